"""Gated and 8-bit experts at the ends of the number range, against the formulas in 64 bits.

Where act'(z) is 0 or 1 to more places than its type has (|z| >= 30 in every activation but SiLU), dHpre is a product of dH that carries
fp32 sums of d terms (2^-23 sqrt(d) of the root of the sum of their squares, six standard deviations of errors uniform in that: `sums`) and
one rounding per factor and for the type, u = finfo(t).eps / 2.
"""
import math

import pytest
import torch

from test_gated_ffn import SPREAD, Case, act64, decode, dot, float32_by_default, sums  # noqa: F401
from test_i8_experts import Ffn

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
LARGE = (1e19, -1e19, 6e19, -6e19, 1e25, -1e25, 1e33, -1e33, 30.0, -30.0)


def _b():
    from paper_2304_03946_amd import binding as B
    B.load_library()
    return B


def d_hidden(c, rows, dt):
    """dH = dY W2^T and its noise."""
    dh, noise = (torch.zeros(c.A, c.f, dtype=torch.float64, device="cuda") for _ in range(2))
    for e in range(c.E):
        r = torch.nonzero(rows == e).flatten()
        w2t = c.w2[e].double().T.contiguous()
        dh[r] = c.dy[r].double() @ w2t
        noise[r] = SPREAD * sums(c.d) * dot(c.dy[r].double(), w2t)
    return dh, noise


# rows, d, f: few rows; 256 x 256 tiles, contractions in whole rounds of 128 and not
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "gelu_erf", "gelu_tanh"])
@pytest.mark.parametrize("A,d,f", [(40, 64, 72), (7300, 2048, 1024), (7400, 2056, 1032)])
def test_slopes_of_gates_far_from_zero(A, d, f, act, dtype):
    if dtype == "f32" and A > 1000:
        A, d, f = 1600, 136, 264
    c = Case(A, d, f, 2, 3, dtype, act, True, seed=7)
    far = torch.arange(f, device="cuda") % 3 != 0
    gate = torch.tensor(LARGE, device="cuda")[torch.arange(f, device="cuda") % len(LARGE)]
    c.b1[:, :f] = torch.where(far, gate, torch.zeros_like(gate)).to(c.dt)
    c.w1[:, :, :f][:, :, far] = 0
    c.fwd()
    g, up = decode(c.hpre)[:, :f], decode(c.hpre)[:, f:]
    assert torch.isfinite(c.y).all() and (g[:, far].abs() >= 29).all()
    dh, noise = d_hidden(c, c.rows, c.dt)
    u = c.u()
    for kept in (True, False):
        c.bwd(kept)
        got = c.ws[:A * 2 * f * c.dxp.element_size()].view(c.dt).view(A, 2 * f).double()
        for t in (got, c.dxp, c.dw1, c.dw2):
            assert torch.isfinite(t).all()
        slope = (g > 0).double()
        for name, v, want, n in (("dG", got[:, :f], dh * up * slope, noise * up.abs() * slope),
                                 ("dU", got[:, f:], dh * g * slope, noise * g.abs() * slope)):
            tol = (u + 2.0 ** -21) * want.abs() + (1 + u) * n + 1e-37
            if act != "relu":                     # at |z| = 30 the lower tail is below 1e-12 of |z|; the fp32 forms' sums cancel to 2^-22
                tol = tol + 2.0 ** -22 * dh.abs() * (up.abs() if name == "dG" else g.abs().clamp(max=30))
            worst = float(((v - want).abs() / tol)[:, far].max())
            assert worst <= 1 + 2 * u, (name, kept, worst)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,A,d,f", [("bf16", 40, 64, 72), ("bf16", 40, 128, 72), ("bf16", 7400, 2056, 1032), ("bf16", 7300, 2048, 1024),
                                         ("f32", 40, 64, 72), ("f32", 1600, 136, 264)])
@pytest.mark.parametrize("act", ["relu", "gelu_erf", "gelu_tanh"])
def test_slopes_far_from_zero_without_a_gate(dtype, A, d, f, act):
    """The same for ungated layers: GELU from its table (d a multiple of 128), evaluated, and in fp32."""
    B = _b()
    c = Case(A, d, f, 2, 3, dtype, act, False, seed=8)
    hpre = torch.tensor(LARGE, device="cuda").to(c.dt)[torch.arange(A * f, device="cuda") % len(LARGE)].view(A, f).clone()
    w1 = c.w1[:, :, :f].contiguous()
    dw1 = torch.empty_like(w1)
    dh, noise = d_hidden(c, c.rows, c.dt)
    u = c.u()
    ws = torch.empty(B.flexmoe_workspace_bytes(A, d, f, 2, 1, 3, B.BF16 if dtype == "bf16" else B.F32), dtype=torch.uint8, device="cuda")
    B.flexmoe_expert_ffn_bwd(c.dy, c.x, hpre, w1, c.w2, c.voff, c.owner, c.code, c.dxp, dw1, c.dw2, ws)
    got = ws[:A * f * c.dxp.element_size()].view(c.dt).view(A, f).double()
    for t in (got, c.dxp, dw1, c.dw2):
        assert torch.isfinite(t).all()
    slope = (hpre > 0).double()
    tol = (u + 2.0 ** -21) * (dh * slope).abs() + (1 + u) * noise * slope + 2.0 ** -22 * dh.abs() + 1e-37
    worst = float(((got - dh * slope).abs() / tol).max())
    assert worst <= 1 + 2 * u, worst


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "silu", "gelu_erf"])
@pytest.mark.parametrize("A,d,f", [(40, 64, 72), (7300, 2048, 1024), (7400, 2056, 1032)])
def test_closed_gates_keep_large_factors_out(A, d, f, act, dtype):
    """dG = dH U act'(G) where dH U is beyond fp32 and act'(G) next to nothing: the product fits, or is zero."""
    if dtype == "f32" and A > 1000:
        A, d, f = 1600, 136, 264
    c = Case(A, d, f, 2, 3, dtype, act, True, seed=6)
    c.w1.zero_()
    c.b1[:, :f] = -60.0 if act == "silu" else -8.0
    c.b1[:, f:] = 1e25
    c.dy *= 1e20
    c.fwd()
    dh, noise = d_hidden(c, c.rows, c.dt)
    assert float(dh.abs().max()) * 1e25 > 3.5e38
    g, up = decode(c.hpre)[:, :f], decode(c.hpre)[:, f:]
    slope = act64(act, g)[1]
    want = dh * up * slope
    for kept in (True, False):
        c.bwd(kept)
        dz = c.ws[:A * 2 * f * c.dxp.element_size()].view(c.dt).view(A, 2 * f)
        for t in (dz, c.dxp, c.dw1, c.dw2):
            assert torch.isfinite(t).all()
        if act == "relu":
            assert not dz.any() and not c.dxp.any() and not c.dw1.any() and not c.dw2.any()
        if act == "silu":                         # one rounding of z / ln 2 in the exponent: 2^-24 of 87, and as much for the constant
            u = c.u()
            tol = (u + 2.0 ** -15) * want.abs() + (1 + u) * noise * (up * slope).abs()
            assert float(((dz[:, :f].double() - want).abs() / tol).max()) <= 1 + 2 * u


def hidden_alone(z, act, gated, dtype):
    """H = act(z) (times 1) of 8-bit experts, one expert for each z, read from the scales: x = 0, so the pre-activations are the biases, all
    of a row's H are equal, its integers are 127 and y is 127 times their scale."""
    B = _b()
    E, d, f = len(z), 16, 16
    cols = 2 * f if gated else f
    b1 = torch.ones(E, cols, device="cuda")
    b1[:, :f] = z[:, None]
    i32 = dict(dtype=torch.int32, device="cuda")
    w2 = torch.zeros(E, d, f, dtype=torch.int8, device="cuda")
    w2[:, :, 0] = 1
    y = torch.empty(E, d, dtype=DT[dtype], device="cuda")
    ws = torch.empty(B.flexmoe_i8_workspace_bytes(E, d, f, E, 1, E, int(gated)), dtype=torch.uint8, device="cuda")
    code = dict(relu=B.RELU, gelu_erf=B.GELU_ERF, gelu_tanh=B.GELU_TANH, silu=B.SILU)[act]
    B.flexmoe_expert_ffn_i8_fwd(torch.zeros(E, d, device="cuda", dtype=DT[dtype]), torch.arange(E, **i32), 1, torch.arange(E + 1, **i32),
                                torch.arange(E, **i32), torch.zeros(E, cols, d, dtype=torch.int8, device="cuda"), torch.ones(E, cols, device="cuda"),
                                b1.to(DT[dtype]), w2, torch.ones(E, d, device="cuda"), None, gated, code, y, ws)
    assert torch.equal(y, y[:, :1].expand(E, d))
    return y[:, 0].double()


@pytest.mark.gpu
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("act", ["relu", "gelu_erf", "gelu_tanh", "silu"])
def test_fp32_activations_of_8_bit_experts(act, gated):
    """H of fp32 layers is what the other fp32 layers make: SiLU to 2^-21 of its value (an exponential within 2^-23, and five roundings of
    2^-24: the sum, the quotient, the product, H / 127 and 127 times that), GELU to 2^-22 |z| (an error function or tanh within 2^-23, halved, next to 1)."""
    z = torch.cat([-torch.logspace(-3, math.log10(80), 100), torch.logspace(-3, 2, 100)]).float().cuda()
    want = act64(act, z.double())[0]
    got = hidden_alone(z, act, gated, "f32")
    tol = 2.0 ** -21 * want.abs() + (2.0 ** -22 * z.double().abs() if act.startswith("gelu") else 0) + 1e-43
    worst = (got - want).abs() / tol
    assert float(worst.max()) <= 1, (float(z[worst.argmax()]), float(worst.max()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_weight_channels_that_are_not_finite(bad, dtype):
    """Their scale is NaN and their integers are zeros; the other channels are as without them, and what is multiplied by them is NaN."""
    B = _b()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(2)
    E, K, NC = 2, 80, 72
    w = torch.randn(E, K, NC, generator=gen, device="cuda").to(DT[dtype])

    def quantized():
        q, s = torch.full((E, NC, K), 99, dtype=torch.int8, device="cuda"), torch.full((E, NC), 9.0, device="cuda")
        B.flexmoe_quantize_weights(w, q, s)
        return q, s
    q0, s0 = quantized()
    w[1, 79, 65] = bad
    q, s = quantized()
    other = torch.ones(E, NC, dtype=torch.bool, device="cuda")
    other[1, 65] = False
    assert torch.isnan(s[1, 65]) and not q[1, 65].any()
    assert torch.equal(s[other], s0[other]) and torch.equal(q[other], q0[other])
    i32 = dict(dtype=torch.int32, device="cuda")
    x, y = torch.ones(4, K, dtype=torch.int8, device="cuda"), torch.zeros(4, NC, dtype=DT[dtype], device="cuda")
    ws = torch.empty(B.flexmoe_i8_workspace_bytes(4, K, NC, E, 1, 2, 0), dtype=torch.uint8, device="cuda")
    B.flexmoe_expert_matmul_i8(x, torch.ones(4, device="cuda"), None, 1, torch.tensor([0, 2, 4], **i32), torch.tensor([0, 1], **i32), q, s, None, y, ws)
    assert torch.isnan(y[2:, 65]).all() and int(torch.isnan(y).sum()) == 2


# few rows on 16- and 64-row tiles; 256 x 256 tiles, with a gate and without
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "gelu_erf", "gelu_tanh", "silu"])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("N,d,f,E,k,V", [(5, 64, 80, 4, 2, 5), (300, 64, 80, 4, 2, 5), (4000, 2064, 2048, 4, 2, 6)])
def test_tokens_that_are_not_finite(N, d, f, E, k, V, gated, act, dtype):
    """A NaN or an infinity in a token makes all of that token's rows NaN, whatever the activation, and no other row."""
    c = Ffn(N, d, f, E, k, V, gated, act, dtype, False, seed=3)
    y = c.run().clone()
    c.x[N // 2, 3] = float("nan")
    c.x[N // 3, 0] = -float("inf")
    c.run()
    bad = (c.t.token == N // 2) | (c.t.token == N // 3)
    assert torch.equal(c.y[~bad], y[~bad]) and torch.isnan(c.y[bad]).all() and torch.isfinite(y).all()
