"""8-bit integer expert products and the FFN made of them, against the formulas in 64 bits.

Tolerances.  Integers and scales of rows and weights are exact.  A product's integer sum is exact; turning it into y takes the scales'
product, the sum as fp32, their product with the bias added (2^-24 each, so 2^-22 of |y - b| + |b| covers them) and the rounding to dtype.
The hidden activations H of the FFN are known to the kernel up to such errors, 2^-20 (|z| + 1) of the activation included; what can come out
for their integers is found by quantising H at both ends of those errors, and y may be off by the integers' range times the weights.
"""
import math

import numpy as np
import pytest
import torch

from test_gated_ffn import act64, buckets, float32_by_default, split  # noqa: F401

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
TINY = 2.0 ** -126


def _b():
    from paper_2304_03946_amd import binding as B
    B.load_library()
    return B


def scale64(x):
    """fp32 scales of rows, as doubles (torch divides by a number on the GPU as a product with its reciprocal, so in 64 bits: the quotient
    rounded to 53 and then to 24 bits is the one rounded to 24)."""
    largest = x.abs().amax(1).double()
    return (largest / torch.full_like(largest, 127)).float().clamp(min=TINY).double()


def whole64(x, s):
    return torch.clamp(torch.round(x / s[:, None]), -127, 127)


def quantize(x):
    q = torch.full(x.shape, 99, dtype=torch.int8, device="cuda")
    s = torch.full((x.shape[0],), 99.0, device="cuda")
    _b().flexmoe_quantize_rows(x, q, s)
    return q, s


# ---- quantisers ----------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K", [(1, 16), (5, 1008), (4, 1024), (7, 1040), (300, 2048), (9000, 64), (3, 100000)])
def test_rows(M, K, dtype):
    x = (torch.randn(M, K, device="cuda") * torch.exp(4 * torch.randn(M, 1, device="cuda"))).to(DT[dtype])
    q, s = quantize(x)
    want = scale64(x)
    assert torch.equal(s.double(), want) and torch.equal(q.double(), whole64(x.double(), want))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_the_borders(dtype):
    """Ties (scales that are powers of two and odd multiples of their halves), zeros, the smallest and largest magnitudes, signs."""
    rows = []
    for e in (-20, 0, 3):
        n = torch.arange(-64, 64, dtype=torch.float64)
        rows.append(torch.cat([n + 0.5, torch.tensor([127.0]), torch.zeros(15, dtype=torch.float64)]) * 2.0 ** e)
    rows.append(torch.zeros(144, dtype=torch.float64))
    rows.append(torch.linspace(-1, 1, 144, dtype=torch.float64) * 2.0 ** -126)      # scales below the smallest
    rows.append(torch.linspace(-1, 1, 144, dtype=torch.float64) * 2.0 ** -133)      # subnormal in fp32 and bf16
    rows.append(torch.linspace(-1, 1, 144, dtype=torch.float64) * 3.3e38)
    rows.append(torch.where(torch.arange(144) % 2 == 0, 1.0, -1.0).double() * 7)
    x = torch.stack(rows).cuda().to(DT[dtype])
    q, s = quantize(x)
    want = scale64(x)
    assert torch.equal(s.double(), want)
    assert torch.equal(q.double(), whole64(x.double(), want))


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite(bad):
    x = torch.randn(5, 64, device="cuda", dtype=torch.bfloat16)
    x[2, 17] = bad
    q, s = quantize(x)
    assert torch.isnan(s[2]) and not q[2].any()
    other = torch.tensor([0, 1, 3, 4], device="cuda")
    assert torch.equal(q[other].double(), whole64(x[other].double(), scale64(x[other])))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("E,K,NC", [(1, 16, 8), (3, 80, 72), (2, 1024, 520), (5, 272, 64)])
def test_weights(E, K, NC, dtype):
    w = (torch.randn(E, K, NC, device="cuda") * torch.exp(torch.randn(E, 1, NC, device="cuda"))).to(DT[dtype])
    w[0, :, 3] = 0
    q, s = torch.full((E, NC, K), 99, dtype=torch.int8, device="cuda"), torch.full((E, NC), 9.0, device="cuda")
    _b().flexmoe_quantize_weights(w, q, s)
    rows = w.transpose(1, 2).contiguous().view(E * NC, K)
    want = scale64(rows)
    assert torch.equal(s.view(-1).double(), want) and torch.equal(q.view(-1, K).double(), whole64(rows.double(), want))


# ---- products ------------------------------------------------------------------------------------
class Routed:
    """N tokens, k assignments each, in buckets; src as the router leaves it."""

    def __init__(self, N, E, k, V, seed, counts=None):
        rng = np.random.default_rng(seed)
        off, owner, rows = buckets(split(N * k, V, rng) if counts is None else counts, E, seed)
        self.voff, self.owner = torch.from_numpy(off).cuda(), torch.from_numpy(owner).cuda()
        self.expert = torch.from_numpy(rows).cuda()
        self.src = torch.from_numpy(rng.permutation(N * k).astype(np.int32)).cuda()
        self.token = self.src.long() // k


def weights(E, NC, K, gen):
    q = torch.randint(-127, 128, (E, NC, K), generator=gen, device="cuda", dtype=torch.int8)
    return q, torch.rand(E, NC, generator=gen, device="cuda") * 2e-4 + 1e-5


def check_product(y, q, s, wq, ws, bias, rows, expert, dtype):
    u = torch.finfo(DT[dtype]).eps / 2
    for e in range(wq.shape[0]):
        p = torch.nonzero(expert == e).flatten()
        if len(p) == 0:
            continue
        r = rows[p]
        prod = (q[r].double() @ wq[e].double().T.contiguous()) * (s[r].double()[:, None] * ws[e].double())
        b = bias[e].double() if bias is not None else torch.zeros(1, device="cuda", dtype=torch.float64)
        want = prod + b
        tol = u * want.abs() + (1 + u) * 2.0 ** -22 * (prod.abs() + b.abs()) + 1e-37
        worst = float(((y[p].double() - want).abs() / tol).max())
        assert worst <= 1, (e, worst)


# tokens, K, NC, experts, per token, vExperts: one row; few rows with and without segments; K in no whole stages; 256 x 256 tiles (2056 columns); many
# rows on 64-row tiles, in two segments; one expert on 256 x 256 tiles
PRODUCTS = [(1, 16, 8, 1, 1, 1), (3, 64, 72, 4, 2, 5), (16, 2048, 512, 8, 2, 12), (130, 336, 912, 12, 3, 15), (900, 272, 256, 4, 1, 9),
            (2500, 2048, 2056, 4, 3, 6), (7300, 2048, 1000, 3, 1, 3), (7300, 2064, 1024, 3, 1, 3), (7300, 2048, 2048, 1, 1, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("N,K,NC,E,k,V", PRODUCTS)
def test_product(N, K, NC, E, k, V, gather, dtype):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N + K)
    t = Routed(N, E, k, V, N + K)
    M = N if gather else N * k
    q = torch.randint(-127, 128, (M, K), generator=gen, device="cuda", dtype=torch.int8)
    s = torch.rand(M, generator=gen, device="cuda") + 0.01
    wq, ws = weights(E, NC, K, gen)
    bias = torch.randn(E, NC, generator=gen, device="cuda").to(DT[dtype]) if K % 32 == 0 else None
    y = torch.full((N * k, NC), 3.0, device="cuda", dtype=DT[dtype])
    work = torch.empty(_b().flexmoe_i8_workspace_bytes(N, 16, 16, E, k, V, 0), dtype=torch.uint8, device="cuda")
    _b().flexmoe_expert_matmul_i8(q, s, t.src if gather else None, k, t.voff, t.owner, wq, ws, bias, y, work)
    rows = t.token if gather else torch.arange(N * k, device="cuda")
    check_product(y, q, s, wq, ws, bias, rows, t.expert, dtype)


@pytest.mark.gpu
def test_sums_at_the_end_of_their_range():
    """K just below 2^17, every product 127 * 127."""
    K, NC = (1 << 17) - 16, 8
    q = torch.full((2, K), 127, dtype=torch.int8, device="cuda")
    q[1] = -127
    wq = torch.full((1, NC, K), 127, dtype=torch.int8, device="cuda")
    one = torch.ones(2, device="cuda")
    off, own = torch.tensor([0, 2], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    y = torch.empty(2, NC, device="cuda")
    work = torch.empty(_b().flexmoe_i8_workspace_bytes(2, 16, 16, 1, 1, 1, 0), dtype=torch.uint8, device="cuda")
    _b().flexmoe_expert_matmul_i8(q, one, None, 1, off, own, wq, torch.ones(1, NC, device="cuda"), None, y, work)
    assert torch.equal(y.cpu(), torch.tensor([[127.0 * 127 * K]] * 1 + [[-127.0 * 127 * K]]).expand(2, NC).float())


# ---- FFN -----------------------------------------------------------------------------------------
class Ffn:
    def __init__(self, N, d, f, E, k, V, gated, act, dtype, bias, seed=0):
        B = _b()
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.__dict__.update(N=N, d=d, f=f, E=E, k=k, V=V, gated=gated, act=act, dtype=dtype)
        self.t = Routed(N, E, k, V, seed)
        dt = DT[dtype]
        cols = 2 * f if gated else f
        self.x = torch.randn(N, d, generator=gen, device="cuda").to(dt)
        self.x[:, :: 37] *= 5
        (self.w1, self.s1), (self.w2, self.s2) = weights(E, cols, d, gen), weights(E, d, f, gen)
        self.s1 *= 100 / math.sqrt(d)
        self.b1 = torch.randn(E, cols, generator=gen, device="cuda").to(dt) if bias else None
        self.b2 = torch.randn(E, d, generator=gen, device="cuda").to(dt) if bias else None
        self.y = torch.full((N * k, d), 3.0, device="cuda", dtype=dt)
        self.code = dict(relu=B.RELU, gelu_erf=B.GELU_ERF, gelu_tanh=B.GELU_TANH, silu=B.SILU)[act]
        self.ws = torch.empty(B.flexmoe_i8_workspace_bytes(N, d, f, E, k, V, int(gated)), dtype=torch.uint8, device="cuda")

    def run(self):
        _b().flexmoe_expert_ffn_i8_fwd(self.x, self.t.src, self.k, self.t.voff, self.t.owner, self.w1, self.s1, self.b1, self.w2, self.s2,
                                       self.b2, self.gated, self.code, self.y, self.ws)
        return self.y

    def check(self):
        dt, f = DT[self.dtype], self.f
        u = torch.finfo(dt).eps / 2
        x = self.x.double()
        xs = scale64(self.x)
        xq = whole64(x, xs)
        for e in range(self.E):
            p = torch.nonzero(self.t.expert == e).flatten()
            if len(p) == 0:
                continue
            r = self.t.token[p]
            prod = (xq[r] @ self.w1[e].double().T.contiguous()) * (xs[r][:, None] * self.s1[e].double())
            b1 = self.b1[e].double() if self.b1 is not None else torch.zeros(1, device="cuda", dtype=torch.float64)
            z, nz = prod + b1, 2.0 ** -22 * (prod.abs() + b1.abs())
            g = z[:, :f]
            a = act64(self.act, g)[0]
            if self.gated:
                up = z[:, f:]
                h = a * up
                nh = 1.13 * nz[:, :f] * up.abs() + nz[:, f:] * a.abs() + 2.0 ** -20 * (g.abs() + 1) * up.abs()
            else:
                h, nh = a, 1.13 * nz + 2.0 ** -20 * (g.abs() + 1)
            ends = []
            for sign in (-1, 1):
                hs = ((h.abs() + sign * nh).amax(1) / 127 * (1 + sign * 2.0 ** -23)).clamp(min=TINY)
                for hh in (h - nh, h + nh):
                    ends.append(whole64(hh.to(dt).double(), hs) * hs[:, None])
            ends = torch.stack(ends)
            low, high = ends.amin(0), ends.amax(0)
            mid = (low + high) / 2
            w2 = (self.w2[e].double() * self.s2[e].double()[:, None]).T.contiguous()
            b2 = self.b2[e].double() if self.b2 is not None else torch.zeros(1, device="cuda", dtype=torch.float64)
            prod = mid @ w2
            want = prod + b2
            noise = ((high - low) / 2) @ w2.abs() + 2.0 ** -22 * (prod.abs() + b2.abs())
            worst = float(((self.y[p].double() - want).abs() / (u * want.abs() + (1 + u) * noise + 1e-37)).max())
            assert worst <= 1 + 2 * u, (e, worst)
            # the range that H's integers leave is a small part of what they add up to: the check means something
            assert float(noise.mean()) <= 0.02 * float(prod.abs().mean()) + 1e-6


FFNS = [(1, 16, 16, 1, 1, 1), (3, 64, 80, 4, 2, 5), (16, 1024, 512, 8, 2, 12), (130, 336, 912, 12, 3, 15), (900, 272, 256, 4, 1, 9),
        (4000, 2048, 1024, 4, 2, 6), (4000, 2048, 1104, 4, 2, 6), (7400, 2064, 1024, 3, 1, 5), (30000, 256, 512, 2, 1, 40)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated,act,bias", [(True, "silu", False), (True, "gelu_erf", True), (False, "gelu_tanh", True), (False, "relu", False),
                                            (False, "silu", False)])
@pytest.mark.parametrize("N,d,f,E,k,V", FFNS)
def test_ffn(N, d, f, E, k, V, gated, act, bias, dtype):
    if dtype == "f32" and N * k * f > 9_000_000:
        N //= 8
    c = Ffn(N, d, f, E, k, V, gated, act, dtype, bias, seed=N + d)
    c.run()
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("act,gated", [("silu", True), ("gelu_erf", True), ("gelu_tanh", False), ("relu", False)])
def test_a_row_depends_on_nothing_else(act, gated):
    """The same bits for a token alone, in a few-rows batch and in a large one."""
    big = Ffn(4000, 2048, 1024, 4, 2, 6, gated, act, "bf16", True, seed=4)
    y = big.run().clone()
    shared = ("w1", "s1", "b1", "w2", "s2", "b2")
    at = torch.nonzero(big.t.token == 17).flatten()
    for p in at.tolist():
        one = Ffn(1, 2048, 1024, 4, 1, 4, gated, act, "bf16", True, seed=4)
        e = int(big.t.expert[p])
        one.x = big.x[17:18].clone()
        one.__dict__.update({n: getattr(big, n) for n in shared})
        one.t.owner = torch.arange(4, dtype=torch.int32, device="cuda")
        one.t.voff = (torch.arange(5, device="cuda") > e).int()
        one.t.src = torch.zeros(1, dtype=torch.int32, device="cuda")
        assert torch.equal(one.run()[0], y[p])
    some = Ffn(130, 2048, 1024, 4, 2, 6, gated, act, "bf16", True, seed=5)
    some.x = big.x[:130].clone()
    some.__dict__.update({n: getattr(big, n) for n in shared})
    some.run()
    where = {(t, e): p for p, (t, e) in enumerate(zip(big.t.token.tolist(), big.t.expert.tolist()))}
    both = [(p, where[te]) for p, te in enumerate(zip(some.t.token.tolist(), some.t.expert.tolist())) if te in where]
    assert len(both) > 40
    here, there = torch.tensor(both, device="cuda").T
    assert torch.equal(some.y[here], y[there])


@pytest.mark.gpu
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("M,K,NC", [(540_000, 4096, 64), (540_000, 64, 4096)])
def test_offsets_past_32_bits(M, K, NC, gather):
    """Rows and outputs of more than 2^31 elements: the last rows as in a call of their own, bit for bit; their integers too."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(M)
    B, last = _b(), 300
    x = torch.randn(M, K, generator=gen, device="cuda", dtype=torch.bfloat16)
    q, s = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    B.flexmoe_quantize_rows(x, q, s)
    ql, sl = torch.empty(last, K, dtype=torch.int8, device="cuda"), torch.empty(last, device="cuda")
    B.flexmoe_quantize_rows(x[-last:].contiguous(), ql, sl)
    assert torch.equal(ql, q[-last:]) and torch.equal(sl, s[-last:])
    del x
    wq, ws = weights(2, NC, K, gen)
    own = torch.arange(2, dtype=torch.int32, device="cuda")

    def product(q, s, first):
        n = len(q)
        y = torch.empty(n, NC, dtype=torch.bfloat16, device="cuda")
        work = torch.empty(B.flexmoe_i8_workspace_bytes(n, 16, 16, 2, 1, 2, 0), dtype=torch.uint8, device="cuda")
        off = torch.tensor([0, first, n], dtype=torch.int32, device="cuda")
        B.flexmoe_expert_matmul_i8(q, s, torch.arange(n, dtype=torch.int32, device="cuda") if gather else None, 1, off, own, wq, ws, None, y, work)
        return y
    assert torch.equal(product(q, s, M - last + 100)[-last:], product(ql, sl, 100))


@pytest.mark.gpu
@pytest.mark.parametrize("N,d,f,E,k,V", [(40, 64, 80, 4, 2, 5), (4000, 2048, 1024, 4, 2, 6)])
@pytest.mark.parametrize("act,gated", [("relu", False), ("silu", True)])
def test_non_finite_tokens_stay_where_they_are(N, d, f, E, k, V, act, gated):
    c = Ffn(N, d, f, E, k, V, gated, act, "bf16", False, seed=3)
    y = c.run().clone()
    c.x[N // 2, 3] = float("nan")
    c.x[N // 3, 0] = -float("inf")
    c.run()
    bad = (c.t.token == N // 2) | (c.t.token == N // 3)
    assert torch.equal(c.y[~bad], y[~bad]) and torch.isnan(c.y[bad]).all()


@pytest.mark.gpu
def test_no_tokens_and_rows_behind_the_last_bucket():
    c = Ffn(3, 64, 80, 4, 2, 5, True, "silu", "bf16", False)
    old = c.y.clone()
    c.t.voff.zero_()
    c.run()
    assert torch.equal(c.y, old)
    big = Ffn(4000, 2048, 1024, 4, 2, 6, True, "silu", "bf16", False)
    y = big.run().clone()
    cut = int(big.t.voff[-1]) - int((big.t.voff[-1] - big.t.voff[-2]) // 2) - 1
    big.t.voff.clamp_(max=cut)            # (the last bucket may be empty: the offsets stay ascending)
    big.y.fill_(3)
    big.run()
    assert torch.equal(big.y[:cut], y[:cut]) and (big.y[cut:] == 3).all()
    B = _b()
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    B.flexmoe_quantize_rows(e, torch.empty(0, 64, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("N,d,f,E,k,V", [(16, 1024, 512, 8, 2, 12), (4000, 2048, 1024, 4, 2, 6)])
def test_equal_calls_streams_and_graphs(N, d, f, E, k, V):
    c = Ffn(N, d, f, E, k, V, True, "silu", "bf16", True, seed=11)
    want = c.run().clone()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = c.run().clone()
    s.synchronize()
    assert torch.equal(want, got)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    x0, off0 = c.x.clone(), c.t.voff.clone()
    for i in range(3):
        c.x.copy_(x0 * (i + 2))
        c.t.voff[1:-1] = torch.sort(torch.randint(0, N * k + 1, (V - 1,), device="cuda", dtype=torch.int32)).values
        eager = c.run().clone()
        c.y.fill_(3)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager, c.y), i
        c.x.copy_(x0)
        c.t.voff.copy_(off0)
        assert torch.equal(want, c.run())


# ---- the layer -------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("gated,act", [(True, "SILU"), (False, "GELU_ERF")])
@pytest.mark.parametrize("N", [24, 3000])
def test_layer_trains_and_serves(N, gated, act):
    """MoELayer: a training step (every gradient), then the same tokens on the quantised weights: y within the error that 8 bits leave.
    A number is off by at most half a scale of its row or channel, 1 / 254 of the largest: x, W1, H and W2 each put a relative error of
    about (largest / rms) / 254 / sqrt(3) into terms that add up independently; largest / rms stays below 6 here."""
    from paper_2304_03946_amd import layer as L
    B = _b()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N)
    d, f, E, k, V = 256, 512, 8, 2, 10
    f1 = 2 * f if gated else f

    def new(*s, std):
        return (torch.randn(*s, generator=gen, device="cuda") * std).bfloat16()
    x, wg, dy = new(N, d, std=1), new(d, E, std=d ** -0.5), new(N, d, std=1)
    w1, w2, b1, b2 = new(E, d, f1, std=d ** -0.5), new(E, f, d, std=f ** -0.5), new(E, f1, std=0.1), new(E, d, std=0.1)
    off, ids = np.array([0, 2, 4, 5, 6, 7, 8, 9, 10], np.int32), np.arange(10, dtype=np.int32)
    m = L.MoELayer(N, d, f, E, k, V, B.BF16, getattr(B, act), backward=True, gated=gated)
    y = m.forward(x, wg, w1, w2, off, ids, b1, b2).double().clone()
    grads = {n: t.clone() for n, t in m.backward_full(dy, wg, w1, w2).items()}
    assert grads["dw1"].shape == w1.shape and grads["db1"].shape == b1.shape
    assert all(torch.isfinite(t).all() and t.any() for t in grads.values())
    dx, dw1, dw2 = m.backward(dy, w1, w2)
    assert torch.equal(dw1, grads["dw1"]) and torch.equal(dw2, grads["dw2"])
    assert m.profile_token_cost(w1, w2, reps=1) >= 1
    q = L.QuantizedExperts(w1, w2, b1, b2)
    assert q.gated == gated
    y8 = m.forward_i8(x, wg, q, off, ids).double()
    rel = float((y8 - y).norm() / y.norm())
    assert 0 < rel < 2 * 6 / 254 / math.sqrt(3) * 1.5, rel      # sqrt(4) errors, and as much again for the gate's two factors
    with pytest.raises(ValueError):
        L.MoELayer(N, d, f, E, k, V, B.BF16, B.RELU, gated=not gated).forward_i8(x, wg, q, off, ids)
    if gated:
        for call in ((m.forward_fused, (x, wg, w1, w2, off, ids)), (m.forward_top1, (x, wg, w1, w2, off, ids)), (m.backward_top1, (dy, w1, w2))):
            with pytest.raises(ValueError):
                call[0](*call[1])


# ---- refusals ----------------------------------------------------------------------------------------
def test_refusals():
    import ctypes
    B = _b()
    lib = B.load_library()
    null, one, odd, big = ctypes.c_void_p(None), ctypes.c_void_p(16), ctypes.c_void_p(24), 1 << 40

    def rows(x=one, M=4, K=64, dtype=B.BF16, q=one, s=one):
        return lib.flexmoe_quantize_rows(x, M, K, dtype, q, s, null)

    def wts(w=one, E=4, K=64, NC=64, dtype=B.BF16, q=one, s=one):
        return lib.flexmoe_quantize_weights(w, E, K, NC, dtype, q, s, null)

    def mm(x=one, xs=one, src=null, off=one, own=one, w=one, s=one, b=null, N=4, k=1, K=64, NC=64, E=4, V=4, dtype=B.BF16, y=one, ws=one, size=big):
        return lib.flexmoe_expert_matmul_i8(x, xs, src, off, own, w, s, b, N, k, K, NC, E, V, dtype, y, ws, size, null)

    def ffn(x=one, src=one, off=one, own=one, w1=one, s1=one, b1=null, w2=one, s2=one, b2=null, N=4, k=1, d=64, f=64, E=4, V=4, gated=1,
            act=B.SILU, dtype=B.BF16, y=one, ws=one, size=big):
        return lib.flexmoe_expert_ffn_i8_fwd(x, src, off, own, w1, s1, b1, w2, s2, b2, N, k, d, f, E, V, gated, act, dtype, y, ws, size, null)
    for call in (rows, wts, mm, ffn):
        assert call(dtype=2) == B.UNSUPPORTED and call(dtype=-1) == B.UNSUPPORTED
    for kw in (dict(M=-1), dict(M=1 << 30), dict(K=0), dict(K=24), dict(K=1 << 20), dict(x=null), dict(x=odd), dict(q=null), dict(q=odd),
               dict(s=null)):
        assert rows(**kw) == B.INVALID_ARG, kw
    for kw in (dict(E=0), dict(E=257), dict(K=0), dict(K=8), dict(K=1 << 17), dict(NC=4), dict(NC=12), dict(NC=1 << 20),
               dict(K=65536, NC=32768), dict(w=null), dict(w=odd), dict(q=null), dict(s=odd)):
        assert wts(**kw) == B.INVALID_ARG, kw
    for kw in (dict(N=-1), dict(N=1 << 29, k=2), dict(k=0), dict(k=9), dict(K=8), dict(K=1 << 17), dict(NC=4), dict(K=65536, NC=32768), dict(E=0),
               dict(E=257, V=300), dict(V=3), dict(V=513), dict(x=null), dict(x=odd), dict(xs=null), dict(off=null), dict(own=null), dict(w=null),
               dict(w=odd), dict(s=null), dict(b=odd), dict(y=null), dict(y=odd), dict(ws=null), dict(ws=odd)):
        assert mm(**kw) == B.INVALID_ARG, kw
    for kw in (dict(N=-1), dict(k=0), dict(d=0), dict(d=24), dict(f=8), dict(f=24), dict(d=1 << 17), dict(f=1 << 17), dict(d=65536, f=16384), dict(E=0),
               dict(V=3), dict(x=null), dict(x=odd), dict(src=null), dict(off=null), dict(w1=null), dict(w2=odd), dict(s1=null), dict(s2=odd), dict(b1=odd),
               dict(b2=odd), dict(y=null), dict(ws=null), dict(ws=odd)):
        assert ffn(**kw) == B.INVALID_ARG, kw
    for kw in (dict(act=4), dict(act=-1), dict(gated=2)):
        assert ffn(**kw) == B.UNSUPPORTED, kw
    need = B.flexmoe_i8_workspace_bytes(4, 64, 64, 4, 1, 4, 1)
    assert need > 0 and ffn(size=need - 256) == B.WORKSPACE_TOO_SMALL and mm(size=64) == B.WORKSPACE_TOO_SMALL
    for bad in ((4, 24, 64, 4, 1, 4, 1), (4, 64, 20, 4, 1, 4, 0), (4, 64, 64, 4, 9, 4, 0), (-1, 64, 64, 4, 1, 4, 0), (4, 64, 64, 4, 1, 3, 0)):
        assert B.flexmoe_i8_workspace_bytes(*bad) == 0
    last = 0
    for N in list(range(0, 3000)) + list(range(3000, 200000, 97)):
        size = B.flexmoe_i8_workspace_bytes(N, 256, 512, 8, 2, 12, 1)
        assert size >= last
        last = size
