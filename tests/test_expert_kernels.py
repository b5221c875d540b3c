"""Gated and 8-bit experts: every kernel that the host's rules choose between has a case here that is known to reach it, and the sizes at the
ends of what the calls take."""
import ctypes

import pytest
import torch

from test_gated_ffn import float32_by_default  # noqa: F401
from test_i8_experts import DT, Routed, check_product, weights


def _b():
    from paper_2304_03946_amd import binding as B
    B.load_library()
    return B


# ---- sizes -----------------------------------------------------------------------------------------
WIDE = [1 << 17, (1 << 17) + 8, (1 << 20) - 8]


@pytest.mark.parametrize("NC", WIDE)
def test_workspace_of_wide_products(NC):
    """A product has up to 2^20 - 8 columns, eight times what a contraction may have: its workspace is known, and enough."""
    B = _b()
    lib, null, one = B.load_library(), ctypes.c_void_p(None), ctypes.c_void_p(16)
    need = B.flexmoe_i8_workspace_bytes(4, 64, NC, 4, 1, 4, 0)
    assert 0 < need <= B.flexmoe_i8_workspace_bytes(4, 64, NC // 2, 4, 1, 4, 1)
    assert need <= B.flexmoe_i8_workspace_bytes(5, 64, NC, 4, 1, 4, 0)

    def call(size):
        return lib.flexmoe_expert_matmul_i8(one, one, null, one, one, one, one, null, 4, 1, 64, NC, 4, 4, B.BF16, one, one, size, null)
    assert call(need - 1) == B.WORKSPACE_TOO_SMALL


def test_workspace_of_sizes_that_nothing_takes():
    B = _b()
    for bad in ((4, 64, 1 << 20, 4, 1, 4, 0), (4, 64, 1 << 19, 4, 1, 4, 1), (4, 1 << 16, 1 << 15, 4, 1, 4, 0), (4, 1 << 17, 64, 4, 1, 4, 0),
                (4, 64, (1 << 31) - 8, 4, 1, 4, 1), (4, 64, -8, 4, 1, 4, 0)):
        assert B.flexmoe_i8_workspace_bytes(*bad) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 700])
def test_wide_product(N, dtype):
    NC, K, E, k, V = WIDE[1], 80, 2, 2, 3
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N)
    t = Routed(N, E, k, V, N)
    q = torch.randint(-127, 128, (N, K), generator=gen, device="cuda", dtype=torch.int8)
    s = torch.rand(N, generator=gen, device="cuda") + 0.01
    wq, ws = weights(E, NC, K, gen)
    bias = torch.randn(E, NC, generator=gen, device="cuda").to(DT[dtype])
    y = torch.full((N * k, NC), 3.0, device="cuda", dtype=DT[dtype])
    work = torch.empty(_b().flexmoe_i8_workspace_bytes(N, K, NC, E, k, V, 0), dtype=torch.uint8, device="cuda")
    _b().flexmoe_expert_matmul_i8(q, s, t.src, k, t.voff, t.owner, wq, ws, bias, y, work)
    check_product(y, q, s, wq, ws, bias, t.token, t.expert, dtype)


# ---- the layer's checks ------------------------------------------------------------------------------
def test_experts_that_do_not_fit():
    """Shapes that the kernels would take at their word (they get E, d and f from one of the tensors) are refused on the host."""
    from types import SimpleNamespace
    from paper_2304_03946_amd import layer as L
    B = _b()
    new = torch.zeros
    for w1, w2, b1, b2 in (((2, 16, 48), (2, 32, 16), None, None), ((3, 16, 32), (2, 32, 16), None, None), ((2, 32, 32), (2, 32, 16), None, None),
                           ((2, 16, 96), (2, 32, 16), None, None), ((2, 16, 64), (2, 32, 16), (2, 32), None), ((2, 16, 32), (2, 32, 16), (2, 64), None),
                           ((2, 16, 32), (2, 32, 16), None, (2, 32)), ((2, 16, 32), (2, 32, 16), None, (1, 16))):
        with pytest.raises(ValueError):
            L.QuantizedExperts(new(w1), new(w2), None if b1 is None else new(b1), None if b2 is None else new(b2))
    m = L.MoELayer(4, 16, 32, 2, 1, 2, B.BF16, B.RELU, device="cpu")
    fits = dict(sizes=(2, 16, 32), gated=False, b1=None, b2=None)
    for wrong in (dict(sizes=(1, 16, 32)), dict(sizes=(2, 32, 32)), dict(sizes=(2, 16, 16)), dict(gated=True), dict(b1=new(2, 32)), dict(b2=new(2, 16))):
        with pytest.raises(ValueError):
            m.forward_i8(new(4, 16), new(16, 2), SimpleNamespace(**{**fits, **wrong}), [0, 1, 2], [0, 1])
