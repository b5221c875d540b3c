"""Gated and 8-bit experts: every kernel that the host's rules choose between has a case here that is known to reach it, and the sizes at the
ends of what the calls take."""
import ctypes

import numpy as np
import pytest
import torch

from test_gated_ffn import Case, buckets, float32_by_default, split  # noqa: F401
from test_i8_experts import DT, Ffn, Routed, check_product, weights


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


# ---- which kernels run -------------------------------------------------------------------------------
# The host's rules are asked (flexmoe_debug_gated_paths, flexmoe_debug_i8_paths), with the row tiles that a case's buckets have.
def gated_paths(A, d, f, E, V, row_tiles=0):
    fn = _b().load_library().flexmoe_debug_gated_paths
    fn.restype, fn.argtypes = None, [ctypes.c_int] * 6 + [ctypes.c_void_p]
    out = (ctypes.c_longlong * 10)()
    fn(A, d, f, E, V, row_tiles, out)
    names = ("tile", "past", "turns", "first", "second")
    return dict(zip(names, out[:5])), dict(zip(names, out[5:]))


def i8_paths(N, k, K, columns, E, V, gathered, row_tiles=0):
    fn = _b().load_library().flexmoe_debug_i8_paths
    fn.restype, fn.argtypes = None, [ctypes.c_int] * 8 + [ctypes.c_void_p]
    out = (ctypes.c_longlong * 3)()
    fn(N, k, K, columns, E, V, int(gathered), row_tiles, out)
    return dict(zip(("tile", "ragged", "segments"), out))


def row_tiles(counts, E, seed, tile):
    """Row tiles of the few-rows kernels: every expert's rows in tiles of their own."""
    rows = np.bincount(buckets(counts, E, seed)[2], minlength=E)
    return int(sum(-(-rows // tile))) if tile else 0


def cut(segments):
    return segments if segments <= 3 else "more"


def one_bucket(rows, V):
    return [rows if v == V // 2 else 0 for v in range(V)]


def gated_forms(A, d, f, E, V, counts=None):
    """What a bf16 training step with these rows runs: (product, kernel, form)."""
    counts = split(A, V, np.random.default_rng(A + d)) if counts is None else counts

    def ask(which):
        tile = gated_paths(A, d, f, E, V)[which]["tile"]
        return gated_paths(A, d, f, E, V, row_tiles(counts, E, A + d, tile))[which]
    fwd, bwd = ask(0), ask(1)
    whole = {True: "whole", False: "ragged"}
    forms = {("past the line", fwd["past"], bwd["past"])}
    if fwd["tile"]:
        forms |= {("first", fwd["tile"], "turns" if fwd["turns"] else "mixed", cut(fwd["first"])), ("second", fwd["tile"], cut(fwd["second"]))}
    else:
        forms |= {("first", 256, whole[d % 128 == 0]), ("second", 256, whole[f % 128 == 0])}
    if bwd["tile"]:
        forms |= {("dh", bwd["tile"], cut(bwd["first"]))}
    else:
        forms |= {("dh", 256, whole[d % 128 == 0]), ("dx", 256, whole[2 * f % 128 == 0])}
    return forms


# beside the cases of test_gated_ffn.py: few experts with rows, so that the halves of W1 in turn are cut into two and three segments; second
# products in three; dH of 64-row tiles in two; as many experts and vExperts as there may be
GATED = [(40, 1032, 4096, 32, 32, one_bucket(40, 32)), (100, 1544, 4104, 16, 16, one_bucket(100, 16)), (40, 1024, 776, 32, 32, [2] * 20 + [0] * 12),
         (700, 1280, 1600, 4, 4, [130, 200, 170, 200]), (130, 1032, 256, 2, 2, [65, 65]), (900, 64, 72, 256, 512, None)]


def test_every_gated_kernel_has_a_case():
    import test_gated_ffn as G
    forms = set()
    for c in G.FEW + G.LARGE:
        forms |= gated_forms(*c)
    for c in GATED:
        forms |= gated_forms(*c)
    want = {("first", 256, "whole"), ("first", 256, "ragged"), ("second", 256, "whole"), ("second", 256, "ragged"), ("dh", 256, "whole"),
            ("dh", 256, "ragged"), ("dx", 256, "whole"), ("dx", 256, "ragged"), ("past the line", 1, 1), ("past the line", 0, 1), ("past the line", 0, 0)}
    for tile in (32, 64):
        want |= {("first", tile, "mixed", 1), ("first", tile, "turns", 1), ("dh", tile, 1), ("dh", tile, 2)}
        want |= {("second", tile, s) for s in (1, 2, 3, "more")}
    want |= {("first", 32, "mixed", "more"), ("first", 64, "mixed", 2), ("first", 32, "turns", 2), ("first", 64, "turns", 3)}
    assert not want - forms, want - forms


@pytest.mark.gpu
@pytest.mark.parametrize("act,bias", [("silu", True), ("gelu_tanh", False)])
@pytest.mark.parametrize("at", range(len(GATED)))
def test_gated(at, act, bias):
    A, d, f, E, V, counts = GATED[at]
    c = Case(A, d, f, E, V, "bf16", act, bias, seed=A + d, counts=counts)
    c.fwd()
    c.check_fwd()
    y = c.y.clone()
    c.fwd(keep=False, keep_h=False)
    assert torch.equal(y, c.y)
    for kept in (True, False):
        c.bwd(kept)
        c.check_bwd(kept)


# tokens, K, columns, experts, per token, vExperts, rows per bucket: beside those of test_i8_experts.py 256 x 256 tiles with a contraction in no whole
# rounds, gathered and not; two, three and sixteen segments; as many experts and vExperts as there may be
PRODUCTS = [(2500, 2064, 2056, 4, 3, 6, None), (640, 3104, 2048, 1, 1, 1, None), (33, 3088, 256, 40, 1, 40, [1] * 33 + [0] * 7), (1, 16400, 72, 1, 1, 1, None),
            (100, 16400, 136, 1, 1, 1, None), (300, 2064, 512, 3, 2, 3, [200, 200, 200]), (600, 64, 80, 256, 2, 512, None)]
# tokens, d, f, experts, per token, vExperts: 256 x 256 tiles with and without a gate, whole and ragged
FFNS = [(4000, 2048, 2048, 4, 2, 6), (4000, 2064, 2064, 4, 2, 6), (9000, 1040, 1040, 2, 1, 3), (600, 64, 80, 256, 2, 512)]


def i8_forms():
    """What the tests of 8-bit experts run, here and in test_i8_experts.py: (dtype, product, kernel, form)."""
    import test_i8_experts as I
    forms = set()

    def add(dtype, what, N, k, K, columns, E, V, gathered, counts, seed):
        tile = i8_paths(N, k, K, columns, E, V, gathered)["tile"]
        counts = split(N * k, V, np.random.default_rng(seed)) if counts is None else counts
        p = i8_paths(N, k, K, columns, E, V, gathered, row_tiles(counts, E, seed, tile))
        forms.add((dtype, what, tile, cut(p["segments"])) if tile else (dtype, what, 256, "ragged" if p["ragged"] else "whole"))
    for dtype in ("bf16", "f32"):
        for N, K, NC, E, k, V, *counts in I.PRODUCTS + PRODUCTS:
            for gathered in (True, False):
                add(dtype, "gathered" if gathered else "rows", N, k, K, NC, E, V, gathered, counts[0] if counts else None, N + K)
        for here, (N, d, f, E, k, V) in [(False, c) for c in I.FFNS] + [(True, c) for c in FFNS]:
            if dtype == "f32" and not here and N * k * f > 9_000_000:      # (as test_ffn there does)
                N //= 8
            for what, columns in (("gate", 2 * f), ("act", f)):
                add(dtype, what, N, k, d, columns, E, V, True, None, N + d)
            add(dtype, "rows", N, k, f, d, E, V, False, None, N + d)
    return forms


def test_every_8_bit_kernel_has_a_case():
    forms = i8_forms()
    for dtype in ("bf16", "f32"):
        want = {(dtype, what, 256, form) for what in ("gathered", "rows", "gate", "act") for form in ("whole", "ragged")}
        want |= {(dtype, what, tile, 1) for what in ("gathered", "rows", "gate", "act") for tile in (16, 64)}
        want |= {(dtype, what, tile, s) for what in ("gathered", "rows") for tile in (16, 64) for s in (2, 3, "more")}
        assert not want - forms, want - forms


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("at", range(len(PRODUCTS)))
def test_product(at, gather, dtype):
    N, K, NC, E, k, V, counts = PRODUCTS[at]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N + K)
    t = Routed(N, E, k, V, N + K, counts)
    M = N if gather else N * k
    q = torch.randint(-127, 128, (M, K), generator=gen, device="cuda", dtype=torch.int8)
    s = torch.rand(M, generator=gen, device="cuda") + 0.01
    wq, ws = weights(E, NC, K, gen)
    bias = torch.randn(E, NC, generator=gen, device="cuda").to(DT[dtype]) if at % 2 else None
    y = torch.full((N * k, NC), 3.0, device="cuda", dtype=DT[dtype])
    work = torch.empty(_b().flexmoe_i8_workspace_bytes(N, 16, 16, E, k, V, 0), dtype=torch.uint8, device="cuda")
    _b().flexmoe_expert_matmul_i8(q, s, t.src if gather else None, k, t.voff, t.owner, wq, ws, bias, y, work)
    check_product(y, q, s, wq, ws, bias, t.token if gather else torch.arange(N * k, device="cuda"), t.expert, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated,act,bias", [(False, "silu", True), (False, "gelu_erf", False), (False, "gelu_tanh", True), (False, "relu", False),
                                            (False, "relu", True), (True, "relu", True), (True, "gelu_tanh", False)])
@pytest.mark.parametrize("N,d,f,E,k,V", FFNS)
def test_ffn(N, d, f, E, k, V, gated, act, bias, dtype):
    c = Ffn(N, d, f, E, k, V, gated, act, dtype, bias, seed=N + d)
    c.run()
    c.check()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["relu", "gelu_erf", "gelu_tanh", "silu"])
def test_a_row_depends_on_nothing_else(act):
    """Ungated experts on 256 x 256 tiles: a token's bits are those of a batch that takes the few-rows kernels."""
    big = Ffn(4000, 2048, 2048, 4, 2, 6, False, act, "bf16", True, seed=4)
    some = Ffn(130, 2048, 2048, 4, 2, 6, False, act, "bf16", True, seed=5)
    assert i8_paths(4000, 2, 2048, 2048, 4, 6, True)["tile"] == 0 and i8_paths(130, 2, 2048, 2048, 4, 6, True)["tile"] == 64
    some.x = big.x[:130].clone()
    some.__dict__.update({n: getattr(big, n) for n in ("w1", "s1", "b1", "w2", "s2", "b2")})
    big.run()
    some.run()
    where = {(t, e): p for p, (t, e) in enumerate(zip(big.t.token.tolist(), big.t.expert.tolist()))}
    both = [(p, where[te]) for p, te in enumerate(zip(some.t.token.tolist(), some.t.expert.tolist())) if te in where]
    assert len(both) > 40
    here, there = torch.tensor(both, device="cuda").T
    assert torch.equal(some.y[here], big.y[there])


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


# ---- a gated layer as a whole ------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu_erf"])
@pytest.mark.parametrize("N,d,f", [(24, 64, 72), (600, 256, 512), (3000, 200, 264)])
def test_gated_layer_is_its_formula(N, d, f, act, dtype):
    """Output and every gradient (the gate's too) of a layer with biases and replicas against autograd in 64 bits, for the experts that the
    layer's gate chose.  Largest error over largest value as in the other layers' parity tests: fp32 1e-5; bf16 2e-2, of which a value's four
    or five roundings of 2^-9 on its way take a part."""
    from paper_2304_03946_amd import layer as L
    B = _b()
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N + f)
    E, k, V = 8, 2, 10

    def new(*s, std):
        return (torch.randn(*s, generator=gen, device="cuda") * std).to(DT[dtype])
    t = dict(x=new(N, d, std=1), wg=new(d, E, std=d ** -0.5), w1=new(E, d, 2 * f, std=d ** -0.5), w2=new(E, f, d, std=f ** -0.5), b1=new(E, 2 * f, std=0.1),
             b2=new(E, d, std=0.1))
    dy = new(N, d, std=1)
    off, ids = np.array([0, 2, 4, 5, 6, 7, 8, 9, 10], np.int32), np.arange(10, dtype=np.int32)
    m = L.MoELayer(N, d, f, E, k, V, B.BF16 if dtype == "bf16" else B.F32, dict(silu=B.SILU, gelu_erf=B.GELU_ERF)[act], backward=True, gated=True)
    y = m.forward(t["x"], t["wg"], t["w1"], t["w2"], off, ids, t["b1"], t["b2"]).clone()
    got = {n: g.clone() for n, g in m.backward_full(dy, t["wg"], t["w1"], t["w2"]).items()}
    idx = m.topk_idx.long().cpu()
    p = {n: v.double().cpu().requires_grad_() for n, v in t.items()}
    weight = torch.softmax(torch.gather(p["x"] @ p["wg"], 1, idx), 1)
    want = torch.zeros(N, d, dtype=torch.float64)
    for e in range(E):
        tok, slot = torch.nonzero(idx == e, as_tuple=True)
        g, up = (p["x"][tok] @ p["w1"][e] + p["b1"][e]).split(f, 1)
        a = g * torch.sigmoid(g) if act == "silu" else g * 0.5 * torch.erfc(-g / 2 ** 0.5)
        want = want.index_add(0, tok, weight[tok, slot][:, None] * ((a * up) @ p["w2"][e] + p["b2"][e]))
    want.backward(dy.double().cpu())
    pairs = {"y": (y, want.detach()), **{n: (got["d" + n], p[n].grad) for n in p}}
    for name, (v, ref) in pairs.items():
        err = float((v.double().cpu() - ref).abs().max() / ref.abs().max())
        assert err <= (2e-2 if dtype == "bf16" else 1e-5), (name, err)
