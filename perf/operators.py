"""The gated expert FFN and the 8-bit integer expert products: what they are timed on.

Four passes, each on rows that a router has sorted into per-vExpert buckets (bucket v holds rows off[v] .. off[v+1] and
belongs to expert owner[v]):

  gated_fwd    forward pass of gated experts, nothing kept:  y = (act(x Wg + bg) * (x Wu + bu)) W2 + b2
  gated_train  the same with what the backward pass needs, then every gradient: dX, dW1 = [dWg, dWu], dW2 and, with
               biases, db1, db2
  i8_ffn       forward pass with weights in 8 bits and a scale per output channel; rows of x and of the hidden
               activations are quantised on the way, a scale per token
  i8_matmul    rows quantised, then one grouped 8-bit product (one expert: a plain dense product)

Inputs follow workloads.py: x ~ N(0, 1), weights ~ N(0, 0.02^2), upstream gradients ~ N(0, 1), expert loads by a Zipf
law, replicas given to the most loaded experts.  Rows that are quantised have a few channels with larger values, as
trained models' activations do.

With `own` the passes go through the framework's calls, otherwise through their plain form: elementary torch operations
in 32 bits, rounded once at the end (whole numbers by exact rules: the quotients that decide them are taken in 64 bits).
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_TINY = 2.0 ** -126                      # smallest scale: a row or channel of zeros has this one


def _case(name, op, dtype, N, d, f, E, k, V, zipf, act="silu", bias=False, gated=True):
    """op i8_matmul: d is the contraction, f the number of output columns; act and gated mean nothing."""
    c = {"op": op, "dtype": dtype, "N": N, "d": d, "f": f, "E": E, "k": k, "V": V, "zipf": zipf, "act": act, "bias": bias,
         "gated": gated}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one decode step of a small serving batch: a few rows for each of the experts, bound by their weights and by launches
        _case("gated_decode_16", "gated_fwd", "bf16", 16, 1024, 4096, 32, 2, 48, 0.8),
        # a prompt of ragged length through wide experts
        _case("gated_prompt_2000", "gated_fwd", "bf16", 2000, 2048, 4096, 16, 2, 20, 1.0),
        # fp32 training of a small layer: gradient checks, reference runs
        _case("gated_train_fp32", "gated_train", "f32", 1000, 256, 512, 8, 2, 10, 1.0, "gelu", True),
        # sizes that are no multiples of any tile, three experts per token, biases
        _case("gated_train_odd", "gated_train", "bf16", 1501, 328, 904, 12, 3, 15, 1.2, "gelu_tanh", True),
        # the GPT-medium-like layer with gated experts of half the width, training
        _case("gated_train_mid", "gated_train", "bf16", 16384, 1024, 2048, 32, 2, 48, 1.2),
        # a large training batch of wide gated experts
        _case("gated_train_large", "gated_train", "bf16", 32768, 2048, 5632, 32, 2, 40, 1.2),
        # a single token: the smallest serving call
        _case("i8_one_token", "i8_ffn", "bf16", 1, 1024, 4096, 8, 2, 8, 0.0),
        # one decode step of a larger serving batch: nearly every expert's weights for a row or two
        _case("i8_decode_48", "i8_ffn", "bf16", 48, 2048, 4096, 64, 2, 80, 0.8),
        # a ragged prompt through experts without a gate, with biases
        _case("i8_gelu_prompt", "i8_ffn", "bf16", 3001, 784, 2064, 16, 2, 18, 1.0, "gelu", True, False),
        # a large batch of prompts
        _case("i8_large", "i8_ffn", "bf16", 32768, 2048, 5632, 32, 2, 40, 1.2),
        # a dense product over all tokens, as the projections around the experts are
        _case("i8_dense", "i8_matmul", "bf16", 4096, 2048, 6144, 1, 1, 1, 0.0),
        # one projection of small experts, fp32 in and out
        _case("i8_grouped_fp32", "i8_matmul", "f32", 300, 1040, 1000, 8, 2, 10, 0.8, "silu", True),
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    while True:
        op = rng.choice(["gated_fwd", "gated_train", "i8_ffn", "i8_matmul"])
        i8 = op.startswith("i8")
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        step = 16 if i8 else 8
        N, d, f = _log_int(rng, 1, 32768), _log_int(rng, 64, 2048, step), _log_int(rng, 64, 5632, step)
        E = 1 if op == "i8_matmul" and rng.random() < 0.4 else _log_int(rng, 1, 64)
        k = min(E, rng.choice([1, 2, 2, 3, 4]))
        V = E + rng.randint(0, E // 2)
        c = _case(None, op, dtype, N, d, f, E, k, V, rng.choice([0.0, 0.5, 1.0, 1.5]), rng.choice(["silu", "gelu", "gelu_tanh", "relu"]),
                  rng.random() < 0.4, rng.random() < 0.6 or not op == "i8_ffn")
        if work(c)["flops"] <= (1.2e13 if dtype == "bf16" or i8 else 5e11) and E * d * f <= 3.7e8:
            return c


# ---- inputs ----------------------------------------------------------------------------------
def _shares(case):
    p = [(r + 1.0) ** -case["zipf"] for r in range(case["E"])]
    s = sum(p)
    return [v / s for v in p]


def _routing(case, gen):
    """The buckets a router leaves: host offsets and owners, src[p] = assignment of bucket row p, and the device copies."""
    N, E, k, V = case["N"], case["E"], case["k"], case["V"]
    p = torch.tensor(_shares(case), device="cuda")[torch.randperm(E, generator=gen, device="cuda")]
    noise = -torch.log(-torch.log(torch.rand(N, E, generator=gen, device="cuda").clamp(1e-7, 1 - 1e-7)))
    expert = torch.topk(torch.log(p) + noise, k, dim=1).indices.reshape(-1)
    # every expert one vExpert, further ones to whoever has the largest share per replica; ids dealt in that order
    share, reps, owner = p.tolist(), [1] * E, list(range(E))
    while len(owner) < V:
        e = max(range(E), key=lambda i: share[i] / reps[i])
        reps[e] += 1
        owner.append(e)
    ids = [[v for v in range(V) if owner[v] == e] for e in range(E)]
    order = torch.argsort(expert, stable=True)
    counts = torch.bincount(expert, minlength=E).tolist()
    chunks, at, sizes = [None] * V, 0, [0] * V
    for e in range(E):
        n = len(ids[e])
        for r, v in enumerate(ids[e]):
            take = counts[e] // n + (1 if r < counts[e] % n else 0)
            chunks[v], sizes[v] = order[at:at + take], take
            at += take
    off = [0]
    for s in sizes:
        off.append(off[-1] + s)
    return {"off": off, "owner": owner, "src": torch.cat(chunks).int(),
            "voff": torch.tensor(off, dtype=torch.int32, device="cuda"), "vowner": torch.tensor(owner, dtype=torch.int32, device="cuda")}


def _weights_i8(E, K, NC, gen):
    """[E, NC, K] int8 (the contraction contiguous) and [E, NC] fp32, as the framework's quantiser lays them out."""
    q = torch.empty(E, NC, K, dtype=torch.int8, device="cuda")
    s = torch.empty(E, NC, dtype=torch.float32, device="cuda")
    for e in range(E):
        w = torch.randn(NC, K, generator=gen, device="cuda") * 0.02
        s[e] = w.abs().amax(1) / 127
        q[e] = torch.round(w.double() / s[e].double()[:, None]).to(torch.int8)
    return q, s


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, op = _DT[case["dtype"]], case["op"]
    N, d, f, E, k = (case[n] for n in "NdfEk")
    A = N * k

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dt)

    st = {"case": case, "act": case["act"], **_routing(case, gen)}
    x = normal(N, d)
    if op.startswith("gated"):
        st["xp"] = x[st["src"].long() // k].contiguous()
        st["w1"] = torch.empty(E, d, 2 * f, dtype=dt, device="cuda")
        st["w2"] = torch.empty(E, f, d, dtype=dt, device="cuda")
        for e in range(E):
            st["w1"][e], st["w2"][e] = normal(d, 2 * f, std=0.02), normal(f, d, std=0.02)
        st["b1"], st["b2"] = (normal(E, 2 * f, std=0.1), normal(E, d, std=0.1)) if case["bias"] else (None, None)
        if op == "gated_train":
            st["dyp"] = normal(A, d)
        return st
    x[:, ::61] *= 6
    st["x"] = x
    cols = 2 * f if op == "i8_ffn" and case["gated"] else f
    st["w1"], st["s1"] = _weights_i8(E, d, cols, gen)
    st["b1"] = normal(E, cols, std=0.1) if case["bias"] else None
    if op == "i8_ffn":
        st["w2"], st["s2"] = _weights_i8(E, f, d, gen)
        st["b2"] = normal(E, d, std=0.1) if case["bias"] else None
    return st


# ---- the framework's calls ---------------------------------------------------------------------
def _buffers(st):
    """Outputs and workspace, allocated once as a layer does."""
    if "buf" in st:
        return st["buf"]
    from paper_2304_03946_amd import binding as B
    case = st["case"]
    dt, op = _DT[case["dtype"]], case["op"]
    N, d, f, E, k, V = (case[n] for n in ("N", "d", "f", "E", "k", "V"))
    A = N * k

    def new(*shape, dtype=dt):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    b = {"act": {"relu": B.RELU, "gelu": B.GELU_ERF, "gelu_tanh": B.GELU_TANH, "silu": B.SILU}[case["act"]]}
    if op.startswith("gated"):
        ws = B.flexmoe_workspace_bytes(N, d, 2 * f, E, k, V, B.BF16 if case["dtype"] == "bf16" else B.F32)
        b["yp"] = new(A, d)
        if op == "gated_train":
            b.update(hpre=new(A, 2 * f), h=new(A, f), dxp=new(A, d), dw1=new(E, d, 2 * f), dw2=new(E, f, d))
            if case["bias"]:
                b.update(db1=new(E, 2 * f), db2=new(E, d))
    elif op == "i8_ffn":
        ws = B.flexmoe_i8_workspace_bytes(N, d, f, E, k, V, int(case["gated"]))
        b["yp"] = new(A, d)
    else:
        ws = B.flexmoe_i8_workspace_bytes(N, d, f, E, k, V, 0)
        b.update(q=new(N, d, dtype=torch.int8), s=new(N, dtype=torch.float32), yp=new(A, f))
    b["ws"] = new(ws, dtype=torch.uint8)
    st["buf"] = b
    return b


def _run_own(st):
    from paper_2304_03946_amd import binding as B
    case, b = st["case"], _buffers(st)
    op, k = case["op"], case["k"]
    at = (st["voff"], st["vowner"])
    if op == "gated_fwd":
        B.flexmoe_expert_ffn_gated_fwd(st["xp"], *at, st["w1"], st["b1"], st["w2"], st["b2"], b["act"], None, b["yp"], b["ws"])
        return {"yp": b["yp"]}
    if op == "gated_train":
        B.flexmoe_expert_ffn_gated_fwd(st["xp"], *at, st["w1"], st["b1"], st["w2"], st["b2"], b["act"], b["hpre"], b["yp"], b["ws"],
                                       h=b["h"])
        B.flexmoe_expert_ffn_gated_bwd(st["dyp"], st["xp"], b["hpre"], st["w1"], st["w2"], *at, b["act"], b["dxp"], b["dw1"], b["dw2"],
                                       b["ws"], h=b["h"])
        out = {n: b[n] for n in ("yp", "dxp", "dw1", "dw2")}
        if case["bias"]:
            B.flexmoe_expert_bias_grads(st["dyp"], *at, 2 * case["f"], case["E"], b["db1"], b["db2"], b["ws"])
            out.update(db1=b["db1"], db2=b["db2"])
        return out
    if op == "i8_ffn":
        B.flexmoe_expert_ffn_i8_fwd(st["x"], st["src"], k, *at, st["w1"], st["s1"], st["b1"], st["w2"], st["s2"], st["b2"],
                                    int(case["gated"]), b["act"], b["yp"], b["ws"])
        return {"yp": b["yp"]}
    B.flexmoe_quantize_rows(st["x"], b["q"], b["s"])
    B.flexmoe_expert_matmul_i8(b["q"], b["s"], st["src"], k, *at, st["w1"], st["s1"], st["b1"], b["yp"], b["ws"])
    return {"yp": b["yp"]}


# ---- plain forms -------------------------------------------------------------------------------
def _act(kind, z):
    if kind == "relu":
        return torch.clamp(z, min=0)
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))


def _act_grad(kind, z):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (z + 0.044715 * z * z * z))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)


def _quantise(rounded, largest):
    """Whole numbers (as floats) and scales of rows: scale = largest / 127, numbers to the nearest, ties to even."""
    s = torch.clamp(largest.float() / 127, min=_TINY)
    return torch.clamp(torch.round(rounded.double() / s.double()[:, None]), -127, 127).float(), s


def _run_plain(st):
    case = st["case"]
    dt, op, act = _DT[case["dtype"]], case["op"], case["act"]
    f, E, k = case["f"], case["E"], case["k"]
    off, owner = st["off"], st["owner"]
    if op.startswith("gated"):
        xp, train = st["xp"], op == "gated_train"
        out = {"yp": torch.empty_like(xp)}
        if train:
            out["dxp"] = torch.empty_like(xp)
            sums = {}
        for v, e in enumerate(owner):
            lo, hi = off[v], off[v + 1]
            if lo == hi:
                continue
            x, w1, w2 = xp[lo:hi].float(), st["w1"][e].float(), st["w2"][e].float()
            z = x @ w1
            if st["b1"] is not None:
                z = z + st["b1"][e].float()
            g, u = z[:, :f], z[:, f:]
            a = _act(act, g)
            h = a * u
            y = h @ w2
            if st["b2"] is not None:
                y = y + st["b2"][e].float()
            out["yp"][lo:hi] = y.to(dt)
            if train:
                dy = st["dyp"][lo:hi].float()
                dh = dy @ w2.T
                dz = torch.cat([dh * u * _act_grad(act, g), dh * a], 1)
                out["dxp"][lo:hi] = (dz @ w1.T).to(dt)
                parts = [x.T @ dz, h.T @ dy] + ([dz.sum(0), dy.sum(0)] if case["bias"] else [])
                sums[e] = [p + q for p, q in zip(sums[e], parts)] if e in sums else parts
                if e not in owner[v + 1:]:                       # the expert's last bucket
                    for n, p in zip(("dw1", "dw2", "db1", "db2"), sums.pop(e)):
                        out.setdefault(n, torch.zeros(E, *p.shape, dtype=dt, device="cuda"))[e] = p.to(dt)
        if train:
            for e, parts in sums.items():                        # experts whose last bucket is empty
                for n, p in zip(("dw1", "dw2", "db1", "db2"), parts):
                    out.setdefault(n, torch.zeros(E, *p.shape, dtype=dt, device="cuda"))[e] = p.to(dt)
        return out
    q, s = _quantise(st["x"], st["x"].float().abs().amax(1))
    token = st["src"].long() // k
    cols = case["d"] if op == "i8_ffn" else f
    yp = torch.empty(case["N"] * k, cols, dtype=dt, device="cuda")
    for v, e in enumerate(owner):
        lo, hi = off[v], off[v + 1]
        if lo == hi:
            continue
        t = token[lo:hi]
        z = (q[t] @ st["w1"][e].float().T) * (s[t][:, None] * st["s1"][e])
        if st["b1"] is not None:
            z = z + st["b1"][e].float()
        if op == "i8_ffn":
            h = _act(act, z[:, :f]) * z[:, f:] if case["gated"] else _act(act, z)
            hq, hs = _quantise(h.to(dt), h.abs().amax(1))        # numbers of the rows as stored, scales of the rows before that
            z = (hq @ st["w2"][e].float().T) * (hs[:, None] * st["s2"][e])
            if st["b2"] is not None:
                z = z + st["b2"][e].float()
        yp[lo:hi] = z.to(dt)
    return {"yp": yp}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ---------------------------------------------------------------
def _experts_used(case):
    """Experts that some token goes to, on average."""
    return sum(1 - (1 - min(1.0, case["k"] * p)) ** case["N"] for p in _shares(case))


def work(case):
    """Inputs once (the weights of experts with tokens only), outputs once; two operations per product and sum."""
    op, N, d, f, E, k = (case[n] for n in ("op", "N", "d", "f", "E", "k"))
    A, s, used = N * k, 2 if case["dtype"] == "bf16" else 4, _experts_used(case)
    if op == "i8_matmul":
        return {"bytes": N * d * s + used * f * (d + 4 + (s if case["bias"] else 0)) + A * (f * s + 4), "flops": 2 * A * d * f}
    cols = 2 * f if case["gated"] else f
    bias = used * (cols + d) * s if case["bias"] else 0
    product = 2 * A * d * (cols + f)
    if op == "i8_ffn":
        return {"bytes": N * d * s + used * (d * (cols + f) + 4 * (cols + d)) + bias + A * (d * s + 4), "flops": product}
    weights = used * d * (cols + f) * s
    if op == "gated_fwd":
        return {"bytes": 2 * A * d * s + weights + bias, "flops": product}
    # forward and backward: x and dy in, y and dx out, weights in, their gradients out
    return {"bytes": 4 * A * d * s + weights + bias + E * (d * (cols + f) + (cols + d if case["bias"] else 0)) * s, "flops": 3 * product}


# ---- the definition in 64 bits -------------------------------------------------------------------
def _sigma(t):
    return torch.special.expit(t)


_VALUE = {"relu": lambda t: t * (t > 0), "silu": lambda t: t * _sigma(t), "gelu": lambda t: t * torch.special.ndtr(t),
          "gelu_tanh": lambda t: t * _sigma(2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3))}


def _slope(kind, t):
    if kind == "relu":
        return (t > 0).double()
    if kind == "silu":
        return _sigma(t) + t * _sigma(t) * _sigma(-t)
    if kind == "gelu":
        return torch.special.ndtr(t) + t * torch.exp(-t * t / 2) / math.sqrt(2 * math.pi)
    arg = 2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t ** 3)
    return _sigma(arg) + t * _sigma(arg) * _sigma(-arg) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * t ** 2)


def _whole(values, scale):
    ratio = values / scale[:, None]
    return torch.clamp(torch.round(ratio), -127.0, 127.0)


def exact(case, seed):
    """Expert by expert: all rows of an expert at once, whichever bucket they lie in."""
    if work(case)["flops"] > 3e14:
        return None
    st = prepare(case, seed)
    op, kind, f, E, k = case["op"], case["act"], case["f"], case["E"], case["k"]
    lengths = torch.tensor([st["off"][v + 1] - st["off"][v] for v in range(case["V"])], device="cuda")
    row_expert = torch.repeat_interleave(torch.tensor(st["owner"], device="cuda"), lengths)
    width = f if op == "i8_matmul" else case["d"]
    res = {"yp": torch.zeros(case["N"] * k, width, dtype=torch.float64, device="cuda")}
    if op == "gated_train":
        res["dxp"] = torch.zeros_like(res["yp"])
        res["dw1"] = torch.zeros(st["w1"].shape, dtype=torch.float64, device="cuda")
        res["dw2"] = torch.zeros(st["w2"].shape, dtype=torch.float64, device="cuda")
        if case["bias"]:
            res["db1"], res["db2"] = torch.zeros_like(res["dw1"][:, 0]), torch.zeros_like(res["dw2"][:, 0])

    def shift(m, b, e):
        return m if b is None else m + b[e].double()

    if op.startswith("i8"):
        xd = st["x"].double()
        xs = (xd.abs().max(dim=1).values / 127).float().double().clamp(min=_TINY)
        tokens = st["src"].long().div(k, rounding_mode="floor")
        xi = _whole(xd, xs) * xs[:, None]
    for e in range(E):
        rows = torch.nonzero(row_expert == e).flatten()
        if rows.numel() == 0:
            continue
        if op.startswith("gated"):
            xe, w1, w2 = st["xp"][rows].double(), st["w1"][e].double(), st["w2"][e].double()
            pre = shift(torch.mm(xe, w1), st["b1"], e)
            gate, up = pre.split(f, dim=1)
            hidden = _VALUE[kind](gate) * up
            res["yp"][rows] = shift(torch.mm(hidden, w2), st["b2"], e)
            if op == "gated_train":
                dye = st["dyp"][rows].double()
                dhid = torch.mm(dye, w2.t().contiguous())
                dgate, dup = dhid * up * _slope(kind, gate), dhid * _VALUE[kind](gate)
                res["dxp"][rows] = torch.mm(dgate, w1[:, :f].t().contiguous()) + torch.mm(dup, w1[:, f:].t().contiguous())
                xt = xe.t().contiguous()
                res["dw1"][e, :, :f], res["dw1"][e, :, f:] = torch.mm(xt, dgate), torch.mm(xt, dup)
                res["dw2"][e] = torch.mm(hidden.t().contiguous(), dye)
                if case["bias"]:
                    res["db1"][e], res["db2"][e] = torch.cat([dgate.sum(0), dup.sum(0)]), dye.sum(0)
            continue
        w1 = st["w1"][e].double() * st["s1"][e].double()[:, None]
        z = shift(torch.mm(xi[tokens[rows]], w1.t().contiguous()), st["b1"], e)
        if op == "i8_ffn":
            hidden = _VALUE[kind](z[:, :f]) * z[:, f:] if case["gated"] else _VALUE[kind](z)
            hs = (hidden.abs().max(dim=1).values / 127).clamp(min=_TINY)
            hi = _whole(hidden.to(_DT[case["dtype"]]).double(), hs) * hs[:, None]
            z = shift(torch.mm(hi, (st["w2"][e].double() * st["s2"][e].double()[:, None]).t().contiguous()), st["b2"], e)
        res["yp"][rows] = z
    return res
