"""One MoE layer on one GPU: buffers owned here, every step done by libflexmoe.

Forward (paper Section 3.1 workflow on a single GPU):
    gate_topk -> route(placement table) -> permute -> expert_ffn_fwd -> combine
Backward of the expert path for an upstream gradient dY (gate output held constant):
    permute(dY, row_scale = gate weights) -> expert_ffn_bwd -> combine(weights = None)
Gated experts (act(x Wg) * (x Wu), W1 = [Wg, Wu]) take expert_ffn_gated_fwd / _bwd in their place; serving with 8-bit weights
(QuantizedExperts) is gate_topk -> route -> expert_ffn_i8_fwd -> combine.

This class only allocates device memory once and sequences the C-ABI calls; it
does no arithmetic of its own.
"""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B
from . import workloads as W


def to_device(t, device="cuda"):
    """Upload a stored tensor (Bf16Tensor bit patterns or float32 ndarray) unchanged."""
    if t is None:
        return None
    if isinstance(t, W.Bf16Tensor):
        return torch.from_numpy(t.bits.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(t, dtype=np.float32)).to(device)


def to_host_f32(t: torch.Tensor) -> np.ndarray:
    return t.detach().float().cpu().numpy()


class QuantizedExperts:
    """The experts' weights as 8-bit integers with a scale per output channel, for MoELayer.forward_i8: made once from w1 [E, d, f]
    (gated: [E, d, 2 f]) and w2 [E, f, d]; the biases stay as they are."""

    def __init__(self, w1, w2, b1=None, b2=None):
        E, f, d = w2.shape
        cols = w1.shape[-1]
        if tuple(w1.shape) != (E, d, cols) or cols not in (f, 2 * f):
            raise ValueError(f"w1 {tuple(w1.shape)} is neither [E, d, f] nor [E, d, 2 f] for w2 [E, f, d] = {tuple(w2.shape)}")
        for b, n in ((b1, cols), (b2, d)):
            if b is not None and tuple(b.shape) != (E, n):
                raise ValueError(f"a bias of shape {tuple(b.shape)} where [{E}, {n}] belongs")
        self.sizes, self.gated = (E, d, f), cols == 2 * f
        self.b1, self.b2 = b1, b2
        (self.w1, self.s1), (self.w2, self.s2) = self._quantize(w1), self._quantize(w2)

    @staticmethod
    def _quantize(w):
        E, K, NC = w.shape
        q = torch.empty((E, NC, K), dtype=torch.int8, device=w.device)
        scale = torch.empty((E, NC), dtype=torch.float32, device=w.device)
        B.flexmoe_quantize_weights(w, q, scale)
        return q, scale


class MoELayer:
    def __init__(self, N, d, f, E, k, V, dtype, act, backward=False, device="cuda", keep_h=None, gated=False):
        """keep_h (training layers; default on): the forward pass leaves act(Hpre) in a buffer of the layer's
        and the backward pass reads it there instead of computing and storing it again -- A*f more elements
        of saved activations for a shorter backward pass.
        gated: w1 is [E, d, 2 f], the gate's columns first; b1 [E, 2 f].  f stays the width of the hidden activations.  self.hpre of a gated
        bf16 layer holds the 16-bit words that include/flexmoe.h describes, not bf16 numbers, whatever the tensor's type says.
        A layer that only ever serves 8-bit experts holds the other passes' buffers as well."""
        self.N, self.d, self.f, self.E, self.k, self.V = N, d, f, E, k, V
        self.A = N * k
        self.act = act
        self.gated = gated
        f1 = self.f1 = 2 * f if gated else f              # columns of w1 and hpre
        self.dtype_code = dtype
        tdt = torch.bfloat16 if dtype == B.BF16 else torch.float32
        dev = device
        i32 = dict(dtype=torch.int32, device=dev)
        A = self.A
        self.topk_idx = torch.empty((N, k), **i32)
        self.topk_w = torch.empty((N, k), dtype=torch.float32, device=dev)
        self.expert_count = torch.empty(E, **i32)
        self.vexpert_count = torch.empty(V, **i32)
        self.vexpert_off = torch.empty(V + 1, **i32)
        self.vexpert_owner = torch.empty(V, **i32)
        self.dest = torch.empty(A, **i32)
        self.src = torch.empty(A, **i32)
        self.xp = torch.empty((A, d), dtype=tdt, device=dev)
        self.hpre = torch.empty((A, f1), dtype=tdt, device=dev)
        self.yp = torch.empty((A, d), dtype=tdt, device=dev)
        self.y = torch.empty((N, d), dtype=tdt, device=dev)
        ws_bytes = B.flexmoe_workspace_bytes(N, d, f1, E, k, V, dtype)
        if ws_bytes == 0:
            raise ValueError("unsupported layer shape")
        self.ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        self.has_backward = backward
        self.h = None
        if backward and (keep_h is None or keep_h):
            self.h = torch.empty((A, f), dtype=tdt, device=dev)
        if backward:
            self.dyp = torch.empty((A, d), dtype=tdt, device=dev)
            self.dxp = torch.empty((A, d), dtype=tdt, device=dev)
            self.dx = torch.empty((N, d), dtype=tdt, device=dev)
            self.dw1 = torch.empty((E, d, f1), dtype=tdt, device=dev)
            self.dw2 = torch.empty((E, f, d), dtype=tdt, device=dev)

    @classmethod
    def for_config(cls, cfg: W.LayerConfig, device="cuda"):
        return cls(cfg.N, cfg.d, cfg.f, cfg.E, cfg.k, cfg.V, cfg.dtype, cfg.act, cfg.backward, device)

    # -- individual stages ------------------------------------------------
    def _ffn_fwd(self, w1, b1, w2, b2, hpre):
        call = B.flexmoe_expert_ffn_gated_fwd if self.gated else B.flexmoe_expert_ffn_fwd
        call(self.xp, self.vexpert_off, self.vexpert_owner, w1, b1, w2, b2, self.act, hpre, self.yp, self.ws, h=self.h)

    def _ffn_bwd(self, w1, w2):
        call = B.flexmoe_expert_ffn_gated_bwd if self.gated else B.flexmoe_expert_ffn_bwd
        call(self.dyp, self.xp, self.hpre, w1, w2, self.vexpert_off, self.vexpert_owner, self.act, self.dxp, self.dw1, self.dw2,
             self.ws, h=self.h)

    def _ungated_only(self, what):
        if self.gated:
            raise ValueError(f"{what} has no gated form")

    def gate(self, x, wg):
        B.flexmoe_gate_topk(x, wg, self.k, self.topk_idx, self.topk_w, self.ws)

    def route(self, rep_off, rep_ids):
        B.flexmoe_route(self.topk_idx, self.E, rep_off, rep_ids, self.expert_count, self.vexpert_count,
                        self.vexpert_off, self.vexpert_owner, self.dest, self.src, self.ws)

    def post_loads(self):
        """Start copying this step's expert loads I_e (expert_count, as the router wrote it) into
        pinned host memory on the current stream.  Returns (host int32 tensor, event): the host-side
        scheduler reads the tensor once the event has completed -- normally while later steps run --
        so the stream never waits for the host (Section 3.3: the Scheduler monitors the workloads
        next to the training loop)."""
        if not hasattr(self, "_loads_host"):
            self._loads_host = torch.empty(self.E, dtype=torch.int32, pin_memory=True)
        self._loads_host.copy_(self.expert_count, non_blocking=True)
        ev = torch.cuda.Event()
        ev.record()
        return self._loads_host, ev

    def profile_token_cost(self, w1, w2, reps: int = 3) -> int:
        """T_C of Eq. 7 from profiling: nanoseconds of expert computation (forward, plus backward for a
        training layer) per routed token, measured with HIP events around flexmoe_expert_ffn_fwd / _bwd on
        the buckets the layer currently holds (call after `forward`, and after `backward` for a training
        layer: xp, hpre, dyp must be filled).  The integer it returns is the `token_cost` (1 / TPS) the
        scheduler entry points take; a sync_cost table in the same unit (ns) then weighs T_Sync against it."""
        if self.A == 0:
            return 1
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]

        def once():
            self._ffn_fwd(w1, None, w2, None, self.hpre)
            if self.has_backward:
                self._ffn_bwd(w1, w2)
        once()
        ev[0].record()
        for _ in range(reps):
            once()
        ev[1].record()
        ev[1].synchronize()
        ns = ev[0].elapsed_time(ev[1]) * 1e6 / reps
        return max(1, int(round(ns / self.A)))

    def forward(self, x, wg, w1, w2, rep_off, rep_ids, b1=None, b2=None, keep_hpre=True):
        """keep_hpre=False (inference): the pre-activations are not stored; `backward` cannot follow."""
        self.gate(x, wg)
        self.route(rep_off, rep_ids)
        B.flexmoe_permute(x, self.src, None, self.k, self.xp)
        self._ffn_fwd(w1, b1, w2, b2, self.hpre if keep_hpre else None)
        B.flexmoe_combine(self.yp, self.dest, self.topk_w, self.k, self.y)
        return self.y

    def gather_supported(self) -> bool:
        return self.dtype_code == B.BF16 and self.d % 128 == 0 and self.N * self.d < 2 ** 32

    def forward_fused(self, x, wg, w1, w2, rep_off, rep_ids, b1=None, b2=None, keep_hpre=True):
        """Forward-only variant: the permutation is folded into the first expert GEMM (xp is not
        written, so `backward` cannot follow); keep_hpre=False also drops the pre-activations."""
        self._ungated_only("forward_fused")
        self.gate(x, wg)
        self.route(rep_off, rep_ids)
        B.flexmoe_expert_ffn_fwd_gather(x, self.src, self.k, self.vexpert_off, self.vexpert_owner, w1, b1, w2, b2,
                                        self.act, self.hpre if keep_hpre else None, self.yp, self.ws)
        B.flexmoe_combine(self.yp, self.dest, self.topk_w, self.k, self.y)
        return self.y

    def top1_supported(self) -> bool:
        return self.k == 1 and self.gather_supported() and self.f % 128 == 0

    def forward_top1(self, x, wg, w1, w2, rep_off, rep_ids, b1=None, b2=None, keep_hpre=True):
        """Forward-only top-1 layer: gate, route and one expert call that reads x through src and
        stores y through src (neither xp nor yp is written)."""
        self._ungated_only("forward_top1")
        self.gate(x, wg)
        self.route(rep_off, rep_ids)
        B.flexmoe_expert_ffn_fwd_top1(x, self.src, self.vexpert_off, self.vexpert_owner, w1, b1, w2, b2, self.act,
                                      self.hpre if keep_hpre else None, self.y, self.ws)
        return self.y

    def forward_i8(self, x, wg, experts: QuantizedExperts, rep_off, rep_ids):
        """Forward-only pass on 8-bit experts (gated or not, as they were made): x is read through src and quantised row by row;
        neither xp nor hpre is written."""
        if experts.gated != self.gated:
            raise ValueError("the experts were made for a layer of the other kind (gated or not)")
        if experts.sizes != (self.E, self.d, self.f):
            raise ValueError(f"experts of [E, d, f] = {experts.sizes} in a layer of {(self.E, self.d, self.f)}")
        if any(b is not None and b.dtype != self.y.dtype for b in (experts.b1, experts.b2)):
            raise ValueError("the experts' biases have another type than the layer")
        if not hasattr(self, "ws_i8"):
            nbytes = B.flexmoe_i8_workspace_bytes(self.N, self.d, self.f, self.E, self.k, self.V, int(self.gated))
            if nbytes == 0:
                raise ValueError("unsupported layer shape (8-bit experts: d and f multiples of 16)")
            self.ws_i8 = torch.empty(nbytes, dtype=torch.uint8, device=self.y.device)
        self.gate(x, wg)
        self.route(rep_off, rep_ids)
        B.flexmoe_expert_ffn_i8_fwd(x, self.src, self.k, self.vexpert_off, self.vexpert_owner, experts.w1, experts.s1, experts.b1,
                                    experts.w2, experts.s2, experts.b2, self.gated, self.act, self.yp, self.ws_i8)
        B.flexmoe_combine(self.yp, self.dest, self.topk_w, self.k, self.y)
        return self.y

    def backward(self, dy, w1, w2):
        """After `forward` (the one pass that fills xp, hpre and, with keep_h, h)."""
        B.flexmoe_permute(dy, self.src, self.topk_w, self.k, self.dyp)
        self._ffn_bwd(w1, w2)
        B.flexmoe_combine(self.dxp, self.dest, None, self.k, self.dx)
        return self.dx, self.dw1, self.dw2

    def backward_top1(self, dy, w1, w2):
        """`backward` for a top-1 layer: dX comes straight out of the expert backward (no dXp, no combine)."""
        self._ungated_only("backward_top1")
        B.flexmoe_permute(dy, self.src, self.topk_w, self.k, self.dyp)
        B.flexmoe_expert_ffn_bwd_top1(self.dyp, self.xp, self.hpre, w1, w2, self.vexpert_off, self.vexpert_owner,
                                      self.src, self.act, self.dx, self.dw1, self.dw2, self.ws, h=self.h)
        return self.dx, self.dw1, self.dw2

    def backward_full(self, dy, wg, w1, w2):
        """Backward of everything trainable: the expert path as in `backward`, plus the bias
        gradients and the gate path (dW_g, and the gate's share of dX added to self.dx)."""
        dev, tdt = self.dx.device, self.dx.dtype
        if not hasattr(self, "dwg"):
            self.db1 = torch.empty((self.E, self.f1), dtype=tdt, device=dev)
            self.db2 = torch.empty((self.E, self.d), dtype=tdt, device=dev)
            self.dl = torch.empty((self.N, self.k), dtype=torch.float32, device=dev)
            self.dwg = torch.empty((self.d, self.E), dtype=tdt, device=dev)
        B.flexmoe_permute(dy, self.src, self.topk_w, self.k, self.dyp)
        self._ffn_bwd(w1, w2)
        B.flexmoe_expert_bias_grads(self.dyp, self.vexpert_off, self.vexpert_owner, self.f1, self.E, self.db1,
                                    self.db2, self.ws)
        B.flexmoe_combine(self.dxp, self.dest, None, self.k, self.dx)
        B.flexmoe_gate_bwd(wg, self.topk_idx, self.topk_w, dy, self.yp, self.xp, self.dest, self.src,
                           self.vexpert_off, self.vexpert_owner, self.dl, self.dx, self.dwg, self.ws)
        return dict(dx=self.dx, dw1=self.dw1, dw2=self.dw2, db1=self.db1, db2=self.db2, dwg=self.dwg, dl=self.dl)
