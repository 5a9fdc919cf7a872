"""One MoE expert layer on the GPU: torch owns the buffers, libpcmoe computes every step.

Forward (Alg. 3 with the gating of Alg. 7 and the experts of Alg. 6):
    moe_route -> moe_permute -> moe_expert_ffn_fwd -> moe_combine
Backward (Alg. 5 / Alg. 6 and the owner-side router adjoint):
    moe_combine_bwd -> moe_expert_ffn_bwd -> moe_route_bwd (full layer only) -> moe_permute_bwd
With a gate, moe_route_gated and moe_route_gated_bwd take the place of the routing calls. With checkpoint=True the forward
ends in moe_ffn_checkpoint and the backward begins with moe_ffn_restore. forward_q4 runs the experts from 4-bit weights,
forward_q8 in 8-bit integers.
Expert update (the last step of Alg. 6): moe_expert_update over the hosted experts' weights, or moe_expert_update_muon.
MoEStack chains layers with moe_residual_norm between them, and their adjoints.
All calls are enqueued on one stream; no per-expert count ever returns to the host.
"""
from __future__ import annotations

from copy import copy
from dataclasses import dataclass
from typing import Optional

import numpy as np
import torch

from . import pcmoe as P


@dataclass
class LayerWeights:
    x: torch.Tensor
    w_router: torch.Tensor
    logit_bias: Optional[torch.Tensor]
    bias_groups: int
    w_gate: torch.Tensor
    w_up: torch.Tensor
    w_down: torch.Tensor
    dy: Optional[torch.Tensor] = None
    select_bias: Optional[torch.Tensor] = None   # [E] fp32, gated routing only


def torch_dtype(dtype: str):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def upload(inp, device="cuda") -> LayerWeights:
    """Copy a synth.LayerInputs (float32 arrays, bf16-exact for bf16 layers) to the device."""
    cfg = inp.cfg
    dt = torch_dtype(cfg.dtype)
    to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device=device).to(dt)
    bias = None
    if inp.logit_bias is not None:
        bias = torch.from_numpy(np.ascontiguousarray(inp.logit_bias, dtype=np.float32)).to(device)
    return LayerWeights(to(inp.x), to(inp.w_router), bias, cfg.bias_groups, to(inp.w_gate), to(inp.w_up),
                        to(inp.w_down), None if inp.dy is None else to(inp.dy))


@dataclass
class Q4Experts:
    """4-bit codes and group scales of the experts' gate, up and down projections."""
    group: int
    gate: tuple
    up: tuple
    down: tuple

    @staticmethod
    def pack(w: LayerWeights, group: int = 64) -> "Q4Experts":
        names = {torch.bfloat16: "bf16", torch.float32: "f32"}

        def one(t):
            if t.dtype not in names:
                raise ValueError(f"weights of dtype {t.dtype}: bfloat16 or float32 are packed")
            n, rows, cols = t.shape
            codes = torch.empty(n, rows // 16, cols // 128, 4, 16, 4, 4, dtype=torch.uint8, device=t.device)
            scales = torch.empty(n, rows // 16, cols // group, 16, dtype=torch.bfloat16, device=t.device)
            P.moe_q4_pack(n, rows, cols, group, names[t.dtype], t, codes, scales)
            return codes, scales
        return Q4Experts(group, one(w.w_gate), one(w.w_up), one(w.w_down))


@dataclass
class Q8Experts:
    """8-bit codes and channel scales of the experts' gate, up and down projections."""
    gate: tuple
    up: tuple
    down: tuple

    @staticmethod
    def pack(w: LayerWeights) -> "Q8Experts":
        names = {torch.bfloat16: "bf16", torch.float32: "f32"}

        def one(t):
            if t.dtype not in names:
                raise ValueError(f"weights of dtype {t.dtype}: bfloat16 or float32 are packed")
            n, rows, cols = t.shape
            codes = torch.empty(n, rows, cols, dtype=torch.int8, device=t.device)
            scales = torch.empty(n, rows, dtype=torch.float32, device=t.device)
            P.moe_q8_pack(n, rows, cols, names[t.dtype], t, codes, scales)
            return codes, scales
        return Q8Experts(one(w.w_gate), one(w.w_up), one(w.w_down))


class MoELayer:
    """gate: a pcmoe.make_gate(...) for gated routing. checkpoint: keep the activations of the backward in 8 bits;
    `saved`, the buffer of their full form, may then be shared by layers that run one after the other: at least
    MOE_WS_FFN_SAVED bytes of the largest of them."""

    def __init__(self, cfg, device="cuda", backward=None, router_backward=None, gate=None, checkpoint=False, saved=None):
        self.cfg = cfg
        self.gate = gate
        self.checkpoint = checkpoint
        self.device = device
        self.backward_enabled = cfg.backward if backward is None else backward
        self.router_backward = cfg.router_backward if router_backward is None else router_backward
        self.desc = P.make_desc(cfg.T, cfg.d, cfg.f, cfg.E, cfg.k, cfg.local_begin, cfg.n_local, cfg.n_shared,
                                cfg.renormalize, cfg.dtype)
        T, d, f, E, k, S, Eloc = cfg.T, cfg.d, cfg.f, cfg.E, cfg.k, cfg.n_shared, cfg.n_local
        dt = torch_dtype(cfg.dtype)
        R = T * k + S * T
        kw = dict(device=device)
        self.logits = torch.empty(T, E, dtype=torch.float32, **kw)
        self.topk_idx = torch.empty(T, k, dtype=torch.int32, **kw)
        self.topk_w = torch.empty(T, k, dtype=torch.float32, **kw)
        self.counts = torch.empty(max(Eloc, 1), dtype=torch.int32, **kw)
        self.offsets = torch.empty(Eloc + 1, dtype=torch.int32, **kw)
        self.row_to_slot = torch.empty(T * k, dtype=torch.int32, **kw)
        self.slot_to_row = torch.empty(T * k, dtype=torch.int32, **kw)
        self.x_perm = torch.empty(T * k, d, dtype=dt, **kw)
        self.y_perm = torch.empty(R, d, dtype=dt, **kw)
        self.y = torch.empty(T, d, dtype=dt, **kw)
        ws = lambda which: torch.empty(max(P.moe_workspace_size(self.desc, which), 1), dtype=torch.uint8, **kw)
        self.ws_permute = ws(P.MOE_WS_PERMUTE)
        if saved is not None:
            self._check_saved(saved)
        self.saved = ws(P.MOE_WS_FFN_SAVED) if saved is None else saved
        if checkpoint:
            self.ckpt = ws(P.MOE_WS_FFN_CKPT)
        self.ws_q4 = None   # of forward_q4 and forward_q8, allocated by their first calls
        self.ws_q8 = None
        self.saved_nothing = False  # the last forward was forward_q4 or forward_q8
        self.runs = 0       # forwards so far: what the activations are of
        self.ws_ffn_fwd = ws(P.MOE_WS_FFN_FWD)
        if self.backward_enabled:
            G = Eloc + S
            self.dy_perm = torch.empty(T * k, d, dtype=dt, **kw)
            self.dgate = torch.empty(T, k, dtype=torch.float32, **kw)
            self.dx_perm = torch.empty(R, d, dtype=dt, **kw)
            self.dw_gate = torch.empty(G, f, d, dtype=dt, **kw)
            self.dw_up = torch.empty(G, f, d, dtype=dt, **kw)
            self.dw_down = torch.empty(G, d, f, dtype=dt, **kw)
            self.ws_ffn_bwd = ws(P.MOE_WS_FFN_BWD)
            self.dx = torch.empty(T, d, dtype=dt, **kw)
            if self.router_backward:
                self.dlogits = torch.empty(T, E, dtype=torch.float32, **kw)
                self.dw_router = torch.empty(E, d, dtype=torch.float32, **kw)
                self.ws_route_bwd = ws(P.MOE_WS_ROUTE_BWD)

    def _check_saved(self, saved):
        """The calls that write a saved buffer do not take its size, so a caller's is measured here."""
        if not self.checkpoint:
            raise ValueError("a shared saved buffer needs checkpoint=True: it does not outlive the next layer's forward")
        if saved.device != self.logits.device:
            raise ValueError(f"the shared saved buffer is on device {saved.device}, the layer on {self.logits.device}")
        if not saved.is_contiguous():
            raise ValueError("the shared saved buffer is not contiguous")
        need, have = P.moe_workspace_size(self.desc, P.MOE_WS_FFN_SAVED), saved.numel() * saved.element_size()
        if have < need:
            raise ValueError(f"the shared saved buffer has {have} bytes, this layer needs {need} bytes (MOE_WS_FFN_SAVED)")

    # ------------------------------------------------------------------ forward
    def route(self, w: LayerWeights):
        if self.gate is not None:
            P.moe_route_gated(self.desc, self.gate, w.x, w.w_router, w.logit_bias, w.bias_groups, w.select_bias,
                              self.logits, self.topk_idx, self.topk_w)
            return
        P.moe_route(self.desc, w.x, w.w_router, w.logit_bias, w.bias_groups, self.logits, self.topk_idx, self.topk_w)

    def permute(self, w: LayerWeights):
        self.runs += 1
        P.moe_permute(self.desc, self.topk_idx, w.x, self.counts, self.offsets, self.row_to_slot, self.slot_to_row,
                      self.x_perm, self.ws_permute, self.ws_permute.numel())

    def ffn_fwd(self, w: LayerWeights):
        self.saved_nothing = False
        P.moe_expert_ffn_fwd(self.desc, w.x, self.x_perm, self.offsets, w.w_gate, w.w_up, w.w_down, self.y_perm,
                             self.saved, self.ws_ffn_fwd, self.ws_ffn_fwd.numel())
        if self.checkpoint:
            P.moe_ffn_checkpoint(self.desc, self.offsets, self.saved, self.ckpt, self.ckpt.numel())

    def combine(self):
        P.moe_combine(self.desc, self.y_perm, self.slot_to_row, self.topk_w, self.y)

    def forward(self, w: LayerWeights):
        self.route(w)
        self.permute(w)
        self.ffn_fwd(w)
        self.combine()
        return self.y

    def forward_q4(self, w: LayerWeights, q: Q4Experts):
        """The forward with the experts' 4-bit weights (inference: nothing is saved, no backward can
        follow; w's expert weights are not read and may be None)."""
        if self.ws_q4 is None:
            self.ws_q4 = torch.empty(P.moe_workspace_size(self.desc, P.MOE_WS_FFN_Q4), dtype=torch.uint8,
                                     device=self.device)
        self.saved_nothing = True
        self.route(w)
        self.permute(w)
        P.moe_expert_ffn_q4(self.desc, q.group, w.x, self.x_perm, self.offsets, *q.gate, *q.up, *q.down, self.y_perm,
                            self.ws_q4, self.ws_q4.numel())
        self.combine()
        return self.y

    def _check_q8(self, q: Q8Experts):
        G, d, f = self.cfg.n_local + self.cfg.n_shared, self.cfg.d, self.cfg.f
        for name, rows, cols in (("gate", f, d), ("up", f, d), ("down", d, f)):
            for t, shape, dtype in zip(getattr(q, name), ((G, rows, cols), (G, rows)), (torch.int8, torch.float32)):
                if t is not None and (tuple(t.shape) != shape or t.dtype != dtype):
                    raise ValueError(f"8-bit {name}: {tuple(t.shape)} {t.dtype}, this layer takes {shape} {dtype}")

    def forward_q8(self, w: LayerWeights, q: Q8Experts):
        """The forward of a bf16 layer with the experts in 8-bit integers (inference, prompts above all: nothing is saved, no
        backward can follow; w's expert weights are not read and may be None)."""
        if self.cfg.dtype != "bf16":
            raise ValueError("experts in 8-bit integers are for bf16 layers")
        self._check_q8(q)
        if self.ws_q8 is None:
            self.ws_q8 = torch.empty(P.moe_workspace_size(self.desc, P.MOE_WS_FFN_Q8), dtype=torch.uint8,
                                     device=self.device)
        self.saved_nothing = True
        self.route(w)
        self.permute(w)
        P.moe_expert_ffn_q8(self.desc, w.x, self.x_perm, self.offsets, *q.gate, *q.up, *q.down, self.y_perm, self.ws_q8,
                            self.ws_q8.numel())
        self.combine()
        return self.y

    # ----------------------------------------------------------------- backward
    def _need_saved(self):
        if self.saved_nothing:
            raise RuntimeError("the last forward was forward_q4 or forward_q8, which save nothing for a backward")

    def combine_bwd(self, dy):
        P.moe_combine_bwd(self.desc, dy, self.y_perm, self.slot_to_row, self.topk_w, self.dy_perm, self.dgate)

    def ffn_bwd(self, w: LayerWeights, dy):
        self._need_saved()
        if self.checkpoint:
            P.moe_ffn_restore(self.desc, self.offsets, self.ckpt, self.ckpt.numel(), self.saved)
        P.moe_expert_ffn_bwd(self.desc, w.x, self.x_perm, dy, self.dy_perm, self.offsets, w.w_gate, w.w_up, w.w_down,
                             self.saved, self.dx_perm, self.dw_gate, self.dw_up, self.dw_down, self.ws_ffn_bwd,
                             self.ws_ffn_bwd.numel())

    def route_bwd(self, w: LayerWeights):
        if self.gate is not None:
            P.moe_route_gated_bwd(self.desc, self.gate, w.x, self.logits, self.topk_idx, self.topk_w, self.dgate,
                                  self.dlogits, self.dw_router, self.ws_route_bwd, self.ws_route_bwd.numel())
            return
        P.moe_route_bwd(self.desc, w.x, self.logits, self.topk_idx, self.topk_w, self.dgate, self.dlogits,
                        self.dw_router, self.ws_route_bwd, self.ws_route_bwd.numel())

    def permute_bwd(self, w: LayerWeights):
        P.moe_permute_bwd(self.desc, self.dx_perm, self.slot_to_row, self.dlogits if self.router_backward else None,
                          w.w_router, self.dx)

    def backward(self, w: LayerWeights, dy=None):
        self._need_saved()
        dy = w.dy if dy is None else dy
        self.combine_bwd(dy)
        self.ffn_bwd(w, dy)
        if self.router_backward:
            self.route_bwd(w)
        self.permute_bwd(w)
        return self.dx

    # ------------------------------------------------------------- expert update
    def init_update_state(self, w: LayerWeights, master: bool = True):
        """fp32 optimiser state over w_gate, w_up, w_down (in that order): zero moments and, if asked,
        a master copy of the current weights."""
        n = w.w_gate.numel() + w.w_up.numel() + w.w_down.numel()
        kw = dict(device=self.device, dtype=torch.float32)
        self.opt_m = torch.zeros(n, **kw)
        self.opt_v = torch.zeros(n, **kw)
        self.opt_master = self._master(w) if master else None
        self.opt_step = 0

    def _master(self, w: LayerWeights):
        parts = (w.w_gate, w.w_up, w.w_down)
        out = torch.empty(sum(t.numel() for t in parts), device=self.device, dtype=torch.float32)
        o = 0
        for t in parts:  # filled slice by slice: no transient copy of all parameters
            out[o:o + t.numel()].copy_(t.reshape(-1))
            o += t.numel()
        return out

    def update(self, w: LayerWeights, opt: "P.moe_opt"):
        """One optimiser step of the hosted experts from the gradients of the last backward."""
        self.opt_step += 1
        opt.step = self.opt_step
        P.moe_expert_update(self.desc, opt, w.w_gate, w.w_up, w.w_down, self.dw_gate, self.dw_up, self.dw_down,
                            self.opt_master, self.opt_m, self.opt_v)

    def init_muon_state(self, w: LayerWeights, master: bool = True, precise: bool = False):
        """State of update_muon: a zero momentum, the workspace and, if asked, a master copy of the current weights. precise:
        for updates with precise=True, whose workspace is twice the size."""
        n = w.w_gate.numel() + w.w_up.numel() + w.w_down.numel()
        self.muon_m = torch.zeros(n, device=self.device, dtype=torch.float32)
        self.muon_master = self._master(w) if master else None
        which = P.MOE_WS_UPDATE_MUON_PRECISE if precise else P.MOE_WS_UPDATE_MUON
        self.ws_muon = torch.empty(P.moe_workspace_size(self.desc, which), dtype=torch.uint8, device=self.device)

    def update_muon(self, w: LayerWeights, opt: "P.moe_muon"):
        """One step of the hosted experts along their orthogonalised momentum, from the gradients of the last backward."""
        P.moe_expert_update_muon(self.desc, opt, w.w_gate, w.w_up, w.w_down, self.dw_gate, self.dw_up, self.dw_down,
                                 self.muon_master, self.muon_m, self.ws_muon, self.ws_muon.numel())

    def n_local_rows(self) -> int:
        return int(self.offsets[-1].item())


@dataclass
class NormWeights:
    """Weights of what stands between two blocks; None: all ones (the gate: none)."""
    w_post: Optional[torch.Tensor] = None   # [d]
    gate: Optional[torch.Tensor] = None     # [gate_groups, d]
    w_pre: Optional[torch.Tensor] = None    # [d]


class ResidualNorm:
    """Between two blocks: r = alpha x + gate * post(y), h = pre(r), and the adjoint. norm: a pcmoe.make_norm(...). first: before
    the first block, where there is no y. ws: a workspace of the adjoint to share, MOE_WS_NORM_BWD bytes at least."""

    def __init__(self, T, d, norm, dtype="bf16", device="cuda", first=False, backward=True, ws=None):
        self.desc = P.make_desc(T, d, 128, 1, 1, dtype=dtype)
        self.norm, self.first, self.shape, self.dt = norm, first, (T, d), torch_dtype(dtype)
        new = lambda: torch.empty(T, d, dtype=self.dt, device=device)
        self.r = None if first else new()
        self.h = new() if norm.pre != P.MOE_NORM_NONE else None
        self.device, self.backward_enabled = device, backward
        if backward:
            self.dx = new()
            self.dy = None if first else new()
            need = P.moe_workspace_size(self.desc, P.MOE_WS_NORM_BWD)
            self.ws = torch.empty(need, dtype=torch.uint8, device=device) if ws is None else ws
        self.dw_post = self.dgate = self.dw_pre = None   # fp32, allocated by the first backward
        self.y = self.r_of_backward = None   # of the last forward

    def _check(self, what, t, shape, dtype=None):
        if t is not None and (tuple(t.shape) != shape or t.dtype != (dtype or self.dt)):
            raise ValueError(f"{what}: {tuple(t.shape)} {t.dtype}, expected {shape} {dtype or self.dt}")

    def _check_weights(self, w: NormWeights):
        d = self.shape[1]
        self._check("w_post", w.w_post, (d,))
        self._check("w_pre", w.w_pre, (d,))
        self._check("gate", w.gate, (self.norm.gate_groups, d))

    def forward(self, w: NormWeights, x, y=None):
        """r and h (r is x before the first block; h is None without a pre norm). x and y are read again by the backward."""
        self._check_weights(w)
        self._check("x", x, self.shape)
        self._check("y", y, self.shape)
        P.moe_residual_norm(self.desc, self.norm, x, y, w.w_post, w.gate, w.w_pre, self.r, self.h)
        self.y, self.r_of_backward = y, x if self.first else self.r
        return self.r_of_backward, self.h

    def backward(self, w: NormWeights, dr, dh):
        """dx and dy of the last forward; the weights' gradients are left in dw_post, dgate and dw_pre."""
        self._check_weights(w)
        self._check("dr", dr, self.shape)
        self._check("dh", dh, self.shape)
        if not self.backward_enabled:
            raise RuntimeError("a norm built with backward=False has no backward")
        if self.r_of_backward is None:
            raise RuntimeError("a backward needs a forward before it")
        for name, t in (("dw_post", w.w_post), ("dgate", w.gate), ("dw_pre", w.w_pre)):
            if t is None:
                setattr(self, name, None)
            elif getattr(self, name) is None:
                setattr(self, name, torch.empty(t.shape, dtype=torch.float32, device=self.device))
        P.moe_residual_norm_bwd(self.desc, self.norm, dr, dh, self.y, self.r_of_backward, w.w_post, w.gate, w.w_pre, self.dx,
                                self.dy, self.dw_post, self.dgate, self.dw_pre, self.ws, self.ws.numel())
        return self.dx, self.dy


class MoEStack:
    """Layers one after the other with norms, gates and the residual stream around them:
        r_0 = x, h_0 = pre(r_0);  y_i = layer_i(h_i);  r_i+1 = alpha r_i + gate_i+1 * post(y_i), h_i+1 = pre(r_i+1)
    with `final` in place of pre at the end. The result is the last h, or the last r where final is "none". layers: MoELayers of
    one T, d and dtype that host all experts. forward takes the layers' weights (whose x it sets) and len(layers) + 1
    NormWeights. The stack's calls read the layers' inputs from its own buffers, never from the weights' x: other stacks may run
    with the same weights between a forward and its backward, and layers of one stack may share theirs. A backward belongs to
    the last forward of each of its layers."""

    def __init__(self, layers, pre="rms", post="none", final="rms", eps=1e-6, residual_scale=1.0, gate_groups=1):
        if not layers:
            raise ValueError("a stack needs a layer")
        if len({id(l) for l in layers}) < len(layers):
            raise ValueError("a layer holds the activations of one place of a stack: the same layer twice")
        cfg = layers[0].cfg
        for l in layers:
            if (l.cfg.T, l.cfg.d, l.cfg.dtype) != (cfg.T, cfg.d, cfg.dtype):
                raise ValueError("the layers of a stack share T, d and dtype")
            if l.cfg.n_local != l.cfg.E:
                raise ValueError(f"a stack's layers host all experts, got {l.cfg.n_local} of {l.cfg.E}: one party's output is a "
                                 "part of a sum; add the parties' up and join the layers with ResidualNorm")
        if pre == "none":
            raise ValueError("a stack norms the input of its layers: pre is 'rms' or 'layer'")
        self.layers = list(layers)
        self.backward_enabled = all(l.backward_enabled for l in layers)
        self.ran = None   # the layers' runs after the last forward
        self.norms, ws = [], None
        for i in range(len(layers) + 1):
            norm = P.make_norm(final if i == len(layers) else pre, post if i else "none", eps, residual_scale if i else 1.0,
                               gate_groups)
            self.norms.append(ResidualNorm(cfg.T, cfg.d, norm, cfg.dtype, layers[0].device, first=i == 0,
                                           backward=self.backward_enabled, ws=ws))
            ws = getattr(self.norms[-1], "ws", None)

    def _check_counts(self, ws, ns, experts=None):
        n = len(self.layers)
        if len(ws) != n or len(ns) != n + 1 or (experts is not None and len(experts) != n):
            raise ValueError(f"{n} layers take {n} weights, {n + 1} norms and, if any, {n} experts: got {len(ws)}, {len(ns)}"
                             + (f" and {len(experts)}" if experts is not None else ""))

    def _of(self, i, w):
        """Weights w with the input of layer i."""
        w = copy(w)
        w.x = self.norms[i].h
        return w

    def forward(self, x, ws, ns, experts=None):
        """experts: a Q4Experts or Q8Experts for each layer, to run the experts from (no backward can follow)."""
        self._check_counts(ws, ns, experts)
        r, h = self.norms[0].forward(ns[0], x)
        for i, (layer, w) in enumerate(zip(self.layers, ws)):
            w.x = h
            w = self._of(i, w)
            if experts is None:
                y = layer.forward(w)
            else:
                y = (layer.forward_q8 if isinstance(experts[i], Q8Experts) else layer.forward_q4)(w, experts[i])
            r, h = self.norms[i + 1].forward(ns[i + 1], r, y)
        self.ran = [l.runs for l in self.layers]
        return r if h is None else h

    def backward(self, d, ws, ns):
        """The gradient of x from that of forward's result (without what passes through the routing of layers built with
        router_backward=False). Layers leave the gradients of their weights in their buffers, the norms in theirs."""
        self._check_counts(ws, ns)
        if not self.backward_enabled:
            raise RuntimeError("a stack with a layer built with backward=False has no backward")
        if self.ran is None:
            raise RuntimeError("a backward needs a forward before it")
        for layer in self.layers:
            layer._need_saved()
        if [l.runs for l in self.layers] != self.ran:
            raise RuntimeError("a layer ran another forward since this stack's: its activations are of that one")
        dr, dh = (d, None) if self.norms[-1].h is None else (None, d)
        for i in reversed(range(len(self.layers))):
            dr, dy = self.norms[i + 1].backward(ns[i + 1], dr, dh)
            dh = self.layers[i].backward(self._of(i, ws[i]), dy)
        return self.norms[0].backward(ns[0], dr, dh)[0]


def training_footprint(cfg, local_count: int, master: bool = True, checkpoint: bool = False,
                       shared_saved: bool = False, update: str = "adamw") -> dict:
    """Device bytes one party allocates for the expert layer's training step (route, permute, expert FFN forward
    and backward, combine and its adjoint, router adjoint, expert update) when it hosts `local_count` of the
    cfg.E routed experts, by category:
      expert_state  hosted experts' weights and weight gradients (dtype) plus fp32 moments and master copy;
      activations   row-space buffers (capacity T*k + S*T rows), saved activations and the FFN workspaces;
      owner         the owner-side buffers of its own T tokens (input, router, combine, input gradient).
    checkpoint: with the 8-bit checkpoint of a MoELayer(checkpoint=True). shared_saved: without the saved activations, for
    a layer that is given a buffer which all the layers of a stack share, and whose size is returned as `shared_saved`.
    update: "adamw", or "muon" or "muon_precise" for update_muon, with one moment and a workspace, returned as `update_ws`.
    The sizes are those MoELayer, init_update_state and init_muon_state allocate, with workspace sizes from the library."""
    muon_ws = {"muon": P.MOE_WS_UPDATE_MUON, "muon_precise": P.MOE_WS_UPDATE_MUON_PRECISE}
    if update != "adamw" and update not in muon_ws:
        raise ValueError(f"update {update!r} is not 'adamw', 'muon' or 'muon_precise'")
    if shared_saved and not checkpoint:
        raise ValueError("a shared saved buffer needs checkpoint=True")
    T, d, f, E, k, S = cfg.T, cfg.d, cfg.f, cfg.E, cfg.k, cfg.n_shared
    es = 2 if cfg.dtype == "bf16" else 4
    desc = P.make_desc(T, d, f, E, k, 0, local_count, S, cfg.renormalize, cfg.dtype)
    ws = lambda which: max(P.moe_workspace_size(desc, which), 1)
    G, R = local_count + S, T * k + S * T
    params = G * 3 * f * d
    moments = 2 if update == "adamw" else 1
    expert_state = params * es * 2 + params * 4 * (moments + (1 if master else 0))
    update_ws = P.moe_workspace_size(desc, muon_ws[update]) if update in muon_ws else 0
    activations = (T * k * d * es            # x_perm
                   + R * d * es              # y_perm
                   + T * k * d * es          # dy_perm
                   + R * d * es              # dx_perm
                   + (0 if shared_saved else ws(P.MOE_WS_FFN_SAVED)) + (ws(P.MOE_WS_FFN_CKPT) if checkpoint else 0)
                   + ws(P.MOE_WS_FFN_FWD) + ws(P.MOE_WS_FFN_BWD) + ws(P.MOE_WS_PERMUTE)
                   + (local_count + 1) * 4 + max(local_count, 1) * 4 + 2 * T * k * 4)   # offsets, counts, maps
    owner = (T * d * es * 3                  # x, y, dx
             + T * d * es                    # dy
             + E * d * es + E * d * 4        # router weights and their gradient
             + T * E * 4 * 2                 # logits, dlogits
             + T * k * (4 + 4 + 4)           # topk_idx, topk_w, dgate
             + ws(P.MOE_WS_ROUTE_BWD))
    out = {"local_experts": local_count, "expert_state": expert_state, "activations": activations, "owner": owner,
           "total": expert_state + activations + owner + update_ws}
    if update in muon_ws:
        out["update_ws"] = update_ws
    if shared_saved:
        out["shared_saved"] = ws(P.MOE_WS_FFN_SAVED)
    return out
