"""Device-side plumbing around the C ABI: PyTorch holds the device memory and
the stream; these classes only fill the C structs with its addresses and
call the library.  No arithmetic of the method happens here.
"""
from __future__ import annotations

import ctypes as C
import functools
import struct
from typing import Dict, List, Optional, Sequence

import numpy as np
import torch

from . import jnx as J


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream: Optional[torch.cuda.Stream]) -> int:
    s = stream if stream is not None else torch.cuda.current_stream()
    return s.cuda_stream


class DeviceGroup:
    """A plan's arrays copied to the device, wrapped in a jnx_group."""

    DEV = ("cu_seqlens", "sample_slot", "sample_target", "seg_offsets", "gather_src", "pos_ids")

    def __init__(self, plan: J.Plan, device="cuda", non_blocking: bool = False):
        self.plan = plan
        self.h = {k: np.ascontiguousarray(getattr(plan, k), dtype=np.int32)
                  for k in ("cu_seqlens", "seg_offsets", "slot_tenant")}
        self.d = {}
        for k in self.DEV:
            a = torch.from_numpy(np.ascontiguousarray(getattr(plan, k), dtype=np.int32))
            if non_blocking:
                a = a.pin_memory()
            self.d[k] = a.to(device, non_blocking=non_blocking)
        hp = lambda k: self.h[k].ctypes.data_as(J.P32)
        self.struct = J.jnx_group(
            plan.n_samples, plan.n_tokens, plan.n_slots, plan.max_seqlen,
            *[self.d[k].data_ptr() or None for k in self.DEV],
            hp("cu_seqlens"), hp("seg_offsets"), hp("slot_tenant"), None, 0)
        # the attention work list on the device too, so the backbone's calls
        # read it instead of uploading it (and can be captured into a graph)
        L = J.lib()
        n = L.jnx_group_attn_items(C.byref(self.struct), None, 0)
        if n < 0:
            J.check(n)
        items = np.zeros(2 * max(n, 1), dtype=np.int32)
        got = L.jnx_group_attn_items(C.byref(self.struct), items.ctypes.data, n)
        if got != n:
            J.check(got if got < 0 else J.JNX_ERR_INVALID_ARG)
        t = torch.from_numpy(items)
        if non_blocking:
            t = t.pin_memory()
        self.d["attn_items"] = t.to(device, non_blocking=non_blocking)
        self.struct.attn_items = self.d["attn_items"].data_ptr() if n else None
        self.struct.n_attn_items = n

    @property
    def ref(self):
        return C.byref(self.struct)


class DeviceBackbone:
    """Frozen backbone weights on the device in the library's layout: the
    fused [W_q; W_k; W_v] rows and the 128-row interleaved gate/up matrix
    (built by jnx_pack_gate_up)."""

    def __init__(self, cfg, weights: Dict, n_tenants: int = 1, stream=None):
        self.cfg = cfg
        L = J.lib()
        self.keep: List[torch.Tensor] = []
        self.layers = (J.jnx_layer * max(1, cfg.n_layers))()
        s = _stream(stream)
        for i, lw in enumerate(weights["layers"]):
            w_qkv = torch.cat([lw["wq"], lw["wk"], lw["wv"]], dim=0).contiguous()
            w_gu = torch.empty((2 * cfg.d_ff, cfg.d), dtype=torch.bfloat16, device=w_qkv.device)
            J.check(L.jnx_pack_gate_up(lw["wg"].data_ptr(), lw["wu"].data_ptr(), cfg.d_ff, cfg.d,
                                       w_gu.data_ptr(), s))
            ent = dict(attn_norm=lw["attn_norm"], w_qkv=w_qkv, w_o=lw["wo"],
                       ffn_norm=lw["ffn_norm"], w_gu=w_gu, w_down=lw["wd"])
            names = ["attn_norm", "w_qkv", "w_o", "ffn_norm", "w_gu", "w_down"]
            if cfg.lora_rank:
                for p in ("q", "k", "v", "o"):
                    ent["lora_a_" + p] = lw["lora_a_" + p].contiguous()
                    ent["lora_b_" + p] = lw["lora_b_" + p].contiguous()
                    names += ["lora_a_" + p, "lora_b_" + p]
            self.keep += list(ent.values())
            self.layers[i] = J.jnx_layer(**{k: ent[k].data_ptr() for k in names})
        self.text_table = weights["text_table"]
        self.final_norm = weights["final_norm"]
        self.struct = J.jnx_backbone(cfg.n_layers, cfg.d, cfg.n_heads, cfg.n_kv_heads,
                                     cfg.head_dim, cfg.d_ff, cfg.glu, cfg.lora_rank, n_tenants,
                                     cfg.vocab, cfg.vision_tokens, cfg.eps, cfg.rope_theta,
                                     self.text_table.data_ptr(), self.final_norm.data_ptr(),
                                     C.cast(self.layers, C.POINTER(J.jnx_layer)))

    def workspace_bytes(self, n_tokens: int) -> int:
        return J.lib().jnx_backbone_workspace_bytes(C.byref(self.struct), n_tokens)

    def forward(self, group: DeviceGroup, vision: torch.Tensor, text_ids: torch.Tensor,
                pooled: Optional[torch.Tensor], hidden: Optional[torch.Tensor],
                ws: torch.Tensor, stream=None) -> None:
        J.check(J.lib().jnx_backbone_forward(
            C.byref(self.struct), group.ref, vision.data_ptr(), vision.shape[0],
            text_ids.data_ptr(), text_ids.shape[0], _ptr(pooled), _ptr(hidden),
            ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)))

    # ---- trainable adapters ------------------------------------------------
    def saved_bytes(self, n_tokens: int) -> int:
        return J.lib().jnx_backbone_saved_bytes(C.byref(self.struct), n_tokens)

    def backward_workspace_bytes(self, n_tokens: int) -> int:
        return J.lib().jnx_backbone_backward_workspace_bytes(C.byref(self.struct), n_tokens)

    def prepare_backward(self, stream=None) -> None:
        """Transposed copies of the frozen weights (built once on the device)
        and zeroed fp32 adapter-gradient buffers, one set per layer."""
        cfg, L, s = self.cfg, J.lib(), _stream(stream)
        n = max(1, cfg.n_layers)
        self.layers_t = (J.jnx_layer_t * n)()
        self.lgarr = (J.jnx_lora_grads * n)()
        self.keep_t: List[torch.Tensor] = []
        self.lora_grads: List[Dict[str, torch.Tensor]] = []
        per = len(self.keep) // max(1, cfg.n_layers)
        for i in range(cfg.n_layers):
            ent = self.keep[i * per:(i + 1) * per]
            w_qkv, w_o, w_gu, w_down = ent[1], ent[2], ent[4], ent[5]
            outs = []
            for w in (w_qkv, w_o, w_gu, w_down):
                t = torch.empty((w.shape[1], w.shape[0]), dtype=torch.bfloat16, device=w.device)
                J.check(L.jnx_transpose(w.data_ptr(), 1, w.shape[0], w.shape[1], t.data_ptr(), s))
                outs.append(t)
            self.keep_t += outs
            self.layers_t[i] = J.jnx_layer_t(*[t.data_ptr() for t in outs])
            lw = dict(zip(["attn_norm", "w_qkv", "w_o", "ffn_norm", "w_gu", "w_down",
                           "lora_a_q", "lora_b_q", "lora_a_k", "lora_b_k", "lora_a_v",
                           "lora_b_v", "lora_a_o", "lora_b_o"], ent))
            g = {}
            for name in J.LORA_GRADS:
                src = lw.get("lora_" + name)
                g[name] = (torch.zeros(src.shape, dtype=torch.float32, device=src.device)
                           if src is not None else None)
            self.lora_grads.append(g)
            self.lgarr[i] = J.jnx_lora_grads(*[_ptr(g[k]) for k in J.LORA_GRADS])

    def lora_pairs(self):
        """(adapter [n_tenants, ...] bf16, its gradient buffer) of every layer,
        for TenantAdamW (the adapters are updated in place)."""
        per = len(self.keep) // max(1, self.cfg.n_layers)
        out = []
        for i in range(self.cfg.n_layers):
            ent = self.keep[i * per:(i + 1) * per][6:]
            for name, p in zip(J.LORA_GRADS, ent):
                out.append((p, self.lora_grads[i][name]))
        return out

    def forward_train(self, group: DeviceGroup, vision, text_ids, pooled, hidden, saved, ws,
                      stream=None) -> None:
        J.check(J.lib().jnx_backbone_forward_train(
            C.byref(self.struct), group.ref, vision.data_ptr(), vision.shape[0],
            text_ids.data_ptr(), text_ids.shape[0], _ptr(pooled), _ptr(hidden),
            saved.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)))

    def backward_lora(self, group: DeviceGroup, saved, d_hidden, ws, accumulate: bool = False,
                      stream=None) -> None:
        """Every group tenant's adapter gradients into self.lora_grads (its
        slice only), from dloss/d(final normed rows)."""
        J.check(J.lib().jnx_backbone_backward_lora(
            C.byref(self.struct), self.layers_t, group.ref, saved.data_ptr(), d_hidden.data_ptr(),
            self.lgarr, 1 if accumulate else 0, ws.data_ptr(), ws.numel() * ws.element_size(),
            _stream(stream)))


class DeviceHeads:
    """One head slot per tenant (bf16 parameters) and fp32 gradient slots."""

    def __init__(self, tenants: Sequence, d: int, heads: List[Dict], device="cuda"):
        n = len(tenants)
        self.n = n
        self.arr = (J.jnx_head * max(1, n))()
        self.garr = (J.jnx_head_grads * max(1, n))()
        self.grads: List[Dict[str, torch.Tensor]] = []
        self.keep = []
        for t, (tn, hw) in enumerate(zip(tenants, heads)):
            if tn.head_kind == J.JNX_HEAD_MLP:
                self.arr[t] = J.jnx_head(tn.head_kind, d, tn.d_hidden, 0, 0, tn.width,
                                         hw["w1"].data_ptr(), hw["b1"].data_ptr(),
                                         hw["w2"].data_ptr(), hw["b2"].data_ptr(),
                                         None, None, None, None, None)
                g = {k: torch.zeros(hw[k].shape, dtype=torch.float32, device=device)
                     for k in ("w1", "b1", "w2", "b2")}
                self.garr[t] = J.jnx_head_grads(*[g[k].data_ptr() for k in ("w1", "b1", "w2",
                                                                             "b2")],
                                                None, None, None, None, None)
            else:
                self.arr[t] = J.jnx_head(tn.head_kind, d, 0, tn.n_queries, tn.q_dim, tn.width,
                                         None, None, None, None, hw["q"].data_ptr(),
                                         hw["wk"].data_ptr(), hw["wv"].data_ptr(),
                                         hw["wout"].data_ptr(), hw["bout"].data_ptr())
                g = {k: torch.zeros(hw[k].shape, dtype=torch.float32, device=device)
                     for k in ("q", "wk", "wv", "wout", "bout")}
                self.garr[t] = J.jnx_head_grads(None, None, None, None,
                                                *[g[k].data_ptr() for k in ("q", "wk", "wv",
                                                                            "wout", "bout")])
            self.grads.append(g)
            self.keep.append(hw)

    def workspace_bytes(self, group: DeviceGroup) -> int:
        return J.lib().jnx_heads_workspace_bytes(self.arr, self.n, group.ref)

    def forward(self, group: DeviceGroup, pooled, hidden, targets, preds, loss, ws,
                stream=None) -> None:
        """targets and loss may both be None (inference: predictions only)."""
        J.check(J.lib().jnx_heads_forward(
            self.arr, self.n, group.ref, _ptr(pooled), _ptr(hidden), _ptr(targets),
            preds.data_ptr(), _ptr(loss), ws.data_ptr(), ws.numel() * ws.element_size(),
            _stream(stream)))

    def backward(self, group: DeviceGroup, pooled, hidden, targets, ws, stream=None,
                 accumulate: bool = False) -> None:
        """Gradients into each group tenant's slot: overwritten, or added to
        what is there (gradient accumulation) with accumulate=True."""
        fn = J.lib().jnx_heads_backward_accumulate if accumulate else J.lib().jnx_heads_backward
        J.check(fn(self.arr, self.n, group.ref, _ptr(pooled), _ptr(hidden), targets.data_ptr(),
                   self.garr, ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)))

    def backward_input(self, group: DeviceGroup, pooled, hidden, targets, d_hidden, ws,
                       stream=None) -> None:
        """backward, and also dloss/d(final normed row) of every token row."""
        J.check(J.lib().jnx_heads_backward_input(
            self.arr, self.n, group.ref, _ptr(pooled), _ptr(hidden), targets.data_ptr(),
            self.garr, d_hidden.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(),
            _stream(stream)))

    def init_optimizer(self) -> None:
        """Tenant-private AdamW state: an fp32 master copy of every head
        parameter (from its bf16 value) and zero moments, per tenant."""
        self.opt = (J.jnx_head_opt * max(1, self.n))()
        self.opt_state: List[Dict[str, Dict[str, torch.Tensor]]] = []
        for t, hw in enumerate(self.keep):
            st = {}
            for k, name in enumerate(J.HEAD_PARAMS):
                if name not in hw:
                    continue
                p = hw[name]
                st[name] = dict(master=p.float().clone(), m=torch.zeros_like(p, dtype=torch.float32),
                                v=torch.zeros_like(p, dtype=torch.float32))
                self.opt[t].master[k] = st[name]["master"].data_ptr()
                self.opt[t].m[k] = st[name]["m"].data_ptr()
                self.opt[t].v[k] = st[name]["v"].data_ptr()
            self.opt_state.append(st)

    def adamw_step(self, group: DeviceGroup, lr: float, beta1: float = 0.9,
                   beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0,
                   stream=None) -> None:
        """One AdamW step on every group tenant's head from its gradients
        (bf16 parameters updated in place; the tenant's step and policy
        version counters increment)."""
        hp = J.jnx_adamw(lr, beta1, beta2, eps, weight_decay)
        J.check(J.lib().jnx_heads_adamw(self.arr, self.garr, self.opt, self.n, group.ref,
                                        C.byref(hp), _stream(stream)))

    def backward_adamw(self, group: DeviceGroup, pooled, hidden, targets, ws, lr: float,
                       beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                       weight_decay: float = 0.0, accumulate: bool = False, d_hidden=None,
                       stream=None) -> None:
        """The heads backward with every group tenant's AdamW step fused into
        it: the same result as backward() then adamw_step(), without storing
        the gradients (with accumulate=True the gradients already in the
        slots are added first).  d_hidden, if given, receives the gradient at
        the final normed rows (as backward_input)."""
        hp = J.jnx_adamw(lr, beta1, beta2, eps, weight_decay)
        J.check(J.lib().jnx_heads_backward_adamw(
            self.arr, self.n, group.ref, _ptr(pooled), _ptr(hidden), _ptr(targets), self.garr,
            1 if accumulate else 0, self.opt, C.byref(hp), _ptr(d_hidden), ws.data_ptr(),
            ws.numel() * ws.element_size(), _stream(stream)))

    def version(self, t: int) -> int:
        return int(self.opt[t].version)


class DeviceFlowHeads:
    """Flow-matching action experts (DiT heads) of n_tenants tenants with the
    same dimensions: stacked bf16 parameters (the gate/up pair of each block
    packed by jnx_pack_gate_up) and fp32 gradient buffers of the same shapes."""

    def __init__(self, dims: Dict, weights: Dict, stream=None):
        L, s = J.lib(), _stream(stream)
        self.dims = dims
        T, dm, F = dims["n_tenants"], dims["d_model"], dims["d_ff"]
        self.keep = {k: weights[k].contiguous() for k in J.FLOW_PARAMS}
        self.blocks = []
        for B in weights["blocks"]:
            w_gu = torch.empty((T, 2 * F, dm), dtype=torch.bfloat16, device=B["wg"].device)
            for t in range(T):
                J.check(L.jnx_pack_gate_up(B["wg"][t].contiguous().data_ptr(),
                                           B["wu"][t].contiguous().data_ptr(), F, dm,
                                           w_gu[t].data_ptr(), s))
            self.blocks.append(dict(w_qkv=B["w_qkv"].contiguous(), w_kvc=B["w_kvc"].contiguous(),
                                    w_o=B["w_o"].contiguous(), w_gu=w_gu,
                                    w_d=B["w_d"].contiguous()))
        nb = max(1, len(self.blocks))
        self.barr = (J.jnx_flow_block * nb)(*[J.jnx_flow_block(
            *[b[k].data_ptr() for k in J.FLOW_BLOCK_PARAMS]) for b in self.blocks])
        self.struct = J.jnx_flow_head(
            dm, F, len(self.blocks), dims["chunk"], dims["action_dim"], dims["d_in"], T,
            *[self.keep[k].data_ptr() for k in J.FLOW_PARAMS],
            C.cast(self.barr, C.POINTER(J.jnx_flow_block)))
        dev = self.keep["w_in"].device
        self.grads = {k: torch.zeros(self.keep[k].shape, dtype=torch.float32, device=dev)
                      for k in J.FLOW_PARAMS}
        self.block_grads = [{k: torch.zeros(b[k].shape, dtype=torch.float32, device=dev)
                             for k in J.FLOW_BLOCK_PARAMS} for b in self.blocks]
        self.bgarr = (J.jnx_flow_block_grads * nb)(*[J.jnx_flow_block_grads(
            *[g[k].data_ptr() for k in J.FLOW_BLOCK_PARAMS]) for g in self.block_grads])
        self.gstruct = J.jnx_flow_grads(*[self.grads[k].data_ptr() for k in J.FLOW_PARAMS],
                                        C.cast(self.bgarr, C.POINTER(J.jnx_flow_block_grads)))

    def workspace_bytes(self, group: DeviceGroup) -> int:
        return J.lib().jnx_flow_workspace_bytes(C.byref(self.struct), group.ref)

    def param_pairs(self):
        """(stacked parameter, its gradient buffer) of every expert tensor
        (the packed gate/up pair as one), for TenantAdamW."""
        out = [(self.keep[k], self.grads[k]) for k in J.FLOW_PARAMS]
        for b, g in zip(self.blocks, self.block_grads):
            out += [(b[k], g[k]) for k in J.FLOW_BLOCK_PARAMS]
        return out

    def forward(self, group: DeviceGroup, hidden, actions, noise, tau, velocity, loss, ws,
                stream=None) -> None:
        J.check(J.lib().jnx_flow_forward(
            C.byref(self.struct), group.ref, hidden.data_ptr(), actions.data_ptr(),
            noise.data_ptr(), tau.data_ptr(), velocity.data_ptr(), loss.data_ptr(),
            ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)))

    def backward(self, group: DeviceGroup, hidden, ws, accumulate: bool = False,
                 stream=None) -> None:
        J.check(J.lib().jnx_flow_backward(
            C.byref(self.struct), group.ref, hidden.data_ptr(), C.byref(self.gstruct),
            1 if accumulate else 0, ws.data_ptr(), ws.numel() * ws.element_size(),
            _stream(stream)))

    def sample(self, group: DeviceGroup, hidden, noise, n_steps: int, actions, ws,
               stream=None) -> None:
        J.check(J.lib().jnx_flow_sample(
            C.byref(self.struct), group.ref, hidden.data_ptr(), noise.data_ptr(), n_steps,
            actions.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)))


class TenantAdamW:
    """Tenant-private AdamW over stacked per-tenant parameters: for every
    (parameter [n_tenants, ...] bf16, gradient [n_tenants, ...] fp32) pair an
    fp32 master copy and zero moments; step(tenants) updates only those
    tenants' slices, each slice with its own step counter
    (jnx_adamw_tensors)."""

    def __init__(self, pairs):
        self.pairs = [(p, g) for p, g in pairs]
        self.master = [p.float().clone() for p, _ in self.pairs]
        self.m = [torch.zeros_like(x) for x in self.master]
        self.v = [torch.zeros_like(x) for x in self.master]
        self.counts: Dict = {}

    def steps(self, i: int, t: int) -> int:
        c = self.counts.get((i, t))
        return int(c.value) if c is not None else 0

    def step(self, tenants, lr: float, beta1: float = 0.9, beta2: float = 0.999,
             eps: float = 1e-8, weight_decay: float = 0.0, stream=None) -> None:
        arr = []
        for i, (p, g) in enumerate(self.pairs):
            for t in tenants:
                cnt = self.counts.setdefault((i, t), C.c_int32(0))
                arr.append(J.jnx_adam_tensor(p[t].data_ptr(), self.master[i][t].data_ptr(),
                                             self.m[i][t].data_ptr(), self.v[i][t].data_ptr(),
                                             g[t].data_ptr(), p[t].numel(), C.pointer(cnt)))
        tab = (J.jnx_adam_tensor * max(1, len(arr)))(*arr)
        hp = J.jnx_adamw(lr, beta1, beta2, eps, weight_decay)
        J.check(J.lib().jnx_adamw_tensors(tab, len(arr), C.byref(hp), _stream(stream)))


def check_status(ws: torch.Tensor, stream=None) -> None:
    J.check(J.lib().jnx_check_status(ws.data_ptr(), _stream(stream)))


class GroupedStep:
    """One grouped step through the C ABI: backbone forward over the packed
    batch, then every group tenant's head forward, loss and backward."""

    def __init__(self, backbone: DeviceBackbone, heads: DeviceHeads, group: DeviceGroup,
                 device="cuda"):
        self.bb, self.heads, self.group = backbone, heads, group
        cfg = backbone.cfg
        S, N = group.plan.n_samples, group.plan.n_tokens
        kinds = {heads.arr[t].kind for t in group.plan.slot_tenant.tolist()}
        self.need_hidden = J.JNX_HEAD_XATTN in kinds
        self.need_pooled = J.JNX_HEAD_MLP in kinds or not kinds
        self.pooled = torch.zeros((max(S, 1), cfg.d), dtype=torch.float32, device=device)
        self.hidden = (torch.zeros((max(N, 1), cfg.d), dtype=torch.bfloat16, device=device)
                       if self.need_hidden else None)
        self.ws_bb = torch.zeros(max(backbone.workspace_bytes(N), 256), dtype=torch.uint8,
                                 device=device)
        self.ws_h = torch.zeros(max(heads.workspace_bytes(group), 256), dtype=torch.uint8,
                                device=device)
        self.loss = torch.full((max(heads.n, 1),), float("nan"), dtype=torch.float32, device=device)

    def run(self, vision, text_ids, targets, preds, stream=None) -> None:
        self.bb.forward(self.group, vision, text_ids,
                        self.pooled if self.need_pooled else None, self.hidden, self.ws_bb, stream)
        self.heads.forward(self.group, self.pooled, self.hidden, targets, preds, self.loss,
                           self.ws_h, stream)
        self.heads.backward(self.group, self.pooled, self.hidden, targets, self.ws_h, stream)

    def infer(self, vision, text_ids, preds, stream=None) -> None:
        """Inference: the shared backbone forward and every group tenant's
        head forward (predictions only; no targets, loss or backward)."""
        self.bb.forward(self.group, vision, text_ids,
                        self.pooled if self.need_pooled else None, self.hidden, self.ws_bb, stream)
        self.heads.forward(self.group, self.pooled, self.hidden, None, preds, None, self.ws_h,
                           stream)


class LoraTrainStep(GroupedStep):
    """One grouped training step of the tenants' adapters and heads through
    the C ABI: the shared forward keeping each block's residual input, every
    group tenant's head forward, loss and backward (with the gradient at its
    features), then the adapter backward through the frozen backbone.  Head
    gradients land in heads.grads, adapter gradients in backbone.lora_grads,
    each tenant's in its own slice."""

    def __init__(self, backbone: DeviceBackbone, heads: DeviceHeads, group: DeviceGroup,
                 device="cuda"):
        super().__init__(backbone, heads, group, device)
        if not hasattr(backbone, "layers_t"):
            backbone.prepare_backward()
        N, d = group.plan.n_tokens, backbone.cfg.d
        self.saved = torch.empty(max(backbone.saved_bytes(N) // 4, 1), dtype=torch.float32,
                                 device=device)
        self.d_hidden = torch.zeros((max(N, 1), d), dtype=torch.float32, device=device)
        self.ws_bwd = torch.zeros(max(backbone.backward_workspace_bytes(N), 256),
                                  dtype=torch.uint8, device=device)

    def run(self, vision, text_ids, targets, preds, stream=None, accumulate: bool = False) -> None:
        self.bb.forward_train(self.group, vision, text_ids,
                              self.pooled if self.need_pooled else None, self.hidden, self.saved,
                              self.ws_bb, stream)
        self.heads.forward(self.group, self.pooled, self.hidden, targets, preds, self.loss,
                           self.ws_h, stream)
        self.heads.backward_input(self.group, self.pooled, self.hidden, targets, self.d_hidden,
                                  self.ws_h, stream)
        self.bb.backward_lora(self.group, self.saved, self.d_hidden, self.ws_bwd,
                              accumulate=accumulate, stream=stream)


class StepPipeline:
    """Grouped steps fed from pinned host memory, each step's preparation
    overlapped with the step before it.

    While step i runs on the compute stream, the host plans step i+1 and a
    copy stream moves its inputs into the second of two device input
    buffers; step i+1 waits only for that copy (and its group's plan arrays,
    which go up on the compute stream behind step i).  Every step's per-slot
    loss and predictions come back to pinned host memory on the compute
    stream and are handed to `on_result(i, loss, preds)` once step i is done
    (while step i+1 is already queued on the GPU).  All steps share the
    GroupedStep's buffers and workspaces, so each step's group must need no
    more than the group the GroupedStep was built for."""

    def __init__(self, step: GroupedStep, vision_rows: int, n_text: int, targets_shape,
                 device="cuda"):
        self.step = step
        self.dev = device
        d = step.bb.cfg.d
        self.vis = [torch.empty((max(vision_rows, 1), d), dtype=torch.bfloat16, device=device)
                    for _ in range(2)]
        self.tid = [torch.empty(max(n_text, 1), dtype=torch.int32, device=device)
                    for _ in range(2)]
        self.tgt = [torch.empty(targets_shape, dtype=torch.float32, device=device)
                    for _ in range(2)]
        self.preds = torch.zeros(targets_shape, dtype=torch.float32, device=device)
        self.copy_stream = torch.cuda.Stream(device=device)
        self.copied = [torch.cuda.Event() for _ in range(2)]
        self.done = [torch.cuda.Event() for _ in range(2)]
        self.loss_h = [torch.empty(step.loss.shape, dtype=torch.float32).pin_memory()
                       for _ in range(2)]
        self.preds_h = [torch.empty(targets_shape, dtype=torch.float32).pin_memory()
                        for _ in range(2)]
        self.groups: List[Optional[DeviceGroup]] = [None, None]
        self.h2d_bytes = 0
        self.max_tokens = step.group.plan.n_tokens
        self.max_samples = step.group.plan.n_samples

    def _fits(self, g: DeviceGroup) -> None:
        s = self.step
        if (g.plan.n_tokens > self.max_tokens or g.plan.n_samples > self.max_samples
                or s.ws_h.numel() < s.heads.workspace_bytes(g)
                or s.ws_bb.numel() < s.bb.workspace_bytes(g.plan.n_tokens)):
            raise ValueError("StepPipeline: a step's group is larger than the step's buffers")
        kinds = {s.heads.arr[t].kind for t in g.plan.slot_tenant.tolist()}
        if ((J.JNX_HEAD_XATTN in kinds and not s.need_hidden)
                or (J.JNX_HEAD_MLP in kinds and not s.need_pooled)):
            raise ValueError("StepPipeline: a step's group has a head kind the step was not built for")

    def _stage(self, i: int, host: Dict[str, torch.Tensor], plan) -> None:
        b = i & 1
        g = DeviceGroup(plan, device=self.dev, non_blocking=True)
        self._fits(g)
        cs = self.copy_stream
        cs.wait_event(self.done[b])  # step i-2 has finished reading buffer b
        with torch.cuda.stream(cs):
            for dst, k in ((self.vis[b], "vision"), (self.tid[b], "text_ids"),
                           (self.tgt[b], "targets")):
                src = host[k]
                dst.view(-1)[:src.numel()].copy_(src.view(-1), non_blocking=True)
                self.h2d_bytes += src.numel() * src.element_size()
        self.copied[b].record(cs)
        self.groups[b] = g

    def run(self, batches: Sequence[Dict[str, torch.Tensor]], plan_fn, on_result=None) -> None:
        """batches[i]: pinned host tensors 'vision', 'text_ids', 'targets' of
        step i; plan_fn(i) returns step i's plan (called on the host while
        step i-1 runs)."""
        ks = torch.cuda.current_stream(self.dev)
        n = len(batches)
        if n == 0:
            return
        self._stage(0, batches[0], plan_fn(0))
        for i in range(n):
            b = i & 1
            ks.wait_event(self.copied[b])
            self.step.group = self.groups[b]
            self.step.run(self.vis[b], self.tid[b], self.tgt[b], self.preds, ks)
            self.loss_h[b].copy_(self.step.loss, non_blocking=True)
            self.preds_h[b].copy_(self.preds, non_blocking=True)
            self.done[b].record(ks)
            if i >= 1:
                self.done[b ^ 1].synchronize()
                if on_result is not None:
                    on_result(i - 1, self.loss_h[b ^ 1], self.preds_h[b ^ 1])
            if i + 1 < n:
                self._stage(i + 1, batches[i + 1], plan_fn(i + 1))
        self.done[(n - 1) & 1].synchronize()
        if on_result is not None:
            on_result(n - 1, self.loss_h[(n - 1) & 1], self.preds_h[(n - 1) & 1])


# ---------------------------------------------------------------------------
# operators of text tenants
# ---------------------------------------------------------------------------

_BF16, _I32, _F32 = torch.bfloat16, torch.int32, torch.float32


def _refuse(t: torch.Tensor, dtype, shape) -> None:
    raise ValueError(f"expected a {dtype} CUDA tensor {shape}, its last axis contiguous, got "
                     f"{t.dtype} {tuple(t.shape)} strides {t.stride()} on {t.device}")


def _bf16(t: torch.Tensor, *shape) -> torch.Tensor:
    if t.dtype is not _BF16 or not t.is_cuda or t.shape != shape or \
            (t.stride(-1) != 1 and shape[-1] > 1):
        _refuse(t, _BF16, shape)
    return t


def _view(t: torch.Tensor, shape):
    """Head rows [n, heads, head_dim] of any row and head stride: what jnx_head_rows holds."""
    s = t.stride()
    if t.dtype is not _BF16 or t.shape != shape or s[2] != 1 or not t.is_cuda:
        _refuse(t, _BF16, shape)
    return t.data_ptr(), s[0], s[1]


def _dense(t: torch.Tensor, dtype, *shape) -> int:
    if t.dtype is not dtype or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        _refuse(t, dtype, shape)
    return t.data_ptr()


def _cache(k: torch.Tensor, v: torch.Tensor, heads):
    """A cache [slots, room, kv heads, head_dim], k and v of one layout: jnx_kv_cache's fields."""
    s, t, shape = k.stride(), v.stride(), k.shape
    # (an axis of length one, as a single key head's, has no stride to agree on)
    if k.dtype is not _BF16 or v.dtype is not _BF16 or v.shape != shape or \
            (s != t and any(a != b for a, b, n in zip(s, t, shape) if n > 1)) or \
            shape[2:] != heads or s[3] != 1 or not k.is_cuda or not v.is_cuda:
        raise ValueError(f"expected bf16 CUDA caches [slots, room, {heads[0]}, {heads[1]}] of one "
                         f"layout, got {k.dtype} {tuple(shape)} strides {s} and {v.dtype} "
                         f"{tuple(v.shape)} strides {v.stride()}")
    return k.data_ptr(), v.data_ptr(), shape[0], shape[1], s[0], s[1], s[2]


class _Views:
    """The structs that a call's tensors are described in, filled in one go: making one of
    each for every call took as long as the rest of a short call."""

    def __init__(self, *kinds):
        self._mem = C.create_string_buffer(sum(C.sizeof(k) for k in kinds))
        at, self.refs, form = C.addressof(self._mem), [], "="
        for k in kinds:
            self.refs.append(C.cast(at, C.POINTER(k)))
            at += C.sizeof(k)
            form += "Qqq" if k is J.jnx_head_rows else "QQiiqqq"
        self.fill = functools.partial(struct.Struct(form).pack_into, self._mem, 0)


class _TextOperator:
    """What the operators share: the status word their kernels report to and scratch
    memory, both the object's own (calls on several streams or threads at once take an
    object each)."""

    def __init__(self, ws_bytes: int = 0, device="cuda"):
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.ws = torch.empty(max(int(ws_bytes), 16), dtype=torch.uint8, device=device)
        self._status, self._ws, self._nws = (self.status.data_ptr(), self.ws.data_ptr(),
                                             self.ws.numel())
        self._lib, self._device = J.lib(), self.ws.device.index
        self._held = [self.status, self.ws]  # the object's device memory
        home = torch.cuda.current_stream(self._device)
        self._known, self._made = {home.cuda_stream}, None
        if not torch.cuda.is_current_stream_capturing():
            self._made = torch.cuda.Event()
            self._made.record(home)

    def _on(self, stream: Optional[torch.cuda.Stream]) -> int:
        handle = (stream.cuda_stream if stream is not None
                  else torch._C._cuda_getCurrentRawStream(self._device))
        if handle not in self._known:
            self._first_use(stream or torch.cuda.current_stream(self._device))
        return handle

    def _first_use(self, stream: torch.cuda.Stream) -> None:
        """A stream other than the one that the object was made on: its memory is ready there,
        and is not handed out again, once the object is gone, before the stream is through."""
        for t in self._held:
            t.record_stream(stream)
        with torch.cuda.stream(stream):
            if torch.cuda.is_current_stream_capturing():
                return  # (a capture cannot wait for what lies outside it)
        if self._made is not None:
            stream.wait_event(self._made)
        self._known.add(stream.cuda_stream)

    def check(self) -> None:
        """Raise what kernels reported since the last check, of calls on any stream (waits for
        the device: torch's streams do not order with one another)."""
        torch.cuda.synchronize(self._device)
        code = int(self.status.item())
        if code != J.JNX_OK:
            self.status.zero_()
            torch.cuda.synchronize(self._device)  # a later call's report is not wiped
            raise J.JnxError(code, "reported by a kernel")


class QKNormRope(_TextOperator):
    """Norms of each query and key head (gains gamma_q, gamma_k; None: no norm) and
    rotate-half RoPE over one or more position axes, `sections` frequencies to each."""

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int,
                 gamma_q: Optional[torch.Tensor] = None, gamma_k: Optional[torch.Tensor] = None,
                 sections: Optional[Sequence[int]] = None, theta: float = 10000.0,
                 eps: float = 1e-6, device="cuda"):
        self.sections = tuple(sections) if sections is not None else (head_dim // 2,)
        if len(self.sections) > 4:
            raise ValueError("at most four position axes")
        self.dims = (n_heads, n_kv_heads, head_dim)
        self.gains = tuple(None if g is None else _bf16(g, head_dim) for g in (gamma_q, gamma_k))
        self.struct = J.jnx_qk_rope(n_heads, n_kv_heads, head_dim, len(self.sections),
                                    (J.C.c_int32 * 4)(*self.sections), theta, eps,
                                    _ptr(gamma_q), _ptr(gamma_k))
        self._ref = C.byref(self.struct)
        # enough for any number of tokens: the gradient's CTAs are bounded
        super().__init__(J.lib().jnx_op_qk_norm_rope_backward_workspace_bytes(self._ref, 1 << 30),
                         device)

        rows, cache = J.jnx_head_rows, J.jnx_kv_cache
        self._qk, self._qc = _Views(rows, rows), _Views(rows, cache)

    def _args(self, qkv: torch.Tensor, pos: torch.Tensor):
        h, hkv, hd = self.dims
        n = qkv.shape[0]
        _bf16(qkv, n, (h + 2 * hkv) * hd)
        return n, qkv.data_ptr(), qkv.stride(0), _dense(pos, _I32, len(self.sections), n)

    def forward(self, qkv: torch.Tensor, pos: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                stream=None) -> None:
        """q [n, H, hd] and k [n, Hkv, hd] from qkv [n, (H + 2 Hkv) hd] at pos [axes, n]."""
        h, hkv, hd = self.dims
        n, x, ld, p = self._args(qkv, pos)
        self._qk.fill(*_view(q, (n, h, hd)), *_view(k, (n, hkv, hd)))
        J.check(self._lib.jnx_op_qk_norm_rope(self._ref, x, ld, p, n, *self._qk.refs,
                                              self._on(stream)))

    def append(self, qkv: torch.Tensor, pos: torch.Tensor, q: torch.Tensor,
               k_cache: torch.Tensor, v_cache: torch.Tensor, slot: torch.Tensor,
               at: torch.Tensor, stream=None) -> None:
        """q as forward; key and value rows go to cache rows [slot[i], at[i]]."""
        h, hkv, hd = self.dims
        n, x, ld, p = self._args(qkv, pos)
        self._qc.fill(*_view(q, (n, h, hd)), *_cache(k_cache, v_cache, (hkv, hd)))
        J.check(self._lib.jnx_op_qk_norm_rope_append(
            self._ref, x, ld, p, n, *self._qc.refs, _dense(slot, _I32, n),
            _dense(at, _I32, n), self._status, self._on(stream)))

    def backward(self, qkv: torch.Tensor, pos: torch.Tensor, dq: torch.Tensor, dk: torch.Tensor,
                 dqkv: torch.Tensor, dgamma_q: Optional[torch.Tensor] = None,
                 dgamma_k: Optional[torch.Tensor] = None, stream=None) -> None:
        """dqkv's query and key columns (same strides as qkv) and the gains' gradients."""
        h, hkv, hd = self.dims
        n, x, ld, p = self._args(qkv, pos)
        _bf16(dqkv, *qkv.shape)
        if n > 1 and dqkv.stride(0) != ld:
            raise ValueError("dqkv and qkv differ in their row strides")
        gains = [None if g is None else _dense(g, _F32, hd) for g in (dgamma_q, dgamma_k)]
        self._qk.fill(*_view(dq, (n, h, hd)), *_view(dk, (n, hkv, hd)))
        J.check(self._lib.jnx_op_qk_norm_rope_backward(
            self._ref, x, ld, p, n, *self._qk.refs, dqkv.data_ptr(), *gains, self._ws, self._nws,
            self._on(stream)))


class PromptPlan:
    """Packed prompts: query and key lengths of each sequence and the keys at its start
    that every row sees.  The queries are the last of a sequence's positions."""

    def __init__(self, q_lens: Sequence[int], kv_lens: Optional[Sequence[int]] = None,
                 prefix: Optional[Sequence[int]] = None, device="cuda"):
        kv_lens = q_lens if kv_lens is None else kv_lens
        if len(kv_lens) != len(q_lens) or (prefix is not None and len(prefix) != len(q_lens)):
            raise ValueError("lengths of different numbers of sequences")
        cu = lambda n: np.concatenate([[0], np.cumsum(n, dtype=np.int64)]).astype(np.int64)
        both = [cu(q_lens), cu(kv_lens)]
        if any(int(x[-1]) >= 2 ** 31 for x in both):
            raise ValueError("2^31 rows or more")
        self.h = [x.astype(np.int32) for x in both]
        if prefix is not None and any(prefix):
            self.h.append(np.asarray(prefix, dtype=np.int32))
        self.n_seqs, self.device = len(q_lens), device
        self.n_q, self.n_kv = int(self.h[0][-1]), int(self.h[1][-1])
        self.d = [torch.from_numpy(x).to(device) for x in self.h]

    def struct(self, n_heads: int, n_kv_heads: int, head_dim: int):
        """The prompt with its work lists for a head layout, and what they lie in."""
        ptrs = [x.data_ptr() for x in self.d] + [None] * (3 - len(self.d))
        host = [x.ctypes.data_as(J.P32) for x in self.h] + [None] * (3 - len(self.h))
        p = J.jnx_prompt(self.n_seqs, *ptrs, *host, None, 0, 0, 0, 0)
        L = J.lib()
        n = L.jnx_prompt_items(C.byref(p), n_heads, n_kv_heads, head_dim, None, 0)
        if n < 0:
            J.check(n)
        items = np.zeros((max(n, 1), 2), dtype=np.int32)
        L.jnx_prompt_items(C.byref(p), n_heads, n_kv_heads, head_dim, items.ctypes.data, n)
        items = torch.from_numpy(items).to(self.device)
        p.items = items.data_ptr()
        return p, items


class PromptAttention(_TextOperator):
    """Attention of packed prompts, causal behind the plan's prefixes, and its gradients."""

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, plan: PromptPlan,
                 gradients: bool = False):
        self.plan, self.dims = plan, (n_heads, n_kv_heads, head_dim)
        self.struct, self.items = plan.struct(*self.dims)
        self._ref = C.byref(self.struct)
        super().__init__(J.lib().jnx_op_prompt_attention_backward_workspace_bytes(
            self._ref, *self.dims) if gradients else 0, plan.device)
        self._held += [self.items, *plan.d]
        self.gradients = gradients
        rows = J.jnx_head_rows
        self._qs, self._ks = (plan.n_q, n_heads, head_dim), (plan.n_kv, n_kv_heads, head_dim)
        self._fwd, self._bwd = _Views(*[rows] * 4), _Views(*[rows] * 8)

    def forward(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                lse: Optional[torch.Tensor] = None, stream=None) -> None:
        """out [n_q, H, hd]; lse [n_q, H] fp32 where the gradients are wanted later."""
        qs, ks = self._qs, self._ks
        if lse is not None:
            lse = _dense(lse, _F32, *qs[:2])
        self._fwd.fill(*_view(q, qs), *_view(k, ks), *_view(v, ks), *_view(out, qs))
        J.check(self._lib.jnx_op_prompt_attention(self._ref, *self.dims, *self._fwd.refs, None, lse,
                                                  self._status, self._on(stream)))

    def backward(self, q, k, v, out, lse, dout, dq, dk, dv, stream=None) -> None:
        """dq, dk, dv from dout, with out and lse of the forward of the same q, k and v.  Nothing
        is kept from a forward to its backward."""
        if not self.gradients:
            raise ValueError("made for the forward only (gradients=False)")
        qs, ks, r = self._qs, self._ks, self._bwd.refs
        self._bwd.fill(*_view(q, qs), *_view(k, ks), *_view(v, ks), *_view(out, qs),
                       *_view(dout, qs), *_view(dq, qs), *_view(dk, ks), *_view(dv, ks))
        J.check(self._lib.jnx_op_prompt_attention_backward(
            self._ref, *self.dims, *r[:4], None, _dense(lse, _F32, *qs[:2]), *r[4:],
            self._ws, self._nws, self._status, self._on(stream)))


class DecodeAttention(_TextOperator):
    """Attention of one new token of each live sequence against its cache."""

    def __init__(self, n_heads: int, n_kv_heads: int, head_dim: int, max_batch: int,
                 device="cuda"):
        self.dims, self.max_batch = (n_heads, n_kv_heads, head_dim), max_batch
        super().__init__(J.lib().jnx_op_decode_attention_workspace_bytes(max_batch, n_heads,
                                                                         head_dim), device)

        self._views = _Views(J.jnx_kv_cache, J.jnx_head_rows, J.jnx_head_rows)

    def forward(self, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                slot: torch.Tensor, n_cached: torch.Tensor, out: torch.Tensor,
                stream=None) -> None:
        """out [b, H, hd] of q [b, H, hd] over the first n_cached[i] tokens of slot[i] in
        the cache [slots, room, Hkv, hd]."""
        h, hkv, hd = self.dims
        b = q.shape[0]
        if b > self.max_batch:
            raise ValueError(f"batch of {b}, at most {self.max_batch}")
        rows, r = (b, h, hd), self._views.refs
        self._views.fill(*_cache(k_cache, v_cache, (hkv, hd)), *_view(q, rows), *_view(out, rows))
        J.check(self._lib.jnx_op_decode_attention(
            r[0], b, h, hkv, hd, r[1], _dense(slot, _I32, b),
            _dense(n_cached, _I32, b), r[2], self._ws, self._nws, self._status,
            self._on(stream)))


class VocabLoss(_TextOperator):
    """Next-token losses of hidden rows over a vocabulary w [vocab, d], and their
    gradients; the logits are never stored."""

    def __init__(self, w: torch.Tensor, max_rows: int, gradients: bool = True,
                 piece_rows: int = 0):
        self.w, (self.vocab, self.d) = _bf16(w, *w.shape), w.shape
        self.max_rows, self.piece_rows, self.gradients = max_rows, piece_rows, gradients
        L = J.lib()
        need = L.jnx_op_vocab_loss_workspace_bytes(max_rows, self.vocab, self.d)
        if gradients:
            need = max(need, L.jnx_op_vocab_loss_train_workspace_bytes(max_rows, self.vocab,
                                                                       self.d, piece_rows))
        super().__init__(need, w.device)

    def _args(self, h: torch.Tensor, targets: torch.Tensor):
        n = h.shape[0]
        if n > self.max_rows:
            raise ValueError(f"{n} rows, at most {self.max_rows}")
        _bf16(h, n, self.d)
        return n, h.data_ptr(), h.stride(0), self.w.data_ptr(), self.w.stride(0), \
            _dense(targets, _I32, n)

    def loss(self, h: torch.Tensor, targets: torch.Tensor, loss: torch.Tensor,
             stream=None) -> None:
        """loss [n] fp32 of h [n, d]; 0 where targets [n] is negative."""
        n, *args = self._args(h, targets)
        J.check(self._lib.jnx_op_vocab_loss(
            *args, n, self.vocab, self.d, _dense(loss, _F32, n), self._ws, self._nws,
            self._status, self._on(stream)))

    def train(self, h: torch.Tensor, targets: torch.Tensor, row_weight: torch.Tensor,
              loss: torch.Tensor, dh: torch.Tensor, dw: Optional[torch.Tensor] = None,
              stream=None) -> None:
        """Also the gradients of sum(row_weight * loss): dh [n, d] and dw [vocab, d] (None:
        a frozen vocabulary), bf16."""
        if not self.gradients:
            raise ValueError("made for losses only (gradients=False)")
        n, *args = self._args(h, targets)
        _bf16(dh, n, self.d)
        grads = [dh.data_ptr(), dh.stride(0), None, 0]
        if dw is not None:
            _bf16(dw, self.vocab, self.d)
            grads[2:] = [dw.data_ptr(), dw.stride(0)]
        J.check(self._lib.jnx_op_vocab_loss_train(
            *args, _dense(row_weight, _F32, n), n, self.vocab, self.d, self.piece_rows,
            _dense(loss, _F32, n), *grads, self._ws, self._nws, self._status,
            self._on(stream)))
