"""One MoE expert layer step through the C ABI.

PyTorch only allocates device memory and provides the stream; every step of
the layer runs in the library's kernels (see _lib.py for the entry points).
"""
from __future__ import annotations

import dataclasses
from typing import Optional

import torch

from . import _lib as L


@dataclasses.dataclass
class LayerShape:
    T: int
    d: int
    E: int
    k: int
    F: int

    @property
    def rows_cap(self) -> int:
        return L.moe_perm_rows_max(self.T, self.k, self.E)


@dataclasses.dataclass
class BalanceLoss:
    """Auxiliary losses of a layer's router (moe_balance_loss): the load-balance loss over the batch, or per
    packed sequence with seq_offsets [n + 1] int32, and the z-loss. token_mask [T] uint8: 0 for padding.
    forward() keeps the fields' values of the moment for its backward(), so the object may be set anew and used
    again in between; the tensors are not copied and stay as they are until that backward."""
    coef: float
    z_coef: float = 0.0
    token_mask: Optional[torch.Tensor] = None
    seq_offsets: Optional[torch.Tensor] = None

    @property
    def n_seq(self) -> int:
        return 1 if self.seq_offsets is None else self.seq_offsets.numel() - 1


def _alloc_routing(o, s: LayerShape, dev, balance_seqs: int):
    """What the backward needs of a routing, as attributes of o (balance_seqs: most sequences of a
    BalanceLoss, 0: none)."""
    f32, i32 = torch.float32, torch.int32
    o.topk_idx = torch.empty(s.T, s.k, dtype=i32, device=dev)
    o.topk_gate = torch.empty(s.T, s.k, dtype=f32, device=dev)
    o.counts = torch.empty(s.E, dtype=i32, device=dev)
    o.group_offsets = torch.empty(s.E + 1, dtype=i32, device=dev)
    o.group_counts = torch.empty(s.E, dtype=i32, device=dev)
    o.row_of_assignment = torch.empty(s.T, s.k, dtype=i32, device=dev)
    # of the forward, for the backward: its BalanceLoss (a copy), number of sequences and mask
    o.balance, o.balance_n, o.balance_mask = None, 0, None
    o.balance_seqs = balance_seqs
    if balance_seqs:
        o.loss = torch.empty(2, dtype=f32, device=dev)
        o.balance_counts = torch.empty(balance_seqs, s.E, dtype=i32, device=dev)
        o.balance_prob = torch.empty(balance_seqs, s.E, dtype=f32, device=dev)
        o.balance_tokens = torch.empty(balance_seqs + 2, dtype=i32, device=dev)
        o.lse = torch.empty(s.T, dtype=f32, device=dev)


class MoECheckpoint:
    """What one layer keeps from its forward to its backward, with the activations in 8 bits: the routing,
    x and the pre-activations [A|B] (T*d + 2*F*rows_cap bytes and 1/32 of that in scales; with
    balance_seqs also the fp32 logits). Pass it to forward() and backward(); the MoELayerBuffers
    (ckpt=True) of the calls may serve other layers in between."""

    def __init__(self, shape: LayerShape, device="cuda", balance_seqs: int = 0):
        s, dev, u8 = shape, torch.device(device), torch.uint8
        if s.d % 128 or s.F % 128:
            raise ValueError("d_model and d_ff must be multiples of 128")
        self.shape = s
        _alloc_routing(self, s, dev, balance_seqs)
        self.logits = torch.empty(s.T, s.E, dtype=torch.float32, device=dev) if balance_seqs else None
        self.x_q = torch.empty(s.T, s.d, dtype=u8, device=dev)
        self.x_scale = torch.empty(s.T, s.d // 32, dtype=u8, device=dev)
        self.ab_q = torch.empty(s.rows_cap, 2 * s.F, dtype=u8, device=dev)
        self.ab_scale = torch.empty(s.rows_cap, 2 * s.F // 32, dtype=u8, device=dev)


class MoELayerBuffers:
    """Device buffers of one layer step (activations, grouped layout, grads).

    gather=False (default): moe_permute writes X_perm and the GEMMs read it with tile
    loads. gather=True: the grouped operand is read from x through token_of_row by the
    GEMMs' 4-row TMA gathers (moe_permute_map and the *_gather calls), so X_perm is not
    allocated; the results are identical, but on GB300 the gathers make the two GEMMs
    that read X_perm about 3.3x slower (32 gathers of 4 x 128 bytes per 128-row k-block
    against one tile load), far more than the separate gather pass costs.

    fused_combine=True: the combine runs in the down GEMM's epilogue
    (moe_grouped_ffn_fwd_combine, fp32 atomics into y_acc; the last bits of y can
    change from run to run); O is then stored only when a backward follows.

    balance_seqs=n: buffers for a BalanceLoss over up to n sequences (forward's balance argument).

    ckpt=True: for calls with a MoECheckpoint only, which keeps what a layer's backward needs; one
    object then serves any number of layers of the shape (ab is not allocated)."""

    def __init__(self, shape: LayerShape, device="cuda", backward: bool = True,
                 gather: bool = False, fused_combine: bool = False, balance_seqs: int = 0,
                 ckpt: bool = False):
        s = shape
        self.shape = s
        self.gather = gather
        self.fused_combine = fused_combine
        if fused_combine and gather:
            raise ValueError("fused_combine reads X_perm: use it with gather=False")
        self.ckpt = ckpt
        if ckpt and (gather or fused_combine):
            raise ValueError("the checkpointed forward has neither gather nor fused_combine")
        self.x = None  # the forward's input, kept for the backward
        R = s.rows_cap
        dev = torch.device(device)
        bf16, f32, i32 = torch.bfloat16, torch.float32, torch.int32
        self.ws_bytes = max(L.moe_workspace_size(s.T, s.d, s.E, s.k, s.F), 256)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        self.logits = torch.empty(s.T, s.E, dtype=f32, device=dev)
        _alloc_routing(self, s, dev, balance_seqs)
        if balance_seqs:
            self.balance_ws = torch.empty(L.moe_balance_workspace_size(s.T, s.E, balance_seqs), dtype=torch.uint8,
                                          device=dev)
        if gather:
            self.token_of_row = torch.empty(R, dtype=i32, device=dev)
            self.x_perm = None
        else:
            self.token_of_row = None
            self.x_perm = torch.empty(R, s.d, dtype=bf16, device=dev)
        self.ab = None if ckpt else torch.empty(R, 2 * s.F, dtype=bf16, device=dev)
        self.h = torch.empty(R, s.F, dtype=bf16, device=dev)
        self.out_perm = (torch.empty(R, s.d, dtype=bf16, device=dev)
                         if backward or not fused_combine else None)
        self.y_acc = torch.empty(s.T, s.d, dtype=f32, device=dev) if fused_combine else None
        self.y = torch.empty(s.T, s.d, dtype=bf16, device=dev)
        if backward:
            self.d_out_perm = torch.empty(R, s.d, dtype=bf16, device=dev)
            self.d_gate = torch.empty(s.T, s.k, dtype=f32, device=dev)
            self.d_ab = torch.empty(R, 2 * s.F, dtype=bf16, device=dev)
            self.dx_perm = torch.empty(R, s.d, dtype=bf16, device=dev)
            self.dw_gate_up = torch.empty(s.E, 2 * s.F, s.d, dtype=bf16, device=dev)
            self.dw_down = torch.empty(s.E, s.d, s.F, dtype=bf16, device=dev)
            self.d_logits = torch.empty(s.T, s.k, dtype=f32, device=dev)
            self.dw_router = torch.empty(s.d, s.E, dtype=f32, device=dev)
            self.dx = torch.empty(s.T, s.d, dtype=bf16, device=dev)
            self.dz = torch.empty(s.T, s.E, dtype=f32, device=dev) if balance_seqs else None
            self.x_back = torch.empty(s.T, s.d, dtype=bf16, device=dev) if ckpt else None
            # second stream: the router backward and the unpermute-sum run beside
            # the grouped GEMMs (whose CTAs leave registers and threads free)
            self.side = torch.cuda.Stream(device=dev) if dev.type == "cuda" else None


def route(b: MoELayerBuffers, x, w_router, bias, active_mask=None, logits_in=None,
          keep_logits: bool = False, stream=None):
    _route(b, b, b.logits if keep_logits else None, x, w_router, bias, active_mask, logits_in, stream)


def _route(b, kept, logits, x, w_router, bias, active_mask, logits_in, stream):
    s = b.shape
    L.moe_route(x, w_router, bias, active_mask, s.T, s.d, s.E, s.k, logits_in, logits, kept.topk_idx,
                kept.topk_gate, kept.counts, b.ws, b.ws_bytes, stream)


def _kept(b: MoELayerBuffers, ckpt: Optional[MoECheckpoint]):
    """What holds the routing: b, or the layer's checkpoint."""
    if (ckpt is not None) != b.ckpt:
        raise ValueError("buffers made with ckpt=True go with a MoECheckpoint, others without")
    if ckpt is not None and (ckpt.shape != b.shape or ckpt.topk_idx.device != b.h.device):
        raise ValueError("the checkpoint is of another shape or device")
    return b if ckpt is None else ckpt


def _check_balance(b, kept, balance: BalanceLoss):
    if not 1 <= balance.n_seq <= min(kept.balance_seqs, b.balance_seqs):
        raise ValueError(f"balance over {balance.n_seq} sequences: more than the buffers' balance_seqs")
    off, tok, dev = balance.seq_offsets, balance.token_mask, kept.topk_idx.device
    if off is not None and (off.dtype != torch.int32 or not off.is_contiguous() or off.device != dev):
        raise ValueError("seq_offsets: a contiguous int32 tensor on the layer's device")
    if tok is not None and (tok.dtype not in (torch.uint8, torch.bool) or not tok.is_contiguous()
                            or tok.numel() != b.shape.T or tok.device != dev):
        raise ValueError("token_mask: a contiguous uint8 or bool tensor of T values on the layer's device")


def _check_d_loss(kept, d_loss):
    if kept.balance is None:
        raise ValueError("d_loss: the forward had no balance")
    if (d_loss.dtype != torch.float32 or d_loss.numel() != 2 or not d_loss.is_contiguous()
            or d_loss.device != kept.topk_idx.device):
        raise ValueError("d_loss: two contiguous fp32 values on the layer's device")


def forward(b: MoELayerBuffers, x, w_router, bias, w_gate_up, w_down, active_mask=None,
            logits_in=None, keep_logits: bool = False, stream=None,
            balance: Optional[BalanceLoss] = None, ckpt: Optional[MoECheckpoint] = None):
    """route -> permute -> grouped SwiGLU FFN -> combine (in the down GEMM's epilogue
    when b.fused_combine). Returns b.y.

    keep_logits: b.logits [T, E] receives the masked logits.
    balance: adds the router's auxiliary losses; loss [2] (balance, z), balance_counts, balance_prob
    [sequences, E] are then in b (in ckpt, when given), and backward() adds their gradient.
    ckpt: the layer's checkpoint (for b with ckpt=True): receives the routing (in the place of b's
    attributes), x and the pre-activations in 8 bits."""
    s = b.shape
    R = s.rows_cap
    kept = _kept(b, ckpt)
    if balance is not None:
        _check_balance(b, kept, balance)
    stream = L.stream_handle(stream)  # once for all calls
    logits = kept.logits if balance is not None else b.logits if keep_logits else None
    _route(b, kept, logits, x, w_router, bias, active_mask, logits_in, stream)
    if keep_logits and logits is not b.logits:  # (the routing of these logits is the same one)
        _route(b, kept, b.logits, x, w_router, bias, active_mask, logits, stream)
    kept.balance = None
    if balance is not None:
        balance = dataclasses.replace(balance)  # the caller's object may change before the backward
        kept.balance, kept.balance_n, kept.balance_mask = balance, balance.n_seq, active_mask
        L.moe_balance_loss(logits, kept.topk_idx, active_mask, balance.token_mask, balance.seq_offsets,
                           balance.n_seq, s.T, s.E, s.k, balance.coef, balance.z_coef, kept.loss,
                           kept.balance_counts, kept.balance_prob, kept.balance_tokens, kept.lse,
                           b.balance_ws, b.balance_ws.numel(), stream)
    if ckpt is not None:
        L.moe_permute(x, kept.topk_idx, kept.counts, s.T, s.d, s.E, s.k, R, kept.group_offsets,
                      kept.group_counts, kept.row_of_assignment, b.x_perm, b.ws, b.ws_bytes, stream)
        L.moe_ckpt_pack(x, s.T, s.d, ckpt.x_q, ckpt.x_scale, stream)
        L.moe_grouped_ffn_fwd_ckpt(b.x_perm, kept.group_offsets, s.E, s.d, s.F, R, w_gate_up, w_down,
                                   ckpt.ab_q, ckpt.ab_scale, b.h, b.out_perm, b.ws, b.ws_bytes, stream)
        L.moe_unpermute_combine(b.out_perm, kept.row_of_assignment, kept.topk_gate, s.T, s.d, s.k, b.y,
                                stream)
        return b.y
    b.x = x
    if b.gather:
        L.moe_permute_map(b.topk_idx, b.counts, s.T, s.E, s.k, R, b.group_offsets,
                          b.group_counts, b.row_of_assignment, b.token_of_row, b.ws, b.ws_bytes,
                          stream)
        L.moe_grouped_ffn_fwd_gather(x, b.token_of_row, s.T, b.group_offsets, s.E, s.d, s.F, R,
                                     w_gate_up, w_down, b.ab, b.h, b.out_perm, b.ws, b.ws_bytes,
                                     stream)
    else:
        L.moe_permute(x, b.topk_idx, b.counts, s.T, s.d, s.E, s.k, R, b.group_offsets,
                      b.group_counts, b.row_of_assignment, b.x_perm, b.ws, b.ws_bytes, stream)
        if b.fused_combine:
            L.moe_grouped_ffn_fwd_combine(b.x_perm, b.group_offsets, s.E, s.d, s.F, R, w_gate_up,
                                          w_down, b.row_of_assignment, b.topk_gate, s.T, s.k,
                                          b.ab, b.h, b.out_perm, b.y_acc, b.y, b.ws, b.ws_bytes,
                                          stream)
            return b.y
        L.moe_grouped_ffn_fwd(b.x_perm, b.group_offsets, s.E, s.d, s.F, R, w_gate_up, w_down,
                              b.ab, b.h, b.out_perm, b.ws, b.ws_bytes, stream)
    L.moe_unpermute_combine(b.out_perm, b.row_of_assignment, b.topk_gate, s.T, s.d, s.k, b.y,
                            stream)
    return b.y


def backward(b: MoELayerBuffers, dy, w_router, w_gate_up, w_down, stream=None,
             overlap: bool = False, active_mask=None, d_loss=None,
             ckpt: Optional[MoECheckpoint] = None):
    """combine bwd -> grouped FFN dgrad (with the gate gradient and the router's term of dx)
    -> router bwd -> permute bwd -> grouped FFN wgrad.

    active_mask: the LAEP mask the forward routed with (None: all experts live). Pruned
    experts' weight gradients are not written (their buffers keep what they held); live
    experts without tokens get exact zeros.

    With overlap, the router backward and the unpermute-sum (after the dgrad GEMMs) run on
    a second stream while the main stream computes the weight gradients; the main stream
    waits for them at the end. The
    default is one stream: on GB300 at T=65536, d_model=7168 the step is power-capped,
    and running those memory-bound kernels beside the GEMMs slowed the GEMMs by more
    than it hid (96.1-96.7 against 97.0-97.3 ms per step).

    After a forward with balance, dw_router and dx hold the auxiliary losses' gradient too (dx is then rounded to bf16
    once more, where the losses' share is added); d_loss [2]
    fp32 on the device: the gradient of the losses (None: ones).
    ckpt: the layer's checkpoint, as in forward(): X_perm, x and H come from its 8 bits.
    Returns (dx, dw_gate_up, dw_down, dw_router)."""
    s = b.shape
    R = s.rows_cap
    kept = _kept(b, ckpt)
    if d_loss is not None:
        _check_d_loss(kept, d_loss)
    if kept.balance is not None and getattr(b, "dz", None) is None:
        raise ValueError("the forward had a balance loss: its backward needs buffers made with balance_seqs")
    if overlap:
        main = torch.cuda.current_stream() if stream is None else stream
        side = b.side
    else:
        main = side = L.stream_handle(stream)  # once for all calls
    # d_out_perm = g * dy; the gate gradient comes from the dH GEMM (below), so the combine
    # backward does not read out_perm
    L.moe_unpermute_combine_bwd(dy, None, kept.row_of_assignment, kept.topk_gate,
                                kept.group_offsets, kept.group_counts, s.T, s.d, s.E, s.k,
                                b.d_out_perm, None, main)
    # dH (+ the gate gradient into b.d_gate), dX with the router's term of dx added to the
    # grouped rows in its epilogue
    if ckpt is not None:
        x = b.x_back
        L.moe_ckpt_permute(ckpt.x_q, ckpt.x_scale, ckpt.row_of_assignment, ckpt.group_offsets,
                           ckpt.group_counts, s.T, s.d, s.E, s.k, R, x, b.x_perm, main)
        L.moe_grouped_ffn_bwd_dgrad_ckpt(b.d_out_perm, ckpt.ab_q, ckpt.ab_scale, ckpt.group_offsets, s.E,
                                         s.d, s.F, R, w_gate_up, w_down, ckpt.topk_gate, None,
                                         ckpt.row_of_assignment, w_router, s.T, s.k, b.d_gate, b.h,
                                         b.d_ab, b.dx_perm, b.ws, b.ws_bytes, main)
    else:
        x = b.x
        L.moe_grouped_ffn_bwd_dgrad(b.d_out_perm, b.ab, b.group_offsets, s.E, s.d, s.F, R,
                                    w_gate_up, w_down, b.topk_gate, None, b.row_of_assignment,
                                    w_router, s.T, s.k, b.d_gate, b.d_ab, b.dx_perm, b.ws,
                                    b.ws_bytes, main)
    if overlap:
        ev = torch.cuda.Event()
        ev.record(main)
        side.wait_event(ev)
    bal = kept.balance
    if bal is not None:
        L.moe_balance_loss_bwd(kept.logits, kept.balance_mask, bal.seq_offsets, kept.balance_n, s.T, s.E,
                               s.k, bal.coef, bal.z_coef, kept.balance_counts, kept.balance_tokens,
                               kept.lse, d_loss, b.dz, side)
        L.moe_route_bwd_dense(x, kept.topk_idx, kept.topk_gate, b.d_gate, b.dz, s.T, s.d, s.E, s.k,
                              b.d_logits, b.dw_router, b.ws, b.ws_bytes, side)
    else:
        L.moe_route_bwd(x, kept.topk_idx, kept.topk_gate, b.d_gate, s.T, s.d, s.E, s.k, b.d_logits,
                        b.dw_router, b.ws, b.ws_bytes, side)
    L.moe_permute_bwd(b.dx_perm, kept.row_of_assignment, kept.topk_idx, None, None, s.T, s.d, s.E,
                      s.k, b.dx, b.ws, b.ws_bytes, side)
    if bal is not None:
        # dx is rounded to bf16 by the call above and again by this one: half a step more, as much as each of the
        # k rows of dx_perm has. An fp32 sum in between would be 2 T d more bytes written and read (~280 us at T=65536,
        # d_model=7168, beside ~1,500 for the two calls).
        L.moe_route_dx(b.dz, w_router, b.dx, s.T, s.d, s.E, s.k, b.dx, b.ws, b.ws_bytes, side)
    if b.gather:
        L.moe_grouped_ffn_bwd_wgrad_gather(b.d_out_perm, b.x, b.token_of_row, s.T, b.h, b.d_ab,
                                           b.group_offsets, active_mask, s.E, s.d, s.F, R,
                                           b.dw_gate_up, b.dw_down, b.ws, b.ws_bytes, main)
    else:
        L.moe_grouped_ffn_bwd_wgrad(b.d_out_perm, b.x_perm, b.h, b.d_ab, kept.group_offsets,
                                    active_mask, s.E, s.d, s.F, R, b.dw_gate_up, b.dw_down, b.ws,
                                    b.ws_bytes, main)
    if overlap:
        ev = torch.cuda.Event()
        ev.record(side)
        main.wait_event(ev)
    return b.dx, b.dw_gate_up, b.dw_down, b.dw_router


def prune_from_counts(counts_host, S: int, k: int, *, prune_count: int = -1,
                      alpha: float = 0.0, beta: float = 0.0):
    """LAEP decision on a host histogram; returns (mask uint8 tensor on CPU, n_pruned)."""
    mask, n = L.laep_prune_mask([int(c) for c in counts_host], S, k, alpha, beta, prune_count)
    return torch.tensor(mask, dtype=torch.uint8), n
