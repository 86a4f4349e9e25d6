"""Measured operators beside the MoE layer's own: the balance loss with its gradients, and 8-bit
activation checkpoints with their use in the backward pass.

What a training program calls, in five kinds of case:
  balance  moe_balance_loss + moe_balance_loss_bwd: loss, per-expert counts, the logits' gradient
  router   moe_route_bwd_dense + moe_route_dx: that gradient into the router's weight and the layer's input
  rows     moe_ckpt_pack + moe_ckpt_permute: the layer's input in 8 bits, back as rows of the groups
  ffn_fwd  moe_grouped_ffn_fwd_ckpt + moe_ckpt_unpack_ab: the experts' forward with the pre-activations
           [A|B] kept in 8 bits, and what is kept read back
  ffn_bwd  moe_grouped_ffn_bwd_dgrad_ckpt + moe_grouped_ffn_bwd_wgrad: the experts' backward from them
`own` false: the same results from elementary torch operations in 32 bits or more. `own` true: the
framework's calls. Inputs are synthetic and seeded, with the distributions of the package's own workloads.

A case: kind, T tokens, d = d_model, E experts, k experts per token, F = d_ff, bias ("none", "zipf" with
zipf_s: the load's skew), pruned (experts masked out), seqs (packed sequences; 0: one, over all tokens),
padded (share of the tokens that a mask leaves out).
"""
import math

import torch

own = False

PAD = 128      # rows of a group are padded to this
BLOCK = 32     # values that share a scale
E4M3_MAX = 448.0
BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


def _case(name, kind, T, d, E, k, F=0, bias="zipf", zipf_s=1.0, pruned=0, seqs=0, padded=0.0):
    c = {"kind": kind, "T": T, "d": d, "E": E, "k": k, "F": F, "bias": bias, "zipf_s": zipf_s,
         "pruned": pruned, "seqs": seqs, "padded": padded}
    return {"name": name, **c} if name else c


def listed():
    return [
        # ---- the balance loss and its gradient
        # a validation pass over a few short sequences: launches and latency count
        _case("balance_few_tokens", "balance", 37, 0, 64, 6, seqs=3),
        # a training step on packed sequences, 16 of 64 experts pruned, the batch's tail padded
        _case("balance_packed", "balance", 16384, 0, 64, 8, pruned=16, seqs=24, padded=0.06),
        # the largest layer before pruning, one loss over the whole batch
        _case("balance_large", "balance", 65536, 0, 256, 8, zipf_s=0.8),
        # ---- that gradient into the router's weight and the layer's input
        # a small model on a ragged token count
        _case("router_ragged", "router", 1021, 512, 32, 4),
        # the largest layer after pruning
        _case("router_large", "router", 65536, 7168, 171, 8),
        # ---- the layer's input in 8 bits and back
        # a micro-batch of ragged length
        _case("rows_ragged", "rows", 1021, 2048, 64, 6),
        # the 128-expert layer under skewed load
        _case("rows_large", "rows", 32768, 4096, 128, 8),
        # ---- the experts, with [A|B] in 8 bits between forward and backward
        # a small model on a ragged token count, d_ff not a multiple of 256
        _case("ffn_fwd_small", "ffn_fwd", 1021, 512, 32, 4, 384, zipf_s=0.8),
        # a training step's experts; the balance loss has evened the load
        _case("ffn_fwd_large", "ffn_fwd", 16384, 4096, 64, 8, 2048, bias="none"),
        # their backward passes, and one of a micro-batch of ragged length
        _case("ffn_bwd_small", "ffn_bwd", 1021, 512, 32, 4, 384, zipf_s=0.8),
        _case("ffn_bwd_ragged", "ffn_bwd", 2039, 2048, 64, 6, 1408, zipf_s=0.5),
        _case("ffn_bwd_large", "ffn_bwd", 16384, 4096, 64, 8, 2048, bias="none"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithms."""
    top = {c["kind"]: c for c in listed()}  # the last of a kind is its largest
    while True:
        kind = rng.choice(("balance", "balance", "router", "router", "rows", "rows", "ffn_fwd", "ffn_bwd"))
        ffn = kind.startswith("ffn")
        E = _log_int(rng, 4, 256)
        step = 128 if ffn else 8
        d = 0 if kind == "balance" else step * _log_int(rng, 256 // step, 7168 // step)
        c = _case("", kind, _log_int(rng, 1, 65536), d, E, rng.randint(1, min(8, E)),
                  128 * _log_int(rng, 1, 16) if ffn else 0, rng.choice(("none", "zipf", "zipf")),
                  0.5 if ffn else rng.choice((0.8, 1.0, 1.2)))
        if kind == "balance":
            c["pruned"] = rng.choice((0, 0, (E - c["k"]) // 4))
            c["seqs"] = rng.choice((0, _log_int(rng, 1, 64)))
            c["padded"] = rng.choice((0.0, 0.0, 0.1))
        w, m = work(c), work(top[kind])
        if w["bytes"] <= m["bytes"] and w["flops"] <= m["flops"]:
            if ffn and E * 2 * c["T"] * c["k"] * (c["d"] + c["F"]) > 1 << 35:
                continue  # (the plain form's per-expert copies)
            return c


# ---------------------------------------------------------------- inputs


def _rows_cap(c):
    return c["T"] * c["k"] + PAD * c["E"]


def _randn(g, *shape, std=1.0, dtype=BF16):
    return torch.empty(*shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _logits(c, g):
    """Router logits as the top-k leaves them (pruned experts -inf), the mask of live experts or None."""
    E = c["E"]
    bias = torch.zeros(E, device="cuda", dtype=F64)
    if c["bias"] == "zipf":
        bias = -c["zipf_s"] * torch.log(1.0 + torch.randperm(E, generator=g, device="cuda").double())
    z = _randn(g, c["T"], E, dtype=F32) + bias.float()
    mask = None
    if c["pruned"]:
        mask = torch.ones(E, dtype=torch.uint8, device="cuda")
        mask[torch.argsort(bias, stable=True)[:c["pruned"]]] = 0
        z[:, mask == 0] = -math.inf
    return z, mask


def _topk(z, k):
    """The k largest logits, ties to the lower index, and the softmax over them."""
    v, idx = torch.sort(z, dim=1, descending=True, stable=True)
    return idx[:, :k].to(I32).contiguous(), torch.softmax(v[:, :k], dim=1).contiguous()


def _layout(idx, E):
    """Grouped layout of a routing: group_offsets, group_counts, row_of_assignment."""
    flat = idx.reshape(-1).long()
    counts = torch.bincount(flat, minlength=E)
    padded = (counts + PAD - 1) // PAD * PAD
    off = torch.zeros(E + 1, dtype=torch.long, device=flat.device)
    off[1:] = torch.cumsum(padded, 0)
    first = torch.cumsum(counts, 0) - counts
    order = torch.argsort(flat, stable=True)
    row = torch.empty_like(flat)
    e = flat[order]
    row[order] = off[e] + torch.arange(flat.numel(), device=flat.device) - first[e]
    return off.to(I32), counts.to(I32), row.reshape(idx.shape).to(I32)


def _grouped(c, rows, row, scale=None):
    """[R, d] with rows[t] (times scale[t, j]) at the row of every assignment, zeros elsewhere."""
    out = torch.zeros(_rows_cap(c), rows.shape[1], dtype=rows.dtype, device=rows.device)
    v = rows[:, None, :] if scale is None else (rows.float()[:, None, :] * scale[:, :, None]).to(rows.dtype)
    out[row.long().reshape(-1)] = v.expand(-1, c["k"], -1).reshape(-1, rows.shape[1])
    return out


def _sequences(c, g):
    """Offsets of packed sequences (some may be empty, a few rows may lie behind the last), or None."""
    if not c["seqs"]:
        return None
    cut = torch.randint(0, c["T"] + 1, (c["seqs"],), generator=g, device="cuda")
    off = torch.zeros(c["seqs"] + 1, dtype=I32, device="cuda")
    off[1:] = torch.sort(cut)[0].to(I32)
    off[-1] = c["T"] - c["T"] // 64
    return torch.cummax(off, 0)[0].to(I32).clamp(max=c["T"] - c["T"] // 64).contiguous()


def prepare(case, seed):
    c, T, d, E, k, F, R = case, case["T"], case["d"], case["E"], case["k"], case["F"], _rows_cap(case)
    g = torch.Generator(device="cuda").manual_seed(1000 + int(seed))
    s = {"case": c}

    def empty(*shape, dtype=BF16):
        return torch.zeros(*shape, dtype=dtype, device="cuda")

    z, s["mask"] = _logits(c, g)
    s["idx"], s["gate"] = _topk(z, k)
    if c["kind"] == "balance":
        s["z"], S = z, max(1, c["seqs"])
        s["seq"] = _sequences(c, g)
        s["tokens"] = None
        if c["padded"]:  # a padded batch: its tail, and a few tokens in between
            keep = torch.rand(T, generator=g, device="cuda") >= c["padded"] / 2
            keep[T - int(T * c["padded"] / 2):] = False
            s["tokens"] = keep.to(torch.uint8)
        s["coef"], s["z_coef"] = 0.01, 0.001
        s["d_loss"] = 0.5 + torch.rand(2, generator=g, device="cuda")
        s["loss"], s["lse"], s["dz"] = empty(2, dtype=F32), empty(T, dtype=F32), empty(T, E, dtype=F32)
        s["counts"], s["prob"] = empty(S, E, dtype=I32), empty(S, E, dtype=F32)
        s["n_tokens"] = empty(S + 2, dtype=I32)
    elif c["kind"] == "router":
        p = torch.softmax(z, dim=1)
        f = torch.bincount(s["idx"].reshape(-1).long(), minlength=E).float() * (E / (T * k))
        s["g_dz"] = (p * (f - (p * f).sum(1, keepdim=True))).contiguous()
        s["x"], s["dx_in"] = _randn(g, T, d), _randn(g, T, d, std=0.02)
        s["w"] = _randn(g, d, E, std=1.0 / math.sqrt(d), dtype=F32)
        s["d_gate"] = _randn(g, T, k, dtype=F32)
        s["d_logits"], s["dw"], s["dx"] = empty(T, k, dtype=F32), empty(d, E, dtype=F32), empty(T, d)
    else:
        s["off"], s["count"], s["row"] = _layout(s["idx"], E)
        if c["kind"] == "rows":
            # a residual stream: a few columns are much larger than the others
            s["x"] = (_randn(g, T, d, dtype=F32)
                      * torch.exp(0.8 * _randn(g, d, dtype=F32))).to(BF16)
            s["q"], s["scale"] = empty(T, d, dtype=torch.uint8), empty(T, -(-d // BLOCK), dtype=torch.uint8)
            s["x_out"], s["x_perm"] = empty(T, d), empty(R, d)
        else:
            s["w_gate_up"], s["w_down"] = _randn(g, E, 2 * F, d, std=0.02), _randn(g, E, d, F, std=0.02)
            s["x_perm"] = _grouped(c, _randn(g, T, d), s["row"])
            if c["kind"] == "ffn_fwd":
                s["ab_q"] = empty(R, 2 * F, dtype=torch.uint8)
                s["ab_scale"] = empty(R, 2 * F // BLOCK, dtype=torch.uint8)
                s["h"], s["out"], s["ab"], s["h_back"] = empty(R, F), empty(R, d), empty(R, 2 * F), empty(R, F)
            else:
                ab = _randn(g, R, 2 * F, std=0.02 * math.sqrt(d), dtype=F32)
                pad = torch.ones(R, 1, dtype=torch.bool, device="cuda")
                pad[s["row"].long().reshape(-1)] = False
                s["ab_q"], s["ab_scale"] = _pack_ab(ab.masked_fill(pad, 0.0))
                del ab
                s["d_out"] = _grouped(c, _randn(g, T, d), s["row"], s["gate"])
                s["h_back"], s["d_ab"], s["dx_perm"] = empty(R, F), empty(R, 2 * F), empty(R, d)
                s["d_gate"] = empty(T, k, dtype=F32)
                s["dw_gate_up"], s["dw_down"] = empty(E, 2 * F, d), empty(E, d, F)
            # where the plain form finds a group's rows: [E, most rows of a group]
            cap = max(1, int(s["count"].max()))
            s["at"] = s["off"][:E, None].long() + torch.arange(cap, device="cuda")
            s["live"] = torch.arange(cap, device="cuda") < s["count"][:, None]
            s["at"] = torch.where(s["live"], s["at"], R - 1)
    return s


# ---------------------------------------------------------------- the framework's calls


def _own(s):
    from paper_2601_14327_gb300 import _lib as L
    c = s["case"]
    T, d, E, k, F, R, S = c["T"], c["d"], c["E"], c["k"], c["F"], _rows_cap(c), max(1, c["seqs"])
    if "ws" not in s and c["kind"] != "rows":  # kept with the other buffers of the shape
        n = L.moe_balance_workspace_size(T, E, S) if c["kind"] == "balance" else L.moe_workspace_size(T, d, E, k, F)
        s["ws"] = torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    if c["kind"] == "balance":
        L.moe_balance_loss(s["z"], s["idx"], s["mask"], s["tokens"], s["seq"], S, T, E, k, s["coef"],
                           s["z_coef"], s["loss"], s["counts"], s["prob"], s["n_tokens"], s["lse"],
                           s["ws"], s["ws"].numel())
        L.moe_balance_loss_bwd(s["z"], s["mask"], s["seq"], S, T, E, k, s["coef"], s["z_coef"],
                               s["counts"], s["n_tokens"], s["lse"], s["d_loss"], s["dz"])
        return {n: s[n] for n in ("loss", "counts", "prob", "n_tokens", "lse", "dz")}
    if c["kind"] == "router":
        L.moe_route_bwd_dense(s["x"], s["idx"], s["gate"], s["d_gate"], s["g_dz"], T, d, E, k,
                              s["d_logits"], s["dw"], s["ws"], s["ws"].numel())
        L.moe_route_dx(s["g_dz"], s["w"], s["dx_in"], T, d, E, k, s["dx"], s["ws"], s["ws"].numel())
        return {n: s[n] for n in ("d_logits", "dw", "dx")}
    if c["kind"] == "rows":
        L.moe_ckpt_pack(s["x"], T, d, s["q"], s["scale"])
        L.moe_ckpt_permute(s["q"], s["scale"], s["row"], s["off"], s["count"], T, d, E, k, R, s["x_out"],
                           s["x_perm"])
        return {"x": s["x_out"], "x_perm": s["x_perm"]}
    if c["kind"] == "ffn_fwd":
        L.moe_grouped_ffn_fwd_ckpt(s["x_perm"], s["off"], E, d, F, R, s["w_gate_up"], s["w_down"], s["ab_q"],
                                   s["ab_scale"], s["h"], s["out"], s["ws"], s["ws"].numel())
        L.moe_ckpt_unpack_ab(s["ab_q"], s["ab_scale"], s["off"], E, F, R, s["ab"], s["h_back"])
        return {"out": s["out"], "ab": s["ab"], "h": s["h_back"]}
    L.moe_grouped_ffn_bwd_dgrad_ckpt(s["d_out"], s["ab_q"], s["ab_scale"], s["off"], E, d, F, R,
                                     s["w_gate_up"], s["w_down"], s["gate"], None, s["row"], None, T, k,
                                     s["d_gate"], s["h_back"], s["d_ab"], s["dx_perm"], s["ws"],
                                     s["ws"].numel())
    L.moe_grouped_ffn_bwd_wgrad(s["d_out"], s["x_perm"], s["h_back"], s["d_ab"], s["off"], None, E, d, F, R,
                                s["dw_gate_up"], s["dw_down"], s["ws"], s["ws"].numel())
    return {"h": s["h_back"], "d_gate": s["d_gate"], "dx_perm": s["dx_perm"],
            "dw_gate_up": s["dw_gate_up"], "dw_down": s["dw_down"]}


# ---------------------------------------------------------------- the plain forms


def _sums(member, v):
    """Sums of v [T, n] over the tokens of each sequence (member [S, T]), in 64 bits."""
    return member @ v.double()


def _plain_balance(s):
    c, z, seq = s["case"], s["z"], s["seq"]
    T, E, k, dev = c["T"], c["E"], c["k"], z.device
    live = torch.ones(E, dtype=torch.bool, device=dev) if s["mask"] is None else s["mask"] != 0
    z = torch.where(live, z, -math.inf)
    top = z.amax(1)
    ok = top > -math.inf
    if s["tokens"] is not None:
        ok = ok & (s["tokens"] != 0)
    of = torch.zeros(T, dtype=torch.long, device=dev)
    if seq is not None:
        t = torch.arange(T, device=dev)
        of = torch.searchsorted(seq[1:], t.to(I32), right=True)
        ok = ok & (t >= seq[0]) & (of < seq.numel() - 1)
        of = of.clamp(max=seq.numel() - 2)
    ex = torch.exp(z - torch.where(ok, top, 0.0)[:, None])
    den = ex.sum(1)
    lse = torch.where(ok, top + torch.log(den), -math.inf)
    p = torch.where(ok[:, None], ex / den[:, None], 0.0)
    member = (ok & (of == torch.arange(s["counts"].shape[0], device=dev)[:, None])).double()   # [S, T]
    n = member.sum(1).long()
    chosen = torch.zeros(T, E, device=dev).scatter_(1, s["idx"].long(), 1.0)
    counts = _sums(member, chosen)                                      # [S, E]
    each = n.clamp(min=1).double()[:, None]
    prob = _sums(member, p) / each
    over = counts * live.sum() / (k * each) - (n > 0).double()[:, None]  # f - 1
    seqs, m = (n > 0).sum(), n.sum()
    loss_b = s["coef"] * ((over + 1) * prob).sum() / seqs.clamp(min=1)
    sq = torch.where(ok, lse, 0.0).double()
    loss_z = s["z_coef"] * (sq * sq).sum() / m.clamp(min=1)
    # gradient (f - 1 in the place of f: the probabilities sum to one)
    a = (s["d_loss"][0].double() * s["coef"] / (seqs.clamp(min=1) * each)).float()[of]   # [T, 1]
    b = (s["d_loss"][1].double() * (2 * s["z_coef"]) / m.clamp(min=1)).float()
    f = over.float()[of]
    dz = p * (a * (f - (p * f).sum(1, keepdim=True)) + b * sq.float()[:, None])
    return {"loss": torch.stack((loss_b, loss_z)).float(), "counts": counts.to(I32), "prob": prob.float(),
            "n_tokens": torch.cat((n, m[None], seqs[None])).to(I32), "lse": lse, "dz": dz}


def _plain_router(s):
    g, dg = s["gate"], s["d_gate"]
    d_logits = g * (dg - (g * dg).sum(1, keepdim=True))
    dz = s["g_dz"].scatter_add(1, s["idx"].long(), d_logits)
    dw = s["x"].float().T @ dz
    dx = s["dx_in"].float() + s["g_dz"] @ s["w"].T
    return {"d_logits": d_logits, "dw": dw, "dx": dx.to(BF16)}


def _power(e):
    """2^e in fp32 for whole e (the exponent's bits: exact)."""
    return ((e.to(I32) + 127) << 23).view(F32)


def _codes(v):
    """fp32 [..., n] in blocks of 32 [..., n/32, 32]: E4M3 codes, and the block's exponent."""
    b = torch.nn.functional.pad(v, (0, -v.shape[-1] % BLOCK)).unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(b.abs().amax(-1, keepdim=True))      # m in [0.5, 1); 448 = 0.875 * 2^9
    e = (e - 9 + (m > E4M3_MAX / 512)).clamp(min=-126)
    return (b * _power(-e)).to(torch.float8_e4m3fn), e


def _round_8bit(v):
    """fp32 [..., n] through E4M3 with a power-of-two scale per 32 values: the values that come back."""
    q, e = _codes(v)
    return (q.float() * _power(e)).flatten(-2)[..., :v.shape[-1]]


def _tiles(m, n):
    """[R, C] row-major -> the order of the kept pre-activations: blocks of 32 rows (those that are whole),
    in each the rows of n columns after one another."""
    out, C, W = torch.zeros_like(m), m.shape[1], m.shape[0] // 32 * 32
    out[:W] = m[:W].reshape(W // 32, 32, C // n, n).transpose(1, 2).reshape(W, C)
    return out


def _untiled(m, n):
    out, C, W = torch.zeros_like(m), m.shape[1], m.shape[0] // 32 * 32
    out[:W] = m[:W].reshape(W // 32, C // n, 32, n).transpose(1, 2).reshape(W, C)
    return out


def _pack_ab(ab):
    """What the forward keeps of [A|B] (fp32 [R, 2F]): codes and scales, 16 and 1 columns to a tile row."""
    q, e = _codes(ab)
    return (_tiles(q.flatten(-2).view(torch.uint8), 16).contiguous(),
            _tiles((e.squeeze(-1) + 127).to(torch.uint8), 1).contiguous())


def _unpack_ab(q, scale):
    q = _untiled(q, 16).view(torch.float8_e4m3fn).float().unflatten(-1, (-1, BLOCK))
    return (q * _power(_untiled(scale, 1).to(I32) - 127)[:, :, None]).flatten(-2)


def _plain_rows(s):
    c = s["case"]
    x = _round_8bit(s["x"].float()).to(BF16)
    out = torch.zeros(_rows_cap(c), c["d"], dtype=BF16, device=x.device)
    out[s["row"].long().reshape(-1)] = x[:, None, :].expand(-1, c["k"], -1).reshape(-1, c["d"])
    return {"x": x, "x_perm": out}


def _plain_ffn(s):
    F, R, at, live = s["case"]["F"], _rows_cap(s["case"]), s["at"], s["live"][:, :, None]

    def back(v):  # [E, rows, n] -> [R, n], zeros on padding rows and behind the last group
        out = torch.zeros(R + 1, v.shape[2], dtype=BF16, device=v.device)
        out[torch.where(s["live"], at, R).reshape(-1)] = v.to(BF16).flatten(0, 1)
        return out[:R]

    x = torch.where(live, s["x_perm"][at].float(), 0.0)
    wu, wd = s["w_gate_up"].float(), s["w_down"].float()
    if s["case"]["kind"] == "ffn_fwd":
        ab = x @ wu.transpose(1, 2)
        h = ab[..., :F] * torch.sigmoid(ab[..., :F]) * ab[..., F:]
        out = h @ wd.transpose(1, 2)
        ab = _round_8bit(ab)                                 # what the backward has
        h = ab[..., :F] * torch.sigmoid(ab[..., :F]) * ab[..., F:]
        return {"out": back(out), "ab": _tiles(back(ab), 8), "h": back(h)}
    ab = _unpack_ab(s["ab_q"], s["ab_scale"])[at]
    a, b = ab[..., :F], ab[..., F:]
    sg = torch.sigmoid(a)
    h = a * sg * b
    do = torch.where(live, s["d_out"][at].float(), 0.0)
    dh = do @ wd
    share = torch.zeros(R + 1, device=x.device)
    share[torch.where(s["live"], at, R).reshape(-1)] = (dh * h).sum(-1).reshape(-1)
    d_gate = share[s["row"].long()] / s["gate"]
    dab = torch.cat((dh * b * (sg * (1 + a * (1 - sg))), dh * a * sg), -1)
    return {"h": back(h), "d_gate": d_gate, "dx_perm": back(dab @ wu),
            "dw_gate_up": (dab.transpose(1, 2) @ x).to(BF16), "dw_down": (do.transpose(1, 2) @ h).to(BF16)}


def run(s):
    if own:
        return _own(s)
    return {"balance": _plain_balance, "router": _plain_router, "rows": _plain_rows,
            "ffn_fwd": _plain_ffn, "ffn_bwd": _plain_ffn}[s["case"]["kind"]](s)


# ---------------------------------------------------------------- what a pass needs


def work(case):
    """Bytes with every input read once and every output written once, and the operations."""
    c = case
    T, d, E, k, F = c["T"], c["d"], c["E"], c["k"], c["F"]
    A, S = T * k, max(1, c["seqs"])
    if c["kind"] == "balance":   # z, idx, mask, offsets; lse, dz, counts and prob
        return {"bytes": 8 * T * E + 4 * A + 4 * T + (T if c["padded"] else 0) + 8 * S * E, "flops": 12 * T * E}
    if c["kind"] == "router":    # x, dx_in, dx; dz, W, dW; idx, gate, d_gate, d_logits
        return {"bytes": 6 * T * d + 4 * T * E + 8 * d * E + 16 * A, "flops": 4 * T * d * E}
    if c["kind"] == "rows":      # x, codes and scales, x back, the groups' rows; row
        return {"bytes": T * d * 2 + T * d + T * -(-d // BLOCK) + T * d * 2 + A * d * 2 + 4 * A, "flops": 4 * T * d}
    # the weights of experts with rows; the codes and scales of [A|B]
    live, ab = min(E, A), 2 * A * F + 2 * A * F // BLOCK
    if c["kind"] == "ffn_fwd":   # x; out; [A|B] and h read back
        return {"bytes": 6 * live * d * F + 4 * A * d + ab + 6 * A * F, "flops": 6 * A * d * F}
    # x, d_out; dx, h, the weights' gradients; gates
    return {"bytes": 6 * live * d * F + 6 * E * d * F + 6 * A * d + 2 * A * F + ab + 12 * A,
            "flops": 12 * A * d * F}


# ---------------------------------------------------------------- in 64 bits, from the definitions


def _two(e):
    """2^e in 64 bits for whole e."""
    return ((e.long() + 1023) << 52).view(F64)


def _exact_8bit(v):
    """Nearest E4M3 value (ties to the even code) times the block's power of two, in 64 bits."""
    out = torch.zeros_like(v)
    for j in range(0, v.shape[-1], BLOCK):
        b = v[..., j:j + BLOCK]
        most = b.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(most > 0, most, 1.0) / E4M3_MAX))
        e = torch.where(most > E4M3_MAX * _two(e), e + 1, e)   # (where the logarithm rounded)
        e = torch.where(most <= E4M3_MAX * _two(e - 1), e - 1, e)
        y = b * _two(-e)
        step = _two(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(max=8) - 3)
        out[..., j:j + BLOCK] = torch.round(y / step) * step * _two(e)
    return out


def _exact_balance(s):
    c = s["case"]
    T, E, k = c["T"], c["E"], c["k"]
    live = list(range(E)) if s["mask"] is None else torch.nonzero(s["mask"]).flatten().tolist()
    off = [0, T] if s["seq"] is None else s["seq"].tolist()
    S = len(off) - 1
    z, dev = s["z"].double()[:, live], s["z"].device
    ok = torch.ones(T, dtype=torch.bool, device=dev) if s["tokens"] is None else s["tokens"].bool()
    lse = torch.full((T,), -math.inf, dtype=F64, device=dev)
    dz = torch.zeros(T, E, dtype=F64, device=dev)
    counts, prob = torch.zeros(S, E, dtype=I32, device=dev), torch.zeros(S, E, dtype=F64, device=dev)
    inside = [torch.arange(off[i], off[i + 1], device=dev) for i in range(S)]
    inside = [t[ok[t]] for t in inside]
    n = [t.numel() for t in inside]
    seqs, m = max(1, sum(v > 0 for v in n)), max(1, sum(n))
    g0, g1 = s["d_loss"].double().tolist()
    total = torch.zeros(2, dtype=F64, device=dev)
    for i, t in enumerate(inside):
        if not n[i]:
            continue
        lse[t] = torch.logsumexp(z[t], 1)
        p = torch.exp(z[t] - lse[t][:, None])
        counts[i] = torch.bincount(s["idx"][t].flatten().long(), minlength=E).to(I32)
        prob[i, live] = p.mean(0)
        f = counts[i, live].double() * len(live) / (k * n[i])
        total[0] += s["coef"] / seqs * (f * p.mean(0)).sum()
        total[1] += s["z_coef"] / m * (lse[t] ** 2).sum()
        d_prob = g0 * s["coef"] / seqs * f / n[i]
        dp = p * (d_prob - (p * d_prob).sum(1, keepdim=True)) + g1 * 2 * s["z_coef"] / m * lse[t][:, None] * p
        dz[t[:, None], torch.tensor(live, device=dev)] = dp
    many = torch.tensor(n + [sum(n), sum(v > 0 for v in n)], dtype=I32, device=dev)
    return {"loss": total, "counts": counts, "prob": prob, "n_tokens": many, "lse": lse, "dz": dz}


def _exact_router(s):
    g, dg = s["gate"].double(), s["d_gate"].double()
    dl = g * dg - g * (g * dg).sum(1, keepdim=True)
    dz = s["g_dz"].double()
    dx = s["dx_in"].double() + dz @ s["w"].double().T
    for j in range(s["case"]["k"]):
        dz[torch.arange(dz.shape[0], device=dz.device), s["idx"][:, j].long()] += dl[:, j]
    return {"d_logits": dl, "dw": s["x"].double().T @ dz, "dx": dx}


def _exact_rows(s):
    x = _exact_8bit(s["x"].double())
    out = torch.zeros(s["x_perm"].shape, dtype=F64, device=x.device)
    for j in range(s["case"]["k"]):
        out[s["row"][:, j].long()] = x
    return {"x": x, "x_perm": out}


def _exact_ffn(s):
    c = s["case"]
    d, F, R, E, fwd = c["d"], c["F"], _rows_cap(c), c["E"], c["kind"] == "ffn_fwd"

    def zeros(*n):
        return torch.zeros(*n, dtype=F64, device="cuda")

    off, count, h_back = s["off"].tolist(), s["count"].tolist(), zeros(R, F)
    if fwd:
        out, ab = zeros(R, d), zeros(R, 2 * F)
    else:
        dx, share, dwu, dwd = zeros(R, d), zeros(R), zeros(E, 2 * F, d), zeros(E, d, F)
        kept = _unpack_ab(s["ab_q"], s["ab_scale"])
    for e in range(E):
        r = slice(off[e], off[e] + count[e])
        x = s["x_perm"][r].double()
        wg, wu, wd = s["w_gate_up"][e, :F].double(), s["w_gate_up"][e, F:].double(), s["w_down"][e].double()
        if fwd:
            a, b = x @ wg.T, x @ wu.T
            out[r] = (a / (1 + torch.exp(-a)) * b) @ wd.T
            a, b = _exact_8bit(a), _exact_8bit(b)
            ab[r] = torch.cat((a, b), 1)
            h_back[r] = a / (1 + torch.exp(-a)) * b
            continue
        a, b, do = kept[r, :F].double(), kept[r, F:].double(), s["d_out"][r].double()
        sg = 1 / (1 + torch.exp(-a))
        h = a * sg * b
        dh = do @ wd
        da, db = dh * b * (sg + a * sg * (1 - sg)), dh * a * sg
        h_back[r], share[r] = h, (dh * h).sum(1)
        dx[r] = da @ wg + db @ wu
        dwd[e] = do.T @ h
        dwu[e, :F], dwu[e, F:] = da.T @ x, db.T @ x
    if fwd:
        return {"out": out, "ab": _tiles(ab, 8), "h": h_back}
    return {"h": h_back, "d_gate": share[s["row"].long()] / s["gate"].double(), "dx_perm": dx,
            "dw_gate_up": dwu, "dw_down": dwd}


def exact(case, seed):
    if case["kind"].startswith("ffn") and work(case)["flops"] > 8e12:
        return None
    s = prepare(case, seed)
    return {"balance": _exact_balance, "router": _exact_router, "rows": _exact_rows,
            "ffn_fwd": _exact_ffn, "ffn_bwd": _exact_ffn}[case["kind"]](s)
