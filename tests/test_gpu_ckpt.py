"""8-bit activation checkpoints on the GPU: bit-exact packing, the grouped layout, the experts' forward
and backward through them, and whole layer steps with checkpoints and a balance loss."""
import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from paper_2601_14327_gb300 import _lib as L
from paper_2601_14327_gb300 import layer

from gpu_helpers import assert_close, case_inputs, oracle_inputs, to_np, unblock_ab

pytestmark = pytest.mark.gpu

BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


@pytest.fixture(autouse=True)
def _clean_device_error():
    L.moe_device_error(clear=True)
    yield
    assert L.moe_device_error(clear=True) == 0


def _values(rows, cols, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(2 * torch.randn(rows, cols, generator=g))
    return x.to(BF16)


def _pack(x):
    rows, cols = x.shape
    q = torch.full((rows + 1, cols), 0x55, dtype=U8, device="cuda")
    s = torch.full((rows + 1, -(-cols // 32)), 0x55, dtype=U8, device="cuda")
    L.moe_ckpt_pack(x.cuda(), rows, cols, q, s)
    assert (q[rows:] == 0x55).all() and (s[rows:] == 0x55).all()  # nothing behind the last row
    return q[:rows], s[:rows]


def _same(a, b):
    return np.array_equal(np.asarray(a, np.float64), np.asarray(b, np.float64), equal_nan=True)


@pytest.mark.parametrize("rows,cols", [(1, 8), (1, 32), (3, 40), (5, 256), (2, 1000), (37, 2048), (1, 7168), (700, 136),
                                       (1300, 1032), (5000, 512)])
def test_pack_and_unpack_bit_exact(rows, cols):
    x = _values(rows, cols, rows + cols)
    v, s = O.ckpt_round(x.double().numpy())
    q, got_s = _pack(x)
    assert (got_s.cpu().numpy() == s).all()
    out = torch.full((rows + 1, cols), 7.0, dtype=BF16, device="cuda")
    L.moe_ckpt_unpack(q, got_s, rows, cols, out)
    assert _same(out[:rows].double().cpu().numpy(), v) and (out[rows:] == 7).all()
    # packing what was unpacked changes nothing
    q2, s2 = _pack(out[:rows].cpu())
    again = torch.empty(rows, cols, dtype=BF16, device="cuda")
    L.moe_ckpt_unpack(q2, s2, rows, cols, again)
    assert torch.equal(again, out[:rows])


def test_pack_extremes():
    """Zeros, the smallest and largest values, scales at both ends, infinities and NaN (in their block only)."""
    x = torch.zeros(8, 96)
    x[0, 0], x[0, 1], x[0, 40] = 448.0, 17.0, 450.0
    x[1, 3], x[1, 70] = 3.38e38, -1e-38
    x[2, 5], x[2, 33], x[2, 34] = 1e-40, 2.0 ** -133, 2.0 ** -126
    x[3] = torch.linspace(-1, 1, 96)
    x[4, 10] = float("inf")
    x[5, 40], x[5, 41] = float("nan"), 3.0
    x[6, 95] = -float("inf")
    x[7] = 2.0 ** torch.arange(-48.0, 48.0)
    x = x.to(BF16)
    v, s = O.ckpt_round(x.double().numpy())
    q, got_s = _pack(x)
    assert (got_s.cpu().numpy() == s).all()
    out = torch.empty(8, 96, dtype=BF16, device="cuda")
    L.moe_ckpt_unpack(q, got_s, 8, 96, out)
    want = torch.from_numpy(v).to(BF16)  # (values below 2^-133 round to bf16's smallest or to zero)
    assert _same(out.double().cpu().numpy(), want.double().numpy())
    assert torch.isnan(out[4, :32]).all() and torch.isfinite(out[4, 32:]).all()


def _layout(idx, E, rows_cap):
    T, k = idx.shape
    d = 8
    n = L.moe_workspace_size(T, d, E, k, 128)
    ws = torch.empty(n, dtype=U8, device="cuda")
    off, cnt = torch.empty(E + 1, dtype=I32, device="cuda"), torch.empty(E, dtype=I32, device="cuda")
    row, xp = torch.empty(T, k, dtype=I32, device="cuda"), torch.empty(rows_cap, d, dtype=BF16, device="cuda")
    L.moe_permute(torch.zeros(T, d, dtype=BF16, device="cuda"), idx, None, T, d, E, k, rows_cap, off, cnt, row, xp, ws, n)
    return off, cnt, row


def _routing(T, E, k, seed):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(T, E, generator=g) - torch.log1p(torch.arange(E).float())
    return torch.argsort(z, dim=1, descending=True)[:, :k].to(I32).contiguous().cuda()


@pytest.mark.parametrize("T,d,E,k", [(1, 8, 1, 1), (1, 7168, 16, 8), (37, 2048, 64, 6), (151, 264, 5, 3), (700, 72, 128, 4),
                                     (1021, 512, 32, 4), (3000, 40, 256, 8), (4097, 1024, 17, 2)])
def test_ckpt_permute_is_permute_of_the_unpacked_rows(T, d, E, k):
    R = L.moe_perm_rows_max(T, k, E) + 64
    idx = _routing(T, E, k, T)
    off, cnt, row = _layout(idx, E, R)
    x = _values(T, d, T + d)
    q, s = _pack(x)
    plain = torch.empty(T, d, dtype=BF16, device="cuda")
    L.moe_ckpt_unpack(q, s, T, d, plain)
    n = L.moe_workspace_size(T, d, E, k, 128)
    want = torch.full((R, d), 9.0, dtype=BF16, device="cuda")
    L.moe_permute(plain, idx, None, T, d, E, k, R, off, cnt, row, want, torch.empty(n, dtype=U8, device="cuda"), n)
    got, back = torch.full((R, d), 9.0, dtype=BF16, device="cuda"), torch.empty(T, d, dtype=BF16, device="cuda")
    L.moe_ckpt_permute(q, s, row, off, cnt, T, d, E, k, R, back, got)
    assert torch.equal(got, want) and torch.equal(back, plain)
    assert (got[int(off[E]):] == 9).all()
    # without x; an assignment whose row is out of range is left out
    row[0, 0] = R
    got2 = torch.full((R, d), 9.0, dtype=BF16, device="cuda")
    L.moe_ckpt_permute(q, s, row, off, cnt, T, d, E, k, R, None, got2)
    same = (got2 == got).all(dim=1)
    assert (~same).sum() <= 1


FFN = [(40, 128, 4, 2, 128), (1021, 512, 32, 4, 384), (300, 256, 16, 8, 256), (1500, 384, 12, 4, 640),
       # CTA pairs with 256 and 128 columns, an odd number of row blocks
       (6000, 256, 4, 2, 256), (3000, 640, 3, 2, 896), (4100, 2048, 8, 4, 1408),
       # 2^18 rows and more: a group's odd last block goes to the other kernel
       (66000, 128, 5, 4, 128)]


class Ffn:
    def __init__(self, T, d, E, k, F, seed=0):
        self.T, self.d, self.E, self.k, self.F = T, d, E, k, F
        self.R = R = L.moe_perm_rows_max(T, k, E)
        g = torch.Generator(device="cuda").manual_seed(seed + T)
        self.idx = _routing(T, E, k, seed + T)
        self.gate = torch.softmax(torch.randn(T, k, generator=g, device="cuda"), 1)
        self.off, self.cnt, self.row = _layout(self.idx, E, R)
        self.used = int(self.off[E])
        self.live = torch.zeros(R, dtype=torch.bool, device="cuda")
        self.live[self.row.reshape(-1).long()] = True

        def rows(n):
            v = torch.zeros(R, n, dtype=BF16, device="cuda")
            v[self.live] = torch.randn(T * k, n, generator=g, device="cuda").to(BF16)
            return v

        self.x, self.dout = rows(d), rows(d)
        self.wu = (0.05 * torch.randn(E, 2 * F, d, generator=g, device="cuda")).to(BF16)
        self.wd = (0.05 * torch.randn(E, d, F, generator=g, device="cuda")).to(BF16)
        self.wr = torch.randn(d, E, generator=g, device="cuda") / d ** 0.5
        self.n = L.moe_workspace_size(T, d, E, k, F)
        self.ws = torch.empty(self.n, dtype=U8, device="cuda")

    def buf(self, cols, dtype=BF16, fill=3.0):
        return torch.full((self.R, cols), fill, dtype=dtype, device="cuda")

    def forward(self):
        q, s = self.buf(2 * self.F, U8, 0x55), self.buf(2 * self.F // 32, U8, 0x55)
        h, out = self.buf(self.F), self.buf(self.d)
        L.moe_grouped_ffn_fwd_ckpt(self.x, self.off, self.E, self.d, self.F, self.R, self.wu, self.wd, q, s, h, out,
                                   self.ws, self.n)
        return q, s, h, out


def _decode(q, s, F):
    """Values and scales of the kept [A|B], [rows, 2F] and [rows, 2F/32], from the documented layout."""
    R = q.shape[0] // 32 * 32
    v = q[:R].reshape(R // 32, 2 * F // 16, 32, 16).transpose(1, 2).reshape(R, 2 * F).contiguous().view(torch.float8_e4m3fn)
    sc = s[:R].reshape(R // 32, 2 * F // 32, 32).transpose(1, 2).reshape(R, 2 * F // 32)
    scale = torch.exp2(sc.double() - 127)
    return v.double() * scale.repeat_interleave(32, dim=1), scale


@pytest.mark.parametrize("T,d,E,k,F", FFN)
def test_ffn_forward_keeps_8_bits(T, d, E, k, F):
    f = Ffn(T, d, E, k, F)
    q, s, h, out = f.forward()
    ab, h0, out0 = f.buf(2 * F), f.buf(F), f.buf(d)
    L.moe_grouped_ffn_fwd(f.x, f.off, E, d, F, f.R, f.wu, f.wd, ab, h0, out0, f.ws, f.n)
    assert torch.equal(h, h0) and torch.equal(out, out0)
    assert (q[f.used:] == 0x55).all() and (s[f.used:] == 0x55).all()
    got, scale = _decode(q, s, F)
    off = f.off.tolist()
    for e in range(E):
        r = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            continue
        x, w = f.x[r].double(), f.wu[e].double()
        ref, size = x @ w.T, x.abs() @ w.abs().T
        sc = scale[r].repeat_interleave(32, dim=1)
        # half a step of the code: 2^-4 of the value, or 2^-10 scales; the fp32 accumulation before it
        # (tensor-core sums: d * 2^-23 of the absolute products)
        bound = torch.maximum(ref.abs() * 2 ** -4, sc * 2 ** -10) + (1 + 2 ** -4) * size * d * 2 ** -23
        assert ((got[r] - ref).abs() <= bound + 1e-37).all()
        # the scale: the smallest that holds the block's largest value, but for that accumulation
        amax = ref.abs().reshape(ref.shape[0], -1, 32).amax(2)
        eps = size.reshape(ref.shape[0], -1, 32).amax(2) * d * 2 ** -23
        assert (amax - eps <= 448 * scale[r]).all()
        assert ((amax + eps >= 224 * scale[r]) | (scale[r] == 2.0 ** -126)).all()


@pytest.mark.parametrize("T,d,E,k,F", FFN)
def test_unpack_ab_reads_what_was_kept(T, d, E, k, F):
    f = Ffn(T, d, E, k, F)
    q, s, _, _ = f.forward()
    ab, h = f.buf(2 * F), f.buf(F)
    L.moe_ckpt_unpack_ab(q, s, f.off, E, F, f.R, ab, h)
    want, _ = _decode(q, s, F)
    got = torch.from_numpy(unblock_ab(to_np(ab), F)[:f.used]).double().cuda()
    assert torch.equal(got, want[:f.used])
    a, b = want[:f.used, :F], want[:f.used, F:]
    ref = a * torch.sigmoid(a) * b
    # sigmoid: exp and the quick divide, 2 ulp each, then the rounding to bf16
    assert ((h[:f.used].double() - ref).abs() <= (2 ** -8 + 2 ** -20) * ref.abs() + 1e-37).all()
    assert (ab.reshape(-1)[f.used * 2 * F:] == 3).all() and (h[f.used:] == 3).all()
    only = f.buf(F)
    L.moe_ckpt_unpack_ab(q, s, f.off, E, F, f.R, None, only)
    assert torch.equal(only, h)


@pytest.mark.parametrize("router", [False, True])
@pytest.mark.parametrize("T,d,E,k,F", FFN)
def test_ffn_backward_from_8_bits(T, d, E, k, F, router):
    """Bit for bit the plain backward on the unpacked pre-activations, which other tests hold to the oracle."""
    f = Ffn(T, d, E, k, F)
    q, s, _, _ = f.forward()
    ab, h = f.buf(2 * F), f.buf(F)
    L.moe_ckpt_unpack_ab(q, s, f.off, E, F, f.R, ab, h)
    wr = f.wr if router else None
    dg = [torch.full((T, k), 5.0, device="cuda") for _ in range(2)]
    dab, dx, h8 = [f.buf(2 * F) for _ in range(2)], [f.buf(d) for _ in range(2)], f.buf(F)
    L.moe_grouped_ffn_bwd_dgrad(f.dout, ab, f.off, E, d, F, f.R, f.wu, f.wd, f.gate, None, f.row, wr, T, k, dg[0],
                                dab[0], dx[0], f.ws, f.n)
    f.ws.fill_(255)
    L.moe_grouped_ffn_bwd_dgrad_ckpt(f.dout, q, s, f.off, E, d, F, f.R, f.wu, f.wd, f.gate, None, f.row, wr, T, k, dg[1],
                                     h8, dab[1], dx[1], f.ws, f.n)
    assert torch.equal(dab[0], dab[1]) and torch.equal(dx[0], dx[1]) and torch.equal(dg[0], dg[1])
    assert torch.equal(h8, h)  # (rows behind the last group as they were)
    # and against 64 bits: d_gate, from the definition
    if not router:
        v, _ = _decode(q, s, F)
        share, size = torch.zeros(f.R, dtype=torch.float64, device="cuda"), torch.zeros(f.R, dtype=torch.float64, device="cuda")
        off = f.off.tolist()
        for e in range(E):
            r = slice(off[e], off[e + 1])
            a, b = v[r, :F], v[r, F:]
            hh = a * torch.sigmoid(a) * b
            share[r] = ((f.dout[r].double() @ f.wd[e].double()) * hh).sum(1)
            size[r] = ((f.dout[r].double().abs() @ f.wd[e].double().abs()) * hh.abs()).sum(1)
        ref = share[f.row.long()] / f.gate.double()
        # fp32 accumulation over d and F (tensor cores: d * 2^-23), sigmoid 4 ulp
        bound = size[f.row.long()] / f.gate.double() * (d * 2 ** -23 + F * 2 ** -24 + 2 ** -20)
        assert ((dg[1].double() - ref).abs() <= bound + 1e-30).all()


def test_ffn_ckpt_zero_and_infinite_rows():
    """A zero row keeps zeros; a row whose products overflow reads back as NaN, and no other row does."""
    f = Ffn(200, 256, 4, 2, 128)
    r0, r1 = int(f.row[3, 0]), int(f.row[5, 1])
    f.x[r0] = 0
    f.x[r1] = 3e38
    q, s, _, out = f.forward()
    v, _ = _decode(q, s, 128)
    assert (v[r0] == 0).all() and torch.isnan(v[r1]).any()
    keep = [r for r in range(f.used) if r != r1]
    assert torch.isfinite(v[keep]).all()


# ---------------------------------------------------------------- whole layer steps


def _layer_inputs(T, d, E, k, F, masked, seed=3):
    inp = case_inputs(T, d, E, k, F, seed=seed)
    o = oracle_inputs(inp)
    mask = None
    if masked:
        mask = np.ones(E, np.uint8)
        mask[np.argsort(o["bias"], kind="stable")[:masked]] = 0
    z = O.apply_mask(O.router_logits(o["x"], o["w_router"], o["bias"]), mask)
    return inp, o, mask, z


def _step(b, g, mask, z, balance=None, d_loss=None, ckpt=None, overlap=False):
    layer.forward(b, g["x"], g["w_router"], g["bias"], g["w_gate_up"], g["w_down"], mask, z, balance=balance, ckpt=ckpt)
    return layer.backward(b, g["dy"], g["w_router"], g["w_gate_up"], g["w_down"], active_mask=mask, d_loss=d_loss,
                          ckpt=ckpt, overlap=overlap)


@pytest.mark.parametrize("overlap", [False, True])
@pytest.mark.parametrize("T,d,E,k,F,masked", [(300, 256, 8, 2, 256, 0), (1021, 512, 32, 4, 384, 6), (77, 128, 16, 3, 128, 2)])
def test_layer_with_balance_loss_against_oracle(T, d, E, k, F, masked, overlap):
    """The layer's gradients with the auxiliary losses: the oracle's layer gradients plus the losses'."""
    inp, o, mask, z = _layer_inputs(T, d, E, k, F, masked)
    g = {n: v.cuda() for n, v in inp.items()}
    m = None if mask is None else torch.from_numpy(mask).cuda()
    off = torch.tensor([0, T // 3, T // 3, T - 5], dtype=I32, device="cuda")
    tok = (torch.arange(T, device="cuda") % 7 != 0).to(U8)
    b = layer.MoELayerBuffers(layer.LayerShape(T, d, E, k, F), "cuda", balance_seqs=4)
    # a large coefficient, so that the losses are a good part of the router's gradient
    bal, dl = layer.BalanceLoss(50.0 * T, 0.5 * T, tok, off), torch.tensor([0.8, 1.2], device="cuda")
    dx, dgu, ddn, dr = _step(b, g, m, torch.from_numpy(z).cuda(), bal, dl, overlap=overlap)
    ref = O.moe_layer(o["x"], o["w_router"], o["bias"], mask, k, o["w_gate_up"], o["w_down"], dy=o["dy"], logits32=z)
    aux = O.balance_loss(z, ref["topk_idx"], mask, tok.cpu().numpy(), off.cpu().numpy(), 50.0 * T, 0.5 * T, (0.8, 1.2))
    np.testing.assert_allclose(b.loss.cpu().numpy(), aux["loss"], rtol=1.2e-5)
    assert (b.balance_counts[:3].cpu().numpy() == aux["counts"]).all()
    assert_close("dx", to_np(dx), ref["dx"] + aux["dz"] @ o["w_router"].T)
    assert_close("dw_router", to_np(dr), ref["dw_router"] + o["x"].T @ aux["dz"])
    assert np.abs(o["x"].T @ aux["dz"]).max() > 0.1 * np.abs(ref["dw_router"]).max()
    live = np.ones(E, bool) if mask is None else mask != 0
    assert_close("dw_gate_up", to_np(dgu)[live], ref["dw_gate_up"][live])
    assert_close("dw_down", to_np(ddn)[live], ref["dw_down"][live])
    # a step without the losses through the same buffers: as if they had never been there
    plain = layer.MoELayerBuffers(layer.LayerShape(T, d, E, k, F), "cuda")
    for got, want in zip(_step(b, g, m, torch.from_numpy(z).cuda()), _step(plain, g, m, torch.from_numpy(z).cuda())):
        if got.shape[0] == E and got.dim() == 3:
            got, want = got[torch.from_numpy(live).cuda()], want[torch.from_numpy(live).cuda()]
        assert torch.equal(got, want)


def _oracle_from_8_bits(o, z, ref, mask, k, c, F, row):
    """The layer's backward in 64 bits from what the checkpoint holds: x and [A|B] as unpacked."""
    x8, _ = O.ckpt_round(o["x"])
    ab = _decode(c.ab_q, c.ab_scale, F)[0].cpu().numpy()
    T, d = o["x"].shape
    E = o["w_router"].shape[1]
    idx, gate = ref["topk_idx"], ref["topk_gate"] if "topk_gate" in ref else None
    if gate is None:
        _, gate = O.route_topk(z, k)
    gate = np.asarray(gate, np.float64)
    dwu, dwd = np.zeros((E, 2 * F, d)), np.zeros((E, d, F))
    dxa, dgate = np.zeros((T, d)), np.zeros((T, k))
    for e in range(E):
        t, j = np.nonzero(idx == e)
        r = row[t, j]
        a, b = ab[r, :F], ab[r, F:]
        sg = 1 / (1 + np.exp(-a))
        h = a * sg * b
        do = gate[t, j][:, None] * o["dy"][t]
        dh = do @ o["w_down"][e]
        dgate[t, j] = (o["dy"][t] @ o["w_down"][e] * h).sum(1)
        dab = np.concatenate([dh * b * (sg * (1 + a * (1 - sg))), dh * a * sg], 1)
        dwu[e], dwd[e] = dab.T @ x8[t], do.T @ h
        np.add.at(dxa, t, dab @ o["w_gate_up"][e])
    dl, dwr = O.router_backward(x8, idx, gate, dgate, E)
    for j in range(k):
        dxa += dl[:, j:j + 1] * o["w_router"].T[idx[:, j]]
    return dxa, dwu, dwd, dwr, x8


@pytest.mark.parametrize("overlap", [False, True])
@pytest.mark.parametrize("T,d,E,k,F,masked", [(300, 256, 8, 2, 256, 0), (1021, 512, 32, 4, 384, 6), (1, 128, 4, 2, 128, 0)])
def test_layers_share_buffers_through_checkpoints(T, d, E, k, F, masked, overlap):
    """Two layers forward and then backward through one set of buffers, each with its checkpoint: gradients
    as the oracle computes them from what the checkpoints hold."""
    b = layer.MoELayerBuffers(layer.LayerShape(T, d, E, k, F), "cuda", balance_seqs=1, ckpt=True)
    layers = []
    for seed in (3, 4):
        inp, o, mask, z = _layer_inputs(T, d, E, k, F, masked, seed)
        g = {n: v.cuda() for n, v in inp.items()}
        m = None if mask is None else torch.from_numpy(mask).cuda()
        c = layer.MoECheckpoint(b.shape, "cuda", balance_seqs=1)
        bal = layer.BalanceLoss(20.0 * T, 0.1 * T) if seed == 4 else None
        y = layer.forward(b, g["x"], g["w_router"], g["bias"], g["w_gate_up"], g["w_down"], m, torch.from_numpy(z).cuda(),
                          balance=bal, ckpt=c)
        ref = O.moe_layer(o["x"], o["w_router"], o["bias"], mask, k, o["w_gate_up"], o["w_down"], dy=o["dy"], logits32=z)
        assert_close("y", to_np(y), ref["y"])
        layers.append((o, mask, z, g, m, c, bal, ref))
    for o, mask, z, g, m, c, bal, ref in reversed(layers):
        dx, dgu, ddn, dr = layer.backward(b, g["dy"], g["w_router"], g["w_gate_up"], g["w_down"], active_mask=m, ckpt=c,
                                          overlap=overlap)
        torch.cuda.synchronize()
        row = c.row_of_assignment.cpu().numpy()
        rdx, rdu, rdd, rdr, x8 = _oracle_from_8_bits(o, z, ref, mask, k, c, F, row)
        if bal is not None:
            aux = O.balance_loss(z, ref["topk_idx"], mask, None, None, bal.coef, bal.z_coef)
            rdx, rdr = rdx + aux["dz"] @ o["w_router"].T, rdr + x8.T @ aux["dz"]
        live = np.ones(E, bool) if mask is None else mask != 0
        assert_close("dx", to_np(dx), rdx)
        assert_close("dw_router", to_np(dr), rdr)
        assert_close("dw_gate_up", to_np(dgu)[live], rdu[live])
        assert_close("dw_down", to_np(ddn)[live], rdd[live])


def test_layer_without_tokens_with_checkpoint_and_balance():
    s = layer.LayerShape(0, 128, 4, 2, 128)
    b, c = layer.MoELayerBuffers(s, "cuda", balance_seqs=1, ckpt=True), layer.MoECheckpoint(s, "cuda", balance_seqs=1)
    e = torch.empty(0, 128, dtype=BF16, device="cuda")
    wr, wu = torch.zeros(128, 4, device="cuda"), torch.zeros(4, 256, 128, dtype=BF16, device="cuda")
    wd = torch.zeros(4, 128, 128, dtype=BF16, device="cuda")
    layer.forward(b, e, wr, None, wu, wd, balance=layer.BalanceLoss(1.0, 1.0), ckpt=c)
    dx, dgu, ddn, dr = layer.backward(b, e, wr, wu, wd, ckpt=c)
    assert (c.loss == 0).all() and (dgu == 0).all() and (ddn == 0).all() and (dr == 0).all() and dx.shape == (0, 128)


def test_graph_of_a_checkpointed_step_replays():
    """Forward and backward of a layer with checkpoint and balance loss, captured once, on new inputs."""
    T, d, E, k, F = 600, 256, 16, 4, 256
    s = layer.LayerShape(T, d, E, k, F)
    sets = []
    for seed in (5, 6):
        inp, o, mask, z = _layer_inputs(T, d, E, k, F, 0, seed)
        sets.append({n: v.cuda() for n, v in inp.items()})
    bal = layer.BalanceLoss(10.0, 0.1)
    eager_b, eager_c = layer.MoELayerBuffers(s, "cuda", balance_seqs=1, ckpt=True), layer.MoECheckpoint(s, "cuda", 1)
    want = []
    for g in sets:
        want.append([t.clone() for t in _step(eager_b, g, None, None, bal, None, eager_c)] + [eager_c.loss.clone()])
    b, c = layer.MoELayerBuffers(s, "cuda", balance_seqs=1, ckpt=True), layer.MoECheckpoint(s, "cuda", 1)
    g = {n: v.clone() for n, v in sets[0].items()}
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        _step(b, g, None, None, bal, None, c)
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = _step(b, g, None, None, bal, None, c)
    for i in (1, 0):
        for n, v in sets[i].items():
            g[n].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for got, ref in zip(list(out) + [c.loss], want[i]):
            assert torch.equal(got, ref)


def test_offsets_past_32_bits():
    """More than 2^31 codes in rows and in the kept [A|B]: the last rows are as a small call has them."""
    g = torch.Generator(device="cuda").manual_seed(7)
    rows, cols = 263000, 8200
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    tail = torch.randn(40, cols, generator=g, device="cuda").to(BF16)
    x[-40:] = tail
    q, s = torch.empty(rows, cols, dtype=U8, device="cuda"), torch.empty(rows, -(-cols // 32), dtype=U8, device="cuda")
    L.moe_ckpt_pack(x, rows, cols, q, s)
    q2, s2 = _pack(tail.cpu())
    assert rows * cols > 2 ** 31 and torch.equal(q[-40:], q2) and torch.equal(s[-40:], s2)
    x.fill_(7)
    L.moe_ckpt_unpack(q, s, rows, cols, x)
    assert _same(x[-40:].double().cpu().numpy(), O.ckpt_round(tail.double().cpu().numpy())[0])
    assert (x[:-40:997] == 0).all()
    del x, q, s
    # the experts: one group of 263,040 rows, the last 128 of which hold values; 8,192 columns of [A|B]
    d, E, F, R = 128, 1, 4096, 263040
    xp = torch.zeros(R, d, dtype=BF16, device="cuda")
    xp[-128:] = torch.randn(128, d, generator=g, device="cuda").to(BF16)
    wu = (0.1 * torch.randn(E, 2 * F, d, generator=g, device="cuda")).to(BF16)
    wd = (0.1 * torch.randn(E, d, F, generator=g, device="cuda")).to(BF16)
    ws = torch.empty(256, dtype=U8, device="cuda")

    def run(xs):
        n = xs.shape[0]
        off = torch.tensor([0, n], dtype=I32, device="cuda")
        q, s = torch.empty(n, 2 * F, dtype=U8, device="cuda"), torch.empty(n, 2 * F // 32, dtype=U8, device="cuda")
        h, out = torch.empty(n, F, dtype=BF16, device="cuda"), torch.empty(n, d, dtype=BF16, device="cuda")
        L.moe_grouped_ffn_fwd_ckpt(xs, off, E, d, F, n, wu, wd, q, s, h, out, ws, 256)
        h8, dab, dx = torch.empty_like(h), torch.empty(n, 2 * F, dtype=BF16, device="cuda"), torch.empty_like(out)
        L.moe_grouped_ffn_bwd_dgrad_ckpt(xs, q, s, off, E, d, F, n, wu, wd, None, None, None, None, 0, 1, None, h8, dab,
                                         dx, ws, 256)
        ab = torch.empty(n, 2 * F, dtype=BF16, device="cuda")
        L.moe_ckpt_unpack_ab(q, s, off, E, F, n, ab, None)
        return [t[-128:].clone() for t in (q, s, h, out, h8, dab, dx, ab)]

    assert R * 2 * F > 2 ** 31
    for a, b in zip(run(xp), run(xp[-128:].contiguous())):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T,d,E,k", [(37, 2048, 64, 6), (700, 72, 16, 4)])
def test_ckpt_permute_leaves_out_rows_out_of_range(T, d, E, k):
    """Entries outside [0, rows_cap): their rows stay as they were, and so does what lies before and behind x_perm."""
    R, rim = L.moe_perm_rows_max(T, k, E), 40
    idx = _routing(T, E, k, T)
    off, cnt, row = _layout(idx, E, R)
    q, s = _pack(_values(T, d, T + d))

    def run(r):
        whole = torch.full((rim + R + rim, d), 9.0, dtype=BF16, device="cuda")
        L.moe_ckpt_permute(q, s, r, off, cnt, T, d, E, k, R, None, whole[rim:rim + R])
        return whole

    want, bad = run(row), row.clone()
    dropped = []
    for i, (t, j) in enumerate([(0, 0), (T - 1, k - 1), (T // 2, 1), (3, 2), (5, 0)]):
        dropped.append(rim + int(row[t, j]))
        bad[t, j] = (R, -1, R + rim - 1, -rim, R + 1)[i]
    got = run(bad)
    differ = (got != want).any(dim=1).nonzero().flatten().tolist()
    assert differ == sorted(dropped)
    assert (got[dropped] == 9).all() and (got[:rim] == 9).all() and (got[rim + R:] == 9).all()


@pytest.mark.parametrize("kw", [{"gather": True}, {"fused_combine": True}])
@pytest.mark.parametrize("T,d,E,k,F,masked", [(300, 256, 8, 2, 256, 0), (1021, 512, 32, 4, 384, 6)])
def test_balance_loss_in_the_other_forms_of_the_layer(T, d, E, k, F, masked, kw):
    """Gathered dispatch and fused combine with a balance loss: losses and gradients of the default form, bit for bit
    (y too, but for the order of the fused combine's sums)."""
    inp, o, mask, z = _layer_inputs(T, d, E, k, F, masked)
    g = {n: v.cuda() for n, v in inp.items()}
    m = None if mask is None else torch.from_numpy(mask).cuda()
    off = torch.tensor([0, T // 3, T - 5], dtype=I32, device="cuda")
    got = []
    for form in ({}, kw):
        b = layer.MoELayerBuffers(layer.LayerShape(T, d, E, k, F), "cuda", balance_seqs=2, **form)
        b.dw_gate_up.zero_()
        b.dw_down.zero_()
        out = _step(b, g, m, torch.from_numpy(z).cuda(), layer.BalanceLoss(20.0 * T, 0.3 * T, seq_offsets=off))
        got.append([t.clone() for t in out] + [b.loss, b.balance_counts, b.balance_prob, b.y.clone()])
    for n, (u, v) in enumerate(zip(*got)):
        if n == 7 and "fused_combine" in kw:
            assert_close("y", to_np(v), to_np(u))
        else:
            assert torch.equal(u, v), n


def test_kept_logits_beside_a_checkpoint():
    """keep_logits with a checkpoint and a balance loss: the same logits in the buffers, and the same step."""
    T, d, E, k, F = 333, 128, 12, 3, 128
    inp, o, mask, z = _layer_inputs(T, d, E, k, F, 2)
    g, m = {n: v.cuda() for n, v in inp.items()}, torch.from_numpy(mask).cuda()
    s = layer.LayerShape(T, d, E, k, F)
    got = []
    for keep in (False, True):
        b, c = layer.MoELayerBuffers(s, "cuda", balance_seqs=1, ckpt=True), layer.MoECheckpoint(s, "cuda", 1)
        b.logits.fill_(7.0)
        y = layer.forward(b, g["x"], g["w_router"], g["bias"], g["w_gate_up"], g["w_down"], m, keep_logits=keep,
                          balance=layer.BalanceLoss(0.3, 0.1), ckpt=c)
        got.append([y, c.loss, c.topk_idx, c.topk_gate, c.counts, c.logits])
        assert torch.equal(b.logits, c.logits) if keep else (b.logits == 7).all()
    for u, v in zip(*got):
        assert torch.equal(u, v)
