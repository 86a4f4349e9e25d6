"""8-bit checkpoints without a GPU: the oracle's rounding, and the refusals of the entry points and of
the layer (nothing is launched)."""
import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from paper_2601_14327_gb300 import _lib as L
from paper_2601_14327_gb300 import build as B
from paper_2601_14327_gb300 import layer


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()


def test_oracle_rounding_is_the_nearest_code():
    """Against every finite E4M3 value: none is nearer, and at equal distance the even code won."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 100)) * np.exp(3 * rng.standard_normal((40, 100)))
    v, s = O.ckpt_round(x)
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert codes[-1] == 448
    for r in range(40):
        for b in range(4):
            j = slice(32 * b, min(32 * b + 32, 100))
            scale = 2.0 ** (int(s[r, b]) - 127)
            assert np.abs(x[r, j]).max() <= 448 * scale < 2 * np.abs(x[r, j]).max() * (1 + 1e-15)
            d = np.abs(np.abs(x[r, j])[:, None] / scale - codes)
            assert (np.abs(x[r, j] - v[r, j]) / scale <= d.min(axis=1)).all()
    # ties: 17 lies between 16 and 18, 19 between 18 and 20 (448 sets the scale to one)
    t = np.zeros((1, 32))
    t[0, :6] = 448, 17, 19, -17, 2.0 ** -10, 3 * 2.0 ** -10
    v, s = O.ckpt_round(t)
    assert s[0, 0] == 127 and v[0, :6].tolist() == [448, 16, 20, -16, 0, 2.0 ** -8]


@pytest.mark.parametrize("amax,s", [(448.0, 127), (449.0, 128), (1.75, 119), (1.7578125, 120), (1.0, 119), (0.0, 1),
                                    (2.0 ** -130, 1), (3.3e38, 247), (float("inf"), 255), (float("nan"), 255)])
def test_oracle_scale(amax, s):
    x = np.zeros((1, 32))
    x[0, 5] = -amax
    v, got = O.ckpt_round(x)
    assert got[0, 0] == s and (np.isnan(v).all() if s == 255 else np.isfinite(v).all())


def _pack(**kw):
    a = dict(x=16, rows=10, cols=64, q=16, scale=1)
    a.update(kw)
    L.moe_ckpt_pack(*a.values(), stream=0)


def _unpack(**kw):
    a = dict(q=16, scale=1, rows=10, cols=64, x=16)
    a.update(kw)
    L.moe_ckpt_unpack(*a.values(), stream=0)


def _permute(**kw):
    a = dict(q=16, scale=1, row=16, off=16, cnt=16, T=10, d=64, E=8, k=2, rows_cap=10 * 2 + 8 * 128, x=None, x_perm=16)
    a.update(kw)
    L.moe_ckpt_permute(*a.values(), stream=0)


def _unpack_ab(**kw):
    a = dict(q=16, scale=16, off=16, E=8, F=128, rows_cap=4096, ab=16, h=16)
    a.update(kw)
    L.moe_ckpt_unpack_ab(*a.values(), stream=0)


@pytest.mark.parametrize("call,bad,status", [
    (_pack, {"cols": 12}, -1), (_pack, {"cols": 0}, -1), (_pack, {"rows": -1}, -1), (_pack, {"rows": 1 << 31}, -1),
    (_pack, {"x": None}, -1), (_pack, {"x": 24}, -1), (_pack, {"q": 12}, -1), (_pack, {"q": None}, -1),
    (_pack, {"scale": None}, -1),
    (_unpack, {"cols": 4}, -1), (_unpack, {"rows": -5}, -1), (_unpack, {"x": 8}, -1), (_unpack, {"q": 4}, -1),
    (_unpack, {"scale": None}, -1), (_unpack, {"x": None}, -1),
    (_permute, {"E": 257}, -1), (_permute, {"k": 9}, -1), (_permute, {"d": 12}, -1), (_permute, {"T": -1}, -1),
    (_permute, {"rows_cap": 100}, -1), (_permute, {"rows_cap": 1 << 31}, -2), (_permute, {"x_perm": None}, -1),
    (_permute, {"x": 24}, -1), (_permute, {"q": 4}, -1), (_permute, {"row": None}, -1), (_permute, {"cnt": None}, -1),
    (_unpack_ab, {"F": 64}, -1), (_unpack_ab, {"E": 0}, -1), (_unpack_ab, {"rows_cap": 64}, -1),
    (_unpack_ab, {"ab": None, "h": None}, -1), (_unpack_ab, {"ab": 24}, -1), (_unpack_ab, {"h": 8}, -1),
    (_unpack_ab, {"q": 8}, -1), (_unpack_ab, {"scale": 8}, -1), (_unpack_ab, {"off": None}, -1)])
def test_ckpt_refusals(call, bad, status):
    with pytest.raises(L.MoEError) as e:
        call(**bad)
    assert e.value.status == status


def test_ckpt_calls_without_rows_do_nothing():
    _pack(rows=0, x=None, q=None, scale=None)
    _unpack(rows=0, x=None, q=None, scale=None)
    _permute(T=0, q=None, scale=None, row=None, x_perm=None)


def _fwd(**kw):
    a = dict(x=16, off=16, E=8, d=256, F=256, rows_cap=4096, wu=16, wd=16, q=16, scale=16, h=16, out=16, ws=16,
             ws_bytes=256)
    a.update(kw)
    L.moe_grouped_ffn_fwd_ckpt(*a.values(), stream=0)


def _dgrad(**kw):
    a = dict(dout=16, q=16, scale=16, off=16, E=8, d=256, F=256, rows_cap=4096, wu=16, wd=16, gate=None, d_gate=None,
             row=None, w=None, T=0, k=1, dg_out=None, h=16, d_ab=16, dx=16, ws=16, ws_bytes=256)
    a.update(kw)
    L.moe_grouped_ffn_bwd_dgrad_ckpt(*a.values(), stream=0)


@pytest.mark.parametrize("call,bad,status", [
    (_fwd, {"d": 100}, -2), (_fwd, {"F": 64}, -2), (_fwd, {"E": 300}, -2), (_fwd, {"q": None}, -1), (_fwd, {"q": 24}, -1),
    (_fwd, {"scale": None}, -1), (_fwd, {"scale": 8}, -1), (_fwd, {"h": None}, -1), (_fwd, {"ws_bytes": 128}, -6),
    (_fwd, {"rows_cap": 64}, -1),
    (_dgrad, {"d": 100}, -2), (_dgrad, {"q": None}, -1), (_dgrad, {"scale": None}, -1), (_dgrad, {"h": None}, -1),
    (_dgrad, {"h": 8}, -1), (_dgrad, {"ws": None}, -6), (_dgrad, {"d_gate": 16}, -1), (_dgrad, {"gate": 16}, -1),
    (_dgrad, {"dg_out": 16, "T": 10, "k": 2, "ws_bytes": 1 << 24}, -1), (_dgrad, {"rows_cap": 10}, -1)])
def test_ffn_ckpt_refusals(call, bad, status):
    with pytest.raises(L.MoEError) as e:
        call(**bad)
    assert e.value.status == status


def test_layer_refuses_mixed_buffers():
    s = layer.LayerShape(8, 128, 4, 2, 128)
    for kw in ({"gather": True}, {"fused_combine": True}):
        with pytest.raises(ValueError):
            layer.MoELayerBuffers(s, "cpu", ckpt=True, **kw)
    with pytest.raises(ValueError):
        layer.MoECheckpoint(layer.LayerShape(8, 136, 4, 2, 128), "cpu")
    plain, shared = layer.MoELayerBuffers(s, "cpu"), layer.MoELayerBuffers(s, "cpu", ckpt=True)
    c = layer.MoECheckpoint(s, "cpu")
    other = layer.MoECheckpoint(layer.LayerShape(9, 128, 4, 2, 128), "cpu")
    for b, ckpt in ((plain, c), (shared, None), (shared, other)):
        with pytest.raises(ValueError):
            layer.forward(b, None, None, None, None, None, ckpt=ckpt)
        with pytest.raises(ValueError):
            layer.backward(b, None, None, None, None, ckpt=ckpt)
    off = torch.zeros(4, dtype=torch.int32)
    for b, ckpt in ((plain, None), (layer.MoELayerBuffers(s, "cpu", balance_seqs=2), None),
                    (layer.MoELayerBuffers(s, "cpu", balance_seqs=3, ckpt=True), c)):
        with pytest.raises(ValueError):  # three sequences
            layer.forward(b, None, None, None, None, None, balance=layer.BalanceLoss(0.1, seq_offsets=off), ckpt=ckpt)
    b = layer.MoELayerBuffers(s, "cpu", balance_seqs=3)
    for bad in ({"seq_offsets": off.long()}, {"seq_offsets": torch.zeros(8, dtype=torch.int32)[::2]},
                {"seq_offsets": off[:1]}, {"token_mask": torch.ones(8)}, {"token_mask": torch.ones(7, dtype=torch.uint8)}):
        with pytest.raises(ValueError):
            layer.forward(b, None, None, None, None, None, balance=layer.BalanceLoss(0.1, **bad))


def test_layer_refuses_tensors_of_another_device_and_other_d_loss():
    s = layer.LayerShape(8, 128, 4, 2, 128)
    b = layer.MoELayerBuffers(s, "cpu", balance_seqs=1)
    for bad in ({"seq_offsets": torch.empty(2, dtype=torch.int32, device="meta")},
                {"token_mask": torch.empty(8, dtype=torch.uint8, device="meta")}):
        with pytest.raises(ValueError):
            layer.forward(b, None, None, None, None, None, balance=layer.BalanceLoss(0.1, **bad))
    with pytest.raises(ValueError):
        layer.forward(layer.MoELayerBuffers(s, "cpu", ckpt=True), None, None, None, None, None,
                      ckpt=layer.MoECheckpoint(s, "meta"))
    with pytest.raises(ValueError):  # no forward with a balance loss came before
        layer.backward(b, None, None, None, None, d_loss=torch.ones(2))
    b.balance = layer.BalanceLoss(0.1)
    for bad in (torch.ones(1), torch.ones(2, dtype=torch.float64), torch.ones(4)[::2], torch.empty(2, device="meta")):
        with pytest.raises(ValueError):
            layer.backward(b, None, None, None, None, d_loss=bad)
