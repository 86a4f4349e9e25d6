"""What the layer hands to the library's calls, without a GPU: every call is replaced by a recorder."""
import inspect

import pytest
import torch

from paper_2601_14327_gb300 import _lib as L
from paper_2601_14327_gb300 import build as B
from paper_2601_14327_gb300 import layer

S = layer.LayerShape(8, 128, 4, 2, 128)
HOST = ("moe_workspace_size", "moe_balance_workspace_size", "moe_perm_rows_max")


@pytest.fixture(autouse=True)
def _lib():
    B.build()


@pytest.fixture
def calls(monkeypatch):
    """[(name, {argument: value})] of the calls made, in order."""
    seen = []
    for name in [n for n in vars(L) if n.startswith("moe_") and n not in HOST]:
        sig = inspect.signature(getattr(L, name))

        def record(*a, _name=name, _sig=sig, **kw):
            seen.append((_name, dict(_sig.bind(*a, **kw).arguments)))

        monkeypatch.setattr(L, name, record)
    return seen


def _offsets(*at):
    return torch.tensor(at, dtype=torch.int32)


def _forward(b, bal, ckpt=None, mask=None, **kw):
    layer.forward(b, None, None, None, None, None, mask, stream=1, balance=bal, ckpt=ckpt, **kw)


def _backward(b, ckpt=None, **kw):
    layer.backward(b, None, None, None, None, stream=1, ckpt=ckpt, **kw)


def _args(calls, name):
    found = [a for n, a in calls if n == name]
    assert len(found) == 1, [n for n, _ in calls]
    return found[0]


@pytest.mark.parametrize("ckpt", [False, True])
def test_backward_takes_the_forwards_balance_loss(calls, ckpt):
    """One BalanceLoss object for all micro-batches, its fields set anew before each forward: the backward of the
    first micro-batch gets what that one's forward got."""
    b = layer.MoELayerBuffers(S, "cpu", balance_seqs=2, ckpt=ckpt)
    kept = [layer.MoECheckpoint(S, "cpu", 2) if ckpt else None for _ in range(2)]
    bal = layer.BalanceLoss(0.1, 0.01, seq_offsets=_offsets(0, 5, 8))
    first = bal.seq_offsets
    _forward(b, bal, kept[0])
    if ckpt:  # another micro-batch in between
        bal.coef, bal.seq_offsets = 0.3, _offsets(0, 8)
        _forward(b, bal, kept[1])
    bal.coef, bal.z_coef, bal.seq_offsets = 0.5, 0.05, _offsets(0, 1, 2, 3, 4, 8)
    calls.clear()
    _backward(b, kept[0])
    got = _args(calls, "moe_balance_loss_bwd")
    assert (got["n_seq"], got["coef"], got["z_coef"]) == (2, 0.1, 0.01) and got["seq_offsets"] is first
    assert got["n_seq"] + 2 <= got["n_tokens"].numel() and got["n_seq"] <= got["counts"].shape[0]
    if ckpt:
        calls.clear()
        _backward(b, kept[1])
        got = _args(calls, "moe_balance_loss_bwd")
        assert (got["n_seq"], got["coef"]) == (1, 0.3)


def test_backward_takes_the_forwards_number_of_sequences(calls):
    """Offsets that were resized in place since the forward: still the forward's number of sequences."""
    b = layer.MoELayerBuffers(S, "cpu", balance_seqs=2)
    bal = layer.BalanceLoss(0.1, seq_offsets=_offsets(0, 5, 8))
    _forward(b, bal)
    bal.seq_offsets.resize_(9)
    calls.clear()
    _backward(b)
    assert _args(calls, "moe_balance_loss_bwd")["n_seq"] == 2


@pytest.mark.parametrize("kw", [{}, {"balance_seqs": 1, "backward": False}])
def test_backward_refuses_buffers_without_room_for_the_losses_gradient(calls, kw):
    """The checkpoint's forward had a balance loss, the backward's buffers have no dz (or no backward at all): refused
    before the first launch."""
    c = layer.MoECheckpoint(S, "cpu", 1)
    _forward(layer.MoELayerBuffers(S, "cpu", balance_seqs=1, ckpt=True), layer.BalanceLoss(0.1), c)
    calls.clear()
    with pytest.raises(ValueError):
        _backward(layer.MoELayerBuffers(S, "cpu", ckpt=True, **kw), c)
    assert not calls
    _backward(layer.MoELayerBuffers(S, "cpu", balance_seqs=1, ckpt=True), c)
    assert calls


@pytest.mark.parametrize("balance", [False, True])
@pytest.mark.parametrize("ckpt", [False, True])
def test_kept_logits_are_in_the_buffers(calls, balance, ckpt):
    """keep_logits: the last call that writes b.logits makes them this routing's, also where a checkpoint keeps the
    logits for the balance loss."""
    b = layer.MoELayerBuffers(S, "cpu", balance_seqs=1, ckpt=ckpt)
    c = layer.MoECheckpoint(S, "cpu", 1) if ckpt else None
    _forward(b, layer.BalanceLoss(0.1) if balance else None, c, mask=5, keep_logits=True, logits_in=7)
    routes = [a for n, a in calls if n == "moe_route"]
    assert routes[-1]["logits_out"] is b.logits and all(a["active_mask"] == 5 for a in routes)
    # a second call has the first one's logits, so it writes the same routing
    assert routes[0]["logits_in"] == 7 and all(a["logits_in"] is c.logits for a in routes[1:])
    if balance:
        assert any(a["logits_out"] is (c or b).logits for a in routes)
    calls.clear()
    _forward(b, layer.BalanceLoss(0.1) if balance else None, c, logits_in=7)
    assert len([n for n, _ in calls if n == "moe_route"]) == 1
