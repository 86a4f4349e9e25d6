"""The balance loss without a GPU: the oracle against autograd and differences, and the refusals of the
entry points (nothing is launched)."""
import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from paper_2601_14327_gb300 import _lib as L
from paper_2601_14327_gb300 import build as B


@pytest.fixture(scope="module", autouse=True)
def _lib():
    B.build()


def _case(T, E, k, S, seed, masked=0, padded=False):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((T, E)) * 2
    mask = np.ones(E, np.uint8)
    mask[rng.permutation(E)[:masked]] = 0
    z[:, mask == 0] = -np.inf
    idx = np.argsort(-z, axis=1, kind="stable")[:, :k]
    off = None
    if S:
        off = np.concatenate([[0], np.sort(rng.integers(0, T + 1, S))])
        off[-1] = max(off[-2], T - 2)
    tok = (rng.random(T) > 0.3).astype(np.uint8) if padded else None
    return z, idx, mask, tok, off


@pytest.mark.parametrize("T,E,k,S,masked,padded", [(9, 6, 2, 0, 0, False), (20, 8, 3, 4, 2, True),
                                                   (1, 4, 1, 0, 0, False), (12, 5, 5, 3, 0, True)])
def test_oracle_gradient_against_autograd_and_differences(T, E, k, S, masked, padded):
    z, idx, mask, tok, off = _case(T, E, k, S, T + E, masked, padded)
    kw = dict(active_mask=mask, token_mask=tok, seq_offsets=off, coef=0.3, z_coef=0.2)
    ref = O.balance_loss(z, idx, d_loss=(0.7, 1.9), **kw)
    live = mask != 0
    zt = torch.tensor(z[:, live], dtype=torch.float64, requires_grad=True)
    bounds = [0, T] if off is None else list(off)
    lose, zl, seqs = 0.0, 0.0, [s for s in range(len(bounds) - 1) if ref["n_tokens"][s] > 0]
    for s in seqs:
        t = np.arange(bounds[s], bounds[s + 1])
        t = t if tok is None else t[tok[t] != 0]
        f = np.bincount(idx[t].reshape(-1), minlength=E)[live] * live.sum() / (k * len(t))
        lose = lose + 0.3 / len(seqs) * (torch.tensor(f) * torch.softmax(zt[t], 1).mean(0)).sum()
        zl = zl + 0.2 * (torch.logsumexp(zt[t], 1) ** 2).sum() / ref["n_tokens"][-2]
    np.testing.assert_allclose(ref["loss"], [lose.item(), zl.item()], rtol=1e-12)
    (0.7 * lose + 1.9 * zl).backward()
    np.testing.assert_allclose(ref["dz"][:, live], zt.grad.numpy(), rtol=1e-10, atol=1e-14)
    assert (ref["dz"][:, ~live] == 0).all()
    h = 1e-6
    for t, e in [(0, int(np.flatnonzero(live)[0])), (T // 2, int(np.flatnonzero(live)[-1]))]:
        zp, zm = z.copy(), z.copy()
        zp[t, e] += h
        zm[t, e] -= h
        d = (O.balance_loss(zp, idx, **kw)["loss"] - O.balance_loss(zm, idx, **kw)["loss"]) / (2 * h)
        # the difference's own error: curvature (~1) h^2 and the loss's rounding 2^-52 / h
        assert abs(0.7 * d[0] + 1.9 * d[1] - ref["dz"][t, e]) < 1e-8


def test_even_load_gives_the_coefficient():
    T, E, k = 12, 6, 2
    z = np.zeros((T, E))
    idx = np.stack([(np.arange(T) * 2) % E, (np.arange(T) * 2 + 1) % E], axis=1)
    ref = O.balance_loss(z, idx, coef=0.01)
    np.testing.assert_allclose(ref["loss"], [0.01, 0.0], rtol=1e-12)
    assert np.abs(ref["dz"]).max() < 1e-18


def _loss(**kw):
    a = dict(logits=16, topk_idx=16, active_mask=None, token_mask=None, seq_offsets=None, n_seq=1, T=10,
             E=8, k=2, coef=0.01, z_coef=0.0, loss=16, counts=16, prob=16, n_tokens=16, lse=16, ws=16,
             ws_bytes=1 << 20)
    a.update(kw)
    L.moe_balance_loss(*a.values(), stream=0)


def _bwd(**kw):
    a = dict(logits=16, active_mask=None, seq_offsets=None, n_seq=1, T=10, E=8, k=2, coef=0.01,
             z_coef=0.0, counts=16, n_tokens=16, lse=16, d_loss=None, dz=16)
    a.update(kw)
    L.moe_balance_loss_bwd(*a.values(), stream=0)


@pytest.mark.parametrize("call", [_loss, _bwd])
@pytest.mark.parametrize("bad,status", [
    ({"E": 0}, -2), ({"E": 257}, -2), ({"k": 0}, -2), ({"k": 9}, -2), ({"k": 8, "E": 7}, -2), ({"T": -1}, -1),
    ({"T": (1 << 30) + 1}, -1), ({"n_seq": 0}, -1), ({"n_seq": -3}, -1), ({"n_seq": 2}, -1), ({"n_seq": (1 << 20) + 1, "seq_offsets": 16}, -1),
    ({"coef": float("nan")}, -1), ({"z_coef": float("inf")}, -1), ({"logits": None}, -1), ({"lse": None}, -1),
    ({"counts": None}, -1), ({"n_tokens": None}, -1)])
def test_balance_refusals(call, bad, status):
    with pytest.raises(L.MoEError) as e:
        call(**bad)
    assert e.value.status == status


@pytest.mark.parametrize("bad,status", [
    ({"topk_idx": None}, -1), ({"loss": None}, -1), ({"prob": None}, -1), ({"ws": None}, -6),
    ({"ws_bytes": 512}, -6), ({"ws": 24}, -1)])
def test_balance_forward_refusals(bad, status):
    with pytest.raises(L.MoEError) as e:
        _loss(**bad)
    assert e.value.status == status


def test_balance_backward_refuses_no_output():
    with pytest.raises(L.MoEError) as e:
        _bwd(dz=None)
    assert e.value.status == -1


def test_balance_workspace_sizes():
    # per chunk or sequence a row of E fp32 sums and E counts
    assert L.moe_balance_workspace_size(65536, 256, 1) >= 152 * 256 * 8
    assert L.moe_balance_workspace_size(0, 8, 1) > 0
    assert L.moe_balance_workspace_size(16, 8, 1000) >= 1000 * 8 * 8
    for bad in ((-1, 8, 1), (8, 0, 1), (8, 8, 0)):
        assert L.moe_balance_workspace_size(*bad) == 0


def _dense(**kw):
    a = dict(x=16, topk_idx=16, topk_gate=16, d_gate=16, dz=16, T=10, d=128, E=8, k=2, d_logits=16,
             dw_router=16, ws=16, ws_bytes=1 << 24)
    a.update(kw)
    L.moe_route_bwd_dense(*a.values(), stream=0)


def _dx(**kw):
    a = dict(dz=16, w_router=16, dx_in=None, T=10, d=128, E=8, k=2, dx=16, ws=16, ws_bytes=1 << 24)
    a.update(kw)
    L.moe_route_dx(*a.values(), stream=0)


@pytest.mark.parametrize("call,bad,status", [
    (_dense, {"dz": None}, -1), (_dense, {"x": None}, -1), (_dense, {"x": 24}, -1), (_dense, {"E": 257}, -1),
    (_dense, {"d": 12}, -1), (_dense, {"T": -1}, -1), (_dense, {"k": 9}, -1), (_dense, {"dw_router": None}, -1),
    # the gates' arguments go together
    (_dense, {"topk_idx": None}, -1), (_dense, {"d_gate": None}, -1), (_dense, {"d_logits": None}, -1),
    (_dense, {"ws_bytes": 64}, -6), (_dense, {"ws": 24}, -1),
    (_dx, {"dz": None}, -1), (_dx, {"w_router": None}, -1), (_dx, {"dx": None}, -1), (_dx, {"dx": 24}, -1),
    (_dx, {"dx_in": 24}, -1), (_dx, {"E": 0}, -1), (_dx, {"E": 257}, -1), (_dx, {"d": 4}, -1), (_dx, {"T": -1}, -1),
    (_dx, {"k": 0}, -1), (_dx, {"ws": None}, -1), (_dx, {"ws_bytes": 64}, -6)])
def test_dense_router_backward_refusals(call, bad, status):
    with pytest.raises(L.MoEError) as e:
        call(**bad)
    assert e.value.status == status


@pytest.mark.parametrize("E,n_seq", [(1, 1), (64, 3), (256, 1 << 20)])
def test_balance_workspace_size_of_any_number_of_tokens(E, n_seq):
    """Ascending in T up to the largest int, also where the entry points refuse T."""
    sizes = [L.moe_balance_workspace_size(T, E, n_seq) for T in (0, 1, 1000, 1 << 20, 1 << 30, 2 ** 31 - 200, 2 ** 31 - 1)]
    assert sizes == sorted(sizes) and sizes[-1] < 1 << 40, sizes
    assert L.moe_balance_workspace_size(-1, E, n_seq) == 0
