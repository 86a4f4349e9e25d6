"""Balance loss, its gradient, and the products that carry it on, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from paper_2601_14327_gb300 import _lib as L

pytestmark = pytest.mark.gpu

F32, I32 = torch.float32, torch.int32


@pytest.fixture(autouse=True)
def _clean_device_error():
    L.moe_device_error(clear=True)
    yield
    assert L.moe_device_error(clear=True) == 0


def _inputs(T, E, k, S, masked=0, padded=0.0, seed=0, scale=2.0):
    rng = np.random.default_rng(seed + 7 * T + E)
    z = (rng.standard_normal((T, E)) * scale).astype(np.float32)
    z -= np.log1p(rng.permutation(E)).astype(np.float32)
    mask = None
    if masked:
        mask = np.ones(E, np.uint8)
        mask[rng.permutation(E)[:masked]] = 0
        z[:, mask == 0] = -np.inf
    idx = np.argsort(-z, axis=1, kind="stable")[:, :k].astype(np.int32)
    off = None
    if S:
        off = np.concatenate([[0], np.sort(rng.integers(0, T + 1, S))]).astype(np.int32)
        off[-1] = max(off[-2], T - T // 16)
    tok = (rng.random(T) >= padded).astype(np.uint8) if padded else None
    return z, idx, mask, tok, off


def _dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Balance:
    """The two calls with buffers of their own, filled with what must not be left there."""

    def __init__(self, T, E, k, S):
        self.T, self.E, self.k, self.S = T, E, k, max(1, S)
        nan = float("nan")
        self.loss = torch.full((2,), nan, device="cuda")
        self.counts = torch.full((self.S, E), -7, dtype=I32, device="cuda")
        self.prob = torch.full((self.S, E), nan, device="cuda")
        self.n_tokens = torch.full((self.S + 2,), -7, dtype=I32, device="cuda")
        self.lse = torch.full((T,), nan, device="cuda")
        self.dz = torch.full((T, E), nan, device="cuda")
        self.ws = torch.full((L.moe_balance_workspace_size(T, E, self.S),), 255, dtype=torch.uint8, device="cuda")

    def __call__(self, z, idx, mask, tok, off, coef, z_coef, d_loss=None, stream=None):
        L.moe_balance_loss(z, idx, mask, tok, off, self.S, self.T, self.E, self.k, coef, z_coef, self.loss,
                           self.counts, self.prob, self.n_tokens, self.lse, self.ws, self.ws.numel(), stream)
        L.moe_balance_loss_bwd(z, mask, off, self.S, self.T, self.E, self.k, coef, z_coef, self.counts,
                               self.n_tokens, self.lse, d_loss, self.dz, stream)
        return {n: getattr(self, n).cpu().numpy() for n in ("loss", "counts", "prob", "n_tokens", "lse", "dz")}


def _check(got, ref, coef, z_coef, d_loss, k):
    assert (got["counts"] == ref["counts"]).all()
    assert (got["n_tokens"] == ref["n_tokens"]).all()
    ok = ref["lse"] > -np.inf
    assert (np.isneginf(got["lse"]) == ~ok).all()
    # exp 2 ulp (2^-22), its argument's rounding weighted by p (|x| e^-|x| summed: < ln 256 * 2^-24), 13
    # additions, log 1 ulp, the final addition
    err = np.abs(got["lse"][ok] - ref["lse"][ok])
    assert (err <= 2e-6 + 2 ** -23 * np.abs(ref["lse"][ok])).all(), err.max()
    # p: 2^-22 + |z - m| 2^-24 (|z - m| <= 88: 5.3e-6) and the quotient; < 80 additions of 2^-24 each
    np.testing.assert_allclose(got["prob"], ref["prob"], rtol=1.2e-5, atol=1e-36)
    np.testing.assert_allclose(got["loss"], ref["loss"], rtol=1.2e-5, atol=1e-36)
    # gradient: p as above twice (its own and the weights of the mean), a, b, f - 1 and the sums' roundings,
    # relative to the sizes of its terms
    T, E = ref["dz"].shape
    scale = np.zeros((T, E))
    off = ref["off"]
    N, M, El = ref["n_tokens"][-1], ref["n_tokens"][-2], ref["live"].sum()
    for s in range(len(off) - 1):
        t = np.arange(off[s], off[s + 1])
        t = t[ok[t]]
        if len(t):
            f = np.abs(ref["counts"][s] * (El / (k * len(t))) - 1)
            p = ref["p"][t]
            scale[t] = p * (abs(d_loss[0]) * coef / (N * len(t)) * (f + (p * f).sum(1, keepdims=True))
                            + abs(d_loss[1]) * 2 * z_coef / M * np.abs(ref["lse"][t])[:, None])
    bad = np.abs(got["dz"] - ref["dz"]) > 2e-5 * scale + 1e-37
    assert not bad.any(), (bad.sum(), np.abs(got["dz"] - ref["dz"])[bad].max())
    assert (got["dz"][~ok] == 0).all() and (got["dz"][:, ~ref["live"]] == 0).all()


CASES = [
    # T, E, k, sequences (0: no offsets), pruned, padded
    (1, 1, 1, 0, 0, 0.0), (1, 256, 8, 0, 0, 0.0), (3, 5, 2, 2, 1, 0.0),
    # experts at the edges of the lanes per token
    (130, 16, 2, 3, 0, 0.2), (131, 17, 3, 0, 4, 0.0), (100, 32, 4, 1, 0, 0.0), (257, 33, 4, 5, 7, 0.3),
    (77, 64, 6, 2, 0, 0.0), (300, 65, 8, 0, 20, 0.0), (201, 128, 8, 4, 0, 0.5), (99, 129, 8, 1, 0, 0.0),
    (515, 171, 8, 7, 30, 0.1), (90, 192, 7, 2, 0, 0.0), (64, 193, 8, 0, 0, 0.0), (1000, 256, 8, 33, 85, 0.1),
    # a chunk per 8 tokens up to 4864, then longer ones; more sequences than tokens
    (4864, 64, 8, 3, 0, 0.0), (4865, 24, 4, 11, 3, 0.05), (20001, 96, 6, 40, 0, 0.0), (50, 12, 3, 200, 0, 0.2),
    # one block: at most three sequences and four rounds of tokens, and just more than that
    (200, 64, 6, 3, 3, 0.1), (200, 64, 6, 4, 0, 0.1), (384, 60, 4, 0, 0, 0.0), (385, 60, 4, 0, 0, 0.0),
    (192, 250, 8, 2, 9, 0.0), (193, 250, 8, 2, 9, 0.0),
    # every token masked
    (40, 20, 2, 3, 0, 1.0)]


@pytest.mark.parametrize("T,E,k,S,masked,padded", CASES)
def test_balance_against_oracle(T, E, k, S, masked, padded):
    z, idx, mask, tok, off = _inputs(T, E, k, S, masked, padded)
    coef, z_coef, d = 0.013, 0.002, (0.6, 1.7)
    ref = O.balance_loss(z, idx, mask, tok, off, coef, z_coef, d)
    ref["off"] = [0, T] if off is None else off
    b = Balance(T, E, k, S)
    got = b(_dev(z), _dev(idx), _dev(mask), _dev(tok), _dev(off), coef, z_coef, torch.tensor(d, device="cuda"))
    _check(got, ref, coef, z_coef, d, k)
    # twice the same inputs through the same workspace: the same bits
    again = b(_dev(z), _dev(idx), _dev(mask), _dev(tok), _dev(off), coef, z_coef, torch.tensor(d, device="cuda"))
    assert all((got[n] == again[n]).all() for n in got)
    # d_loss NULL: ones
    one = b(_dev(z), _dev(idx), _dev(mask), _dev(tok), _dev(off), coef, z_coef)
    _check(one, {**O.balance_loss(z, idx, mask, tok, off, coef, z_coef), "off": ref["off"]}, coef, z_coef, (1, 1), k)


def test_balance_without_tokens():
    E, k, S = 10, 2, 3
    got = Balance(0, E, k, S)(None, None, None, None, torch.zeros(S + 1, dtype=I32, device="cuda"), 1.0, 1.0)
    assert (got["loss"] == 0).all() and (got["counts"] == 0).all() and (got["prob"] == 0).all()
    assert (got["n_tokens"] == 0).all()


def test_balance_large_logits_and_masked_rubbish():
    """Logits near 1000 (their sum's rounding is common to a token's probabilities), masked tokens and
    pruned experts that hold infinities and NaN, rows without a live logit, rows behind the last sequence."""
    T, E, k = 200, 40, 4
    z, idx, mask, tok, off = _inputs(T, E, k, 3, masked=6, padded=0.2)
    z[np.ix_(np.arange(0, T, 3), mask != 0)] += 1000
    z[5, :] = -np.inf
    z[17, :] = -np.inf
    coef, z_coef, d = 0.01, 1e-4, (1, 1)
    ref = O.balance_loss(z, idx, mask, tok, off, coef, z_coef)
    ref["off"] = off
    dirty = z.copy()
    dirty[:, mask == 0] = np.nan
    dirty[tok == 0] = np.inf
    dirty[off[-1]:] = np.nan
    bad_idx = idx.copy()
    bad_idx[tok == 0] = -1
    bad_idx[off[-1]:] = 9999
    bad_idx[[5, 17]] = E
    got = Balance(T, E, k, 3)(_dev(dirty), _dev(bad_idx), _dev(mask), _dev(tok), _dev(off), coef, z_coef)
    _check(got, ref, coef, z_coef, d, k)


@pytest.mark.parametrize("T", [60, 3000])
def test_balance_rows_of_the_lowest_value(T):
    """Masks as the type's lowest value: such a logit has no probability beside an ordinary one; a row of nothing
    else is a row of equal logits. Also very large ones."""
    E, k = 20, 3
    z, idx, _, _, _ = _inputs(T, E, k, 0)
    low = np.finfo(np.float32).min
    z[:, 4] = low
    z[1::7] = low
    z[2::7, 3] = -low
    z[3::7] += 3e9
    z[4::7, 5:] *= 1e5
    idx = np.argsort(-z, axis=1, kind="stable")[:, :k].astype(np.int32)
    off = np.array([0, T // 2, T], np.int32)
    ref = O.balance_loss(z, idx, None, None, off, 0.5, 0.0)
    ref["off"] = off
    got = Balance(T, E, k, 2)(_dev(z), _dev(idx), None, None, _dev(off), 0.5, 0.0)
    assert got["loss"][1] == 0 and (ref["p"][1] == 1 / E).all()
    # a log-sum-exp this large has no room for the sum of exponentials: the log-sum-exp itself, and
    # then p (from it) only where it is exact, near logits of ordinary size, or from the sums of p
    # (2e-6 + 2^-23 |lse| as in _check: where m + log(sum) cancels, the roundings of m, up to 8 here, and of the
    # logarithm stay, 8 * 2^-24 + 2^-22)
    np.testing.assert_allclose(got["lse"], ref["lse"], rtol=2 ** -23, atol=2e-6)
    np.testing.assert_allclose(got["prob"], ref["prob"], rtol=1.2e-5, atol=1e-36)
    np.testing.assert_allclose(got["loss"], ref["loss"], rtol=1.2e-5)
    assert np.isfinite(got["dz"]).all()
    few = np.abs(ref["lse"]) < 100
    assert (np.abs(got["dz"] - ref["dz"])[few] <= 2e-5 * np.abs(ref["dz"][few]).max()).all()
    # rows of equal logits: p is divided by its sum, so their rounding does not matter
    np.testing.assert_allclose(got["dz"][1::7], ref["dz"][1::7], rtol=2e-5, atol=2e-5 * np.abs(ref["dz"]).max())


@pytest.mark.parametrize("T,E", [(60, 64), (61, 13), (3001, 64), (3000, 250)])
def test_balance_bits_do_not_depend_on_other_tokens(T, E):
    """What masked tokens, tokens behind the last sequence and pruned experts hold, and which tokens share a warp with
    one, changes no bit of the results."""
    z, idx, mask, tok, off = _inputs(T, E, 2, 2, masked=3, padded=0.3)
    d = torch.tensor((0.6, 1.7), device="cuda")
    got = []
    for fill in (0.0, 1e30, np.inf, -3e38):
        y = z.copy()
        y[tok == 0] = fill
        y[off[-1]:] = fill
        y[:, mask == 0] = fill
        got.append(Balance(T, E, 2, 2)(_dev(y), _dev(idx), _dev(mask), _dev(tok), _dev(off), 0.013, 0.002, d))
    for g in got[1:]:
        assert all((g[n] == got[0][n]).all() for n in g)
    # a token with a logit of 1e5 (a log-sum-exp of its own kind) beside the others: their bits stay, but for the
    # sequence's means in dz
    y = z.copy()
    t = int(np.flatnonzero(tok[:off[1]])[0]) if tok[:off[1]].any() else 0
    y[t, np.flatnonzero(mask)[0]] = 1e5
    far = Balance(T, E, 2, 2)(_dev(y), _dev(idx), _dev(mask), _dev(tok), _dev(off), 0.013, 0.002, d)
    same = np.arange(T) != t
    assert (far["lse"][same] == got[0]["lse"][same]).all() and (far["dz"][same] == got[0]["dz"][same]).all()


def test_balance_nan_reaches_its_sequence_only():
    T, E, k = 64, 8, 2
    z, idx, _, _, _ = _inputs(T, E, k, 0)
    off = np.array([0, 30, 64], np.int32)
    z[40, 3] = np.nan
    got = Balance(T, E, k, 2)(_dev(z), _dev(idx), None, None, _dev(off), 1.0, 0.0)
    assert np.isnan(got["loss"][0]) and np.isfinite(got["prob"][0]).all() and np.isnan(got["prob"][1]).any()
    assert np.isfinite(got["dz"][:30]).all() and np.isnan(got["dz"][40]).all()
    assert np.isfinite(np.delete(got["lse"], 40)).all()


@pytest.mark.parametrize("T,E", [(40, 64), (9000, 64), (700, 256)])
def test_balance_unaligned_rows_and_late_first_sequence(T, E):
    """Rows of whole 16-byte vectors that start off a 16-byte boundary; rows before the first sequence."""
    k = 4
    z, idx, mask, tok, _ = _inputs(T, E, k, 0, masked=3, padded=0.1)
    off = np.array([T // 8, T // 8, T // 2, T - 3], np.int32)
    ref = O.balance_loss(z, idx, mask, tok, off, 0.02, 0.003)
    ref["off"] = off
    b = Balance(T, E, k, 3)
    args = [_dev(idx), _dev(mask), _dev(tok), _dev(off), 0.02, 0.003]
    aligned = b(_dev(z), *args)
    _check(aligned, ref, 0.02, 0.003, (1, 1), k)
    shifted = torch.empty(T * E + 1, device="cuda")[1:].view(T, E)
    shifted.copy_(_dev(z))
    b.dz = torch.full((T * E + 3,), float("nan"), device="cuda")[3:].view(T, E)
    _check(b(shifted, *args), ref, 0.02, 0.003, (1, 1), k)


def test_balance_flags_bad_ids_and_offsets():
    T, E, k = 50, 6, 2
    z, idx, _, _, _ = _inputs(T, E, k, 0)
    idx[7, 1] = E
    idx[9, 0] = -1
    got = Balance(T, E, k, 0)(_dev(z), _dev(idx), None, None, None, 1.0, 0.0)
    assert L.moe_device_error(clear=True) == 1  # MOE_DEV_BAD_EXPERT
    assert (got["counts"] == O.balance_loss(z, idx)["counts"]).all()
    idx = np.clip(idx, 0, E - 1)
    for off in ([0, 30, 20], [-1, 30, 50], [0, 20, T + 1]):
        Balance(T, E, k, 2)(_dev(z), _dev(idx), None, None, _dev(np.array(off, np.int32)), 1.0, 0.0)
        assert L.moe_device_error(clear=True) == 6, off  # MOE_DEV_BAD_OFFSETS


def test_balance_in_a_graph_and_on_another_stream():
    """Captured once and replayed on new inputs; two graphs with workspaces of their own."""
    T, E, k, S = 700, 48, 4, 5
    z, idx, mask, tok, off = _inputs(T, E, k, S, 5, 0.1)
    z2, idx2, _, tok2, _ = _inputs(T, E, k, S, 0, 0.1, seed=1)
    z2[:, mask == 0] = -np.inf
    idx2 = np.argsort(-z2, axis=1, kind="stable")[:, :k].astype(np.int32)
    bufs = [_dev(z), _dev(idx), _dev(mask), _dev(tok), _dev(off)]
    b, e = Balance(T, E, k, S), Balance(T, E, k, S)
    want = [e(*bufs, 0.01, 0.001), e(_dev(z2), _dev(idx2), bufs[2], _dev(tok2), bufs[4], 0.01, 0.001)]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()

    def calls(stream):
        L.moe_balance_loss(*bufs, S, T, E, k, 0.01, 0.001, b.loss, b.counts, b.prob, b.n_tokens, b.lse, b.ws,
                           b.ws.numel(), stream)
        L.moe_balance_loss_bwd(bufs[0], bufs[2], bufs[4], S, T, E, k, 0.01, 0.001, b.counts, b.n_tokens, b.lse, None,
                               b.dz, stream)

    calls(st)
    st.synchronize()
    with torch.cuda.graph(g, stream=st):
        calls(torch.cuda.current_stream())
    for i, new in ((0, None), (1, (z2, idx2, tok2)), (0, (z, idx, tok))):
        if new is not None:
            for at, v in zip((0, 1, 3), new):
                bufs[at].copy_(_dev(v))
        g.replay()
        torch.cuda.synchronize()
        for n, v in want[i].items():
            assert (getattr(b, n).cpu().numpy() == v).all(), (i, n)


# ---------------------------------------------------------------- into the router's weight and the input


def _router_inputs(T, d, E, k, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g).to(torch.bfloat16)
    w = torch.randn(d, E, generator=g) / d ** 0.5
    z = torch.randn(T, E, generator=g)
    idx = torch.argsort(z, dim=1, descending=True)[:, :k].to(I32).contiguous()
    gate = torch.softmax(torch.gather(z, 1, idx.long()), 1).contiguous()
    dg = torch.randn(T, k, generator=g)
    dz = torch.randn(T, E, generator=g) * torch.softmax(3 * z, 1)
    dx_in = (0.1 * torch.randn(T, d, generator=g)).to(torch.bfloat16)
    return x, w, idx, gate, dg, dz, dx_in


ROUTER = [(1, 8, 1, 1), (3, 72, 5, 2), (130, 136, 13, 2), (257, 256, 17, 4), (333, 200, 64, 6), (128, 512, 128, 8),
          (1000, 384, 100, 4), (515, 776, 171, 8), (129, 1024, 256, 8), (2500, 264, 48, 3), (4097, 2048, 33, 8)]


@pytest.mark.parametrize("T,d,E,k", ROUTER)
def test_dense_router_backward_against_oracle(T, d, E, k):
    x, w, idx, gate, dg, dz, _ = _router_inputs(T, d, E, k, T + E)
    n = L.moe_workspace_size(T, d, E, k, 128)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    dl = torch.full((T, k), float("nan"), device="cuda")
    dw = torch.full((d, E), float("nan"), device="cuda")
    L.moe_route_bwd_dense(x.cuda(), idx.cuda(), gate.cuda(), dg.cuda(), dz.cuda(), T, d, E, k, dl, dw, ws, n)
    dl_ref, dw_ref = O.router_backward(x.double().numpy(), idx.numpy(), gate.double().numpy(),
                                       dg.double().numpy(), E)
    xd, zd = x.double().numpy(), dz.double().numpy()
    dw_ref = dw_ref + xd.T @ zd
    g64, dg64 = gate.double().numpy(), dg.double().numpy()
    zs = np.abs(g64) * (np.abs(dg64) + np.sum(np.abs(g64 * dg64), axis=1, keepdims=True))
    assert (np.abs(dl.cpu().numpy() - dl_ref) <= 2e-6 * zs + 1e-30).all()
    size = np.abs(zd)
    np.put_along_axis(size, idx.numpy().astype(np.int64),
                      np.take_along_axis(size, idx.numpy().astype(np.int64), 1) + zs, 1)
    # dZ carried to 2^-24, products exact, 48 truncated additions (2^-23 each) per accumulator, then one
    # fp32 addition per 256 tokens and one per split: (48 * 2 + T / 256 + 64) * 2^-24 < 1e-5
    assert (np.abs(dw.cpu().double().numpy() - dw_ref) <= 1e-5 * (np.abs(xd).T @ size) + 1e-30).all()
    # without the gates' part; with a zero dz moe_route_bwd's gradient, and its d_logits bit for bit
    only = torch.full_like(dw, float("nan"))
    L.moe_route_bwd_dense(x.cuda(), None, None, None, dz.cuda(), T, d, E, k, None, only, ws, n)
    assert (np.abs(only.cpu().double().numpy() - xd.T @ zd) <= 1e-5 * (np.abs(xd).T @ np.abs(zd)) + 1e-30).all()
    none, plain, dl2 = torch.empty_like(dw), torch.empty_like(dw), torch.empty_like(dl)
    L.moe_route_bwd_dense(x.cuda(), idx.cuda(), gate.cuda(), dg.cuda(), torch.zeros(T, E, device="cuda"), T, d, E, k,
                          dl, none, ws, n)
    L.moe_route_bwd(x.cuda(), idx.cuda(), gate.cuda(), dg.cuda(), T, d, E, k, dl2, plain, ws, n)
    gates = np.zeros((T, E))
    np.put_along_axis(gates, idx.numpy().astype(np.int64), zs, 1)
    bound = 2e-5 * (np.abs(xd).T @ gates) + 1e-30  # (either is within 1e-5 of it)
    assert ((none - plain).abs().cpu().double().numpy() <= bound).all() and torch.equal(dl, dl2)


@pytest.mark.parametrize("T,d,E", [(65536, 256, 171), (65536, 264, 64), (40000, 8, 256), (65537, 128, 20)])
def test_dense_router_backward_over_many_tokens(T, d, E):
    """Sums over many tokens stay near 64 bits in the 2-norm too: an accumulator holds at most 48 truncated
    additions, off by 2^-24 of it each on average (2.9e-6, were it as large as at its end all along)."""
    g = torch.Generator(device="cuda").manual_seed(T + E)
    x = torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)
    dz = torch.randn(T, E, generator=g, device="cuda")
    n = L.moe_workspace_size(T, d, E, 8, 128)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    dw, again = torch.empty(d, E, device="cuda"), torch.empty(d, E, device="cuda")
    L.moe_route_bwd_dense(x, None, None, None, dz, T, d, E, 8, None, dw, ws, n)
    L.moe_route_bwd_dense(x, None, None, None, dz, T, d, E, 8, None, again, ws, n)
    ref = x.double().T @ dz.double()
    assert torch.equal(dw, again)
    assert float((dw.double() - ref).norm() / ref.norm()) < 2.9e-6


def test_dense_router_backward_ids_twice_and_outside():
    T, d, E, k = 100, 64, 10, 3
    x, w, idx, gate, dg, dz, _ = _router_inputs(T, d, E, k, 9)
    idx[:, 1] = idx[:, 0]
    idx[::5, 2] = E
    idx[1::5, 2] = -1
    n = L.moe_workspace_size(T, d, E, k, 128)
    dl, dw = torch.empty(T, k, device="cuda"), torch.empty(d, E, device="cuda")
    L.moe_route_bwd_dense(x.cuda(), idx.cuda(), gate.cuda(), dg.cuda(), dz.cuda(), T, d, E, k, dl, dw,
                          torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    g64, dg64 = gate.double().numpy(), dg.double().numpy()
    dl_ref = g64 * (dg64 - (g64 * dg64).sum(1, keepdims=True))
    zz = dz.double().numpy().copy()
    for j in range(k):
        t = np.flatnonzero((idx[:, j].numpy() >= 0) & (idx[:, j].numpy() < E))
        np.add.at(zz, (t, idx[t, j].numpy()), dl_ref[t, j])
    assert np.abs(dl.cpu().numpy() - dl_ref).max() < 1e-5
    size = np.abs(x.double().numpy()).T @ (np.abs(dz.double().numpy()) + 3 * np.abs(dl_ref).max())
    assert (np.abs(dw.cpu().double().numpy() - x.double().numpy().T @ zz) <= 1e-5 * size).all()


def test_router_dx_beside_the_experts_backward():
    """moe_route_dx on a second stream beside moe_grouped_ffn_bwd_dgrad with one workspace: both as alone."""
    T, d, E, k, F = 4000, 512, 16, 4, 1024
    g = torch.Generator(device="cuda").manual_seed(1)
    R = L.moe_perm_rows_max(T, k, E)

    def rnd(*n, dtype=torch.bfloat16, s=1.0):
        return (s * torch.randn(*n, generator=g, device="cuda")).to(dtype)

    idx = torch.argsort(rnd(T, E, dtype=F32), dim=1)[:, :k].to(I32).contiguous()
    gate, n = torch.full((T, k), 1 / k, device="cuda"), L.moe_workspace_size(T, d, E, k, F)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    off, cnt = torch.empty(E + 1, dtype=I32, device="cuda"), torch.empty(E, dtype=I32, device="cuda")
    row, xp = torch.empty(T, k, dtype=I32, device="cuda"), torch.zeros(R, d, dtype=torch.bfloat16, device="cuda")
    L.moe_permute(rnd(T, d), idx, None, T, d, E, k, R, off, cnt, row, xp, ws, n)
    ab, wu, wd = rnd(R, 2 * F), rnd(E, 2 * F, d, s=0.02), rnd(E, d, F, s=0.02)
    dz, w, dx_in = rnd(T, E, dtype=F32), rnd(d, E, dtype=F32), rnd(T, d)
    dab, dx = torch.empty(R, 2 * F, dtype=torch.bfloat16, device="cuda"), torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    dxp, dg = torch.zeros(R, d, dtype=torch.bfloat16, device="cuda"), torch.empty(T, k, device="cuda")
    side = torch.cuda.Stream()

    def dgrad():
        L.moe_grouped_ffn_bwd_dgrad(xp, ab, off, E, d, F, R, wu, wd, gate, None, row, None, T, k, dg, dab, dxp, ws, n)

    def route(stream=None):
        L.moe_route_dx(dz, w, dx_in, T, d, E, k, dx, ws, n, stream)

    dgrad()
    route()
    torch.cuda.synchronize()
    want = [t.clone() for t in (dx, dg, dxp)]
    for _ in range(20):
        for t in (dx, dg, dxp):
            t.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            dgrad()
            route(side)
        torch.cuda.synchronize()
        for a, b in zip((dx, dg, dxp), want):
            assert torch.equal(a, b)


def test_dense_router_backward_without_tokens():
    dw = torch.full((64, 6), float("nan"), device="cuda")
    n = L.moe_workspace_size(0, 64, 6, 2, 128)
    L.moe_route_bwd_dense(None, None, None, None, None, 0, 64, 6, 2, None, dw,
                          torch.empty(n, dtype=torch.uint8, device="cuda"), n)
    assert (dw == 0).all()
    L.moe_route_dx(None, None, None, 0, 64, 6, 2, None, None, 0)


def _dx(dz, w, dx_in, k, out=None):
    T, E = dz.shape
    d = w.shape[0]
    n = L.moe_workspace_size(T, d, E, k, 128)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((T, d), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    L.moe_route_dx(dz.cuda(), w.cuda(), dx_in, T, d, E, k, out, ws, n)
    torch.cuda.synchronize()
    return out


def _dx_bound(ref, size):
    # the result's rounding to bf16 (2^-8); both factors in half precision (2^-11 each, powers of two
    # taken out), products exact, up to 256 fp32 additions (2^-24 each)
    return 2 ** -8 * np.abs(ref) + (2 ** -10 + 2 ** -16) * (1 + 2 ** -8) * size + 1e-37


@pytest.mark.parametrize("T,d,E,k", ROUTER)
def test_route_dx_against_64_bits(T, d, E, k):
    _, w, _, _, _, dz, dx_in = _router_inputs(T, d, E, k, T + E + 1)
    prod, size = dz.double().numpy() @ w.double().numpy().T, dz.abs().double().numpy() @ w.abs().double().numpy().T
    got = _dx(dz, w, None, k).double().cpu().numpy()
    assert (np.abs(got - prod) <= _dx_bound(prod, size)).all()
    ref = prod + dx_in.double().numpy()
    out = _dx(dz, w, dx_in.cuda(), k)
    assert (np.abs(out.double().cpu().numpy() - ref) <= _dx_bound(ref, size)).all()
    # in place: the same bits; no token's gradient: dx_in
    buf = dx_in.cuda()
    assert torch.equal(_dx(dz, w, buf, k, out=buf), out)
    assert torch.equal(_dx(torch.zeros(T, E), w, dx_in.cuda(), k), dx_in.cuda())


def test_route_dx_wide_ranges():
    """Rows and columns of very different sizes: each row of the result is as near as its own size asks."""
    T, d, E, k = 300, 272, 60, 4
    _, w, _, _, _, dz, _ = _router_inputs(T, d, E, k, 5)
    dz = dz * torch.exp2(torch.arange(T)[:, None] % 61 - 50.0)
    w = w * torch.exp2(torch.arange(d)[:, None] % 41 - 30.0)
    dz[7] = 0
    w[9] = 0
    # smaller than the row's largest by up to 2^20
    dz[:, ::3] *= 2.0 ** -20
    prod, size = dz.double().numpy() @ w.double().numpy().T, dz.abs().double().numpy() @ w.abs().double().numpy().T
    got = _dx(dz, w, None, k).double().cpu().numpy()
    assert (np.abs(got - prod) <= _dx_bound(prod, size)).all()
    assert (got[7] == 0).all() and (got[:, 9] == 0).all()


def test_route_dx_largest_and_smallest_factors():
    """Gradients up to fp32's largest beside weights that bring the product back, and the other way round."""
    T, d, E, k = 280, 136, 40, 2
    _, w, _, _, _, dz, _ = _router_inputs(T, d, E, k, 8)
    dz, w = dz / dz.abs().max(), w / w.abs().max()
    for a, b in ((2.0 ** 127, 2.0 ** -60), (2.0 ** 127, 2.0 ** -100), (2.0 ** -80, 2.0 ** 117), (2.0 ** -100, 2.0 ** 60)):
        y, v = dz * a, w * b
        prod, size = y.double().numpy() @ v.double().numpy().T, y.abs().double().numpy() @ v.abs().double().numpy().T
        got = _dx(y, v, None, k).double().cpu().numpy()
        assert (np.abs(got - prod) <= _dx_bound(prod, size)).all(), (a, b)


def test_route_dx_infinities_stay_in_their_row():
    T, d, E, k = 140, 136, 20, 2
    _, w, _, _, _, dz, dx_in = _router_inputs(T, d, E, k, 6)
    clean = _dx(dz, w, dx_in.cuda(), k)
    dz[3, 4], dz[100, 0] = float("nan"), float("inf")
    got = _dx(dz, w, dx_in.cuda(), k)
    keep = [t for t in range(T) if t not in (3, 100)]
    assert torch.equal(got[keep], clean[keep])
    assert torch.isnan(got[3]).all() and not torch.isfinite(got[100]).any()


def test_balance_and_router_past_32_bits():
    """More than 2^31 logits; the last rows against 64 bits."""
    T, E, k, d = 8_500_000, 256, 1, 8
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn(T, E, generator=g, device="cuda")
    idx = z.argmax(1, keepdim=True).to(I32)
    b = Balance(T, E, k, 0)
    L.moe_balance_loss(z, idx, None, None, None, 1, T, E, k, 1.0, 0.5, b.loss, b.counts, b.prob, b.n_tokens, b.lse, b.ws,
                       b.ws.numel())
    L.moe_balance_loss_bwd(z, None, None, 1, T, E, k, 1.0, 0.5, b.counts, b.n_tokens, b.lse, None, b.dz)
    assert T * E > 2 ** 31 and int(b.counts.sum()) == T
    zt = z[-500:].double()
    lse = torch.logsumexp(zt, 1)
    assert ((b.lse[-500:].double() - lse).abs() <= 2e-6 + 2 ** -23 * lse.abs()).all()
    p, f = torch.exp(zt - lse[:, None]), b.counts[0].double() * E / T - 1
    dz = p * ((f - (p * f).sum(1, keepdim=True)) / T + lse[:, None] / T)
    size = p * ((f.abs() + (p * f.abs()).sum(1, keepdim=True)) / T + lse[:, None].abs() / T)
    assert ((b.dz[-500:].double() - dz).abs() <= 2e-5 * size).all()
    del z
    n = L.moe_workspace_size(T, d, E, k, 128)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    w = torch.randn(d, E, generator=g, device="cuda")
    b.dz *= T
    out = torch.full((T, d), 9.0, dtype=torch.bfloat16, device="cuda")
    L.moe_route_dx(b.dz, w, None, T, d, E, k, out, ws, n)
    ref, size = b.dz[-500:].double() @ w.double().T, b.dz[-500:].double().abs() @ w.double().abs().T
    err = (out[-500:].double() - ref).abs().cpu().numpy()
    assert (err <= _dx_bound(ref.cpu().numpy(), size.cpu().numpy())).all()
    # x^T dZ over the last rows alone: the others' x is zero
    x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    x[-500:] = torch.randn(500, d, generator=g, device="cuda").to(torch.bfloat16)
    dw = torch.empty(d, E, device="cuda")
    L.moe_route_bwd_dense(x, None, None, None, b.dz, T, d, E, k, None, dw, ws, n)
    xt, zt = x[-500:].double(), b.dz[-500:].double()
    assert ((dw.double() - xt.T @ zt).abs() <= 1e-5 * (xt.abs().T @ zt.abs()) + 1e-30).all()


@pytest.mark.parametrize("T,d,E", [(64, 136, 256), (63, 264, 1), (65, 128, 65), (256, 384, 80), (250, 1032, 171), (256, 136, 240),
                                   (257, 384, 100), (1, 8, 33)])
def test_dense_router_backward_in_one_split(T, d, E):
    """One k-block, and up to four of more than 64 experts, are written without partial sums; just more are not."""
    g = torch.Generator().manual_seed(T * d + E)
    x, dz = torch.randn(T, d, generator=g).to(torch.bfloat16), torch.randn(T, E, generator=g)
    n = L.moe_workspace_size(T, d, E, 1, 128)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    dw = torch.full((d + 1, E), 7.0, device="cuda")
    L.moe_route_bwd_dense(x.cuda(), None, None, None, dz.cuda(), T, d, E, 1, None, dw, ws, n)
    xd, zd = x.double().numpy(), dz.double().numpy()
    assert (np.abs(dw[:d].cpu().double().numpy() - xd.T @ zd) <= 1e-5 * (np.abs(xd).T @ np.abs(zd)) + 1e-30).all()
    assert (dw[d] == 7).all()  # nothing behind the last row


def _sums_64(z, idx, off, k):
    """counts, prob and sum of lse^2 of each sequence, in 64 bits and slices."""
    E, out = z.shape[1], []
    for a, b in zip(off[:-1], off[1:]):
        p, q = torch.zeros(E, dtype=torch.float64, device="cuda"), 0.0
        for t in range(a, b, 1 << 20):
            y = z[t:min(b, t + (1 << 20))].double()
            lse = torch.logsumexp(y, 1)
            p += torch.exp(y - lse[:, None]).sum(0)
            q += float((lse * lse).sum())
        c = torch.bincount(idx[a:b].reshape(-1).long(), minlength=E)
        out.append((c, p / max(1, b - a), q))
    return out


def _check_sums(z, idx, off, k):
    T, E = z.shape
    S = len(off) - 1
    b = Balance(T, E, k, S)
    coef, z_coef = 0.7, 0.3
    L.moe_balance_loss(z, idx, None, None, None if S == 1 else torch.tensor(off, dtype=I32, device="cuda"), S, T, E, k,
                       coef, z_coef, b.loss, b.counts, b.prob, b.n_tokens, b.lse, b.ws, b.ws.numel())
    ref = _sums_64(z, idx, off, k)
    N, M = sum(hi > lo for lo, hi in zip(off[:-1], off[1:])), off[-1] - off[0]
    loss = 0.0
    for s, (c, p, _) in enumerate(ref):
        n = off[s + 1] - off[s]
        assert int(b.n_tokens[s]) == n and torch.equal(b.counts[s].long(), c)
        # fp32 additions one after another: 80 of a lane, 3 of a warp's tokens, 24 warps, then rows of chunks
        # (64 and T / 2^20 at most) and 32 warps, 2^-24 each; p itself: exp and the quotient 2^-22 each, the exponent's
        # argument |z - m| 2^-23 (|z - m| < 16)
        tol = (80 + 3 + 24 + 64 + T / 2 ** 20 + 32 + 4) * 2 ** -24 + 2 ** -21 + 2 ** -19
        assert ((b.prob[s].double() - p).abs() <= tol * p).all(), float(((b.prob[s].double() - p).abs() / p).max())
        if n:
            loss += coef / N * float((c.double() * E / (k * n) * p).sum())
    # (a few more roundings: the quotients, the products, the sums over experts and sequences)
    tol += 24 * 2 ** -24
    assert abs(float(b.loss[0]) - loss) <= tol * loss
    lz = z_coef * sum(r[2] for r in ref) / M
    assert abs(float(b.loss[1]) - lz) <= tol * lz, (float(b.loss[1]), lz)


def test_balance_sums_of_many_equal_tokens():
    """Equal addends round the same way: sums of one after another would be off by more the more tokens there are."""
    T, E, k = 1 << 26, 4, 1
    row = torch.log(torch.tensor([0.8694458658865812, 0.06, 0.04, 0.0305541341134188], dtype=torch.float64)) + 1.3
    z = row.float().cuda().expand(T, E).contiguous()
    _check_sums(z, torch.zeros(T, k, dtype=I32, device="cuda"), [0, T], k)


@pytest.mark.parametrize("T,E,k,S", [(1_500_000, 96, 4, 5), (4_000_000, 16, 2, 1), (2_400_000, 40, 8, 300)])
def test_balance_sums_of_many_tokens(T, E, k, S):
    """More chunks than SMs: sums of probabilities and squares against 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(T + E)
    z = torch.randn(T, E, generator=g, device="cuda") - torch.log1p(torch.arange(E, device="cuda").float())
    idx = torch.randint(0, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
    cut = torch.sort(torch.randint(0, T + 1, (S - 1,), generator=g, device="cuda"))[0].tolist()
    _check_sums(z, idx, [0] + cut + [T], k)


@pytest.mark.parametrize("T,d,E", [(1 << 22, 64, 20), ((1 << 20) + 77, 136, 171), (65536, 256, 64)])
def test_dense_router_backward_of_many_tokens_of_one_sign(T, d, E):
    """Sums that grow all along, so that every addition rounds in the size of the result: against 64 bits in slices."""
    g = torch.Generator(device="cuda").manual_seed(T + E)
    x = (1 + 0.1 * torch.randn(T, d, generator=g, device="cuda")).to(torch.bfloat16)
    dz = 1 + 0.1 * torch.rand(T, E, generator=g, device="cuda")
    n = L.moe_workspace_size(T, d, E, 8, 128)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    dw = torch.empty(d, E, device="cuda")
    L.moe_route_bwd_dense(x, None, None, None, dz, T, d, E, 8, None, dw, ws, n)
    ref = torch.zeros(d, E, dtype=torch.float64, device="cuda")
    for t in range(0, T, 1 << 18):
        ref += x[t:t + (1 << 18)].double().T @ dz[t:t + (1 << 18)].double()
    # (up to 256 features: 64 splits.) dZ carried to 2^-24; 48 truncated additions of 2^-23 in an accumulator, one
    # rounded addition per 256 tokens of a split, two of the terms, one per split
    kb = -(-T // 64)
    chain = -(-(-(-kb // 64)) // 4)
    tol = (1 + 2 * 48 + chain + 2 + 64) * 2 ** -24
    assert ((dw.double() - ref).abs() <= tol * ref).all(), float(((dw.double() - ref).abs() / ref).max())


def _dx_bound_cancelled(ref, size, E, dz, w):
    # the result's rounding to bf16 (2^-8); factors of two half-precision terms (2^-22 of a value, or 2^-39 of its row's
    # largest), the product of both second terms left out (2^-22), three fp32 additions per 16 experts that truncate (2^-23)
    small = 2.0 ** -39 * E * 2 * np.abs(dz).max(1, keepdims=True) * np.abs(w).max(1)
    return 2 ** -8 * np.abs(ref) + (1 + 2 ** -8) * ((3 * 2 ** -22 + 3 * -(-E // 16) * 2 ** -23) * size + small) + 1e-37


@pytest.mark.parametrize("T,d,E,k", ROUTER + [(700, 296, 192, 4), (300, 520, 240, 4), (130, 264, 65, 2), (300, 72, 130, 2), (200, 2872, 225, 8)])
def test_route_dx_carries_more_bits_than_its_result(T, d, E, k):
    """dx_in cancels the product but for bf16's rounding: what is left of the product's own error shows."""
    _, w, _, _, _, dz, _ = _router_inputs(T, d, E, k, T + E + 3)
    z64, w64 = dz.double().numpy(), w.double().numpy()
    prod, size = z64 @ w64.T, np.abs(z64) @ np.abs(w64).T
    dx_in = torch.from_numpy(-prod).to(torch.bfloat16)
    ref = prod + dx_in.double().numpy()
    got = _dx(dz, w, dx_in.cuda(), k).double().cpu().numpy()
    bound = _dx_bound_cancelled(ref, size, E, z64, w64)
    assert (np.abs(got - ref) <= bound).all(), (np.abs(got - ref) / bound).max()
