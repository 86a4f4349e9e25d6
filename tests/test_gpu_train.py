"""The vocabulary loss and the orthogonalised update on the GPU, through the package's calls, against the oracle
in 64 bits."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import moe_oracle as O
from paper_2601_14327_gb300 import _lib as L
from paper_2601_14327_gb300 import layer, train

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U16 = 2.0 ** -8   # half a step of bf16, relative


def dev_ok():
    torch.cuda.synchronize()
    assert L.moe_device_error(clear=True) == 0


def npf(t):
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------- vocabulary loss


def vocab_case(T, d, V, seed, std=2.0, ignored=0.0, sure=0.0):
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(V, d, generator=g) * (std / d ** 0.5)).to(BF16)
    target = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    h = (torch.randn(T, d, generator=g) + sure * w[target.long()].float()).to(BF16)
    if ignored:
        target[torch.rand(T, generator=g) < ignored] = -1
    return h, w, target


def loss_tolerance(h, w, ref):
    """Error bound of lse and nll. Logits: products of bf16 are exact in fp32; one rounding (or truncation, 2^-23) per
    16-wide step of the accumulation, each of at most sum |h w|. Exponentials: their argument's and their own rounding,
    2^-21 together where they weigh; sums: chains of 32 + 2 in a tile, V/4096 + 5 over tiles; logarithm and last
    additions 2^-23 relative to the values."""
    d, V = h.shape[1], w.shape[0]
    zabs = (np.abs(h) @ np.abs(w).T).max(axis=1)
    tz = (d / 16 + 2) * 2.0 ** -23 * zabs
    return tz, tz + 2.0 ** -21 + (44 + V / 4096) * 2.0 ** -24 + 2.0 ** -22 * np.abs(ref["lse"])


def check_vocab(out, h, w, target, z_coef, d_loss=(1.0, 1.0), tokens=None):
    ref = O.vocab_loss(npf(h), npf(w), target.numpy(), z_coef, d_loss)
    hn, wn = npf(h), npf(w)
    tz, tl = loss_tolerance(hn, wn, ref)
    T, V = len(target), w.shape[0]
    assert int(out["n_valid"]) == ref["n_valid"]
    assert (np.abs(out["lse"] - ref["lse"]) <= tl).all()
    bad = (target.numpy() < 0) | (target.numpy() >= V)
    assert (np.abs(out["nll"] - ref["nll"]) <= tl + tz + 2.0 ** -23 * np.abs(ref["z"]).max(axis=1)).all()
    assert (out["nll"][bad] == 0).all()
    n = max(1, ref["n_valid"])
    e0 = (tl + tz)[~bad].sum() / n + 2.0 ** -18 * abs(ref["loss"][0])
    e1 = z_coef * (2 * np.abs(ref["lse"]) * tl)[~bad].sum() / n + 2.0 ** -18 * abs(ref["loss"][1])
    assert abs(out["loss"][0] - ref["loss"][0]) <= e0 + 1e-30 and abs(out["loss"][1] - ref["loss"][1]) <= e1 + 1e-30
    if "d_hidden" not in out:
        return
    # dz: half steps of half precision (2^-11, or 2^-25 of the block's maximum) and of bf16 (2^-8), what lse and the
    # logits are off, the exponentials' 2^-20
    dz = ref["dz"]
    rel = U16 + 2.0 ** -11 + 2.0 ** -20 + (2 * tl + 2 * tz)[:, None]
    scale = (abs(d_loss[0]) + 2 * z_coef * abs(d_loss[1]) * np.abs(ref["lse"])) / n
    ddz = np.abs(dz) * rel + (scale * ~bad)[:, None] * 2.0 ** -25
    # z's own coefficient b lse cancels in part with a (p - 1) at the target
    rows = np.flatnonzero(~bad)
    t = target.numpy()[rows]
    ddz[rows, t] += scale[rows] * (2.0 ** -20 + (2 * tl + 2 * tz)[rows])
    for name, other, k, want, err in [("d_hidden", np.abs(wn), V, ref["d_hidden"], lambda a: a @ np.abs(wn)),
                                      ("d_w", np.abs(hn), T, ref["d_w"], lambda a: a.T @ np.abs(hn))]:
        if name not in out:
            continue
        got = out[name]
        tol = err(ddz) + (k / 16 + 66) * 2.0 ** -23 * err(np.abs(dz)) + U16 * np.abs(want) + 1e-38
        assert (np.abs(got - want) <= tol).all(), name
        # as a whole: two independent half steps, each uniform up to 2^-8 (rms 2^-8 / 3^0.5 times the mantissas' mean 0.72
        # = 1.6e-3), are 2.3e-3 off together; 4e-3 where few values average less
        norm = np.linalg.norm(want)
        assert np.linalg.norm(got - want) <= 4e-3 * norm + 1e-37 * want.size ** 0.5, name


def run_vocab(h, w, target, z_coef=0.0, d_loss=None, backward=True, piece=None, **kw):
    T, d = h.shape
    b = train.VocabLossBuffers(T, d, w.shape[0], "cuda", backward=backward, piece=piece)
    for t in (b.loss, b.nll, b.lse):
        t.fill_(float("nan"))
    b.ws.fill_(0xff)  # NaN in every type: nothing may be used that the call has not written
    args = (b, h.cuda(), w.cuda(), target.cuda())
    if backward:
        b.d_hidden.fill_(float("nan"))
        b.d_w.fill_(float("nan"))
        dl = None if d_loss is None else torch.tensor(d_loss, dtype=F32).cuda()
        train.vocab_loss_grad(*args, z_coef=z_coef, d_loss=dl, **kw)
    else:
        train.vocab_loss(*args, z_coef=z_coef)
    torch.cuda.synchronize()
    out = {"loss": npf(b.loss), "nll": npf(b.nll), "lse": npf(b.lse), "n_valid": b.n_valid.item()}
    if backward:
        out.update({"d_hidden": npf(b.d_hidden), "d_w": npf(b.d_w)})
    return out


VOCAB_SIZES = [(1, 8, 1), (1, 64, 7), (3, 8, 129), (2, 136, 128), (37, 200, 1000), (129, 256, 256), (257, 136, 513),
               (300, 520, 4099), (255, 64, 2049), (1021, 72, 300), (5, 16, 20001), (64, 72, 20001), (65, 600, 20001), (128, 24, 19457),
               (600, 136, 9000)]


@pytest.mark.parametrize("T,d,V", VOCAB_SIZES)
def test_vocab_loss_alone(T, d, V):
    h, w, t = vocab_case(T, d, V, T + V, ignored=0.2 if T > 2 else 0.0, sure=1.0)
    out = run_vocab(h, w, t, z_coef=0.01, backward=False)
    dev_ok()
    check_vocab(out, h, w, t, 0.01)


@pytest.mark.parametrize("T,d,V", VOCAB_SIZES)
def test_vocab_loss_with_gradients(T, d, V):
    h, w, t = vocab_case(T, d, V, 2 * T + V, ignored=0.2 if T > 2 else 0.0, sure=1.0)
    out = run_vocab(h, w, t, z_coef=0.01, d_loss=(0.7, 1.9))
    dev_ok()
    check_vocab(out, h, w, t, 0.01, (0.7, 1.9))


@pytest.mark.parametrize("T,d,V", [(300, 16, 115000), (1024, 24, 130), (1500, 72, 300), (2048, 24, 130), (2049, 16, 200), (513, 64, 2000)])
def test_vocab_either_side_of_the_forms_borders(T, d, V):
    h, w, t = vocab_case(T, d, V, T + 2 * V, ignored=0.1, sure=0.5)
    out = run_vocab(h, w, t, z_coef=0.02, d_loss=(1.3, 0.4))
    alone = run_vocab(h, w, t, z_coef=0.02, backward=False)
    dev_ok()
    check_vocab(out, h, w, t, 0.02, (1.3, 0.4))
    for k in ("loss", "nll", "lse"):
        assert (out[k] == alone[k]).all(), k  # in the same order with and without gradients


@pytest.mark.parametrize("T,d,V", [(1, 128, 300), (2, 2048, 77), (3, 264, 5000), (31, 72, 1000), (32, 136, 20001)])
def test_vocab_gradients_of_few_tokens_are_rounded_once(T, d, V):
    """Up to 32 tokens: dz in two terms (2^-16 left), so that what remains beside the outputs' half step is the kept
    exponentials' 2^-11 (2^-25 of their block's maximum), exp's 2^-20 and what lse and the logits are off. The target's
    own share a (p - 1) comes from nll: 2^-20 of a and the same."""
    h, w, t = vocab_case(T, d, V, 3 * T + V, sure=0.7)
    t[1:2] = -1
    out = run_vocab(h, w, t)
    dev_ok()
    ref = O.vocab_loss(npf(h), npf(w), t.numpy(), 0.0, (1.0, 1.0))
    tz, tl = loss_tolerance(npf(h), npf(w), ref)
    ok, off = (t.numpy() >= 0), 2 * (tl + tz)
    ddz = np.abs(ref["dz"]) * (2.0 ** -16 + 2.0 ** -11 + 2.0 ** -20 + off[:, None])
    ddz[ok] += 2.0 ** -25 / ok.sum()
    ddz[ok, t.numpy()[ok]] += (2.0 ** -20 + off[ok]) / ok.sum()
    for name, k, err in [("d_hidden", V, lambda a: a @ np.abs(npf(w))), ("d_w", 64, lambda a: a.T @ np.abs(npf(h)))]:
        tol = err(ddz) + (k / 16 + 66) * 2.0 ** -23 * err(np.abs(ref["dz"])) + U16 * np.abs(ref[name]) + 1e-38
        assert (np.abs(out[name] - ref[name]) <= tol).all(), name


@pytest.mark.parametrize("piece", [1, 100, 256, 299, 300, 1000])
def test_vocab_pieces(piece):
    h, w, t = vocab_case(300, 72, 777, 5, ignored=0.3)
    whole = run_vocab(h, w, t, z_coef=0.1, backward=False)
    alone = run_vocab(h, w, t, z_coef=0.1, backward=False, piece=piece)
    for k in whole:
        np.testing.assert_array_equal(whole[k], alone[k])
    out = run_vocab(h, w, t, z_coef=0.1, piece=piece)
    dev_ok()
    for k in whole:
        np.testing.assert_array_equal(whole[k], out[k])
    check_vocab(out, h, w, t, 0.1)


def test_vocab_sure_tokens_and_large_logits():
    # logits up to ~400: p - 1 from 1e-30 to 1, exponentials that underflow in every block but one
    h, w, t = vocab_case(64, 64, 500, 3, std=8.0)
    h[:32] = (w[t[:32].long()].float() * torch.linspace(0.2, 3, 32)[:, None] * 8).to(BF16)
    out = run_vocab(h, w, t, z_coef=0.0)
    dev_ok()
    check_vocab(out, h, w, t, 0.0)


def test_vocab_equal_logits():
    h = torch.zeros(5, 16, dtype=BF16)
    w = torch.randn(1000, 16).to(BF16)
    t = torch.tensor([0, 999, 127, 128, -1], dtype=torch.int32)
    out = run_vocab(h, w, t)
    np.testing.assert_allclose(out["lse"], np.log(1000.0), rtol=1e-6)
    check_vocab(out, h, w, t, 0.0)


def test_vocab_without_targets_and_without_tokens():
    h, w, t = vocab_case(70, 64, 333, 9)
    t[:] = -100
    out = run_vocab(h, w, t, z_coef=0.5)
    assert out["n_valid"] == 0 and (out["loss"] == 0).all() and (out["nll"] == 0).all()
    assert (out["d_hidden"] == 0).all() and (out["d_w"] == 0).all()
    check_vocab(out, h, w, t, 0.5)
    out = run_vocab(h[:0], w, t[:0], z_coef=0.5)
    assert out["n_valid"] == 0 and (out["loss"] == 0).all() and (out["d_w"] == 0).all()
    dev_ok()


def test_vocab_target_out_of_range():
    h, w, t = vocab_case(40, 64, 333, 11)
    t[7], t[39] = 333, 2 ** 31 - 1
    out = run_vocab(h, w, t, z_coef=0.2)
    assert L.moe_device_error(clear=True) == 7
    check_vocab(out, h, w, t, 0.2)
    assert (out["d_hidden"][[7, 39]] == 0).all()


def test_vocab_nan_stays_with_its_token():
    h, w, t = vocab_case(300, 64, 333, 13)
    good = run_vocab(h, w, t, backward=False)
    h2 = h.clone()
    h2[17, 3] = float("nan")
    h2[260, 0] = float("inf")
    t2 = t.clone()
    t2[17] = t2[260] = -1
    out = run_vocab(h2, w, t2, backward=False)
    keep = np.ones(300, bool)
    keep[[17, 260]] = False
    np.testing.assert_array_equal(out["lse"][keep], good["lse"][keep])
    assert np.isnan(out["lse"][[17, 260]]).all() and (out["nll"][[17, 260]] == 0).all()
    assert np.isfinite(out["loss"]).all()
    dev_ok()


def test_vocab_logits_of_minus_infinity():
    # entries that no token can have: the target's own gives an infinite nll, lse is the others'
    h = torch.ones(4, 8, dtype=BF16)
    w = torch.randn(300, 8, generator=torch.Generator().manual_seed(1)).to(BF16)
    w[[5, 200, 299]] = float("-inf")
    t = torch.tensor([5, 6, 299, -1], dtype=torch.int32)
    out = run_vocab(h, w, t, backward=False)
    keep = [i for i in range(300) if i not in (5, 200, 299)]
    ref = O.vocab_loss(npf(h), npf(w[keep]), np.array([-1, 5, -1, -1]))
    np.testing.assert_allclose(out["lse"], ref["lse"], rtol=1e-6)
    assert np.isposinf(out["nll"][[0, 2]]).all() and out["nll"][3] == 0 and np.isposinf(out["loss"][0])
    np.testing.assert_allclose(out["nll"][1], ref["nll"][1], rtol=1e-5)
    dev_ok()


def test_vocab_sure_tokens_keep_their_digits():
    # nll from 4e-6 to 0.9: z_t is off by (d / 16 + 2) 2^-23 sum |h w| as the others are, their difference by twice that, and
    # nll by as much relative to itself (d nll / d (z_t - z_v) <= nll); exponentials and sums 2^-19 more
    d, V = 64, 400
    g = torch.Generator().manual_seed(4)
    w = (torch.randn(V, d, generator=g) * 0.1).to(BF16)
    t = torch.arange(24, dtype=torch.int32)
    u = w[:24].float()
    h = (u / u.square().sum(1, keepdim=True) * torch.linspace(6, 22, 24)[:, None]).to(BF16)
    ref = O.vocab_loss(npf(h), npf(w), t.numpy())
    assert ref["nll"].min() < 1e-5
    out = run_vocab(h, w, t)
    dev_ok()
    tz, _ = loss_tolerance(npf(h), npf(w), ref)
    assert (np.abs(out["nll"] - ref["nll"]) <= ref["nll"] * (2 * tz + 2.0 ** -19)).all()
    check_vocab(out, h, w, t, 0.0)


def test_vocab_one_gradient_alone():
    h, w, t = vocab_case(200, 64, 777, 21)
    both = run_vocab(h, w, t)
    only_h = run_vocab(h, w, t, need_w=False)
    only_w = run_vocab(h, w, t, need_hidden=False)
    np.testing.assert_array_equal(both["d_hidden"], only_h["d_hidden"])
    np.testing.assert_array_equal(both["d_w"], only_w["d_w"])
    assert np.isnan(only_h["d_w"]).all() and np.isnan(only_w["d_hidden"]).all()
    dev_ok()


def test_vocab_gradient_against_differences():
    h, w, t = vocab_case(24, 32, 200, 31)
    z = 0.05
    out = run_vocab(h, w, t, z_coef=z)
    g = np.random.default_rng(0)
    # along random directions the oracle's loss (both parts) changes by the gradient's product with them
    for name, base in [("d_hidden", npf(h)), ("d_w", npf(w))]:
        v = g.standard_normal(base.shape)
        e = 1e-5
        a = [(base + s * e * v) for s in (1, -1)]
        f = [O.vocab_loss(x, npf(w), t.numpy(), z)["loss"].sum() if name == "d_hidden"
             else O.vocab_loss(npf(h), x, t.numpy(), z)["loss"].sum() for x in a]
        diff = (f[0] - f[1]) / (2 * e)
        # the product's terms are 2^-8 + 2^-8 off each; differences ~1e-9
        assert abs((out[name] * v).sum() - diff) <= 2 * U16 * (np.abs(out[name]) * np.abs(v)).sum() / v.size ** 0.5 * 4 + 1e-8


def test_vocab_captured_and_replayed_on_another_stream():
    h, w, t = vocab_case(130, 64, 777, 41, ignored=0.1)
    want = run_vocab(h, w, t, z_coef=0.1)
    b = train.VocabLossBuffers(130, 64, 777, "cuda")
    gh, gw, gt = torch.zeros_like(h).cuda(), w.cuda(), t.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        train.vocab_loss_grad(b, gh, gw, gt, z_coef=0.1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            train.vocab_loss_grad(b, gh, gw, gt, z_coef=0.1)
        gh.copy_(h)
        graph.replay()
        graph.replay()
    s.synchronize()
    for k in ("loss", "nll", "lse", "d_hidden", "d_w"):
        np.testing.assert_array_equal(npf(getattr(b, k)), want[k])
    dev_ok()


# ---------------------------------------------------------------- orthogonalised update


def stack(n, rows, cols, seed, kind="tokens"):
    g = torch.Generator().manual_seed(seed)
    if kind == "gauss":
        x = torch.randn(n, rows, cols, generator=g)
    elif kind == "rank1":
        x = torch.randn(n, rows, 1, generator=g) @ torch.randn(n, 1, cols, generator=g)
    else:
        x = torch.randn(n, rows, 40, generator=g) @ torch.randn(n, 40, cols, generator=g)
        x = x * torch.exp(torch.randn(1, 1, cols, generator=g)) * 1e-3
    return x.to(BF16)


def run_orth(g, batch=None, mask=None, out=None, **kw):
    n, rows, cols = g.shape
    b = train.MuonBuffers(n, rows, cols, "cuda", batch=batch)
    b.ws.fill_(0xff)
    gd = g.cuda()
    out = torch.full_like(gd, float("nan")) if out is None else out
    train.orthogonalize(b, gd, out, active_mask=mask, **kw)
    dev_ok()
    return out.cpu()


def orth_bound(g, coef=(3.4445, -4.7750, 2.0315), steps=5, eps=1e-7):
    """Largest possible 2-norm of the result's error. With h = 2^-11 (half a step of half precision, relative): X enters
    the products h off, A is then 2h + h, B = b A + c A A is 3h + h and 6h + h off in its parts, B X another h: 5h and 8h
    of |b| |X|^2 |X|_F and |c| |X|^4 |X|_F a step. An error e of X grows by the largest |p'| or |p(s) / s| over the
    singular values s (the polynomial acts on them). In the end half a step of bf16."""
    x = npf(g)
    s = np.linalg.svd(x / (np.linalg.norm(x) + eps), compute_uv=False)
    h, e = 2.0 ** -11, 0.0
    for a, b, c in ([coef] * steps if np.isscalar(coef[0]) else coef):
        top = s.max() + e
        grow = max(np.abs(a + b * s ** 2 + c * s ** 4).max(), np.abs(a + 3 * b * s ** 2 + 5 * c * s ** 4).max())
        e = grow * e + h * (5 * abs(b) * top ** 2 + 8 * abs(c) * top ** 4) * np.linalg.norm(s)
        s = np.abs(a * s + b * s ** 3 + c * s ** 5)
    return e + U16 * (np.linalg.norm(s) + e)


def check_orth(got, g, **kw):
    """One rounding to bf16 (rms 1.65e-3 of the values) and the products' half-precision operands: simulated with those
    roundings on spectra flat, decaying to 1e-4, and of rank 16 to 200 in 256 x 512 to 512 x 1,792: 4e-4 to 1.3e-3.
    Together 2.1e-3; the bar leaves two fifths. Largest: 8 rms of either. A matrix of fewer than 1,000 values does not
    average over its roundings (one value: all of them may point one way): orth_bound."""
    for i in range(g.shape[0]):
        ref = O.newton_schulz(npf(g[i]), **kw)
        d = npf(got[i]) - ref
        norm = np.linalg.norm(ref)
        if ref.size < 1000:
            assert np.linalg.norm(d) <= orth_bound(g[i], **kw), (i, np.linalg.norm(d) / norm)
            continue
        assert np.linalg.norm(d) <= 3e-3 * norm, (i, np.linalg.norm(d) / norm)
        rms = norm / ref.size ** 0.5
        assert np.abs(d).max() <= U16 * np.abs(ref).max() + 8 * 1.5e-3 * max(rms, np.abs(ref).max() / 8)


@pytest.mark.parametrize("n,rows,cols", [(1, 1, 1), (2, 1, 64), (2, 40, 1), (3, 16, 24), (3, 33, 7), (2, 65, 130), (2, 256, 256),
                                         (2, 256, 512), (2, 512, 256), (1, 257, 300), (1, 300, 257), (1, 129, 1030),
                                         (1, 1030, 129), (1, 515, 640), (1, 128, 384), (2, 128, 385), (1, 2999, 100), (1, 100, 3000),
                                         (40, 17, 700), (90, 64, 90), (1, 128, 3100), (1, 127, 6000)])
@pytest.mark.parametrize("kind", ["gauss", "tokens"])
def test_orthogonalize(n, rows, cols, kind):
    g = stack(n, rows, cols, rows + cols, kind)
    check_orth(run_orth(g), g)


@pytest.mark.parametrize("rows,cols", [(96, 200), (200, 96), (300, 300)])
def test_orthogonalize_rank_one(rows, cols):
    g = stack(2, rows, cols, 1, "rank1")
    check_orth(run_orth(g), g)


@pytest.mark.parametrize("n,rows,cols", [(2, 40, 5000), (1, 5001, 100), (2, 128, 6144), (1, 6144, 16), (1, 33, 6145), (3, 3100, 64),
                                         (20, 128, 3500), (1, 65, 3329)])
def test_orthogonalize_long_and_narrow(n, rows, cols):
    g = stack(n, rows, cols, n + cols)
    check_orth(run_orth(g), g)


def test_orthogonalize_coefficients_and_steps():
    g = stack(2, 70, 90, 3, "gauss")
    check_orth(run_orth(g, steps=1), g, steps=1)
    rows = [(4.0, -6.0, 2.5), (3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5)]
    check_orth(run_orth(g, coef=rows, steps=3), g, coef=rows, steps=3)
    check_orth(run_orth(g, coef=(2.0, -1.5, 0.5), steps=7), g, coef=(2.0, -1.5, 0.5), steps=7)


def test_orthogonalize_sizes_of_the_values():
    # values from 2^-120 to 2^126: the result does not depend on their size, and eps counts where it is larger
    g = stack(3, 48, 80, 5, "gauss")
    want = run_orth(g, eps=1e-37)
    for e in (-115, -70, 60, 123):
        got = run_orth((g.float() * 2.0 ** e).to(BF16), eps=1e-37)
        # eps is below the norms here and the power of two exact: only eps's share, 1e-37 / 2^-115 = 4e-3 at most, differs
        d = (got.double() - want.double()).norm() / want.double().norm()
        assert d <= (5e-3 if e == -115 else 0), e
    small = (g.float() * 2.0 ** -40).to(BF16)
    got, ref = run_orth(small, eps=1e-7), O.newton_schulz(npf(small[0]), eps=1e-7)
    assert np.linalg.norm(npf(got[0]) - ref) <= 4e-3 * np.linalg.norm(ref)


def test_orthogonalize_zero_and_nan_matrices():
    g = stack(5, 40, 72, 7)
    want = run_orth(g)
    g2 = g.clone()
    g2[1] = 0
    g2[2, 3, 5] = float("nan")
    g2[4, 39, 71] = float("inf")
    got = run_orth(g2)
    assert torch.equal(got[[0, 3]], want[[0, 3]])
    assert (got[1] == 0).all() and torch.isnan(got[2]).all() and torch.isnan(got[4]).all()


@pytest.mark.parametrize("batch", [1, 3, 8])
def test_orthogonalize_mask_batches_and_in_place(batch):
    g = stack(8, 72, 100, 9)
    want = run_orth(g)
    mask = torch.tensor([1, 0, 0, 1], dtype=torch.uint8).cuda()
    out = torch.full_like(g, 7.0).cuda()
    got = run_orth(g, batch=batch, mask=mask, out=out)
    live = torch.tensor([0, 1, 6, 7])
    assert torch.equal(got[live], want[live]) and (got[2:6] == 7.0).all()
    b = train.MuonBuffers(8, 72, 100, "cuda", batch=batch)
    gd = g.cuda()
    train.orthogonalize(b, gd, gd, active_mask=mask)
    dev_ok()
    assert torch.equal(gd.cpu()[live], want[live]) and torch.equal(gd.cpu()[2:6], g[2:6])
    gd = g.cuda()
    train.orthogonalize(b, gd, gd, active_mask=torch.zeros(4, dtype=torch.uint8).cuda())
    dev_ok()
    assert torch.equal(gd.cpu(), g)


@pytest.mark.parametrize("rows,cols,nesterov,use_master", [(40, 72, True, False), (72, 40, False, True), (33, 65, True, True),
                                                           (65, 33, True, False), (256, 264, False, False)])
def test_muon_step(rows, cols, nesterov, use_master):
    check_muon_step(rows, cols, nesterov, use_master, lambda length, n: 8 * 1.5e-3 * length / n ** 0.5)


def check_muon_step(rows, cols, nesterov, use_master, bar):
    n = 6
    rng = torch.Generator().manual_seed(rows)
    w0 = (torch.randn(n, rows, cols, generator=rng) * 0.02)
    grad, m0 = stack(n, rows, cols, 3), stack(n, rows, cols, 4).float() * 3 + 1e-4
    mask = torch.tensor([1, 0, 1], dtype=torch.uint8).cuda()
    w, m = w0.to(BF16).cuda(), m0.clone().cuda()
    master = w0.clone().cuda() if use_master else None
    b = train.MuonBuffers(n, rows, cols, "cuda", batch=4)
    kw = dict(lr=0.02, weight_decay=0.1, mu=0.9, nesterov=nesterov, scale=2.0)
    start = w0 if use_master else w0.to(BF16).float()
    train.muon_step(b, w, grad.cuda(), m, active_mask=mask, master=master, **kw)
    dev_ok()
    for i in range(n):
        if i // 2 == 1:
            assert torch.equal(w[i].cpu(), w0[i].to(BF16)) and torch.equal(m[i].cpu(), m0[i])
            continue
        rw, rm = O.muon_step(npf(start[i]), npf(grad[i]), npf(m0[i]), **kw)
        assert np.abs(npf(m[i]) - rm).max() <= 2.0 ** -23 * (np.abs(rm).max() + np.abs(npf(m0[i])).max())
        o = (start[i].double().numpy() * (1 - 0.002) - rw) / 0.04  # the update itself
        # The update is 1.5e-3 off (see check_orth). Every step multiplies the vectors along the short side: X' = P X, or
        # X P where rows > cols, so that the error of such a vector x is dP x + P dx, in proportion to its own length
        # (lengths differ: the gradients' features do): 8 times its rms at most, and the weight's roundings.
        short = 0 if rows <= cols else 1
        tol = 0.04 * bar(np.linalg.norm(o, axis=short, keepdims=True), min(rows, cols))
        if use_master:
            assert (np.abs(npf(master[i]) - rw) <= tol + 2.0 ** -22 * np.abs(rw).max()).all()
            assert torch.equal(w[i], master[i].to(BF16))
        else:
            assert (np.abs(npf(w[i]) - rw) <= tol + U16 * np.abs(rw) + 1e-9).all()


@pytest.mark.parametrize("rows,cols,nesterov,use_master", [(24, 4100, True, True), (4104, 100, True, False), (4099, 65, False, True),
                                                           (128, 5000, True, False)])
def test_muon_step_long_and_narrow(rows, cols, nesterov, use_master):
    """A value's error is at most its vector's, |e_j| <= |e|, and that 1.5e-3 of the vector's length, twice for a vector
    that is worse off than most (check_orth's bar for the whole): 3e-3 |o|. No value's share of |e| is assumed: over
    thousands of vectors some value has more than 8 rms of it where the error lies in few values (the products' roundings
    are relative to the operands' values, which differ as the features do)."""
    check_muon_step(rows, cols, nesterov, use_master, lambda length, n: 3e-3 * length)


def test_muon_captured_and_replayed():
    g, m, w = stack(4, 130, 72, 3), stack(4, 130, 72, 4).float(), stack(4, 130, 72, 5, "gauss")
    want_w, want_m = w.cuda(), m.cuda()
    b = train.MuonBuffers(4, 130, 72, "cuda")
    for _ in range(2):
        train.muon_step(b, want_w, g.cuda(), want_m, lr=0.1)
    gd, md, wd = g.cuda(), m.cuda(), w.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        train.muon_step(b, wd, gd, md, lr=0.1)
    graph.replay()
    graph.replay()
    dev_ok()
    assert torch.equal(wd, want_w) and torch.equal(md, want_m)


@pytest.mark.parametrize("form", [{"MOE_MUON_SMALL": "0", "MOE_DENSE_SMALL": "0"}, {"MOE_MUON_SMALL": "0", "MOE_DENSE_SMALL": "1"},
                                  {"MOE_MUON_SMALL": "1"}])
def test_other_forms_of_the_updates(form):
    """The tests above with each form of the products forced (the variables are read once, so in a child process)."""
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-p", "no:cacheprovider", "-k",
                        "orthogonalize or muon_step or muon_captured", os.path.abspath(__file__)],
                       env={**os.environ, **form}, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:]


# ---------------------------------------------------------------- together


def test_training_steps_of_a_small_model():
    """hidden -> expert layer -> vocabulary loss, its gradient back through the layer, Muon on the experts: against the
    oracle's step on the same routing."""
    T, d, E, k, F, V = 200, 128, 8, 2, 256, 500
    gen = torch.Generator().manual_seed(0)
    x = torch.randn(T, d, generator=gen).to(BF16)
    wr = torch.randn(d, E, generator=gen) / d ** 0.5
    wgu = (torch.randn(E, 2 * F, d, generator=gen) * 0.05).to(BF16)
    wdn = (torch.randn(E, d, F, generator=gen) * 0.05).to(BF16)
    wv = (torch.randn(V, d, generator=gen) * 0.2).to(BF16)
    target = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    mask = torch.ones(E, dtype=torch.uint8)
    mask[3] = 0
    s = layer.LayerShape(T, d, E, k, F)
    b = layer.MoELayerBuffers(s, "cuda")
    vb = train.VocabLossBuffers(T, d, V, "cuda")
    gu, dn = train.MuonBuffers(2 * E, F, d, "cuda"), train.MuonBuffers(E, d, F, "cuda")
    c = {n: t.cuda() for n, t in dict(x=x, wr=wr, wgu=wgu, wdn=wdn, wv=wv, target=target, mask=mask).items()}
    m_gu, m_dn = torch.zeros(E, 2 * F, d, device="cuda"), torch.zeros(E, d, F, device="cuda")
    y = layer.forward(b, c["x"], c["wr"], None, c["wgu"], c["wdn"], c["mask"], keep_logits=True)
    loss, dy, _ = train.vocab_loss_grad(vb, y, c["wv"], c["target"])
    b.dw_gate_up.fill_(float("nan"))  # (pruned experts' gradients are not written, nor read by the step)
    b.dw_down.fill_(float("nan"))
    dx, dgu, ddn, dr = layer.backward(b, dy, c["wr"], c["wgu"], c["wdn"], active_mask=c["mask"])
    train.muon_step(gu, c["wgu"], dgu, m_gu, lr=0.1, active_mask=c["mask"])
    train.muon_step(dn, c["wdn"], ddn, m_dn, lr=0.1, active_mask=c["mask"])
    dev_ok()
    ref = O.moe_layer(npf(x), npf(wr), None, mask.numpy(), k, npf(wgu), npf(wdn), dy=npf(dy), logits32=b.logits.cpu().numpy())
    lr_ = O.vocab_loss(npf(y), npf(wv), target.numpy())
    assert abs(loss[0].item() - lr_["loss"][0]) <= 1e-4
    for got, want in [(y, ref["y"]), (dy, lr_["d_hidden"]), (dx, ref["dx"])]:
        assert np.abs(npf(got) - want).max() <= 2e-2 * np.abs(want).max()
    # the weights' step from the gradients that the layer gave
    for w0, w1, g, mats in [(wgu, c["wgu"], dgu, 2), (wdn, c["wdn"], ddn, 1)]:
        w0, w1, g = (npf(t).reshape(E * mats, -1, t.shape[-1]) for t in (w0, w1, g))
        for i in range(E * mats):
            if i // mats == 3:
                assert (w1[i] == w0[i]).all()
                continue
            rw, _ = O.muon_step(w0[i], g[i], 0 * g[i], lr=0.1, scale=0.2 * max(g.shape[1:]) ** 0.5)
            assert np.linalg.norm(w1[i] - rw) <= 3e-3 * np.linalg.norm(rw)
    assert (m_gu[3] == 0).all() and (m_dn[3] == 0).all()
