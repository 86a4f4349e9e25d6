"""Measured operators at the two ends of a training step around the expert layer: the vocabulary loss that
the layer's output gradient comes from, and the orthogonalised update that the experts' gradients go into.

What a training program calls, in four kinds of case:
  loss  train.vocab_loss: cross entropy over the vocabulary and its z-loss, no gradient (validation, scoring)
  grad  train.vocab_loss_grad: the same with the gradients of the hidden states and of the vocabulary's weight
  orth  train.orthogonalize: Newton-Schulz products over a stack of gradients
  muon  train.muon_step: momentum, its orthogonalised update, new weights
`own` false: the same results from elementary torch operations in 32 bits. `own` true: the framework's calls.
Inputs are synthetic and seeded.

A case of the losses: T tokens, d = d_model, V vocabulary entries, ignored (share of the tokens without a
target), z_coef. A case of the updates: E experts, per matrices of rows x cols to an expert, pruned (experts
masked out), rank (of the gradients' main part: tokens that reached the expert).
"""
import math

import torch

own = False

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
COEF, STEPS, EPS = (3.4445, -4.7750, 2.0315), 5, 1e-7
LR, DECAY, MU = 2e-3, 0.1, 0.95


def _loss(name, kind, T, d, V, ignored=0.0, z_coef=0.0):
    c = {"kind": kind, "T": T, "d": d, "V": V, "ignored": ignored, "z_coef": z_coef}
    return {"name": name, **c} if name else c


def _update(name, kind, E, per, rows, cols, pruned=0, rank=256):
    c = {"kind": kind, "E": E, "per": per, "rows": rows, "cols": cols, "pruned": pruned, "rank": rank}
    return {"name": name, **c} if name else c


def listed():
    return [
        # ---- the loss alone
        # scoring one short answer: the weight's 131 MB and the launches count
        _loss("loss_few_tokens", "loss", 37, 2048, 32000),
        # a validation batch of ragged length, a vocabulary of odd size
        _loss("loss_ragged", "loss", 2039, 1024, 50257, ignored=0.1, z_coef=1e-4),
        # a validation batch at the large layer's width
        _loss("loss_large", "loss", 8192, 7168, 129280),
        # ---- with both gradients
        # a small model's micro-batch
        _loss("grad_small", "grad", 512, 512, 32000, z_coef=1e-4),
        # a micro-batch of ragged length, prompts left out of the loss
        _loss("grad_ragged", "grad", 2039, 2048, 50257, ignored=0.3),
        # a training step's tokens at the width of the 64-expert layer
        _loss("grad_large", "grad", 16384, 4096, 131072, z_coef=1e-4),
        # ---- the orthogonalised update alone
        # the smallest layer's down projections: launches and latency count
        _update("orth_small", "orth", 16, 1, 256, 512),
        # odd sizes; few tokens reached the expert
        _update("orth_odd", "orth", 5, 1, 1021, 333, rank=64),
        # the down projections of the 64-expert layer, 16 experts pruned
        _update("orth_large", "orth", 64, 1, 4096, 2048, pruned=16),
        # ---- with momentum and weights
        # gate and up projections of a small model's experts
        _update("muon_small", "muon", 32, 2, 384, 512),
        # gate and up projections of the skewed 64-expert layer
        _update("muon_mid", "muon", 64, 2, 1408, 2048, rank=700),
        # of the 64-expert layer, 16 experts pruned
        _update("muon_large", "muon", 64, 2, 2048, 4096, pruned=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithms."""
    top = {c["kind"]: work(c) for c in listed()}  # the last of a kind is its largest
    while True:
        kind = rng.choice(("loss", "grad", "grad", "orth", "muon"))
        if kind in ("loss", "grad"):
            c = _loss("", kind, _log_int(rng, 1, 16384), 8 * _log_int(rng, 16, 896), _log_int(rng, 1000, 151936),
                      rng.choice((0.0, 0.1, 0.5)), rng.choice((0.0, 1e-4)))
        else:
            E = _log_int(rng, 1, 64)
            c = _update("", kind, E, rng.choice((1, 2)), _log_int(rng, 16, 7168), _log_int(rng, 16, 7168),
                        rng.choice((0, E // 4)), _log_int(rng, 32, 1024))
        w, m = work(c), top[kind]
        if w["bytes"] <= m["bytes"] and w["flops"] <= m["flops"]:
            return c


# ---------------------------------------------------------------- inputs


def _randn(g, *shape, std=1.0, dtype=BF16):
    return torch.empty(*shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _prepare_loss(c, g):
    T, d, V = c["T"], c["d"], c["V"]
    w = _randn(g, V, d, std=2.0 / math.sqrt(d))
    # targets as frequent as words are (1 / rank), in any order of the ids
    u = torch.rand(T, generator=g, device="cuda", dtype=F64)
    target = torch.randperm(V, generator=g, device="cuda")[torch.exp(u * math.log(V)).long().clamp(max=V - 1)]
    # hidden states that predict their target, some not at all and some almost surely
    sure = 6.0 * torch.rand(T, 1, generator=g, device="cuda") / math.sqrt(d)
    h = (_randn(g, T, d, dtype=F32) + sure * w[target].float() * math.sqrt(d)).to(BF16)
    if c["ignored"]:
        target[torch.rand(T, generator=g, device="cuda") < c["ignored"]] = -1
    s = {"case": c, "h": h, "w": w, "target": target.to(I32),
         "d_loss": torch.rand(2, generator=g, device="cuda") + 0.5}
    if own:
        from paper_2601_14327_gb300 import train
        s["b"] = train.VocabLossBuffers(T, d, V, "cuda", backward=c["kind"] == "grad")
    return s


def _gradient(c, g):
    """Gradients of a stack of matrices: products of the tokens that reached the expert, features of unequal size."""
    n, r, k = c["E"] * c["per"], c["rank"], c["cols"]
    scale = torch.exp(_randn(g, 1, 1, k, dtype=F32))
    return (_randn(g, n, c["rows"], r, std=1e-2) @ (_randn(g, n, r, k, dtype=F32) * scale).to(BF16)).to(BF16)


def _prepare_update(c, g):
    n, E = c["E"] * c["per"], c["E"]
    s = {"case": c, "g": _gradient(c, g), "mask": None}
    if c["pruned"]:
        s["mask"] = torch.ones(E, dtype=torch.uint8, device="cuda")
        s["mask"][torch.randperm(E, generator=g, device="cuda")[:c["pruned"]]] = 0
    if c["kind"] == "muon":
        s["w"] = _randn(g, n, c["rows"], c["cols"], std=0.02)
        s["m"] = _gradient(c, g).float() * 5 + _gradient(c, g).float()
        s["scale"] = 0.2 * math.sqrt(max(c["rows"], c["cols"]))
    else:
        s["out"] = torch.zeros_like(s["g"])
    if own:
        from paper_2601_14327_gb300 import train
        s["b"] = train.MuonBuffers(n, c["rows"], c["cols"], "cuda")
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (_prepare_loss if case["kind"] in ("loss", "grad") else _prepare_update)(case, g)


# ---------------------------------------------------------------- the framework's calls


def _own(s):
    from paper_2601_14327_gb300 import train
    c = s["case"]
    if c["kind"] in ("loss", "grad"):
        b = s["b"]
        if c["kind"] == "loss":
            train.vocab_loss(b, s["h"], s["w"], s["target"], z_coef=c["z_coef"])
            return {"loss": b.loss, "nll": b.nll, "lse": b.lse, "n_valid": b.n_valid}
        train.vocab_loss_grad(b, s["h"], s["w"], s["target"], z_coef=c["z_coef"], d_loss=s["d_loss"])
        return {"loss": b.loss, "nll": b.nll, "lse": b.lse, "n_valid": b.n_valid, "d_hidden": b.d_hidden,
                "d_w": b.d_w}
    if c["kind"] == "orth":
        return train.orthogonalize(s["b"], s["g"], s["out"], active_mask=s["mask"], coef=COEF, steps=STEPS, eps=EPS)
    train.muon_step(s["b"], s["w"], s["g"], s["m"], lr=LR, weight_decay=DECAY, mu=MU, nesterov=True,
                    scale=s["scale"], active_mask=s["mask"], coef=COEF, steps=STEPS, eps=EPS)
    return {"w": s["w"], "momentum": s["m"]}


# ---------------------------------------------------------------- plain forms


def _plain_loss(s):
    c, t = s["case"], s["target"].long()
    h, w = s["h"].float(), s["w"].float()
    z = h @ w.T
    top = z.amax(1, keepdim=True)
    at = t.clamp(min=0)[:, None]
    ok = t >= 0
    zt = z.gather(1, at)[:, 0]
    e = z.sub_(top).exp_()
    total = e.sum(1)
    lse = top[:, 0] + torch.log(total)
    nll = torch.where(ok, lse - zt, 0.0)
    n = ok.sum()
    m = n.clamp(min=1)
    loss = torch.stack((nll.double().sum() / m, c["z_coef"] * torch.where(ok, lse, 0.0).double().square().sum() / m))
    out = {"loss": loss.float(), "nll": nll, "lse": lse, "n_valid": n[None].to(I32)}
    if c["kind"] == "loss":
        return out
    a = s["d_loss"][0] / m
    b = s["d_loss"][1] * (2 * c["z_coef"]) / m * lse
    dz = e.mul_(torch.where(ok, (a + b) / total, 0.0)[:, None])
    # p - 1 at the target without what the difference loses
    back = torch.where(ok, a * torch.expm1(-nll) + b * torch.exp(-nll), 0.0)
    dz.scatter_(1, at, back[:, None])
    out["d_hidden"], out["d_w"] = (dz @ w).to(BF16), (dz.T @ h).to(BF16)
    return out


def _orthogonal(u):
    """fp32 [n, rows, cols] -> the Newton-Schulz products of each matrix."""
    x = u / (u.double().square().sum((1, 2), keepdim=True).sqrt().float() + EPS)
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    for _ in range(STEPS):
        a = x @ x.transpose(1, 2)
        x = COEF[0] * x + (COEF[1] * a + COEF[2] * (a @ a)) @ x
    return x.transpose(1, 2) if tall else x


def _live(s):
    """Indices of the matrices that are updated."""
    c = s["case"]
    mask = torch.ones(c["E"], dtype=torch.uint8, device="cuda") if s["mask"] is None else s["mask"]
    return torch.nonzero(mask.repeat_interleave(c["per"]))[:, 0]


def _plain_orth(s):
    at = _live(s)
    s["out"][at] = _orthogonal(s["g"][at].float()).to(BF16)
    return s["out"]


def _plain_muon(s):
    at = _live(s)
    g = s["g"][at].float()
    m = MU * s["m"][at] + g
    s["m"][at] = m
    step = _orthogonal(g + MU * m)
    s["w"][at] = (s["w"][at].float() * (1 - LR * DECAY) - LR * s["scale"] * step).to(BF16)
    return {"w": s["w"], "momentum": s["m"]}


def run(s):
    if own:
        return _own(s)
    return {"loss": _plain_loss, "grad": _plain_loss, "orth": _plain_orth, "muon": _plain_muon}[s["case"]["kind"]](s)


# ---------------------------------------------------------------- what a pass needs


def work(case):
    """Bytes with every input read once and every output written once, and the operations (of symmetric products
    one half)."""
    c = case
    if c["kind"] in ("loss", "grad"):
        T, d, V = c["T"], c["d"], c["V"]
        twice = 2 if c["kind"] == "grad" else 1
        return {"bytes": 2 * (T + V) * d * twice + 12 * T, "flops": (6 if c["kind"] == "grad" else 2) * T * V * d}
    n, k = min(c["rows"], c["cols"]), max(c["rows"], c["cols"])
    mats = (c["E"] - c["pruned"]) * c["per"]
    return {"bytes": mats * n * k * (14 if c["kind"] == "muon" else 4), "flops": mats * STEPS * (3 * n * n * k + n ** 3)}


# ---------------------------------------------------------------- in 64 bits, from the definitions


def _exact_loss(s):
    c = s["case"]
    T, V = c["T"], c["V"]
    w, grad = s["w"].double(), c["kind"] == "grad"
    lse, nll = (torch.zeros(T, dtype=F64, device="cuda") for _ in range(2))
    target = s["target"].long()
    counted = [int(t) for t in torch.nonzero(target >= 0)[:, 0].tolist()]
    m = max(1, len(counted))
    d0, d1 = (float(v) / m for v in s["d_loss"].double())
    dh = torch.zeros(T, c["d"], dtype=F64, device="cuda") if grad else None
    dw = torch.zeros(V, c["d"], dtype=F64, device="cuda") if grad else None
    for lo in range(0, T, 1024):
        r = slice(lo, min(T, lo + 1024))
        x, t = s["h"][r].double(), target[r]
        logp = x @ w.T
        lse[r] = torch.logsumexp(logp, 1)
        logp -= lse[r][:, None]
        has = t >= 0
        rows = torch.nonzero(has)[:, 0]
        nll[r][rows] = -logp[rows, t[rows]]
        if grad:
            p = torch.exp(logp)
            dz = p * (2 * c["z_coef"] * d1 * lse[r][:, None] + d0)
            dz[rows, t[rows]] = 2 * c["z_coef"] * d1 * lse[r][rows] * p[rows, t[rows]] + d0 * torch.expm1(-nll[r][rows])
            dz[~has] = 0
            dh[r] = dz @ w
            dw += dz.T @ x
    z2 = lse[target >= 0].square().sum()
    out = {"loss": torch.stack((nll.sum() / m, c["z_coef"] * z2 / m)), "nll": nll, "lse": lse,
           "n_valid": torch.tensor([len(counted)], dtype=I32, device="cuda")}
    return {**out, "d_hidden": dh, "d_w": dw} if grad else out


def _exact_orthogonal(u):
    """One matrix in 64 bits, the products taken from the side that the rows are on or not, whichever is short."""
    x = u / (torch.linalg.vector_norm(u) + EPS)
    a, b, c = COEF
    eye = torch.eye(min(x.shape), dtype=F64, device=x.device)
    for _ in range(STEPS):
        gram = x.T @ x if x.shape[0] > x.shape[1] else x @ x.T
        poly = a * eye + gram @ (b * eye + c * gram)
        x = x @ poly if x.shape[0] > x.shape[1] else poly @ x
    return x


def _exact_update(s):
    c = s["case"]
    muon = c["kind"] == "muon"
    out = {"w": s["w"].double(), "momentum": s["m"].double()} if muon else s["out"].double()
    for i in range(c["E"] * c["per"]):
        if s["mask"] is not None and not int(s["mask"][i // c["per"]]):
            continue
        g = s["g"][i].double()
        if muon:
            m = out["momentum"][i] * MU + g
            out["momentum"][i] = m
            out["w"][i] -= LR * (DECAY * out["w"][i] + s["scale"] * _exact_orthogonal(g + MU * m))
        else:
            out[i] = _exact_orthogonal(g)
    return out


def exact(case, seed):
    if work(case)["flops"] > 8e12:
        return None
    s = prepare(case, seed)
    return (_exact_loss if case["kind"] in ("loss", "grad") else _exact_update)(s)
