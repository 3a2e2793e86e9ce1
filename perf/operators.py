"""Scoring of tokens, its gradient, and the update made of a gradient, as cases that can be timed and compared.

Four kinds of work:

  score   log-probs, entropy and the top alternatives of tokens whose logits exist;
  grad    the same, then the gradient with respect to the logits, as a training step takes it;
  head    log-probs and entropy from hidden states and the LM head ("forward"), or with the gradients of
          both ("train"): the logits are the operator's own;
  update  a weight gradient orthogonalised ("orthogonalize"), or the whole momentum step on the weights ("muon").

Where `own` is false, `run` computes the plain form in 32 bits with elementary torch operations; where it is true,
it makes the calls of `paper_2509_13232_amd.binding`.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
HIDDEN, VOCAB = 4096, 151936                   # the large LM head of this repository's configurations
ENTROPY_WEIGHT = 0.01
COEFFS, STEPS, EPS = (3.4445, -4.7750, 2.0315), 5, 1e-7
LR, MOMENTUM, WEIGHT_DECAY = 2e-3, 0.95, 0.1


def _score(name, dtype, T, V, K, mask=0.0, pad=0):
    """K: alternatives per token; mask: share of tokens left out; pad: columns behind the vocabulary in the logits' rows."""
    return dict(name=name, kind="score", dtype=dtype, T=T, V=V, K=K, mask=mask, pad=pad)


def _grad(name, dtype, T, V, K, mask=0.0):
    return dict(name=name, kind="grad", dtype=dtype, T=T, V=V, K=K, mask=mask, pad=0)


def _head(name, path, T, H, V, mask=0.0, hv=False):
    """hv: the head as [H, V]."""
    return dict(name=name, kind="head", path=path, T=T, H=H, V=V, mask=mask, hv=hv)


def _update(name, path, dtype, L, m, n, split=False, weights="fp32"):
    """L matrices of m x n; dtype: of the gradient; split: products of fp32 grade; weights: type of W ("muon")."""
    return dict(name=name, kind="update", path=path, dtype=dtype, L=L, m=m, n=n, split=split, weights=weights)


def listed():
    return [
        # one generated token: what a server reports beside it
        _score("score_token", "bf16", 1, VOCAB, 20),
        # evaluation of a few hundred tokens, fp32 logits of a vocabulary of odd size in padded rows, some of them prompt
        _score("score_odd_fp32", "fp32", 713, 100003, 5, mask=0.25, pad=61),
        # the smallest training run's step with alternatives (distillation from a few of a teacher's)
        _grad("grad_small_fp32", "fp32", 512, 1000, 8),
        # log-prob and entropy terms over logits that a model's own head has formed
        _grad("grad_bf16", "bf16", 8192, VOCAB, 0, mask=0.2),
        # one generated token, scored from its hidden state
        _head("head_token", "forward", 1, HIDDEN, VOCAB),
        # a few short responses, scored
        _head("head_score", "forward", 1191, HIDDEN, VOCAB),
        # an odd little batch of a model that keeps its head as [H, V], tool output masked
        _head("head_ragged_hv", "train", 713, 256, 3000, mask=0.25, hv=True),
        # the small model's step: 64 responses of 128 tokens over the full vocabulary
        _head("head_small_model", "train", 8192, 1024, VOCAB),
        # eight small projections of odd shape at once
        _update("orthogonalize_small", "orthogonalize", "bf16", 8, 257, 1000),
        # one large square matrix
        _update("orthogonalize_large", "orthogonalize", "bf16", 1, 4096, 4096),
        # one matrix of the small model, weights and products of fp32 grade
        _update("muon_fp32", "muon", "fp32", 1, 1024, 1024, split=True),
        # four layers' projections of the small model at once, tall ones
        _update("muon_layers", "muon", "bf16", 4, 4096, 1024),
    ]


# ------------------------------------------------------------------ drawn cases
def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rows(rng):
    V = VOCAB if rng.random() < 0.4 else _log_uniform(rng, 500, VOCAB)
    dtype, mask = rng.choice(["fp32", "bf16"]), rng.choice([0.0, 0.0, 0.25])
    if rng.random() < 0.5:
        return _score("", dtype, _log_uniform(rng, 1, 1024), V, rng.choice([0, 1, 5, 20, 64]), mask, rng.choice([0, 0, 64, 61]))
    K = rng.choice([0, 0, 8])
    return _grad("", dtype, _log_uniform(rng, 1, 1024 if K else min(8192, (1 << 29) // V)), V, K, mask)


def _draw_head(rng):
    H = 64 * _log_uniform(rng, 2, 64)
    V = VOCAB if rng.random() < 0.4 else _log_uniform(rng, 1000, VOCAB)
    T = _log_uniform(rng, 1, max(1, min(8192, 8192 * 1024 * VOCAB // (H * V))))
    return _head("", rng.choice(["forward", "forward", "train"]), T, H, V, rng.choice([0.0, 0.0, 0.2]), rng.random() < 0.25)


def _draw_update(rng):
    m, n = _log_uniform(rng, 32, 4096), _log_uniform(rng, 32, 4096)
    L = _log_uniform(rng, 1, max(1, min(8, 4096 ** 3 // (m * n * min(m, n)))))
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    # results in fp32 are asked for with products of that grade, bf16 ones with the faster products
    return _update("", rng.choice(["orthogonalize", "muon"]), dtype, L, m, n, dtype == "fp32", rng.choice(["fp32", "fp32", "bf16"]))


def draw(rng):
    case = rng.choice([_draw_rows, _draw_rows, _draw_head, _draw_update])(rng)
    del case["name"]
    return case


# ------------------------------------------------------------------ inputs
def _dtype(name):
    return {"fp32": torch.float32, "bf16": torch.bfloat16}[name]


def _generator(seed, stream):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 64 + stream)
    return g


def _tokens(case, seed):
    """Sampled ids, the loss mask in spans, and what a policy-gradient loss with an entropy bonus sends back."""
    T, V = case["T"], case["V"]
    g = _generator(seed, 1)
    target = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    mask = None
    if case["mask"]:
        span = max(1, T // 16)                                          # whole spans of tool output or prompt
        off = torch.rand((T + span - 1) // span, generator=g, device=DEV) < case["mask"]
        mask = (~off.repeat_interleave(span)[:T]).to(torch.uint8)
    ratio = torch.exp(0.1 * torch.randn(T, generator=g, device=DEV))
    d_logp = -torch.randn(T, generator=g, device=DEV) * ratio / T       # advantage times ratio over the number of tokens
    d_entropy = torch.full((T,), -ENTROPY_WEIGHT / T, device=DEV)
    return dict(target=target, mask=mask, d_logp=d_logp, d_entropy=d_entropy)


def _prepare_rows(case, seed):
    T, V, K = case["T"], case["V"], case["K"]
    g = _generator(seed, 2)
    s = dict(case, **_tokens(case, seed))
    # logits of a model: a spread of 2, a handful of tokens that carry most of the probability
    rows = torch.randn((T, V + case["pad"]), generator=g, device=DEV) * 2.0
    likely = (torch.randint(0, V, (T, 1), generator=g, device=DEV) + torch.arange(24, device=DEV) * (V // 24)) % V
    rows.scatter_(1, likely, 9.0 + 3.0 * torch.randn((T, 24), generator=g, device=DEV))
    s["logits"] = rows.to(_dtype(case["dtype"]))[:, :V]
    # a sampled token is a likely one, most of the time
    use = torch.rand(T, generator=g, device=DEV) < 0.8
    s["target"] = torch.where(use, likely[:, 0].to(torch.int32), s["target"])
    s["d_top"] = torch.rand((T, K), generator=g, device=DEV) * (-0.1 / T) if K else None
    return s


def _prepare_head(case, seed):
    T, H, V = case["T"], case["H"], case["V"]
    g = _generator(seed, 3)
    s = dict(case, **_tokens(case, seed))
    s["hidden"] = torch.randn((T, H), generator=g, device=DEV).to(torch.bfloat16)
    shape = (H, V) if case["hv"] else (V, H)
    s["W"] = (torch.randn(shape, generator=g, device=DEV) * (1.5 / math.sqrt(H))).to(torch.bfloat16)
    return s


def _prepare_update(case, seed):
    L, m, n = case["L"], case["m"], case["n"]
    g = _generator(seed, 4)

    def gradients():
        # a sum of outer products: few directions carry most of it, the rest is noise of the batch
        r = min(m, n, 64)
        left = torch.randn((L, m, r), generator=g, device=DEV) * torch.arange(1, r + 1, device=DEV) ** -0.5
        return (left @ torch.randn((L, r, n), generator=g, device=DEV) + torch.randn((L, m, n), generator=g, device=DEV)) * 1e-3

    s = dict(case, grad=gradients().to(_dtype(case["dtype"])))
    if case["path"] == "muon":
        s["momentum"] = 10.0 * gradients()
        s["W"] = (torch.randn((L, m, n), generator=g, device=DEV) / math.sqrt(n)).to(_dtype(case["weights"]))
    return s


def prepare(case, seed):
    return {"score": _prepare_rows, "grad": _prepare_rows, "head": _prepare_head, "update": _prepare_update}[case["kind"]](case, seed)


# ------------------------------------------------------------------ one pass, plain
def _scores(z, s):
    """(log-softmax, log-prob, log-sum-exp, entropy) of fp32 rows; rows that the mask leaves out give zeros."""
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = top + torch.log(total)
    logq = z - lse
    entropy = -(e / total * logq).sum(dim=1)
    logp = logq.gather(1, s["target"].long()[:, None])[:, 0]
    lse = lse[:, 0]
    if s["mask"] is not None:
        zero = torch.zeros_like(lse)
        live = s["mask"].bool()
        logp, lse, entropy = torch.where(live, logp, zero), torch.where(live, lse, zero), torch.where(live, entropy, zero)
    return logq, logp, lse, entropy


def _alternatives(z, logq, s):
    """Ids and log-probs of the K largest, ties to the lowest id: the largest of (value, -id) as one whole number."""
    V = z.shape[1]
    bits = (z + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    key = order * (1 << 32) + (V - 1 - torch.arange(V, device=z.device))
    ids = (V - 1 - (torch.topk(key, s["K"], dim=1).values & 0xFFFFFFFF)).to(torch.int32)
    top = logq.gather(1, ids.long())
    if s["mask"] is not None:
        live = s["mask"].bool()[:, None]
        ids, top = torch.where(live, ids, torch.full_like(ids, -1)), torch.where(live, top, torch.zeros_like(top))
    return ids, top


def _d_logits(logq, entropy, s, ids=None):
    """The gradient with respect to the logits."""
    a, e = s["d_logp"], s["d_entropy"]
    total = a if ids is None else a + s["d_top"].sum(dim=1)
    dz = -torch.exp(logq) * (total[:, None] + e[:, None] * (logq + entropy[:, None]))
    dz.scatter_add_(1, s["target"].long()[:, None], a[:, None])
    if ids is not None:
        dz.scatter_add_(1, ids.long().clamp(min=0), s["d_top"])
    if s["mask"] is not None:
        dz = torch.where(s["mask"].bool()[:, None], dz, torch.zeros_like(dz))
    return dz


def _plain_rows(s):
    z = s["logits"].float()
    logq, logp, lse, entropy = _scores(z, s)
    out = dict(logp=logp, lse=lse, entropy=entropy)
    if s["K"]:
        out["top_id"], out["top_logp"] = _alternatives(z, logq, s)
    if s["kind"] == "grad":
        out["d_logits"] = _d_logits(logq, entropy, s, out.get("top_id")).to(s["logits"].dtype)
    return out


def _plain_head(s):
    X, W = s["hidden"].float(), s["W"].float()
    z = X @ W if s["hv"] else X @ W.t()
    logq, logp, lse, entropy = _scores(z, s)
    out = dict(logp=logp, lse=lse, entropy=entropy)
    if s["path"] == "train":
        dz = _d_logits(logq, entropy, s)
        out["d_hidden"] = (dz @ (W.t() if s["hv"] else W)).to(torch.bfloat16)
        out["d_W"] = (X.t() @ dz if s["hv"] else dz.t() @ X).to(torch.bfloat16)
    return out


def _orthogonal(X):
    a, b, c = COEFFS
    X = X / (torch.sqrt((X * X).sum(dim=(1, 2), keepdim=True)) + EPS)
    tall = X.shape[1] > X.shape[2]
    for _ in range(STEPS):
        A = X.mT @ X if tall else X @ X.mT
        B = b * A + c * (A @ A)
        X = a * X + (X @ B if tall else B @ X)
    return X


def _muon_scale(s):
    return math.sqrt(max(1.0, s["m"] / s["n"]))


def _plain_update(s):
    G = s["grad"].float()
    if s["path"] == "orthogonalize":
        return dict(out=_orthogonal(G).to(s["grad"].dtype))
    M, W = s["momentum"], s["W"]
    M.mul_(MOMENTUM).add_(G)
    O = _orthogonal(G + MOMENTUM * M)
    W.copy_((1.0 - LR * WEIGHT_DECAY) * W.float() - LR * _muon_scale(s) * O)
    return dict(W=W, momentum=M)


# ------------------------------------------------------------------ one pass, through the framework
def _kept(s, name, make):
    """What a program makes once for its buffers and keeps: the descriptor and the workspaces."""
    if name not in s:
        s[name] = make()
    return s[name]


def _space(nbytes):
    return torch.empty(max(256, int(nbytes)), dtype=torch.uint8, device=DEV)


def _own_rows(s):
    from paper_2509_13232_amd import binding as spo
    d = _kept(s, "desc", lambda: spo.make_logprob_desc(None, None, s["target"], s["mask"], logits=s["logits"], top_k=s["K"]))
    ws = _kept(s, "ws_fwd", lambda: _space(spo.spo_logprob_fwd_workspace_bytes(d)))
    logp, lse, entropy, ids, top = spo.spo_logprob_fwd(d, workspace=ws)
    out = dict(logp=logp, lse=lse, entropy=entropy)
    if s["K"]:
        out["top_id"], out["top_logp"] = ids, top
    if s["kind"] == "grad":
        ws = _kept(s, "ws_bwd", lambda: _space(spo.spo_logprob_bwd_workspace_bytes(d)))
        out["d_logits"] = spo.spo_logprob_bwd(d, lse, entropy, s["d_logp"], s["d_entropy"], ids, s["d_top"], workspace=ws)
    return out


def _own_head(s):
    from paper_2509_13232_amd import binding as spo
    d = _kept(s, "desc", lambda: spo.make_logprob_desc(s["hidden"], s["W"], s["target"], s["mask"],
                                                       w_layout=spo.SPO_W_HV if s["hv"] else spo.SPO_W_VH))
    ws = _kept(s, "ws_fwd", lambda: _space(spo.spo_logprob_fwd_workspace_bytes(d)))
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(d, workspace=ws)
    out = dict(logp=logp, lse=lse, entropy=entropy)
    if s["path"] == "train":
        ws = _kept(s, "ws_bwd", lambda: _space(spo.spo_logprob_bwd_workspace_bytes(d)))
        out["d_hidden"], out["d_W"] = spo.spo_logprob_bwd(d, lse, entropy, s["d_logp"], s["d_entropy"], d_W_dtype=torch.bfloat16,
                                                          workspace=ws)
    return out


def _own_update(s):
    from paper_2509_13232_amd import binding as spo
    products = spo.SPO_PRODUCTS_SPLIT if s["split"] else spo.SPO_PRODUCTS_FP16
    ws = _kept(s, "ws", lambda: _space(spo.spo_orthogonalize_workspace_bytes(s["L"], s["m"], s["n"], products)))
    if s["path"] == "orthogonalize":
        return dict(out=spo.spo_orthogonalize(s["grad"], steps=STEPS, coeffs=COEFFS, eps=EPS, products=products, workspace=ws))
    spo.spo_muon_update(s["W"], s["momentum"], s["grad"], lr=LR, mu=MOMENTUM, weight_decay=WEIGHT_DECAY, scale=_muon_scale(s),
                        steps=STEPS, coeffs=COEFFS, eps=EPS, products=products, workspace=ws)
    return dict(W=s["W"], momentum=s["momentum"])


def run(state):
    kind = "rows" if state["kind"] in ("score", "grad") else state["kind"]
    plain = {"rows": _plain_rows, "head": _plain_head, "update": _plain_update}
    framework = {"rows": _own_rows, "head": _own_head, "update": _own_update}
    return (framework if own else plain)[kind](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "update":
        L, m, n = case["L"], case["m"], case["n"]
        k = min(m, n)
        elt = 4 if case["dtype"] == "fp32" else 2
        # in and out, and for the whole step the weights and the momentum read and written
        moved = 2 * elt if case["path"] == "orthogonalize" else elt + 2 * (4 if case["weights"] == "fp32" else 2) + 8
        # the two symmetric products count half
        return {"bytes": moved * L * m * n, "flops": float(STEPS) * L * (3.0 * k * m * n + float(k) ** 3)}
    T, V = case["T"], case["V"]
    live = T * (1.0 - case["mask"])
    if case["kind"] == "head":
        H = case["H"]
        if case["path"] == "forward":
            return {"bytes": 2 * (T * H + H * V), "flops": 2.0 * live * H * V}
        return {"bytes": 4 * (T * H + H * V), "flops": 6.0 * live * H * V}
    elt = 4 if case["dtype"] == "fp32" else 2
    # every live row read once, and for the gradient all rows written
    return {"bytes": elt * V * live + (elt * V * T if case["kind"] == "grad" else 0), "flops": 0}


# ------------------------------------------------------------------ from the definition, in 64 bits
def _exact_rows(z, s, K):
    """Rows in 64 bits -> outputs and, with K None, what the gradient needs."""
    p = torch.softmax(z, dim=1)
    lse = torch.logsumexp(z, dim=1)
    entropy = torch.special.entr(p).sum(dim=1)
    rows = torch.arange(z.shape[0], device=z.device)
    logp = z[rows, s["target"].long()] - lse
    live = torch.ones_like(lse) if s["mask"] is None else s["mask"].double()
    out = dict(logp=torch.where(live > 0, logp, 0.0), lse=torch.where(live > 0, lse, 0.0), entropy=torch.where(live > 0, entropy, 0.0))
    ids = None
    if K:
        ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :K]
        out["top_id"] = torch.where(live[:, None] > 0, ids, -1).to(torch.int32)
        out["top_logp"] = torch.where(live[:, None] > 0, z.gather(1, ids) - lse[:, None], 0.0)
    return out, p, lse, entropy, live, ids


def _exact_d_logits(z, s, p, lse, entropy, live, ids):
    a, e = s["d_logp"].double() * live, s["d_entropy"].double() * live
    onehot = torch.zeros_like(z)
    rows = torch.arange(z.shape[0], device=z.device)
    onehot[rows, s["target"].long()] = a
    if ids is not None:
        b = s["d_top"].double() * live[:, None]
        onehot.scatter_add_(1, ids, b)
        a = a + b.sum(dim=1)
    # d entropy / d z_i = -p_i (log p_i + entropy); p log p vanishes with p
    return onehot - a[:, None] * p + e[:, None] * (torch.special.entr(p) - entropy[:, None] * p)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "update":
        a, b, c = COEFFS
        G = s["grad"].double()
        U = G
        if case["path"] == "muon":
            M = MOMENTUM * s["momentum"].double() + G
            U = G + MOMENTUM * M
        X = U / (torch.linalg.vector_norm(U, dim=(1, 2), keepdim=True) + EPS)
        flip = case["m"] > case["n"]
        X = X.mT.contiguous() if flip else X
        for _ in range(STEPS):
            S = X @ X.mT
            X = a * X + b * (S @ X) + c * (S @ (S @ X))
        X = X.mT.contiguous() if flip else X
        if case["path"] == "orthogonalize":
            return dict(out=X)
        return dict(W=s["W"].double() * (1.0 - LR * WEIGHT_DECAY) - LR * _muon_scale(s) * X, momentum=M)
    if case["kind"] == "head":
        X, W = s["hidden"].double(), s["W"].double()
        W = W if case["hv"] else W.t()
        z = X @ W
        out, p, lse, entropy, live, ids = _exact_rows(z, s, 0)
        if case["path"] == "train":
            dz = _exact_d_logits(z, s, p, lse, entropy, live, None)
            out["d_hidden"] = dz @ W.t()
            out["d_W"] = X.t() @ dz if case["hv"] else dz.t() @ X
        return out
    z = s["logits"].double()
    out, p, lse, entropy, live, ids = _exact_rows(z, s, case["K"])
    if case["kind"] == "grad":
        out["d_logits"] = _exact_d_logits(z, s, p, lse, entropy, live, ids)
    return out
