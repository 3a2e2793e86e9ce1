"""Token scores, their gradient and orthogonalised updates from their definitions, in 64 bits with plain torch operations on
the CPU (nothing of the library), and the inputs that their tests share."""
import torch

NEWTON_SCHULZ = (3.4445, -4.7750, 2.0315)


def log_softmax(z):
    # about the row's largest entry: beside a logit of 1e38 the logarithm of a sum has no digits left
    d = z - z.amax(dim=1, keepdim=True)
    return d - torch.log(torch.exp(d).sum(dim=1, keepdim=True))


def scores(z, target=None, mask=None, K=0):
    """z [T, V] float64: dict of logp, lse, entropy, top_id, top_logp."""
    T, V = z.shape
    lse = torch.logsumexp(z, dim=1)
    logq = log_softmax(z)
    p = torch.exp(logq)
    h = -torch.where(p > 0, p * logq, torch.zeros_like(p)).sum(dim=1)
    out = dict(lse=lse, entropy=torch.where(torch.isfinite(lse), h, torch.full_like(h, float("nan"))))
    if target is not None:
        ok = (target >= 0) & (target < V)
        zy = logq.gather(1, target.long().clamp(0, V - 1)[:, None])[:, 0]
        out["logp"] = torch.where(ok, zy, torch.full_like(zy, float("nan")))
    if K:
        ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :K]
        out["top_id"], out["top_logp"] = ids, logq.gather(1, ids)
    if mask is not None:
        live = mask.bool()
        for k, v in out.items():
            off = torch.full_like(v, -1 if k == "top_id" else 0)
            out[k] = torch.where(live if v.dim() == 1 else live[:, None], v, off)
    return out


def d_logits(z, target, mask, a=None, e=None, ids=None, b=None):
    """Gradient of sum(a logp) + sum(e entropy) + sum(b top_logp) with respect to z [T, V] float64."""
    T, V = z.shape
    logq = log_softmax(z)
    p = torch.exp(logq)
    plogp = torch.where(p > 0, p * logq, torch.zeros_like(p))
    h = -plogp.sum(dim=1, keepdim=True)
    zero = torch.zeros(T, dtype=torch.float64)
    a = zero if a is None else a.double()
    e = zero if e is None else e.double()
    hot = torch.zeros_like(z)
    total = a.clone()
    if target is not None:
        ok = (target >= 0) & (target < V)
        hot.scatter_add_(1, target.long().clamp(0, V - 1)[:, None], torch.where(ok, a, zero)[:, None])
    if b is not None:
        hot.scatter_add_(1, ids.long().clamp(min=0), b.double())
        total = total + b.double().sum(dim=1)
    dz = hot - p * total[:, None] - e[:, None] * (plogp + h * p)
    return dz if mask is None else torch.where(mask.bool()[:, None], dz, torch.zeros_like(dz))


def orthogonal(U, steps=5, coeffs=NEWTON_SCHULZ, eps=1e-7):
    a, b, c = coeffs
    X = U.double()
    X = X / (torch.sqrt((X * X).sum(dim=(-2, -1), keepdim=True)) + eps)
    tall = X.shape[-2] > X.shape[-1]
    X = X.mT.contiguous() if tall else X
    for _ in range(steps):
        S = X @ X.mT
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.mT.contiguous() if tall else X


def rel(x, want):
    x, want = x.double().cpu(), want.double().cpu()
    n = want.norm()
    return float((x - want).norm() / n) if n > 0 else float(x.norm())


def logits(T, V, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((T, V), generator=g) * spread).to(dtype)


def mask_of(T, seed, share=0.3):
    g = torch.Generator().manual_seed(seed + 77)
    m = (torch.rand(T, generator=g) >= share).to(torch.uint8)
    return m


def targets(T, V, seed):
    g = torch.Generator().manual_seed(seed + 99)
    return torch.randint(0, V, (T,), generator=g, dtype=torch.int32)


def factors(shape, seed):
    g = torch.Generator().manual_seed(seed + 55)
    return torch.randn(shape, generator=g)
