"""Token scores and updates of arrays with more than 2^31 elements (and 2^32 bytes): samples from both ends and the middle against
64-bit products of the inputs' own rows.  Tolerances as in the small tests of the same operators."""
import pytest
import torch

import score_cases as sc
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def gauss(shape, dtype, seed, std=1.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def say(text):
    print(text, flush=True)


def test_logits():
    T, V, K = 14400, 151936, 3
    z = gauss((T, V + 24), BF16, 1, 2.0)[:, 3:V + 3]     # rows apart, off 16-byte boundaries
    assert z.stride(0) * (T - 1) > 1 << 31
    g = torch.Generator().manual_seed(2)
    target = torch.randint(0, V, (T,), generator=g).int()
    a, e, b = torch.randn(T, generator=g), torch.randn(T, generator=g), torch.randn((T, K), generator=g)
    d = spo.make_logprob_desc(None, None, target.cuda(), logits=z, top_k=K)
    say("logits: forward")
    logp, lse, entropy, ids, top = spo.spo_logprob_fwd(d)
    rows = [0, 1, 7000, T // 2, T - 2, T - 1]
    want = sc.scores(z[rows].double().cpu(), target[rows], None, K)
    for x, name in ((logp, "logp"), (lse, "lse"), (entropy, "entropy"), (top, "top_logp")):
        torch.testing.assert_close(x[rows].double().cpu(), want[name], atol=2e-5, rtol=2e-6)
    assert torch.equal(ids[rows].cpu().long(), want["top_id"])
    say("logits: gradient")
    dz = spo.spo_logprob_bwd(d, lse, entropy, a.cuda(), e.cuda(), ids, b.cuda())
    want = sc.d_logits(z[rows].double().cpu(), target[rows], None, a[rows], e[rows], ids[rows].cpu(), b[rows])
    assert sc.rel(dz[rows], want) < 3e-3


@pytest.mark.parametrize("T", [1, 3, 40])
def test_head(T):
    V, H = 151936, 16384
    W = gauss((V, H), BF16, 3, H ** -0.5)
    assert W.numel() > 1 << 31
    X = gauss((T, H), BF16, 4, 2.0)
    g = torch.Generator().manual_seed(5)
    target = torch.randint(0, V, (T,), generator=g).int()
    target[-1] = V - 1
    d = spo.make_logprob_desc(X, W, target.cuda())
    say(f"head: forward of {T}")
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    z = torch.cat([X.double() @ W[v:v + 16384].double().t() for v in range(0, V, 16384)], dim=1)
    want = sc.scores(z.cpu(), target)
    for x, name in ((logp, "logp"), (lse, "lse"), (entropy, "entropy")):
        torch.testing.assert_close(x.double().cpu(), want[name], atol=2e-4, rtol=2e-6)
    if T != 40:
        return
    say("head: gradients")
    a, e = torch.randn(T, generator=g), torch.randn(T, generator=g)
    dX, dW = spo.spo_logprob_bwd(d, lse, entropy, a.cuda(), e.cuda())
    dz = sc.d_logits(z.cpu(), target, None, a, e).cuda()
    assert sc.rel(dX, sum(dz[:, v:v + 16384] @ W[v:v + 16384].double() for v in range(0, V, 16384))) < 1e-2
    vs = torch.cat([target.long(), torch.tensor([0, 1, V // 2, V - 2])])
    assert sc.rel(dW[vs], (dz[:, vs].t() @ X.double()).cpu()) < 1e-2


def _one_step(U, rows, coeffs):
    """Rows of a X + (b A + c A A) X, A = X X^T, X = U / |U|, by products of single rows with the whole matrix, in 64 bits."""
    a, b, c = coeffs
    k, part = U.shape[0], 4000
    blocks = [slice(i, min(i + part, k)) for i in range(0, k, part)]
    norm = sum((U[s].double() ** 2).sum() for s in blocks).sqrt()
    x = U[rows].double() / norm
    gram = lambda y: torch.cat([y @ (U[s].double() / norm).t() for s in blocks], dim=1)    # y X^T
    back = lambda w: sum(w[:, s] @ (U[s].double() / norm) for s in blocks)                 # w X
    ax = back(gram(x))
    return a * x + b * ax + c * back(gram(ax))


@pytest.mark.parametrize("turned", [False, True])
def test_one_matrix(turned):
    k, L = 36000, 60000
    assert k * L > 1 << 31
    G = gauss((L, k) if turned else (k, L), BF16, 6)
    say(f"update of {tuple(G.shape)}")
    out = spo.spo_orthogonalize(G, steps=1, out_dtype=F32)
    rows = [0, 1, 17999, 31111, k - 1]
    U = G.t().contiguous() if turned else G
    del G
    got = (out[:, rows].t() if turned else out[rows]).contiguous()
    del out
    assert sc.rel(got, _one_step(U, rows, spo.NEWTON_SCHULZ)) < 3e-3


def test_a_stack():
    L, n, lr = 3, 27000, 0.5
    assert (L - 1) * n * n < 1 << 31 < L * n * n
    G, W, M = gauss((L, n, n), BF16, 7), gauss((L, n, n), BF16, 8), torch.zeros((L, n, n), device="cuda")
    rows = [0, 13333, n - 1]
    before = [W[i, rows].double() for i in range(L)]
    say("momentum step of a stack")
    spo.spo_muon_update(W, M, G, lr=lr, mu=0.5, nesterov=False, scale=n ** 0.5, steps=1)
    for i in range(L):
        assert torch.equal(M[i, ::1111], G[i, ::1111].float())
        want = before[i] - lr * n ** 0.5 * _one_step(G[i], rows, spo.NEWTON_SCHULZ)
        assert sc.rel(W[i, rows], want) < 4e-3
