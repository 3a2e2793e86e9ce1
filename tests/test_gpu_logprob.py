"""Log-probs, entropy and alternatives, and their gradient, against their definitions in 64 bits.

Tolerances, from the arithmetic: a log-sum-exp or entropy of fp32 sums carries the rounding of exponents up to ~30 (30 * 2^-24 =
2e-6 relative per term) and of a result up to ~20 (1e-6): 2e-5 absolute.  Gradients in fp32 inherit 2e-6 relative per
entry: 1e-5 in 2-norm; in bf16 one rounding of at most 2^-9: 3e-3 in 2-norm.  The head form has fp32 sums over the hidden size
before (logits to ~1e-5: 2e-4 absolute, as the loss) and bf16 logit gradients behind (1e-2 in 2-norm, as the loss)."""
import pytest
import torch

import score_cases as sc
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
GRAD = {F32: 1e-5, BF16: 3e-3}


def cuda(t):
    return None if t is None else t.cuda()


def run_fwd(z, target, mask, K, **kw):
    d = spo.make_logprob_desc(None, None, cuda(target), cuda(mask), logits=z, top_k=K)
    return d, spo.spo_logprob_fwd(d, **kw)


def close(x, want, atol=2e-5, rtol=2e-6):
    torch.testing.assert_close(x.double().cpu(), want, atol=atol, rtol=rtol, equal_nan=True)


def check_fwd(z_host, out, target, mask, K, **kw):
    want = sc.scores(z_host.double(), target, mask, K)
    logp, lse, entropy, ids, top = out
    close(lse, want["lse"], **kw)
    close(entropy, want["entropy"], **kw)
    if target is not None:
        close(logp, want["logp"], **kw)
    if K:
        assert torch.equal(ids.cpu().long(), want["top_id"].long())
        close(top, want["top_logp"], **kw)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (1, 151936, 20), (3, 7, 7), (5, 64, 64), (33, 100, 64), (300, 1000, 8), (17, 4099, 5),
                                   (2, 100003, 64), (70, 8192, 1), (9, 16392, 3), (700, 2056, 0), (40, 30001, 0), (2500, 130, 4)])
def test_forward(dtype, T, V, K):
    z = sc.logits(T, V, dtype, T + V)
    target, mask = sc.targets(T, V, T), sc.mask_of(T, V) if T > 4 else None
    _, out = run_fwd(z.cuda(), target, mask, K)
    check_fwd(z, out, target, mask, K)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_apart_and_off_16_byte_boundaries(dtype):
    T, V, K = 21, 5003, 12
    z = sc.logits(T, V + 61, dtype, 3)
    for off in (0, 1, 3):
        part = z.cuda()[:, off:off + V]
        target = sc.targets(T, V, off)
        _, out = run_fwd(part, target, None, K)
        check_fwd(z[:, off:off + V], out, target, None, K)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [50, 3000, 40000])
def test_ties_go_to_the_lowest_id(dtype, V):
    g = torch.Generator().manual_seed(V)
    rows = [torch.zeros(V), torch.full((V,), -3.5), torch.randint(0, 3, (V,), generator=g).float(),
            torch.randint(-2, 40, (V,), generator=g).float(), torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)]
    z = torch.stack(rows).to(dtype)
    for K in (1, 20, min(64, V)):
        _, out = run_fwd(z.cuda(), None, None, K)
        assert out[0] is None
        check_fwd(z, out, None, None, K)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [70, 20000])
def test_masked_logits(dtype, V):
    # what constrained sampling and padded vocabularies leave in rows
    low = torch.finfo(dtype).min
    z = sc.logits(8, V, F32, V)
    z[0, V // 2:] = float("-inf")
    z[1, 3:] = float("-inf")               # fewer finite entries than alternatives
    z[2, :] = float("-inf")                # nothing left
    z[3, 10:] = low
    z[4, :] = low                          # the type's lowest value throughout
    z[5, :-1] = -1e30
    z[6, ::3] = -1e30
    z = z.to(dtype)
    target = torch.tensor([1, 2, 0, 4, 5, V - 1, 1, 0], dtype=torch.int32)
    K = 20
    d, out = run_fwd(z.cuda(), target, None, K)
    check_fwd(z, out, target, None, K)
    # gradients of rows with something left
    rows = torch.tensor([0, 1, 3, 4, 5, 6, 7])
    a, e = sc.factors(8, 1), sc.factors(8, 2)
    got = spo.spo_logprob_bwd(d, out[1], out[2], a.cuda(), e.cuda()).cpu()
    want = sc.d_logits(z.double()[rows], target[rows], None, a[rows], e[rows])
    assert torch.isfinite(got[rows].float()).all()
    for i, r in enumerate(rows):
        assert sc.rel(got[r], want[i]) < GRAD[dtype], r


def test_large_logits_keep_their_scores():
    z = sc.logits(6, 5000, F32, 9)
    z[0] += 1e6
    z[1] *= 1e5
    z[2] -= 3e37
    z[3, 17] = 3e38
    target = torch.full((6,), 17, dtype=torch.int32)
    d, out = run_fwd(z.cuda(), target, None, 3)
    want = sc.scores(z.double(), target, None, 3)
    close(out[1], want["lse"], atol=2e-5, rtol=3e-7)
    close(out[2], want["entropy"])
    close(out[0], want["logp"], atol=2e-5, rtol=3e-7)
    close(out[4], want["top_logp"], atol=2e-5, rtol=3e-7)
    assert torch.equal(out[3].cpu().long(), want["top_id"])
    a, e = sc.factors(6, 1), sc.factors(6, 2)
    dz = spo.spo_logprob_bwd(d, out[1], out[2], a.cuda(), e.cuda())
    want = sc.d_logits(z.double(), target, None, a, e)
    for i in range(6):
        assert sc.rel(dz[i], want[i]) < GRAD[F32], i


def test_left_out_rows_are_not_read():
    T, V, K = 12, 9000, 5
    z = sc.logits(T, V, BF16, 4)
    mask = sc.mask_of(T, 1, 0.5)
    z[mask == 0] = float("nan")
    target = sc.targets(T, V, 2)
    target[mask == 0] = 1 << 30
    d, out = run_fwd(z.cuda(), target, mask, K)
    live = mask.bool()
    want = sc.scores(z.double()[live], target[live], None, K)
    for x, k in ((out[0], "logp"), (out[1], "lse"), (out[2], "entropy"), (out[4], "top_logp")):
        close(x[live.cuda()], want[k])
        assert (x[~live.cuda()] == 0).all()
    assert (out[3][~live.cuda()] == -1).all()
    a, e, b = sc.factors(T, 1), sc.factors(T, 2), sc.factors((T, K), 3)
    dz = spo.spo_logprob_bwd(d, out[1], out[2], a.cuda(), e.cuda(), out[3], b.cuda()).cpu()
    assert (dz[~live] == 0).all()
    assert sc.rel(dz[live], sc.d_logits(z.double()[live], target[live], None, a[live], e[live], want["top_id"], b[live])) < GRAD[BF16]


def test_nan_rows_and_bad_targets_say_so():
    z = sc.logits(4, 700, F32, 1)
    z[1, 300] = float("nan")
    target = torch.tensor([-1, 5, 700, 6], dtype=torch.int32)
    d, out = run_fwd(z.cuda(), target, None, 4)
    logp, lse, entropy, ids, top = (x.cpu() for x in out)
    assert torch.isnan(logp[:3]).all() and torch.isfinite(logp[3])
    assert torch.isnan(lse[1]) and torch.isnan(entropy[1]) and torch.isnan(top[1]).all()
    assert ((ids >= 0) & (ids < 700)).all() and torch.isfinite(lse[[0, 2, 3]]).all()
    a = sc.factors(4, 3)
    dz = spo.spo_logprob_bwd(d, out[1], None, a.cuda()).cpu()
    rows = torch.tensor([0, 2, 3])
    assert sc.rel(dz[rows], sc.d_logits(z.double()[rows], target[rows], None, a[rows])) < GRAD[F32]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,V,K", [(1, 5, 5), (3, 151936, 20), (130, 1000, 8), (65, 4099, 64), (11, 100003, 0), (600, 264, 3), (7, 16392, 1)])
@pytest.mark.parametrize("parts", ["logp", "entropy", "top", "all"])
def test_gradient(dtype, T, V, K, parts):
    if parts == "top" and not K:
        pytest.skip("no alternatives")
    z = sc.logits(T, V, dtype, T * 3 + V)
    target, mask = sc.targets(T, V, T), sc.mask_of(T, V) if T > 4 else None
    target[0] = int(z[0].float().argmax())     # the target among the alternatives
    d, out = run_fwd(z.cuda(), target, mask, K)
    a = sc.factors(T, 1) if parts in ("logp", "all") else None
    e = sc.factors(T, 2) if parts in ("entropy", "all") else None
    b = sc.factors((T, K), 3) if parts in ("top", "all") and K else None
    dz = spo.spo_logprob_bwd(d, out[1], out[2] if e is not None else None, cuda(a), cuda(e), out[3] if b is not None else None, cuda(b))
    want = sc.d_logits(z.double(), target, mask, a, e, None if b is None else out[3].cpu(), b)
    assert dz.dtype == dtype and sc.rel(dz, want) < GRAD[dtype]


def test_gradient_against_differences():
    T, V, K, h = 5, 400, 6, 1e-4
    z = sc.logits(T, V, F32, 8)
    target = sc.targets(T, V, 8)
    d, out = run_fwd(z.cuda(), target, None, K)
    a, e, b = sc.factors(T, 1), sc.factors(T, 2), sc.factors((T, K), 3)
    dz = spo.spo_logprob_bwd(d, out[1], out[2], a.cuda(), e.cuda(), out[3], b.cuda()).double().cpu()
    way = sc.factors((T, V), 4).double()

    def total(x):
        s = sc.scores(x, target)
        top = x.gather(1, out[3].cpu().long()) - s["lse"][:, None]
        return (a.double() * s["logp"]).sum() + (e.double() * s["entropy"]).sum() + (b.double() * top).sum()

    by_difference = (total(z.double() + h * way) - total(z.double() - h * way)) / (2 * h)
    assert abs(float((dz * way).sum() - by_difference)) < 1e-4 * float(dz.norm() * way.norm())


def test_no_gradient_writes_zeros():
    z = sc.logits(6, 3001, BF16, 2)
    z[2] = float("inf")
    d, out = run_fwd(z.cuda(), sc.targets(6, 3001, 1), None, 0)
    zero = torch.zeros(6)
    assert (spo.spo_logprob_bwd(d, out[1], out[2], zero.cuda(), zero.cuda()) == 0).all()
    assert (spo.spo_logprob_bwd(d, out[1]) == 0).all()


def test_empty_batch_and_streams():
    d, out = run_fwd(torch.empty((0, 40), device="cuda"), torch.empty(0, dtype=torch.int32), None, 3)
    assert out[0].shape == (0,) and out[3].shape == (0, 3)
    assert spo.spo_logprob_bwd(d, out[1]).shape == (0, 40)
    z = sc.logits(50, 20000, BF16, 1)
    target = sc.targets(50, 20000, 1)
    _, want = run_fwd(z.cuda(), target, None, 9)
    side = torch.cuda.Stream()
    zc, tc = z.cuda(), target.cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        _, got = run_fwd(zc, tc, None, 9)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))       # bit for bit


def test_a_captured_pass_replays():
    T, V, K = 24, 20000, 7
    z = torch.empty((T, V), dtype=BF16, device="cuda")
    target = sc.targets(T, V, 1).cuda()
    a, e, b = (sc.factors(s, i).cuda() for i, s in enumerate(((T,), (T,), (T, K))))
    d = spo.make_logprob_desc(None, None, target, None, logits=z, top_k=K)
    ws = torch.empty(spo.spo_logprob_fwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")

    def step():
        out = spo.spo_logprob_fwd(d, workspace=ws)
        return (*out, spo.spo_logprob_bwd(d, out[1], out[2], a, e, out[3], b))

    z.copy_(sc.logits(T, V, BF16, 0))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (1, 2, 3):
        z.copy_(sc.logits(T, V, BF16, seed))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(captured, step()):
            assert torch.equal(x, y)


# ------------------------------------------------------------------ from hidden states and the head
def head_inputs(T, H, V, dtype, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    X = torch.randn((T, H), generator=g).to(dtype)
    W = (torch.randn((V, H), generator=g) * (spread / H ** 0.5)).to(dtype)
    return X, W


@pytest.mark.parametrize("hv", [False, True])
@pytest.mark.parametrize("dtype,T,H,V", [(BF16, 1, 64, 10), (BF16, 1, 256, 3001), (BF16, 5, 1024, 5000), (BF16, 16, 4096, 2000), (BF16, 17, 128, 1000),
                                         (BF16, 32, 192, 4096), (BF16, 713, 256, 3000), (BF16, 300, 64, 40000), (F32, 40, 128, 1000),
                                         (F32, 1, 64, 777)])
def test_head_forward(hv, dtype, T, H, V):
    X, W = head_inputs(T, H, V, dtype, T + V)
    target, mask = sc.targets(T, V, T), sc.mask_of(T, H) if T > 4 else None
    layout = spo.SPO_W_HV if hv else spo.SPO_W_VH
    d = spo.make_logprob_desc(X.cuda(), (W.t().contiguous() if hv else W).cuda(), target.cuda(), cuda(mask), w_layout=layout)
    logp, lse, entropy, ids, top = spo.spo_logprob_fwd(d)
    want = sc.scores(X.double() @ W.double().t(), target, mask)
    tol = 2e-4 if dtype == BF16 else 5e-5
    for x, k in ((logp, "logp"), (lse, "lse"), (entropy, "entropy")):
        close(x, want[k], atol=tol)
    assert ids is None and top is None
    # without a target, without the entropy
    d = spo.make_logprob_desc(X.cuda(), (W.t().contiguous() if hv else W).cuda(), None, cuda(mask), w_layout=layout)
    logp, lse2, entropy, _, _ = spo.spo_logprob_fwd(d, want_entropy=False)
    assert logp is None and entropy is None and torch.equal(lse, lse2)


@pytest.mark.parametrize("T", [1, 2, 3, 7, 16])
@pytest.mark.parametrize("H,V", [(64, 1), (64, 17), (448, 3000), (1024, 501), (1088, 20000), (2112, 300), (4096, 1111), (4160, 640), (8192, 95)])
def test_a_few_tokens(T, H, V):
    X, W = head_inputs(T, H, V, BF16, T + V + H)
    target = sc.targets(T, V, T + H)
    target[-1] = V - 1
    mask = None
    if T > 2:
        mask = torch.ones(T, dtype=torch.uint8)
        mask[1] = 0
        target[0] = V           # outside the vocabulary
    d = spo.make_logprob_desc(X.cuda(), W.cuda(), target.cuda(), cuda(mask))
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    want = sc.scores(X.double() @ W.double().t(), target, mask)
    for x, k in ((logp, "logp"), (lse, "lse"), (entropy, "entropy")):
        close(x, want[k], atol=2e-4)
    again = spo.spo_logprob_fwd(d)
    assert torch.equal(again[1], lse) and torch.equal(again[2], entropy)


@pytest.mark.parametrize("T", [1, 2, 5, 20])
def test_an_infinite_weight_does_not_reach_other_tokens(T):
    H, V = 192, 700
    X, W = head_inputs(T, H, V, BF16, T)
    X[:, 5] = 0
    X[0, 5] = 1
    W[333, 5] = float("-inf")     # bans an entry for the first token; for the others 0 * inf
    d = spo.make_logprob_desc(X.cuda(), W.cuda(), torch.zeros(T, dtype=torch.int32, device="cuda"))
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    z = X.double() @ W.double().t()
    want = sc.scores(z[:1], torch.zeros(1, dtype=torch.int32))
    for x, k in ((logp, "logp"), (lse, "lse"), (entropy, "entropy")):
        close(x[:1], want[k], atol=2e-4)
    assert T == 1 or torch.isnan(lse[1:]).all()


@pytest.mark.parametrize("hv", [False, True])
@pytest.mark.parametrize("T,H,V,chunk", [(1, 64, 10, 0), (5, 128, 1003, 0), (713, 256, 3000, 0), (600, 64, 500, 256), (300, 1024, 2111, 0)])
@pytest.mark.parametrize("parts", ["logp", "entropy", "both"])
def test_head_gradient(hv, T, H, V, chunk, parts):
    X, W = head_inputs(T, H, V, BF16, T + V)
    target, mask = sc.targets(T, V, T), sc.mask_of(T, H) if T > 4 else None
    a = sc.factors(T, 1) if parts != "entropy" else None
    e = sc.factors(T, 2) if parts != "logp" else None
    if a is not None and T > 3:
        a[1] = 0.0
    Wl = W.t().contiguous() if hv else W
    d = spo.make_logprob_desc(X.cuda(), Wl.cuda(), target.cuda(), cuda(mask), w_layout=spo.SPO_W_HV if hv else spo.SPO_W_VH)
    _, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    args = (d, lse, entropy if e is not None else None, cuda(a), cuda(e))
    dz = sc.d_logits(X.double() @ W.double().t(), target, mask, a, e)
    want_x, want_w = dz @ W.double(), dz.t() @ X.double()
    want_w = want_w.t() if hv else want_w
    dx, dw = spo.spo_logprob_bwd(*args, chunk_tokens=chunk)
    assert dx.dtype == BF16 and dw.dtype == F32
    assert sc.rel(dx, want_x) < 1e-2 and sc.rel(dw, want_w) < 1e-2
    dead = (dz == 0).all(dim=1)
    assert (dx.cpu()[dead] == 0).all()
    # other types, one of the two alone, and added to what is there
    dx, dw = spo.spo_logprob_bwd(*args, d_hidden_dtype=F32, d_W_dtype=BF16, chunk_tokens=chunk)
    assert sc.rel(dx, want_x) < 1e-2 and sc.rel(dw, want_w) < 1e-2
    only, none = spo.spo_logprob_bwd(*args, want_d_W=False, chunk_tokens=chunk)
    assert none is None and sc.rel(only, want_x) < 1e-2
    held = torch.ones(Wl.shape, device="cuda")
    none, acc = spo.spo_logprob_bwd(*args, d_W=held, accumulate_dW=True, want_d_hidden=False, chunk_tokens=chunk)
    assert none is None and sc.rel(acc.cpu() - 1.0, want_w) < 1.1e-2


def test_head_and_logits_forms_agree():
    # the softmax part on its own: peaked rows, where it is as large as the one-hot part
    T, H, V = 200, 128, 2000
    X, W = head_inputs(T, H, V, BF16, 5, spread=6.0)
    target = sc.targets(T, V, 3)
    z = X.double() @ W.double().t()
    e = sc.factors(T, 2)
    d = spo.make_logprob_desc(X.cuda(), W.cuda(), target.cuda())
    _, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    dx, dw = spo.spo_logprob_bwd(d, lse, entropy, None, e.cuda(), d_hidden_dtype=F32)
    dl = spo.make_logprob_desc(None, None, target.cuda(), logits=z.float().cuda())
    _, lse_l, entropy_l, _, _ = spo.spo_logprob_fwd(dl)
    close(lse, lse_l.double().cpu(), atol=2e-4)
    close(entropy, entropy_l.double().cpu(), atol=2e-4)
    dz = spo.spo_logprob_bwd(dl, lse_l, entropy_l, None, e.cuda()).double().cpu()
    assert sc.rel(dx, dz @ W.double()) < 1e-2 and sc.rel(dw, dz.t() @ X.double()) < 1e-2


def test_head_batches_without_tokens_or_factors():
    X, W = head_inputs(4, 64, 300, BF16, 1)
    d = spo.make_logprob_desc(X.cuda()[:0], W.cuda(), torch.empty(0, dtype=torch.int32, device="cuda"))
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    assert lse.shape == (0,)
    dx, dw = spo.spo_logprob_bwd(d, lse, entropy, lse, lse)
    assert dx.shape == (0, 64) and (dw == 0).all()
    d = spo.make_logprob_desc(X.cuda(), W.cuda(), sc.targets(4, 300, 1).cuda(), torch.zeros(4, dtype=torch.uint8, device="cuda"))
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    assert (lse == 0).all() and (entropy == 0).all() and (logp == 0).all()
    ones = torch.ones(4, device="cuda")
    dx, dw = spo.spo_logprob_bwd(d, lse, entropy, ones, ones)
    assert (dx == 0).all() and (dw == 0).all()


# ------------------------------------------------------------------ plain calls of the binding
@pytest.mark.parametrize("K", [0, 6])
@pytest.mark.parametrize("given", [True, False])
def test_plain_calls_give_the_same_bits(monkeypatch, K, given):
    z = sc.logits(20, 3000, BF16, 1).cuda()
    target = sc.targets(20, 3000, 1).cuda() if given else None
    d = spo.make_logprob_desc(None, None, target, sc.mask_of(20, 3).cuda(), logits=z, top_k=K)
    ws = torch.empty(spo.spo_logprob_fwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    a, e, b = sc.factors(20, 1).cuda() if given else None, sc.factors(20, 2).cuda(), sc.factors((20, K), 3).cuda() if K else None
    X, W = head_inputs(20, 64, 300, BF16, 1)
    h = spo.make_logprob_desc(X.cuda(), W.cuda(), target if target is None else target % 300)
    wh = torch.empty(spo.spo_logprob_fwd_workspace_bytes(h), dtype=torch.uint8, device="cuda")

    def calls():
        out = spo.spo_logprob_fwd(d, workspace=ws)
        return (*out, spo.spo_logprob_bwd(d, out[1], out[2], a, e, out[3], b), *spo.spo_logprob_fwd(h, workspace=wh))

    real, taken = spo._plain_calls(), []

    class Watch:
        def __getattr__(self, name):
            def f(*args):
                out = getattr(real, name)(*args)
                taken.append((name, out is not None))
                return out
            return f

    class Nothing:
        def __getattr__(self, name):
            return lambda *args: None

    results = []
    for way in (Watch(), Nothing()):
        with monkeypatch.context() as m:
            m.setattr(spo, "_calls", way)
            results.append(calls())
    assert taken == [("logprob_fwd", True), ("logprob_bwd", True), ("logprob_fwd", True)]
    for x, y in zip(*results):
        assert (x is None and y is None) or (x.dtype == y.dtype and x.shape == y.shape and torch.equal(x, y))
    # what is not plain goes the general way: its errors, and calls that are right all the same
    with pytest.raises(TypeError):
        spo.spo_logprob_bwd(d, out_of(results)[1].double())
    with pytest.raises(ValueError):
        spo.spo_logprob_bwd(d, out_of(results)[1][:3])
    bad = spo.make_logprob_desc(None, None, target, None, logits=z, top_k=65)
    with pytest.raises(spo.SpoError):
        spo.spo_logprob_fwd(bad, workspace=ws)


def out_of(results):
    return results[0]


# ------------------------------------------------------------------ refusals
def test_refusals():
    z = torch.zeros((4, 100), device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    X, W = torch.zeros((4, 64), dtype=BF16, device="cuda"), torch.zeros((100, 64), dtype=BF16, device="cuda")
    status = lambda f, *a, **k: pytest.raises(spo.SpoError, f, *a, **k).value.status
    for K, want in ((-1, -1), (101, -1), (65, -3)):
        assert status(spo.spo_logprob_fwd, spo.make_logprob_desc(None, None, t, logits=z, top_k=K)) == want
    assert status(spo.spo_logprob_fwd, spo.make_logprob_desc(X, W, t, top_k=2)) == -5
    assert status(spo.spo_logprob_fwd, spo.make_logprob_desc(X[:, :32].contiguous(), W[:, :32].contiguous(), t)) == -5
    d = spo.make_logprob_desc(None, None, None, logits=z)
    _, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    assert status(spo.spo_logprob_bwd, d, lse, None, lse) == -2              # a log-prob's gradient without a target
    assert status(spo.spo_logprob_bwd, d, lse, None, None, lse) == -2        # an entropy's without the entropy
    f = spo.make_logprob_desc(X.float(), W.float(), t)
    _, lse, entropy, _, _ = spo.spo_logprob_fwd(f)
    assert status(spo.spo_logprob_bwd, f, lse, entropy, lse) == -5
    b = spo.make_logprob_desc(X, W, t)
    assert status(spo.spo_logprob_bwd, b, lse, entropy, lse, d_W=torch.zeros((100, 64), dtype=BF16, device="cuda"), accumulate_dW=True) == -1
    assert status(spo.spo_logprob_bwd, b, lse, entropy, lse, chunk_tokens=-1) == -1
    with pytest.raises(TypeError):
        spo.make_logprob_desc(None, None, t, logits=z.t())
    with pytest.raises(TypeError):
        spo.make_logprob_desc(None, None, t, logits=z.half())
    with pytest.raises(TypeError):
        spo.make_logprob_desc(None, None, t.long(), logits=z)
    with pytest.raises(ValueError):
        spo.make_logprob_desc(None, None, t[:3], logits=z)
    with pytest.raises(ValueError):
        spo.make_logprob_desc(X, W[:, :32].contiguous(), t)
    with pytest.raises(ValueError):
        spo.spo_logprob_fwd(d, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
