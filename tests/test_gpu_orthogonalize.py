"""Orthogonalised updates and the momentum step against their definitions in 64 bits.

Tolerances: in 64 bits with the kernels' roundings, five steps are 2e-4 to 1.7e-3 off with fp16 products (bound 3e-3; a bf16
output adds one rounding of at most 2^-9: 4e-3) and 3e-7 to 5e-6 with split ones (bound 1.5e-5)."""
import pytest
import torch

import score_cases as sc
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
FP16, SPLIT = spo.SPO_PRODUCTS_FP16, spo.SPO_PRODUCTS_SPLIT
BOUND = {FP16: 3e-3, SPLIT: 1.5e-5}


def matrices(shape, seed, kind="gradient"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if kind == "gradient":  # few directions carry most of it
        r = min(shape[-1], shape[-2], 16)
        left = torch.randn((*shape[:-1], r), generator=g) * torch.arange(1, r + 1) ** -0.5
        x = x + left @ torch.randn((*shape[:-2], r, shape[-1]), generator=g)
    elif kind == "low_rank":
        r = min(shape[-1], shape[-2], 4)
        x = 0.05 * x + torch.randn((*shape[:-1], r), generator=g) @ torch.randn((*shape[:-2], r, shape[-1]), generator=g)
    return x


SHAPES = [(1, 1), (1, 7), (9, 1), (16, 16), (3, 200), (64, 64), (65, 63), (130, 257), (257, 130), (200, 1000), (1000, 200), (512, 512), (384, 640)]


@pytest.mark.parametrize("products", [FP16, SPLIT])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", ["gradient", "low_rank"])
def test_orthogonalize(products, shape, kind):
    G = matrices(shape, sum(shape), kind)
    out = spo.spo_orthogonalize(G.cuda(), products=products)
    assert out.dtype == F32 and sc.rel(out, sc.orthogonal(G)) < BOUND[products]
    B = G.to(BF16)
    out = spo.spo_orthogonalize(B.cuda(), products=products)
    assert out.dtype == BF16 and sc.rel(out, sc.orthogonal(B)) < 4e-3


@pytest.mark.parametrize("products", [FP16, SPLIT])
@pytest.mark.parametrize("shape", [(5, 40, 100), (3, 300, 130), (2, 1, 1), (20, 256, 256), (40, 300, 200), (3, 1100, 1030)])
def test_stacks(products, shape):
    G = matrices(shape, 3)
    G[0] *= 1e-6        # each matrix has its own norm
    if shape[0] > 2:
        G[2] = 0
    out = spo.spo_orthogonalize(G.cuda(), products=products)
    want = sc.orthogonal(G)
    for i in range(shape[0]):
        if i == 2:
            assert (out[i] == 0).all()
        elif i == 0:    # eps is 1e-7: seen beside a norm of 1e-4
            assert sc.rel(out[i], want[i]) < BOUND[products]
        else:
            assert sc.rel(out[i], want[i]) < BOUND[products]


@pytest.mark.parametrize("steps,coeffs", [(0, sc.NEWTON_SCHULZ), (1, sc.NEWTON_SCHULZ), (2, (2.0, -1.5, 0.5)), (12, (1.875, -1.25, 0.375))])
def test_steps_and_coefficients(steps, coeffs):
    for shape in ((70, 50), (96, 300)):
        G = matrices(shape, 5, "gauss")
        for products, dtype in ((FP16, BF16), (SPLIT, F32)):
            x = G.to(dtype)
            out = spo.spo_orthogonalize(x.cuda(), steps=steps, coeffs=coeffs, products=products)
            assert sc.rel(out, sc.orthogonal(x, steps, coeffs)) < (4e-3 if dtype == BF16 else 1.5e-5)


def test_rows_and_matrices_apart():
    whole = matrices((3, 90, 170), 8)
    for part in (whole[:, 2:80, 5:155], whole[::2, ::3, 1:60], whole[1:2, :, :91], whole[0, 3:4, 7:150], whole.transpose(0, 1)[:, 1:2, 3:50]):
        g = whole.cuda()
        sub = g.as_strided(part.size(), part.stride(), part.storage_offset())
        out = spo.spo_orthogonalize(sub, products=SPLIT)
        assert out.is_contiguous() and sc.rel(out, sc.orthogonal(part)) < 1.5e-5


def test_output_types_and_in_place():
    G = matrices((120, 77), 4)
    want = sc.orthogonal(G)
    assert sc.rel(spo.spo_orthogonalize(G.cuda(), out_dtype=BF16), want) < 4e-3
    held = G.cuda()
    assert spo.spo_orthogonalize(held, out=held, products=SPLIT) is held and sc.rel(held, want) < 1.5e-5
    again = [spo.spo_orthogonalize(G.cuda()) for _ in range(2)]
    assert torch.equal(*again)


def test_values_far_from_one():
    G = matrices((100, 140), 6)
    for f in (1e-18, 1e18):      # squares beyond fp32
        assert sc.rel(spo.spo_orthogonalize((G * f).cuda(), products=SPLIT, eps=0.0), sc.orthogonal(G * f, eps=0.0)) < 1.5e-5
    G[3, 5] = float("nan")
    assert torch.isnan(spo.spo_orthogonalize(G.cuda())).any()
    assert (spo.spo_orthogonalize(torch.zeros((50, 60), device="cuda"), eps=0.0) == 0).all()


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("shape,g_dtype,w_dtype", [((96, 200), F32, F32), ((300, 130), BF16, F32), ((4, 64, 77), BF16, BF16), ((2, 33, 20), F32, BF16)])
def test_momentum_step(nesterov, shape, g_dtype, w_dtype):
    lr, mu, wd, scale = 0.02, 0.9, 0.1, 1.7
    W, M = matrices(shape, 1, "gauss").to(w_dtype), matrices(shape, 2)
    w, m = W.cuda(), M.cuda()
    W64, M64 = W.double(), M.double()
    for step in range(3):
        G = matrices(shape, 10 + step).to(g_dtype)
        spo.spo_muon_update(w, m, G.cuda(), lr=lr, mu=mu, nesterov=nesterov, weight_decay=wd, scale=scale, products=SPLIT)
        M64 = mu * M64 + G.double()
        U = G.double() + mu * M64 if nesterov else M64
        W64 = (1 - lr * wd) * W64 - lr * scale * sc.orthogonal(U)
        assert sc.rel(m, M64) < 1e-6
        # the update itself, to the bound of split products and the rounding of W (2^-24 of it, per step; bf16 2^-9)
        assert sc.rel(w, W64) < (2e-6 if w_dtype == F32 else 6e-3)
        if w_dtype == BF16:
            W64 = w.double().cpu()
    # fp16 products: 3e-3 of an update, which is a hundredth of W
    w2, m2 = W.cuda(), M.cuda()
    G = matrices(shape, 10).to(g_dtype)
    spo.spo_muon_update(w2, m2, G.cuda(), lr=lr, mu=mu, nesterov=nesterov)
    M64 = mu * M.double() + G.double()
    O = sc.orthogonal(G.double() + mu * M64 if nesterov else M64)
    s = max(1.0, shape[-2] / shape[-1]) ** 0.5
    if w_dtype == F32:
        assert sc.rel((W.cuda() - w2) / (lr * s), O) < 3e-3 + 1e-4     # 2^-24 of W beside lr of it


def test_a_captured_step_replays():
    W, M, G = (matrices((3, 100, 60), i).cuda() for i in range(3))
    ws = torch.empty(spo.spo_orthogonalize_workspace_bytes(3, 100, 60), dtype=torch.uint8, device="cuda")
    step = lambda w, m: spo.spo_muon_update(w, m, G, lr=0.1, weight_decay=0.01, workspace=ws)
    step(W.clone(), M.clone())
    torch.cuda.synchronize()
    w, m = W.clone(), M.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(w, m)
    w.copy_(W), m.copy_(M)
    we, me = W.clone(), M.clone()
    for i in range(3):
        G.copy_(matrices((3, 100, 60), 20 + i))
        graph.replay()
        torch.cuda.synchronize()
        step(we, me)
        assert torch.equal(w, we) and torch.equal(m, me)


def test_refusals():
    G = torch.zeros((8, 9), device="cuda")
    status = lambda f, *a, **k: pytest.raises(spo.SpoError, f, *a, **k).value.status
    for kw in (dict(steps=-1), dict(products=7), dict(eps=-1.0), dict(eps=float("nan"))):
        assert status(spo.spo_orthogonalize, G, **kw) == -1
    assert status(spo.spo_orthogonalize, G, steps=65) == -3
    assert status(spo.spo_orthogonalize, torch.zeros((1, 65537), device="cuda")) == -3
    for kw in (dict(mu=1.0), dict(mu=-0.1), dict(lr=-1.0), dict(weight_decay=-1.0), dict(scale=float("nan"))):
        assert status(spo.spo_muon_update, G.clone(), G.clone(), G, **{"lr": 0.1, **kw}) == -1
    with pytest.raises(TypeError):
        spo.spo_orthogonalize(G.t())
    with pytest.raises(TypeError):
        spo.spo_orthogonalize(G.half())
    with pytest.raises(TypeError):
        spo.spo_orthogonalize(G[:1].expand(4, 9))
    with pytest.raises(ValueError):
        spo.spo_orthogonalize(G[0])
    with pytest.raises(ValueError):
        spo.spo_orthogonalize(G, out=torch.zeros((8, 8), device="cuda"))
    with pytest.raises(TypeError):
        spo.spo_muon_update(G, G.to(BF16), G, lr=0.1)
    with pytest.raises(ValueError):
        spo.spo_muon_update(G, G.clone(), G[:4].contiguous(), lr=0.1)
