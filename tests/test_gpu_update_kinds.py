"""Orthogonalised updates of five steps on every kind of tiles in each product, against 64 bits.

Tolerances, from the steps carried out in 64 bits with the kernels' roundings of stored values and sums in fp32, 32 entries at a time:
matrices of more than 64 rows with fp16 products are 1.5e-4 to 9.4e-4 off, from 128 on at most 7.2e-4 (1.1e-3 and more without what
keeps the diagonals out of fp16): 9e-4.  Split products of matrices whose singular values are all of a size: 3e-7 to 6e-7, and the order
of the sums is another one: 2e-6; of nearly low rank 2.4e-6 to 3.4e-6: 7e-6."""
import pytest
import torch

import score_cases as sc
import update_kinds as uk
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu
BOUND = {uk.FP16: {"gradient": 9e-4, "low_rank": 9e-4}, uk.SPLIT: {"gradient": 2e-6, "low_rank": 7e-6}}


def stack(batch, rows, cols, kind, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    gauss = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    if kind == "gradient":  # few directions carry most of it
        left = gauss(batch, rows, 16) * torch.arange(1, 17, device="cuda") ** -0.5
        return torch.stack([gauss(rows, cols) + left[i] @ gauss(16, cols) for i in range(batch)])
    return torch.stack([0.05 * gauss(rows, cols) + gauss(rows, 4) @ gauss(4, cols) for i in range(batch)])


def off(x, want):
    return float((x.double() - want).norm() / want.norm())


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("case", uk.STACKS, ids=lambda c: "-".join(map(str, c)))
def test_orthogonalize(case, turned):
    batch, rows, cols, products = case[:4]
    if turned:
        rows, cols = cols, rows
    some = sorted({0, batch // 2, batch - 1})
    for kind in ("gradient", "low_rank"):
        G = stack(batch, rows, cols, kind, rows + batch)
        out = spo.spo_orthogonalize(G, products=products)
        for i in some:
            assert off(out[i], sc.orthogonal(G[i])) < BOUND[products][kind], (kind, i)
        assert torch.equal(out, spo.spo_orthogonalize(G, products=products))


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("case", uk.STACKS, ids=lambda c: "-".join(map(str, c)))
def test_momentum_step(case, turned):
    batch, rows, cols, products = case[:4]
    if turned:
        rows, cols = cols, rows
    lr, decay, scale, mu = 0.5, 0.1, 1.3, 0.9
    G, M, W = stack(batch, rows, cols, "gradient", 1), stack(batch, rows, cols, "gradient", 2), stack(batch, rows, cols, "gradient", 3) * 1e-3
    w, m = W.clone(), M.clone()
    spo.spo_muon_update(w, m, G, lr=lr, mu=mu, weight_decay=decay, scale=scale, products=products)
    for i in sorted({0, batch // 2, batch - 1}):
        M64 = mu * M[i].double() + G[i].double()
        assert off(m[i], M64) < 1e-6
        step = (w[i].double() - (1 - lr * decay) * W[i].double()) / (-lr * scale)
        # (W's own rounding, 2^-24 of entries that are no larger than the step's)
        assert off(step, sc.orthogonal(G[i].double() + mu * M64)) < BOUND[products]["gradient"] + 5e-7
