"""Orthogonalised updates of entries over fp32's whole range, and of matrices that are not finite.

Tolerance: that of split products elsewhere (3e-7 to 5e-6 in 64 bits with the kernels' roundings), 1.5e-5."""
import pytest
import torch

import score_cases as sc
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(100, 140), (140, 100), (2, 30, 70)])
@pytest.mark.parametrize("factor", [1e-37, 1e-30, 1e30, 1e37])
@pytest.mark.parametrize("steps", [0, 5])
def test_whole_range_of_entries(shape, factor, steps):
    G = torch.randn(shape, generator=torch.Generator().manual_seed(6)) * factor
    out = spo.spo_orthogonalize(G.cuda(), steps=steps, products=spo.SPO_PRODUCTS_SPLIT, eps=0.0)
    assert sc.rel(out, sc.orthogonal(G, steps=steps, eps=0.0)) < 1.5e-5


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("shape", [(70, 200), (200, 70)])
@pytest.mark.parametrize("steps", [0, 5])
def test_a_matrix_that_is_not_finite_is_nan_and_alone_so(bad, shape, steps):
    G = torch.randn((3, *shape), generator=torch.Generator().manual_seed(2))
    want = spo.spo_orthogonalize(G.cuda(), steps=steps)
    G[1, 5, 9] = bad
    out = spo.spo_orthogonalize(G.cuda(), steps=steps)
    assert torch.isnan(out[1]).all()
    assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])
