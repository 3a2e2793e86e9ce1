"""Gradients of scores of rows that lie far from zero, where a log-sum-exp rounded to fp32 is no longer exact beside them.

Tolerances as in the other tests of scores: 1e-5 in 2-norm in fp32, 3e-3 in bf16 (one rounding)."""
import pytest
import torch

import score_cases as sc
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu
GRAD = {torch.float32: 1e-5, torch.bfloat16: 3e-3}


# rows within one segment, of two, of a few, of many; few rows and many
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (9, 300, 4), (300, 700, 0), (5, 1001, 64), (7, 5000, 0), (1, 151936, 20), (300, 20000, 3), (40, 100003, 0)])
@pytest.mark.parametrize("offset", [100.0, -150.0, -3000.0, 2e4, 6e4, -3e5])
def test_gradient(dtype, T, V, K, offset):
    g = torch.Generator().manual_seed(T + V)
    z = (torch.randn((T, V + 5), generator=g) * 3 + offset).to(dtype)
    z[T // 2] = sc.logits(1, V + 5, dtype, 1)[0]         # an ordinary row among them
    part, target, mask = z[:, 2:V + 2], sc.targets(T, V, T), sc.mask_of(T, V) if T > 8 else None
    d = spo.make_logprob_desc(None, None, target.cuda(), None if mask is None else mask.cuda(), logits=z.cuda()[:, 2:V + 2], top_k=K)
    _, lse, entropy, ids, _ = spo.spo_logprob_fwd(d)
    a, e, b = sc.factors(T, 1), sc.factors(T, 2), sc.factors((T, K), 3) if K else None
    dz = spo.spo_logprob_bwd(d, lse, entropy, a.cuda(), e.cuda(), ids, None if b is None else b.cuda())
    again = spo.spo_logprob_bwd(d, lse, entropy, a.cuda(), e.cuda(), ids, None if b is None else b.cuda())
    want = sc.d_logits(part.double(), target, mask, a, e, None if b is None else ids.cpu(), b)
    assert sc.rel(dz, want) < GRAD[dtype] and torch.equal(dz, again)
