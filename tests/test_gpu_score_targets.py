"""Target ids outside the vocabulary: a NaN log-prob, and no one-hot term in any gradient, whatever the bits of the id.

Tolerances as in the other tests of scores: head gradients 1e-2 in 2-norm (bf16 logit gradients); from logits in fp32 1e-5."""
import pytest
import torch

import score_cases as sc
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu
LOWEST = -(1 << 31)


def _ids(V):
    # the first half is valid; an id must not come back as another one when a bit of it is taken off, nor as a padded entry
    return torch.tensor([0, 5, V - 1, 7, LOWEST, LOWEST + 5, LOWEST + V - 1, -1, -100, V, V + 1, V + 20, 1 << 30, (1 << 31) - 1], dtype=torch.int32)


@pytest.mark.parametrize("hv", [False, True])
@pytest.mark.parametrize("V", [10, 700, 3000])
@pytest.mark.parametrize("copies", [1, 30])
def test_head_gradient(hv, V, copies):
    target = _ids(V).repeat(copies)
    T, H = target.numel(), 128
    g = torch.Generator().manual_seed(V + copies)
    X = torch.randn((T, H), generator=g).to(torch.bfloat16)
    W = (torch.randn((V, H), generator=g) * 0.2).to(torch.bfloat16)
    a, e = sc.factors(T, 1), 0.1 * sc.factors(T, 2)
    d = spo.make_logprob_desc(X.cuda(), (W.t().contiguous() if hv else W).cuda(), target.cuda(), w_layout=spo.SPO_W_HV if hv else spo.SPO_W_VH)
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    assert torch.equal(torch.isnan(logp).cpu(), (target < 0) | (target >= V)) and torch.isfinite(lse).all()
    dx, dw = spo.spo_logprob_bwd(d, lse, entropy, a.cuda(), e.cuda(), d_hidden_dtype=torch.float32)
    dz = sc.d_logits(X.double() @ W.double().t(), target, None, a, e)
    want_x, want_w = dz @ W.double(), dz.t() @ X.double()
    assert sc.rel(dx, want_x) < 1e-2 and sc.rel(dw, want_w.t() if hv else want_w) < 1e-2
    outside = (target < 0) | (target >= V)
    assert sc.rel(dx[outside.cuda()], want_x[outside]) < 1e-2      # on their own: softmax parts only


@pytest.mark.parametrize("V", [10, 700, 9000])
def test_logits_gradient(V):
    target = _ids(V)
    T = target.numel()
    z = sc.logits(T, V, torch.float32, V)
    a, e = sc.factors(T, 1), sc.factors(T, 2)
    d = spo.make_logprob_desc(None, None, target.cuda(), logits=z.cuda())
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    assert torch.equal(torch.isnan(logp).cpu(), (target < 0) | (target >= V))
    dz = spo.spo_logprob_bwd(d, lse, entropy, a.cuda(), e.cuda())
    assert sc.rel(dz, sc.d_logits(z.double(), target, None, a, e)) < 1e-5
