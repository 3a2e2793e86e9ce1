"""Scores from hidden states whose logits lie far from zero: the same for few tokens and for batches, exact to the sums.

The products are exact here (one-hot hidden states, weights of few bits), so what is left is the scores' own arithmetic.
Tolerance: that of the head form, 2e-4 absolute."""
import pytest
import torch

import score_cases as sc
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hv", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(1, 3000), (2, 700), (16, 40000), (17, 700), (40, 40000), (713, 3000)])
@pytest.mark.parametrize("base", [0.0, 100.0, -2944.0, 9984.0, -60928.0])
def test_forward(hv, dtype, T, V, base):
    H = 64
    g = torch.Generator().manual_seed(T + V)
    X = torch.zeros((T, H))
    X[:, 0] = 1
    X[torch.arange(T), 1 + torch.arange(T) % 9] = 1
    W = torch.randint(-128, 129, (V, H), generator=g) / 16.0     # base + W is exact in fp32, base and W are exact in bf16
    W[:, 0] = base
    X, W = X.to(dtype), W.to(dtype)
    z = X.double() @ W.double().t()
    assert torch.equal(z, z.float().double())
    target, mask = sc.targets(T, V, T), sc.mask_of(T, 2) if T > 20 else None
    d = spo.make_logprob_desc(X.cuda(), (W.t().contiguous() if hv else W).cuda(), target.cuda(), None if mask is None else mask.cuda(),
                              w_layout=spo.SPO_W_HV if hv else spo.SPO_W_VH)
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(d)
    want = sc.scores(z, target, mask)
    for x, name in ((logp, "logp"), (entropy, "entropy"), (lse, "lse")):
        torch.testing.assert_close(x.double().cpu(), want[name], atol=2e-4, rtol=2e-6)
