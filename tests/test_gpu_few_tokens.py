"""Scores of a few tokens from hidden states: heads whose blocks of entries are shared by the wavefronts of a workgroup, and heads
where each has its own; all shapes against 64 bits.

Tolerance: that of the head form, 2e-4 absolute (fp32 sums over the hidden size)."""
import pytest
import torch

import score_cases as sc
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [2, 3, 16])
@pytest.mark.parametrize("H,V", [(64, 16384), (64, 16400), (192, 40001), (320, 9000), (704, 25000), (768, 24000), (768, 30000), (1024, 33000),
                                 (2048, 16385), (4096, 33000), (4352, 17000)])
def test_shared_and_own_blocks(T, H, V):
    g = torch.Generator().manual_seed(H + V + T)
    X = torch.randn((T, H), generator=g).to(torch.bfloat16)
    W = (torch.randn((V, H), generator=g) * H ** -0.5).to(torch.bfloat16)
    target = torch.randint(0, V, (T,), generator=g).int()
    target[0], target[-1] = V - 1, -1
    mask = torch.ones(T, dtype=torch.uint8)
    mask[1] = 0
    desc = spo.make_logprob_desc(X.cuda(), W.cuda(), target.cuda(), mask.cuda())
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(desc)
    again = spo.spo_logprob_fwd(desc)
    want = sc.scores(X.double() @ W.double().t(), target, mask)
    for x, y, name in ((logp, again[0], "logp"), (lse, again[1], "lse"), (entropy, again[2], "entropy")):
        torch.testing.assert_close(x.double().cpu(), want[name], atol=2e-4, rtol=2e-6, equal_nan=True)
        assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))     # and bit for bit the same again
