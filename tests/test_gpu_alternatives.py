"""Many alternatives of small vocabularies, where one bound leaves most logits as candidates: against a stable sort; and rows
that lie far from zero.

Ids are whole numbers and have to be equal; log-probs as in the other tests of scores (2e-5)."""
import pytest
import torch

import score_cases as sc
from paper_2509_13232_amd import binding as spo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 684, 1025, 1500, 2049, 3000])
@pytest.mark.parametrize("K", [33, 64])
@pytest.mark.parametrize("kind", ["noise", "ties", "falling", "rising", "negative", "sparse"])
def test_small_vocabularies(dtype, V, K, kind):
    g = torch.Generator().manual_seed(V + K)
    z = torch.randn((6, V), generator=g) * 3
    if kind == "ties":
        z = z.round()
    elif kind == "falling":
        z = -torch.arange(V).float().repeat(6, 1) / 8
    elif kind == "rising":
        z = torch.arange(V).float().repeat(6, 1) / 8 - 1000
    elif kind == "negative":
        z = -z.abs() - 1e4
    elif kind == "sparse":
        z[:, 40:] = float("-inf")
        z[3:] = z[3:].nan_to_num(neginf=torch.finfo(dtype).min)
    z = z.to(dtype)
    _, lse, _, ids, top = spo.spo_logprob_fwd(spo.make_logprob_desc(None, None, None, logits=z.cuda(), top_k=K))
    want = sc.scores(z.double(), None, None, K)
    assert torch.equal(ids.cpu().long(), want["top_id"])
    torch.testing.assert_close(top.double().cpu(), want["top_logp"], atol=2e-5, rtol=2e-6, equal_nan=True)
    torch.testing.assert_close(lse.double().cpu(), want["lse"], atol=2e-5, rtol=2e-6)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [700, 20000])
@pytest.mark.parametrize("offset", [100.0, -3000.0, 2e4, -1e5, 3e5])
def test_rows_far_from_zero(dtype, V, offset):
    g = torch.Generator().manual_seed(V)
    z = (torch.randn((5, V), generator=g) * 3 * (1 if dtype == torch.float32 else abs(offset) / 100) + offset).to(dtype)
    target = torch.randint(0, V, (5,), generator=g).int()
    logp, lse, entropy, _, _ = spo.spo_logprob_fwd(spo.make_logprob_desc(None, None, target.cuda(), logits=z.cuda()))
    want = sc.scores(z.double(), target)
    for x, name in ((logp, "logp"), (lse, "lse"), (entropy, "entropy")):
        torch.testing.assert_close(x.double().cpu(), want[name], atol=2e-5, rtol=2e-6)
