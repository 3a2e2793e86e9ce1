"""AdamW steps at their edges."""
import pytest
import torch

from pg_cases import say
from test_gpu_adamw import Case, spo  # noqa: F401

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def bits(u, dtype):
    """A number of these bits."""
    return torch.tensor([u - (1 << 32) if u >> 31 else u], dtype=torch.int32).view(F32) if dtype == F32 else \
        torch.tensor([u - (1 << 16) if u >> 15 else u], dtype=torch.int16).view(BF16)


@pytest.mark.parametrize("dtype,u", [(BF16, 0xffff), (BF16, 0xfff9), (BF16, 0xffc0), (BF16, 0x7fff), (F32, 0xffffffff), (F32, 0xfff80001), (F32, 0xff800001), (F32, 0x7fffffff)])
@pytest.mark.parametrize("zero_state", [False, True])
def test_gradients_of_any_nan_spoil_their_blocks(spo, dtype, u, zero_state):  # noqa: F811
    # memory filled with ones is one of them
    say(f"adamw, 8 bits, a gradient of {u:x}")
    c, clean = (Case(spo, [1000], 8, BF16, dtype, zero_state=zero_state) for _ in range(2))
    c.dev_g[0][70:71] = bits(u, dtype).cuda()
    c.dev_g[0][960:] = bits(u, dtype).cuda()
    assert bool(torch.isnan(c.dev_g[0][70])) and bool(torch.isnan(c.dev_g[0][999]))
    c.update(2), clean.update(2)
    spoilt = torch.zeros(1000, dtype=torch.bool)
    spoilt[64:128] = spoilt[960:] = True
    for got, want in zip(spo.spo_adamw_state_values(c.states[0]), spo.spo_adamw_state_values(clean.states[0])):
        assert torch.equal(got.cpu()[~spoilt], want.cpu()[~spoilt]) and bool(torch.isnan(got.cpu()[spoilt]).all())
    nan = torch.isnan(c.dev_p[0].cpu())
    assert bool(nan[70]) and bool(nan[960:].all()) and int(nan.sum()) == 41
    # and stay so
    c.dev_g[0].zero_()
    c.update(3)
    assert all(bool(torch.isnan(t.cpu()[spoilt]).all()) for t in spo.spo_adamw_state_values(c.states[0]))
