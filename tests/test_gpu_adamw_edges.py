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


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-37, 1e-40, 1e-46, 1e-300])
@pytest.mark.parametrize("on_device", [False, True])
def test_any_eps_above_zero_keeps_what_has_no_moments(spo, bits, eps, on_device):  # noqa: F811
    say(f"adamw, {bits} bits, eps {eps}")
    n = 1000
    p0 = torch.linspace(-1, 1, n).cuda()
    p, g = p0.clone(), torch.zeros(n, device="cuda")
    g[100:400] = 1e-3
    d = spo.make_adamw_desc([p], [g], [spo.adamw_state(p, bits)])
    spo.spo_adamw_update(d, 1e-2, torch.zeros(1, dtype=torch.int64, device="cuda") if on_device else 1, eps=eps)
    still = g == 0
    assert torch.equal(p[still], p0[still])
    # the others take the first step's lr: 12 roundings of 2^-24 of it, and one of p's
    assert float((p0[~still] - p[~still] - 1e-2).abs().max()) < 1e-2 * 1e-6 + 2.0 ** -24


def test_workspaces_in_host_memory_or_with_holes_are_refused(spo):  # noqa: F811
    say("workspaces that are refused")
    U8 = torch.uint8
    x, w, p = torch.zeros((5, 100), device="cuda"), torch.zeros(100, device="cuda"), torch.zeros(5, device="cuda")
    norm, step = spo.make_norm_desc(x, w), spo.make_adamw_desc([p], [torch.zeros_like(p)], [spo.adamw_state(p)])
    a, idx, r = torch.ones(16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    score = spo.make_logprob_desc(None, None, idx, logits=torch.zeros((4, 64), device="cuda"))
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    calls = [
        lambda ws: spo.spo_norm_bwd(norm, p, p, x, workspace=ws),
        lambda ws: spo.spo_grad_norm(step, workspace=ws),
        lambda ws: spo.spo_adamw_update(step, 0.1, count, workspace=ws),
        lambda ws: spo.spo_logprob_fwd(score, workspace=ws),
        lambda ws: spo.spo_sample_prompts(a, a.clone(), 4, workspace=ws),
        lambda ws: spo.spo_advantages(a, a.clone(), idx, r, workspace=ws),
        lambda ws: spo.spo_tracker_update(a, a.clone(), idx, r, r, 0.25, 0.875, 0.96, ids_unique=False, workspace=ws),
    ]
    room = torch.zeros(1 << 21, dtype=U8, device="cuda")
    for k, call in enumerate(calls):
        for bad in (torch.zeros(1 << 20, dtype=U8), torch.zeros(1 << 20, dtype=U8, pin_memory=True), room[::2], room[:1].expand(1 << 20)):
            with pytest.raises(ValueError, match="workspace"):
                call(bad)
        call(room)
    torch.cuda.synchronize()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("on_device", [False, True])
def test_a_norm_without_a_limit_clips_nothing(spo, bits, on_device):  # noqa: F811
    say(f"adamw with a norm and no limit, {bits} bits")
    c, bad = Case(spo, [5000, 64], bits), float("inf")
    number = torch.full((1,), 1, dtype=torch.int64, device="cuda") if on_device else 2
    c.update(number, grad_norm=spo.spo_grad_norm(c.desc))
    c.check(2, factor=torch.tensor(1.0))
    c.dev_g[0][17] = bad
    before = [t.clone() for t in (*c.dev_p, *(x for s in c.states for x in s if x is not None))]
    c.update(number if on_device else 3, grad_norm=spo.spo_grad_norm(c.desc))
    assert all(torch.equal(a, b) for a, b in zip((*c.dev_p, *(x for s in c.states for x in s if x is not None)), before))
