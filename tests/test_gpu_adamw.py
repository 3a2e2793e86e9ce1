"""AdamW steps over many tensors, the norm of their gradients and 8-bit states, against their definitions.

Bounds.  Moments are chains of single roundings in fp32: they are compared with the same chain on the CPU, bit for bit, and so are
codes (a code's place among its neighbours is exact arithmetic).  The change of a weight is a handful of fp32 operations on factors
that are rounded once each: 12 roundings of 2^-24 = 7.2e-7 of its size, bounded by 1e-6; then one rounding to the weight's type."""
import math

import pytest
import torch

import train_cases as tc
from pg_cases import say

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
B1, B2, EPS = 0.9, 0.999, 1e-8


@pytest.fixture(scope="module")
def spo():
    from paper_2509_13232_amd import binding
    binding.lib()
    return binding


def place(t, shift=0):
    """A copy on the GPU, `shift` elements behind an aligned address."""
    out = torch.zeros(t.numel() + shift + 8, dtype=t.dtype, device="cuda")
    out[shift:shift + t.numel()] = t.cuda()
    return out[shift:shift + t.numel()]


class Case:
    """Tensors of the given sizes on the CPU, with a state that some steps have left."""

    def __init__(self, spo, sizes, bits, p_dtype=F32, g_dtype=F32, seed=0, shift=0, copies=False, decay=0.01, zero_state=False):
        g = torch.Generator().manual_seed(seed * 7 + len(sizes))
        self.spo, self.bits, self.sizes, self.decay, self.shift = spo, bits, sizes, decay, shift
        rand = lambda n: torch.randn(n, generator=g)   # noqa: E731
        scale = [1e-2 * torch.exp(rand(-(-n // 64))).repeat_interleave(64)[:n] for n in sizes]
        self.p = [(rand(n) * 0.1).to(p_dtype) for n in sizes]
        self.g = [(rand(n) * s).to(g_dtype) for n, s in zip(sizes, scale)]
        self.m = [rand(n) * 0.3 * s for n, s in zip(sizes, scale)]
        self.v = [(torch.exp(0.5 * rand(n)) * s) for n, s in zip(sizes, scale)]        # the root, so far
        for m, v in zip(self.m, self.v):
            if zero_state:
                m.zero_(), v.zero_()
        if bits == 32:
            self.v = [v * v for v in self.v]
            states = [spo.AdamwState(place(m, shift), place(v, shift)) for m, v in zip(self.m, self.v)]
        else:
            coded = [(tc.encode(m, 3, 5), tc.encode(v, 4, 5)) for m, v in zip(self.m, self.v)]
            self.m = [tc.decode(*c[0], 3) for c in coded]
            self.v = [tc.decode(*c[1], 4) for c in coded]
            states = [spo.AdamwState(*(place(t, shift) for t in (a[0], b[0], a[1], b[1]))) for a, b in coded]
        self.states = states
        self.dev_p, self.dev_g = [place(p, shift) for p in self.p], [place(t, shift) for t in self.g]
        self.copies = [place(torch.zeros(n, dtype=BF16), shift) for n in sizes] if copies else None
        decays = decay if isinstance(decay, list) else [decay] * len(sizes)
        self.decays = decays
        self.desc = spo.make_adamw_desc(self.dev_p, self.dev_g, states, weight_decay=decay, copies=self.copies)

    def update(self, step, lr=1e-3, **kw):
        self.spo.spo_adamw_update(self.desc, lr, step, beta1=B1, beta2=B2, eps=EPS, **kw)
        torch.cuda.synchronize()

    def check(self, step, lr=1e-3, factor=None, p_bound=1.0):
        """The state and the weights after the step from what they were; remembers what they are."""
        for i, n in enumerate(self.sizes):
            g = self.g[i].float()
            if factor is not None:
                g = g * factor
            m, v = tc.moments(g, self.m[i], self.v[i], B1, B2, root=self.bits == 8)
            s = self.states[i]
            if self.bits == 32:
                assert torch.equal(s.m.cpu(), m) and torch.equal(s.v.cpu(), v), (i, n)
                v64 = self.v[i].double()
                new_state = m, v
            else:
                (mc, ms), (vc, vs) = tc.encode(m, 3, step), tc.encode(tc.root(v), 4, step)
                for got, want, name in ((s.m, mc, "m"), (s.m_scale, ms, "m_scale"), (s.v, vc, "v"), (s.v_scale, vs, "v_scale")):
                    bad = (got.cpu() != want).nonzero()
                    assert not bad.numel(), (i, n, name, len(bad), bad[:4].tolist())
                v64 = self.v[i].double() ** 2
                new_state = tc.decode(mc, ms, 3), tc.decode(vc, vs, 4)
            want, _, _, size = tc.adamw(self.p[i].double(), g.double(), self.m[i].double(), v64, step, lr, B1, B2, EPS, self.decays[i])
            p = self.dev_p[i].cpu()
            tc.off(p, want, 1e-6 * size + tc.EPS_HALF[p.dtype] * p_bound * 1.01 * want.abs() + 2.0 ** -24 * want.abs(), ("param", i, n))
            if self.copies:
                assert torch.equal(self.copies[i].cpu(), p.to(BF16))
            self.p[i] = p
            self.m[i], self.v[i] = new_state


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_dtype,g_dtype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("sizes", [[1], [64], [4096], [7, 63, 65, 2048, 8191, 8192, 8193], [100000, 3, 0, 513]])
def test_steps_follow_the_definition(spo, bits, p_dtype, g_dtype, sizes):
    say(f"adamw {bits} bits {p_dtype} {g_dtype} {sizes}")
    c = Case(spo, sizes, bits, p_dtype, g_dtype, copies=p_dtype == F32)
    for step in (1, 2, 100, 5000):
        c.update(step)
        c.check(step)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [1, 3])
def test_tensors_that_are_not_aligned(spo, bits, shift):
    say(f"adamw {bits} bits, {shift} elements off")
    for p_dtype in (F32, BF16):
        c = Case(spo, [5, 1000, 20001], bits, p_dtype, BF16, shift=shift, copies=p_dtype == F32)
        before = [t._base.clone() for t in c.dev_p] if c.dev_p[0]._base is not None else None
        c.update(3)
        c.check(3)
        if before is not None:     # what lies around the tensors stays
            for t, b, n in zip(c.dev_p, before, c.sizes):
                assert torch.equal(t._base[:shift], b[:shift]) and torch.equal(t._base[shift + n:], b[shift + n:])


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_launch_takes(spo, bits):
    say(f"adamw of 333 tensors, {bits} bits")
    g = torch.Generator().manual_seed(4)
    sizes = [int(10 ** (torch.rand(1, generator=g) * 4)) for _ in range(333)]
    c = Case(spo, sizes, bits, F32, BF16, copies=True, decay=[0.0 if i % 3 else 0.1 for i in range(333)])
    norm = spo.spo_grad_norm(c.desc)
    want = torch.sqrt(sum((t.double() ** 2).sum() for t in c.g)).float()
    assert float(norm) == float(want)
    limit = float(want) / 3
    c.update(7, grad_norm=norm, max_norm=limit)
    c.check(7, factor=torch.tensor(limit, dtype=F32) / norm.cpu())


@pytest.mark.parametrize("bits", [32, 8])
def test_state_from_zero(spo, bits):
    say(f"adamw from a state of zeros, {bits} bits")
    c = Case(spo, [1000, 77], bits, zero_state=True)
    fresh = [spo.adamw_state(p, bits) for p in c.dev_p]
    for a, b in zip(fresh, c.states):
        assert all(x is None and y is None or torch.equal(x, y) or name.endswith("scale") for x, y, name in zip(a, b, a._fields))
    c.states = fresh
    c.desc = spo.make_adamw_desc(c.dev_p, c.dev_g, fresh, weight_decay=c.decay)
    c.g[0][100:200] = 0      # (no gradient: the weights only decay)
    c.dev_g[0][100:200] = 0
    for step in (1, 2, 3):
        c.update(step)
        c.check(step)


# ------------------------------------------------------------------ the norm, clipping
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("sizes", [[1], [8193, 5, 300000], [0], [], [1 << 22, 100]])
def test_norm_of_gradients_is_the_rounded_one(spo, dtype, sizes):
    say(f"norm of gradients {sizes} {dtype}")
    c = Case(spo, sizes, 32, F32, dtype)
    want = torch.sqrt(sum(((t.double() ** 2).sum() for t in c.g), torch.zeros((), dtype=torch.float64)))
    got = spo.spo_grad_norm(c.desc).cpu().double()
    # sums of exact squares in 64 bits: n roundings of 2^-53 at most, and one of 2^-24
    assert abs(float(got) - float(want)) <= float(want) * (2.0 ** -24 + sum(sizes) * 2.0 ** -53)


@pytest.mark.parametrize("value,want", [(1e30, 1e30 * 30), (1e-30, 1e-30 * 30), (float("inf"), float("inf")), (float("nan"), float("nan")), (3e38, float("inf"))])
def test_norm_over_the_whole_range(spo, value, want):
    say(f"norm of gradients of {value}")
    grad = torch.full((900,), value, device="cuda")
    p = torch.zeros(900, device="cuda")
    got = float(spo.spo_grad_norm(spo.make_adamw_desc([p], [grad], [spo.adamw_state(p)])))
    assert got == pytest.approx(want, rel=1e-6, nan_ok=True)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("limit", [1e9, 0.3, 0.0])
def test_clipping(spo, bits, limit):
    say(f"adamw clipped to {limit}, {bits} bits")
    c = Case(spo, [5000, 64], bits)
    norm = spo.spo_grad_norm(c.desc)
    c.update(2, grad_norm=norm, max_norm=limit)
    n = norm.cpu()
    c.check(2, factor=torch.tensor(limit, dtype=F32) / n if float(n) > limit else torch.tensor(1.0))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("on_device", [False, True])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_norm_that_is_not_finite_changes_nothing(spo, bits, on_device, bad):
    say(f"adamw skipped, {bits} bits, norm {bad}")
    c = Case(spo, [5000, 64], bits, copies=True)
    c.dev_g[0][17] = bad
    before = [t.clone() for t in (*c.dev_p, *c.copies, *(x for s in c.states for x in s if x is not None))]
    step = torch.full((1,), 6, dtype=torch.int64, device="cuda") if on_device else 7
    c.update(step, grad_norm=spo.spo_grad_norm(c.desc), max_norm=1.0)
    after = (*c.dev_p, *c.copies, *(x for s in c.states for x in s if x is not None))
    assert all(torch.equal(a, b) for a, b in zip(after, before)) and int(step) == (6 if on_device else 7)
    c.dev_g[0][17] = c.g[0][17]
    c.update(step, grad_norm=spo.spo_grad_norm(c.desc), max_norm=1e9)
    assert int(step) == 7
    c.check(7, factor=torch.tensor(1.0))


@pytest.mark.parametrize("bits", [32, 8])
def test_without_a_norm_what_is_not_finite_stays_in_its_place(spo, bits):
    say(f"adamw with gradients that are not finite, {bits} bits")
    c = Case(spo, [1000], bits)
    clean = Case(spo, [1000], bits)
    c.dev_g[0][70], c.dev_g[0][700] = float("nan"), float("inf")
    c.update(2), clean.update(2)
    where = torch.zeros(1000, dtype=torch.bool)
    where[70] = where[700] = True
    p, q = c.dev_p[0].cpu(), clean.dev_p[0].cpu()
    assert torch.equal(p[~where], q[~where]) and bool(torch.isnan(p[where]).all())
    held = spo.spo_adamw_state_values(c.states[0]) if bits == 8 else c.states[0][:2]
    others = spo.spo_adamw_state_values(clean.states[0]) if bits == 8 else clean.states[0][:2]
    spoilt = torch.zeros(1000, dtype=torch.bool)     # in 8 bits a block is held together
    spoilt[64:128] = spoilt[640:704] = True
    if bits == 32:
        spoilt = where
    for a, b in zip(held, others):
        assert torch.equal(a.cpu()[~spoilt], b.cpu()[~spoilt]) and not bool(torch.isfinite(a.cpu()[spoilt]).any())


# ------------------------------------------------------------------ numbers on the device, graphs
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr_there", [False, True])
@pytest.mark.parametrize("step_there", [False, True])
def test_step_and_rate_on_the_device(spo, bits, lr_there, step_there):
    say(f"adamw, numbers on the device, {bits} bits")
    here, there = Case(spo, [3000, 5], bits, BF16, BF16), Case(spo, [3000, 5], bits, BF16, BF16)
    lr = float(torch.tensor(3e-4, dtype=F32))
    lr_t = torch.full((1,), lr, device="cuda") if lr_there else lr
    step_t = torch.full((1,), 8, dtype=torch.int64, device="cuda")
    for step in (9, 10, 11):
        here.update(step, lr=lr, rounding=spo.SPO_ROUND_THRESHOLD)
        there.update(step_t if step_there else step, lr=lr_t, rounding=spo.SPO_ROUND_THRESHOLD)
    assert int(step_t) == (11 if step_there else 8)
    for a, b in zip(here.dev_p + [x for s in here.states for x in s if x is not None], there.dev_p + [x for s in there.states for x in s if x is not None]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_replay_from_graphs(spo, bits):
    # two graphs of the same program share a workspace, and eager steps go between their replays
    say(f"adamw in graphs, {bits} bits")
    sizes = [4096, 999, 70000]
    eager, caught = (Case(spo, sizes, bits, F32, BF16, copies=True) for _ in range(2))
    lr = torch.full((1,), 1e-3, device="cuda")
    ws = torch.empty(max(spo.spo_grad_norm_workspace_bytes(caught.desc), 256), dtype=torch.uint8, device="cuda")
    steps = [torch.zeros(1, dtype=torch.int64, device="cuda") for _ in range(2)]

    def step(c, count):
        norm = spo.spo_grad_norm(c.desc, workspace=ws)
        spo.spo_adamw_update(c.desc, lr, count, grad_norm=norm, max_norm=0.5, workspace=ws)
        return norm

    def snapshot(c):
        return [t.clone() for t in (*c.dev_p, *c.copies, *(x for s in c.states for x in s if x is not None))]

    start = snapshot(caught)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caught, steps[1])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            norm = step(caught, steps[1])
    for t, s in zip((*caught.dev_p, *caught.copies, *(x for s in caught.states for x in s if x is not None)), start):
        t.copy_(s)
    steps[1].zero_()
    for k in range(6):
        g = torch.Generator().manual_seed(100 + k)
        for a, b in zip(eager.dev_g, caught.dev_g):
            fresh = (torch.randn(a.numel(), generator=g) * 0.01).to(a)
            a.copy_(fresh), b.copy_(fresh)
        lr.fill_(1e-3 / (k + 1))
        step(eager, steps[0])
        if k == 4:
            step(caught, steps[1])
        else:
            graphs[k % 2].replay()
        torch.cuda.synchronize()
        (torch.randn(1 << 20, device="cuda") * 1.0001).sin_()
        torch.cuda.synchronize()
        assert int(steps[0]) == int(steps[1]) == k + 1
        assert all(torch.equal(a, b) for a, b in zip(snapshot(eager), snapshot(caught))), k
    assert float(norm) > 0


def test_on_another_stream(spo):
    say("adamw on a stream")
    a, b = Case(spo, [70000], 8), Case(spo, [70000], 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        spo.spo_adamw_update(a.desc, 1e-3, 3, grad_norm=spo.spo_grad_norm(a.desc), max_norm=0.1)
    torch.cuda.synchronize()
    b.update(3, grad_norm=spo.spo_grad_norm(b.desc), max_norm=0.1)
    assert torch.equal(a.dev_p[0], b.dev_p[0]) and torch.equal(a.states[0].m, b.states[0].m)


# ------------------------------------------------------------------ rounding to few bits
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 8191, 100000])
def test_values_of_a_state(spo, n, dtype):
    say(f"values of {n} codes")
    g = torch.Generator().manual_seed(n)
    codes = [torch.randint(0, 256, (n,), generator=g).to(torch.uint8) for _ in range(2)]
    scales = [torch.randint(15, 256, (-(-n // 64),), generator=g).to(torch.uint8) for _ in range(2)]
    for s in scales:
        s[0] = 15
    m, root = spo.spo_adamw_state_values(spo.AdamwState(*(t.cuda() for t in (*codes, *scales))), dtype=dtype)
    for got, c, s, mantissa in ((m, codes[0], scales[0], 3), (root, codes[1], scales[1], 4)):
        want = tc.decode(c, s, mantissa)
        assert got.dtype == dtype and torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
        ok = ~torch.isnan(want)
        assert torch.equal(got.cpu().float()[ok], want[ok])      # bf16 holds them exactly


def test_every_step_reaches_codes_as_defined(spo):
    # thresholds of many steps, beyond 2^32 of them too; small and large numbers; blocks that end early
    say("codes over steps")
    c = Case(spo, [64 * 40 + 9], 8)
    c.dev_g[0][:64] *= 1e-30
    c.dev_g[0][64:128] *= 1e18
    c.g[0] = c.dev_g[0].cpu()
    for step in (1, 2, 3, 4, 5, 1000, 12345678, (1 << 32) + 7, (1 << 40) + 3):
        c.update(step, lr=0.0)
        c.check(step, lr=0.0)


@pytest.mark.parametrize("scale", [1.0, 1e-19, 1e-22])
def test_codes_of_many_elements(spo, scale):
    # enough roots that hundreds lie beside a code's border, and squares down to where fp32 has no more of them
    say(f"8-bit codes of many elements, {scale}")
    n = 6 << 20
    g = torch.Generator().manual_seed(11)
    grad = torch.randn(n, generator=g) * torch.exp(2 * torch.randn(n, generator=g)) * scale
    p = torch.zeros(n, device="cuda")
    state = spo.adamw_state(p, 8)
    desc = spo.make_adamw_desc([p], [grad.cuda()], [state])
    m, v = torch.zeros(n), torch.zeros(n)
    for step in (1, 2, 3):
        spo.spo_adamw_update(desc, 1e-3, step, beta1=B1, beta2=B2, eps=EPS)
        torch.cuda.synchronize()
        m, v = tc.moments(grad, m, v, B1, B2, root=True)
        (mc, ms), (vc, vs) = tc.encode(m, 3, step), tc.encode(tc.root(v), 4, step)
        assert torch.equal(state.m_scale.cpu(), ms) and torch.equal(state.v_scale.cpu(), vs), step
        assert torch.equal(state.m.cpu(), mc) and torch.equal(state.v.cpu(), vc), step
        m, v = tc.decode(mc, ms, 3), tc.decode(vc, vs, 4)


def test_small_changes_add_up_over_steps(spo):
    # gradients that stay: r^2 goes to g^2 by a thousandth of the way per step, 60 times less than half a code.  A value that
    # moves evenly is at most one code from its place when it is rounded, and reaches the next one within one more on either
    # side: three codes of 1/16 at the most
    say("8-bit moments over 600 steps")
    n = 2048
    g = torch.Generator().manual_seed(11)
    grad = (torch.exp(1.5 * torch.randn(n, generator=g)) * 1e-3).cuda()
    p = torch.zeros(n, device="cuda")
    s = spo.adamw_state(p, 8)
    d = spo.make_adamw_desc([p], [grad], [s])
    for step in range(1, 601):
        spo.spo_adamw_update(d, 0.0, step)
        if step % 100 == 0:
            m, root = spo.spo_adamw_state_values(s, dtype=F32)
            want = math.sqrt(1 - B2 ** step) * grad
            assert float((root / want - 1).abs().max()) < 3 / 16, step
            assert float((root / want - 1).mean().abs()) < 1 / 32, step
    # the first moment goes all the way within some dozens of steps; codes are 1/8 apart, and those 2^14 below a block's largest wider
    top = grad.view(-1, 64).amax(dim=1, keepdim=True).expand(-1, 64).reshape(-1)
    assert float(((m - grad).abs() / torch.maximum(grad, top * 2.0 ** -14)).max()) < 1 / 4


def test_weights_in_bf16_move_by_less_than_half_a_place(spo):
    # each step takes a weight of 1 to 2 by lr = 2^-14 (its place is 2^-7): lost by rounding to nearest, kept by thresholds, within
    # a place (2^-7) and what the moments are off by at the start
    say("bf16 weights by thresholds")
    n = 4096
    p0 = (1 + torch.rand(n, generator=torch.Generator().manual_seed(1))).to("cuda", BF16)
    for rounding, moved in ((spo.SPO_ROUND_NEAREST, False), (spo.SPO_ROUND_THRESHOLD, True)):
        p, g = p0.clone(), torch.full((n,), 1e-3, device="cuda")
        d = spo.make_adamw_desc([p], [g], [spo.adamw_state(p)])
        for step in range(1, 513):
            spo.spo_adamw_update(d, 2.0 ** -14, step, rounding=rounding)
        went = (p0.float() - p.float()).cpu()
        if moved:
            assert float((went - 512 * 2.0 ** -14).abs().max()) <= 2.0 ** -7 + 1e-4
        else:
            assert not went.any()


def test_weights_by_thresholds_keep_what_is_not_finite(spo):
    say("bf16 weights that are not finite")
    p = torch.tensor([float("inf"), -float("inf"), float("nan"), 1.0, -0.0, 3e38], dtype=BF16, device="cuda")
    d = spo.make_adamw_desc([p], [torch.zeros(6, dtype=BF16, device="cuda")], [spo.adamw_state(p)])
    for step in range(1, 20):
        spo.spo_adamw_update(d, 1e-3, step, rounding=spo.SPO_ROUND_THRESHOLD)
    got = p.cpu().float()
    assert got[0] == float("inf") and got[1] == -float("inf") and torch.isnan(got[2]) and got[3] == 1 and got[4] == 0 and got[5] == torch.tensor(3e38, dtype=BF16).float()


# ------------------------------------------------------------------ sizes
def where(t):
    """Places that are not zero, looked for in pieces."""
    piece = 1 << 28
    return torch.cat([t[i:i + piece].nonzero()[:, 0] + i for i in range(0, t.numel(), piece)])


@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_2_to_the_31_elements(spo, bits):
    n = (1 << 31) + 5000
    say(f"adamw of {n} elements, {bits} bits")
    p = torch.zeros(n, dtype=BF16, device="cuda")
    g = torch.zeros(n, dtype=BF16, device="cuda")
    s = spo.adamw_state(p, bits)
    at = torch.tensor([0, 1, 8191, 8192, (1 << 31) - 1, 1 << 31, (1 << 31) + 4097, n - 1], device="cuda")
    g[at] = torch.arange(1, 9, device="cuda").to(BF16)
    d = spo.make_adamw_desc([p], [g], [s])
    norm = spo.spo_grad_norm(d)
    assert float(norm) == float(torch.tensor(204.0).sqrt())
    spo.spo_adamw_update(d, 0.5, 1)
    torch.cuda.synchronize()
    assert torch.equal(where(p), at)
    assert bool(((p[at].float() + 0.5).abs() < 0.5 * 2.0 ** -8 + 1e-6).all())
    if bits == 8:
        m, root = spo.spo_adamw_state_values(s)
        assert torch.equal(where(m), at) and torch.equal(where(root), at)
    else:
        assert torch.equal(where(s.m), at) and torch.equal(where(s.v), at)


def test_no_tensors(spo):
    say("adamw of nothing")
    d = spo.make_adamw_desc([], [], [])
    spo.spo_adamw_update(d, 1e-3, 1)
    e = torch.empty(0, device="cuda")
    d = spo.make_adamw_desc([e], [e], [spo.adamw_state(e, 8)])
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    spo.spo_adamw_update(d, 1e-3, count)
    assert float(spo.spo_grad_norm(d)) == 0.0 and int(count) == 1
