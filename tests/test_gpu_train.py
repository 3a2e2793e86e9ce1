"""Normalisation, head, AdamW step and norm of gradients together, as a training step uses them.

Tolerances.  Hidden states, head and logit gradients are rounded to bf16 (2^-9 each) before sums over many terms: 1e-2 of a gradient.
A step's tensors: those of their own tests, from the gradients that the library itself gave."""
import sys

import pytest
import torch

import score_cases as sc
import test_gpu_plain_calls as pc
import train_cases as tc
from paper_2509_13232_amd import iteration
from pg_cases import say
from test_gpu_iteration import _through_bf16

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
spo = iteration.spo


def _batch(policy):
    batch = iteration.respond(policy, torch.arange(policy.prompts, dtype=torch.int32, device="cuda"))
    # ratios of about 1, 0.7 and 1.5: inside and outside of the clip
    batch["old_logp"] += torch.tensor([0.0, 0.357, -0.405], device="cuda").repeat(14)[:batch["old_logp"].numel()]
    return batch, torch.randn(policy.prompts, generator=torch.Generator().manual_seed(5)).cuda()


def _fp64_gradients(policy, batch, adv, bonus):
    x = batch["x"].double().cpu()
    leaf = lambda t: t.double().cpu().requires_grad_()   # noqa: E731
    P, W = leaf(policy.P.to(BF16)), leaf(policy.W)
    w, b = (leaf(t) for t in policy.norm)
    pre = _through_bf16(x @ P)
    h = torch.nn.functional.layer_norm(pre, pre.shape[1:], w, b, 1e-6)
    logq = torch.log_softmax(_through_bf16(h) @ W.t(), dim=1)
    logp = logq.gather(1, batch["target"].long().cpu()[:, None])[:, 0]
    ratio = torch.exp(logp - batch["old_logp"].double().cpu())
    A = adv.double().cpu().repeat_interleave(policy.tokens)
    loss = -torch.minimum(ratio * A, ratio.clamp(0.8, 1.28) * A).mean()
    entropy = -(torch.exp(logq) * logq).sum(dim=1).mean()
    (loss - bonus * entropy).backward()
    return [t.grad for t in ((P, W, w, b) if policy.train_head else (P, w, b))]


@pytest.mark.parametrize("step", ["muon", "adamw"])
@pytest.mark.parametrize("bonus", [0.0, 0.05])
def test_gradients_through_the_normalisation(step, bonus):
    say(f"training step's gradients, {step}, bonus {bonus}")
    policy = iteration.Policy(prompts=8, tokens=5, hidden=128, vocab=1000, top_k=8, seed=3, normalise=True, step=step)
    policy.norm[0].copy_(1 + 0.3 * torch.randn(128, generator=torch.Generator().manual_seed(1)))
    policy.norm[1].copy_(0.2 * torch.randn(128, generator=torch.Generator().manual_seed(2)))
    batch, adv = _batch(policy)
    got, want = iteration.gradients(policy, batch, adv, bonus), _fp64_gradients(policy, batch, adv, bonus)
    assert len(got) == len(want) == (4 if step == "adamw" else 3)
    for g, w in zip(got, want):
        assert g.shape == w.shape and g.dtype == F32 and sc.rel(g, w) < 1e-2


@pytest.mark.parametrize("bits", [32, 8])
def test_a_whole_step_is_its_parts(bits):
    say(f"training step, states in {bits} bits")
    policy = iteration.Policy(prompts=8, tokens=5, hidden=128, vocab=1000, top_k=8, seed=3, normalise=True, step="adamw", state_bits=bits)
    batch, adv = _batch(policy)
    for step in (1, 2):
        grads = iteration.gradients(policy, batch, adv, 0.01)
        host = lambda ts: [t.clone().cpu() for t in ts]   # noqa: E731
        before, g = host(t.view(-1) for t in policy.adamw), host(t.reshape(-1) for t in grads)
        if bits == 32:
            m, v = host(s.m.view(-1) for s in policy.states), host(s.v.view(-1) for s in policy.states)
        else:
            m = [tc.decode(s.m.view(-1).cpu(), s.m_scale.cpu(), 3) for s in policy.states]
            v = [tc.decode(s.v.view(-1).cpu(), s.v_scale.cpu(), 4) for s in policy.states]
        iteration.update(policy, grads, adamw_lr=1e-3, max_norm=0.05)
        torch.cuda.synchronize()
        assert int(policy.steps) == step
        norm = float(torch.cat([t.double() for t in g]).norm())
        assert norm > 0.05                                                  # the limit is felt
        factor = float(torch.tensor(0.05) / torch.tensor(norm, dtype=F32))  # as fp32 divides
        for i, t in enumerate(policy.adamw):
            clipped = (g[i] * torch.tensor(factor, dtype=F32)).double()
            m64 = 0.9 * m[i].double() + 0.1 * clipped
            old = v[i].double() if bits == 32 else v[i].double() ** 2
            root = (0.999 * old + 0.001 * clipped ** 2).sqrt()
            change = 1e-3 / (1 - 0.9 ** step) * m64 / (root / (1 - 0.999 ** step) ** 0.5 + 1e-8)
            size = 1e-3 / (1 - 0.9 ** step) * (0.9 * m[i].double().abs() + 0.1 * clipped.abs()) / (root / (1 - 0.999 ** step) ** 0.5 + 1e-8)
            p = before[i].double()
            want = p - change - 1e-3 * policy.decay[i] * p
            # the step's own 1e-6, the betas' four and the limit's two roundings to fp32 (3.6e-7 in all), and the weight's two
            tc.off(t.view(-1), want, 2e-6 * size + 2.0 ** -23 * p.abs() + 1e-12, "weights")
        assert torch.equal(policy.W, policy.master.to(BF16))


@pytest.mark.parametrize("bits", [32, 8])
def test_training_steps_replay_from_a_graph(bits):
    say(f"training steps from a graph, states in {bits} bits")

    def fresh():
        policy = iteration.Policy(prompts=8, tokens=5, hidden=128, vocab=1000, top_k=8, seed=3, normalise=True, step="adamw", state_bits=bits)
        return policy, *_batch(policy)

    def step(policy, batch, adv):
        x = batch["x"]
        norm = spo.make_norm_desc(x, *policy.norm)
        h, mean, rstd = spo.spo_norm_fwd(norm)
        loss = spo.make_desc(h, policy.W, batch["target"], batch["old_logp"], None, adv, batch["cu_seqlens"], 0.2, 0.28)
        _, logp, lse, _ = spo.spo_pg_loss_fwd(loss)
        d_h, d_W = spo.spo_pg_loss_bwd(loss, logp, lse, d_hidden_dtype=F32)
        _, d_w, d_b = spo.spo_norm_bwd(norm, mean, rstd, d_h, want_dx=False)
        desc = spo.make_adamw_desc(policy.adamw[1:], [d_W, d_w, d_b], policy.states[1:], weight_decay=policy.decay[1:], copies=policy.copies[1:])
        spo.spo_adamw_update(desc, 1e-3, policy.steps, grad_norm=spo.spo_grad_norm(desc), max_norm=0.05)

    def held(policy):
        return [t.clone() for t in (policy.W, policy.steps, *policy.adamw, *(t for s in policy.states for t in s if t is not None))]

    eager, captured = fresh(), fresh()
    want = []
    for _ in range(4):
        step(*eager)
        want.append(held(eager[0]))
    step(*captured)     # (what a first call makes, it makes outside of the graph)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*captured)
    for k in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        (torch.randn(1 << 20, device="cuda") * 1.0001).sin_()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held(captured[0]), want[k])), k


@pytest.mark.parametrize("options", [["--normalise"], ["--step", "adamw"], ["--normalise", "--step", "adamw", "--state-bits", "8"]])
def test_command(monkeypatch, capsys, options):
    say(f"iterations {options}")
    monkeypatch.setattr(sys, "argv", ["iteration", "--iterations", "2", *options])
    iteration.main()
    lines = capsys.readouterr().out.strip().splitlines()
    lines = [line for line in lines if line.startswith("iteration ")]
    assert len(lines) == 2 and all("reward" in line and "nan" not in line for line in lines[-2:]), lines


# ------------------------------------------------------------------ plain calls against the general way
@pytest.mark.parametrize("kind", [spo.SPO_NORM_LAYER, spo.SPO_NORM_RMS])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_plain_calls_of_normalisations(monkeypatch, kind, dtype):
    say(f"plain calls of normalisations, {kind} {dtype}")
    g = torch.Generator().manual_seed(1)
    x, dy = (torch.randn((50, 300), generator=g).to("cuda", dtype) for _ in range(2))
    w, b = (torch.randn(300, generator=g).cuda() for _ in range(2))
    for weight, bias in ((w, b), (w, None), (None, None)):
        d = spo.make_norm_desc(x, weight, bias, kind=kind)
        def call():
            y, mean, rstd = spo.spo_norm_fwd(d)
            return y, mean, rstd, spo.spo_norm_bwd(d, mean, rstd, dy)
        pc.same(*pc.both_ways(spo, monkeypatch, call))


@pytest.mark.parametrize("bits", [32, 8])
def test_plain_calls_of_steps(monkeypatch, bits):
    say(f"plain calls of steps, {bits}")
    g = torch.Generator().manual_seed(1)
    sizes = [(3, 100), (7,), (5000,)]
    p0 = [torch.randn(s, generator=g).cuda() for s in sizes]
    grads = [torch.randn(s, generator=g).to("cuda", BF16) for s in sizes]
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    def call():
        p, states = [t.clone() for t in p0], [spo.adamw_state(t, bits) for t in p0]
        copies = [torch.zeros(t.shape, dtype=BF16, device="cuda") for t in p0[:2]] + [None]
        desc = spo.make_adamw_desc(p, grads, states, weight_decay=[0.1, 0.0, 0.2], copies=copies)
        norm = spo.spo_grad_norm(desc, workspace=ws)
        spo.spo_adamw_update(desc, 1e-3, 1, grad_norm=norm, max_norm=0.5)
        spo.spo_adamw_update(desc, 2e-3, 7, 0.8, 0.99, 1e-6)
        held = [t for s in states for t in s if t is not None]
        return norm, p, copies, held, list(spo.spo_adamw_state_values(states[0])) if bits == 8 else None
    pc.same(*pc.both_ways(spo, monkeypatch, call))


def test_errors_are_those_of_the_general_way(monkeypatch):
    say("plain calls of normalisations and steps: errors")
    x, w = torch.zeros((5, 100), device="cuda"), torch.zeros(100, device="cuda")
    d, stat = spo.make_norm_desc(x, w), torch.zeros(5, device="cuda")
    p, g, s = torch.zeros(10, device="cuda"), torch.zeros(10, device="cuda"), spo.adamw_state(torch.zeros(10, device="cuda"))
    step, e = spo.make_adamw_desc([p], [g], [s]), spo.adamw_state(p, 8)
    u = spo.spo_adamw_update
    calls = [
        lambda: spo.spo_norm_fwd(spo.make_norm_desc(x, w, eps=-1.0)),
        lambda: spo.spo_norm_fwd(d, out=x[:4]),
        lambda: spo.spo_norm_bwd(d, None, stat, x),
        lambda: spo.spo_norm_bwd(d, stat, stat[:4], x),
        lambda: spo.spo_norm_bwd(d, stat, stat, x.half()),
        lambda: spo.spo_norm_bwd(d, stat, stat, x[:, :99]),
        lambda: spo.spo_norm_bwd(d, stat, stat, x.cpu()),
        lambda: spo.make_adamw_desc([p], [g[:9]], [s]),
        lambda: spo.make_adamw_desc([p], [p], [s]),
        lambda: spo.make_adamw_desc([p, p], [g, g], [s, spo.adamw_state(p)]),
        lambda: spo.make_adamw_desc([p.half()], [g], [s]),
        lambda: spo.make_adamw_desc([p], [g], [s], weight_decay=[]),
        lambda: spo.make_adamw_desc([p], [g], [e._replace(m_scale=None)]),
        lambda: spo.make_adamw_desc([p], [g], [s], copies=[g]),
        lambda: spo.spo_adamw_update(spo.make_adamw_desc([p], [g], [s], weight_decay=-1.0), 0.1, 1),
        lambda: u(step, -0.1, 1), lambda: u(step, float("nan"), 1), lambda: u(step, 0.1, 0), lambda: u(step, 0.1, 1, beta1=1.0),
        lambda: u(step, 0.1, 1, beta2=-0.5), lambda: u(step, 0.1, 1, eps=-1.0), lambda: u(step, 10 ** 400, 1), lambda: u(step, 0.1, 1 << 70),
        lambda: u(step, 0.1, 1.5), lambda: u(step, "a", 1), lambda: u(step, stat, 1), lambda: u(step, 0.1, stat), lambda: u(step, 0.1, 1, rounding=2),
        lambda: u(step, 0.1, 1, grad_norm=stat), lambda: u(step, 0.1, 1, grad_norm=stat[:1], max_norm=-1.0), lambda: u(step, 0.1, 1, grad_norm=1.0),
        lambda: spo.spo_adamw_state_values(s), lambda: spo.spo_adamw_state_values(e._replace(v=e.v[:9])),
        lambda: spo.spo_adamw_state_values(e, torch.float16),
    ]
    for i, call in enumerate(calls):
        seen = []
        for way in (spo._plain_calls(), pc.Nothing()):
            with monkeypatch.context() as m:
                m.setattr(spo, "_calls", way)
                try:
                    seen.append(call())
                except Exception as err:
                    seen.append((type(err), str(err), getattr(err, "status", None)))
        assert isinstance(seen[0], tuple) and seen[0] == seen[1], (i, seen)


def test_calls_on_two_streams_at_once():
    say("normalisations and steps on two streams at once")
    g = torch.Generator().manual_seed(6)
    make = lambda *s: torch.randn(s, generator=g).cuda()   # noqa: E731

    class Lane:
        def __init__(self, N):
            self.x, self.dy, self.w, self.b = make(3000, N), make(3000, N), make(N), make(N)
            self.p, self.grads = [make(N), make(70000)], [make(N), make(70000)]
            self.norm = spo.make_norm_desc(self.x, self.w, self.b)
            self.ws = torch.empty(spo.spo_norm_bwd_workspace_bytes(self.norm), dtype=torch.uint8, device="cuda")
            self.states, self.first = [spo.adamw_state(t, 8) for t in self.p], [t.clone() for t in self.p]
            self.step = spo.make_adamw_desc(self.p, self.grads, self.states)
            self.count, self.room = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.empty(1 << 18, dtype=torch.uint8, device="cuda")

        def run(self):
            y, mean, rstd = spo.spo_norm_fwd(self.norm)
            out = spo.spo_norm_bwd(self.norm, mean, rstd, self.dy, workspace=self.ws)
            size = spo.spo_grad_norm(self.step, workspace=self.room)
            spo.spo_adamw_update(self.step, 1e-3, self.count, grad_norm=size, max_norm=1.0)
            return [y, *out, size]

        def again(self):
            for t, u in zip(self.p, self.first):
                t.copy_(u)
            for s in self.states:
                for t in s:
                    t.zero_()
            self.count.zero_()

        def held(self):
            return [t.clone() for t in (*self.p, *(t for s in self.states for t in s), self.count)]

    lanes, streams = [Lane(1000), Lane(5000)], [torch.cuda.Stream(), torch.cuda.Stream()]
    want = []
    for lane in lanes:
        for _ in range(6):
            out = lane.run()
        want.append((out, lane.held()))
        lane.again()
    torch.cuda.synchronize()
    got = [None, None]
    for _ in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = lanes[i].run()
    torch.cuda.synchronize()
    for i, lane in enumerate(lanes):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i][0])) and all(torch.equal(a, b) for a, b in zip(lane.held(), want[i][1])), i
