"""Normalisations and AdamW steps on the host (no GPU needed): refusals of the C entry points under the sanitizers, what would be
launched, workspaces that serve smaller problems, 8-bit codes, the binding's own checks, and what the compiler says of registers."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import train_cases as tc
from paper_2509_13232_amd import binding as spo
from paper_2509_13232_amd import build
from test_score_update_cpu import OnDevice, _dev, _refused, reached  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "san")
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(spo.LIB_PATH):
        build.build()
    return spo.lib()


@pytest.mark.timeout(900)
def test_argument_checks_run_clean_under_asan_and_ubsan(tmp_path):
    exe = build.build_sanitized_driver(os.path.join(SAN, "train_driver.cpp"), str(tmp_path / "train_san"))
    # the HIP runtime keeps allocations of its own until the process ends: leaks are not looked for here
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "normalisation and step host-side sanitizer run ok" in r.stdout


@pytest.mark.timeout(600)
def test_launches_stay_within_their_limits(L, tmp_path):
    here = os.path.dirname(spo.LIB_PATH)
    exe = str(tmp_path / "train_launch")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-w", "-rdynamic", "-I" + build.INCLUDE, "-I/opt/rocm/include",
                    os.path.join(SAN, "train_launch_driver.cpp"), "-o", exe, "-L" + here, "-l:" + os.path.basename(spo.LIB_PATH),
                    "-Wl,-rpath," + here, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    assert "launches within their limits" in r.stdout


# ---------------------------------------------------------------- workspaces
def _never_shrinks(sizes):
    return all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0


@pytest.mark.parametrize("kind", [spo.SPO_NORM_LAYER, spo.SPO_NORM_RMS])
def test_gradient_workspace_of_the_largest_batch_serves_smaller_ones(L, kind):
    def size(rows, cols):
        d = spo.NormDesc()
        d.struct_size, d.kind, d.rows, d.cols = C.sizeof(spo.NormDesc), kind, rows, cols
        return L.spo_norm_bwd_workspace_bytes(C.byref(d))
    rows = sorted({0, 1, 255, 256, 257, 1023, 1025, 100000} | {int(1.4 ** i) for i in range(1, 40)})
    cols = sorted({1, 63, 64, 65, 16384, 16385, 65536} | {int(1.2 ** i) for i in range(1, 60)})
    for n in cols:
        assert _never_shrinks([size(t, n) for t in rows]), n
    for t in rows:
        assert _never_shrinks([size(t, n) for n in cols]), t


# ---------------------------------------------------------------- 8-bit codes
@pytest.fixture(scope="module")
def state8(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("state8") / "state8")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-ffp-contract=off", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall", "-Wextra",
                    "-I" + build.CSRC, os.path.join(SAN, "state8_driver.cpp"), "-o", exe], check=True)

    def run(x, mantissa, step):
        """(codes, scales, values) of whole blocks."""
        text = "\n".join(f"{mantissa} {step} " + " ".join(f"{u & 0xffffffff:x}" for u in b) for b in x.view(-1, 64).view(torch.int32).tolist())
        r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-3000:]
        rows = [line.split() for line in r.stdout.splitlines()]
        codes = torch.tensor([[int(c) for c in row[1::2]] for row in rows], dtype=torch.uint8).view(-1)
        values = torch.tensor([[int(v, 16) - (1 << 32 if int(v, 16) >> 31 else 0) for v in row[2::2]] for row in rows], dtype=torch.int32).view(F32).view(-1)
        return codes, torch.tensor([int(row[0]) for row in rows], dtype=torch.uint8), values
    return run


@pytest.mark.parametrize("mantissa", [3, 4])
@pytest.mark.parametrize("scale", [1e-44, 1e-40, 1e-38, 1e-30, 1e-8, 1.0, 1e20, 1e36])
def test_codes_are_those_of_the_definition(state8, mantissa, scale):
    g = torch.Generator().manual_seed(7)
    x = (torch.randn(64 * 30, generator=g) * torch.exp(4 * torch.randn(64 * 30, generator=g)) * scale).clamp(-3e38, 3e38)
    x = x if mantissa == 3 else x.abs().double().clamp(min=2.0 ** -74.5).float()      # a root of a positive number is no smaller
    x[64:128] = 0
    x[130:190] = 0
    for step in (1, 2, 777, (1 << 32) + 5):
        codes, scales, values = state8(x, mantissa, step)
        want, want_scales = tc.encode(x, mantissa, step)
        ok = (want_scales != 255).repeat_interleave(64)
        assert torch.equal(scales, want_scales) and torch.equal(codes[ok], want[ok])
        held = tc.decode(want, want_scales, mantissa)
        assert torch.equal(values[ok], held[ok]) and torch.equal(held[ok], held[ok].to(BF16).float())   # bf16 holds them
        if mantissa == 4:
            assert bool(((values > 0) == (x > 0))[ok].all())
        # a value goes to one of its two neighbours, which are 2^-3 or 2^-4 of its binade apart, or of the lowest binade's, 2^14 below
        top = x.abs().view(-1, 64).amax(dim=1, keepdim=True).expand(-1, 64).reshape(-1)
        gap = torch.maximum(x.abs(), top * 2.0 ** -13).double() * 2.0 ** -mantissa + 2.0 ** -129
        assert bool(((values.double() - x.double()).abs() <= gap)[ok].all())


@pytest.mark.parametrize("mantissa", [3, 4])
@pytest.mark.parametrize("bad", [float("inf"), float("nan"), 3.4e38])
def test_a_block_that_is_not_finite_is_nan(state8, mantissa, bad):
    x = torch.linspace(0, 1, 192)
    x[70] = bad
    _, scales, values = state8(x, mantissa, 3)
    assert scales[1] == 255 and bool(torch.isnan(values[64:128]).all())
    assert bool(torch.isfinite(values[:64]).all()) and bool(torch.isfinite(values[128:]).all())


def test_thresholds_visit_all_places_evenly():
    # of any number n of steps the share below a bound is off by (log n + 2) / n at most: sequences by the golden ratio are that even
    for place in (0, 1, 63):
        t = torch.tensor([int(tc.turns(step, tc.ROOT)[place]) for step in range(1, 3001)], dtype=torch.float64) / 2 ** 32
        for n in (10, 100, 3000):
            for bound in (0.01, 0.25, 0.6):
                assert abs(float((t[:n] < bound).double().mean()) - bound) < (torch.tensor(float(n)).log().item() + 2) / n


# -------------------------------------------------------- the binding's checks
def test_normalisations_look_at_their_tensors(reached):  # noqa: F811
    x, w, b = _dev(5, 100), _dev(100), _dev(100)
    make = spo.make_norm_desc
    _refused(TypeError, "x", make, torch.zeros(5, 100))
    _refused(TypeError, "x", make, _dev(5, 100, dtype=torch.float16))
    _refused(TypeError, "x", make, OnDevice(torch.zeros(100, 5).t()))
    _refused(TypeError, "x", make, OnDevice(torch.zeros(1, 100).expand(5, 100)))
    _refused(TypeError, "x", make, OnDevice(torch.zeros(5, 200)[:, ::2]))
    _refused(ValueError, "x", make, _dev(100))
    _refused(ValueError, "x", make, _dev(2, 5, 100))
    _refused(ValueError, "weight", make, x, _dev(99))
    _refused(TypeError, "weight", make, x, _dev(100, dtype=torch.float16))
    _refused(TypeError, "weight", make, x, torch.zeros(100))
    _refused(TypeError, "bias", make, x, None, OnDevice(torch.zeros(200)[::2]))
    _refused(TypeError, "one type", make, x, w, _dev(100, dtype=BF16))
    d = make(x, w, b)
    mean, rstd, dy = _dev(5), _dev(5), _dev(5, 100)
    _refused(ValueError, "out", spo.spo_norm_fwd, d, out=_dev(5, 99))
    _refused(TypeError, "out", spo.spo_norm_fwd, d, out=_dev(5, 100, dtype=BF16))
    _refused(TypeError, "out", spo.spo_norm_fwd, d, out=OnDevice(torch.zeros(1, 100).expand(5, 100)))
    back = spo.spo_norm_bwd
    _refused(TypeError, "mean", back, d, None, rstd, dy)
    _refused(ValueError, "mean", back, d, _dev(4), rstd, dy)
    _refused(TypeError, "rstd", back, d, mean, _dev(5, dtype=BF16), dy)
    _refused(ValueError, "dy", back, d, mean, rstd, _dev(5, 101))
    _refused(ValueError, "dy", back, d, mean, rstd, _dev(100, 5))
    _refused(TypeError, "dy", back, d, mean, rstd, OnDevice(torch.zeros(1, 100).expand(5, 100)))
    _refused(TypeError, "dy", back, d, mean, rstd, OnDevice(torch.zeros(()).expand(5, 100)))
    _refused(ValueError, "dx", back, d, mean, rstd, dy, dx=_dev(100, 5))
    _refused(TypeError, "dx", back, d, mean, rstd, dy, dx=OnDevice(torch.zeros(5, 200)[:, :100]))
    _refused(ValueError, "d_weight", back, d, mean, rstd, dy, d_weight=_dev(101))
    _refused(TypeError, "one type", back, d, mean, rstd, dy, d_weight=_dev(100), d_bias=_dev(100, dtype=BF16))
    _refused(ValueError, "accumulate", back, d, mean, rstd, dy, accumulate=True)
    _refused(ValueError, "accumulate", back, d, mean, rstd, dy, d_weight=_dev(100), accumulate=True)
    _refused(ValueError, "workspace", back, d, mean, rstd, dy, workspace=_dev(8, dtype=torch.uint8))
    # what is written has a place of its own, or is the input itself
    wide = torch.zeros(6, 220)
    part = lambda t: OnDevice(t)   # noqa: E731
    dw = make(part(wide[:5, :100]), w, b)
    _refused(ValueError, "out: overlaps x", spo.spo_norm_fwd, dw, out=part(wide[1:, :100]))
    _refused(ValueError, "out: overlaps x", spo.spo_norm_fwd, dw, out=part(wide[:5, 99:199]))
    _refused(ValueError, "out: overlaps weight", spo.spo_norm_fwd, make(x, part(wide.view(-1)[:100])), out=part(wide[:5, :100]))
    _refused(ValueError, "dx: overlaps x", back, make(part(wide.view(-1)[:500].view(5, 100))), mean, rstd, dy, dx=part(wide.view(-1)[8:508].view(5, 100)))
    _refused(ValueError, "d_weight: overlaps dy", back, d, mean, rstd, part(wide[:5, :100]), d_weight=part(wide[0, :100]))
    _refused(ValueError, "d_bias: overlaps d_weight", back, d, mean, rstd, dy, d_weight=part(wide[0, :100]), d_bias=part(wide[0, 99:199]))
    assert not reached
    spo.spo_norm_fwd(dw, out=part(wide[:5, 100:200]))                               # other columns of the same rows
    spo.spo_norm_fwd(dw, out=dw[1][0])
    back(d, mean, rstd, dy, dx=dy)
    assert reached == ["spo_norm_fwd", "spo_norm_fwd", "spo_norm_bwd"]
    reached.clear()
    spo.spo_norm_fwd(d, out=OnDevice(torch.zeros(5, 120)[:, 3:103]))
    back(d, mean, rstd, dy, dx=_dev(5, 100), d_weight=_dev(100), d_bias=_dev(100), accumulate=True)
    back(make(x, kind=spo.SPO_NORM_RMS), None, rstd, dy)
    assert reached == ["spo_norm_fwd", "spo_norm_bwd", "spo_norm_bwd"]


def _state(n, bits=32):
    if bits == 32:
        return spo.AdamwState(_dev(n), _dev(n))
    u8 = lambda k: _dev(k, dtype=torch.uint8)   # noqa: E731
    return spo.AdamwState(u8(n), u8(n), u8(-(-n // 64)), u8(-(-n // 64)))


def test_steps_look_at_their_tensors(reached):  # noqa: F811
    make = spo.make_adamw_desc
    p, g = [_dev(10), _dev(3, 5)], [_dev(10), _dev(15)]
    s = [_state(10), _state(15)]
    _refused(ValueError, "grads", make, p, g[:1], s)
    _refused(ValueError, "states", make, p, g, s[:1])
    _refused(ValueError, "weight_decay", make, p, g, s, weight_decay=[0.1])
    _refused(ValueError, "copies", make, p, g, s, copies=[None])
    _refused(TypeError, r"params\[1\]", make, [p[0], _dev(15, dtype=torch.float16)], g, s)
    _refused(TypeError, r"params\[0\]", make, [torch.zeros(10), p[1]], g, s)
    _refused(TypeError, r"params\[1\]", make, [p[0], OnDevice(torch.zeros(5, 3).t())], g, s)
    _refused(ValueError, r"grads\[1\]", make, p, [g[0], _dev(14)], s)
    _refused(TypeError, r"grads\[0\]", make, p, [_dev(10, dtype=torch.float64), g[1]], s)
    _refused(ValueError, r"states\[1\].v", make, p, g, [s[0], s[1]._replace(v=_dev(16))])
    _refused(TypeError, r"states\[1\].m", make, p, g, [s[0], s[1]._replace(m=_dev(15, dtype=BF16))])
    _refused(TypeError, r"states\[1\].m", make, p, g, [s[0], _state(15, 8)])        # kinds are not mixed
    _refused(TypeError, r"states\[0\].m_scale", make, p, g, [s[0]._replace(m_scale=_dev(1, dtype=torch.uint8)), s[1]])
    eight = [_state(10, 8), _state(15, 8)]
    _refused(TypeError, r"states\[1\].v_scale", make, p, g, [eight[0], eight[1]._replace(v_scale=None)])
    _refused(ValueError, r"states\[1\].m_scale", make, p, g, [eight[0], eight[1]._replace(m_scale=_dev(2, dtype=torch.uint8))])
    _refused(TypeError, r"copies\[0\]", make, p, g, s, copies=[_dev(10), None])
    _refused(ValueError, r"copies\[1\]", make, p, g, s, copies=[None, _dev(14, dtype=BF16)])
    _refused(TypeError, r"copies\[0\]", make, [_dev(10, dtype=BF16), p[1]], g, s, copies=[_dev(10, dtype=BF16), None])
    # the same tensor twice, and arrays that share memory
    _refused(ValueError, "overlaps", make, [p[0], p[0]], [g[0], g[0]], [_state(10), _state(10)])
    _refused(ValueError, "overlaps", make, p, g, [s[0], s[1]._replace(v=s[1].m)])
    _refused(ValueError, "overlaps", make, [p[0]], [p[0]], [s[0]])
    flat = torch.zeros(30)
    _refused(ValueError, "overlaps", make, [OnDevice(flat[:10]), OnDevice(flat[9:24])], g, s)
    make([OnDevice(flat[:10]), OnDevice(flat[10:25])], g, s)
    make([p[0], _dev(10)], [g[0], g[0]], [_state(10), _state(10)])                  # a gradient may serve two tensors
    d = make(p, g, s, weight_decay=[0.1, 0.0], copies=[_dev(10, dtype=BF16), None])
    assert d[0].state_bits == 32 and d[0].count == 2 and d[0].tensors[0].weight_decay == 0.1 and d[0].tensors[1].copy is None
    assert make(p, g, eight)[0].state_bits == 8
    _refused(TypeError, "lr", spo.spo_adamw_update, d, torch.zeros(1), 1)
    _refused(TypeError, "step", spo.spo_adamw_update, d, 0.1, torch.zeros(1))
    _refused(ValueError, "grad_norm", spo.spo_adamw_update, d, 0.1, 1, grad_norm=_dev(2))
    _refused(TypeError, "grad_norm", spo.spo_adamw_update, d, 0.1, 1, grad_norm=torch.zeros(1))
    _refused(ValueError, "workspace", spo.spo_grad_norm, d, workspace=_dev(8, dtype=torch.uint8))
    _refused(TypeError, "8 bits", spo.spo_adamw_state_values, s[0]._replace(m=_dev(10, dtype=torch.uint8), v=_dev(10, dtype=torch.uint8)))
    _refused(ValueError, "v_scale", spo.spo_adamw_state_values, eight[0]._replace(v_scale=_dev(2, dtype=torch.uint8)))
    _refused(ValueError, "bits", spo.adamw_state, torch.zeros(3), 16)
    assert not reached
    spo.spo_grad_norm(d)
    spo.spo_adamw_update(d, 0.1, 1, grad_norm=_dev(1), max_norm=1.0)
    spo.spo_adamw_state_values(eight[0])
    assert reached == ["spo_grad_norm", "spo_adamw_update", "spo_adamw_state_values"]


def test_a_tensor_of_another_device_is_refused(reached, monkeypatch):  # noqa: F811
    class Elsewhere(OnDevice):
        device = torch.device("cuda", 1)

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x, far = _dev(5, 100), Elsewhere(torch.zeros(5, 100))
    _refused(ValueError, "current device", spo.make_norm_desc, far)
    _refused(ValueError, "current device", spo.make_norm_desc, x, Elsewhere(torch.zeros(100)))
    d = spo.make_norm_desc(x)
    _refused(ValueError, "current device", spo.spo_norm_bwd, d, _dev(5), _dev(5), far)
    _refused(ValueError, "current device", spo.spo_norm_bwd, d, Elsewhere(torch.zeros(5)), _dev(5), _dev(5, 100))
    step = spo.make_adamw_desc([_dev(5)], [_dev(5)], [_state(5)])
    _refused(ValueError, "grad_norm: is on", spo.spo_adamw_update, step, 0.1, 1, grad_norm=Elsewhere(torch.zeros(1)))
    _refused(ValueError, "current device", spo.make_adamw_desc, [Elsewhere(torch.zeros(5))], [_dev(5)], [_state(5)])
    _refused(ValueError, "current device", spo.make_adamw_desc, [_dev(5)], [Elsewhere(torch.zeros(5))], [_state(5)])
    assert not reached


def test_state_of_a_tensor():
    p = torch.zeros(3, 50, dtype=BF16)
    a, b = spo.adamw_state(p), spo.adamw_state(p, 8)
    assert a.m.shape == a.v.shape == p.shape and a.m.dtype == F32 and a.m_scale is None and not a.m.any()
    assert b.m.dtype == torch.uint8 and b.v.shape == p.shape and b.m_scale.shape == b.v_scale.shape == (3,) and not b.v.any()


# ------------------------------------------------------------------- registers
@pytest.mark.timeout(900)
@pytest.mark.parametrize("src", ["adamw.hip", "norm_fwd.hip", "norm_bwd.hip"])
def test_kernels_keep_their_values_in_registers(tmp_path, src):
    r = subprocess.run([build._hipcc(), *build.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
                        os.path.join(build.CSRC, src), "-o", str(tmp_path / "k.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    scratch, name = {}, None
    for line in r.stderr.splitlines():
        if m := re.search(r"remark: .*Function Name: (\S+)", line):
            name = m[1]
        elif m := re.search(r"remark: .*ScratchSize \[bytes/lane\]: (\d+)", line):
            scratch[name] = int(m[1])
    assert len(scratch) > 4
    # rows of more than 8192 elements, four and more eights per thread, keep some of what they hold elsewhere; nothing else does
    long_rows = r"norm_fwd_kernelI.*Li0ELi(12|16)ELi[48]E|norm_fwd_kernelI.*Li0ELi8ELi4E|norm_bwd_kernelI.*Li0ELi0ELi2E"
    assert not any(v for k, v in scratch.items() if not re.search(long_rows, k)), {k: v for k, v in scratch.items() if v}
