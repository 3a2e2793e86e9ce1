"""Normalisations and AdamW steps on the host, at their edges (no GPU needed)."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2509_13232_amd import binding as spo
from paper_2509_13232_amd import build
from test_binding_cpu import _desc
from test_score_update_cpu import OnDevice, _dev, _refused, reached  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---------------------------------------------------------------- 8-bit codes
@pytest.fixture(scope="module")
def tops(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("state8") / "top")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wall", "-Wextra", "-I" + build.CSRC,
                    os.path.join(ROOT, "tests", "san", "state8_top_driver.cpp"), "-o", exe], check=True)

    def run(blocks, mantissa):
        """[(scale, whether all is NaN)] of blocks of 64 numbers, as bits."""
        text = "\n".join(f"{mantissa} " + " ".join(f"{u:x}" for u in b) for b in blocks)
        r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-3000:]
        return [tuple(int(v) for v in line.split()) for line in r.stdout.splitlines()]
    return run


@pytest.mark.parametrize("mantissa", [3, 4])
def test_every_nan_and_infinity_spoils_its_block(tops, mantissa):
    # NaNs of any sign and payload: memory filled with ones is one of them
    bad = [0x7f800000, 0x7f800001, 0x7fc00000, 0x7fffffff, 0xff800000, 0xff800001, 0xffc00000, 0xffefffff, 0xfff00000, 0xfff00001, 0xfff80000, 0xfff80001, 0xffff0000,
           0xffffffff]
    if mantissa == 4:
        bad.remove(0xff800000)       # (no root is -infinity; -NaN is what a root of a NaN may be)
    ones = [0x3f800000 + i for i in range(64)]
    blocks = [ones[:i % 64] + [u] + ones[i % 64 + 1:] for i, u in enumerate(bad)]
    assert tops(blocks, mantissa) == [(255, 1)] * len(bad)
    assert tops([[u] * 64 for u in bad], mantissa) == [(255, 1)] * len(bad)
    # the largest number that a block holds, and the next one
    largest = 0x7f800000 - (1 << (23 - mantissa))
    assert tops([ones[1:] + [largest]], mantissa) == [(254, 0)] and tops([ones[1:] + [largest + 1]], mantissa) == [(255, 1)]
    assert tops([ones, [0] * 64, [1] * 64], mantissa) == [(127, 0), (15, 0), (15, 0)]


# -------------------------------------------------------- the binding's checks
class Elsewhere(OnDevice):
    device = torch.device("cuda", 1)


def _state(n, bits=32):
    if bits == 32:
        return spo.AdamwState(_dev(n), _dev(n))
    u8 = lambda k: _dev(k, dtype=torch.uint8)   # noqa: E731
    return spo.AdamwState(u8(n), u8(n), u8(-(-n // 64)), u8(-(-n // 64)))


def test_a_workspace_is_looked_at(reached):  # noqa: F811
    # kernels write to it: in host memory, with holes, or on another device it is refused
    U8 = torch.uint8
    x, w, f, i, r = _dev(5, 100), _dev(100), _dev(16), _dev(4, dtype=torch.int32), _dev(4)
    norm, step = spo.make_norm_desc(x, w), spo.make_adamw_desc([_dev(5)], [_dev(5)], [_state(5)])
    loss, logp, lse = _desc(spo.SPO_W_VH)
    calls = [
        lambda ws: spo.spo_norm_bwd(norm, _dev(5), _dev(5), _dev(5, 100), workspace=ws),
        lambda ws: spo.spo_norm_bwd(norm, _dev(5), _dev(5), _dev(5, 100), want_dx=False, workspace=ws),
        lambda ws: spo.spo_grad_norm(step, workspace=ws),
        lambda ws: spo.spo_pg_loss_fwd(loss, workspace=ws),
        lambda ws: spo.spo_pg_loss_bwd(loss, logp, lse, d_W=_dev(100, 64), workspace=ws),
        lambda ws: spo.spo_pg_loss_fwd_bwd(loss, d_W=_dev(100, 64), workspace=ws),
        lambda ws: spo.spo_sample_prompts(f, f, 4, workspace=ws),
        lambda ws: spo.spo_advantages(f, f, i, r, workspace=ws),
        lambda ws: spo.spo_tracker_update(f, f, i, r, r, 0.25, 0.875, 0.96, ids_unique=False, workspace=ws),
    ]

    def at256(t, of=OnDevice):
        if of is not None:
            t = of(t)
            t.data_ptr = lambda: 256
        return t

    host = torch.zeros(1 << 20, dtype=U8)
    host = host[-host.data_ptr() % 256:]
    for k, call in enumerate(calls):
        for bad in (host, at256(torch.zeros(1 << 21, dtype=U8)[::2]), at256(torch.zeros(1, dtype=U8).expand(1 << 20)), at256(torch.zeros(1 << 20, dtype=U8), Elsewhere)):
            with pytest.raises(ValueError, match="workspace"):
                call(bad)
        assert not reached, k
        call(at256(torch.zeros(1 << 20, dtype=U8)))
        assert len(reached) == 1, k
        reached.clear()


def test_states_and_copies_of_another_device_are_refused(reached, monkeypatch):  # noqa: F811
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    U8 = torch.uint8
    make = lambda s, **kw: spo.make_adamw_desc([_dev(100)], [_dev(100)], [s], **kw)   # noqa: E731
    for bits in (32, 8):
        whole = _state(100, bits)
        make(whole)
        for name, t in zip(whole._fields, whole):
            if t is not None:
                _refused(ValueError, rf"states\[0\].{name}: is on cuda:1", make, whole._replace(**{name: Elsewhere(torch.zeros(t.shape, dtype=t.dtype))}))
    _refused(ValueError, r"copies\[0\]: is on cuda:1", make, _state(100), copies=[Elsewhere(torch.zeros(100, dtype=torch.bfloat16))])
    for name in spo.AdamwState._fields:
        whole = _state(100, 8)
        _refused(ValueError, f"{name}: is on cuda:1", spo.spo_adamw_state_values, whole._replace(**{name: Elsewhere(torch.zeros(getattr(whole, name).shape, dtype=U8))}))
    assert not reached


def test_a_norm_without_a_limit_clips_nothing(reached, monkeypatch):  # noqa: F811
    # a norm alone is for leaving out steps that are not finite; a limit of zero has to be asked for
    step, given = spo.make_adamw_desc([_dev(5)], [_dev(5)], [_state(5)]), []

    class Steps:
        def spo_adamw_update(self, *a):
            given.append(a[9])
            return 0

    monkeypatch.setattr(spo, "lib", Steps)
    plain = []
    for calls in (lambda *a: None, lambda *a: plain.append(a[8]) or True):
        monkeypatch.setattr(spo, "_calls", type("Calls", (), {"adamw_update": staticmethod(calls)}))
        for kw in ({}, {"max_norm": None}, {"max_norm": 0.0}, {"max_norm": 2.5}):
            spo.spo_adamw_update(step, 0.1, 1, grad_norm=_dev(1), **kw)
    infinite = float("inf")
    assert given == plain == [infinite, infinite, 0.0, 2.5]


def test_workspace_queries_of_what_is_refused_say_nothing():
    if not os.path.exists(spo.LIB_PATH):
        build.build()
    L = C.CDLL(spo.LIB_PATH)
    L.spo_grad_norm_workspace_bytes.restype = C.c_size_t
    d = spo.AdamwDesc()
    d.struct_size, d.state_bits = C.sizeof(spo.AdamwDesc), 32
    sizes = []
    for count in (0, 1, 160, 161, 1 << 24):
        d.count = count
        sizes.append(L.spo_grad_norm_workspace_bytes(C.byref(d)))
    assert sizes == sorted(sizes) and sizes[0] > 0
    for count in ((1 << 24) + 1, 1 << 45, 1 << 62, (1 << 63) - 1, -1):
        d.count = count
        assert L.spo_grad_norm_workspace_bytes(C.byref(d)) == 0, count


# ------------------------------------------------------------------- registers
# What is kept outside of registers, in bytes per lane at most: rows beyond 32768 elements in the forward, and the sums of two types in LDS
OUTSIDE = {"norm_fwd.hip": [(r"norm_fwd_kernelI..Li0ELi16ELi8E", 256)], "norm_bwd.hip": [(r"norm_bwd_kernelI(ft|tf)Li0ELi0ELi2ELb1E", 32)]}


@pytest.mark.timeout(900)
@pytest.mark.parametrize("src", list(OUTSIDE))
def test_little_is_kept_outside_of_registers(tmp_path, src):
    r = subprocess.run([build._hipcc(), *build.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
                        os.path.join(build.CSRC, src), "-o", str(tmp_path / "k.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    scratch, scalars, name = {}, {}, None
    for line in r.stderr.splitlines():
        if m := re.search(r"remark: .*Function Name: (\S+)", line):
            name = m[1]
        elif m := re.search(r"remark: .*ScratchSize \[bytes/lane\]: (\d+)", line):
            scratch[name] = int(m[1])
        elif m := re.search(r"remark: .*TotalSGPRs: (\d+)", line):
            scalars[name] = int(m[1])
    assert len(scratch) > 100
    too_much = {k: v for k, v in scratch.items() if v > max([most for kernel, most in OUTSIDE[src] if re.search(kernel, k)], default=0)}
    assert not too_much
    if src == "norm_fwd.hip":     # (the kernels' own bound)
        assert max(scalars.values()) <= 80
