"""Token scores and orthogonalised updates on the host (no GPU needed): refusals of the C entry points under the sanitizers,
workspaces that serve smaller problems, the binding's own checks, and what the compiler says about the kernels' registers."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2509_13232_amd import binding as spo
from paper_2509_13232_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(spo.LIB_PATH):
        build.build()
    return spo.lib()


@pytest.mark.timeout(600)
def test_argument_checks_run_clean_under_asan_and_ubsan(tmp_path):
    exe = build.build_sanitized_driver(os.path.join(ROOT, "tests", "san", "score_update_driver.cpp"), str(tmp_path / "score_update_san"))
    # the HIP runtime keeps allocations of its own until the process ends: leaks are not looked for here
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert "score and update host-side sanitizer run ok" in r.stdout


# ---------------------------------------------------------------- workspaces
def _scores(T, V, H=0, dtype=1, top_k=0, w_layout=0, mask=False):
    """A descriptor for the workspace queries, which read sizes only (H = 0: logits-in)."""
    d = spo.LogprobDesc()
    d.struct_size = C.sizeof(spo.LogprobDesc)
    d.dtype, d.w_layout, d.T, d.H, d.V, d.top_k = dtype, w_layout, T, H, V, top_k
    for f in ("target",) + (("hidden", "W") if H else ("logits",)):
        setattr(d, f, 256)
    d.mask = 256 if mask else None
    return C.byref(d)


def _never_shrinks(sizes):
    return all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0


TOKENS = sorted({0, 1, 2, 16, 17, 255, 257} | {int(1.2 ** i) for i in range(1, 60)} | set(range(256, 20000, 256)))
VOCABS = sorted({1, 4096, 4097, 8192, 8193, 151936} | {int(1.3 ** i) for i in range(1, 47)})


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("H,w_layout,top_k", [(0, 0, 0), (0, 0, 1), (64, 0, 0), (64, 1, 0), (4096, 0, 0)])
def test_forward_workspace_of_the_largest_batch_serves_smaller_ones(L, dtype, H, w_layout, top_k):
    size = lambda T, V: L.spo_logprob_fwd_workspace_bytes(_scores(T, V, H, dtype, top_k, w_layout))
    for V in VOCABS:
        assert _never_shrinks([size(T, V) for T in TOKENS]), V
    for T in TOKENS[::5]:
        assert _never_shrinks([size(T, V) for V in VOCABS]), T


@pytest.mark.parametrize("mask", [False, True])
def test_gradient_workspace_of_long_chunks_serves_short_ones(L, mask):
    size = lambda T, V, H, chunk: L.spo_logprob_bwd_workspace_bytes(_scores(T, V, H, 1, 0, 0, mask), chunk)
    for T in (1, 256, 257, 3000, 9000):
        for V, H in ((300, 64), (3000, 1024), (30000, 4096)):
            assert _never_shrinks([size(T, V, H, c) for c in [*range(256, 10000, 256), 0]]), (T, V, H)
    for V, H in ((300, 64), (151936, 4096)):
        for chunk in (0, 256, 4096):
            assert _never_shrinks([size(T, V, H, chunk) for T in TOKENS]), (V, H, chunk)


@pytest.mark.parametrize("products", [spo.SPO_PRODUCTS_FP16, spo.SPO_PRODUCTS_SPLIT])
def test_update_workspace_of_the_largest_matrices_serves_smaller_ones(L, products):
    size = lambda batch, rows, cols: spo.spo_orthogonalize_workspace_bytes(batch, rows, cols, products)
    sides = sorted({1, 63, 64, 65, 127, 129, 65536} | {int(1.25 ** i) for i in range(1, 49)})
    for other in (1, 64, 200, 1024, 5000, 65536):
        assert _never_shrinks([size(3, n, other) for n in sides]), other
        assert _never_shrinks([size(3, other, n) for n in sides]), other
        assert _never_shrinks([size(n, other, 300) for n in range(1, 200)]), other
        assert [size(2, n, other) for n in sides] == [size(2, other, n) for n in sides]


# -------------------------------------------------------- the binding's checks
class OnDevice:
    """A tensor that says it is on the GPU."""

    is_cuda = True

    def __init__(self, t):
        self._t = t

    def __getattr__(self, name):
        return getattr(self._t, name)


class Recorder:
    def __init__(self, called):
        self._called = called

    def __getattr__(self, name):
        def f(*a):
            if name.endswith("_bytes"):
                return 256
            self._called.append(name)
            return 0
        return f


@pytest.fixture
def reached(monkeypatch):
    """Names of the library's functions that were called."""
    called = []

    class NoPlain:
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(spo, "lib", lambda: Recorder(called))
    monkeypatch.setattr(spo, "_calls", NoPlain())
    monkeypatch.setattr(spo, "_stream", lambda: 0)
    return called


def _dev(*shape, dtype=torch.float32):
    return OnDevice(torch.zeros(shape, dtype=dtype))


def _refused(error, match, f, *a, **kw):
    with pytest.raises(error, match=match):
        f(*a, **kw)


def test_scores_look_at_their_tensors(reached):
    z, target, X, W = _dev(5, 100), _dev(5, dtype=torch.int32), _dev(5, 64, dtype=torch.bfloat16), _dev(100, 64, dtype=torch.bfloat16)
    make = spo.make_logprob_desc
    _refused(TypeError, "logits", make, None, None, target, logits=torch.zeros(5, 100))
    _refused(TypeError, "logits", make, None, None, target, logits=_dev(5, 100, dtype=torch.float64))
    _refused(TypeError, "logits", make, None, None, target, logits=OnDevice(torch.zeros(100, 5).t()))
    _refused(TypeError, "logits", make, None, None, target, logits=OnDevice(torch.zeros(1, 100).expand(5, 100)))
    _refused(TypeError, "target", make, None, None, _dev(5), logits=z)
    _refused(ValueError, "target", make, None, None, _dev(4, dtype=torch.int32), logits=z)
    _refused(TypeError, "mask", make, None, None, target, mask=_dev(5), logits=z)
    _refused(ValueError, "mask", make, None, None, target, mask=_dev(6, dtype=torch.uint8), logits=z)
    _refused(TypeError, "hidden", make, torch.zeros(5, 64), W, target)
    _refused(TypeError, "W", make, X, _dev(100, 64), target)
    _refused(ValueError, "W", make, X, W, target, w_layout=spo.SPO_W_HV)
    _refused(ValueError, "W", make, X, _dev(100, 128, dtype=torch.bfloat16), target)

    d = make(None, None, target, logits=z, top_k=3)
    lse, top = _dev(5), _dev(5, 3)
    ids = _dev(5, 3, dtype=torch.int32)
    _refused(ValueError, "lse", spo.spo_logprob_bwd, d, _dev(4))
    _refused(ValueError, "entropy", spo.spo_logprob_bwd, d, lse, _dev(6))
    _refused(TypeError, "d_logp", spo.spo_logprob_bwd, d, lse, None, _dev(5, dtype=torch.bfloat16))
    _refused(ValueError, "d_top_logp", spo.spo_logprob_bwd, d, lse, None, None, None, ids, _dev(5, 2))
    _refused(ValueError, "top_id", spo.spo_logprob_bwd, d, lse, None, None, None, _dev(5, 2, dtype=torch.int32), top)
    head = make(X, W, target)
    _refused(TypeError, "d_W", spo.spo_logprob_bwd, head, lse, None, lse, d_W=torch.zeros(100, 64))
    _refused(ValueError, "d_W", spo.spo_logprob_bwd, head, lse, None, lse, d_W=_dev(99, 64))
    _refused(ValueError, "accumulate_dW", spo.spo_logprob_bwd, head, lse, None, lse, accumulate_dW=True)
    small = _dev(8, dtype=torch.uint8)
    _refused(ValueError, "workspace", spo.spo_logprob_fwd, head, workspace=small)
    assert not reached
    spo.spo_logprob_bwd(head, lse, None, lse, d_W=_dev(100, 64))
    assert reached == ["spo_logprob_bwd"]


def test_updates_look_at_their_tensors(reached):
    W, m, g = _dev(6, 8), _dev(6, 8), _dev(6, 8)
    _refused(TypeError, "G", spo.spo_orthogonalize, torch.zeros(6, 8))
    _refused(TypeError, "G", spo.spo_orthogonalize, _dev(6, 8, dtype=torch.float16))
    _refused(TypeError, "G", spo.spo_orthogonalize, OnDevice(torch.zeros(8, 6).t()))
    _refused(TypeError, "overlap", spo.spo_orthogonalize, OnDevice(torch.zeros(1, 8).expand(6, 8)))
    _refused(TypeError, "overlap", spo.spo_orthogonalize, OnDevice(torch.zeros(1, 6, 8).expand(3, 6, 8)))
    _refused(ValueError, "G", spo.spo_orthogonalize, _dev(6))
    _refused(ValueError, "out", spo.spo_orthogonalize, g, out=_dev(6, 7))
    _refused(TypeError, "out", spo.spo_orthogonalize, g, out=torch.zeros(6, 8))
    _refused(ValueError, "W", spo.spo_muon_update, _dev(6), m, g, lr=0.1)
    _refused(TypeError, "W", spo.spo_muon_update, _dev(6, 8, dtype=torch.float64), m, g, lr=0.1)
    _refused(TypeError, "W", spo.spo_muon_update, OnDevice(torch.zeros(8, 6).t()), m, g, lr=0.1)
    _refused(TypeError, "momentum", spo.spo_muon_update, W, _dev(6, 8, dtype=torch.bfloat16), g, lr=0.1)
    _refused(ValueError, "momentum", spo.spo_muon_update, W, _dev(6, 7), g, lr=0.1)
    _refused(ValueError, "grad", spo.spo_muon_update, W, m, _dev(5, 8), lr=0.1)
    _refused(TypeError, "grad", spo.spo_muon_update, W, m, _dev(6, 8, dtype=torch.float16), lr=0.1)
    assert not reached
    spo.spo_muon_update(W, m, g, lr=0.1)
    assert reached == ["spo_muon_update"]


# ------------------------------------------------------------------- registers
@pytest.mark.timeout(600)
def test_kernels_keep_their_values_in_registers(tmp_path):
    scratch = {}
    for src in ("logprob.hip", "orthogonalize.hip"):
        r = subprocess.run([build._hipcc(), *build.FLAGS, "--cuda-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
                            os.path.join(build.CSRC, src), "-o", str(tmp_path / "k.o")], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        name = None
        for line in r.stderr.splitlines():
            if m := re.search(r"remark: .*Function Name: (\S+)", line):
                name = m[1]
            elif m := re.search(r"remark: .*ScratchSize \[bytes/lane\]: (\d+)", line):
                scratch[name] = int(m[1])
    assert any("score_rows" in k for k in scratch) and any("orth_few" in k for k in scratch)
    # products on tiles of 256 keep a few addresses outside of their main loops; nothing else does
    large = {k: v for k, v in scratch.items() if "orth_product_kernelINS_4TileILi256E" in k}
    assert len(large) == 6 and max(large.values()) <= 128, large
    assert not any(v for k, v in scratch.items() if k not in large), scratch
