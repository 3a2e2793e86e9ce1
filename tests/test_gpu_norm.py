"""Normalisation of rows, forward and backward, against the definition in 64 bits.

Bounds.  A thread sums at most 64 elements in turn and joins them over 1024 threads in 6 + 16 more additions: sums are off by at
most 90 roundings of 2^-24 = 5.4e-6 of the sum of sizes, the variance by twice that and rstd by half of the variance's, so h by
6e-6 (1 + |h|) with what the mean is off by, in units of the row's deviation.  1e-5 (1 + |h|) |w| bounds y, beside the one
rounding to its type; dx is a difference of three terms, each within 2e-5; sums over rows within (rows in turn + 32) 2^-24, h's
own 1e-5 and a rounding."""
import pytest
import torch

import train_cases as tc
from pg_cases import say

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def spo():
    from paper_2509_13232_amd import binding
    binding.lib()
    return binding


def rows(T, N, dtype, pad=0, seed=0, mean=0.3, scale=1.0):
    g = torch.Generator().manual_seed(seed * 1000003 + T * 7919 + N)
    wide = torch.randn((T, N + pad), generator=g) * scale * torch.exp(0.5 * torch.randn((T, 1), generator=g)) + mean * scale
    return wide.to("cuda", dtype)[:, :N]


def vector(N, dtype, seed, mean=0.0):
    g = torch.Generator().manual_seed(seed * 31 + N)
    return (mean + 0.2 * torch.randn(N, generator=g)).to("cuda", dtype)


def cpu(*ts):
    return [None if t is None else t.double().cpu() for t in ts]


def check(spo, x, w, b, dy, layer, y_dtype, eps=1e-6, dx_dtype=None, dw_dtype=F32):
    T, N = x.shape
    d = spo.make_norm_desc(x, w, b, eps=eps, kind=spo.SPO_NORM_LAYER if layer else spo.SPO_NORM_RMS, y_dtype=y_dtype)
    y, mean, rstd = spo.spo_norm_fwd(d)
    dx, dw, db = spo.spo_norm_bwd(d, mean, rstd, dy, dx_dtype=dx_dtype, d_w_dtype=dw_dtype)
    torch.cuda.synchronize()
    assert y.dtype == y_dtype and y.shape == x.shape and (mean is None) != layer and dx.dtype == (dx_dtype or x.dtype)
    x64, w64, b64, dy64 = cpu(x, w, b, dy)
    want, h, mean64, rstd64 = tc.norm(x64, w64, b64, eps, layer)
    aw = torch.ones(N, dtype=torch.float64) if w is None else w64.abs()
    tc.off(rstd, rstd64, 1e-5 * rstd64, "rstd")
    if layer:
        tc.off(mean, mean64, 1e-5 * x64.abs().mean(dim=1), "mean")
    slack = 1e-5 * (1 + h.abs())
    tc.off(y, want, slack * aw + tc.EPS_HALF[y_dtype] * 1.01 * want.abs() + 2.0 ** -23 * (want.abs() + (0 if b is None else b64.abs())), "y")
    dx64, dw64, db64, size = tc.norm_grad(h, rstd64, dy64, w64, layer)
    tc.off(dx, dx64, 2e-5 * size + tc.EPS_HALF[dx.dtype] * 1.01 * dx64.abs(), "dx")
    ulps = (T / 256 + 64) * 2.0 ** -24
    for got, exact, sizes, of, name in ((dw, dw64, (dy64.abs() * (h.abs() * ulps + slack)).sum(dim=0), w, "d_weight"),
                                        (db, db64, dy64.abs().sum(dim=0) * ulps, b, "d_bias")):
        assert (got is None) == (of is None)
        if got is not None:
            assert got.dtype == dw_dtype
            tc.off(got, exact, sizes + tc.EPS_HALF[dw_dtype] * 1.01 * exact.abs() + 1e-37, name)
    return y, dx, dw, db


SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 64), (17, 513), (70, 1000), (33, 1024), (9, 1025), (300, 2048), (10, 2049), (700, 4096), (5, 4097),
          (3, 8192), (4, 8193), (3, 16384), (2, 16385), (3, 40001), (2, 65536), (2000, 100), (5000, 64), (300, 17000)]


@pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])
@pytest.mark.parametrize("T,N", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_against_the_definition(spo, T, N, dtype, layer):
    say(f"norm {T} x {N} {dtype} layer={layer}")
    x, dy = rows(T, N, dtype), rows(T, N, dtype, seed=1, mean=0.05)
    check(spo, x, vector(N, dtype, 2, 1.0), vector(N, dtype, 3), dy, layer, dtype)


@pytest.mark.parametrize("x_dtype", [F32, BF16])
@pytest.mark.parametrize("y_dtype", [F32, BF16])
@pytest.mark.parametrize("w_dtype", [F32, BF16])
@pytest.mark.parametrize("N", [96, 1500, 5001, 16500])
def test_types_mix(spo, x_dtype, y_dtype, w_dtype, N):
    say(f"norm types {x_dtype} {y_dtype} {w_dtype} {N}")
    x, dy = rows(37, N, x_dtype), rows(37, N, y_dtype, seed=1)
    for dx_dtype in (F32, BF16):
        check(spo, x, vector(N, w_dtype, 2, 1.0), vector(N, w_dtype, 3), dy, True, y_dtype, dx_dtype=dx_dtype, dw_dtype=w_dtype)


@pytest.mark.parametrize("T,N,pad", [(50, 1001, 23), (21, 4096, 1), (7, 300, 3), (3, 16401, 7), (40, 64, 64), (1, 33, 5)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_apart_and_not_aligned(spo, T, N, pad, dtype):
    say(f"norm rows apart {T} x {N} + {pad} {dtype}")
    x = rows(T + 1, N, dtype, pad=pad)[1:]
    wide = torch.zeros((T, N + pad + 1), device="cuda", dtype=dtype)
    dy = wide[:, 1:1 + N]
    dy.copy_(rows(T, N, dtype, seed=1))
    w = vector(N + 1, dtype, 2, 1.0)[1:]
    y, *_ = check(spo, x, w, None, dy, True, dtype)
    # into rows of a wider buffer: what lies between them stays
    out = torch.full((T, N + pad + 2), 7.0, device="cuda", dtype=dtype)
    d = spo.make_norm_desc(x, w, None)
    got, _, _ = spo.spo_norm_fwd(d, out=out[:, 1:1 + N])
    torch.cuda.synchronize()
    assert torch.equal(got, y) and bool((out[:, 0] == 7).all()) and bool((out[:, 1 + N:] == 7).all())


@pytest.mark.parametrize("w,b", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("layer", [True, False])
def test_without_weight_or_bias(spo, w, b, layer):
    say(f"norm weight={w} bias={b} layer={layer}")
    x, dy = rows(40, 777, BF16), rows(40, 777, BF16, seed=1)
    check(spo, x, vector(777, BF16, 2, 1.0) if w else None, vector(777, BF16, 3) if b else None, dy, layer, BF16)


@pytest.mark.parametrize("N", [100, 1000, 4096, 9000, 20000])
def test_rows_far_from_zero_keep_their_digits(spo, N):
    # means of 1e4 deviations, whose fp32 rounding is 5e-4 of one
    say(f"norm far from zero {N}")
    g = torch.Generator().manual_seed(N)
    x = (torch.randn((30, N), generator=g) + 1e4 * (1 + torch.rand((30, 1), generator=g))).cuda()
    check(spo, x, vector(N, F32, 2, 1.0), vector(N, F32, 3), rows(30, N, F32, seed=1), True, F32)


@pytest.mark.parametrize("N", [100, 1000, 4096, 9000, 20000])
@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("scale", [1e-27, 1e25])
def test_squares_beyond_fp32(spo, N, layer, scale):
    say(f"norm of numbers around {scale}, {N}")
    x = rows(5, N, F32, scale=scale)
    dy = rows(5, N, F32, seed=1, scale=min(1.0, scale))
    check(spo, x, vector(N, F32, 2, 1.0), None, dy, layer, F32, eps=0.0)


@pytest.mark.parametrize("N", [100, 4096, 9000, 20000])
@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_row_that_is_not_finite_stays_alone(spo, N, layer, bad):
    say(f"norm with {bad} in a row of {N}")
    x, dy, w = rows(9, N, BF16), rows(9, N, BF16, seed=1), vector(N, BF16, 2, 1.0)
    kind = spo.SPO_NORM_LAYER if layer else spo.SPO_NORM_RMS
    run = lambda d: (lambda f: (f, spo.spo_norm_bwd(d, f[1], f[2], dy)))(spo.spo_norm_fwd(d))   # noqa: E731
    clean, clean_b = run(spo.make_norm_desc(x, w, None, kind=kind))
    broken = x.clone()
    broken[4, N // 2] = bad
    f, b = run(spo.make_norm_desc(broken, w, None, kind=kind))
    torch.cuda.synchronize()
    assert bool(torch.isnan(b[1]).any())
    if layer or bad != bad:
        assert bool(torch.isnan(f[0][4]).all()) and bool(torch.isnan(b[0][4]).all())
    keep = torch.arange(9, device="cuda") != 4
    assert torch.equal(f[0][keep], clean[0][keep]) and torch.equal(b[0][keep], clean_b[0][keep])


@pytest.mark.parametrize("N", [64, 4096])
def test_rows_of_zeros_and_of_one_value(spo, N):
    say(f"norm of constant rows {N}")
    x = torch.zeros((4, N), device="cuda")
    x[1], x[2] = 3.0, -1e5
    d = spo.make_norm_desc(x, None, None, eps=1e-5)
    y, mean, rstd = spo.spo_norm_fwd(d)
    dx, _, _ = spo.spo_norm_bwd(d, mean, rstd, torch.ones_like(x))
    torch.cuda.synchronize()
    assert bool((y[:3] == 0).all()) and bool(torch.isfinite(dx).all()) and mean.tolist() == [0.0, 3.0, -1e5, 0.0]
    tc.off(rstd, torch.full((4,), 1e-5, dtype=torch.float64) ** -0.5, torch.full((4,), 316.3 * 1e-5), "rstd")


def test_no_rows(spo):
    say("norm of no rows")
    x = torch.empty((0, 300), device="cuda")
    w, b = vector(300, F32, 2), vector(300, F32, 3)
    d = spo.make_norm_desc(x, w, b)
    y, mean, rstd = spo.spo_norm_fwd(d)
    dx, dw, db = spo.spo_norm_bwd(d, mean, rstd, x)
    torch.cuda.synchronize()
    assert y.shape == dx.shape == (0, 300) and mean.numel() == 0 and not dw.any() and not db.any()
    dw, db = torch.ones(300, device="cuda"), torch.full((300,), 2.0, device="cuda")
    spo.spo_norm_bwd(d, mean, rstd, x, d_weight=dw, d_bias=db, accumulate=True)
    torch.cuda.synchronize()
    assert bool((dw == 1).all()) and bool((db == 2).all())


@pytest.mark.parametrize("T,N", [(3, 50), (900, 1500), (30, 20000)])
def test_gradients_are_added_to_and_left_out(spo, T, N):
    say(f"norm accumulates {T} x {N}")
    x, dy, w, b = rows(T, N, F32), rows(T, N, F32, seed=1), vector(N, F32, 2, 1.0), vector(N, F32, 3)
    d = spo.make_norm_desc(x, w, b)
    y, mean, rstd = spo.spo_norm_fwd(d)
    dx, dw, db = spo.spo_norm_bwd(d, mean, rstd, dy)
    dw2, db2 = torch.full_like(w, 0.5), torch.full_like(b, -0.25)
    out = spo.spo_norm_bwd(d, mean, rstd, dy, d_weight=dw2, d_bias=db2, accumulate=True)
    assert torch.equal(out[0], dx) and out[1] is dw2 and torch.equal(dw2, dw + 0.5) and torch.equal(db2, db - 0.25)
    none, dw3, db3 = spo.spo_norm_bwd(d, mean, rstd, dy, want_dx=False)
    assert none is None and torch.equal(dw3, dw) and torch.equal(db3, db)
    dx4, n1, n2 = spo.spo_norm_bwd(d, mean, rstd, dy, want_dw=False)
    assert n1 is None and n2 is None and torch.equal(dx4, dx)
    dw5 = spo.spo_norm_bwd(spo.make_norm_desc(x, w, None), mean, rstd, dy)[1]
    assert torch.equal(dw5, dw)
    y2, m2, r2 = spo.spo_norm_fwd(d, want_stats=False)
    assert m2 is None and r2 is None and torch.equal(y2, y)


@pytest.mark.parametrize("T,N", [(300, 700), (3, 5000), (5, 30000)])
def test_in_place(spo, T, N):
    say(f"norm in place {T} x {N}")
    x, dy, w = rows(T, N, BF16), rows(T, N, BF16, seed=1), vector(N, BF16, 2, 1.0)
    d = spo.make_norm_desc(x, w, None)
    y, mean, rstd = spo.spo_norm_fwd(d)
    dx, dw, _ = spo.spo_norm_bwd(d, mean, rstd, dy)
    over = dy.clone()
    got = spo.spo_norm_bwd(d, mean, rstd, over, dx=over)
    assert got[0] is over and torch.equal(over, dx) and torch.equal(got[1], dw)
    z = x.clone()
    dz = spo.make_norm_desc(z, w, None)
    got = spo.spo_norm_bwd(dz, mean, rstd, dy, dx=z)
    assert torch.equal(z, dx) and torch.equal(got[1], dw)
    z.copy_(x)
    assert spo.spo_norm_fwd(dz, out=z)[0] is z and torch.equal(z, y)


# rows enough that a group of threads takes two of them side by side, with a last one that is alone; widths of every such group
MANY = [(131080, 32), (131073, 17), (65601, 64), (32801, 128), (32769, 100), (16401, 256), (8201, 512), (8197, 511), (8199, 1000), (2055, 2000), (2051, 4000),
        (2053, 3999)]


@pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])
@pytest.mark.parametrize("T,N", MANY)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_many_rows(spo, T, N, dtype, layer):
    say(f"norm of many rows {T} x {N} {dtype} layer={layer}")
    x, dy = rows(T, N, dtype), rows(T, N, dtype, seed=1, mean=0.05)
    check(spo, x, vector(N, dtype, 2, 1.0), vector(N, dtype, 3), dy, layer, dtype)


@pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])
@pytest.mark.parametrize("T,N", [(131073, 32), (32, 64), (8199, 1000), (50, 1400), (2051, 2000), (2053, 4000), (40, 6000), (30, 8192), (20, 12288), (11, 20000)])
def test_rows_of_all_kinds_side_by_side(spo, T, N, layer):
    # ordinary rows beside rows that begin with an outlier, that lie far from zero, and whose squares leave fp32
    say(f"norm of rows of all kinds {T} x {N} layer={layer}")
    x, dy = rows(T, N, F32), rows(T, N, F32, seed=1)
    x[1::5, 0] = 1e4
    x[2::5, 0] *= 1e-3
    x[3::5] *= 1e25
    x[4::5] += 1e3
    dy[3::5] *= 1e-3
    check(spo, x, vector(N, F32, 2, 1.0), vector(N, F32, 3), dy, layer, F32)
    y, dx, _, _ = check(spo, x, None, None, dy, layer, F32)
    # a row's result is its own: alone, and in any order
    order = torch.randperm(T, generator=torch.Generator().manual_seed(4)).cuda()
    kind = spo.SPO_NORM_LAYER if layer else spo.SPO_NORM_RMS
    d = spo.make_norm_desc(x[order], kind=kind)
    other, mean, rstd = spo.spo_norm_fwd(d)
    d_other, _, _ = spo.spo_norm_bwd(d, mean, rstd, dy[order])
    assert torch.equal(other, y[order]) and torch.equal(d_other, dx[order])


@pytest.mark.parametrize("N", [1100, 1280, 1536, 1537, 2560, 5120, 6000, 8192, 10240, 12288, 24577, 33000])
def test_widths(spo, N):
    say(f"norm widths {N}")
    for dtype in (F32, BF16):
        x, dy = rows(25, N, dtype), rows(25, N, dtype, seed=1)
        check(spo, x, vector(N, dtype, 2, 1.0), vector(N, dtype, 3), dy, True, dtype)


@pytest.mark.parametrize("T,N", [(131073, 20), (8199, 700), (2051, 3000)])
def test_many_rows_in_place_and_into_others(spo, T, N):
    say(f"norm of many rows in place {T} x {N}")
    x, w = rows(T, N, BF16), vector(N, BF16, 2, 1.0)
    d = spo.make_norm_desc(x, w, None)
    y, mean, rstd = spo.spo_norm_fwd(d)
    out = torch.full((T + 2, N + 3), 7.0, device="cuda", dtype=BF16)
    got, _, _ = spo.spo_norm_fwd(d, out=out[1:-1, 2:-1])
    assert torch.equal(got, y) and bool((out[0] == 7).all()) and bool((out[-1] == 7).all())
    assert bool((out[:, :2] == 7).all()) and bool((out[:, -1] == 7).all())
    z = x.clone()
    assert torch.equal(spo.spo_norm_fwd(spo.make_norm_desc(z, w, None), out=z)[0], y)


def test_gradient_against_differences(spo):
    # central differences of sum(dy y) along random directions, in fp32 calls: y is off by 1e-5, a step of 2^-6 of the row's size,
    # third derivatives of order one: (2e-5 / 2^-5 + 2^-12) of the directions' norms
    say("norm gradients against differences")
    for layer in (True, False):
        T, N = 6, 200
        x, w, b = rows(T, N, F32), vector(N, F32, 2, 1.0), vector(N, F32, 3)
        dy = rows(T, N, F32, seed=1, mean=0.0)
        kind = spo.SPO_NORM_LAYER if layer else spo.SPO_NORM_RMS

        def total(x, w, b):
            return float((spo.spo_norm_fwd(spo.make_norm_desc(x, w, b, kind=kind))[0].double() * dy.double()).sum())
        d = spo.make_norm_desc(x, w, b, kind=kind)
        _, mean, rstd = spo.spo_norm_fwd(d)
        grads = spo.spo_norm_bwd(d, mean, rstd, dy)
        g = torch.Generator().manual_seed(9)
        for i, (t, grad) in enumerate(zip((x, w, b), grads)):
            v = torch.randn(t.shape, generator=g).cuda()
            step = 2.0 ** -6 / float(v.abs().max())
            up, down = [[x, w, b] for _ in range(2)]
            up[i], down[i] = t + step * v, t - step * v
            slope = (total(*up) - total(*down)) / (2 * step)
            size = float(dy.double().norm() * N ** 0.5)
            assert abs(slope - float((grad.double() * v.double()).sum())) < 1e-3 * size, (layer, i)


def test_results_do_not_depend_on_the_run_nor_on_what_the_workspace_held(spo):
    say("norm twice")
    x, dy, w, b = rows(3000, 1000, BF16), rows(3000, 1000, BF16, seed=1), vector(1000, BF16, 2, 1.0), vector(1000, BF16, 3)
    d = spo.make_norm_desc(x, w, b)
    _, mean, rstd = spo.spo_norm_fwd(d)
    ws = torch.empty(spo.spo_norm_bwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    first = spo.spo_norm_bwd(d, mean, rstd, dy, workspace=ws.fill_(255))
    second = spo.spo_norm_bwd(d, mean, rstd, dy, workspace=ws.fill_(0))
    assert all(torch.equal(p, q) for p, q in zip(first, second))


@pytest.mark.parametrize("T,N", [(500, 1200), (40, 12000), (20, 20000)])
def test_on_another_stream_and_in_a_graph(spo, T, N):
    say(f"norm on a stream and in a graph, {T} x {N}")
    x, dy, w, b = rows(T, N, BF16), rows(T, N, BF16, seed=1), vector(N, BF16, 2, 1.0), vector(N, BF16, 3)
    d = spo.make_norm_desc(x, w, b)
    ws = torch.empty(spo.spo_norm_bwd_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    dw, db = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")

    def both():
        y, mean, rstd = spo.spo_norm_fwd(d)
        dx, _, _ = spo.spo_norm_bwd(d, mean, rstd, dy, d_weight=dw, d_bias=db, accumulate=True, workspace=ws)
        return y, mean, rstd, dx

    want = [t.clone() for t in both()]
    one = dw.clone(), db.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    dw.zero_(), db.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    torch.cuda.synchronize()
    total = [torch.zeros_like(t) for t in one]
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        (torch.randn(1 << 20, device="cuda") * 1.0001).sin_()
        torch.cuda.synchronize()
        total = [t + o for t, o in zip(total, one)]
        assert all(torch.equal(p, q) for p, q in zip(out, want)), k
        assert torch.equal(dw, total[0]) and torch.equal(db, total[1]), k
    # and on other inputs in the same places
    x.copy_(rows(T, N, BF16, seed=5))
    want = [t.clone() for t in both()]
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, want))


@pytest.mark.parametrize("N", [4096, 40000])
def test_more_than_2_to_the_31_elements(spo, N):
    T = (1 << 31) // N + 300
    say(f"norm of {T} x {N} bf16")
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((T, N), device="cuda", dtype=BF16).normal_(generator=g)
    w = vector(N, BF16, 2, 1.0)
    d = spo.make_norm_desc(x, w, None)
    y, mean, rstd = spo.spo_norm_fwd(d)
    dx, dw, _ = spo.spo_norm_bwd(d, mean, rstd, y)
    some = torch.cat([torch.arange(3), torch.arange(T - 5, T), torch.randint(0, T, (8,), generator=torch.Generator().manual_seed(1))]).cuda()
    ds = spo.make_norm_desc(x[some].contiguous(), w, None)
    ys, ms, rs = spo.spo_norm_fwd(ds)
    dxs, _, _ = spo.spo_norm_bwd(ds, ms, rs, ys)
    torch.cuda.synchronize()
    assert torch.equal(y[some], ys) and torch.equal(mean[some], ms) and torch.equal(dx[some], dxs)
    # y w^-1 = h: the weight's gradient is sum y h, within the bf16 rounding of y (2^-8) of the sum of h^2 |w|, T rows of it
    assert float(((dw.double() / w.double()) / T - 1).abs().max()) < 2.0 ** -8 + 6 * (2.0 / T) ** 0.5
