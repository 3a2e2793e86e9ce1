"""Normalisation of rows at the ends of fp32's range against the definition in 64 bits: the bounds of
test_gpu_norm.py.

Rows there are summed in 64 bits from the row itself, so the bounds leave room.  rstd of the widest rows is 2^-128 and more, a
subnormal number: its rounding takes 2^-150 2^128 = 2.4e-7 of it at most, within the bound of 1e-5."""
import pytest
import torch

import train_cases as tc
from pg_cases import say
from test_gpu_norm import check, cpu, rows, spo, vector  # noqa: F401

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
KINDS = pytest.mark.parametrize("layer", [True, False], ids=["layer", "rms"])


def beside_others(x, many):
    """x among ordinary rows, as its first and third ones; `many`: as many rows as make a group of threads take two of them."""
    out = rows(many, x.shape[1], x.dtype, seed=8)
    out[0], out[2] = x[0], x[-1]
    return out


WIDE = [(3, 9), (20, 9), (20, 131073), (100, 9), (700, 9), (700, 8201), (1400, 9), (2000, 2053), (4096, 9), (9000, 9), (12288, 9), (20000, 9), (30000, 5),
        (40000, 5), (65536, 3)]


def wide_rows(N, many, dtype):
    """Among others, rows of both signs whose difference is no number of fp32: a few of one sign first, and half of each."""
    wide = torch.full((2, N), -3e38, dtype=dtype, device="cuda")
    wide[0, :min(8, N - 1)] = 3e38
    wide[1, ::2] = 3.3e38
    return beside_others(wide, many)


@TYPES
@KINDS
@pytest.mark.parametrize("N,many", WIDE)
def test_differences_beyond_fp32(spo, N, many, dtype, layer):  # noqa: F811
    say(f"norm of rows wider than fp32, {many} x {N} {dtype} layer={layer}")
    x, w, b = wide_rows(N, many, dtype), vector(N, F32, 2, 1.0), vector(N, F32, 3)
    y, mean, rstd = spo.spo_norm_fwd(spo.make_norm_desc(x, w, b, kind=spo.SPO_NORM_LAYER if layer else spo.SPO_NORM_RMS))
    torch.cuda.synchronize()
    x64, w64, b64 = cpu(x, w, b)
    want, h, mean64, rstd64 = tc.norm(x64, w64, b64, layer=layer)
    tc.off(rstd, rstd64, 1e-5 * rstd64, "rstd")
    if layer:
        tc.off(mean, mean64, 1e-5 * x64.abs().mean(dim=1), "mean")
    tc.off(y, want, 1e-5 * (1 + h.abs()) * w64.abs() + tc.EPS_HALF[dtype] * 1.01 * want.abs() + 2.0 ** -23 * (want.abs() + b64.abs()), "y")


@TYPES
@pytest.mark.parametrize("N", [1, 2, 3, 5, 7, 100])
def test_rows_of_the_largest_value(spo, N, dtype):  # noqa: F811
    say(f"norm of rows of the largest number, {N} {dtype}")
    x = torch.full((3, N), torch.finfo(dtype).max, dtype=dtype, device="cuda")
    x[1] *= -1
    d = spo.make_norm_desc(x, None, None, eps=1e-6, y_dtype=F32)
    y, mean, rstd = spo.spo_norm_fwd(d)
    dx, _, _ = spo.spo_norm_bwd(d, mean, rstd, torch.ones_like(x))
    torch.cuda.synchronize()
    # the mean is the value itself: of sums in 64 bits, exactly
    assert bool((y == 0).all()) and torch.equal(mean, x[:, 0].float()) and bool(torch.isfinite(dx).all())
    tc.off(rstd, torch.full((3,), 1e3, dtype=torch.float64), torch.full((3,), 1e-2), "rstd")


@KINDS
@pytest.mark.parametrize("N,many", [(100, 9), (100, 32769), (1400, 9), (2000, 2053), (4096, 9), (9000, 9), (20000, 9), (65536, 3)])
@pytest.mark.parametrize("size,lead", [(1e18, 3e22), (1e25, 1e29), (1e-18, 1e-14), (1e-27, 3e-23)])
def test_large_first_elements_where_squares_leave_fp32(spo, N, many, size, lead, layer):  # noqa: F811
    say(f"norm of {many} rows of {N} around {size} that begin with {lead}")
    g = torch.Generator().manual_seed(N)
    far = torch.randn((2, N), generator=g).cuda() * size
    far[:, :4] = lead
    x = beside_others(far, many)
    dy = rows(many, N, F32, seed=1)
    dy[0] *= min(1.0, size)
    dy[2] *= min(1.0, size)
    check(spo, x, vector(N, F32, 2, 1.0), vector(N, F32, 3), dy, layer, F32, eps=0.0)


@TYPES
@pytest.mark.parametrize("T,N", [(9, 100), (131073, 20), (9, 4096), (5, 40000)])
def test_in_place_beyond_fp32(spo, T, N, dtype):  # noqa: F811
    say(f"norm in place beyond fp32, {T} x {N} {dtype}")
    x = rows(T, N, dtype)
    x[1] = -3e38
    x[1, :3] = 3e38
    x[3] *= 1e25
    y, _, _ = spo.spo_norm_fwd(spo.make_norm_desc(x))
    z = x.clone()
    assert bool(torch.isfinite(y).all()) and torch.equal(spo.spo_norm_fwd(spo.make_norm_desc(z), out=z)[0], y)


@TYPES
@KINDS
@pytest.mark.parametrize("N,many", WIDE)
def test_gradients_of_differences_beyond_fp32(spo, N, many, dtype, layer):  # noqa: F811
    say(f"norm gradients of rows wider than fp32, {many} x {N} {dtype} layer={layer}")
    dy = rows(many, N, dtype, seed=1)
    dy[0] *= 1e20    # (gradients are divided by the rows' deviations)
    dy[2] *= 1e20
    check(spo, wide_rows(N, many, dtype), vector(N, F32, 2, 1.0), vector(N, F32, 3), dy, layer, dtype)


@pytest.mark.parametrize("x_dtype,y_dtype", [(F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("N", [100, 1000, 5000, 9000, 17000])
def test_gradients_of_differences_beyond_fp32_of_two_types(spo, N, x_dtype, y_dtype):  # noqa: F811
    say(f"norm gradients of rows wider than fp32, {N} {x_dtype} {y_dtype}")
    dy = rows(9, N, y_dtype, seed=1)
    dy[0] *= 1e20
    dy[2] *= 1e20
    check(spo, wide_rows(N, 9, x_dtype), vector(N, F32, 2, 1.0), vector(N, F32, 3), dy, True, y_dtype)


@KINDS
@pytest.mark.parametrize("N", [100, 1000, 5000, 9000, 17000])
def test_gradients_of_subnormal_rows(spo, N, layer):  # noqa: F811
    # deviations of 2^-128: rstd is near fp32's end, and half of an element loses its last place, 2^-150 or 2^-22 = 2.4e-7 of a deviation
    say(f"norm gradients of rows of 3e-39, {N} layer={layer}")
    x = torch.randn((9, N), generator=torch.Generator().manual_seed(N)).cuda() * 4e-39
    dy = rows(9, N, F32, seed=1, scale=1e-30)
    check(spo, x, vector(N, F32, 2, 1.0), vector(N, F32, 3), dy, layer, F32, eps=0.0)


@KINDS
@pytest.mark.parametrize("T,N", [(131073, 20), (40, 64), (8199, 1000), (50, 1400), (2053, 4000), (12, 12288), (9, 40000)])
def test_a_row_is_its_own_beside_any_other(spo, T, N, layer):  # noqa: F811
    # ordinary rows, also with outputs at bf16's lower end, beside rows that are summed in 64 bits
    say(f"norm of rows beside those in 64 bits, {T} x {N} layer={layer}")
    x = rows(T, N, BF16)
    x[3::7] *= 1e25
    w, b = vector(N, F32, 2, 1.0), vector(N, F32, 3)
    w[::3] *= 1e-38
    b[::3] = 0
    kind = spo.SPO_NORM_LAYER if layer else spo.SPO_NORM_RMS
    want = spo.spo_norm_fwd(spo.make_norm_desc(x, w, b, kind=kind))
    order = torch.cat([torch.arange(i, T, 7) for i in range(7)]).cuda()      # those of a kind together
    got = spo.spo_norm_fwd(spo.make_norm_desc(x[order], w, b, kind=kind))
    for p, q in zip(got, want):
        assert p is None and q is None or torch.equal(p, q[order])
