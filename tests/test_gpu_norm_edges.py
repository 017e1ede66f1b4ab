"""Norm and quantisation of rows that hold no numbers, or numbers at the ends of the range, in calls of few rows and of many: the same rows
get the same answers."""
import numpy as np
import pytest
import torch

import rows8
from paper_2211_17192_b200 import binding
from test_gpu_rows8 import NORM_REL, normal

pytestmark = pytest.mark.gpu
E4M3, F32, BF16, F16 = torch.float8_e4m3fn, torch.float32, torch.bfloat16, torch.float16
WIDTHS = [2048, 4096, 8192, 16384]  # (a kernel of its own each in calls of many rows)


def same(a, b):
    return torch.equal(a.float().nan_to_num(12345.0), b.float().nan_to_num(12345.0))


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_quantize_rows_at_the_ends(d, dtype):
    if d == 16384 and dtype == F32:
        d = 14336  # (56 KB, the longest row that many rows of this type take the same way)
    x = normal(d, 300, d)
    if dtype != F16:
        x[1] *= 1e30
        x[2] *= 1e-30
        x[6, 3] = 3e38
    x[3] = 0
    x[4, d - 1] = float("nan")
    x[5, d // 2] = -float("inf")
    x[7] = float("nan")
    x[299, 0] = float("inf")
    x = x.to(dtype).cuda()
    codes, scales = binding.spec_quantize_fp8(x)
    none = [4, 5, 7, 299]
    fine = [r for r in range(300) if r not in none]
    rows8.check_codes(codes[fine], scales[fine], x[fine], E4M3)
    assert not torch.isfinite(scales[none]).any() and torch.isnan(codes[none].float() * scales[none, None]).all()
    for rows in (list(range(8)), none):
        few = binding.spec_quantize_fp8(x[rows].contiguous())
        assert same(few[0], codes[rows]) and same(few[1], scales[rows])


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype,h_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("summed", [True, False])
def test_norm_rows_that_are_no_numbers(d, dtype, h_dtype, summed):
    rows = 160
    if (dtype, d, summed) == (F32, 16384, True):
        d = 6144  # (48 KB a row with its residual)
    x, residual, gain = normal(d, rows, d).to(dtype), normal(d + 1, rows, d).to(h_dtype) if summed else None, 1 + 0.1 * normal(d + 2, d)
    x[1, 3] = float("nan")
    x[2, d - 1] = float("inf")
    x[3] = 0
    if summed:
        residual[3] = 0
        residual[4, 5] = -float("inf")
        none = [1, 2, 4]
    else:
        none = [1, 2]
    gain[3] = 0.0  # (takes the NaN out of the products, not out of the row)
    gain[d - 1] = 0.0
    args = lambda r: (x[r].contiguous().cuda(), gain.cuda(), 1e-6, None if residual is None else residual[r].contiguous().cuda())
    codes, scales, _ = binding.spec_norm_fp8(*args(slice(None)))
    assert torch.isnan(codes[none].float() * scales[none, None]).all() and not torch.isfinite(scales[none]).any()
    fine = [r for r in range(rows) if r not in none]
    w = x.float() + (residual.float() if summed else 0)
    w = (w.to(h_dtype) if summed else w).double()
    y = w * gain.double() / torch.sqrt((w * w).mean(-1, keepdim=True) + 1e-6)
    rows8.check_codes(codes[fine], scales[fine], y[fine], E4M3, NORM_REL)
    few = binding.spec_norm_fp8(*args(slice(0, 6)))
    assert torch.equal(torch.isnan(few[1]), torch.isnan(scales[:6])) and torch.equal(torch.isnan(few[0].float()), torch.isnan(codes[:6].float()))


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_gain_that_is_no_number_is_in_every_row(d, dtype, value):
    x, gain = normal(d, 160, d).to(dtype).cuda(), torch.ones(d, device="cuda")
    gain[5] = value
    x[7, 5] = 0  # (0 * inf)
    x[8] = 0
    for part in (x, x[:9].contiguous()):
        codes, scales, _ = binding.spec_norm_fp8(part, gain)
        assert not torch.isfinite(scales).any() and torch.isnan(codes.float() * scales[:, None]).all()


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_squares_past_the_range_are_not_a_row_of_zeros(d, dtype):
    x, gain = normal(d, 160, d), 1 + 0.1 * normal(d + 1, d)
    x[1] *= 1e25
    x[2] *= 1e15      # (squares of 1e30: within it)
    x[3] = 0
    x[3, 1] = 2e19
    x[4] = 0
    x[4, 1] = 1e19
    x = x.to(dtype)
    for rows in (slice(0, 5), slice(None)):
        codes, scales, _ = binding.spec_norm_fp8(x[rows].contiguous().cuda(), gain.cuda())
        fine = [0, 2, 4]
        assert torch.isnan(scales[[1, 3]]).all() and torch.isnan(codes[[1, 3]].float()).all()
        w = x[fine].double()
        rows8.check_codes(codes[fine], scales[fine], w * gain.double() / torch.sqrt((w * w).mean(-1, keepdim=True) + 1e-6), E4M3, NORM_REL)


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size,gain,eps", [(1e-18, 1e-18, 1e-30), (1e-20, 1e-16, 1e-36), (1e-19, 1e-18, 1e-30), (1e-25, 1e-12, 1e-38), (1e-15, 1e-25, 1e-30),
                                           (1e-18, 1e-17, 2.0 ** -90), (1e-20, 1e-17, 2.0 ** -90)])
def test_tiny_rows_under_a_tiny_eps(d, dtype, size, gain, eps):
    # h * gain of about 10^-36: 448 of that is past fp32's range, y itself is not small.  (In the third case y is below 448 of the least
    # scale, 2^-80.  The last eps is the least that calls of many rows take to the kernel for these.)
    x = (normal(d, 160, d) * size).to(dtype)
    x[:, 1::7] = 0
    x[2] = 0
    gains = torch.full((d,), gain)
    for rows in (slice(0, 5), slice(None)):
        codes, scales, _ = binding.spec_norm_fp8(x[rows].contiguous().cuda(), gains.cuda(), eps)
        w = x[rows].double()
        e = torch.tensor(eps, dtype=F32).double()  # (as the kernel is given it)
        # h * gain is rounded to fp32, among the subnormals too (by 2^-150, which is much of a small element): the same product here.  Squares
        # and their sums are off by 2^-150 each there, d of them at most, which is in the row's factor.
        y = (x[rows].float() * gains).double() / torch.sqrt((w * w).mean(-1, keepdim=True) + e)
        small = float(d * 2.0 ** -150 / ((w * w).mean(-1) + e).min())
        rows8.check_codes(codes, scales, y, E4M3, NORM_REL + small)


@pytest.mark.parametrize("rows,d", [(5, 768), (3, 4104), (300, 2048), (200, 4096), (160, 11003)])
@pytest.mark.parametrize("dtype,h_dtype", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
def test_a_sum_that_is_not_stored(rows, d, dtype, h_dtype):
    # the library's form without h: the sum is not rounded to h's type on its way (16-bit sums are of two 16-bit values: exact in fp32 or
    # off by 2^-24)
    kinds = {F32: 0, BF16: 1, F16: 2}
    x, residual, gain = normal(d, rows, d).to(dtype).cuda(), (normal(d + 1, rows, d) * 5).to(h_dtype).cuda(), (1 + 0.1 * normal(d + 2, d)).cuda()
    kept = residual.clone()
    codes, scales = torch.empty(rows, d, dtype=E4M3, device="cuda"), torch.empty(rows, device="cuda")
    assert binding.lib().spec_norm_fp8(x.data_ptr(), kinds[dtype], residual.data_ptr(), None, kinds[h_dtype], gain.data_ptr(), 1e-6, rows, d,
                                       codes.data_ptr(), scales.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    w = (x.float() + residual.float()).double()
    rows8.check_codes(codes, scales, w * gain.double() / torch.sqrt((w * w).mean(-1, keepdim=True) + 1e-6), E4M3, NORM_REL)
    assert torch.equal(residual, kept)
