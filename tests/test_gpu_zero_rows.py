"""Attention over 8-bit pools in which some V rows are zeros (a sink's, a cleared token's): the format gives these the scale 1, which may be
far above the scales of the others and says nothing about what they add."""
import numpy as np
import pytest
import torch

import rows8
from paper_2211_17192_b200 import binding

pytestmark = pytest.mark.gpu
E4M3, INT8, BF16, F16 = torch.float8_e4m3fn, torch.int8, torch.bfloat16, torch.float16


def cache_with_zero_rows(seed, kind, n_kv, d, size, batch, width, sinks, size_of_v, lead):
    """Pages in order; V rows at the positions `sinks` of every sequence are zeros, and their keys lead by `lead` for a query whose first
    element is one."""
    rng = np.random.default_rng(seed)
    pages = batch * width
    x = torch.from_numpy(rng.standard_normal((pages, 2, n_kv, size, d), dtype=np.float32))
    x[:, 1] *= size_of_v
    x[:, 0, :, :, 0] = 0
    for b in range(batch):
        for p in sinks:
            page, slot = b * width + p // size, p % size
            x[page, 0, :, slot] = 0
            x[page, 0, :, slot, 0] = lead
            x[page, 1, :, slot] = 0
    scales = rows8.scale64(x.double(), kind).float()
    z = x * (1.0 / scales)[..., None]
    codes = z.clamp(-448, 448).to(kind) if kind == E4M3 else z.round().to(kind)
    if kind == E4M3:  # (a zero may be a negative one)
        codes.view(torch.uint8)[:, 1, :, :, 1::2] |= (codes.view(torch.uint8)[:, 1, :, :, 1::2] == 0).to(torch.uint8) * 128
    table = torch.arange(pages, dtype=torch.int32).view(batch, width).cuda()
    return codes.cuda(), scales.cuda(), table


@pytest.mark.parametrize("kind,dtype", [(E4M3, BF16), (E4M3, F16), (INT8, BF16), (INT8, F16)])
@pytest.mark.parametrize("rows,group", [(2, 3), (4, 4), (7, 4), (12, 4)])
@pytest.mark.parametrize("d,size_of_v,lead", [(64, 0.1, 8.0), (128, 0.05, 10.0), (64, 1e-3, 12.0), (128, 1e-7, 9.0), (64, 300.0, -3.0), (64, 1.0, 0.0)])
def test_a_row_of_zeros_leaves_the_others_their_weights(kind, dtype, rows, group, d, size_of_v, lead):
    n_kv, size, width = 2, 64, 24
    lengths = [1500, 70, 6, 1400]
    pool, scales, table = cache_with_zero_rows(rows, kind, n_kv, d, size, 4, width, [3, 5, 63, 1399, 1496], size_of_v, lead)
    assert float(scales[0, 1, 0, 5]) == 1.0
    rng = np.random.default_rng(d)
    q = 0.1 * torch.from_numpy(rng.standard_normal((4, rows, n_kv * group, d), dtype=np.float32))
    q[..., 0] = 1.0
    q = q.to(dtype).cuda()
    at = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got = binding.spec_paged_attention(q, pool, scales, table, at, scale=1.0)
    want, bound = rows8.attention64(q, pool, scales, table, at, 1.0)
    # (the bound's last term is a step of fp16's subnormals, which an output in bf16 does not have; without a key it is zero altogether)
    if dtype == BF16:
        bound = (bound - 2.0 ** -25).clamp_min(0)
    err = (got.cpu().double() - want).abs()
    assert torch.all(err <= bound), float((err - bound).max())


@pytest.mark.parametrize("kind", [E4M3, INT8])
@pytest.mark.parametrize("rows", [3, 40])
def test_rows_of_zeros_alone_give_zeros(kind, rows):
    pool, scales, table = cache_with_zero_rows(1, kind, 1, 64, 32, 2, 4, list(range(128)), 1.0, 5.0)
    q = torch.ones(2, rows, 2, 64, dtype=F16, device="cuda")
    at = torch.tensor([128, 50], dtype=torch.int32, device="cuda")
    assert not binding.spec_paged_attention(q, pool, scales, table, at).float().any()
    # one row among them that is not
    pool.view(torch.uint8)[1, 1, 0, 2] = 0x38 if kind == E4M3 else 1
    scales[1, 1, 0, 2] = 2.0 ** -60
    q = q.to(BF16)
    got = binding.spec_paged_attention(q, pool, scales, table, at)
    want, bound = rows8.attention64(q, pool, scales, table, at, 64 ** -0.5)
    assert want[0].any() and torch.all((got.cpu().double() - want).abs() <= (bound - 2.0 ** -25).clamp_min(0))


@pytest.mark.parametrize("kind", [E4M3, INT8])
@pytest.mark.parametrize("rows", [2, 12])
def test_rows_of_zeros_count_beside_large_ones(kind, rows):
    # half of the rows are zeros, of a weight of e^-10 each: together a few per cent of the sum, whatever the others' sizes
    batch, width, size = 2, 12, 64
    pool, scales, table = cache_with_zero_rows(2, kind, 1, 64, size, batch, width, list(range(1, width * size, 2)), 1e12, -10.0)
    rng = np.random.default_rng(9)
    q = 0.1 * torch.from_numpy(rng.standard_normal((batch, rows, 4, 64), dtype=np.float32))
    q[..., 0] = 1.0
    q = q.to(BF16).cuda()
    pool.view(torch.uint8)[:, 0, :, 0::2] = 0  # (keys without a score)
    at = torch.tensor([768, 200], dtype=torch.int32, device="cuda")
    got = binding.spec_paged_attention(q, pool, scales, table, at, scale=1.0)
    want, bound = rows8.attention64(q, pool, scales, table, at, 1.0)
    assert torch.all((got.cpu().double() - want).abs() <= bound)
