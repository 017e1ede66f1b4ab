"""Attention of fp16 queries whose elements lie far apart: each is multiplied as it is."""
import numpy as np
import pytest
import torch

import rows8
from paper_2211_17192_b200 import binding

pytestmark = pytest.mark.gpu
E4M3, INT8, F16 = torch.float8_e4m3fn, torch.int8, torch.float16


@pytest.mark.parametrize("kind", [F16, E4M3, INT8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,group", [(1, 1), (3, 4), (7, 4), (9, 6)])
def test_small_elements_beside_a_large_one(kind, d, rows, group):
    # the first element of a query is 2^15 and of every key zero: the scores are made of the others, of about 2^-11, and keys of 10^3
    rng = np.random.default_rng(rows)
    x = torch.from_numpy(rng.standard_normal((6, 2, 2, 32, d), dtype=np.float32))
    x[:, 0] *= 1000.0
    x[:, 0, ..., 0] = 0
    scales = None
    if kind in rows8.TOP:
        scales = rows8.scale64(x.double(), kind).float()
        z = x * (1.0 / scales)[..., None]
        x = z.clamp(-448, 448) if kind == E4M3 else z.round()
        scales = scales.cuda()
    pool = x.to(kind).cuda()
    table = torch.tensor([[4, 0, 2], [1, 3, 5]], dtype=torch.int32, device="cuda")
    q = 2.0 ** -11 * torch.from_numpy(rng.standard_normal((2, rows, 2 * group, d), dtype=np.float32))
    q[..., 0] = 2.0 ** 15
    q = q.to(F16).cuda()
    at = torch.tensor([90, 65], dtype=torch.int32, device="cuda")
    got = binding.spec_paged_attention(q, pool, scales, table, at, scale=0.5)
    want, bound = rows8.attention64(q, pool, scales, table, at, 0.5)
    err = (got.cpu().double() - want).abs()
    assert torch.all(err <= bound), float((err - bound).max())
