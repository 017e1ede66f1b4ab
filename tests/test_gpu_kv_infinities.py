"""Elements that are no numbers on their way through the paged cache: what is appended as such is read back, and attended to, as such."""
import numpy as np
import pytest
import torch

from paper_2211_17192_b200 import binding

pytestmark = pytest.mark.gpu
E4M3, INT8, F32, BF16, F16 = torch.float8_e4m3fn, torch.int8, torch.float32, torch.bfloat16, torch.float16
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("kind", [E4M3, INT8, F16, BF16])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("d", [64, 128])
def test_append_and_read(kind, dtype, d):
    rng = np.random.default_rng(d)
    rows = 8
    k, v = (torch.from_numpy(rng.standard_normal((1, rows, 2, d), dtype=np.float32)) for _ in range(2))
    for x in (k, v):
        x[0, 1, 0, 3] = INF
        x[0, 2, 1, d - 1] = -INF
        x[0, 3, 0, d // 2] = NAN
        x[0, 4, 1, 0] = 6e4
        if dtype != F16:
            x[0, 5, 0, 7] = 1e6
            x[0, 6, 1, d // 2 + 1] = -3e38
    k, v = k.to(dtype).cuda(), v.to(dtype).cuda()
    pool = torch.zeros(2, 2, 2, 32, d, dtype=kind, device="cuda")
    scales = torch.ones(2, 2, 2, 32, device="cuda") if kind in (E4M3, INT8) else None
    table, start = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"), torch.tensor([29], dtype=torch.int32, device="cuda")
    binding.spec_kv_append(k, v, pool, scales, table, start)
    for got, x in zip(binding.spec_kv_read(pool, scales, table, start, rows), (k, v)):
        if scales is not None:
            # a scale for a row: all of it is none
            none = ~torch.isfinite(x.float()).all(-1)
            assert got[none].isnan().all() and torch.isfinite(got[~none]).all()
        else:
            want = x.float()
            if kind == F16:  # (the largest value for what is beyond, and still a number)
                want = torch.where(torch.isfinite(want), want.clamp(-65504.0, 65504.0), want)
            want = want.to(kind).float()
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0, posinf=1e39, neginf=-1e39), want.nan_to_num(0.0, posinf=1e39, neginf=-1e39))


@pytest.mark.parametrize("kind,dtype", [(E4M3, BF16), (INT8, F16), (F16, F16), (BF16, BF16)])
@pytest.mark.parametrize("rows", [3, 40])
@pytest.mark.parametrize("which", [0, 1])
def test_attention_sees_them(kind, dtype, rows, which):
    rng = np.random.default_rng(3)
    k, v = (torch.from_numpy(rng.standard_normal((1, 70, 1, 64), dtype=np.float32)).to(dtype).cuda() for _ in range(2))
    (k, v)[which][0, 69, 0, 5] = INF  # the last token: for the last row alone
    pool = torch.zeros(3, 2, 1, 32, 64, dtype=kind, device="cuda")
    scales = torch.ones(3, 2, 1, 32, device="cuda") if kind in (E4M3, INT8) else None
    table, start = torch.tensor([[1, 0, 2]], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.spec_kv_append(k, v, pool, scales, table, start)
    q = torch.from_numpy(rng.standard_normal((1, rows, 2, 64), dtype=np.float32)).to(dtype).cuda()
    q[..., 5] = q[..., 5].abs() + 1
    out = binding.spec_paged_attention(q, pool, scales, table, start + 70).float()
    assert torch.isfinite(out[0, :-1]).all() and not torch.isfinite(out[0, -1]).all(-1).any()
