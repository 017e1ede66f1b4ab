"""Sizes and arguments that the 8-bit operators have no form for are refused, with all outputs given and with none."""
import pytest
import torch

from paper_2211_17192_b200 import binding

pytestmark = pytest.mark.gpu
E4M3, BF16, F16 = torch.float8_e4m3fn, torch.bfloat16, torch.float16


def test_a_row_count_past_32_bits_is_refused():
    # (2^32 + 4 rows would be four in the library's 32 bits)
    rows = 2 ** 32 + 4
    x, gain = torch.empty(rows, 1, dtype=BF16, device="cuda"), torch.ones(1, device="cuda")
    codes, scales = torch.empty(rows, 1, dtype=E4M3, device="cuda"), torch.empty(rows, device="cuda")
    codes.view(torch.uint8)[:8] = 7
    for given in (dict(), dict(codes=codes, scales=scales)):
        with pytest.raises(ValueError, match="32 bits"):
            binding.spec_quantize_fp8(x, **given)
        with pytest.raises(ValueError, match="32 bits"):
            binding.spec_norm_fp8(x, gain, **given)
    assert torch.all(codes.view(torch.uint8)[:8] == 7)


def test_a_page_table_past_32_bits_is_refused():
    pool, table = torch.zeros(1, 2, 1, 32, 64, dtype=F16, device="cuda"), torch.zeros(1, 2 ** 32 + 1, dtype=torch.int32, device="cuda")
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    k = torch.ones(1, 1, 1, 64, dtype=F16, device="cuda")
    with pytest.raises(ValueError, match="32 bits"):
        binding.spec_kv_append(k, k, pool, None, table, start)
    with pytest.raises(ValueError, match="32 bits"):
        binding.spec_kv_read(pool, None, table, start, 1)
    with pytest.raises(ValueError, match="32 bits"):
        binding.spec_paged_attention(k, pool, None, table, start + 1)
    assert not pool.any()


def test_what_is_no_tensor_and_what_has_no_heads():
    i32 = dict(dtype=torch.int32, device="cuda")
    pool, table, start = torch.zeros(1, 2, 1, 32, 64, dtype=F16, device="cuda"), torch.zeros(1, 1, **i32), torch.zeros(1, **i32)
    k = torch.ones(1, 1, 1, 64, dtype=F16, device="cuda")
    for kw in (dict(q=[k]), dict(q=k.tolist(), q_out=k), dict(rope=[[1.0, 0.0]]), dict(rope=torch.tensor(1.0, device="cuda")), dict(q=k[0])):
        with pytest.raises(ValueError):
            binding.spec_kv_append(k, k, pool, None, table, start, **kw)
    work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    none = torch.zeros(1, 2, 0, 32, 64, dtype=F16, device="cuda")
    flat = torch.zeros(1, 2, 1, 32, 0, dtype=F16, device="cuda")
    for q, cache in ((k.sum(), pool), (k[0], pool), (k[..., :0], flat), (k[..., :0], pool), (k, none), (k.tolist(), pool)):
        for given in (dict(), dict(out=torch.empty_like(k), workspace=work)):
            with pytest.raises(ValueError):
                binding.spec_paged_attention(q, cache, None, table, start + 1, **given)
    assert not pool.any()
