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
