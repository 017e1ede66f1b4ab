"""Attention over paged rows in 8 and 16 bits against the formula in 64 bits."""
import numpy as np
import pytest
import torch

import rows8
from paper_2211_17192_b200 import binding

pytestmark = pytest.mark.gpu
E4M3, INT8, BF16, F16 = torch.float8_e4m3fn, torch.int8, torch.bfloat16, torch.float16


def compare(seed, kind, dtype, d, n_kv, group, size, rows, lengths, scale=None, table=None, extra=2, sharp=1.0):
    rng = np.random.default_rng(seed)
    batch, width = len(lengths), max(1, max(-(-l // size) for l in lengths))
    used = [-(-max(l, 0) // size) for l in lengths]
    pages = sum(used) + extra
    pool, scales = rows8.make_cache(rng, pages, n_kv, size, d, kind)
    if table is None:
        table = rows8.make_table(rng, pages, batch, width, used)
    q = (sharp * torch.from_numpy(rng.standard_normal((batch, rows, n_kv * group, d), dtype=np.float32))).to(dtype).cuda()
    at = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    need = binding.spec_paged_attention_workspace_bytes(batch, rows, n_kv * group, n_kv, d)
    workspace = torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda")  # (NaN, and a border behind it)
    out = torch.full_like(q, float("nan"))
    got = binding.spec_paged_attention(q, pool, scales, table, at, scale=scale, out=out, workspace=workspace[:need])
    assert got is out
    want, bound = rows8.attention64(q, pool, scales, table, at, d ** -0.5 if scale is None else scale)
    err = (out.cpu().double() - want).abs()
    assert torch.all(err <= bound), (float((err - bound).max()), float(err.max()))
    assert torch.all(workspace[need:] == 0xff)
    again = binding.spec_paged_attention(q, pool, scales, table, at, scale=scale)
    assert torch.equal(again, out)
    return q, pool, scales, table, at, out


KINDS = [(E4M3, BF16), (E4M3, F16), (INT8, BF16), (INT8, F16), (F16, F16), (BF16, BF16)]


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,n_kv,group", [(1, 2, 1), (1, 1, 4), (3, 2, 4), (7, 1, 1), (5, 2, 8), (9, 1, 12)])
def test_types_and_head_layouts(kind, dtype, d, rows, n_kv, group):
    compare(rows, kind, dtype, d, n_kv, group, 64, rows, [200, 1, 65, 128, 63])


@pytest.mark.parametrize("kind,dtype", [(E4M3, BF16), (INT8, F16), (F16, F16), (BF16, BF16)])
@pytest.mark.parametrize("size", [32, 64, 128, 256])
@pytest.mark.parametrize("lengths", [[0], [1], [2], [31, 32, 33], [0, 0, 64, 0], [1000], [257, 0, 5, 511], [2, 700, 0]])
def test_lengths_and_pages(kind, dtype, size, lengths):
    compare(size + len(lengths), kind, dtype, 128, 2, 2, size, 3, lengths)


@pytest.mark.parametrize("kind,dtype", [(E4M3, F16), (INT8, BF16), (F16, F16)])
def test_long_and_many(kind, dtype):
    compare(1, kind, dtype, 64, 1, 4, 256, 1, [20001])                 # one segment for all SMs
    compare(2, kind, dtype, 64, 1, 2, 32, 2, [7] * 300 + [0] * 20 + [130])  # more sequences than threads
    compare(3, kind, dtype, 64, 3, 1, 64, 1, [3000, 10, 0, 777, 64])
    compare(4, kind, dtype, 64, 2, 1, 64, 70, [75, 300])               # more queries than a block holds
    compare(5, kind, dtype, 64, 1, 8, 64, 33, [40, 20, 500])


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_peaked_scores_and_scales_far_apart(kind, dtype):
    compare(1, kind, dtype, 128, 1, 4, 64, 2, [300], sharp=12.0)
    compare(2, kind, dtype, 64, 1, 2, 64, 1, [500], scale=0.0)
    compare(3, kind, dtype, 64, 1, 2, 64, 1, [90], scale=-0.3)


@pytest.mark.parametrize("kind", [E4M3, INT8])
def test_rows_whose_sizes_differ_by_powers_of_ten(kind):
    # tokens with tiny, huge and zero V rows in one softmax: the weights' sum must not lose the tiny ones' tokens
    rng = np.random.default_rng(0)
    d, size, length = 64, 32, 150
    pool, scales = rows8.make_cache(rng, 6, 1, size, d, kind)
    scales[:, 1] *= torch.from_numpy(10.0 ** rng.uniform(-9, 3, scales[:, 1].shape)).float().cuda()
    pool.view(torch.uint8)[1, 1, 0, 3:9] = 0
    scales[1, 1, 0, 3:9] = 1.0
    table = rows8.make_table(rng, 6, 1, 5, [5])
    q = torch.from_numpy(rng.standard_normal((1, 2, 3, d), dtype=np.float32)).to(F16).cuda()
    lengths = torch.tensor([length], dtype=torch.int32, device="cuda")
    got = binding.spec_paged_attention(q, pool, scales, table, lengths)
    want, bound = rows8.attention64(q, pool, scales, table, lengths, d ** -0.5)
    assert torch.all((got.cpu().double() - want).abs() <= bound)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_what_a_row_cannot_see_does_not_reach_it(kind, dtype):
    # the last two tokens are NaN / infinite: rows before them are as without them, rows behind are NaN; what lies past the length or on
    # pages of nobody is NaN too and reaches no one
    rng = np.random.default_rng(1)
    d, size, rows, group = 64, 32, 5, 2
    lengths = [69, 64, 3]
    used = [-(-l // size) for l in lengths]
    pool, scales = rows8.make_cache(rng, sum(used) + 2, 1, size, d, kind)
    table = rows8.make_table(rng, sum(used) + 2, 3, 3, used)
    q = torch.from_numpy(rng.standard_normal((3, rows, group, d), dtype=np.float32)).to(dtype).cuda()
    at = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    clean = binding.spec_paged_attention(q, pool, scales, table, at)
    bad = []
    for b, length in enumerate(lengths):
        for position in list(range(length - 2, length)) + list(range(length, used[b] * size)):
            bad.append((int(table[b, position // size]), position % size))
    unused = sorted(set(range(pool.shape[0])) - set(table.flatten().tolist()))
    nothing = float("nan")
    for i, (page, slot) in enumerate(bad):
        if kind in rows8.TOP:
            scales[page, :, :, slot] = nothing if i % 2 else float("inf")
            if kind == E4M3:
                pool.view(torch.uint8)[page, :, :, slot, 5] = 0x7f
        else:
            pool[page, :, :, slot, i % d] = nothing if i % 2 else float("inf")
    for page in unused:
        if kind in rows8.TOP:
            scales[page] = nothing
        else:
            pool[page] = nothing
    got = binding.spec_paged_attention(q, pool, scales, table, at)
    assert torch.equal(got[:2, :3], clean[:2, :3])
    assert not torch.isfinite(got[:2, 3:].float()).all(-1).any()
    assert torch.equal(got[2, :3], clean[2, :3])  # (positions -2, -1 see nothing, position 0 the first token)
    assert not got[2, :2].float().any()


def test_pages_outside_the_pool_hold_no_keys():
    rng = np.random.default_rng(2)
    pages, size = 6, 32
    table = torch.tensor([[0, 1, 2], [3, 17, 4], [-5, 5, pages], [-1, -1, -1]], dtype=torch.int32, device="cuda")
    for kind, dtype in KINDS:
        compare(4, kind, dtype, 64, 1, 2, size, 2, [90, 80, 96, 50], table=table, extra=pages - 11)
    del rng


def test_lengths_past_the_table_and_negative():
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(3)
    for kind, dtype in KINDS:
        pool, scales = rows8.make_cache(rng, 4, 2, 32, 64, kind)
        q = torch.from_numpy(rng.standard_normal((2, 3, 4, 64), dtype=np.float32)).to(dtype).cuda()
        for lengths in ([70, -4], [2 ** 31 - 1, 64], [-2 ** 31, 65]):
            at = torch.tensor(lengths, dtype=torch.int32, device="cuda")
            got = binding.spec_paged_attention(q, pool, scales, table, at)
            want, bound = rows8.attention64(q, pool, scales, table, at, 0.125)
            assert torch.all((got.cpu().double() - want).abs() <= bound)


@pytest.mark.parametrize("kind,dtype", [(E4M3, BF16), (BF16, BF16)])
def test_queries_inside_a_fused_projection(kind, dtype):
    rng = np.random.default_rng(4)
    pool, scales = rows8.make_cache(rng, 8, 2, 64, 128, kind)
    table = rows8.make_table(rng, 8, 2, 3, [3, 2])
    qkv = torch.from_numpy(rng.standard_normal((2, 4, 8 * 128), dtype=np.float32)).to(dtype).cuda()
    q = qkv[..., :512].view(2, 4, 4, 128)
    at = torch.tensor([170, 70], dtype=torch.int32, device="cuda")
    assert torch.equal(binding.spec_paged_attention(q, pool, scales, table, at), binding.spec_paged_attention(q.contiguous(), pool, scales, table, at))
    with pytest.raises(ValueError):
        binding.spec_paged_attention(q.transpose(1, 2), pool, scales, table, at)


def test_a_captured_call_follows_its_inputs():
    rng = np.random.default_rng(5)
    pool, scales = rows8.make_cache(rng, 40, 2, 32, 128, INT8)
    table = rows8.make_table(rng, 40, 2, 20, [20, 20])
    q = torch.from_numpy(rng.standard_normal((2, 3, 8, 128), dtype=np.float32)).to(BF16).cuda()
    at = torch.tensor([600, 5], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    work = torch.empty(binding.spec_paged_attention_workspace_bytes(2, 3, 8, 2, 128), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.spec_paged_attention(q, pool, scales, table, at, out=out, workspace=work)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            binding.spec_paged_attention(q, pool, scales, table, at, out=out, workspace=work)
    torch.cuda.current_stream().wait_stream(side)
    for lengths in ([600, 5], [1, 640], [0, 0], [333, 64]):
        at.copy_(torch.tensor(lengths, dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, binding.spec_paged_attention(q, pool, scales, table, at))


def test_a_short_workspace_is_refused():
    rng = np.random.default_rng(6)
    pool, scales = rows8.make_cache(rng, 2, 1, 32, 64, INT8)
    q = torch.zeros(1, 1, 1, 64, dtype=F16, device="cuda")
    table, at = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    with pytest.raises(binding.SpecError, match="workspace"):
        binding.spec_paged_attention(q, pool, scales, table, at, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
