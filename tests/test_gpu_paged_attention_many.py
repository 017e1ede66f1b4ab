"""Attention over paged rows with more than 32 queries to a KV head (prompts, passes of many heads) against the formula in 64 bits."""
import numpy as np
import pytest
import torch

import rows8
from paper_2211_17192_b200 import binding
from test_gpu_paged_attention import BF16, E4M3, F16, INT8, KINDS, compare

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows,n_kv,group", [(33, 2, 1), (9, 2, 8), (17, 1, 4), (128, 1, 1), (129, 1, 1), (11, 1, 12), (1, 1, 40)])
def test_types_and_head_layouts(kind, dtype, d, rows, n_kv, group):
    compare(rows, kind, dtype, d, n_kv, group, 64, rows, [200, 1, 65, 128, 63, 0, 300])


@pytest.mark.parametrize("kind,dtype", [(E4M3, BF16), (INT8, F16), (F16, F16), (BF16, BF16)])
@pytest.mark.parametrize("size", [32, 64, 128, 256])
@pytest.mark.parametrize("lengths", [[0], [1], [39, 40, 41], [0, 64, 0, 63], [1000], [2, 700, 0]])
def test_lengths_and_pages(kind, dtype, size, lengths):
    compare(size + len(lengths), kind, dtype, 128, 2, 2, size, 40, lengths)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_long_and_many(kind, dtype):
    compare(1, kind, dtype, 64, 1, 8, 256, 5, [20001])                       # one segment for all SMs
    compare(2, kind, dtype, 128, 1, 8, 32, 5, [7] * 200 + [0] * 20 + [130])  # more sequences than threads, segments of one tile
    compare(3, kind, dtype, 128, 3, 4, 64, 10, [2000, 10, 0, 777, 64])       # several segments to a CTA and several CTAs to a segment
    compare(4, kind, dtype, 64, 2, 1, 64, 300, [310, 300, 40])               # prompts: blocks that see few keys, and none


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_peaked_scores(kind, dtype):
    # the maximum moves in later tiles: what has been added up is scaled down
    compare(1, kind, dtype, 128, 1, 8, 64, 5, [700], sharp=12.0)
    compare(2, kind, dtype, 64, 1, 8, 64, 5, [500], scale=0.0)
    compare(3, kind, dtype, 64, 1, 8, 64, 5, [290], scale=-0.3)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_row_cannot_see_does_not_reach_it(kind, dtype, d):
    # the last two tokens are NaN / infinite: rows before them are as without them, rows behind are NaN; what lies past the length or on
    # pages of nobody is NaN too and reaches no one
    rng = np.random.default_rng(1)
    size, rows, group = 32, 5, 9
    lengths = [69, 64, 3, 200]
    used = [-(-l // size) for l in lengths]
    pool, scales = rows8.make_cache(rng, sum(used) + 2, 1, size, d, kind)
    table = rows8.make_table(rng, sum(used) + 2, 4, max(used), used)
    q = torch.from_numpy(rng.standard_normal((4, rows, group, d), dtype=np.float32)).to(dtype).cuda()
    at = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    want, bound = rows8.attention64(q, pool, scales, table, at, d ** -0.5)
    pool, scales = pool.clone(), None if scales is None else scales.clone()
    bad = [(int(table[b, p // size]), p % size) for b, length in enumerate(lengths) for p in range(length - 2, used[b] * size)]
    nothing = float("nan")
    for i, (page, slot) in enumerate(bad):
        if kind in rows8.TOP:
            if kind == INT8 or i % 3:
                scales[page, :, :, slot] = nothing if i % 2 else float("inf")
            if kind == E4M3:
                pool.view(torch.uint8)[page, :, :, slot, 5] = 0x7f
        else:
            pool[page, :, :, slot, i % d] = nothing if i % 2 else float("inf")
    for page in sorted(set(range(pool.shape[0])) - set(table.flatten().tolist())):
        (pool if scales is None else scales)[page] = nothing
    got = binding.spec_paged_attention(q, pool, scales, table, at).cpu().double()
    for b in (0, 1, 3):
        assert torch.all((got[b, :3] - want[b, :3]).abs() <= bound[b, :3])
        assert not torch.isfinite(got[b, 3:]).all(-1).any()
    assert not got[2, :2].any() and torch.all((got[2, 2] - want[2, 2]).abs() <= bound[2, 2])  # (positions -2, -1 see nothing, position 0 the first token)
    # a query that is no number is one for its row alone
    q[3, 1, 2, 7] = nothing
    pool, scales = rows8.make_cache(np.random.default_rng(1), sum(used) + 2, 1, size, d, kind)
    got = binding.spec_paged_attention(q, pool, scales, table, at).cpu().double()
    assert got[3, 1, 2].isnan().all()
    got[3, 1, 2] = want[3, 1, 2]
    assert torch.all((got - want).abs() <= bound)


def test_pages_outside_the_pool_hold_no_keys():
    pages, size = 6, 32
    table = torch.tensor([[0, 1, 2], [3, 17, 4], [-5, 5, pages], [-1, -1, -1]], dtype=torch.int32, device="cuda")
    for kind, dtype in KINDS:
        compare(4, kind, dtype, 64, 1, 2, size, 20, [90, 80, 96, 50], table=table, extra=pages - 11)


def test_lengths_past_the_table_and_negative():
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    rng = np.random.default_rng(3)
    for kind, dtype in KINDS:
        pool, scales = rows8.make_cache(rng, 4, 2, 32, 64, kind)
        q = torch.from_numpy(rng.standard_normal((2, 3, 24, 64), dtype=np.float32)).to(dtype).cuda()
        for lengths in ([70, -4], [2 ** 31 - 1, 64], [-2 ** 31, 65]):
            at = torch.tensor(lengths, dtype=torch.int32, device="cuda")
            got = binding.spec_paged_attention(q, pool, scales, table, at)
            want, bound = rows8.attention64(q, pool, scales, table, at, 0.125)
            assert torch.all((got.cpu().double() - want).abs() <= bound)


@pytest.mark.parametrize("kind,dtype", [(E4M3, BF16), (F16, F16), (BF16, BF16)])
def test_queries_with_a_stride_and_off_sixteen_bytes(kind, dtype):
    rng = np.random.default_rng(4)
    pool, scales = rows8.make_cache(rng, 8, 1, 64, 128, kind)
    table = rows8.make_table(rng, 8, 2, 3, [3, 2])
    qkv = torch.from_numpy(rng.standard_normal((2, 12, 516), dtype=np.float32)).to(dtype).cuda()
    at = torch.tensor([170, 70], dtype=torch.int32, device="cuda")
    for first in (0, 4):  # (rows 1032 bytes apart: on 8 bytes)
        q = qkv[..., first:first + 512].unflatten(-1, (4, 128))
        assert torch.equal(binding.spec_paged_attention(q, pool, scales, table, at), binding.spec_paged_attention(q.contiguous(), pool, scales, table, at))


def test_captured_calls_follow_their_inputs():
    # two calls in a graph with workspaces of their own, replayed over other lengths
    rng = np.random.default_rng(5)
    pool, scales = rows8.make_cache(rng, 80, 2, 32, 128, INT8)
    table = rows8.make_table(rng, 80, 2, 40, [40, 40])
    qs = [torch.from_numpy(rng.standard_normal((2, rows, 16, 128), dtype=np.float32)).to(BF16).cuda() for rows in (7, 100)]
    at = torch.tensor([600, 5], dtype=torch.int32, device="cuda")
    outs = [torch.empty_like(q) for q in qs]
    works = [torch.empty(binding.spec_paged_attention_workspace_bytes(2, q.shape[1], 16, 2, 128), dtype=torch.uint8, device="cuda") for q in qs]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        for q, out, work in zip(qs, outs, works):
            binding.spec_paged_attention(q, pool, scales, table, at, out=out, workspace=work)
    for lengths in ([600, 5], [1, 1280], [0, 0], [333, 64], [1280, 1279]):
        at.copy_(torch.tensor(lengths, dtype=torch.int32))
        for out in outs:
            out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for q, out in zip(qs, outs):
            assert torch.equal(out, binding.spec_paged_attention(q, pool, scales, table, at))


@pytest.mark.parametrize("kind,dtype", [(INT8, BF16), (F16, F16)])
@pytest.mark.parametrize("rows", [2, 12])
def test_pages_past_32_bits_of_the_pool(kind, dtype, rows):
    rng = np.random.default_rng(6)
    heads, size, d = 2, 256, 128
    pages = 2 ** 32 // (2 * heads * size * d) + 5  # elements: past 2^32
    small, small_scales = rows8.make_cache(rng, 6, heads, size, d, kind)
    pool = torch.zeros(pages, 2, heads, size, d, dtype=kind, device="cuda")
    scales = torch.ones(pool.shape[:4], device="cuda") if kind in rows8.TOP else None
    pool.view(torch.uint8)[pages - 6:] = small.view(torch.uint8)
    if scales is not None:
        scales[pages - 6:] = small_scales
    table = rows8.make_table(rng, 6, 2, 3, [3, 2])
    q = torch.from_numpy(rng.standard_normal((2, rows, 8, d), dtype=np.float32)).to(dtype).cuda()
    at = torch.tensor([700, 300], dtype=torch.int32, device="cuda")
    far = torch.where(table >= 0, table + pages - 6, table)
    assert torch.equal(binding.spec_paged_attention(q, pool, scales, far, at), binding.spec_paged_attention(q, small, small_scales, table, at))


def test_calls_on_two_streams_at_once():
    # attention and a linear layer, both with tensor memory of an SM, beside each other
    rng = np.random.default_rng(7)
    pool, scales = rows8.make_cache(rng, 120, 2, 32, 128, E4M3)
    table = rows8.make_table(rng, 120, 4, 30, [30] * 4)
    q = torch.from_numpy(rng.standard_normal((4, 100, 16, 128), dtype=np.float32)).to(BF16).cuda()
    at = torch.tensor([960, 100, 333, 901], dtype=torch.int32, device="cuda")
    x, w = (binding.spec_quantize_fp8(torch.from_numpy(rng.standard_normal((n, 1024), dtype=np.float32)).cuda()) for n in (200, 2000))
    want = [binding.spec_paged_attention(q, pool, scales, table, at), binding.spec_linear_fp8(*x, *w), binding.spec_linear_fp8(x[0][:5], x[1][:5], *w)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [[] for _ in streams]
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(binding.spec_paged_attention(q, pool, scales, table, at) if i == 0 else
                              binding.spec_linear_fp8(*x, *w) if i == 1 else binding.spec_linear_fp8(x[0][:5], x[1][:5], *w))
    torch.cuda.synchronize()
    for results, expected in zip(got, want):
        for result in results:
            assert torch.equal(result, expected)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("slow", [0, 3])
def test_a_warp_that_is_behind_the_others(kind, dtype, slow):
    # 32 neighbouring queries (a warp's) meet a higher score in every tile, so that all they have added up is scaled down each time; the
    # others' largest is in the first tile.  Segments of two tiles and more, many to a CTA: each one's end and the next one's start.
    rng = np.random.default_rng(8)
    batch, heads, d, size, rows = 40, 8, 128, 64, 128
    lengths = [128 + 64 * (b % 5) for b in range(batch)]
    used = [-(-l // size) for l in lengths]
    x = torch.from_numpy(rng.standard_normal((sum(used), 2, heads, size, d), dtype=np.float32))
    table = rows8.make_table(rng, sum(used), batch, max(used), used)
    x[:, 0, :, :, 0] = 0
    for b in range(batch):
        for j in range(used[b]):
            x[int(table[b, j]), 0, :, :, 0] = 4.0 * j
    scales = None
    if kind in rows8.TOP:
        scales = rows8.scale64(x.double(), kind).float()
        z = x * (1.0 / scales)[..., None]
        x = z.clamp(-448, 448) if kind == E4M3 else z.round()
        scales = scales.cuda()
    pool = x.to(kind).cuda()
    q = torch.from_numpy(rng.standard_normal((batch, rows, heads, d), dtype=np.float32)) * 0.1
    q[..., 0] = -8.0
    q[:, 32 * slow:32 * slow + 32, :, 0] = 8.0
    q = q.to(dtype).cuda()
    at = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got = binding.spec_paged_attention(q, pool, scales, table, at, scale=1.0)
    some = torch.tensor([0, 1, 2, 18, 39])
    want, bound = rows8.attention64(q[some], pool, scales, table[some.cuda()], at[some.cuda()], 1.0)
    assert torch.all((got[some].cpu().double() - want).abs() <= bound)
    for _ in range(20):
        assert torch.equal(binding.spec_paged_attention(q, pool, scales, table, at, scale=1.0), got)
    assert binding.spec_device_error() == 0
