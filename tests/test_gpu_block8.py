"""A decoder block made of the 8-bit operators, as a caller with a model of its own runs it: ragged prompts into a paged cache, a
verification pass of gamma + 1 rows, a ragged roll-back, the pass of the next iteration.  Every operator's output is checked
against its formula in 64 bits on the inputs that it was given."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import rows8
from paper_2211_17192_b200 import binding
from test_gpu_rows8 import NORM_REL, act64, rope_table, rotated64

pytestmark = pytest.mark.gpu
E4M3, INT8, F32, BF16, F16 = torch.float8_e4m3fn, torch.int8, torch.float32, torch.bfloat16, torch.float16
D_MODEL, HEADS, KV_HEADS, D_HEAD, D_FF, PAGE, WIDTH = 512, 8, 2, 64, 1088, 32, 8


class Block:
    def __init__(self, seed, kind, batch):
        rng = np.random.default_rng(seed)

        def weight(n, k):
            return binding.spec_quantize_fp8(torch.from_numpy(rng.standard_normal((n, k), dtype=np.float32) / np.float32(np.sqrt(k))).cuda())

        qkv = (HEADS + 2 * KV_HEADS) * D_HEAD
        self.w = {"qkv": weight(qkv, D_MODEL), "o": weight(D_MODEL, HEADS * D_HEAD), "in": weight(2 * D_FF, D_MODEL), "out": weight(D_MODEL, D_FF)}
        self.gain = [(1 + 0.1 * torch.from_numpy(rng.standard_normal(D_MODEL, dtype=np.float32))).cuda() for _ in range(2)]
        self.kind, self.batch = kind, batch
        pages = batch * WIDTH + 3
        self.pool = torch.full((pages, 2, KV_HEADS, PAGE, D_HEAD), 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) if kind == E4M3 else \
            torch.full((pages, 2, KV_HEADS, PAGE, D_HEAD), 99 if kind == INT8 else float("nan"), dtype=kind, device="cuda")
        self.scales = torch.full(self.pool.shape[:4], float("nan"), device="cuda") if kind in rows8.TOP else None
        self.table = rows8.make_table(rng, pages, batch, WIDTH, [WIDTH] * batch)
        self.rope = rope_table(PAGE * WIDTH, D_HEAD).cuda()

    def __call__(self, h, start, counts, check=True):
        """h [B, rows, d] the residual stream (updated in place), start [B] positions, counts [B] rows that are no padding."""
        batch, rows, _ = h.shape
        flat = h.view(batch * rows, D_MODEL)
        before = flat.clone()
        codes, scales, _ = binding.spec_norm_fp8(flat, self.gain[0])
        qkv = binding.spec_linear_fp8(codes, scales, *self.w["qkv"], dtype=BF16 if self.kind != F16 else F16)
        q, k, v = (t.view(batch, rows, -1, D_HEAD) for t in qkv.view(batch, rows, -1).split([HEADS * D_HEAD, KV_HEADS * D_HEAD, KV_HEADS * D_HEAD], -1))
        rotated = binding.spec_kv_append(k, v, self.pool, self.scales, self.table, start, counts=counts, rope=self.rope, q=q)
        # padding rows stand behind the real ones: with the length of all rows they see more keys, and nobody reads them
        lengths = start + rows
        attended = binding.spec_paged_attention(rotated, self.pool, self.scales, self.table, lengths)
        a_codes, a_scales = binding.spec_quantize_fp8(attended.view(batch * rows, -1))
        binding.spec_linear_fp8(a_codes, a_scales, *self.w["o"], residual=flat, y=flat)
        middle = flat.clone()
        m_codes, m_scales, _ = binding.spec_norm_fp8(flat, self.gain[1])
        act = binding.spec_linear_fp8(m_codes, m_scales, *self.w["in"], act="swiglu", dtype=BF16)
        f_codes, f_scales = binding.spec_quantize_fp8(act)
        binding.spec_linear_fp8(f_codes, f_scales, *self.w["out"], residual=flat, y=flat)
        if check:
            live = torch.cat([torch.arange(rows) < int(c) for c in counts])
            self.norm(before, self.gain[0], codes, scales)
            self.linear(codes, scales, "qkv", "none", None, qkv)
            for b in range(batch):
                for i in range(int(counts[b])):
                    self.rows(q[b, i], k[b, i], v[b, i], int(start[b]) + i, b, rotated[b, i])
            want, bound = rows8.attention64(rotated, self.pool, self.scales, self.table, lengths, D_HEAD ** -0.5)
            err = (attended.cpu().double() - want).abs().view(batch * rows, -1)[live]
            assert torch.all(err <= bound.view(batch * rows, -1)[live])
            rows8.check_codes(a_codes[live.cuda()], a_scales[live.cuda()], attended.view(batch * rows, -1)[live.cuda()], E4M3)
            self.linear(a_codes, a_scales, "o", "none", before, middle, live)
            self.norm(middle, self.gain[1], m_codes, m_scales, live)
            self.linear(m_codes, m_scales, "in", "swiglu", None, act, live)
            rows8.check_codes(f_codes[live.cuda()], f_scales[live.cuda()], act[live.cuda()], E4M3)
            self.linear(f_codes, f_scales, "out", "none", middle, flat, live)
        return h

    @staticmethod
    def norm(x, gain, codes, scales, live=slice(None)):
        w = x.double().cpu()
        y = w * gain.double().cpu() / torch.sqrt((w * w).mean(-1, keepdim=True) + 1e-6)
        rows8.check_codes(codes.cpu()[live], scales.cpu()[live], y[live], E4M3, NORM_REL)

    def linear(self, codes, scales, name, act, residual, y, live=slice(None)):
        wc, ws = self.w[name]
        x, w = codes.float().double() * scales.double()[:, None], wc.float().double() * ws.double()[:, None]
        z, size = x @ w.T, x.abs() @ w.abs().T
        off = size * (2 * (x.shape[1] / 32) + 16) * 2.0 ** -23  # (as derived beside the operator's own test)
        n = y.shape[1]
        want = act64(z, act, n)
        bound = off if act == "none" else (off[:, :n] * 1.13 + z[:, :n].abs() * 2.0 ** -20) * (z[:, n:].abs() + off[:, n:]) + z[:, :n].abs() * off[:, n:]
        if residual is not None:
            want = want + residual.double()
            bound = bound + want.abs() * 2.0 ** -24
        bound = bound + want.abs() * rows8.HALF_STEP[y.dtype] * 1.01 + 2.0 ** -25
        assert torch.all(((y.double() - want).abs() <= bound).cpu()[live])

    def rows(self, q, k, v, position, b, rotated):
        page, slot = int(self.table[b, position // PAGE]), position % PAGE
        at = torch.tensor(position)
        want = rotated64(q.double().cpu(), at, self.rope.cpu())
        assert torch.all((rotated.cpu().double() - want).abs() <= want.abs() * rows8.HALF_STEP[q.dtype] * 1.01 + q.abs().max().double().cpu() * 2.0 ** -21)
        for which, x in ((0, rotated64(k.double().cpu(), at, self.rope.cpu())), (1, v.double().cpu())):
            got = rows8.dequantised(self.pool[page, which, :, slot], None if self.scales is None else self.scales[page, which, :, slot])
            if self.kind in rows8.TOP:
                s = self.scales[page, which, :, slot].double().cpu()[:, None]
                z = x / s
                slack = x.abs().amax(-1, keepdim=True) / s * 2.0 ** -20  # (a rotation in fp32, the scale's two roundings, a reciprocal and a product)
                assert torch.all((got / s - z).abs() <= rows8.half_step_of_code(z.abs() + slack, self.kind) + slack)
            else:
                assert torch.all((got - x).abs() <= x.abs() * rows8.HALF_STEP[self.kind] * 1.01 + x.abs().amax() * 2.0 ** -20)


def stream(seed, batch, rows):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal((batch, rows, D_MODEL), dtype=np.float32)).cuda()


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kind", [E4M3, INT8, BF16, F16])
def test_prompt_verification_rollback(kind):
    block = Block(1, kind, 3)
    prompts = [40, 1, 97]
    # rows of a padded prompt beyond its count are not in the cache; the pass that needs them as keys is the next one
    block(stream(2, 3, 97), ints(0, 0, 0), ints(*prompts), check=False)
    lengths = ints(*prompts)
    block(stream(3, 3, 5), lengths, ints(5, 5, 5))                     # gamma = 4
    accepted = ints(2, 0, 4)
    lengths = lengths + accepted + 1                                   # each sequence keeps its accepted guesses and one token more
    second = block(stream(4, 3, 5), lengths - 1, ints(5, 5, 5))        # (that token's row is fed here)
    # the same from a cache that never saw the rejected rows
    fresh = Block(1, kind, 3)
    fresh(stream(2, 3, 97), ints(0, 0, 0), ints(*prompts), check=False)
    first = stream(3, 3, 5)
    fresh(first, ints(*prompts), accepted, check=False)
    again = fresh(stream(4, 3, 5), lengths - 1, ints(5, 5, 5), check=False)
    assert torch.equal(second, again)
    assert binding.spec_device_error() == 0


def test_a_captured_block_is_the_same():
    block, start, counts = Block(5, INT8, 2), ints(0, 0), ints(3, 3)
    h = stream(6, 2, 3)
    source = h.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(h, start, counts, check=False)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            h.copy_(source)
            block(h, start, counts, check=False)
    torch.cuda.synchronize()
    eager = Block(5, INT8, 2)
    for step in range(4):
        source.copy_(stream(10 + step, 2, 3))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, eager(source.clone(), start, counts, check=False))
        start += 3


@pytest.mark.parametrize("batch,rows,length", [(1, 3, 40), (9, 7, 64), (64, 64, 64), (3, 5, 65)])
def test_what_follows_attention_waits_for_it(batch, rows, length):
    # contexts of one tile: no CTA has anything to join, and the kernel behind attention reads what it wrote all the same
    rng = np.random.default_rng(batch)
    pool, scales = rows8.make_cache(rng, batch * 2, 2, 64, 128, INT8)
    table = rows8.make_table(rng, batch * 2, batch, 2, [2] * batch)
    lengths = torch.full((batch,), length, dtype=torch.int32, device="cuda")
    qs = [torch.from_numpy(rng.standard_normal((batch, rows, 8, 128), dtype=np.float32)).to(BF16).cuda() for _ in range(2)]
    out = torch.zeros_like(qs[0])
    work = torch.empty(binding.spec_paged_attention_workspace_bytes(batch, rows, 8, 2, 128), dtype=torch.uint8, device="cuda")
    want = []
    for q in qs:
        binding.spec_paged_attention(q, pool, scales, table, lengths, out=out, workspace=work)
        torch.cuda.synchronize()
        want.append([t.clone() for t in binding.spec_quantize_fp8(out.view(batch * rows, -1))])
        torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    taken = [[torch.empty_like(t) for t in want[0]] for _ in range(8)]
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        for i, (c, s) in enumerate(taken):
            binding.spec_paged_attention(qs[i % 2], pool, scales, table, lengths, out=out, workspace=work)
            binding.spec_quantize_fp8(out.view(batch * rows, -1), codes=c, scales=s)
    for _ in range(5):
        graph.replay()
        torch.cuda.synchronize()
        for i, (c, s) in enumerate(taken):
            assert torch.equal(c.view(torch.uint8), want[i % 2][0].view(torch.uint8)) and torch.equal(s, want[i % 2][1])


def test_a_lone_row_whose_stride_means_nothing():
    # [heads, 1, d] turned round: one row, whose stride torch gives as d
    q, k = (torch.randn(n, 1, 64, device="cuda").to(BF16).transpose(0, 1)[None] for n in (4, 2))
    assert k.stride(0) < 2 * 64
    results = []
    for x, y in ((q, k), (q.clone(memory_format=torch.contiguous_format), k.clone(memory_format=torch.contiguous_format))):
        pool, table, start = torch.zeros(2, 2, 2, 32, 64, dtype=BF16, device="cuda"), torch.zeros(1, 2, dtype=torch.int32, device="cuda"), ints(5)
        turned = binding.spec_kv_append(y, y, pool, None, table, start, rope=rope_table(64, 64).cuda(), q=x, q_out=torch.empty(1, 1, 4, 64, dtype=BF16, device="cuda"))
        work = torch.empty(binding.spec_paged_attention_workspace_bytes(1, 1, 4, 2, 64), dtype=torch.uint8, device="cuda")
        out = binding.spec_paged_attention(x, pool, None, table, start + 1, out=torch.empty(1, 1, 4, 64, dtype=BF16, device="cuda"), workspace=work)
        results.append((pool, turned, out))
    for a, b in zip(*results):
        assert torch.equal(a, b)


def test_a_position_past_the_page_table_has_no_page():
    # K and V are left out, q is turned as everywhere
    rope = rope_table(80, 64)
    k, q = torch.randn(1, 4, 1, 64, device="cuda"), torch.randn(1, 4, 2, 64, device="cuda")
    pool = torch.zeros(2, 2, 1, 32, 64, dtype=F16, device="cuda")
    out = binding.spec_kv_append(k, k, pool, None, ints(1)[None], ints(30), rope=rope.cuda(), q=q)
    want = rotated64(q[0].cpu().double(), torch.arange(30, 34), rope)
    assert torch.all((out[0].cpu().double() - want).abs() <= 2.0 ** -21 * (q[0].cpu().double().abs() + q[0].cpu().double().abs().roll(32, -1)))
    assert pool[1, :, :, 30:].all() and not pool[1, :, :, :30].any() and not pool[0].any()
    # (positions 32 and 33: zeros come back)
    k_out, _ = binding.spec_kv_read(pool, None, ints(1)[None], ints(30), 4)
    assert k_out[0, :2].all() and not k_out[0, 2:].any()


def test_calls_without_rows_do_nothing():
    e = lambda *shape, dtype=F32: torch.empty(shape, dtype=dtype, device="cuda")
    codes, scales = binding.spec_quantize_fp8(e(0, 64))
    assert codes.shape == (0, 64) and scales.shape == (0,)
    binding.spec_norm_fp8(e(0, 64), e(64), residual=e(0, 64))
    w, ws = binding.spec_quantize_fp8(torch.ones(32, 64, device="cuda"))
    assert binding.spec_linear_fp8(codes, scales, w, ws).shape == (0, 32)
    pool, table = torch.zeros(2, 2, 1, 32, 64, dtype=INT8, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    s = torch.ones(2, 2, 1, 32, device="cuda")
    binding.spec_kv_append(e(2, 0, 1, 64), e(2, 0, 1, 64), pool, s, table, ints(0, 0))
    assert binding.spec_kv_read(pool, s, table, ints(0, 0), 0)[0].shape == (2, 0, 1, 64)
    assert binding.spec_paged_attention(e(2, 0, 1, 64, dtype=F16), pool, s, table, ints(1, 1)).shape == (2, 0, 1, 64)
    assert binding.spec_paged_attention(e(0, 3, 1, 64, dtype=F16), pool, s, table[:0], ints()).shape == (0, 3, 1, 64)


FIRST = """
import torch
from paper_2211_17192_b200 import binding
B = torch.bfloat16
x, gain = torch.randn(300, 2048, device="cuda").to(B), torch.ones(2048, device="cuda")
w = torch.randn(512, 2048, device="cuda").to(torch.float8_e4m3fn)
codes, scales = torch.empty(300, 2048, dtype=torch.float8_e4m3fn, device="cuda"), torch.ones(300, device="cuda")
ws, y, few = torch.ones(512, device="cuda"), torch.empty(300, 512, device="cuda"), torch.empty(3, 512, device="cuda")
pool = torch.zeros(4, 2, 2, 32, 128, dtype=torch.int8, device="cuda")
ps, table, start = torch.ones(4, 2, 2, 32, device="cuda"), torch.arange(4, dtype=torch.int32, device="cuda").view(1, 4), torch.zeros(1, dtype=torch.int32, device="cuda")
k, out = torch.randn(1, 100, 2, 128, device="cuda").to(B), torch.empty(1, 5, 8, 128, dtype=B, device="cuda")
q, lengths = torch.randn(1, 5, 8, 128, device="cuda").to(B), torch.full((1,), 100, dtype=torch.int32, device="cuda")
ko, vo = torch.empty(1, 100, 2, 128, device="cuda"), torch.empty(1, 100, 2, 128, device="cuda")
work = torch.empty(binding.spec_paged_attention_workspace_bytes(1, 5, 8, 2, 128), dtype=torch.uint8, device="cuda")
def step():
    binding.spec_norm_fp8(x, gain, codes=codes, scales=scales)
    binding.spec_quantize_fp8(x[:2], codes=codes[:2], scales=scales[:2])
    binding.spec_linear_fp8(codes, scales, w, ws, y=y)
    binding.spec_linear_fp8(codes[:3], scales[:3], w, ws, y=few)
    binding.spec_kv_append(k, k, pool, ps, table, start)
    binding.spec_kv_read(pool, ps, table, start, 100, k=ko, v=vo)
    binding.spec_paged_attention(q, pool, ps, table, lengths, out=out, workspace=work)
side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph, stream=side):
    step()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (codes.float(), scales, y, few, ko, out)]
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (codes.float(), scales, y, few, ko, out))) and torch.isfinite(out.float()).all()
print("captured first")
"""


def test_a_first_call_may_be_a_captured_one():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST], cwd=root, capture_output=True, text=True, timeout=180)
    assert done.returncode == 0 and "captured first" in done.stdout, done.stderr[-2000:]
