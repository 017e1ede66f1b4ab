"""Norm, quantisation, linear layer and cache rows in 8 bits against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

import rows8
from paper_2211_17192_b200 import binding

pytestmark = pytest.mark.gpu
E4M3, INT8, F32, BF16, F16 = torch.float8_e4m3fn, torch.int8, torch.float32, torch.bfloat16, torch.float16


def normal(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape, dtype=np.float32))


@pytest.mark.parametrize("rows,d", [(1, 1), (1, 768), (3, 7), (5, 252), (2, 33), (300, 128), (7, 4096), (2, 4104), (3, 11008), (2, 11003), (2, 16384), (1, 32768), (900, 4096), (500, 1544), (1000, 11008), (450, 16384)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_quantize(rows, d, dtype):
    x = (normal(rows * 100003 + d, rows, d) * 3).to(dtype)
    x[0] *= 0 if rows > 2 else 1  # a row of zeros has scale 1
    codes, scales = binding.spec_quantize_fp8(x.cuda())
    rows8.check_codes(codes, scales, x, E4M3)
    if rows > 2:
        assert float(scales[0]) == 1.0 and not codes[0].float().any()


def test_quantize_unaligned_and_extreme_rows():
    x = normal(5, 40, 64)
    x[1] *= 1e30
    x[2] *= 1e-30
    x[3] = 0
    x[3, 5] = 1e-38
    x[4, 7] = float("nan")
    x[5, 9] = float("inf")
    for shift in (0, 1, 2, 3):  # a start that no wide access is aligned to
        buf = torch.zeros(40 * 64 + 8, device="cuda")
        buf[shift:shift + 40 * 64] = x.reshape(-1).cuda()
        codes, scales = binding.spec_quantize_fp8(buf[shift:shift + 40 * 64].view(40, 64))
        fine = [r for r in range(40) if r not in (4, 5)]
        rows8.check_codes(codes[fine], scales[fine], x[fine], E4M3)
        value = codes.float() * scales[:, None]
        assert not torch.isfinite(scales[4:6]).any() and torch.isnan(value[4]).all() and not torch.isfinite(value[5]).any()


# The sum of squares: a thread adds up to 32 of them, then five and five steps across lanes and warps: 42 roundings of 2^-24 at most,
# half of that in the square root, and a few roundings of the factor and of the products.
NORM_REL = (42 / 2 + 6) * 2.0 ** -24


@pytest.mark.parametrize("rows,d", [(1, 1), (1, 768), (4, 7), (2, 250), (130, 256), (3, 4096), (2, 8200), (2, 11008), (1, 32768), (900, 4096), (500, 1544), (450, 11008)])
@pytest.mark.parametrize("dtype,h_dtype", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16)])
def test_norm(rows, d, dtype, h_dtype):
    x, gain = (normal(d, rows, d) * 2).to(dtype), 1 + 0.1 * normal(d + 1, d)
    residual = normal(d + 2, rows, d).to(h_dtype)
    residual[0, 0] = 40
    codes, scales, h = binding.spec_norm_fp8(x.cuda(), gain.cuda(), 1e-6, residual=residual.cuda())
    want = (x.float() + residual.float()).to(h_dtype)
    assert torch.equal(h.cpu(), want)
    w = want.double()
    y = w * gain.double() / torch.sqrt((w * w).mean(-1, keepdim=True) + 1e-6)
    rows8.check_codes(codes, scales, y, E4M3, NORM_REL)
    # in place, and without the sum
    r = residual.cuda()
    again = binding.spec_norm_fp8(x.cuda(), gain.cuda(), 1e-6, residual=r, h=r)
    assert again[2] is r and torch.equal(r.cpu(), want)
    assert torch.equal(again[0].view(torch.uint8), codes.view(torch.uint8)) and torch.equal(again[1], scales)
    alone = binding.spec_norm_fp8(x.cuda(), gain.cuda(), 1e-6)
    assert alone[2] is None
    w = x.double()
    rows8.check_codes(alone[0], alone[1], w * gain.double() / torch.sqrt((w * w).mean(-1, keepdim=True) + 1e-6), E4M3, NORM_REL)


def test_norm_of_zeros_and_of_no_numbers():
    x = torch.zeros(3, 96, device="cuda")
    x[1, 3] = float("nan")
    codes, scales, _ = binding.spec_norm_fp8(x, torch.ones(96, device="cuda"), 1e-6)
    assert float(scales[0]) == 1.0 and not codes[0].float().any() and float(scales[2]) == 1.0
    assert torch.isnan(scales[1]) and torch.isnan(codes[1].float()).all()


ACTS = ["none", "gelu", "silu", "gated_gelu", "swiglu"]


def act64(z, act, n_out):
    g = z[:, :n_out]
    if act in ("gelu", "gated_gelu"):
        g = torch.nn.functional.gelu(g, approximate="tanh")
    elif act in ("silu", "swiglu"):
        g = g * torch.sigmoid(g)
    return g * z[:, n_out:] if act in ("gated_gelu", "swiglu") else g


def linear_case(seed, rows, k, n_out, act, bias, residual, dtype):
    n_w = 2 * n_out if act in ("gated_gelu", "swiglu") else n_out
    x, w = normal(seed, rows, k), normal(seed + 1, n_w, k) / np.sqrt(k)
    (xc, xs), (wc, ws) = binding.spec_quantize_fp8(x.cuda()), binding.spec_quantize_fp8(w.cuda())
    b = normal(seed + 2, n_w) if bias else None
    r = normal(seed + 3, rows, n_out).to(dtype) if residual else None
    y = binding.spec_linear_fp8(xc, xs, wc, ws, bias=None if b is None else b.cuda(), act=act, residual=None if r is None else r.cuda(), dtype=dtype)
    x64, w64 = xc.float().double() * xs.double()[:, None], wc.float().double() * ws.double()[:, None]
    z, size = x64 @ w64.T, x64.abs() @ w64.abs().T
    # An fp32 sum of exact products, 32 of them to an MMA: k / 32 additions, each off by one unit of the last place of what has been
    # added up so far (2^-23, also where the hardware truncates), the alignment of the 32 within an MMA as much again; clusters add eight
    # sums; a few roundings of the scales.
    off = size * (2 * (k / 32) + 16) * 2.0 ** -23
    if b is not None:
        z, off = z + b.cuda().double(), off + b.cuda().double().abs() * 2.0 ** -23
    want = act64(z, act, n_out)
    # |act'| <= 1.13 for both functions; tanhf and expf are within 2^-21 of theirs, and |act(z)| <= |z|
    first, second = off[:, :n_out] * 1.13 + z[:, :n_out].abs() * 2.0 ** -20, off[:, n_out:]
    if act in ("gated_gelu", "swiglu"):
        bound = first * z[:, n_out:].abs() + z[:, :n_out].abs() * second + first * second
    else:
        bound = first
    if r is not None:
        want = want + r.cuda().double()
        bound = bound + want.abs() * 2.0 ** -24
    bound = bound + want.abs() * rows8.HALF_STEP[dtype] * 1.01 + 2.0 ** -25
    err = (y.double() - want).abs()
    assert torch.all(err <= bound), float((err - bound).max())
    return xc, xs, wc, ws, b, r, y


@pytest.mark.parametrize("rows,k,n_out", [(1, 16, 1), (1, 768, 2304), (3, 4096, 512), (16, 112, 96), (17, 144, 130), (5, 2048, 64), (64, 1024, 1000), (112, 400, 257),
                                          (128, 256, 128), (129, 256, 300), (200, 1040, 512), (300, 512, 1040), (1000, 640, 384), (2049, 128, 272), (777, 2064, 1500)])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_linear_sizes(rows, k, n_out, act):
    linear_case(rows + k + n_out, rows, k, n_out, act, False, False, F32)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows", [2, 150, 600])
def test_linear_epilogues(act, dtype, rows):
    for bias in (False, True):
        for residual in (False, True):
            linear_case(rows, rows, 320, 200, act, bias, residual, dtype)
    assert binding.spec_device_error() == 0


@pytest.mark.parametrize("rows", [3, 96, 500])
def test_linear_into_its_residual_and_again(rows):
    xc, xs, wc, ws, b, r, y = linear_case(9, rows, 1024, 384, "none", True, True, F32)
    stream = r.cuda()
    out = binding.spec_linear_fp8(xc, xs, wc, ws, bias=b.cuda(), residual=stream, y=stream)
    assert out is stream and torch.equal(stream, y)
    for _ in range(3):
        assert torch.equal(binding.spec_linear_fp8(xc, xs, wc, ws, bias=b.cuda(), residual=r.cuda()), y)
    # a row's result does not hang on what the other rows hold
    xc2 = xc.clone()
    xc2.view(torch.uint8)[1:] = 0x3a
    assert torch.equal(binding.spec_linear_fp8(xc2, xs, wc, ws, bias=b.cuda(), residual=r.cuda())[0], y[0])


def rotated64(x, positions, table):
    """x [.., heads, d] at `positions` [..]."""
    half = x.shape[-1] // 2
    cs = table.double()[positions]
    c, s = cs[..., None, :, 0], cs[..., None, :, 1]
    a, b = x[..., :half], x[..., half:]
    return torch.cat((a * c - b * s, b * c + a * s), -1)


def rope_table(positions, d):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    return torch.stack((angle.cos(), angle.sin()), -1).float()


@pytest.mark.parametrize("kind", [E4M3, INT8, F16, BF16])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("d,heads,n_kv,size,batch,rows", [(128, 32, 8, 64, 3, 7), (64, 3, 3, 32, 1, 1), (64, 4, 1, 256, 5, 40), (128, 2, 2, 128, 2, 300)])
@pytest.mark.parametrize("fused", [True, False])
def test_append_and_read(kind, dtype, d, heads, n_kv, size, batch, rows, fused):
    rng = np.random.default_rng(rows)
    start = torch.tensor([0, 45, size - 1, 600, 31][:batch], dtype=torch.int32)
    counts = torch.tensor([max(0, rows - 2 * b) for b in range(batch)], dtype=torch.int32)
    width = -(-int((start + rows).max()) // size)
    pages = batch * width + 2
    table = rows8.make_table(rng, pages, batch, width, [width] * batch)
    if batch > 1:
        table[1, 0] = pages  # past the pool: positions before `size` of sequence 1 have no page
    pool = torch.full((pages, 2, n_kv, size, d), 3, dtype=torch.uint8 if kind in rows8.TOP else kind, device="cuda").view(kind)
    scales = torch.full(pool.shape[:4], 7.0, device="cuda") if kind in rows8.TOP else None
    before = pool.clone()
    if fused:
        qkv = (normal(7, batch, rows, (heads + 2 * n_kv) * d)).to(dtype).cuda()
        q, k, v = (t.view(batch, rows, -1, d) for t in qkv.split([heads * d, n_kv * d, n_kv * d], -1))
    else:
        q, k, v = (normal(8 + i, batch, rows, n, d).to(dtype).cuda() for i, n in enumerate((heads, n_kv, n_kv)))
    rope = rope_table(600 + rows - 3, d)  # (the last three positions of the fourth sequence are past the table)
    q_out = torch.full((batch, rows, heads, d), 9.0, dtype=dtype, device="cuda")
    assert binding.spec_kv_append(k, v, pool, scales, table, start.cuda(), counts=counts.cuda(), rope=rope.cuda(), q=q, q_out=q_out) is q_out
    k_out, v_out = binding.spec_kv_read(pool, scales, table, start.cuda(), rows, counts=counts.cuda())
    got, touched = rows8.dequantised(pool, scales), torch.zeros(pool.shape[:4], dtype=torch.bool)
    k, v, q = k.cpu(), v.cpu(), q.cpu()
    tab = table.cpu()
    for b in range(batch):
        n = int(counts[b])
        for i in range(rows):
            position = int(start[b]) + i
            live = i < n and position < rope.shape[0]
            if not live:
                assert torch.all(q_out[b, i].float() == 9.0)
            page = int(tab[b, position // size])
            if not live or not 0 <= page < pages:
                # an unwritten place may still be read where it has a page: what lay there before
                if not (i < n and 0 <= page < pages):
                    assert not k_out[b, i].any() and not v_out[b, i].any()
            if live:
                at = torch.tensor(position)
                want_q = rotated64(q[b, i].double(), at, rope)
                size_q = rotated64(q[b, i].double().abs(), at, rope.abs()).abs() + q[b, i].double().abs().roll(d // 2, -1)
                err = (q_out[b, i].cpu().double() - want_q).abs()
                assert torch.all(err <= want_q.abs() * rows8.HALF_STEP[dtype] * 1.01 + size_q * 2.0 ** -22 + 2.0 ** -25)
            if live and 0 <= page < pages:
                slot = position % size
                touched[page, :, :, slot] = True
                for which, x in ((0, rotated64(k[b, i].double(), torch.tensor(position), rope)), (1, v[b, i].double())):
                    value = got[page, which, :, slot]
                    if kind in rows8.TOP:
                        codes, s = pool[page, which, :, slot].cpu(), scales[page, which, :, slot].cpu()
                        # K: two products and a sum in fp32, each off by 2^-24 of |x| + |y| <= sqrt(2) of the pair: 3 * 2^-24 of the row's largest, at most
                        # twice that where the rotation has made it smaller; the same absolute error counts against small elements
                        y = x
                        top = y.abs().amax(-1, keepdim=True)
                        want = rows8.scale64(y, kind)
                        assert torch.all((s.double() - want).abs() <= want * 2.0 ** -20)
                        z = y / s.double()[:, None]
                        slack = z.abs() * 2.0 ** -21 + (top / s.double()[:, None]) * (2.0 ** -21 if which == 0 else 0.0)
                        assert torch.all((codes.float().double() - z).abs() <= rows8.half_step_of_code(z.abs() + slack, kind) + slack)
                    else:
                        assert torch.all((value - x).abs() <= x.abs() * rows8.HALF_STEP[kind] * 1.01 + x.abs().amax() * 2.0 ** -21)
                    out = (k_out if which == 0 else v_out)[b, i].cpu().double()
                    assert torch.all((out - value).abs() <= value.abs() * 2.0 ** -24)
    # nothing else was written
    same = (pool.view(torch.uint8) == before.view(torch.uint8)).cpu().view(*pool.shape[:4], -1).all(-1)
    assert torch.all(same | touched)
    if scales is not None:
        assert torch.all((scales.cpu() == 7.0) | touched)


def test_append_without_rotation_in_place_and_unaligned():
    # a dense q is rotated in place; an odd start of k and v takes the narrow accesses: the same bits
    rng = np.random.default_rng(3)
    batch, rows, heads, d, size = 2, 5, 2, 64, 32
    table = rows8.make_table(rng, 4, batch, 2, [2, 2])
    rope = rope_table(64, d).cuda()
    start = torch.tensor([3, 30], dtype=torch.int32, device="cuda")
    k, v, q = (normal(20 + i, batch, rows, heads, d).to(BF16).cuda() for i in range(3))
    results = []
    for shift in (0, 1):
        buf = [torch.zeros(k.numel() + 8, dtype=BF16, device="cuda") for _ in range(3)]
        t = []
        for x, y in zip((k, v, q), buf):
            y[shift:shift + x.numel()] = x.reshape(-1)
            t.append(y[shift:shift + x.numel()].view(x.shape))
        pool, scales = torch.zeros(4, 2, heads, size, d, dtype=INT8, device="cuda"), torch.zeros(4, 2, heads, size, device="cuda")
        binding.spec_kv_append(t[0], t[1], pool, scales, table, start, rope=rope, q=t[2], q_out=t[2])
        out = [torch.zeros(k.numel() + 8, device="cuda")[shift:shift + k.numel()].view(k.shape) for _ in range(2)]
        binding.spec_kv_read(pool, scales, table, start, rows, k=out[0], v=out[1])
        results.append((pool, scales, t[2].clone(), *out))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    binding.spec_kv_append(k, v, pool, scales, table, start)  # no rotation: V's treatment for K too
    a, b = binding.spec_kv_read(pool, scales, table, start, rows)
    assert torch.all((a - k.float()).abs() <= k.float().abs().amax(-1, keepdim=True) / 127 * 0.5001)
    assert torch.all((b - v.float()).abs() <= v.float().abs().amax(-1, keepdim=True) / 127 * 0.5001)


def test_rows_past_32_bits_of_the_pool():
    heads, size, d = 8, 256, 128
    pages = 2 ** 32 // (2 * heads * size * d) + 40  # bytes of the pool: past 2^32
    pool = torch.empty(pages, 2, heads, size, d, dtype=INT8, device="cuda")
    scales = torch.ones(pages, 2, heads, size, device="cuda")
    table = torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32, device="cuda")
    k, v = (normal(i, 1, 300, heads, d).to(BF16).cuda() for i in (1, 2))
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.spec_kv_append(k, v, pool, scales, table, start)
    a, b = binding.spec_kv_read(pool, scales, table, start, 300)
    assert torch.all((a - k.float()).abs() <= k.float().abs().amax(-1, keepdim=True) / 127 * 0.5001)
    assert torch.all((b - v.float()).abs() <= v.float().abs().amax(-1, keepdim=True) / 127 * 0.5001)
    q = normal(3, 1, 2, heads, d).to(BF16).cuda()
    lengths = torch.tensor([300], dtype=torch.int32, device="cuda")
    got = binding.spec_paged_attention(q, pool, scales, table, lengths)
    want, bound = rows8.attention64(q, pool, scales, table, lengths, d ** -0.5)
    assert torch.all((got.cpu().double() - want).abs() <= bound)


def test_linear_and_norm_in_a_graph_and_on_another_stream():
    x, gain = normal(1, 5, 512).to(BF16).cuda(), torch.ones(512, device="cuda")
    w, ws = binding.spec_quantize_fp8(normal(2, 256, 512).cuda())
    codes, scales, y = torch.empty(5, 512, dtype=E4M3, device="cuda"), torch.empty(5, device="cuda"), torch.empty(5, 256, device="cuda")

    def step():
        binding.spec_norm_fp8(x, gain, 1e-6, codes=codes, scales=scales)
        binding.spec_linear_fp8(codes, scales, w, ws, act="silu", y=y)

    step()
    want = y.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.zero_()
        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    x.mul_(2.0).add_(1.0)
    graph.replay()
    torch.cuda.synchronize()
    replayed = y.clone()
    step()
    assert torch.equal(y, replayed) and not torch.equal(y, want)
