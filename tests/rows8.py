"""64-bit references of the 8-bit operators, and how far a kernel may be from them."""
import numpy as np
import torch

TOP = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def scale64(y, kind):
    top = y.abs().amax(-1)
    return torch.where(top == 0, torch.ones_like(top), (top / TOP[kind]).clamp_min(2.0 ** -80))


def half_step_of_code(z, kind):
    """Half the distance between the codes around z (e4m3: four significant bits, no step below 2^-9)."""
    if kind == torch.int8:
        return torch.full_like(z, 0.5)
    _, e = torch.frexp(z)
    return torch.exp2((e.double() - 5).clamp_min(-10.0))


def check_codes(codes, scales, y, kind, rel=0.0):
    """codes, scales of rows y (64 bits) that the kernel knows to within `rel` of the row's largest magnitude each and `rel` of
    themselves: the scale is a maximum (off by as much) times a rounded reciprocal, which are two roundings of 2^-24, a code one
    reciprocal, one product and the rounding to the nearest code, each within half a step (the scale's two, the reciprocal and the
    product: 4 * 2^-24 of a value)."""
    y, codes, scales = y.double().cpu(), codes.float().double().cpu(), scales.double().cpu()
    want = scale64(y, kind)
    assert torch.all((scales - want).abs() <= want * (rel + 2 * 2.0 ** -24 * 1.01)), "scales"
    z = y / want[..., None]
    slack = z.abs() * (2 * rel + 4 * 2.0 ** -24)
    # (a value this near to a tie may go to either side: the distance to its code is then half a step and the slack)
    far = (codes - z).abs() - half_step_of_code(z.abs() + slack, kind) - slack
    assert torch.all(far <= 0), f"codes: {float(far.max())} beyond half a step"


def dequantised(pool, scales):
    x = pool.cpu()
    x = x.float().double()
    return x if scales is None else x * scales.double().cpu()[..., None]


def gathered(pool, scales, table, b, length):
    """K and V of a sequence in 64 bits, [2, kv heads, length, d], and which of its keys lie on a page of the pool."""
    pages, _, heads, size, d = pool.shape
    out = torch.zeros(2, heads, length, d, dtype=torch.float64)
    there = torch.zeros(length, dtype=torch.bool)
    row = table[b].tolist()
    for j in range(min(len(row), -(-length // size))):
        n = min(size, length - j * size)
        if 0 <= row[j] < pages and n > 0:
            page = dequantised(pool[row[j]], None if scales is None else scales[row[j]])
            out[:, :, j * size:j * size + n] = page[:, :, :n]
            there[j * size:j * size + n] = True
    return out, there


def attention64(q, pool, scales, table, lengths, scale):
    """(out, bound): the formula in 64 bits, and how far the kernel may be from it.

    The kernel multiplies exact 16-bit values (a power of two per query row is exact but for what lies 2^-25 below the row's
    largest), adds d products in fp32: a score is off by d 2^-24 sum|q||k| scale at most, some roundings of the exponent on top
    (2^-21 of its size, which the scales' logarithms raise by up to 80).  A weight is rounded to 16 bits, half a step of itself,
    or, where it is subnormal in fp16 against the largest p_j s_j of the row, by 2^-25 of that, for each key.  The output is
    rounded once."""
    batch, rows, heads, d = q.shape
    n_kv = pool.shape[2]
    out = torch.zeros(batch, rows, heads, d, dtype=torch.float64)
    bound = torch.zeros_like(out)
    group = heads // n_kv
    weight_step = 2.0 ** -8 if pool.dtype == torch.bfloat16 else 2.0 ** -11
    cap = table.shape[1] * pool.shape[3]
    for b, length in enumerate(lengths.tolist()):
        kv, there = gathered(pool, scales, table, b, max(0, min(length, cap)))
        for i in range(rows):
            seen = min(length - rows + i + 1, kv.shape[2])
            if seen <= 0:
                continue
            at = there[:seen].nonzero()[:, 0]
            if at.numel() == 0:
                continue
            for h in range(n_kv):
                k, v = kv[0, h][at], kv[1, h][at]
                qq = q[b, i, h * group:(h + 1) * group].double().cpu()
                s = qq @ k.T * scale
                p = torch.softmax(s, -1)
                o = p @ v
                size = p @ v.abs()
                delta = (d + 8) * 2.0 ** -24 * (qq.abs() @ k.abs().T).amax(-1, keepdim=True) * abs(scale) + 2.0 ** -21 * (s.abs().amax(-1, keepdim=True) + 80)
                rowmax = v.abs().amax(-1)
                # (8-bit rows: p_j s_j against the largest of them, codes at most 448; 16-bit rows: p_j against the largest, any value)
                largest = (p * rowmax).amax(-1, keepdim=True) if pool.dtype in TOP else p.amax(-1, keepdim=True) * rowmax.max()
                subnormal = 2.0 ** -25 * largest * at.numel()
                out[b, i, h * group:(h + 1) * group] = o
                bound[b, i, h * group:(h + 1) * group] = size * (weight_step + 2 * delta + 2.0 ** -20) + subnormal + o.abs() * HALF_STEP[q.dtype] * 1.01 + 2.0 ** -25
    return out, bound


def make_cache(rng, pages, n_kv, size, d, kind, device="cuda", spread=0.5):
    """A pool filled with quantised random rows whose sizes differ by factors of e^(spread N(0, 1))."""
    x = torch.from_numpy(rng.standard_normal((pages, 2, n_kv, size, d), dtype=np.float32))
    x = x * torch.from_numpy(np.exp(spread * rng.standard_normal((pages, 2, n_kv, size, 1))).astype(np.float32))
    if kind not in TOP:
        return x.to(kind).to(device), None
    s = scale64(x.double(), kind).float()
    z = x * (1.0 / s)[..., None]
    codes = z.clamp(-448, 448).to(kind) if kind == torch.float8_e4m3fn else z.round().to(kind)
    return codes.to(device), s.to(device)


def make_table(rng, pages, batch, width, used, device="cuda"):
    """Distinct pages for the first used[b] entries of every row, -1 behind them."""
    order = rng.permutation(pages)
    table = np.full((batch, width), -1, dtype=np.int32)
    at = 0
    for b in range(batch):
        table[b, :used[b]] = order[at:at + used[b]]
        at += used[b]
    return torch.from_numpy(table).to(device)
