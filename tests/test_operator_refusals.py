"""What the 8-bit operators refuse, without a GPU: a refused call touches no pointer."""
import pytest
import torch

import __graft_entry__ as entry
from paper_2211_17192_b200 import binding

P = 1 << 20  # stands for any aligned address: nothing reads it


@pytest.fixture(scope="module")
def h():
    entry.build()
    return binding.lib()


def refused(h, status, word):
    assert status == -1 and word in h.spec_last_error().decode()


def test_quantize_and_norm(h):
    def quantize(x=P, dt=1, rows=2, d=64, codes=P, scales=P):
        return h.spec_quantize_fp8(x, dt, rows, d, codes, scales, None)

    for kw, word in ((dict(x=None), "null"), (dict(codes=None), "null"), (dict(scales=None), "null"), (dict(dt=3), "dtype"), (dict(rows=-1), "rows"),
                     (dict(d=0), "d="), (dict(d=32769), "d="), (dict(x=P + 1), "aligned"), (dict(scales=P + 2), "aligned")):
        refused(h, quantize(**kw), word)
    assert quantize(rows=0, x=None) == 0

    def norm(x=P, dt=1, residual=P, out=P, hdt=0, gain=P, eps=1e-6, rows=2, d=64, codes=P, scales=P):
        return h.spec_norm_fp8(x, dt, residual, out, hdt, gain, eps, rows, d, codes, scales, None)

    for kw, word in ((dict(x=None), "null"), (dict(gain=None), "null"), (dict(codes=None), "null"), (dict(scales=None), "null"), (dict(dt=4), "dtype"),
                     (dict(hdt=2), "h_dtype"), (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
                     (dict(rows=-3), "rows"), (dict(d=40000), "d="), (dict(residual=P + 2), "aligned"), (dict(out=P + 1), "aligned"), (dict(gain=P + 2), "aligned")):
        refused(h, norm(**kw), word)
    assert norm(rows=0) == 0


def test_linear(h):
    def linear(x=P, xs=P, w=P, ws=P, bias=None, act=0, residual=None, y=P, dt=0, rows=3, n=64, k=64):
        return h.spec_linear_fp8(x, xs, w, ws, bias, act, residual, y, dt, rows, n, k, None)

    for kw, word in ((dict(x=None), "null"), (dict(xs=None), "null"), (dict(w=None), "null"), (dict(ws=None), "null"), (dict(y=None), "null"),
                     (dict(k=0), "k="), (dict(k=24), "multiple of 16"), (dict(n=0), "n_out"), (dict(rows=-1), "rows"), (dict(rows=1 << 23), "rows"),
                     (dict(act=5), "act"), (dict(act=-1), "act"), (dict(dt=3), "y_dtype"), (dict(x=P + 8), "16 bytes"), (dict(w=P + 4), "16 bytes"),
                     (dict(bias=P + 2), "aligned"), (dict(residual=P + 1), "aligned"), (dict(y=P + 2), "aligned")):
        refused(h, linear(**kw), word)
    assert linear(rows=0) == 0


CACHE = ((dict(pool=None), "null"), (dict(table=None), "null"), (dict(scales=None), "null"), (dict(kv=0), "kv_dtype"), (dict(kv=5), "kv_dtype"),
         (dict(pages=0), "pages"), (dict(size=48), "page_size"), (dict(size=16), "page_size"), (dict(size=512), "page_size"), (dict(n_kv=0), "n_kv_heads"),
         (dict(d=96), "d_head"), (dict(width=0), "max_pages"), (dict(width=1 << 30), "max_pages"), (dict(batch=-1), "batch"), (dict(batch=1 << 17), "batch"),
         (dict(rows=-1), "rows"), (dict(pool=P + 8), "aligned"), (dict(scales=P + 2), "aligned"))


def test_cache(h):
    def append(q=None, k=P, v=P, dt=1, qs=0, ks=256, vs=256, heads=0, n_kv=2, d=128, batch=2, rows=3, start=P, counts=None, rope=None, positions=0,
               q_out=None, pool=P, scales=P, kv=4, pages=4, size=64, table=P, width=2):
        return h.spec_kv_append(q, k, v, dt, qs, ks, vs, heads, n_kv, d, batch, rows, start, counts, rope, positions, q_out, pool, scales, kv, pages, size,
                                table, width, None)

    for kw, word in CACHE + ((dict(k=None), "null"), (dict(v=None), "null"), (dict(start=None), "null"), (dict(dt=3), "dtype"), (dict(q=P, heads=2, qs=256), "q_out"),
                             (dict(q_out=P), "q_out"), (dict(q=P, q_out=P, qs=256), "n_heads"), (dict(rope=P), "rope_positions"), (dict(ks=255), "stride"),
                             (dict(vs=0), "stride"), (dict(q=P, q_out=P, heads=3, qs=256), "stride"), (dict(k=P + 1), "aligned"), (dict(rope=P + 4, positions=9), "aligned")):
        refused(h, append(**kw), word)
    assert append(rows=0) == 0 and append(batch=0) == 0

    def read(pool=P, scales=P, kv=4, pages=4, size=64, n_kv=2, d=128, table=P, width=2, batch=2, rows=3, start=P, counts=None, k=P, v=P, dt=0):
        return h.spec_kv_read(pool, scales, kv, pages, size, n_kv, d, table, width, batch, rows, start, counts, k, v, dt, None)

    for kw, word in CACHE + ((dict(k=None), "null"), (dict(v=None), "null"), (dict(start=None), "null"), (dict(dt=4), "dtype"), (dict(k=P + 2), "aligned")):
        refused(h, read(**kw), word)
    assert read(rows=0) == 0


def test_attention(h):
    need = h.spec_paged_attention_workspace_bytes(2, 3, 4, 2, 128)
    assert need > 0 and h.spec_paged_attention_workspace_bytes(2, 3, 3, 2, 128) == 0 and h.spec_paged_attention_workspace_bytes(2, 3, 4, 2, 80) == 0

    def attention(q=P, dt=1, qs=512, pool=P, scales=P, kv=4, pages=4, size=64, table=P, width=2, lengths=P, batch=2, rows=3, heads=4, n_kv=2, d=128, scale=0.1,
                  out=P, ws=P, nbytes=need):
        return h.spec_paged_attention(q, dt, qs, pool, scales, kv, pages, size, table, width, lengths, batch, rows, heads, n_kv, d, scale, out, ws, nbytes, None)

    for kw, word in CACHE + ((dict(q=None), "null"), (dict(out=None), "null"), (dict(lengths=None), "null"), (dict(dt=0), "dtype"), (dict(kv=2), "own type"),
                             (dict(heads=3), "n_heads"), (dict(heads=0), "n_heads"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
                             (dict(qs=500), "stride"), (dict(qs=514), "8 bytes"), (dict(q=P + 4), "8 bytes"), (dict(out=P + 4), "8 bytes"), (dict(ws=None), "workspace"),
                             (dict(ws=P + 128), "workspace"), (dict(nbytes=need - 1), "workspace")):
        refused(h, attention(**kw), word)
    assert attention(rows=0) == 0 and attention(batch=0) == 0


def test_tensors_of_the_host_are_refused():
    x = torch.zeros(2, 64)
    with pytest.raises(ValueError, match="CUDA"):
        binding.spec_quantize_fp8(x)
    with pytest.raises(ValueError, match="CUDA"):
        binding.spec_norm_fp8(x, torch.ones(64))
    c = torch.zeros(2, 64, dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="CUDA"):
        binding.spec_linear_fp8(c, torch.ones(2), c, torch.ones(2))
    with pytest.raises(ValueError, match="act"):
        binding.spec_linear_fp8(c, torch.ones(2), c, torch.ones(2), act="relu")
    pool = torch.zeros(2, 2, 1, 32, 64, dtype=torch.int8)
    table = torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        binding.spec_kv_read(pool, torch.ones(2, 2, 1, 32), table, torch.zeros(1, dtype=torch.int32), 3)
    with pytest.raises(ValueError, match="CUDA"):
        binding.spec_paged_attention(torch.zeros(1, 1, 1, 64, dtype=torch.float16), pool, torch.ones(2, 2, 1, 32), table, torch.ones(1, dtype=torch.int32))
