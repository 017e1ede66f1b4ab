"""The operators of a decoder block with 8-bit weights, activations and cached K,V rows, as a user of
`paper_2211_17192_b200.binding` calls them between two models' passes:

* `norm`: residual addition, root-mean-square norm and an e4m3 output with a scale per row (`spec_norm_fp8`);
* `quantize`: the same output of a tensor as it is (`spec_quantize_fp8`), in front of the block's other two projections;
* `linear`: product of such codes with e4m3 weights, with scales, bias, activation and residual (`spec_linear_fp8`);
* `kv`: K and V rows of new tokens rotated, quantised and appended to a paged cache, then read back (`spec_kv_append`,
  `spec_kv_read`), which is what a prefix that another engine shall have goes through;
* `attention`: the few new tokens of every sequence against its cached rows (`spec_paged_attention`).

With `own` false `run` computes the same in elementary torch operations in 32 bits.
"""

import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TOP = {"e4m3": 448.0, "int8": 127.0}
SMALLEST = 2.0 ** -80  # of a scale
ROPE_BASE = 1e4


# --------------------------------------------------------------------------- #
# the cases
# --------------------------------------------------------------------------- #
def listed():
    return [
        # one draft step of the 160M-shaped model: a single row, latency only
        dict(name="norm_r1_d768", op="norm", rows=1, d=768, dtype="bf16", h_dtype="fp32"),
        # the chunk of a prompt pass, 4096 wide
        dict(name="norm_r2048_d4096", op="norm", rows=2048, d=4096, dtype="bf16", h_dtype="bf16"),
        # the attention output of a batch of 32 sequences and seven rows each
        dict(name="quantize_r224_d4096", op="quantize", rows=224, d=4096, dtype="fp16"),
        # FFN activations of a prompt chunk in front of the last projection
        dict(name="quantize_r2048_d11008", op="quantize", rows=2048, d=11008, dtype="bf16"),
        # the draft's q, k, v projection for one token
        dict(name="linear_r1_768x2304", op="linear", rows=1, k=768, n_out=2304, act="none", bias=True, residual=False, dtype="bf16"),
        # gated FFN of the 7B-shaped target in a verification pass, gamma = 2: bound by the weights' bytes
        dict(name="linear_r3_4096x11008_swiglu", op="linear", rows=3, k=4096, n_out=11008, act="swiglu", bias=False, residual=False, dtype="bf16"),
        # its last projection over a prompt chunk, added to the fp32 residual stream: bound by the tensor pipes
        dict(name="linear_r2048_11008x4096_res", op="linear", rows=2048, k=11008, n_out=4096, act="none", bias=False, residual=True, dtype="fp32"),
        # rows of a verification of 32 sequences, gamma = 6: ragged counts, rotated, appended, read back
        dict(name="kv_b32_r7_e4m3", op="kv", batch=32, rows=7, heads=32, kv_heads=8, d=128, context=900, page=64, dtype="bf16", kv="e4m3", rope=True),
        # two prompts into an int8 cache and out again
        dict(name="kv_b2_r1024_int8", op="kv", batch=2, rows=1024, heads=32, kv_heads=8, d=128, context=0, page=128, dtype="bf16", kv="int8", rope=True),
        # one sequence, gamma = 2, 1024 cached tokens of the 7B shape: latency
        dict(name="attention_b1_r3_l1024_e4m3", op="attention", batch=1, rows=3, heads=32, kv_heads=8, d=128, length=1027, ragged=0.0, page=64, dtype="bf16", kv="e4m3"),
        # a verification pass of a ragged batch, heads of 64 without groups
        dict(name="attention_b32_r7_l2048_fp16", op="attention", batch=32, rows=7, heads=12, kv_heads=12, d=64, length=2048, ragged=0.9, page=32, dtype="fp16", kv="fp16"),
        # one new token each over long contexts
        dict(name="attention_b16_r1_l32768_int8", op="attention", batch=16, rows=1, heads=32, kv_heads=8, d=128, length=32768, ragged=0.5, page=256, dtype="bf16", kv="int8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "quantize", "linear", "linear", "kv", "attention", "attention"])
    half = rng.choice(["bf16", "fp16"])
    if op == "norm":
        d = rng.choice([_log_int(rng, 8, 512) * 2, rng.randrange(1, 65) * 128])
        return dict(op=op, rows=min(_log_int(rng, 1, 4096), 2 ** 23 // d), d=d, dtype=rng.choice(["fp32", half]), h_dtype=rng.choice(["fp32", "same"]))
    if op == "quantize":
        d = rng.choice([_log_int(rng, 8, 2048) * 2, rng.randrange(1, 129) * 128])
        return dict(op=op, rows=min(_log_int(rng, 1, 4096), 2 ** 24 // d), d=d, dtype=rng.choice(["fp32", half]))
    if op == "linear":
        act = rng.choice(["none", "none", "gelu", "silu", "gated_gelu", "swiglu"])
        k, n_out = 16 * _log_int(rng, 4, 688), _log_int(rng, 60, 5500)
        n_out = rng.choice([n_out, n_out // 16 * 16 + 16])
        rows = min(_log_int(rng, 1, 2048), 2 ** 36 // (k * n_out))
        return dict(op=op, rows=rows, k=k, n_out=n_out, act=act, bias=rng.random() < 0.5, residual=rng.random() < 0.5, dtype=rng.choice(["fp32", half]))
    kv = rng.choice(["e4m3", "int8", "e4m3", "int8", half])
    d, page = rng.choice([64, 128]), rng.choice([32, 64, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 12])
    heads = kv_heads * rng.choice([1, 2, 4, 8])
    if op == "kv":
        batch = _log_int(rng, 1, 32)
        return dict(op=op, batch=batch, rows=_log_int(rng, 1, max(1, 2048 // batch)), heads=heads, kv_heads=kv_heads, d=d, context=rng.randrange(0, 3000),
                    page=page, dtype=rng.choice(["fp32", half]) if kv in TOP else kv, kv=kv, rope=rng.random() < 0.7)
    batch, rows = _log_int(rng, 1, 48), rng.choice([1, 1, rng.randrange(1, 10)])
    most = 16 * 32768 * 8 * 128 // (batch * kv_heads * d * (1 if kv in TOP else 2))
    return dict(op=op, batch=batch, rows=rows, heads=heads, kv_heads=kv_heads, d=d, length=_log_int(rng, 1, max(2, min(65536, most // 4))),
                ragged=rng.choice([0.0, 0.5, 1.0]), page=page, dtype=half, kv=kv)


def _lengths(case):
    """Tokens of every sequence: between (1 - ragged) and all of `length`, spread by the golden ratio."""
    return [case["length"] - int(case["ragged"] * case["length"] * (b * 0.6180339887 % 1.0)) for b in range(case["batch"])]


def _counts(case):
    """New rows of every sequence of a padded batch: between half of the rows and all of them."""
    return [case["rows"] - int(0.5 * case["rows"] * (b * 0.6180339887 % 1.0)) for b in range(case["batch"])]


def _size(name):
    return torch.empty(0, dtype=DTYPES[name]).element_size()


def _h_dtype(case):
    return case["dtype"] if case["h_dtype"] == "same" else case["h_dtype"]


def work(case):
    op = case["op"]
    if op in ("norm", "quantize"):
        n = case["rows"] * case["d"]
        if op == "quantize":
            return {"bytes": n * (_size(case["dtype"]) + 1) + 4 * case["rows"], "flops": 3 * n}
        return {"bytes": n * (_size(case["dtype"]) + 2 * _size(_h_dtype(case)) + 1) + 4 * case["rows"] + 4 * case["d"], "flops": 8 * n}
    if op == "linear":
        rows, k, n_out = case["rows"], case["k"], case["n_out"]
        n_w = 2 * n_out if case["act"] in ("gated_gelu", "swiglu") else n_out
        out = rows * n_out * _size(case["dtype"])
        return {"bytes": (rows + n_w) * k + 4 * (rows + n_w) + (4 * n_w if case["bias"] else 0) + out * (2 if case["residual"] else 1), "flops": 2 * rows * n_w * k}
    n_kv, d, scales = case["kv_heads"], case["d"], 4 if case["kv"] in TOP else 0
    if op == "kv":
        tokens = sum(_counts(case))
        q = 2 * tokens * case["heads"] * d * _size(case["dtype"]) + 4 * tokens * d if case["rope"] else 0
        row = d * (_size(case["dtype"]) + 2 * _size(case["kv"]) + 2) + 2 * scales  # written once, read once, 16 bits out
        return {"bytes": q + 2 * tokens * n_kv * row, "flops": 2 * tokens * (case["heads"] + 2 * n_kv) * d}
    tokens = sum(_lengths(case))
    io = 2 * case["batch"] * case["rows"] * case["heads"] * d * _size(case["dtype"])
    return {"bytes": io + 2 * tokens * n_kv * (d * _size(case["kv"]) + scales), "flops": 4 * tokens * case["rows"] * case["heads"] * d}


# --------------------------------------------------------------------------- #
# inputs
# --------------------------------------------------------------------------- #
def _quantize(y, kind):
    """Codes and scales of the last axis."""
    top = y.abs().amax(-1, keepdim=True)
    scale = torch.where(top == 0, torch.ones_like(top), (top / TOP[kind]).clamp_min(SMALLEST))
    code = y * (1.0 / scale)
    return (code.clamp(-448.0, 448.0).to(torch.float8_e4m3fn) if kind == "e4m3" else code.round().to(torch.int8)), scale.squeeze(-1)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    op = case["op"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    def activations(rows, d):  # a few channels are far larger than the rest, as a trained model's are
        wide = torch.ones(d, device=dev)
        wide[torch.randint(0, d, (max(1, d // 256),), generator=g, device=dev)] = 20.0
        return normal(rows, d) * wide

    s = {"case": case}
    if op in ("norm", "quantize"):
        rows, d = case["rows"], case["d"]
        s["x"] = activations(rows, d).to(DTYPES[case["dtype"]])
        s["codes"] = torch.empty(rows, d, dtype=torch.float8_e4m3fn, device=dev)
        s["scales"] = torch.empty(rows, device=dev)
        if op == "norm":
            s["gain"] = 1.0 + 0.1 * normal(d)
            s["residual"] = (3.0 * normal(rows, d)).to(DTYPES[_h_dtype(case)])
            s["h"] = torch.empty_like(s["residual"])
        return s
    if op == "linear":
        rows, k, n_out = case["rows"], case["k"], case["n_out"]
        n_w = 2 * n_out if case["act"] in ("gated_gelu", "swiglu") else n_out
        s["xc"], s["xs"] = _quantize(activations(rows, k), "e4m3")
        s["wc"], s["ws"] = _quantize(normal(n_w, k) / math.sqrt(k), "e4m3")
        s["bias"] = 0.5 * normal(n_w) if case["bias"] else None
        s["residual"] = normal(rows, n_out).to(DTYPES[case["dtype"]]) if case["residual"] else None
        s["y"] = torch.empty(rows, n_out, dtype=DTYPES[case["dtype"]], device=dev)
        return s

    batch, rows, heads, n_kv, d, page = (case[n] for n in ("batch", "rows", "heads", "kv_heads", "d", "page"))
    counts = _counts(case) if op == "kv" else None
    tokens = [case["context"] + c for c in counts] if op == "kv" else _lengths(case)
    need = [-(-t // page) for t in tokens]
    pages, width = sum(need) + 3, max(max(need), 1)
    order = torch.randperm(pages, generator=g, device=dev)[:sum(need)].to(torch.int32)
    table = torch.full((batch, width), -1, dtype=torch.int32, device=dev)
    cells = torch.tensor([b * width + j for b in range(batch) for j in range(need[b])], dtype=torch.int64, device=dev)
    table.view(-1)[cells] = order
    s["table"] = table
    kv = case["kv"]
    shape = (pages, 2, n_kv, page)
    if op == "kv":
        s["pool"] = torch.zeros(*shape, d, dtype=torch.uint8 if kv in TOP else DTYPES[kv], device=dev)
        s["pool"] = s["pool"].view(DTYPES[kv])
        s["scales"] = torch.zeros(shape, device=dev) if kv in TOP else None
        s["start"] = torch.full((batch,), case["context"], dtype=torch.int32, device=dev)
        s["counts"] = torch.tensor(counts, dtype=torch.int32, device=dev)
        # q, k and v are parts of one projection's output
        qkv = normal(batch, rows, (heads + 2 * n_kv) * d).to(DTYPES[case["dtype"]])
        s["q"], s["k"], s["v"] = (t.view(batch, rows, -1, d) for t in qkv.split([heads * d, n_kv * d, n_kv * d], dim=-1))
        s["rope"] = None
        if case["rope"]:
            position = torch.arange(max(tokens), dtype=torch.float64, device=dev)
            angle = position[:, None] * ROPE_BASE ** (-torch.arange(0, d, 2, dtype=torch.float64, device=dev) / d)
            s["rope"] = torch.stack((angle.cos(), angle.sin()), -1).to(torch.float32)
        else:
            s["q"] = None
        s["q_out"] = torch.zeros(batch, rows, heads, d, dtype=DTYPES[case["dtype"]], device=dev) if case["rope"] else None
        out = torch.float16 if case["dtype"] == "fp16" else torch.bfloat16
        s["k_out"], s["v_out"] = (torch.zeros(batch, rows, n_kv, d, dtype=out, device=dev) for _ in range(2))
        return s
    rowscale = torch.exp(0.5 * normal(*shape, 1))  # tokens differ in size
    values = normal(*shape, d) * rowscale
    if kv in TOP:
        s["pool"], s["scales"] = _quantize(values, kv)
    else:
        s["pool"], s["scales"] = values.to(DTYPES[kv]), None
    s["lengths"] = torch.tensor(tokens, dtype=torch.int32, device=dev)
    s["q"] = (1.5 * normal(batch, rows, heads, d)).to(DTYPES[case["dtype"]])
    s["out"] = torch.empty_like(s["q"])
    s["workspace"] = torch.empty(64 << 20, dtype=torch.uint8, device=dev)  # (scratch, as a serving loop keeps it)
    return s


# --------------------------------------------------------------------------- #
# one pass
# --------------------------------------------------------------------------- #
def run(s):
    return _run_own(s) if own else _PLAIN[s["case"]["op"]](s)


def _run_own(s):
    from paper_2211_17192_b200 import binding
    case = s["case"]
    op = case["op"]
    if op == "norm":
        codes, scales, h = binding.spec_norm_fp8(s["x"], s["gain"], 1e-6, residual=s["residual"], h=s["h"], codes=s["codes"], scales=s["scales"])
        return {"codes": codes, "scales": scales, "h": h}
    if op == "quantize":
        codes, scales = binding.spec_quantize_fp8(s["x"], codes=s["codes"], scales=s["scales"])
        return {"codes": codes, "scales": scales}
    if op == "linear":
        return {"y": binding.spec_linear_fp8(s["xc"], s["xs"], s["wc"], s["ws"], bias=s["bias"], act=case["act"], residual=s["residual"], y=s["y"])}
    if op == "kv":
        binding.spec_kv_append(s["k"], s["v"], s["pool"], s["scales"], s["table"], s["start"], counts=s["counts"], rope=s["rope"], q=s["q"], q_out=s["q_out"])
        k, v = binding.spec_kv_read(s["pool"], s["scales"], s["table"], s["start"], case["rows"], counts=s["counts"], k=s["k_out"], v=s["v_out"])
        return {"pool": s["pool"], "scales": s["scales"], "q": s["q_out"], "k": k, "v": v}
    return {"out": binding.spec_paged_attention(s["q"], s["pool"], s["scales"], s["table"], s["lengths"], out=s["out"], workspace=s["workspace"])}


def _plain_norm(s):
    h = (s["x"].float() + s["residual"].float()).to(s["h"].dtype)
    y = h.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * s["gain"]
    codes, scales = _quantize(y, "e4m3")
    return {"codes": codes, "scales": scales, "h": h}


def _plain_quantize(s):
    codes, scales = _quantize(s["x"].float(), "e4m3")
    return {"codes": codes, "scales": scales}


def _act(z, act, n_out):
    if act in ("gelu", "gated_gelu"):
        a = z[:, :n_out]
        a = 0.5 * a * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (a + 0.044715 * a * a * a)))
    elif act in ("silu", "swiglu"):
        a = z[:, :n_out] / (1.0 + torch.exp(-z[:, :n_out]))
    else:
        a = z
    return a * z[:, n_out:] if act in ("gated_gelu", "swiglu") else a


def _plain_linear(s):
    case = s["case"]
    z = (s["xc"].float() @ s["wc"].float().T) * s["xs"][:, None] * s["ws"]
    if s["bias"] is not None:
        z = z + s["bias"]
    y = _act(z, case["act"], case["n_out"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(s["y"].dtype)}


def _rotate(x, cs):
    """x [tokens, heads, d], cs [tokens, d/2, 2]."""
    half = x.shape[-1] // 2
    c, n = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = x[..., :half], x[..., half:]
    return torch.cat((a * c - b * n, b * c + a * n), -1)


def _plain_kv(s):
    case = s["case"]
    kv, page, rows = case["kv"], case["page"], case["rows"]
    new = torch.arange(rows, device=s["table"].device)
    b, i = (new[None, :] < s["counts"][:, None]).nonzero(as_tuple=True)  # what is no padding
    position = s["start"].long()[b] + i
    at, slot = s["table"].long()[b, position // page], position % page
    k, v = s["k"][b, i].float(), s["v"][b, i].float()
    if s["rope"] is not None:
        cs = s["rope"][position]
        k = _rotate(k, cs)
        s["q_out"][b, i] = _rotate(s["q"][b, i].float(), cs).to(s["q_out"].dtype)
    raw = s["pool"].view(torch.uint8) if kv in TOP else s["pool"]
    for which, x, out in ((0, k, s["k_out"]), (1, v, s["v_out"])):
        if kv in TOP:
            codes, scales = _quantize(x, kv)
            raw[at, which, :, slot] = codes.view(torch.uint8)
            s["scales"][at, which, :, slot] = scales
            back = raw[at, which, :, slot].view(s["pool"].dtype).float() * s["scales"][at, which, :, slot][..., None]
        else:
            raw[at, which, :, slot] = x.to(raw.dtype)
            back = raw[at, which, :, slot]
        out[b, i] = back.to(out.dtype)
    return {"pool": s["pool"], "scales": s["scales"], "q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _gather(s, which):
    """K (0) or V (1) of every sequence in fp32: [batch, kv_heads, width * page, d]."""
    kv, table = s["case"]["kv"], s["table"].long().clamp_min(0)
    raw = s["pool"].view(torch.uint8) if kv in TOP else s["pool"]
    x = raw[table, which].view(s["pool"].dtype).float()
    if kv in TOP:
        x = x * s["scales"][table, which][..., None]
    batch, width, n_kv, page, d = x.shape
    return x.transpose(1, 2).reshape(batch, n_kv, width * page, d)


def _plain_attention(s):
    case = s["case"]
    batch, rows, heads, n_kv, d = (case[n] for n in ("batch", "rows", "heads", "kv_heads", "d"))
    k, v = _gather(s, 0), _gather(s, 1)
    q = s["q"].float().view(batch, rows, n_kv, heads // n_kv, d).permute(0, 2, 1, 3, 4)  # [batch, kv head, row, query head, d]
    score = (q.reshape(batch, n_kv, -1, d) @ k.transpose(-1, -2)) / math.sqrt(d)
    last = s["lengths"][:, None] - rows + torch.arange(rows, device=k.device)            # position of every row
    hidden = torch.arange(k.shape[2], device=k.device) > last[..., None]                 # [batch, row, key]
    hidden = hidden[:, None, :, None, :].expand(batch, 1, rows, heads // n_kv, -1).reshape(batch, 1, -1, k.shape[2])
    score = score.masked_fill(hidden, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total == 0, torch.ones_like(total), total)
    out = out.view(batch, n_kv, rows, heads // n_kv, d).permute(0, 2, 1, 3, 4)
    return {"out": out.reshape(batch, rows, heads, d).to(s["q"].dtype)}


_PLAIN = {"norm": _plain_norm, "quantize": _plain_quantize, "linear": _plain_linear, "kv": _plain_kv, "attention": _plain_attention}


# --------------------------------------------------------------------------- #
# the definitions in 64 bits
# --------------------------------------------------------------------------- #
def _codes64(y, kind):
    top = y.abs().max(dim=-1).values
    scale = torch.maximum(top / TOP[kind], torch.full_like(top, SMALLEST))
    scale[top == 0] = 1.0
    z = y / scale[..., None]
    if kind == "int8":
        return torch.round(z), scale
    _, e = torch.frexp(z)  # |z| in [2^(e-1), 2^e): four significant bits, no step below 2^-9
    step = torch.exp2((e.to(torch.float64) - 4).clamp_min(-9.0))
    return torch.round(z / step) * step, scale


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "quantize"):
        if op == "quantize":
            codes, scales = _codes64(s["x"].double(), "e4m3")
            return {"codes": codes, "scales": scales}
        h = (s["x"].double() + s["residual"].double()).to(s["h"].dtype)
        y = h.double()
        y = s["gain"].double() * y / torch.sqrt(torch.sum(y * y, -1, keepdim=True) / case["d"] + 1e-6)
        codes, scales = _codes64(y, "e4m3")
        return {"codes": codes, "scales": scales, "h": s["x"].double() + s["residual"].double()}
    if op == "linear":
        n_out, act = case["n_out"], case["act"]
        z = torch.matmul(s["xc"].double() * s["xs"].double()[:, None], (s["wc"].double() * s["ws"].double()[:, None]).T)
        if s["bias"] is not None:
            z += s["bias"].double()
        if act in ("gelu", "gated_gelu"):
            y = torch.nn.functional.gelu(z[:, :n_out], approximate="tanh")
        elif act in ("silu", "swiglu"):
            y = z[:, :n_out] * torch.sigmoid(z[:, :n_out])
        else:
            y = z
        if act in ("gated_gelu", "swiglu"):
            y = y * z[:, n_out:]
        return {"y": y if s["residual"] is None else y + s["residual"].double()}
    batch, rows, heads, n_kv, d, page, kv = (case[n] for n in ("batch", "rows", "heads", "kv_heads", "d", "page", "kv"))
    table = s["table"].tolist()
    if op == "kv":
        pool, scales = s["pool"].double(), None if s["scales"] is None else s["scales"].double()
        q_out, k_out, v_out = (None if s[n] is None else s[n].double() for n in ("q_out", "k_out", "v_out"))
        freq = ROPE_BASE ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=pool.device) / d)

        def turned(x, at):
            if not case["rope"]:
                return x
            z = torch.complex(x[..., : d // 2], x[..., d // 2:]) * torch.polar(torch.ones_like(at[:, None] * freq), at[:, None] * freq)[:, None]
            return torch.cat((z.real, z.imag), -1)

        for b, count in enumerate(_counts(case)):
            at = torch.arange(case["context"], case["context"] + count, dtype=torch.float64, device=pool.device)
            if q_out is not None:
                q_out[b, :count] = turned(s["q"][b, :count].double(), at)
            for which, x, out in ((0, turned(s["k"][b, :count].double(), at), k_out), (1, s["v"][b, :count].double(), v_out)):
                codes, scale = _codes64(x, kv) if kv in TOP else (x, None)
                out[b, :count] = codes if scale is None else codes * scale[..., None]
                done = 0
                while done < count:  # page by page
                    position = case["context"] + done
                    here = min(count - done, page - position % page)
                    cell = (table[b][position // page], which, slice(None), slice(position % page, position % page + here))
                    pool[cell] = codes[done:done + here].transpose(0, 1)
                    if scale is not None:
                        scales[cell] = scale[done:done + here].transpose(0, 1)
                    done += here
        return {"pool": None if kv == "int8" else pool, "scales": scales, "q": q_out, "k": k_out, "v": v_out}
    out = torch.zeros(batch, rows, heads, d, dtype=torch.float64, device=s["q"].device)
    raw = s["pool"].view(torch.uint8) if kv in TOP else s["pool"]
    for b, length in enumerate(_lengths(case)):
        if length == 0:
            continue
        ids = s["table"][b, : -(-length // page)].long()
        x = raw[ids].view(s["pool"].dtype).double()                            # [pages, 2, kv heads, page, d]
        if kv in TOP:
            x = x * s["scales"][ids].double()[..., None]
        x = x.permute(1, 2, 0, 3, 4).reshape(2, n_kv, -1, d)[:, :, :length].repeat_interleave(heads // n_kv, 1)
        for i in range(rows):
            seen = length - rows + i + 1
            if seen > 0:
                p = torch.softmax(torch.einsum("hd,hld->hl", s["q"][b, i].double(), x[0, :, :seen]) * d ** -0.5, -1)
                out[b, i] = torch.einsum("hl,hld->hd", p, x[1, :, :seen])
    return {"out": out}
