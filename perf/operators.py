"""Microscaled operators as cases: what their speed on one GPU is measured on.

A block of 32 consecutive elements shares a power-of-two scale 2^(s - 127),
one byte s; an element is a 4-bit E2M1 ("fp4") or an 8-bit E4M3 ("fp8")
floating point number.  Four operators, each a `kind`:

  quant   rows are quantized to fp4 blocks and read back
  linear  Y = Q(X) W^T + bias: activations quantized to fp4 in the call, weights
          fp4 blocks already
  cache   new keys and values are quantized into the pages of a cache and read back
  attend  one new token of every sequence attends over its pages of the cache

`run` computes them in elementary torch operations in 32 bits, or, where `own`
is true, by the calls that a user makes of the library.  `exact` computes them
in 64 bits from their definitions.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 32
ROW = 128          # rows of fp4 codes are padded to a multiple of this many elements
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# mantissa bits, least exponent, exponent of the largest element, largest element
FORMATS = {"fp4": (1, 0, 2, 6.0), "fp8": (3, -6, 8, 448.0)}
FP4_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # the hidden state of one token: a call's latency
        dict(name="quant_token", kind="quant", rows=1, d=4096, dtype="bf16", pad=0),
        # activations of odd sizes, a view into wider rows
        dict(name="quant_odd", kind="quant", rows=999, d=2047, dtype="f16", pad=3),
        # the weights of the largest layer of VGG-16's classifier, as the fit takes them
        dict(name="quant_weights", kind="quant", rows=4096, d=25088, dtype="f32", pad=0),
        # one token through a square layer, and four through the largest classifier layer
        dict(name="linear_token", kind="linear", n=1, c=4096, d=4096, dtype="bf16", bias=False),
        dict(name="linear_tokens4", kind="linear", n=4, c=4096, d=25088, dtype="bf16", bias=True),
        # a short prompt at odd sizes
        dict(name="linear_odd", kind="linear", n=77, c=1000, d=2047, dtype="f32", bias=True),
        # a long prompt
        dict(name="linear_prompt", kind="linear", n=8192, c=4096, d=4096, dtype="bf16", bias=False),
        # a decoding step writes one token of each of 64 sequences
        dict(name="cache_tokens", kind="cache", tokens=64, heads=8, dim=128, dtype="bf16", fmt="fp8", page=64),
        # a long prompt is written
        dict(name="cache_prompt", kind="cache", tokens=32768, heads=8, dim=128, dtype="bf16", fmt="fp4", page=16),
        # one short sequence, heads of odd size in odd groups, one of three sequences empty: latency
        dict(name="attend_odd", kind="attend", batch=3, most=517, kv=2, group=7, dim=80, dtype="f32", fmt="fp4", page=48,
             window=300, empty=True),
        # one sequence of a long context
        dict(name="attend_long", kind="attend", batch=1, most=131072, kv=8, group=4, dim=128, dtype="bf16", fmt="fp8",
             page=64, window=0, empty=False),
        # an ordinary decoding step: many sequences of different lengths
        dict(name="attend_batch", kind="attend", batch=32, most=8192, kv=8, group=8, dim=128, dtype="bf16", fmt="fp8",
             page=64, window=0, empty=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("quant", "linear", "cache", "attend"))
    dtype = rng.choice(("f32", "f16", "bf16"))
    if kind == "quant":
        d = _log(rng, 1, 25088)
        return dict(kind=kind, rows=_log(rng, 1, min(65536, 4096 * 25088 // d)), d=d, dtype=dtype,
                    pad=rng.choice((0, 0, 1, 8)))
    if kind == "linear":
        while True:
            n, c, d = _log(rng, 1, 8192), _log(rng, 16, 8192), _log(rng, 17, 25088)
            if n * c * d <= 8192 * 4096 * 4096 and c * d <= 4096 * 25088 and n * d <= 2 ** 26:
                return dict(kind=kind, n=n, c=c, d=d, dtype=dtype, bias=rng.random() < 0.5)
    heads = rng.choice((1, 2, 3, 4, 8, 16))
    dim = rng.choice((32, 40, 64, 80, 96, 128, 128, 192, 256))
    fmt = rng.choice(("fp4", "fp8"))
    page = rng.choice((16, 32, 48, 64, 128, 256))
    if kind == "cache":
        return dict(kind=kind, tokens=_log(rng, 1, min(65536, 2 ** 25 // (heads * dim))), heads=heads, dim=dim,
                    dtype=dtype, fmt=fmt, page=page)
    batch = _log(rng, 1, 64)
    most = _log(rng, 1, min(131072, 2 ** 28 // (batch * heads * dim)))
    return dict(kind=kind, batch=batch, most=most, kv=heads, group=rng.choice((1, 2, 4, 5, 7, 8, 12, 16, 24)), dim=dim,
                dtype=dtype, fmt=fmt, page=page, window=rng.choice((0, 0, 0, max(1, most // 3))),
                empty=batch > 1 and rng.random() < 0.3)


# ---------------------------------------------------------------- the format


def _floor_log2(x):
    return torch.frexp(x)[1] - 1


def _quantize(x, fmt):
    """[..., d] fp32 (d a multiple of 32) -> the values that the elements
    stand for (without the scale) and the scales' exponents + 127."""
    bits, least, top, largest = FORMATS[fmt]
    b = x.reshape(*x.shape[:-1], -1, BLOCK)
    amax = b.abs().amax(-1, keepdim=True)
    e = torch.where(amax > 0, _floor_log2(amax) - top, torch.full_like(amax, -127, dtype=torch.int32)).clamp(-127, 127)
    y = torch.ldexp(b, -e)
    q = torch.ldexp(torch.ones_like(y), _floor_log2(y.abs()).clamp(min=least) - bits)
    y = (torch.round(y / q) * q).clamp(-largest, largest)
    return y.reshape(x.shape), (e + 127).squeeze(-1).to(torch.uint8)


def _scaled(y, s, dtype):
    """The values of elements y [..., d] under the scales s [..., d / 32]."""
    e = s.to(torch.int32) - 127
    return torch.ldexp(y.reshape(*s.shape, BLOCK).to(dtype), e.unsqueeze(-1)).reshape(y.shape)


def _padded(x, to):
    short = -x.shape[-1] % to
    return torch.nn.functional.pad(x, (0, short)) if short else x


def _pack(y, fmt):
    """Elements' values -> their codes: one byte each, or two in a byte (the
    even one in the low half)."""
    if fmt == "fp8":
        return y.to(torch.float8_e4m3fn).view(torch.uint8)
    edges = torch.tensor(FP4_VALUES, device=y.device)
    c = torch.searchsorted(edges, y.abs()).to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _unpack(codes, fmt):
    """Codes -> the elements' values, fp32."""
    if fmt == "fp8":
        return codes.view(torch.float8_e4m3fn).to(torch.float32)
    table = torch.tensor(FP4_VALUES + tuple(-v for v in FP4_VALUES), device=codes.device)
    c = torch.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    return table[c.to(torch.int32)]


def _rounded(c, dim):
    return -(-dim // BLOCK) * BLOCK


# ---------------------------------------------------------------- inputs


def _lengths(c):
    """Lengths spread over 1 .. most, the longest first; with `empty` the last is 0."""
    n = [1 + (c["most"] - 1) * (96 - b * 41 % 97) // 96 for b in range(c["batch"])]
    if c["empty"]:
        n[-1] = 0
    return n


def _heavy(shape, g, dtype):
    """Activations: normal, with channels of different size."""
    x = torch.randn(shape, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(shape[-1], generator=g, device=DEV))
    return x.to(dtype)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dtype = DTYPES[c["dtype"]]
    if c["kind"] == "quant":
        c["X"] = _heavy((c["rows"], c["d"] + c["pad"]), g, dtype)[:, c["pad"]:]
    elif c["kind"] == "linear":
        c["X"] = _heavy((c["n"], c["d"]), g, dtype)
        W = torch.randn((c["c"], c["d"]), generator=g, device=DEV)
        W *= torch.exp(0.5 * torch.randn((c["c"], 1), generator=g, device=DEV)) / math.sqrt(c["d"])
        y, c["scales"] = _quantize(_padded(W, ROW), "fp4")
        c["codes"] = _pack(y, "fp4")
        c["b"] = torch.randn((c["c"],), generator=g, device=DEV) if c["bias"] else None
    elif c["kind"] == "cache":
        shape = (c["tokens"], c["heads"], c["dim"])
        c["K"], c["V"] = _heavy(shape, g, dtype), _heavy(shape, g, dtype)
        pages = -(-c["tokens"] // c["page"]) + 3
        c["slots"] = torch.randperm(pages * c["page"], generator=g, device=DEV)[:c["tokens"]].contiguous()
        wide = _rounded(c, c["dim"])
        row = wide if c["fmt"] == "fp8" else wide // 2
        c["buffers"] = [torch.zeros((pages, c["heads"], c["page"], row), dtype=torch.uint8, device=DEV) for _ in "KV"] + [
            torch.zeros((pages, c["heads"], wide // BLOCK, c["page"]), dtype=torch.uint8, device=DEV) for _ in "KV"]
    else:
        lengths = _lengths(c)
        need = [-(-n // c["page"]) for n in lengths]
        total = sum(need) + 2
        table = torch.full((c["batch"], max(need)), -1, dtype=torch.int32)
        order = torch.randperm(total, generator=g, device=DEV).cpu()
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        c["table"] = table.to(DEV)
        c["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        c["buffers"] = []
        scales = []
        for _ in "KV":
            x = _heavy((total, c["kv"], c["page"], c["dim"]), g, torch.float32)
            y, s = _quantize(_padded(x, BLOCK), c["fmt"])
            c["buffers"].append(_pack(y, c["fmt"]))
            scales.append(s.transpose(-1, -2).contiguous())
            del x, y
        c["buffers"] += scales
        c["Q"] = torch.randn((c["batch"], c["kv"] * c["group"], c["dim"]), generator=g, device=DEV).to(dtype)
        c["scale"] = 1.0 / math.sqrt(c["dim"])
    if own and c["kind"] in ("cache", "attend"):
        from paper_2002_09049_amd import mpq
        k, v, ks, vs = c["buffers"]
        c["handle"] = mpq.MXCache(k, v, ks, vs, head_dim=c["dim"], fmt=c["fmt"])
    if own and c["kind"] in ("linear", "attend"):
        from paper_2002_09049_amd import mpq
        if c["kind"] == "linear":
            nbytes = mpq.mx_linear_workspace(c["n"], c["c"], c["d"])
        else:
            nbytes = c["handle"].attend_workspace(c["batch"], c["kv"] * c["group"], c["table"].shape[1])
        c["workspace"] = torch.empty((nbytes,), dtype=torch.uint8, device=DEV)
    return c


# ---------------------------------------------------------------- one pass


def _run_own(c):
    from paper_2002_09049_amd import mpq
    if c["kind"] == "quant":
        codes, scales = mpq.mx_quantize(c["X"])
        return mpq.mx_dequantize(codes, scales, c["d"], dtype=torch.bfloat16)
    if c["kind"] == "linear":
        return mpq.mx_linear(c["X"], c["codes"], c["scales"], bias=c["b"], workspace=c["workspace"])
    if c["kind"] == "cache":
        c["handle"].write(c["K"], c["V"], c["slots"])
        return c["handle"].read(c["slots"], dtype=c["K"].dtype)
    return c["handle"].attend(c["Q"], c["table"], c["lengths"], scale=c["scale"], window=c["window"], with_lse=True,
                              workspace=c["workspace"])


def run(state):
    c = state
    if own:
        return _run_own(c)
    if c["kind"] == "quant":
        y, s = _quantize(_padded(c["X"].float(), BLOCK), "fp4")
        return _scaled(y, s, torch.float32)[:, :c["d"]].to(torch.bfloat16)
    if c["kind"] == "linear":
        x = _padded(c["X"].float(), ROW)
        x = _scaled(*_quantize(x, "fp4"), torch.float32)
        w = _scaled(_unpack(c["codes"], "fp4"), c["scales"], torch.float32)
        y = x @ w.t()
        if c["b"] is not None:
            y = y + c["b"]
        return y.to(c["X"].dtype)
    if c["kind"] == "cache":
        page, where = c["slots"] // c["page"], c["slots"] % c["page"]
        out = []
        for x, codes, scales in zip((c["K"], c["V"]), c["buffers"][:2], c["buffers"][2:]):
            y, s = _quantize(_padded(x.float(), BLOCK), c["fmt"])
            codes[page, :, where] = _pack(y, c["fmt"])
            scales[page, :, :, where] = s
            back = _scaled(_unpack(codes[page, :, where], c["fmt"]), scales[page, :, :, where], torch.float32)
            out.append(back[..., :c["dim"]].to(x.dtype))
        return tuple(out)
    table = c["table"].clamp(min=0).long()

    def whole(codes, scales):
        """[batch, kv, tokens, dim] values of every sequence's pages."""
        y, s = _unpack(codes[table], c["fmt"]), scales[table].transpose(-1, -2)
        x = _scaled(y, s, torch.float32)[..., :c["dim"]]
        return x.permute(0, 2, 1, 3, 4).reshape(c["batch"], c["kv"], -1, c["dim"])

    k, v, ks, vs = c["buffers"]
    q = c["Q"].float().reshape(c["batch"], c["kv"], c["group"], c["dim"])
    scores = (q @ whole(k, ks).transpose(-1, -2)) * c["scale"]
    j = torch.arange(scores.shape[-1], device=DEV)
    n = c["lengths"].long()[:, None]
    seen = j < n
    if c["window"]:
        seen = seen & (j >= n - c["window"])
    seen = seen[:, None, None, :]
    scores = torch.where(seen, scores, torch.full_like(scores, -math.inf))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    o = (p @ whole(v, vs)) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + torch.log(total)).reshape(c["batch"], -1)
    return o.reshape(c["Q"].shape).to(c["Q"].dtype), lse


def work(case):
    c = case
    size = DTYPES[c["dtype"]].itemsize
    if c["kind"] == "quant":
        n = c["rows"] * c["d"]
        # the rows read, their blocks written and read, the values written
        return {"bytes": n * size + 2 * n * 17 // 32 + 2 * n, "flops": 4 * n}
    if c["kind"] == "linear":
        return {"bytes": (c["n"] * (c["d"] + c["c"]) * size + c["c"] * c["d"] * 17 // 32 + 4 * c["c"] * c["bias"]),
                "flops": 2 * c["n"] * c["c"] * c["d"]}
    held = (33 if c["fmt"] == "fp8" else 17) / 32     # bytes of an element in the cache
    if c["kind"] == "cache":
        n = 2 * c["tokens"] * c["heads"] * c["dim"]
        return {"bytes": int(2 * n * (size + held)) + 2 * 8 * c["tokens"], "flops": 4 * n}
    tokens = sum(min(n, c["window"]) if c["window"] else n for n in _lengths(c))
    heads = c["kv"] * c["group"]
    return {"bytes": int(2 * tokens * c["kv"] * c["dim"] * held) + 2 * c["batch"] * heads * c["dim"] * size
            + 4 * c["batch"] * heads, "flops": 4 * tokens * heads * c["dim"]}


# ---------------------------------------------------------------- in 64 bits


def _exact_elements(x, fmt):
    """The nearest values of the format to each block of x (fp64, [..., d]),
    ties to the even one: by search in the sorted list of the elements'
    values, under the block's power of two."""
    if fmt == "fp4":
        values = torch.tensor(FP4_VALUES, dtype=torch.float64, device=x.device)
    else:
        byte = range(0, 127)
        values = torch.tensor([(b & 7) * 2.0 ** -9 if b < 8 else (8 + (b & 7)) * 2.0 ** ((b >> 3) - 10) for b in byte],
                              dtype=torch.float64, device=x.device)
    d = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -d % BLOCK)).reshape(*x.shape[:-1], -1, BLOCK)
    amax = b.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.floor(torch.log2(torch.where(amax > 0, amax, torch.ones_like(amax)))) - FORMATS[fmt][2])
    y = (b.abs() / scale).clamp(max=float(values[-1]))
    hi = torch.searchsorted(values, y).clamp(max=len(values) - 1)
    lo = (hi - 1).clamp(min=0)
    below, above = y - values[lo], values[hi] - y
    take = torch.where(below == above, torch.where(lo % 2 == 0, lo, hi), torch.where(below < above, lo, hi))
    return (values[take] * scale * torch.sign(b)).reshape(*x.shape[:-1], -1)[..., :d]


def _exact_held(codes, scales, fmt):
    """The values that codes [..., d] under scales [..., d / 32] stand for."""
    if fmt == "fp4":
        low, high = (codes & 15).long(), (codes >> 4).long()
        c = torch.cat((low.unsqueeze(-1), high.unsqueeze(-1)), -1).flatten(-2)
        mag, sign, bits, bias = c & 7, c >> 3, 1, 1
    else:
        mag, sign, bits, bias = (codes & 127).long(), (codes >> 7).long(), 3, 7
    e, m = mag >> bits, (mag & (2 ** bits - 1)).double()
    x = torch.where(e > 0, (1 + m * 2.0 ** -bits) * torch.exp2((e - bias).double()), m * 2.0 ** (1 - bias - bits))
    x = torch.where(sign > 0, -x, x)
    return x * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, -1)


def exact(case, seed):
    c = prepare(case, seed)
    if c["kind"] == "quant":
        step = max(1, 2 ** 23 // c["d"])
        return torch.cat([_exact_elements(x.double(), "fp4") for x in c["X"].split(step)])
    if c["kind"] == "linear":
        step = max(1, 2 ** 23 // c["d"])
        x = torch.cat([_exact_elements(x.double(), "fp4") for x in c["X"].split(step)])
        y = torch.cat([x @ _exact_held(q, s, "fp4")[:, :c["d"]].t()
                       for q, s in zip(c["codes"].split(step), c["scales"].split(step))], -1)
        return y if c["b"] is None else y + c["b"].double()
    if c["kind"] == "cache":
        step = max(1, 2 ** 23 // (c["heads"] * c["dim"]))
        return tuple(torch.cat([_exact_elements(x.double(), c["fmt"]) for x in t.split(step)]) for t in (c["K"], c["V"]))
    k, v, ks, vs = c["buffers"]
    out = torch.zeros(c["Q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(c["Q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_lengths(c)):
        first = max(0, n - c["window"]) if c["window"] else 0
        pages = c["table"][b, :-(-n // c["page"])].long()
        for h in range(c["kv"] if n else 0):
            held = []
            for codes, scales in ((k, ks), (v, vs)):
                x = _exact_held(codes[pages, h], scales[pages, h].transpose(-1, -2), c["fmt"])
                held.append(x.reshape(-1, x.shape[-1])[first:n, :c["dim"]])
            mine = slice(h * c["group"], (h + 1) * c["group"])
            s = c["Q"][b, mine].double() @ held[0].t().contiguous() * c["scale"]
            lse[b, mine] = torch.logsumexp(s, -1)
            out[b, mine] = torch.softmax(s, -1) @ held[1]
    return out, lse
