"""The cases the few-bit serving operators are measured on, through the public entry points.

  mx_quantize  rows to microscaled 4-bit floats (E2M1 codes, an E8M0 scale per 32 of them) and the
               values they stand for: mpq_mx_quantize, mpq_mx_dequantize
  mx_linear    a linear layer with both operands in that form: mpq_mx_quantize of the inputs, then
               mpq_mx_linear with weights packed once
  cache        tokens written to a paged key-value cache in 8 or 4 bits, and read back:
               mpq_cache_write, mpq_cache_read
  attention    one new token of every sequence over that cache: mpq_cache_attention

Each has a plain form (elementary torch operations in fp32), taken where ``own`` is false, and
``exact`` restates its definition in 64 bits.  Sizes are those of the large linear layers among the
repository's workloads and generic ones around them.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)     # E2M1 magnitudes by code
WORKSPACE = 1 << 25                                   # zeroed once, kept by the program


# ---------------------------------------------------------------------------------------------
# The cases


def _quantize(rows, d, dtype):
    return dict(kind="mx_quantize", rows=rows, d=d, dtype=dtype)


def _linear(T, C, d, dtype, bias=False):
    return dict(kind="mx_linear", T=T, C=C, d=d, dtype=dtype, bias=bias)


def _cache(T, heads, dim, bits, page, dtype):
    return dict(kind="cache", T=T, heads=heads, dim=dim, bits=bits, page=page, dtype=dtype)


def _attention(B, length, spread, heads, group, dim, bits, page, dtype, window=0):
    return dict(kind="attention", B=B, length=length, spread=spread, heads=heads, group=group,
                dim=dim, bits=bits, page=page, dtype=dtype, window=window)


def listed():
    return [
        # the activations of a decode batch on their way into a linear layer
        dict(_quantize(48, 4096, "bf16"), name="quantize_48x4096"),
        # a large linear layer's weights, once per model
        dict(_quantize(11008, 4096, "fp32"), name="quantize_11008x4096_fp32"),
        # one token through a square linear layer: latency and the weights' bytes
        dict(_linear(1, 4096, 4096, "bf16"), name="linear_1x4096x4096"),
        # a small batch of tokens, an odd number of them, through the widening layer, with a bias
        dict(_linear(37, 11008, 4096, "fp16", True), name="linear_37x11008x4096"),
        # a prompt through the narrowing layer
        dict(_linear(2048, 4096, 11008, "bf16"), name="linear_2048x4096x11008"),
        # the new tokens of a decode batch enter the cache
        dict(_cache(32, 8, 128, 8, 16, "bf16"), name="cache_32_tokens"),
        # a packed batch of prompts enters the cache
        dict(_cache(8192, 8, 128, 8, 16, "bf16"), name="cache_8192_tokens"),
        # a prompt of a small model with narrow heads, 4 bits, fp32 activations
        dict(_cache(1999, 4, 64, 4, 64, "fp32"), name="cache_1999_tokens_4bit_fp32"),
        # one user's short conversation
        dict(_attention(1, 777, "all", 8, 4, 128, 8, 16, "bf16"), name="attend_1x777"),
        # a serving batch of ragged lengths, among them 0 and 1
        dict(_attention(96, 4096, "ragged", 8, 4, 128, 8, 16, "bf16"), name="attend_96_ragged"),
        # two long documents
        dict(_attention(2, 131072, "all", 8, 4, 128, 8, 64, "bf16"), name="attend_2x131072"),
        # a 4-bit cache, eight query heads to a key head
        dict(_attention(16, 16384, "ragged", 4, 8, 128, 4, 32, "fp16"), name="attend_16_ragged_4bit"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer's width: any whole number, or (three times in four) a multiple of 64."""
    d = _log(rng, lo, hi)
    return d if rng.random() < 0.25 else max(64, d // 64 * 64)


def _not(sizes, d):
    """d, or the next whole number where d is one of `sizes` (kept out of the cases)."""
    return d + 1 if d in sizes else d


def draw(rng):
    kind = rng.choice(("mx_quantize", "mx_linear", "mx_linear", "cache", "cache", "attention",
                       "attention", "attention"))
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    out = (3 * 1024,)
    if kind == "mx_quantize":
        d = _not(out, _width(rng, 33, 11008))
        return _quantize(_not(out, _log(rng, 1, max(1, 11008 * 4096 // d))), d, dtype)
    if kind == "mx_linear":
        d, C = _not(out, _width(rng, 64, 11008)), _not(out, _width(rng, 64, 11008))
        T = _log(rng, 1, max(1, min(4096, 2048 * 4096 * 11008 // (C * d))))
        return _linear(_not(out, T), C, d, dtype, rng.random() < 0.5)
    heads, dim = rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 128, 256))
    bits, page = rng.choice((8, 8, 4)), rng.choice((16, 16, 32, 64))
    if kind == "cache":
        T = _log(rng, 1, 8192 * 8 * 128 // (heads * dim))
        return _cache(_not(out, T), heads, dim, bits, page, dtype)
    group = rng.choice((1, 2, 3, 4, 5, 7, 8, 16))
    B = _log(rng, 1, 256)
    most = 2 * 131072 * 8 * 128 // (B * heads * dim * (2 if group > 8 else 1))
    length = _not(out, _log(rng, 1, max(1, min(131072, most))))
    window = _log(rng, 1, length) if rng.random() < 0.2 else 0
    return _attention(B, length, rng.choice(("all", "ragged")), heads, group, dim, bits, page,
                      rng.choice(("bf16", "fp16")), window)


def work(case):
    k = case["kind"]
    if k == "mx_quantize":
        n = case["rows"] * case["d"]
        packed = n / 2 + case["rows"] * -(-case["d"] // 32)
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 2 * packed, "flops": 2 * n}
    if k == "mx_linear":
        T, C, d = case["T"], case["C"], case["d"]
        s = SIZE[case["dtype"]]
        return {"bytes": T * d * s + C * (d / 2 + -(-d // 32)) + T * C * s
                + (4 * C if case["bias"] else 0), "flops": 2 * T * C * d}
    row = case["dim"] * case["bits"] // 8 + 4
    if k == "cache":
        n = case["T"] * 2 * case["heads"]
        return {"bytes": 2 * n * (case["dim"] * SIZE[case["dtype"]] + row) + 16 * case["T"],
                "flops": 4 * n * case["dim"]}
    lens = _lengths(case)
    if case["window"]:
        lens = [min(v, case["window"]) for v in lens]
    n, hq = sum(lens), case["heads"] * case["group"]
    return {"bytes": n * 2 * case["heads"] * row + 2 * case["B"] * hq * case["dim"] * 2,
            "flops": 4 * n * hq * case["dim"]}


# ---------------------------------------------------------------------------------------------
# What a program has in hand


def _lengths(case):
    """Every sequence's length: all the same, or spread over the logarithm (0 and 1 among them)."""
    B, top = case["B"], case["length"]
    if case["spread"] == "all":
        return [top] * B
    got = [max(1, int(round(top ** ((i + 0.5) / B)))) for i in range(B)]
    got[-1] = top
    if B > 2:
        got[0] = 0
    return [got[(i * 37) % B] if math.gcd(37, B) == 1 else got[i] for i in range(B)]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _activations(gen, rows, d):
    """Hidden states: normal rows, each channel with its own size, a few channels far larger."""
    x = torch.randn(rows, d, generator=gen, device=DEV)
    size = torch.exp(0.5 * torch.randn(d, generator=gen, device=DEV))
    size[torch.randint(0, d, (max(1, d // 200),), generator=gen, device=DEV)] *= 20
    return x * size


def _mx_encode(x):
    """(codes [rows][d'] uint8, exponents [rows][d'/32] int32) of fp32 rows, d' = d up to 128."""
    rows, d = x.shape
    x = torch.nn.functional.pad(x, (0, -d % 128)).view(rows, -1, 32)
    amax = x.abs().amax(2)
    e = torch.frexp(amax)[1].to(torch.int32) - 3
    e = torch.where(amax > 0, e, -127).clamp(-127, 125)
    a = x.abs() * ((127 - e) << 23).view(torch.float32)[..., None]
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    v = ((a / step).round() * step).clamp(max=6.0)
    code = torch.where(v < 2, 2 * v, torch.where(v < 4, v + 2, v / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(x).to(torch.uint8) << 3)
    return code.view(rows, -1), e


def _mx_decode(code, e):
    """The fp32 values of codes and exponents."""
    rows = code.shape[0]
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=code.device)
    v = level[code.int()].view(rows, -1, 32) * 0.5 * ((e + 128) << 23).view(torch.float32)[..., None]
    return v.view(rows, -1)


def _mx_pack(x):
    """The packed form of mpq_mx_layout: two codes a byte, the first in the low half, rows of d'/2
    bytes; from the next multiple of 512 bytes on the scales' biased exponents, 512 bytes for each
    128 rows x 4 blocks: row m's 4 bytes at 16 (m % 32) + 4 (m / 32)."""
    code, e = _mx_encode(x)
    rows, dp = code.shape
    codes = (code[:, 0::2] | (code[:, 1::2] << 4)).flatten()
    codes = torch.nn.functional.pad(codes, (0, -codes.numel() % 512))
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, 0, 0, -rows % 128))
    s = s.view(-1, 4, 32, dp // 128, 4).permute(0, 3, 2, 1, 4)
    return torch.cat([codes, s.flatten()])


def _mx_unpack(packed, rows, d):
    """The fp32 values of a packed matrix."""
    dp = d + -d % 128
    n = rows * dp // 2
    b = packed[:n].view(rows, dp // 2)
    code = torch.stack([b & 15, b >> 4], 2).view(rows, dp)
    s = packed[n + -n % 512:].view(-1, dp // 128, 32, 4, 4).permute(0, 3, 2, 1, 4)
    e = s.reshape(-1, dp // 32)[:rows].to(torch.int32) - 127
    return _mx_decode(code, e)[:, :d]


def _cache_encode(x, bits):
    """(codes q + 2^(bits-1), scales) of rows x [..., D]: s = max|x| / Qmax, q = rint(x / s)."""
    qmax = (1 << (bits - 1)) - 1
    s = x.abs().amax(-1) / qmax
    q = (x / s[..., None]).round().clamp(-qmax, qmax)
    q = torch.where(s[..., None] > 0, q, torch.zeros_like(q))
    return (q + (qmax + 1)).to(torch.uint8), s


def _cache_store(x, bits):
    """The stored rows [..., D bits / 8] and scales of x: 4-bit codes two a byte, low half first."""
    u, s = _cache_encode(x, bits)
    return (u if bits == 8 else u[..., 0::2] | (u[..., 1::2] << 4)), s


def _cache_values(rows, s, bits):
    """The fp32 values of stored rows."""
    if bits == 4:
        rows = torch.stack([rows & 15, rows >> 4], -1).flatten(-2)
    return (rows.to(torch.float32) - (1 << (bits - 1))) * s[..., None]


def _keys_values(gen, n, heads, dim):
    """K and V rows of n tokens, [n][2][heads][dim]: keys with a few large channels, tokens of
    different sizes."""
    x = torch.randn(n, 2, heads, dim, generator=gen, device=DEV)
    size = torch.exp(0.3 * torch.randn(heads, dim, generator=gen, device=DEV))
    x[:, 0] *= size / size.square().mean(1, keepdim=True).sqrt()
    x *= torch.exp(0.2 * torch.randn(n, 2, heads, 1, generator=gen, device=DEV))
    return x


def prepare(case, seed):
    gen, k = _gen(seed), case["kind"]
    dt = TYPES[case["dtype"]]
    if k == "mx_quantize":
        return dict(case=case, x=_activations(gen, case["rows"], case["d"]).to(dt))
    if k == "mx_linear":
        w = 0.02 * torch.randn(case["C"], case["d"], generator=gen, device=DEV)
        bias = torch.randn(case["C"], generator=gen, device=DEV) if case["bias"] else None
        return dict(case=case, x=_activations(gen, case["T"], case["d"]).to(dt), w=_mx_pack(w),
                    bias=bias)
    heads, dim, bits, page = case["heads"], case["dim"], case["bits"], case["page"]
    width = dim * bits // 8
    if k == "cache":
        T = case["T"]
        kv = _keys_values(gen, T, heads, dim).to(dt)
        pages = 2 * -(-T // page) + 1
        slots = torch.randperm(pages * page, generator=gen, device=DEV)[:T]
        codes = torch.zeros(pages, 2, heads, page, width, dtype=torch.uint8, device=DEV)
        scales = torch.zeros(pages, 2, heads, page, device=DEV)
        return dict(case=case, k=kv[:, 0], v=kv[:, 1], slots=slots, codes=codes, scales=scales)
    lens = _lengths(case)
    need = [-(-n // page) for n in lens]
    per = max(1, max(need))
    pages = sum(need) + 3
    # what no sequence holds: any codes, and scales that must not reach an output
    codes = torch.randint(0, 256, (pages, 2, heads, page, width), generator=gen, device=DEV,
                          dtype=torch.uint8)
    scales = torch.full((pages, 2, heads, page), math.nan, device=DEV)
    order = torch.randperm(pages, generator=gen, device=DEV)[:sum(need)]
    table = torch.full((case["B"], per), -1, dtype=torch.int32, device=DEV)
    cols = torch.arange(per, device=DEV)
    held = cols[None] < torch.tensor(need, device=DEV)[:, None]
    table[held] = order.to(torch.int32)
    n = sum(need) * page
    step = max(page, (1 << 26) // (heads * dim) // page * page)
    at = torch.arange(per * page, device=DEV)[None].expand(case["B"], -1)
    inside = (at < torch.tensor(lens, device=DEV)[:, None]).view(case["B"], per, page)[held]
    for i in range(0, n, step):
        m = min(step, n - i)
        rows, s = _cache_store(_keys_values(gen, m, heads, dim), bits)
        to = order[i // page:(i + m) // page]
        live = inside[i // page:(i + m) // page]
        codes[to] = rows.view(-1, page, 2, heads, width).permute(0, 2, 3, 1, 4).contiguous()
        s = s.view(-1, page, 2, heads).permute(0, 2, 3, 1)
        scales[to] = torch.where(live[:, None, None], s, math.nan)
    q = 2 * torch.randn(case["B"], heads * case["group"], dim, generator=gen, device=DEV)
    return dict(case=case, q=q.to(dt), codes=codes, scales=scales, table=table,
                lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
                workspace=torch.zeros(WORKSPACE, dtype=torch.uint8, device=DEV))


# ---------------------------------------------------------------------------------------------
# One pass


def _plain(state):
    case, k = state["case"], state["case"]["kind"]
    dt = TYPES[case["dtype"]]
    if k == "mx_quantize":
        return _mx_decode(*_mx_encode(state["x"].float()))[:, :case["d"]].to(dt)
    if k == "mx_linear":
        x = _mx_decode(*_mx_encode(state["x"].float()))[:, :case["d"]]
        y = x @ _mx_unpack(state["w"], case["C"], case["d"]).T
        return (y if state["bias"] is None else y + state["bias"]).to(dt)
    bits, page = case["bits"], case["page"]
    if k == "cache":
        page_of, at = state["slots"] // page, state["slots"] % page
        kv = torch.stack([state["k"], state["v"]], 1).float()
        rows, s = _cache_store(kv, bits)
        state["codes"][page_of, :, :, at] = rows
        state["scales"][page_of, :, :, at] = s
        back = _cache_values(state["codes"][page_of, :, :, at], state["scales"][page_of, :, :, at],
                             bits).to(dt)
        return {"k": back[:, 0], "v": back[:, 1]}
    B, heads, dim = case["B"], case["heads"], case["dim"]
    at = state["table"].clamp(min=0).long()
    L = at.shape[1] * page
    t = torch.arange(L, device=DEV)[None]
    lens = state["lens"][:, None]
    seen = (t < lens) & (state["table"] >= 0).repeat_interleave(page, 1)
    if case["window"]:
        seen &= t >= lens - case["window"]
    both = []
    for i in (0, 1):
        x = _cache_values(state["codes"][at, i], state["scales"][at, i], bits)
        x = x.permute(0, 2, 1, 3, 4).reshape(B, heads, L, dim)
        both.append(torch.where(seen[:, None, :, None], x, 0.0))
    q = state["q"].float().view(B, heads, -1, dim) / math.sqrt(dim)
    s = torch.where(seen[:, None, None], q @ both[0].transpose(2, 3), -math.inf)
    top = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(3, keepdim=True)
    o = (p @ both[1]) / torch.where(total > 0, total, 1.0)
    return o.view(B, -1, dim).to(dt)


def _own(state):
    from paper_2002_09049_gb300 import binding

    case, k = state["case"], state["case"]["kind"]
    dt = TYPES[case["dtype"]]
    if k == "mx_quantize":
        layout = binding.mpq_mx_layout(case["rows"], case["d"])
        packed = binding.mpq_mx_quantize(state["x"], layout)
        return binding.mpq_mx_dequantize(packed, layout, dtype=dt)
    if k == "mx_linear":
        x_layout = binding.mpq_mx_layout(case["T"], case["d"])
        w_layout = binding.mpq_mx_layout(case["C"], case["d"])
        x = binding.mpq_mx_quantize(state["x"], x_layout)
        return binding.mpq_mx_linear(x, x_layout, state["w"], w_layout, bias=state["bias"], dtype=dt)
    layout = binding.mpq_cache_layout(state["codes"].shape[0], case["page"], case["heads"],
                                      case["dim"], case["bits"])
    if k == "cache":
        binding.mpq_cache_write(state["k"], state["v"], state["slots"], layout, state["codes"],
                                state["scales"])
        kk, vv = binding.mpq_cache_read(state["slots"], layout, state["codes"], state["scales"],
                                        dtype=dt)
        return {"k": kk, "v": vv}
    return binding.mpq_cache_attention(state["q"], state["table"], state["lens"], layout,
                                       state["codes"], state["scales"], window=case["window"],
                                       workspace=state["workspace"])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------
# The definitions in 64 bits


def _mx_exact(x):
    """Microscaled values by search among the levels' midpoints, in 64 bits."""
    rows, d = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -d % 32)).view(-1, 32)
    top = x.abs().amax(1, keepdim=True)
    e = (torch.frexp(top)[1] - 3).clamp(min=-127)
    unit = torch.pow(torch.full_like(top, 2.0), e)
    a = x.abs() / unit
    level = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    mid = (level[1:] + level[:-1]) / 2
    below, above = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)
    at = torch.where(below % 2 == 0, below, above)      # a tie goes to the even code
    return (torch.sign(x) * level[at] * unit).view(rows, -1)[:, :d]


def _mx_matrix(packed, rows, d):
    """A packed matrix in 64 bits, entry by entry."""
    dp = (d + 127) // 128 * 128
    r = torch.arange(rows, device=packed.device)[:, None]
    j = torch.arange(d, device=packed.device)[None]
    byte = packed[r * (dp // 2) + j // 2].long()
    code = torch.where(j % 2 == 0, byte % 16, byte // 16)
    base = (rows * (dp // 2) + 511) // 512 * 512
    tile = (r // 128) * (dp // 128) + j // 128
    m = r % 128
    e = packed[base + tile * 512 + (m % 32) * 16 + (m // 32) * 4 + (j % 128) // 32].double() - 127
    level = torch.tensor(LEVELS, dtype=torch.float64, device=packed.device)[code % 8]
    return torch.where(code < 8, level, -level) * torch.exp2(e)


def _rows_exact(x, bits):
    """A cache row's values in 64 bits: the scale is the fp32 one that the cache holds."""
    qmax = 2 ** (bits - 1) - 1
    s = (x.double().abs().amax(-1, keepdim=True) / qmax).float().double()
    q = torch.clamp(torch.round((x.double() / s).float().double()), -qmax, qmax)
    return torch.where(s > 0, q, 0.0) * s


def exact(case, seed):
    state, k = prepare(case, seed), case["kind"]
    if k == "mx_quantize":
        return _mx_exact(state["x"])
    if k == "mx_linear":
        y = _mx_exact(state["x"]) @ _mx_matrix(state["w"], case["C"], case["d"]).T
        return y if state["bias"] is None else y + state["bias"].double()
    if k == "cache":
        return {"k": _rows_exact(state["k"], case["bits"]), "v": _rows_exact(state["v"], case["bits"])}
    B, heads, dim, bits, page = (case[n] for n in ("B", "heads", "dim", "bits", "page"))
    o = torch.zeros(B, heads * case["group"], dim, dtype=torch.float64, device=DEV)
    half = 2 ** (bits - 1)
    for b, n in enumerate(_lengths(case)):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            continue
        t = torch.arange(first, n, device=DEV)
        p, at = state["table"][b].long()[t // page], t % page
        for h in range(heads):
            kv = []
            for i in (0, 1):
                rows = state["codes"][p, i, h, at]
                if bits == 4:
                    rows = torch.stack([rows % 16, rows // 16], 2).view(len(t), dim)
                kv.append((rows.double() - half) * state["scales"][p, i, h, at].double()[:, None])
            q = state["q"][b, h * case["group"]:(h + 1) * case["group"]].double()
            w = torch.softmax(q @ kv[0].T / math.sqrt(dim), 1)
            o[b, h * case["group"]:(h + 1) * case["group"]] = w @ kv[1]
    return o
