"""The cases the rest of a few-bit decode step is measured on, through the public entry points.

  quantize  a weight matrix to 4-bit integers with a scale for each group of 32, 64 or 128 of a row,
            and the values they stand for: mpq_g4_quantize, mpq_g4_dequantize
  linear    a linear layer with weights in that form and inputs of 16 bits, from one token to a
            prompt: mpq_g4_linear
  rotate    queries' and keys' norms for each head with the position rotation: mpq_rotate
  extend    room for new tokens of every request of a paged cache, their slots and positions:
            mpq_pages_extend
  trim      requests cut back to the tokens they keep, their pages returned: mpq_pages_trim

Each has a plain form (elementary torch operations), taken where ``own`` is false, and ``exact``
restates its definition in 64 bits.  Sizes are those of the large linear layers and of the attention
block among the repository's workloads, and generic ones around them.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
SEVENTH = float(torch.tensor(1.0 / 7.0, dtype=torch.float32))        # the fp32 reciprocals
FIFTEENTH = float(torch.tensor(1.0 / 15.0, dtype=torch.float32))
EPS = 1e-6


# ---------------------------------------------------------------------------------------------
# The cases


def _quantize(rows, d, group, zeros, dtype):
    return dict(kind="quantize", rows=rows, d=d, group=group, zeros=zeros, dtype=dtype)


def _linear(T, C, d, group, zeros, dtype, bias=False):
    return dict(kind="linear", T=T, C=C, d=d, group=group, zeros=zeros, dtype=dtype, bias=bias)


def _rotate(T, q_heads, heads, dim, rot, pairs, norm, far, dtype):
    return dict(kind="rotate", T=T, q_heads=q_heads, heads=heads, dim=dim, rot=rot, pairs=pairs,
                norm=norm, far=far, dtype=dtype)


def _extend(B, length, add, most, page, room):
    return dict(kind="extend", B=B, length=length, add=add, most=most, page=page, room=room)


def _trim(B, length, keep, page):
    return dict(kind="trim", B=B, length=length, keep=keep, page=page)


def listed():
    return [
        # one projection's weights while a model is loaded
        dict(_quantize(4096, 4096, 64, True, "bf16"), name="quantize_4096x4096_zeros"),
        # the widening layer's weights
        dict(_quantize(11008, 4096, 128, False, "fp32"), name="quantize_11008x4096_fp32"),
        # one token through a square layer: latency and the weights' bytes
        dict(_linear(1, 4096, 4096, 128, False, "bf16"), name="linear_1x4096x4096"),
        # a few tokens of a small batch through the widening layer, with zero points and a bias
        dict(_linear(5, 11008, 4096, 64, True, "fp16", True), name="linear_5x11008x4096"),
        # an odd decode batch through the narrowing layer, small groups
        dict(_linear(75, 4096, 11008, 32, False, "bf16"), name="linear_75x4096x11008"),
        # a prompt through the widening layer
        dict(_linear(2048, 11008, 4096, 128, False, "bf16"), name="linear_2048x11008x4096"),
        # a decode batch's queries and keys
        dict(_rotate(48, 32, 8, 128, 128, "halves", True, 131072, "bf16"), name="rotate_48_tokens"),
        # a packed batch of prompts
        dict(_rotate(8192, 32, 8, 128, 128, "halves", True, 4096, "bf16"), name="rotate_8192_tokens"),
        # one more token for every sequence of a serving batch
        dict(_extend(96, 4096, "one", 1, 16, "enough"), name="extend_96_by_one"),
        # prompts of ragged lengths admitted together, more than the pool can hold
        dict(_extend(1024, 2048, "prompts", 4096, 64, "short"), name="extend_1024_prompts"),
        # drafted tokens that were not accepted
        dict(_trim(96, 4096, "drafts", 16), name="trim_96_drafts"),
        # half of many requests done
        dict(_trim(2048, 16384, "done", 16), name="trim_2048_done"),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer's width: any whole number, or (three times in four) a multiple of 64."""
    d = _log(rng, lo, hi)
    return d if rng.random() < 0.25 else max(64, d // 64 * 64)


def draw(rng):
    kind = rng.choice(("quantize", "linear", "linear", "linear", "rotate", "rotate", "extend", "trim"))
    group, zeros = rng.choice((32, 64, 128)), rng.random() < 0.5
    if kind == "quantize":
        d = _width(rng, 33, 11008)
        return _quantize(_log(rng, 1, max(1, 11008 * 4096 // d)), d, group, zeros,
                         rng.choice(("bf16", "fp16", "fp32")))
    if kind == "linear":
        d, C = _width(rng, 64, 11008), _width(rng, 64, 11008)
        T = _log(rng, 1, max(1, min(4096, 2048 * 4096 * 11008 // (C * d))))
        return _linear(T, C, d, group, zeros, rng.choice(("bf16", "bf16", "fp16")), rng.random() < 0.5)
    if kind == "rotate":
        dim = rng.choice((64, 80, 96, 128, 128, 256))
        heads, each = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 5, 8))
        rot = rng.choice((dim, dim, dim // 2))
        T = _log(rng, 1, max(1, 8192 * 40 * 128 // (heads * (each + 1) * dim)))
        return _rotate(T, heads * each, heads, dim, rot, rng.choice(("halves", "halves", "neighbours")),
                       rng.random() < 0.75, _log(rng, 64, 1 << 20), rng.choice(("bf16", "bf16", "fp16", "fp32")))
    B, page = _log(rng, 1, 4096), rng.choice((16, 16, 32, 64))
    length = _log(rng, 1, max(1, min(131072, (1 << 25) // B)))
    if kind == "trim":
        return _trim(B, length, rng.choice(("drafts", "done")), page)
    add, most = rng.choice((("one", 1), ("drafts", 8), ("prompts", 0)))
    if add == "prompts":
        most = _log(rng, 2, max(2, min(131072, (1 << 22) // B)))
    return _extend(B, length, add, most, page, rng.choice(("enough", "enough", "short")))


def _packed_bytes(rows, d, group, zeros):
    return rows * d / 2 + rows * -(-d // group) * (3 if zeros else 2)


def work(case):
    k = case["kind"]
    if k == "quantize":
        n = case["rows"] * case["d"]
        packed = _packed_bytes(case["rows"], case["d"], case["group"], case["zeros"])
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 2 * packed, "flops": 4 * n}
    if k == "linear":
        T, C, d = case["T"], case["C"], case["d"]
        return {"bytes": (T * d + T * C) * SIZE[case["dtype"]]
                + _packed_bytes(C, d, case["group"], case["zeros"]) + (4 * C if case["bias"] else 0),
                "flops": 2 * T * C * d}
    if k == "rotate":
        n = case["T"] * (case["q_heads"] + case["heads"])
        return {"bytes": 2 * n * case["dim"] * SIZE[case["dtype"]] + 4 * case["T"],
                "flops": n * (3 * case["rot"] + (4 * case["dim"] if case["norm"] else 0))}
    B, page = case["B"], case["page"]
    lens = _lengths(B, case["length"])
    if k == "extend":
        add = _added(case)
        N = sum(add)
        need = sum(-(-(n + a) // page) - -(-n // page) for n, a in zip(lens, add))
        return {"bytes": 4 * B * 5 + 8 * need + 12 * N, "flops": N}
    freed = sum(-(-n // page) - -(-k // page) for n, k in zip(lens, _kept(case)))
    return {"bytes": 4 * B * 3 + 8 * freed, "flops": B}


# ---------------------------------------------------------------------------------------------
# What a program has in hand


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _lengths(B, top):
    """The requests' lengths, spread over the logarithm; 0 among those of several."""
    got = [max(1, int(round(top ** ((i + 0.5) / B)))) for i in range(B)]
    got[-1] = top
    if B > 2:
        got[0] = 0
    return [got[(i * 37) % B] if math.gcd(37, B) == 1 else got[i] for i in range(B)]


def _added(case):
    """The new tokens of every request."""
    B, most = case["B"], case["most"]
    if case["add"] == "one":
        return [1] * B
    if case["add"] == "drafts":
        return [1 + (i * 5 + 3) % most for i in range(B)]
    # prompts: none for a third of the requests
    return [0 if i % 3 == 1 and B > 1 else max(1, int(round(most ** (((i * 29) % B + 1) / B))))
            for i in range(B)]


def _kept(case):
    """The tokens every request keeps."""
    lens = _lengths(case["B"], case["length"])
    if case["keep"] == "drafts":
        return [max(0, n - (i * 5) % 9) for i, n in enumerate(lens)]
    return [n if i % 2 else 0 for i, n in enumerate(lens)]


def _activations(gen, rows, d):
    """Hidden states: normal rows, each channel with its own size, a few channels far larger."""
    x = torch.randn(rows, d, generator=gen, device=DEV)
    size = torch.exp(0.5 * torch.randn(d, generator=gen, device=DEV))
    size[torch.randint(0, d, (max(1, d // 200),), generator=gen, device=DEV)] *= 20
    return x * size


def _g4_encode(x, group, zeros):
    """(codes [rows][groups][group] int32, zero points and scales [rows][groups]) of fp32 rows."""
    rows, d = x.shape
    x = torch.nn.functional.pad(x, (0, -d % group)).view(rows, -1, group)
    if zeros:
        low, high = x.amin(2).clamp(max=0.0), x.amax(2).clamp(min=0.0)
        s = (high * FIFTEENTH - low * FIFTEENTH).to(torch.bfloat16).float()
        z = torch.where(s > 0, (-low / s).round().clamp(0, 15), 8.0)
        q = ((x / s[..., None]).round() + z[..., None]).clamp(0, 15)
    else:
        s = (x.abs().amax(2) * SEVENTH).to(torch.bfloat16).float()
        z = torch.full_like(s, 8.0)
        q = (x / s[..., None]).round().clamp(-7, 7) + 8
    q = torch.where(s[..., None] > 0, q, z[..., None])
    return q.int(), z.int(), s


def _g4_values(q, z, s, d):
    return ((q - z[..., None]).float() * s[..., None]).flatten(1)[:, :d]


def _g4_pack(x, group, zeros):
    """The packed form of mpq_g4_layout: tiles of 16 rows x 128 elements, those of 16 rows one after
    another along the row.  A tile holds [16][64] bytes of codes -- word 4 i + m of a row has elements
    32 m + 8 i .. + 7, the even ones in its low half --, [16][128 / group] bf16 scales and, with zeros, as
    many bytes of zero points."""
    rows, d = x.shape
    x = torch.nn.functional.pad(x, (0, -d % 128, 0, -rows % 16))
    q, z, s = _g4_encode(x, group, zeros)
    rt, kt = x.shape[0] // 16, x.shape[1] // 128
    w = q.view(rt, 16, kt, 4, 4, 8).permute(0, 2, 1, 4, 3, 5)
    order = torch.tensor([0, 4, 1, 5, 2, 6, 3, 7], device=x.device)      # nibble of each element
    w = (w.long() << (4 * order)).sum(5)
    w = torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32).contiguous()
    parts = [w.view(rt, kt, -1).view(torch.uint8)]
    per = lambda t: t.view(rt, 16, kt, 128 // group).permute(0, 2, 1, 3).contiguous().view(rt, kt, -1)
    parts.append(per(s.to(torch.bfloat16)).view(torch.uint8))
    if zeros:
        parts.append(per(z.to(torch.uint8)))
    return torch.cat(parts, 2).flatten()


def _g4_unpack(packed, C, d, group, zeros):
    """(codes, zero points, scales) of a packed matrix, as _g4_encode's."""
    rt, kt, n = -(-C // 16), -(-d // 128), 128 // group
    p = packed.view(rt, kt, -1)
    w = p[:, :, :1024].contiguous().view(torch.int32).view(rt, kt, 16, 4, 4, 1).permute(0, 2, 1, 4, 3, 5)
    shift = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], dtype=torch.int32, device=p.device)
    q = ((w >> shift) & 15).reshape(rt * 16, kt * n, group)[:C]
    back = lambda t: t.view(rt, kt, 16, n).permute(0, 2, 1, 3).reshape(rt * 16, kt * n)[:C]
    s = back(p[:, :, 1024:1024 + 32 * n].contiguous().view(torch.bfloat16)).float()
    z = back(p[:, :, 1024 + 32 * n:]).int() if zeros else torch.full_like(s, 8.0).int()
    return q, z, s


def _requests(case, gen, lens, cols, held, spare):
    """Every request's pages (none told twice), and the pool of those left."""
    B = case["B"]
    pages = sum(held) + spare
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
    inside = torch.arange(cols, device=DEV)[None] < torch.tensor(held, device=DEV)[:, None]
    table[inside] = order[:sum(held)]
    pool = torch.full((pages,), -1, dtype=torch.int32, device=DEV)
    pool[:spare] = order[sum(held):]
    free = torch.tensor([spare, 0], dtype=torch.int32, device=DEV)
    return dict(table=table, pool=pool, free=free, lens=torch.tensor(lens, dtype=torch.int32, device=DEV))


def prepare(case, seed):
    gen, k = _gen(seed), case["kind"]
    if k == "quantize":
        w = 0.02 * torch.randn(case["rows"], case["d"], generator=gen, device=DEV)
        w *= torch.exp(0.3 * torch.randn(case["rows"], 1, generator=gen, device=DEV))
        if case["zeros"]:
            w += 0.01 * torch.randn(case["rows"], 1, generator=gen, device=DEV)
        return dict(case=case, x=w.to(TYPES[case["dtype"]]))
    if k == "linear":
        w = 0.02 * torch.randn(case["C"], case["d"], generator=gen, device=DEV)
        bias = torch.randn(case["C"], generator=gen, device=DEV) if case["bias"] else None
        x = _activations(gen, case["T"], case["d"]).to(TYPES[case["dtype"]])
        return dict(case=case, x=x, w=_g4_pack(w, case["group"], case["zeros"]), bias=bias)
    if k == "rotate":
        T, hq, h, dim, dt = case["T"], case["q_heads"], case["heads"], case["dim"], TYPES[case["dtype"]]
        rows = (_activations(gen, T, (hq + 2 * h) * dim)).to(dt).view(T, hq + 2 * h, dim)
        q, key, _ = rows.split((hq, h, h), 1)
        # packed sequences: runs of consecutive positions
        at = torch.arange(T, device=DEV)
        start = torch.randint(0, case["far"], (T,), generator=gen, device=DEV)
        run = max(1, T // 8) if T > 256 else 1
        pos = ((start[at // run] + at % run) % case["far"]).to(torch.int32)
        pos[0] = case["far"] - 1
        freq = 10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])
        mk = lambda: 1 + 0.2 * torch.randn(dim, generator=gen, device=DEV) if case["norm"] else None
        state = dict(case=case, q=q, k=key, pos=pos, freq=freq.to(DEV), q_weight=mk(), k_weight=mk())
        if own:
            from paper_2002_09049_gb300 import binding
            state["turns"] = binding.mpq_rotation(freq.tolist(), device=DEV)
        return state
    page, lens = case["page"], _lengths(case["B"], case["length"])
    held = [-(-n // page) for n in lens]
    if k == "trim":
        state = _requests(case, gen, lens, max(1, max(held)), held, 7)
        state["keep"] = torch.tensor(_kept(case), dtype=torch.int32, device=DEV)
        return dict(state, case=case)
    add = _added(case)
    need = [-(-(n + a) // page) - h for n, a, h in zip(lens, add, held)]
    cols = max(1, max(h + m for h, m in zip(held, need)))
    spare = sum(need) + 3 if case["room"] == "enough" else sum(need) * 7 // 8
    state = _requests(case, gen, lens, cols, held, spare)
    state["add"] = torch.tensor(add, dtype=torch.int32, device=DEV)
    N = sum(add) if case["add"] == "one" else -(-sum(add) // 64) * 64     # a buffer of whole tiles
    return dict(state, case=case, N=N)


# ---------------------------------------------------------------------------------------------
# One pass


def _plain_rotate(x, cos, sin, weight, case):
    x = x.float()
    if case["norm"]:
        x = x / torch.sqrt(x.square().mean(2, keepdim=True) + EPS) * weight
    r = case["rot"]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if case["pairs"] == "halves" else (x[..., 0:r:2], x[..., 1:r:2])
    a, b = a * cos - b * sin, b * cos + a * sin
    y = torch.cat([a, b], 2) if case["pairs"] == "halves" else torch.stack([a, b], 3).flatten(2)
    return torch.cat([y, x[..., r:]], 2).to(TYPES[case["dtype"]])


def _plain_extend(state):
    case, page, N = state["case"], state["case"]["page"], state["N"]
    lens, add = state["lens"].long(), state["add"].long().clamp(min=0)
    table, pool, free = state["table"], state["pool"].long(), state["free"][0].long()
    B, cols = table.shape
    end = add.cumsum(0)
    held = (lens + page - 1) // page
    need = (lens + add + page - 1) // page - held
    fits = (lens + add <= cols * page) & (end <= N)
    need = torch.where(fits, need, 0)
    upto = need.cumsum(0)
    given = fits & ((need == 0) | (upto <= free))
    taken = torch.where(given, add, 0)
    need = torch.where(given, need, 0)
    # new pages into the table: the j-th page given is the j-th from the pool's end
    col = torch.arange(cols, device=DEV)[None]
    new = (col >= held[:, None]) & (col < (held + need)[:, None])
    j = upto[:, None] - need[:, None] + col - held[:, None]
    page_of = pool[(free - 1 - j).clamp(0, pool.numel() - 1)]
    table.copy_(torch.where(new, page_of, table.long()))
    # the packed tokens
    t = torch.arange(N, device=DEV)
    b = (torch.searchsorted(end, t, right=True)).clamp(max=B - 1)
    inside = t < end[-1]
    pos = lens[b] + t - (end - add)[b]
    at = table[b, (pos // page).clamp(0, cols - 1)].long()
    slots = torch.where(inside & given[b] & (at >= 0), at * page + pos % page, -1)
    pos = torch.where(inside, pos, 0)
    left = free - need.sum()
    return {"slots": slots, "positions": pos.int(), "taken": taken.int(), "table": table,
            "lens": (lens + taken).int(), "free": left.int()}


def _plain_trim(state):
    page = state["case"]["page"]
    lens, pool, free, table = state["lens"].long(), state["pool"], state["free"][0].long(), state["table"]
    keep = torch.minimum(state["keep"].long().clamp(min=0), lens)
    first, held = (keep + page - 1) // page, (lens + page - 1) // page
    back = held - first
    before = back.cumsum(0) - back
    total = back.sum()
    col = torch.arange(table.shape[1], device=DEV)[None]
    gone = (col >= first[:, None]) & (col < held[:, None])
    # the j-th page returned goes to place free + total - 1 - j: the order in which it would be given again
    to = torch.where(gone, free + total - 1 - (before[:, None] + col - first[:, None]), pool.numel())
    room = torch.cat([pool, pool[:1]])
    room.scatter_(0, to.flatten(), table.flatten())
    pool.copy_(room[:-1])
    return {"pool": pool, "lens": keep.int(), "free": (free + total).int()}


def _plain(state):
    case, k = state["case"], state["case"]["kind"]
    if k == "extend":
        return _plain_extend(state)
    if k == "trim":
        return _plain_trim(state)
    dt = TYPES[case["dtype"]]
    if k == "quantize":
        return _g4_values(*_g4_encode(state["x"].float(), case["group"], case["zeros"]), case["d"]).to(dt)
    if k == "linear":
        w = _g4_values(*_g4_unpack(state["w"], case["C"], case["d"], case["group"], case["zeros"]), case["d"])
        y = state["x"].float() @ w.T
        return (y if state["bias"] is None else y + state["bias"]).to(dt)
    angle = state["pos"].double()[:, None] * state["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    return {"q": _plain_rotate(state["q"], cos, sin, state["q_weight"], case),
            "k": _plain_rotate(state["k"], cos, sin, state["k_weight"], case)}


def run(state):
    if not own:
        return _plain(state)
    from paper_2002_09049_gb300 import binding
    case, k = state["case"], state["case"]["kind"]
    if k == "quantize":
        lay = binding.mpq_g4_layout(case["rows"], case["d"], case["group"], case["zeros"])
        packed = binding.mpq_g4_quantize(state["x"], lay)
        return binding.mpq_g4_dequantize(packed, lay, dtype=TYPES[case["dtype"]])
    if k == "linear":
        lay = binding.mpq_g4_layout(case["C"], case["d"], case["group"], case["zeros"])
        return binding.mpq_g4_linear(state["x"], state["w"], lay, bias=state["bias"],
                                     dtype=TYPES[case["dtype"]], exact=True)
    if k == "rotate":
        q, key = binding.mpq_rotate(state["q"], state["k"], state["pos"], state["turns"],
                                    norm=case["norm"], q_weight=state["q_weight"],
                                    k_weight=state["k_weight"], eps=EPS,
                                    neighbours=case["pairs"] == "neighbours")
        return {"q": q, "k": key}
    # lengths and the pool's count go to tensors of their own, so that a step can be taken back
    lens, free = torch.empty_like(state["lens"]), torch.empty_like(state["free"])
    if k == "extend":
        slots, pos, taken = binding.mpq_pages_extend(state["add"], state["lens"], state["table"],
                                                     state["pool"], state["free"], case["page"],
                                                     state["N"], new_lens=lens, new_count=free)
        return {"slots": slots, "positions": pos, "taken": taken, "table": state["table"],
                "lens": lens, "free": free[0]}
    binding.mpq_pages_trim(state["keep"], state["lens"], state["table"], state["pool"], state["free"],
                           case["page"], new_lens=lens, new_count=free)
    return {"pool": state["pool"], "lens": lens, "free": free[0]}


# ---------------------------------------------------------------------------------------------
# The definitions in 64 bits


def _group_exact(x, zeros):
    """One group's values of every row, x [rows][n] float64: scales in bf16, quotients as fp32 gives
    them, whole codes between."""
    if zeros:
        top, bottom = torch.clamp(x.max(1).values, min=0.0), torch.clamp(x.min(1).values, max=0.0)
        width = (top * FIFTEENTH).float().double() - (bottom * FIFTEENTH).float().double()
        s = width.float().to(torch.bfloat16).double()
        z = torch.clamp(torch.round((-bottom / s).float().double()), 0, 15)
        q = torch.round((x / s[:, None]).float().double())
        q = torch.minimum(torch.maximum(q, -z[:, None]), 15 - z[:, None])
    else:
        s = (x.abs().max(1).values * SEVENTH).float().to(torch.bfloat16).double()
        q = torch.clamp(torch.round((x / s[:, None]).float().double()), -7, 7)
    return torch.where(s[:, None] > 0, q * s[:, None], 0.0)


def _g4_matrix(packed, C, d, group, zeros):
    """A packed matrix in float64, from the layout's description: byte by byte of every tile."""
    kt = -(-d // 128)
    tiles = packed.view(-1, kt, packed.numel() // (-(-C // 16) * kt)).long()
    w = torch.empty(tiles.shape[0], 16, kt, 128, dtype=torch.float64, device=packed.device)
    for e in range(8):
        # element e of a word: byte e / 4 of its low (even e) or high half, low or high nibble
        byte, high = (e // 4) + 2 * (e % 2), (e // 2) % 2
        b = tiles[:, :, :1024].reshape(-1, kt, 16, 16, 4)[..., byte]
        b = (b // 16 if high else b % 16).double().permute(0, 2, 1, 3)
        for word in range(16):
            w[..., 32 * (word % 4) + 8 * (word // 4) + e] = b[..., word]
    n = 128 // group
    for g in range(n):
        at = slice(1024 + 2 * g, 1024 + 32 * n, 2 * n)
        high = slice(1024 + 2 * g + 1, 1024 + 32 * n, 2 * n)
        s = (tiles[:, :, at] + 256 * tiles[:, :, high]).to(torch.int32) << 16
        s = s.view(torch.float32).double().permute(0, 2, 1)[..., None]
        z = 8.0
        if zeros:
            z = tiles[:, :, 1024 + 32 * n + g::n].double().permute(0, 2, 1)[..., None]
        part = w[..., g * group:(g + 1) * group]
        part.copy_((part - z) * s)
    return w.view(-1, kt * 128)[:C, :d]


def _rotate_exact(x, pos, freq, weight, case):
    x = x.double()
    y = x.clone()
    if case["norm"]:
        y = x * weight.double() * torch.rsqrt((x * x).sum(2, keepdim=True) / x.shape[2] + EPS)
    out = y.clone()
    for i in range(case["rot"] // 2):
        j, m = (i, i + case["rot"] // 2) if case["pairs"] == "halves" else (2 * i, 2 * i + 1)
        turn = torch.polar(torch.ones_like(pos, dtype=torch.float64), pos.double() * freq[i])
        both = torch.complex(y[..., j], y[..., m]) * turn[:, None]
        out[..., j], out[..., m] = both.real, both.imag
    return out


def _pages_exact(state):
    """The page manager's steps one request after another."""
    import numpy as np
    case, page = state["case"], state["case"]["page"]
    lens, table, pool = (state[n].cpu().numpy().copy() for n in ("lens", "table", "pool"))
    free, cols = int(state["free"][0]), table.shape[1]
    back = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    if case["kind"] == "trim":
        returned = []
        for b, keep in enumerate(state["keep"].tolist()):
            keep = min(max(keep, 0), int(lens[b]))
            returned.extend(table[b, -(-keep // page):-(-int(lens[b]) // page)])
            lens[b] = keep
        pool[free:free + len(returned)] = returned[::-1]
        return {"pool": back(pool), "lens": back(lens),
                "free": torch.tensor(free + len(returned), dtype=torch.int32, device=DEV)}
    N = state["N"]
    slots, positions = np.full(N, -1, np.int64), np.zeros(N, np.int32)
    taken, at, asked, top = np.zeros(len(lens), np.int32), 0, 0, free
    for b, add in enumerate(state["add"].tolist()):
        add, n = max(add, 0), int(lens[b])
        held, whole = -(-n // page), -(-(n + add) // page)
        end = at + add
        ok = n + add <= cols * page and end <= N
        if ok:
            asked += whole - held
            ok = whole == held or asked <= free
        p = np.arange(n, n + add)
        positions[at:end] = p[:max(0, min(end, N) - at)]
        if ok:
            for c in range(held, whole):
                top -= 1
                table[b, c] = pool[top]
            slots[at:end] = table[b, p // page].astype(np.int64) * page + p % page
            taken[b], lens[b] = add, n + add
        at = end
    return {"slots": back(slots), "positions": back(positions), "taken": back(taken), "table": back(table),
            "lens": back(lens), "free": torch.tensor(top, dtype=torch.int32, device=DEV)}


def exact(case, seed):
    state, k = prepare(case, seed), case["kind"]
    if k in ("extend", "trim"):
        return _pages_exact(state)
    if k == "quantize":
        x = state["x"].double()
        return torch.cat([_group_exact(x[:, i:i + case["group"]], case["zeros"])
                          for i in range(0, case["d"], case["group"])], 1)
    if k == "linear":
        y = state["x"].double() @ _g4_matrix(state["w"], case["C"], case["d"], case["group"], case["zeros"]).T
        return y if state["bias"] is None else y + state["bias"].double()
    return {n: _rotate_exact(state[n], state["pos"], state["freq"], state[n + "_weight"], case)
            for n in ("q", "k")}
