"""Plain references (numpy, 64 bits) of 4-bit integer weights, the norm and rotation of queries and keys, and the
pages of a cache's requests, as include/mpq.h defines them."""
import numpy as np

GROUPS = (32, 64, 128)


def bf16(x):
    """fp32 to bf16, ties to even, as fp32 (finite values)."""
    u = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)


def g4_encode(x, group, zeros):
    """(codes [rows][padded d], zero points, scales [rows][groups]) of x [rows][d], whole tiles of 128 elements."""
    x = np.asarray(x, np.float32)
    rows, d = x.shape
    x = np.pad(x, ((0, 0), (0, -d % 128))).reshape(rows, -1, group)
    bad = ~np.isfinite(x).all(2)
    v = np.where(bad[..., None], np.float32(0), x)
    with np.errstate(all="ignore"):
        if zeros:
            c = np.float32(1) / np.float32(15)
            lo, hi = np.minimum(v.min(2), np.float32(0)), np.maximum(v.max(2), np.float32(0))
            s = bf16(hi * c - lo * c)
            z = np.where(s > 0, np.clip(np.rint(-lo / s), 0, 15), 8)
            q = np.clip(np.rint(v / s[..., None]) + z[..., None], 0, 15)
        else:
            s = bf16(np.abs(v).max(2) * (np.float32(1) / np.float32(7)))
            z = np.full(s.shape, 8)
            q = np.clip(np.rint(v / s[..., None]), -7, 7) + 8
    dead = bad | ~(s > 0)
    z = np.where(dead, 8, z)
    q = np.where(dead[..., None], 8, q)
    return q.astype(np.uint8).reshape(rows, -1), z.astype(np.uint8), np.where(bad, np.float32(np.nan), s)


def g4_values(q, z, s, d):
    """The values that codes stand for, in 64 bits."""
    group = q.shape[1] // s.shape[1]
    v = (q.astype(np.float64).reshape(len(q), -1, group) - z[..., None]) * s.astype(np.float64)[..., None]
    return v.reshape(len(q), -1)[:, :d]


def g4_pack(q, z, s, zeros):
    """The packed buffer, byte by byte of include/mpq.h's layout."""
    rows, dp = q.shape
    n, kt, rt = 128 * s.shape[1] // dp, dp // 128, -(-rows // 16)
    size = 1024 + (48 if zeros else 32) * n
    out = np.zeros((rt, kt, size), np.uint8)
    bits = s.astype(np.float32).view(np.uint32) >> 16
    for r in range(rt * 16):
        for t in range(kt):
            tile = out[r // 16, t]
            for w in range(16):
                word = 0
                for e in range(8):
                    code = int(q[r, 128 * t + 32 * (w % 4) + 8 * (w // 4) + e]) if r < rows else 8
                    word |= code << (4 * (e // 2) + 16 * (e % 2))
                at = (r % 16) * 64 + 4 * w
                tile[at:at + 4] = np.frombuffer(np.uint32(word).tobytes(), np.uint8)
            for g in range(n):
                i = (r % 16) * n + g
                b = int(bits[r, t * n + g]) if r < rows else 0
                tile[1024 + 2 * i], tile[1025 + 2 * i] = b & 255, b >> 8
                if zeros:
                    tile[1024 + 32 * n + i] = z[r, t * n + g] if r < rows else 8
    return out.reshape(-1)


def rotate(x, positions, freq, norm, weight, eps, neighbours):
    """(y, a bound on the magnitudes that went into each element) of rows x [T][heads][dim], positions as
    Python or 64-bit integers, all in 64 bits."""
    x = np.asarray(x, np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(2, keepdims=True) + np.float64(np.float32(eps)))
        if weight is not None:
            x = x * np.asarray(weight, np.float64)
    half = len(freq)
    angle = np.asarray(positions, np.float64)[:, None, None] * np.asarray(freq, np.float64)
    c, s = np.cos(angle), np.sin(angle)
    y, mag = x.copy(), np.abs(x)
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    mag[..., a] = mag[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, mag


def extend(add, lens, table, pool, count, page, N):
    """(slots, positions, taken, table, lens, count) after mpq_pages_extend, one request after another."""
    lens, table = lens.copy(), table.copy()
    cols, have = table.shape[1], min(max(int(count), 0), len(pool))
    slots, positions = np.full(N, -1, np.int64), np.zeros(N, np.int32)
    taken, at, asked, top = np.zeros(len(lens), np.int32), 0, 0, have
    for b, a in enumerate(add.tolist()):
        a, n = max(a, 0), int(lens[b])
        end = at + a
        ok = n >= 0 and n + a <= cols * page and end <= N
        if ok:
            held, whole = -(-n // page), -(-(n + a) // page)
            asked += whole - held
            ok = whole == held or asked <= have
        p = n + np.arange(max(0, min(end, N) - at))
        positions[at:min(end, N)] = p
        if ok:
            for c in range(held, whole):
                top -= 1
                table[b, c] = pool[top]
            of = table[b, p // page].astype(np.int64)
            slots[at:end] = np.where(of >= 0, of * page + p % page, -1)
            taken[b], lens[b] = a, n + a
        at = end
    return slots, positions, taken, table, lens, top


def trim(keep, lens, table, pool, count, page):
    """(lens, pool, count) after mpq_pages_trim."""
    cols, have = table.shape[1], min(max(int(count), 0), len(pool))
    pool, back, left = pool.copy(), [], []
    for b, k in enumerate(keep.tolist()):
        n = min(max(int(lens[b]), 0), page * cols)
        k = min(max(k, 0), n)
        back.extend(table[b, -(-k // page):-(-n // page)].tolist())
        left.append(k)
    for j, p in enumerate(reversed(back)):
        if have + j < len(pool):
            pool[have + j] = p
    return np.array(left, np.int32), pool, min(have + len(back), len(pool))
