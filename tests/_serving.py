"""Plain references of the few-bit serving operators in 64 bits (numpy), for the parity tests: the
microscaled 4-bit floats of include/mpq.h, the key-value cache's rows and the attention over them."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx_encode(x):
    """(codes [rows][d] 0..15, biased exponents [rows][ceil(d/32)]) of a float array."""
    x = np.asarray(x, np.float64)
    rows, d = x.shape
    nb = -(-d // 32)
    codes = np.zeros((rows, d), np.uint8)
    exps = np.zeros((rows, nb), np.uint8)
    for b in range(nb):
        blk = x[:, 32 * b:32 * b + 32]
        bad = ~np.isfinite(blk).all(1)
        top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(blk), blk, 0.0)).max(1))
        e = np.where(top > 0, np.frexp(top)[1] - 3, -127)
        e = np.maximum(e, -127)
        a = np.abs(np.where(bad[:, None], 0.0, blk)) / np.exp2(e.astype(np.float64))[:, None]
        dist = np.abs(a[..., None] - LEVELS)
        near = dist.min(-1, keepdims=True)
        tied = dist == near
        # of two levels at the same distance, the even code; past the last level, the last
        order = np.where(tied, np.arange(8) % 2, 2)
        code = order.argmin(-1)
        sign = np.signbit(blk) & ~bad[:, None]
        codes[:, 32 * b:32 * b + 32] = code + 8 * sign
        exps[:, b] = np.where(bad, 255, e + 127)
    return codes, exps


def mx_decode(codes, exps):
    v = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127))
    return v * np.repeat(s, 32, axis=1)[:, :codes.shape[1]]


def mx_pack(codes, exps):
    """The packed buffer of include/mpq.h's layout, byte by byte."""
    rows, d = codes.shape
    dp = -(-d // 128) * 128
    full = np.zeros((rows, dp), np.uint8)
    full[:, :d] = codes
    off = -(-(rows * dp // 2) // 512) * 512
    kt, rt = dp // 128, -(-rows // 128)
    out = np.zeros(off + rt * kt * 512, np.uint8)
    out[:rows * dp // 2] = (full[:, 0::2] | (full[:, 1::2] << 4)).ravel()
    for m in range(rows):
        for b in range(exps.shape[1]):
            out[off + ((m // 128) * kt + b // 4) * 512 + (m % 32) * 16 + (m % 128 // 32) * 4 + b % 4] = \
                exps[m, b]
    return out


def mx_unpack(packed, rows, d):
    """(codes, exps) of a packed buffer."""
    dp = -(-d // 128) * 128
    off = -(-(rows * dp // 2) // 512) * 512
    by = packed[:rows * dp // 2].reshape(rows, dp // 2)
    codes = np.stack([by & 15, by >> 4], 2).reshape(rows, dp)
    kt = dp // 128
    m, b = np.arange(rows)[:, None], np.arange(dp // 32)[None]
    at = off + ((m // 128) * kt + b // 4) * 512 + (m % 32) * 16 + (m % 128 // 32) * 4 + b % 4
    return codes[:, :d], packed[at][:, :-(-d // 32)], codes[:, d:], packed[at]


def cache_rows(x, bits):
    """(codes q, fp32 scales) of rows x [..., dim] (fp32 values), by the fp32 operations of Eq. 8."""
    qmax = np.float32(2 ** (bits - 1) - 1)
    x = np.asarray(x, np.float32)
    bad = ~np.isfinite(x).all(-1)
    with np.errstate(all="ignore"):
        s = np.abs(x).max(-1) * (np.float32(1) / qmax)      # the reciprocal rounded, one product
        s = np.where(bad, np.float32(np.nan), s)
        q = np.clip(np.rint(x / s[..., None]), -qmax, qmax)
    q = np.where((s > 0)[..., None], q, 0)
    return q.astype(np.int32), s


def attention(q, k, v, seen, scale):
    """(o, lse, sum p |v| / sum p, largest p |v| unit / sum p, spread of the scores) of one head: q [dim],
    k and v [n][dim], seen [n]; all in 64 bits."""
    dim = q.shape[0]
    if not seen.any():
        z = np.zeros(dim)
        return z, -np.inf, z, 0.0, 0.0
    k, v = k[seen], v[seen]
    s = scale * (k @ q)
    m = s.max()
    p = np.exp(s - m)
    L = p.sum()
    reach = float((np.abs(k) @ np.abs(q)).max() * abs(scale))
    unit = float((p * np.abs(v).max(1)).max()) / L
    return p @ v / L, m + np.log(L), p @ np.abs(v) / L, unit, reach
