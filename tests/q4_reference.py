"""The cache held in 4 bits, in plain numpy: what voxzip_q4_pack must hold bit for bit, the values rows stand for,
and the decode step and the eviction on those values in 64 bits. Written from the format's definition; it shares
no code with the package."""
import numpy as np

GROUP = 32


def bf16(x):
    """fp32 rounded to the nearest bf16 (ties to even), as fp32."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r)


def quantise(x):
    """Rows [..., D] fp32 -> scales [..., D / 32] (bf16 values), codes [..., D] in [-8, 7]."""
    g = np.asarray(x, np.float32).reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    with np.errstate(all="ignore"):
        hi, lo = g.max(-1), g.min(-1)
        s = bf16(np.where(hi >= -lo, hi, lo) * np.float32(-0.125))
        s = np.where(np.abs(s) < np.float32(2.0 ** -126), np.float32(0), s)
        s = np.where(np.isfinite(g).all(-1), s, np.float32(np.nan))
        c = np.clip(np.rint(g * (np.float32(1) / s)[..., None]), -8, 7)
        c = np.where(np.isfinite(s)[..., None] & (s != 0)[..., None], c, 0).astype(np.int32)
    return s.astype(np.float32), c.reshape(x.shape)


def channel_exponents(rows):
    """Rows [n][D] fp32 -> exponents [D]."""
    D = rows.shape[-1]
    if not len(rows):
        return np.zeros(D, np.int32)
    bits = np.abs(rows.astype(np.float32)).view(np.int32).max(0)  # ordered as the magnitudes, NaN above all
    mid = np.sort(bits)[(D - 1) // 2]
    top, m = bits.view(np.float32), mid.view(np.float32)
    with np.errstate(all="ignore"):
        r = (top / m * np.float32(np.sqrt(2.0))).astype(np.float32)
        e = np.clip((r.view(np.int32) >> 23) - 127, -16, 16)
    ok = (top > 0) & np.isfinite(top) & (m > 0) & np.isfinite(m)
    return np.where(ok, e, 0).astype(np.int32)


def k_nibbles(D):
    """Nibble of the row that channel d of K lies in."""
    J = D // GROUP
    return np.array([(d % 32 // 8 * J + d // 32) * 8 + d % 8 // 2 + 4 * (d % 2) for d in range(D)])


def v_nibbles(D):
    J = D // GROUP
    return np.array([(d % 32 // 4 * J + d // 32) * 4 + d % 4 for d in range(D)])


def to_bytes(codes, nibbles):
    D = codes.shape[-1]
    n = np.zeros(codes.shape, np.uint8)
    n[..., nibbles] = (codes + 8).astype(np.uint8)
    return n[..., 0::2] | n[..., 1::2] << 4


def from_bytes(data, nibbles):
    n = np.stack([data & 15, data >> 4], -1).reshape(data.shape[:-1] + (-1,))
    return n[..., nibbles].astype(np.int32) - 8


def values(codes, scales, exps=None):
    """What codes stand for, fp64."""
    x = codes.astype(np.float64) * np.repeat(scales.astype(np.float64), GROUP, -1)
    return x if exps is None else x * 2.0 ** exps


def decode_unit(q, k, v, score, gamma, scale):
    """q [G][D], k and v [n + 1][D] (the appended row last), score [n], all fp64. Returns out [G][D], score [n + 1],
    and what tolerances are made of: sum of p |v| per output, the largest sum of |q k| scale of a head."""
    x = q @ k.T * scale
    p = np.exp(x - x.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ v, gamma * np.append(score, 0.0) + p.sum(0), p @ np.abs(v), (np.abs(q) @ np.abs(k).T * scale).max(), p.sum(0)


def kept_slots(score, pos, n, budget, sink, recent_frac, history, fill):
    """Kept slots of a unit, ascending, and the slot each of the first `budget` slots takes its row from."""
    m = int(np.floor(np.float64(np.float32(recent_frac)) * budget)) if history else budget - sink
    top = budget - sink - m
    order = np.argsort(pos[:n], kind="stable") if fill else np.arange(n)
    hist = order[sink:n - m]
    best = sorted(hist, key=lambda j: (-score[j], pos[j]))[:top]
    kept = np.sort(np.concatenate([order[:sink], order[n - m:] if m else order[:0], np.array(best, int)]).astype(int))
    if not fill:
        return kept, kept
    src = np.arange(budget)
    src[np.setdiff1d(np.arange(budget), kept)] = kept[kept >= budget]
    return kept, src
