"""Plain 64-bit forms of the prompt's operators, from their definitions, with the bounds that their arithmetic gives.

A step of fp32 is at most 2^-24 of a value off, of bf16 2^-8 (half a step)."""
import math

import torch

U32 = 2.0 ** -24
UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def angles(positions, rot):
    """[tokens][pairs] in 64 bits: positions [axes][tokens]."""
    pos = positions if positions.dim() == 2 else positions[None]
    axes = torch.tensor(rot.axes or (0,) * len(rot.freqs), device=pos.device)
    f = torch.tensor(rot.freqs, dtype=torch.float64, device=pos.device)
    return pos.double()[axes].t() * f


def rotate(x, positions, rot):
    """x [layers][tokens][heads][D] rotated, and the sizes |lo| + |hi| of each channel's two terms."""
    half = len(rot.freqs)
    th = angles(positions, rot)[None, :, None]
    x = x.double()
    y, size = x.clone(), torch.zeros_like(x)
    lo = torch.arange(half) if rot.pairing == "halves" else torch.arange(0, 2 * half, 2)
    hi = lo + (half if rot.pairing == "halves" else 1)
    a, b = x[..., lo], x[..., hi]
    y[..., lo], y[..., hi] = a * th.cos() - b * th.sin(), b * th.cos() + a * th.sin()
    size[..., lo] = size[..., hi] = a.abs() + b.abs()
    return y, size


def rotate_bound(want, size, dtype):
    """cos and sin: 2 steps of the function, 1 of its argument; two products and their sum 2; all of terms of `size`.
    64-bit angles of positions up to 2^31: 2^-53 of 2^31 radians. Then one rounding to the dtype."""
    err = (5 * U32 + 2.0 ** -21) * size
    return err + (UNIT[dtype] * (want.abs() + err) if dtype != torch.float32 else U32 * want.abs())


def attention(q, k, v, first, scale):
    """q [m][G][D] over k, v [n][D]: row i sees the first `first + i` keys. Returns out, and sum p |v|, the largest
    |logit| and the largest sum |q k| scale of each row, from which the bounds follow."""
    m, G, D = q.shape
    n = k.shape[0]
    q, k, v = q.double(), k.double(), v.double()
    seen = torch.arange(n, device=q.device)[None] < (first + torch.arange(m, device=q.device))[:, None]  # [m][n]
    x = torch.einsum("mgd,nd->mgn", q, torch.nan_to_num(k, 0.0, 0.0, 0.0) if not seen.all() else k) * scale
    bad = ~torch.isfinite(k).all(-1)
    if bad.any() and not seen.all():  # a row that sees such a key has its logits as they come
        x = torch.where(bad[None, None] & seen[:, None], torch.einsum("mgd,nd->mgn", q, k) * scale, x)
    x = x.masked_fill(~seen[:, None], -math.inf)
    p = torch.softmax(x, -1)
    p = torch.where(seen.any(-1)[:, None, None], p, torch.zeros_like(p))
    out = torch.zeros(m, G, D, dtype=torch.float64, device=q.device)
    mag = torch.zeros_like(out)
    for i in range(m):
        c = int(min(n, max(0, first + i)))
        out[i], mag[i] = p[i, :, :c] @ v[:c], p[i, :, :c] @ v[:c].abs()
    size = (q.abs() @ torch.nan_to_num(k, 0.0, 0.0, 0.0).abs().t()).amax(-1) * scale if n else torch.zeros(m, G, device=q.device)
    return out, mag, size


def attention_bound(want, mag, size, n, D, dtype):
    """Logits: fp32 sums of D products, off by (D + 6) steps of the sum of their sizes (the tensor cores cut sums off
    instead of rounding them: twice that); their scaling and difference to the maximum 6 steps more. A weight is off by
    that, relatively, twice (its own logit, the maximum's), and by 8 steps for its power of two and the sum's terms; the
    sums of n weights and of n products by n steps (cut off: twice that). bf16: the weights 2^-8, the output 2^-8."""
    cut = 2 if dtype == torch.bfloat16 else 1
    logit = cut * (D + 12) * U32 * size[..., None]
    err = (2 * logit + 2 * (logit + 8 * U32) + cut * 2 * (n + 8) * U32) * mag
    if dtype == torch.bfloat16:
        err = err + 2.0 ** -8 * mag
        return err + 2.0 ** -8 * (want.abs() + err)
    return err + U32 * want.abs()
