"""How many bits the 4-bit decode's products keep: outputs and scores against 64 bits, in the L2 norm, with limits that
a coarser form would miss (shown here on the CPU, where the form is emulated and the mistake planted).

fp32 activations, q and weights in three bf16 parts (24 bits). A tensor core's sum of 16 products cuts off what its
largest term's 24 bits do not hold; a group's products, scaled, are of the order of 8, a logit's of 1: some 2^-22
(2.4e-7) per logit, the same again for the exponential, and as much for the sums over tokens, which the three
together keep below 8 x 2^-22 = 2e-6. One part less in the weights leaves 2^-15 of each, 1e-5 and more in the outputs.

bf16 activations, q exact and weights times scales in two parts (a loss d of up to 2^-15). The output is rounded to
bf16 (steps of 2^-8): its error is that of rounding the exact output, to which d adds nothing that shows (limit: a
ratio of 1.02; a weight in one part, 2^-9, makes it 1.3). A loss of d turns the rounding of one output in 2^-8 / d, so
against the rounded exact output the error is about sqrt(2^-8 d), 3.5e-4 at most; some ten turned outputs make it, so
that twice as much is allowed for their sizes: 7e-4. Scores come from weights and logits in fp32: the codes' offset of 8
makes a group's terms up to 8 times as large as above, 8 x 2^-22 = 2e-6 per logit: limit 1e-5.
"""
import math

import numpy as np
import pytest
import torch

import q4_reference as R

F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [(64, 2, 32, 149), (128, 8, 4, 416), (128, 16, 8, 600), (64, 1, 64, 1237), (128, 4, 8, 2317)]  # D, G, Hkv, n
LIMIT_F32, LIMIT_BF16_RATIO, LIMIT_BF16_FLIPS, LIMIT_BF16_SCORE = 2e-6, 1.02, 7e-4, 1e-5


def _values(D, G, H, n, dtype, seed):
    """Per kv-head q [G][D], rows K and V [n + 1][D], as fp32 values of the dtype: N(0, 1), channels of one magnitude."""
    rng = np.random.default_rng([seed, D, G, n])
    x = [rng.standard_normal((H,) + s).astype(np.float32) for s in ((G, D), (n + 1, D), (n + 1, D))]
    return x if dtype == F32 else [R.bf16(a) for a in x]


def _quantised(k, v, n):
    """Scales and codes of a head's rows, the last one appended under the others' exponents."""
    e = R.channel_exponents(k[:n])
    return R.quantise(k * np.float32(2.0) ** -e) + R.quantise(v) + (e,)


def _per_head(f, q, rows, *args):
    """f's outputs [H][G][D] and masses [H][n + 1]."""
    both = [f(q[h], *rows[h], *args) for h in range(len(q))]
    return np.stack([x[0] for x in both]), np.stack([x[1] for x in both])


def _exact(q, ks, kc, vs, vc, e, scale):
    """Output [G][D] and every row's mass in 64 bits."""
    x = q.astype(np.float64) @ R.values(kc, ks, e).T * scale
    p = np.exp(x - x.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    return p @ R.values(vc, vs), p.sum(0)


def _err(a, b):
    return np.linalg.norm(np.asarray(a, np.float64) - b) / np.linalg.norm(b)


# ----------------------------------------------------------------------------- the emulation

def _parts(x, parts):
    """fp64 x as the sum of that many bf16 parts, each the upper 8 bits of what is left (one alone is rounded)."""
    if parts == 1:
        return R.bf16(x.astype(np.float32)).astype(np.float64)
    left, total = x.astype(np.float32), np.zeros(x.shape)
    for _ in range(parts):
        part = (left.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
        total, left = total + part, left - part
    return total


def _emulated(q, ks, kc, vs, vc, e, scale, q_parts, w_parts):
    """The kernel's operands, their products and sums in 64 bits."""
    x = _parts(q.astype(np.float64) * 2.0 ** e, q_parts) @ R.values(kc, ks).T * scale
    p = np.exp(x - x.max(-1, keepdims=True))
    D, out = kc.shape[1], np.zeros(q.shape)
    for j in range(D // 32):
        at = slice(32 * j, 32 * j + 32)
        out[:, at] = _parts(p * vs[:, j].astype(np.float64), w_parts) @ vc[:, at].astype(np.float64)
    z = p.sum(-1, keepdims=True)
    return out / z, (p / z).sum(0)


def _bf16_errors(out, exact):
    rounded = R.bf16(exact.astype(np.float32)).astype(np.float64)
    got = R.bf16(np.asarray(out, np.float32)).astype(np.float64)
    return _err(got, exact) / _err(rounded, exact), np.linalg.norm(got - rounded) / np.linalg.norm(exact)


@pytest.mark.parametrize("D,G,H,n", SHAPES)
@pytest.mark.parametrize("seed", range(2))
def test_a_part_less_would_miss_the_limits(D, G, H, n, seed):
    scale = 1 / math.sqrt(D)
    q, k, v = _values(D, G, H, n, F32, seed)
    rows = [_quantised(k[h], v[h], n) for h in range(H)]
    exact, mass = _per_head(_exact, q, rows, scale)
    out, sc = _per_head(_emulated, q, rows, scale, 3, 3)
    assert _err(out, exact) < LIMIT_F32 / 10 and _err(sc, mass) < LIMIT_F32 / 10
    assert _err(_per_head(_emulated, q, rows, scale, 3, 2)[0], exact) > 2 * LIMIT_F32
    out, sc = _per_head(_emulated, q, rows, scale, 2, 3)
    assert _err(out, exact) > 2 * LIMIT_F32 and _err(sc, mass) > 2 * LIMIT_F32

    q, k, v = _values(D, G, H, n, BF16, seed)
    rows = [_quantised(k[h], v[h], n) for h in range(H)]
    exact, mass = _per_head(_exact, q, rows, scale)
    out, sc = _per_head(_emulated, q, rows, scale, 1, 2)  # q is bf16: one part is exact
    ratio, flips = _bf16_errors(out, exact)
    assert ratio < LIMIT_BF16_RATIO and flips < 0.8 * LIMIT_BF16_FLIPS and _err(sc, mass) < 1e-12
    ratio, flips = _bf16_errors(_per_head(_emulated, q, rows, scale, 1, 1)[0], exact)
    assert ratio > 1.1 * LIMIT_BF16_RATIO and flips > 2 * LIMIT_BF16_FLIPS


# ----------------------------------------------------------------------------- on the GPU

def _np(t):
    return t.float().cpu().numpy() if t.dtype == BF16 else t.cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,G,H,n", SHAPES)
@pytest.mark.parametrize("seed", range(2))
@pytest.mark.parametrize("copies", [1, 100])  # few units, split over clusters; many
def test_decode_keeps_its_bits(D, G, H, n, dtype, seed, copies):
    import paper_2608_08569_gb300 as V
    q, k, v = _values(D, G, H, n, dtype, seed)
    C = -(-(n + 1) // 4) * 4
    desc = V.CacheDesc(copies, 1, G * H, H, D, C, dtype)
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(n)

    def rows(x):
        t = torch.zeros(1, 1, H, C, D, dtype=dtype, device="cuda")
        t[0, 0, :, :n] = torch.from_numpy(x[:, :n]).to(dtype)
        return t.expand(copies, 1, H, C, D).contiguous()
    new = lambda x, h: torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda().reshape(1, 1, h, D).expand(1, copies, h, D).contiguous()
    V.voxzip_q4_pack(desc, qc, 0, 1, rows(k), rows(v))
    out = torch.empty(1, copies, G * H, D, dtype=dtype, device="cuda")
    V.voxzip_decode_step_q4(desc, qc, 0, 1, new(q, G * H), new(k[:, n], H), new(v[:, n], H),
                            torch.zeros(copies, dtype=torch.int32, device="cuda"), 1.0, out, max_len=n + 1)
    assert V.voxzip_get_status() == 0
    exact, mass = _per_head(_exact, q, [_quantised(k[h], v[h], n) for h in range(H)], 1 / math.sqrt(D))
    got, sc = _np(out)[0].reshape(copies, H, G, D), _np(qc["score"])[:, 0, :, :n + 1]
    assert (got == got[:1]).all() and (sc == sc[:1]).all()
    if dtype == F32:
        errors, limits = (_err(got[0], exact), _err(sc[0], mass)), (LIMIT_F32, LIMIT_F32)
    else:
        errors = _bf16_errors(got[0], exact) + (_err(sc[0], mass),)
        limits = LIMIT_BF16_RATIO, LIMIT_BF16_FLIPS, LIMIT_BF16_SCORE
    print("errors", *(f"{x:.2e}" for x in errors))
    assert all(x <= y for x, y in zip(errors, limits)), (errors, limits)
