"""How many bits the prompt attention keeps, against 64 bits in the L2 norm, with limits that a coarser form would miss (the
form emulated and the mistake planted on the CPU).

bf16: q, k and v are exact, logits and sums fp32. A weight is rounded to bf16 before it meets V: half a step is 2^-8 of it, the
root mean square over the mantissas some 1.6e-3, as much as the output's own rounding. With values of V that do not depend on
one another a row's error is the weights', so both together are sqrt(2) times the error of rounding the exact output:
limit 1.5. A bit less in the weights makes it sqrt(5) = 2.2, a fault of the sums or logits of 2^-9 1.5 and more.

fp32: a logit is a chain of D sums whose partial ones grow like the root of their number: 2^-25 D / sqrt(2) of rounding, times
the scale 1 / sqrt(D), is some 2e-7 for D = 128, twice that with the maximum's; the exponential 2^-23; a row's sums over n
keys 2^-25 sqrt(n / 2), 1.4e-6 for n = 4 097. Limit 4e-6; weights of 16 bits leave 6e-6.
"""
import math

import numpy as np
import pytest
import torch

F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [(128, 8, 4, 60, 300), (64, 1, 8, 200, 230), (128, 8, 2, 1, 4097), (64, 16, 2, 33, 1237), (128, 1, 2, 300, 1500)]  # D, G, Hkv, m, n
LIMIT_RATIO, LIMIT_F32 = 1.5, 4e-6


def values(D, G, H, m, n, dtype, seed):
    """q [H][m][G][D], k and v [H][n][D], of the dtype, in 64 bits."""
    g = torch.Generator().manual_seed(1000 * seed + D + G + m + n)
    return [torch.randn(*s, generator=g).to(dtype).double() for s in ((H, m, G, D), (H, n, D), (H, n, D))]


def cut(x, bits):
    """x in 64 bits, rounded to a mantissa of so many bits."""
    f, e = np.frexp(x.numpy())
    return torch.from_numpy(np.ldexp(np.rint(np.ldexp(f, bits)), e - bits))


def attention(q, k, v, bits=None):
    """Rows see n - m + 1 + i keys; weights of `bits` before they meet V, their sum of all of them."""
    m, n = q.shape[1], k.shape[1]
    x = torch.einsum("hmgd,hnd->hmgn", q, k) / math.sqrt(q.shape[-1])
    unseen = torch.arange(n)[None] > torch.arange(n - m, n)[:, None]
    x = x.masked_fill(unseen[None, :, None], -math.inf)
    p = (x - x.amax(-1, keepdim=True)).exp()
    return torch.einsum("hmgn,hnd->hmgd", p if bits is None else cut(p, bits), v) / p.sum(-1, keepdim=True)


def err(a, b):
    return float((a - b).norm() / b.norm())


def ratio(out, exact):
    """The error of bf16 outputs, in that of rounding the exact ones."""
    return err(out.to(BF16).double(), exact) / err(exact.to(BF16).double(), exact)


@pytest.mark.parametrize("D,G,H,m,n", SHAPES)
@pytest.mark.parametrize("seed", range(2))
def test_a_coarser_form_would_miss_the_limits(D, G, H, m, n, seed):
    x = values(D, G, H, m, n, BF16, seed)
    exact = attention(*x)
    assert ratio(attention(*x, bits=8), exact) < 0.98 * LIMIT_RATIO
    assert ratio(attention(*x, bits=7), exact) > 1.2 * LIMIT_RATIO  # (less where the largest weight, 1, outweighs the others)
    x = values(D, G, H, m, n, F32, seed)
    exact = attention(*x)
    assert err(attention(*x, bits=16), exact) > 1.2 * LIMIT_F32


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,G,H,m,n", SHAPES)
@pytest.mark.parametrize("seed", range(2))
@pytest.mark.parametrize("copies", [1, 100])  # keys shared out among CTAs, and whole tiles
def test_attention_keeps_its_bits(D, G, H, m, n, dtype, seed, copies):
    import paper_2608_08569_gb300 as V
    q, k, v = values(D, G, H, m, n, dtype, seed)
    desc = V.CacheDesc(1, copies, G * H, H, D, n, dtype)
    cache = [x.to(dtype).cuda().expand(1, copies, H, n, D).contiguous() for x in (k, v)]
    rows = q.to(dtype).transpose(0, 1).reshape(1, m, G * H, D).cuda().expand(copies, m, G * H, D).contiguous()
    out, ln = torch.empty_like(rows), torch.full((1, copies, H), n, dtype=torch.int32, device="cuda")
    V.voxzip_prompt_attention(desc, 0, copies, rows, torch.tensor([0, m], dtype=torch.int32, device="cuda"), *cache, ln, out)
    assert V.voxzip_get_status() == 0
    assert torch.equal(out, out[:1].expand_as(out))
    got, exact = out[0].cpu().double().view(m, H, G, D).transpose(0, 1), attention(q, k, v)
    if dtype == BF16:
        print("ratio", ratio(got, exact))
        assert ratio(got, exact) <= LIMIT_RATIO
    else:
        print("error", err(got, exact))
        assert err(got, exact) <= LIMIT_F32
