"""A turn's prompt on the GPU where it can go wrong: offsets, hints and pools that do not fit, many items for each CTA,
long page lists, the bits of the weights and of the angles."""
import math
import os
import subprocess
import sys

import pytest
import torch

import prompt_reference as R
import test_prompt_gpu as P
from test_prompt_gpu import BF16, F32, I32, check_attention, check_pages, close, fill, gen, offsets

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu
V, no_error_bits = P.V, P.no_error_bits
LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("off", [[HIGH, LOW, 4], [HIGH, LOW + 40, HIGH], [5, LOW, LOW + 3], [LOW, HIGH, LOW], [LOW, LOW + 1, 8]])
@pytest.mark.parametrize("max_rows", [8, 0])
@pytest.mark.parametrize("paged", [False, True])
def test_offsets_whose_difference_does_not_fit(V, off, max_rows, paged):
    """Ends 2^32 apart: a difference taken in 32 bits would be a few tokens from 2^31 - 1 on."""
    T = 80
    desc, rnd, r = V.CacheDesc(2, 1, 4, 2, 64, 64, BF16), gen(2), V.RotaryDesc.make(64)
    c = fill(V, desc, [10, 20], paged=paged)
    before = {x: t.clone() for x, t in c.items() if isinstance(t, torch.Tensor)}
    q, k, pos = rnd(1, T, 4, 64).to(BF16), rnd(1, T, 2, 64).to(BF16), torch.arange(T, dtype=I32, device="cuda")
    off = torch.tensor(off, dtype=I32, device="cuda")
    P.append(V, desc, c, 0, 1, k, k, pos, off, rotary=r, positions=pos, q=q, q_out=torch.empty_like(q), max_rows=max_rows)
    assert V.voxzip_get_status() == V.DEV_BAD_SPANS
    for x, t in before.items():
        assert torch.equal(torch.nan_to_num(c[x].float()), torch.nan_to_num(t.float())), x
    P.attend(V, desc, c, 0, 1, q, off, torch.empty_like(q))
    assert V.voxzip_get_status() == V.DEV_BAD_SPANS


def attend_rows(V, desc, c, ms, ns, T, **kw):
    """Attention of packed rows of which the last ones belong to no sequence, against the plain form."""
    D, G = desc.head_dim, desc.q_heads // desc.kv_heads
    q = gen(sum(ms))(1, T, desc.q_heads, D).to(desc.dtype)
    out = torch.full_like(q, 7.0)
    P.attend(V, desc, c, 0, 1, q, offsets(ms), out, **kw)
    assert (out[:, sum(ms):] == 7).all()
    end = 0
    for b, (m, n) in enumerate(zip(ms, ns)):
        t = slice(end, end + m)
        end += m
        for h in range(desc.kv_heads):
            k, v = P.unit_rows(c, b, 0, h, n)
            heads = slice(h * G, (h + 1) * G)
            want, mag, size = R.attention(q[0, t, heads], k, v, n - m + 1, 1 / math.sqrt(D))
            close(out[0, t, heads], want, R.attention_bound(want, mag, size, n, D, desc.dtype), (b, h))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("paged", [False, True])
def test_padded_rows_with_a_hint(V, dtype, paged):
    """A buffer of fixed size, of which few rows are of sequences: their keys are shared out."""
    ms, ns = [57, 0, 41, 57, 1], [1300, 40, 1000, 57, 900]
    desc = V.CacheDesc(5, 1, 8, 2, 64, 1344, dtype)
    kw = dict(max_rows=57, max_len=1300)
    assert V.voxzip_prompt_attention_workspace_size(desc, 1, 4096, **kw) > 0
    attend_rows(V, desc, fill(V, desc, ns, paged=paged), ms, ns, 4096, **kw)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Hq,H,D", [(8, 2, 64), (5, 1, 128)])
@pytest.mark.parametrize("ms", [[600, 40, 5], [5, 40, 600]])
@pytest.mark.parametrize("hint", [1, 5, 10, 100])
def test_a_hint_that_is_too_low(V, dtype, Hq, H, D, ms, hint):
    """The workspace has parts for the tiles that the hint allows; tiles beyond them, and longer ones, are done whole."""
    ns = [1500 if m == 600 else 1400 for m in ms]
    desc = V.CacheDesc(3, 1, Hq, H, D, 1536, dtype)
    assert V.voxzip_prompt_attention_workspace_size(desc, 1, 700, max_rows=hint) > 0
    attend_rows(V, desc, fill(V, desc, ns), ms, ns, 700, max_rows=hint)


@pytest.mark.parametrize("max_rows", [60, 0])  # one launch, or a planning one
@pytest.mark.parametrize("free", [1, 3, 9])
@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, F32)])
def test_no_unit_takes_another_ones_page_for_its_next_slot(V, max_rows, free, D, dtype):
    """Eight units fill their page and would like one for the next append's slot; the ninth needs one for its rows, and gets
    it. What is left goes to the others; a unit without new rows takes none."""
    ms, n0 = [54] * 8 + [60, 0], [10] * 9 + [64]
    desc, k = V.CacheDesc(10, 1, 2, 1, D, 192, dtype), gen(1)(1, 492, 1, D).to(dtype)
    c = fill(V, desc, n0, paged=True, pages=11 + free)
    gone = int(c["page_table"][9, 0, 0, 1])
    c["page_table"][9, 0, 0, 1] = -1  # (lost when the pool was empty)
    assert int(c["free_count"]) == free
    V.voxzip_append_paged(desc, c, 0, 1, k, k, torch.zeros(492, dtype=I32, device="cuda"), offsets(ms), max_rows=max_rows)
    assert V.voxzip_get_status() == 0
    assert c["len"].flatten().tolist() == [64] * 8 + [70, 64]
    table = c["page_table"][:, 0, 0].cpu()
    assert (table[:8, 1] >= 0).sum() == free - 1 and int(c["free_count"]) == 0
    assert (table[:, 2] == -1).all() and (table[:8, 1] >= -1).all() and table[9, 1] == -1
    held = table[table >= 0].tolist()
    assert sorted(held + [gone]) == list(range(11 + free))
    for b in range(9):
        assert torch.equal(P.unit_rows(c, b, 0, 0, ms[b] + 10)[1][10:], k[0, sum(ms[:b]):sum(ms[:b + 1]), 0])


@pytest.mark.parametrize("max_rows", [60, 0])
def test_a_skipped_unit_takes_no_page(V, max_rows):
    """Two units need more pages than there are: one gets them, the other none, nor one for its next slot."""
    desc, k = V.CacheDesc(3, 1, 2, 1, 64, 192, BF16), gen(1)(1, 120, 1, 64).to(BF16)
    c = fill(V, desc, [64, 64, 10], paged=True, pages=5)
    lost = [int(c["page_table"][b, 0, 0, 1]) for b in (0, 1)]
    c["page_table"][:2, 0, 0, 1] = -1
    c["free_pages"][:1] = lost[0]
    c["free_count"].fill_(1)
    V.voxzip_append_paged(desc, c, 0, 1, k, k, torch.zeros(120, dtype=I32, device="cuda"), offsets([60, 60, 0]), max_rows=max_rows)
    assert V.voxzip_get_status() == V.DEV_CAPACITY
    got = c["len"].flatten().tolist()
    assert sorted(got[:2]) == [64, 124] and int(c["free_count"]) == 0
    assert sorted(c["page_table"][:2, 0, 0, 1].tolist()) == [-1, lost[0]] and (c["page_table"][:, 0, 0, 2] == -1).all()


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("max_rows", [0, 10 ** 9])
def test_a_turn_of_unknown_rows_and_the_steps_after_it(V, paged, max_rows):
    """max_rows=0: the packed tokens bound a sequence's rows, so the next decode step knows how long a unit may be."""
    from paper_2608_08569_gb300.session import Session
    B, L, Hq, H, D = 2, 2, 4, 2, 64
    desc, rnd = V.CacheDesc(B, L, Hq, H, D, 4096, BF16), gen(3)
    s = Session(desc, [4096, 4096], 0.9, pages=800 if paged else None)
    ms = [1500, 20]
    for turn in range(2):
        T = sum(ms)
        qkv = rnd(L, T, Hq + 2 * H, D).to(BF16)
        out = torch.empty(L, T, Hq, D, dtype=BF16, device="cuda")
        s.extend(qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:], torch.arange(T, dtype=I32, device="cuda"), offsets(ms), out,
                 max_rows=max_rows)
        assert max(ms) * (turn + 1) + turn <= s.n_max <= T * (turn + 1) + turn  # (a step of one row lies between)
        q, k, v = rnd(L, B, Hq, D).to(BF16), rnd(L, B, H, D).to(BF16), rnd(L, B, H, D).to(BF16)
        got = torch.full_like(q, 7.0)
        s.decode(q, k, v, torch.zeros(B, dtype=I32, device="cuda"), got)
        assert V.voxzip_get_status() == 0
        for b, m in enumerate(ms):
            n = (turn + 1) * (m + 1)
            assert (s.cache["len"][b] == n).all()
            for l in range(L):
                for h in range(H):
                    kk, vv = P.unit_rows(s.cache, b, l, h, n)
                    want, mag, size = R.attention(q[l, b, 2 * h:2 * h + 2][None], kk, vv, n, 0.125)
                    # (the step adds its parts up in another order: twice the bound)
                    close(got[l, b, 2 * h:2 * h + 2][None], want, 2 * R.attention_bound(want, mag, size, n, D, BF16))


@pytest.mark.parametrize("paged", [False, True])
def test_items_of_many_keys(V, paged):
    """Whole tiles over 3 million rows (some 25 ms each): the mask warp waits for all keys in front of the masked ones, and
    gives up only where nothing moves. (The checked build's waits are 8 ms.)"""
    n, m, G, D = 3_000_000, 2432, 16, 64  # 152 tiles of 16 tokens: keys are not shared out
    C = n + 64
    desc, rnd = V.CacheDesc(1, 1, G, 1, D, C, BF16), gen(5)
    c = dict(k=rnd(1, 1, 1, C, D).to(BF16), v=rnd(1, 1, 1, C, D).to(BF16))
    at = slice(n - m, n)  # what a token sees of its own turn shows
    c["v"][..., at, :] += 4.0
    if paged:
        pages = C // 64
        table = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).cuda()
        pool = {x: torch.empty(pages, 64, D, dtype=BF16, device="cuda") for x in "kv"}
        for x in "kv":
            pool[x][table] = c[x].view(pages, 64, D)
        z = torch.zeros(1, 1, 1, C, device="cuda")
        pc = dict(k_pool=pool["k"], v_pool=pool["v"], page_table=table.to(I32).view(1, 1, 1, pages), free_pages=torch.zeros(pages, dtype=I32, device="cuda"),
                  free_count=torch.zeros(1, dtype=I32, device="cuda"), score=z, pos=z.to(I32), pages=pages, max_pages=pages)
    ln = torch.full((1, 1, 1), n, dtype=I32, device="cuda")
    q = rnd(1, m, G, D).to(BF16)
    q *= 3  # some keys outweigh the others
    out = torch.full_like(q, 7.0)
    assert V.voxzip_prompt_attention_workspace_size(desc, 1, m) == 0
    if paged:
        V.voxzip_prompt_attention_paged(desc, dict(pc, len=ln), 0, 1, q, offsets([m]), out)
    else:
        V.voxzip_prompt_attention(desc, 0, 1, q, offsets([m]), c["k"], c["v"], ln, out)
    k, v = c["k"][0, 0, 0, :n], c["v"][0, 0, 0, :n]
    for t in (0, 15, 16, 1203, 2430, 2431):
        want, mag, size = R.attention(q[0, t:t + 1, ::5], k, v, n - m + 1 + t, 0.125)
        close(out[0, t:t + 1, ::5], want, R.attention_bound(want, mag, size, n, D, BF16), t)


@pytest.mark.skipif(os.environ.get("VOXZIP_CHECKED", "0") not in ("", "0"), reason="this is the checked run")
def test_checked_build():
    """The range-checked build, whose waits are short, gives the same and no bit of VOXZIP_DEV_BOUNDS."""
    from paper_2608_08569_gb300.build import build_library
    build_library(checked=True)
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider"],
                       cwd=ROOT, env=dict(os.environ, VOXZIP_CHECKED="1"), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]


# ----------------------------------------------------------------------------- the bits that are kept

def exact_cos_sin(positions, freqs):
    """cos and sin of position * freq in 64 bits, the angle reduced in integers of 200 bits after the point: [T][pairs]."""
    from fractions import Fraction
    one = 1 << 200

    def arctan_of_inverse(x):  # of 1 / x, by its series
        total, term, k = 0, one // x, 0
        while term:
            total += (term if k % 2 == 0 else -term) // (2 * k + 1)
            term //= x * x
            k += 1
        return total

    two_pi = 8 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239))  # Machin
    turns = torch.empty(len(positions), len(freqs), dtype=torch.float64)
    for j, f in enumerate(map(Fraction, freqs)):
        step = f.numerator * one * one // (f.denominator * two_pi)  # of a turn, 2^-200 each
        for i, p in enumerate(positions):
            turns[i, j] = ((p * step + one // 2) % one - one // 2) / one
    th = turns.cuda() * (2 * math.pi)
    return th.cos(), th.sin()


@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
@pytest.mark.parametrize("freqs", ["usual", "any"])
def test_angles_at_any_position(V, pairing, freqs):
    """fp32, positions over the whole range. With steps of 2^-24: the angle is 2^-28 + 2^-32 + 2^-34 of a turn off, 0.43 steps
    of radians; CUDA's sincospif by a step of its result's (one unit in the last place, at most 2^-24 below 1); so each of
    the two terms 1.43 steps of its channel's size, another for the products and one for their sum: 3.43 of |lo| + |hi|."""
    D, T = 128, 300
    if freqs == "usual":
        r = V.RotaryDesc.make(D, 1e6, pairing=pairing)
    else:
        g = torch.Generator().manual_seed(1)
        fs = (10.0 ** (torch.rand(64, generator=g, dtype=torch.float64) * 18 - 12)).tolist()  # 1e-12 to 1e6
        r = V.RotaryDesc(tuple(x if i % 2 else -x for i, x in enumerate(fs[:61])) + (0.0, 1e6, -1e6), (), pairing)
    desc, rnd = V.CacheDesc(1, 1, 4, 1, D, 8, F32), gen(9)
    g = torch.Generator().manual_seed(2)
    pos = torch.randint(-2 ** 31, 2 ** 31, (T,), generator=g).to(I32)
    pos[:9] = torch.tensor([0, 1, -1, LOW, HIGH, LOW + 1, 46023, 10 ** 6, -46023], dtype=I32)
    x, got = rnd(1, T, 4, D), torch.empty(1, T, 4, D, device="cuda")
    V.voxzip_rotary(desc, r, pos.cuda(), q=x, q_out=got)
    c, s = (t[None, :, None] for t in exact_cos_sin(pos.tolist(), r.freqs))
    lo = torch.arange(64) if pairing == "halves" else torch.arange(0, D, 2)
    hi = lo + (64 if pairing == "halves" else 1)
    a, b = x.double()[..., lo], x.double()[..., hi]
    for at, want in ((lo, a * c - b * s), (hi, b * c + a * s)):
        steps = (got.double()[..., at] - want).abs() / (R.U32 * (a.abs() + b.abs()))
        print("steps", float(steps.max()))
        assert float(steps.max()) <= 3.43 + 1e-5


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("D,dtype", [(128, BF16), (64, F32)])
def test_a_short_append_of_all_layers_is_that_of_each(V, paged, D, dtype):
    """Many units are planned before their rows, a layer's few take one launch: the same rows, to the bit."""
    B, L, Hq, H, C, ms, n0 = 3, 24, 8, 4, 192, [57, 0, 40], [60, 3, 100]
    desc, r, T = V.CacheDesc(B, L, Hq, H, D, C, dtype), V.RotaryDesc.make(64, sections=(16, 8, 8)), sum(ms) + 2
    assert V.voxzip_append_workspace_size(desc, L, T, 57) > 0 == V.voxzip_append_workspace_size(desc, 1, T, 57)
    qkv = gen(4)(L, T, (Hq + 2 * H) * D).to(dtype)
    q, k, v = (x.unflatten(-1, (-1, D)) for x in qkv.split([Hq * D, H * D, H * D], -1))
    pos, new_pos, off = P.positions_for(3, T), torch.arange(T, dtype=I32, device="cuda"), offsets(ms)
    got = []
    for step in (L, 1):
        c, qo = fill(V, desc, n0, paged=paged), torch.zeros(L, T, Hq, D, dtype=dtype, device="cuda")
        for l in range(0, L, step):
            at = slice(l, l + step)
            P.append(V, desc, c, l, step, k[at], v[at], new_pos, off, rotary=r, positions=pos, q=q[at], q_out=qo[at], max_rows=57)
        if paged:
            check_pages(desc, c)
        got.append((c, qo))
    (a, qa), (b, qb) = got
    assert torch.equal(qa, qb) and all(torch.equal(a[x], b[x]) for x in ("len", "pos", "score"))
    for s, (m, n) in enumerate(zip(ms, n0)):
        for l in range(L):
            for h in range(H):
                for x, y in zip(P.unit_rows(a, s, l, h, n + m), P.unit_rows(b, s, l, h, n + m)):
                    assert torch.equal(x, y)


# ----------------------------------------------------------------------------- many items, long page lists

def plain(q, k, v, first, scale):
    """q [m][G][D] over finite k, v [n][D]: as R.attention, all rows at once."""
    m, n = len(q), len(k)
    if n == 0:
        z = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
        return z, z, z[..., 0]
    q, k, v = q.double(), k.double(), v.double()
    seen = torch.arange(n, device=q.device)[None] < (first + torch.arange(m, device=q.device))[:, None]
    x = (torch.einsum("mgd,nd->mgn", q, k) * scale).masked_fill(~seen[:, None], -math.inf)
    p = torch.softmax(x, -1).nan_to_num(0.0)  # (a row that sees nothing)
    return p @ v, p @ v.abs(), (q.abs() @ k.abs().t()).amax(-1) * scale


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("Hq,H,D,L", [(4, 4, 128, 16), (16, 2, 64, 8), (16, 4, 128, 5)])
def test_several_items_for_each_cta(V, paged, Hq, H, D, L):
    """Four hundred items and more: a CTA takes three or more of them, long and short ones, with one row tile alive or both,
    of units without rows, of rows that see nothing, and with infinities that the mask hides from some."""
    ms, G, C = [1, 300, 700, 0, 129, 513, 31], Hq // H, 1280
    B, T, per = len(ms), sum(ms) + 3, 2 * (128 // G)
    items = sum(-(-m // per) for m in ms) * H * L
    assert items > 3 * 152
    desc = V.CacheDesc(B, L, Hq, H, D, C, BF16)
    assert V.voxzip_prompt_attention_workspace_size(desc, L, T) == 0
    c = fill(V, desc, [C] * B, seed=D + G, paged=paged)
    pick = torch.Generator().manual_seed(G)
    ln = torch.empty(B, L, H, dtype=I32)
    for b, m in enumerate(ms):
        choice = torch.tensor([0, m // 2, m, min(C, m + 37), min(C, m + 128), 1200, C], dtype=I32)
        ln[b] = choice[torch.randint(0, len(choice), (L, H), generator=pick)]
    c["len"].copy_(ln)
    dirty = {}  # of some units, an infinity in V's channel 3 in the middle of the turn
    for b, m in enumerate(ms):
        for l in range(0, L, 2):
            n = int(ln[b, l, 0])
            if m > 20 and n >= m:
                slot = n - m // 2
                dirty[b, l, 0] = slot
                if paged:
                    c["v_pool"][int(c["page_table"][b, l, 0, slot // 64]), slot % 64, 3] = math.inf
                else:
                    c["v"][b, l, 0, slot, 3] = math.inf
    q = gen(31)(L, T, Hq, D).to(BF16)
    out = torch.full_like(q, 7.0)
    P.attend(V, desc, c, 0, L, q, offsets(ms), out)
    assert V.voxzip_get_status() == 0 and (out[:, sum(ms):] == 7).all()
    end = 0
    for b, m in enumerate(ms):
        t = slice(end, end + m)
        end += m
        for l in range(L):
            for h in range(H):
                n, heads = int(ln[b, l, h]), slice(h * G, (h + 1) * G)
                k, v = P.unit_rows(c, b, l, h, n)
                got, slot = out[l, t, heads], dirty.get((b, l, h))
                if slot is not None:
                    sees = torch.arange(n - m, n, device="cuda") >= slot
                    assert (got[sees][..., 3] == math.inf).all() and torch.isfinite(got[~sees]).all()
                    k, v, got = k.clone(), v.clone(), got.clone()
                    v[slot, 3] = 0.0
                want, mag, size = plain(q[l, t, heads], k, v, n - m + 1, D ** -0.5)
                if slot is not None:
                    got[..., 3][sees] = want[..., 3][sees].to(BF16)
                close(got, want, R.attention_bound(want, mag, size, n, D, BF16), (b, l, h))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("L", [1, 10])  # keys shared out, at page offsets of any kind, and whole tiles
def test_units_of_many_pages(V, dtype, L):
    """70 shuffled pages a unit, of which a turn of 2 300 rows takes 36 from the middle of the 34th on."""
    H, G, D, n0, m = 16, 1, 64, 33 * 64 + 29, 2300
    C, n = 72 * 64, n0 + m
    desc, rnd = V.CacheDesc(1, L, H * G, H, D, C, dtype), gen(L)
    c = fill(V, desc, [n0], seed=3, paged=True)
    assert int(c["page_table"].max()) > 64
    k, v = rnd(L, m, H, D).to(dtype), rnd(L, m, H, D).to(dtype)
    V.voxzip_append_paged(desc, c, 0, L, k, v, torch.arange(m, dtype=I32, device="cuda"), offsets([m]))
    assert V.voxzip_get_status() == 0 and (c["len"] == n).all()
    check_pages(desc, c)
    for l in range(L):
        for h in range(H):
            kk, vv = P.unit_rows(c, 0, l, h, n)
            assert torch.equal(kk[n0:], k[l, :, h]) and torch.equal(vv[n0:], v[l, :, h])
    last = 40  # of the turn's tokens attend
    q, off = rnd(L, last, H * G, D).to(dtype), offsets([last])
    out = torch.empty_like(q)
    shared = V.voxzip_prompt_attention_workspace_size(desc, L, last) > 0
    assert shared == (L == 1 or dtype is F32)
    V.voxzip_prompt_attention_paged(desc, c, 0, L, q, off, out)
    for l in range(0, L, 3):
        for h in range(H):
            kk, vv = P.unit_rows(c, 0, l, h, n)
            want, mag, size = plain(q[l, :, h:h + 1], kk, vv, n - last + 1, D ** -0.5)
            close(out[l, :, h:h + 1], want, R.attention_bound(want, mag, size, n, D, dtype), (l, h))
