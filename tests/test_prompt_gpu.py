"""A turn's prompt on the GPU against plain 64-bit forms: rotations, appended rows and attention, within the bounds
that prompt_reference.py derives; what is not theirs to write stays as it was."""
import math
import os
import subprocess
import sys

import pytest
import torch

import prompt_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
I32 = torch.int32


@pytest.fixture(scope="module")
def V():
    import paper_2608_08569_gb300 as V
    V.lib()
    return V


@pytest.fixture(autouse=True)
def no_error_bits(V):
    V.voxzip_get_status()
    yield
    assert V.voxzip_get_status() == 0


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s: torch.randn(*s, generator=g, device="cuda")


def offsets(ms, gap=0):
    """seq_off of sequences of ms tokens behind `gap` rows of no sequence."""
    off = [gap]
    for m in ms:
        off.append(off[-1] + m)
    return torch.tensor(off, dtype=I32, device="cuda")


def close(got, want, bound, what=""):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and not torch.isinf(got[~inf]).any(), what
    fine = torch.isfinite(want)
    over = ((got - want).abs() - bound)[fine]
    assert not over.numel() or float(over.max()) <= 0, (what, float(over.max()), float((got - want).abs()[fine].max()))


ROT = [dict(rotary_dim=128, theta=1e6, sections=(24, 20, 20), in_turns=True), dict(rotary_dim=64, pairing="adjacent", sections=(16, 8, 8)),
       dict(rotary_dim=16, theta=10.0), dict(rotary_dim=48, sections=(4, 20), pairing="adjacent"), dict(rotary_dim=64)]


def positions_for(axes, T, seed=0):
    g = torch.Generator().manual_seed(seed)
    p = torch.randint(-5, 10 ** 6, (axes, T), generator=g, dtype=I32)
    p[:, ::3] = torch.randint(-2 ** 31, 2 ** 31 - 1, (axes, len(range(0, T, 3))), generator=g).to(I32)
    p[0, 0] = 0
    return p.cuda()


# ----------------------------------------------------------------------------- rotary

@pytest.mark.parametrize("D,dtype", [(128, BF16), (64, BF16), (128, F32), (64, F32)])
@pytest.mark.parametrize("rot", range(len(ROT)))
@pytest.mark.parametrize("L,T,Hq,H", [(1, 1, 1, 1), (48, 1, 32, 4), (2, 37, 6, 3), (1, 1500, 14, 2)])
def test_rotary(V, D, dtype, rot, L, T, Hq, H):
    if ROT[rot]["rotary_dim"] > D:
        pytest.skip("more channels than the head has")
    rnd = gen(rot + D)
    desc, r = V.CacheDesc(1, 1, Hq, H, D, 8, dtype), V.RotaryDesc.make(**ROT[rot])
    # views of one projection's output, in which tokens have a gap besides
    qkv = rnd(L, T, (Hq + 2 * H) * D + 16).to(dtype)
    q, k = (x.unflatten(-1, (-1, D)) for x in (qkv[..., :Hq * D], qkv[..., Hq * D:(Hq + H) * D]))
    pos = positions_for(r.num_axes, T)
    qo, ko = torch.full((L, T, Hq, D), math.nan, dtype=dtype, device="cuda"), torch.full((L, T, H, D), math.nan, dtype=dtype, device="cuda")
    V.voxzip_rotary(desc, r, pos, q=q, k=k, q_out=qo, k_out=ko)
    for got, x in ((qo, q), (ko, k)):
        want, size = R.rotate(x, pos, r)
        close(got, want, R.rotate_bound(want, size, dtype))
        assert torch.equal(got[..., r.rotary_dim:], x[..., r.rotary_dim:])
    # one of the two alone, in place, gives the same
    alone = k.contiguous()
    V.voxzip_rotary(desc, r, pos if r.num_axes > 1 else pos[0], k=alone, k_out=alone)
    assert torch.equal(alone, ko)


def test_rotation_of_opposite_positions_is_undone(V):
    """fp32: turning back by the same angle gives the rows again, within the two turns' bounds."""
    rnd = gen(1)
    desc, r = V.CacheDesc(1, 1, 4, 1, 128, 8, F32), V.RotaryDesc.make(128, 1e6)
    q, pos = rnd(1, 333, 4, 128), torch.arange(10 ** 6, 10 ** 6 + 333, dtype=I32, device="cuda")
    out, back = torch.empty_like(q), torch.empty_like(q)
    V.voxzip_rotary(desc, r, pos, q=q, q_out=out)
    V.voxzip_rotary(desc, r, -pos, q=out, q_out=back)
    _, size = R.rotate(q, pos[None], r)
    assert float(((back - q).abs().double() - 4 * R.rotate_bound(q.double(), size, F32)).max()) <= 0


# ----------------------------------------------------------------------------- append

def fill(V, desc, n0, seed=0, paged=False, pages=None, shuffle=True):
    """A cache of random rows with units of n0 (a list per sequence) rows, NaN behind them."""
    rnd = gen(seed)
    B, L, H, C, D = desc.batch, desc.layers, desc.kv_heads, desc.capacity, desc.head_dim
    n = torch.tensor(n0, dtype=I32, device="cuda")[:, None, None].expand(B, L, H).contiguous()
    k, v = (rnd(B, L, H, C, D).to(desc.dtype) for _ in range(2))
    behind = (torch.arange(C, device="cuda") >= n[..., None])[..., None]
    k, v = k.masked_fill(behind, math.nan), v.masked_fill(behind, math.nan)
    score, pos = rnd(B, L, H, C).abs(), torch.arange(C, dtype=I32, device="cuda").expand(B, L, H, C).contiguous()
    if not paged:
        return dict(k=k, v=v, score=score, pos=pos, len=n)
    most = C // 64
    need = [int(x) // 64 + 1 for x in n.flatten().tolist()]
    pages = B * L * H * most if pages is None else pages
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)) if shuffle else torch.arange(pages)
    table, used = torch.full((B * L * H, most), -1, dtype=I32), 0
    for u, c in enumerate(need):
        c = min(c, most)
        table[u, :c] = perm[used:used + c].to(I32)
        used += c
    kp, vp = (torch.full((pages, 64, D), math.nan, dtype=desc.dtype, device="cuda") for _ in range(2))
    t = table.long().cuda()
    live = t >= 0
    kp[t[live]], vp[t[live]] = k.view(-1, most, 64, D)[live], v.view(-1, most, 64, D)[live]
    free = torch.zeros(pages, dtype=I32)
    free[:pages - used] = perm[used:].to(I32)
    return dict(k_pool=kp, v_pool=vp, page_table=table.view(B, L, H, most).cuda(), free_pages=free.cuda(),
                free_count=torch.tensor([pages - used], dtype=I32, device="cuda"), score=score, pos=pos, len=n, pages=pages, max_pages=most)


def unit_rows(c, b, l, h, n):
    """The first n rows of a unit, K and V."""
    if "k" in c:
        return c["k"][b, l, h, :n], c["v"][b, l, h, :n]
    t = c["page_table"][b, l, h, :-(-n // 64)].long()
    assert (t >= 0).all()
    return c["k_pool"][t].flatten(0, 1)[:n], c["v_pool"][t].flatten(0, 1)[:n]


def append(V, desc, c, first, count, k, v, new_pos, off, **kw):
    if "k" in c:
        V.voxzip_append(desc, first, count, k, v, new_pos, off, c["k"], c["v"], c["score"], c["pos"], c["len"], **kw)
    else:
        V.voxzip_append_paged(desc, c, first, count, k, v, new_pos, off, **kw)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("D,dtype", [(128, BF16), (64, F32)])
@pytest.mark.parametrize("ms,n0,gap", [([1], [0], 0), ([0, 5, 0, 64, 1], [3, 63, 64, 0, 127], 2), ([200, 131], [56, 120], 0),
                                       ([1] * 40, list(range(40)), 1)])
def test_append(V, paged, D, dtype, ms, n0, gap):
    B, L, first, count, Hq, H, C = len(ms), 4, 1, 2, 6, 2, 256
    desc, r = V.CacheDesc(B, L, Hq, H, D, C, dtype), V.RotaryDesc.make(64, sections=(16, 8, 8), pairing="adjacent")
    rnd, T = gen(3), gap + sum(ms) + 3
    c = fill(V, desc, n0, seed=5, paged=paged)
    before = {x: t.clone() for x, t in c.items() if isinstance(t, torch.Tensor)}
    qkv = rnd(count, T, (Hq + 2 * H) * D).to(dtype)
    q, k, v = (x.unflatten(-1, (-1, D)) for x in qkv.split([Hq * D, H * D, H * D], -1))
    pos, new_pos, off = positions_for(3, T), torch.arange(1000, 1000 + T, dtype=I32, device="cuda"), offsets(ms, gap)
    qo = torch.full((count, T, Hq, D), 7.0, dtype=dtype, device="cuda")
    append(V, desc, c, first, count, k, v, new_pos, off, rotary=r, positions=pos, q=q, q_out=qo, max_rows=max(ms))
    (want_q, sq), (want_k, sk) = R.rotate(q, pos, r), R.rotate(k, pos, r)
    assert (qo[:, :gap] == 7).all() and (qo[:, gap + sum(ms):] == 7).all()
    live = slice(gap, gap + sum(ms))
    close(qo[:, live], want_q[:, live], R.rotate_bound(want_q, sq, dtype)[:, live])
    end = gap
    for b, (m, n) in enumerate(zip(ms, n0)):
        t = slice(end, end + m)
        end += m
        for l in range(L):
            new = m if first <= l < first + count else 0
            assert (c["len"][b, l] == n + new).all()
            for h in range(H):
                kr, vr = unit_rows(c, b, l, h, n + new)
                k0, v0 = unit_rows(before, b, l, h, n)
                assert torch.equal(kr[:n], k0) and torch.equal(vr[:n], v0)
                if new:
                    close(kr[n:], want_k[l - first, t, h], R.rotate_bound(want_k, sk, dtype)[l - first, t, h])
                    assert torch.equal(vr[n:], v[l - first, t, h])
                    assert (c["score"][b, l, h, n:n + m] == 0).all() and torch.equal(c["pos"][b, l, h, n:n + m], new_pos[t])
                for x in ("score", "pos"):
                    assert torch.equal(c[x][b, l, h, :n], before[x][b, l, h, :n])
                    assert torch.equal(c[x][b, l, h, n + new:], before[x][b, l, h, n + new:])
                if not paged:
                    assert torch.isnan(c["k"][b, l, h, n + new:].float()).all() and torch.isnan(c["v"][b, l, h, n + new:].float()).all()
    if paged:
        check_pages(desc, c)


def check_pages(desc, c):
    """A unit of length n holds the pages of slots [0, n]; each page is held once or free once."""
    table, n = c["page_table"].flatten(0, 2).cpu(), c["len"].flatten().cpu()
    held = table[table >= 0].tolist()
    free = c["free_pages"][:int(c["free_count"])].tolist()
    assert sorted(held + free) == list(range(c["pages"]))
    for u in range(len(n)):
        have = min(int(n[u]) // 64 + 1, table.shape[1])
        assert (table[u, :have] >= 0).all() and (table[u, have:] == -1).all()


def test_append_without_scores_rows_as_they_are(V):
    """A slab that stage 1 will read: no scores, no positions; and rows that are rotated already."""
    desc, rnd = V.CacheDesc(2, 1, 4, 2, 64, 40, BF16), gen(2)
    c = fill(V, desc, [0, 0])
    k, v = rnd(1, 50, 2, 64).to(BF16), rnd(1, 50, 2, 64).to(BF16)
    V.voxzip_append(desc, 0, 1, k, v, None, offsets([30, 20]), c["k"], c["v"], None, None, c["len"])
    assert c["len"].flatten().tolist() == [30, 30, 20, 20]
    assert torch.equal(c["k"][0, 0, 1, :30], k[0, :30, 1]) and torch.equal(c["v"][1, 0, 0, :20], v[0, 30:, 0])


def test_append_skips_a_unit_that_would_overflow(V):
    desc, rnd = V.CacheDesc(3, 1, 4, 2, 64, 64, BF16), gen(2)
    c = fill(V, desc, [10, 61, 60])
    c["len"][0, 0, 1] = -1
    before = {x: t.clone() for x, t in c.items()}
    k = rnd(1, 12, 2, 64).to(BF16)
    V.voxzip_append(desc, 0, 1, k, k, torch.zeros(12, dtype=I32, device="cuda"), offsets([4, 4, 4]), c["k"], c["v"], c["score"],
                    c["pos"], c["len"])
    assert V.voxzip_get_status() == V.DEV_CAPACITY
    assert c["len"].flatten().tolist() == [14, -1, 61, 61, 64, 64]
    assert torch.equal(c["score"][1], before["score"][1]) and torch.equal(c["pos"][0, 0, 1], before["pos"][0, 0, 1])
    assert torch.equal(c["k"][1, 0, :, :61], before["k"][1, 0, :, :61]) and torch.isnan(c["k"][1, 0, :, 61:].float()).all()


@pytest.mark.parametrize("off", [[0, 5, 3], [-1, 4, 8], [0, 4, 9], [5, 4, 8]])
def test_bad_offsets_change_nothing(V, off):
    desc, rnd = V.CacheDesc(2, 1, 4, 2, 64, 64, BF16), gen(2)
    c = fill(V, desc, [10, 20])
    before = {x: t.clone() for x, t in c.items()}
    k, q = rnd(1, 8, 2, 64).to(BF16), rnd(1, 8, 4, 64).to(BF16)
    off = torch.tensor(off, dtype=I32, device="cuda")
    V.voxzip_append(desc, 0, 1, k, k, torch.zeros(8, dtype=I32, device="cuda"), off, c["k"], c["v"], c["score"], c["pos"], c["len"])
    assert V.voxzip_get_status() == V.DEV_BAD_SPANS
    for x in before:
        assert torch.equal(torch.nan_to_num(c[x].float()), torch.nan_to_num(before[x].float()))
    out = torch.full_like(q, 3.0)
    V.voxzip_prompt_attention(desc, 0, 1, q, off, c["k"], c["v"], c["len"], out)
    assert V.voxzip_get_status() & V.DEV_BAD_SPANS


def test_append_takes_all_its_pages_or_none(V):
    """6 free pages; unit 0 (64 rows kept) gets 200 rows, unit 1 (70 kept) 300: 4 and 5 pages."""
    desc, rnd = V.CacheDesc(2, 1, 1, 1, 64, 512, BF16), gen(2)
    c = fill(V, desc, [64, 70], paged=True, pages=10)
    assert int(c["free_count"]) == 6
    k = rnd(1, 500, 1, 64).to(BF16)
    V.voxzip_append_paged(desc, c, 0, 1, k, k, torch.zeros(500, dtype=I32, device="cuda"), offsets([200, 300]))
    assert V.voxzip_get_status() == V.DEV_CAPACITY
    got = c["len"].flatten().tolist()
    assert got in ([264, 70], [64, 370])  # which one comes first is not said
    check_pages(desc, c)
    # room for the rows but not for the page of the next append's slot: the rows are appended
    c = fill(V, desc, [10, 10], paged=True, pages=2)
    V.voxzip_append_paged(desc, c, 0, 1, k[:, :54], k[:, :54], torch.zeros(54, dtype=I32, device="cuda"), offsets([54, 0]))
    assert c["len"].flatten().tolist() == [64, 10] and int(c["free_count"]) == 0
    assert c["page_table"][0, 0, 0, :2].tolist()[1] == -1
    # a full unit has no next slot
    c = fill(V, desc, [500, 0], paged=True)
    V.voxzip_append_paged(desc, c, 0, 1, k[:, :12], k[:, :12], torch.zeros(12, dtype=I32, device="cuda"), offsets([12, 0]))
    assert c["len"].flatten().tolist() == [512, 0]
    check_pages(desc, c)


def test_a_page_outside_the_pool_is_reported(V):
    desc, rnd = V.CacheDesc(1, 1, 2, 1, 64, 192, BF16), gen(2)
    for page in (-7, 3, 2 ** 30):
        c = fill(V, desc, [70], paged=True)
        c["page_table"][0, 0, 0, 1] = page
        pools = c["k_pool"].clone()
        k, q = rnd(1, 3, 1, 64).to(BF16), rnd(1, 3, 2, 64).to(BF16)
        if page >= 0:
            V.voxzip_append_paged(desc, c, 0, 1, k, k, torch.zeros(3, dtype=I32, device="cuda"), offsets([3]))
            assert V.voxzip_get_status() == V.DEV_CAPACITY
            assert torch.equal(torch.nan_to_num(pools), torch.nan_to_num(c["k_pool"]))
        # its rows count as zeros: the logits 0, the values 0
        c["len"].fill_(70)
        c["page_table"][0, 0, 0, 0] = int(c["page_table"][0, 0, 0, 0])
        out = torch.empty_like(q)
        V.voxzip_prompt_attention_paged(desc, c, 0, 1, q, offsets([3]), out)
        assert V.voxzip_get_status() == V.DEV_CAPACITY
        kk, vv = torch.zeros(70, 64, device="cuda").to(BF16), torch.zeros(70, 64, device="cuda").to(BF16)
        at = int(c["page_table"][0, 0, 0, 0])
        kk[:64], vv[:64] = c["k_pool"][at], c["v_pool"][at]
        want, mag, size = R.attention(q[0], kk, vv, 68, 0.125)
        close(out[0], want, R.attention_bound(want, mag, size, 70, 64, BF16))


# ----------------------------------------------------------------------------- attention

def attend(V, desc, c, first, count, q, off, out, **kw):
    if "k" in c:
        V.voxzip_prompt_attention(desc, first, count, q, off, c["k"], c["v"], c["len"], out, **kw)
    else:
        V.voxzip_prompt_attention_paged(desc, c, first, count, q, off, out, **kw)


def check_attention(V, desc, c, ms, ns, first=0, count=None, gap=0, seed=0, scale=0.0, q=None, strided=False, **kw):
    count = desc.layers - first if count is None else count
    D, G, T = desc.head_dim, desc.q_heads // desc.kv_heads, gap + sum(ms) + 2
    rnd = gen(seed + 77)
    if q is None:
        q = rnd(count, T, desc.q_heads + (3 if strided else 0), D).to(desc.dtype)[:, :, :desc.q_heads]
    out = torch.full((count, T, desc.q_heads, D), 7.0, dtype=desc.dtype, device="cuda")
    attend(V, desc, c, first, count, q, offsets(ms, gap), out, sm_scale=scale, **kw)
    assert (out[:, :gap] == 7).all() and (out[:, gap + sum(ms):] == 7).all()
    end = gap
    for b, (m, n) in enumerate(zip(ms, ns)):
        t = slice(end, end + m)
        end += m
        for l in range(count):
            for h in range(desc.kv_heads):
                k, v = unit_rows(c, b, first + l, h, n)
                heads = slice(h * G, (h + 1) * G)
                want, mag, size = R.attention(q[l, t, heads], k, v, n - m + 1, scale or 1 / math.sqrt(D))
                close(out[l, t, heads], want, R.attention_bound(want, mag, size, n, D, desc.dtype), (b, l, h))
    return out


SHAPES = [  # q heads, kv heads, D
    (32, 4, 128), (4, 4, 128), (2, 1, 64), (12, 4, 128), (16, 1, 64), (5, 1, 128), (3, 3, 64), (26, 2, 64)]


@pytest.mark.parametrize("Hq,H,D", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("paged", [False, True])
def test_attention_of_ragged_prompts(V, Hq, H, D, dtype, paged):
    """First prompts and later turns, of one token to a few tiles, an empty one among them."""
    ms, ns = [1, 0, 17, 130, 64, 5, 2], [1, 30, 17, 130, 300, 128, 131]
    desc = V.CacheDesc(len(ms), 2, Hq, H, D, 320, dtype)
    c = fill(V, desc, ns, seed=Hq + D, paged=paged)
    check_attention(V, desc, c, ms, ns, first=1, count=1, gap=3, strided=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 63), (1, 64), (1, 65), (1, 4097), (2, 129), (15, 128), (16, 128), (17, 128), (31, 33), (32, 32),
                                 (33, 257), (128, 128), (129, 1000), (255, 256), (257, 513)])
def test_attention_sizes_around_the_tiles(V, dtype, m, n):
    for Hq, H, D in ((8, 1, 128), (1, 1, 64)):
        desc = V.CacheDesc(1, 1, Hq, H, D, n + 7, dtype)
        check_attention(V, desc, fill(V, desc, [n], seed=m), [m], [n])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hint", [dict(), dict(max_rows=9, max_len=1500), dict(max_rows=1, max_len=1), dict(max_rows=500, max_len=64)])
def test_hints_do_not_change_what_is_computed(V, dtype, hint):
    """Few rows over long caches: the keys are shared out, or not, as the hints say."""
    ms, ns = [9, 3], [1500, 700]
    desc = V.CacheDesc(2, 1, 8, 2, 64, 2048, dtype)
    check_attention(V, desc, fill(V, desc, ns), ms, ns, **hint)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("paged", [False, True])
def test_rows_that_see_nothing_are_zero(V, dtype, paged):
    """A unit shorter than its sequence's tokens (evicted since): the first tokens see no slot; nor does any of an
    empty unit."""
    ms, ns = [40, 6, 200, 3], [10, 0, 130, 2]
    desc = V.CacheDesc(4, 1, 4, 2, 64, 192, dtype)
    out = check_attention(V, desc, fill(V, desc, ns, paged=paged), ms, ns)
    assert (out[0, :30] == 0).all() and (out[0, 40:46] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan, "largest"])
@pytest.mark.parametrize("Hq,H,D,m,n", [(8, 1, 128, 60, 300), (2, 2, 64, 200, 200), (4, 1, 128, 3, 1000)])
def test_what_a_token_does_not_see_has_no_part(V, dtype, value, Hq, H, D, m, n):
    """Infinities, NaN and the type's largest numbers in rows of the turn: tokens before them are as without them, tokens
    from them on have what the formula gives."""
    value = torch.finfo(dtype).max if value == "largest" else value
    desc = V.CacheDesc(1, 1, Hq, H, D, n + 40, dtype)
    for where in ("v", "k"):
        c = fill(V, desc, [n], seed=1)
        clean = check_attention(V, desc, c, [m], [n])
        bad = n - m // 2 - 1  # the slot of a token in the middle of the turn
        c[where][0, 0, :, bad, 5] = value
        T = m + 2
        out = torch.full((1, T, Hq, D), 7.0, dtype=dtype, device="cuda")
        q = gen(77)(1, T, Hq, D).to(dtype)
        V.voxzip_prompt_attention(desc, 0, 1, q, offsets([m]), c["k"], c["v"], c["len"], out)
        before = bad - (n - m)
        assert torch.equal(out[:, :before], clean[:, :before])
        after = out[:, before:m]
        if where == "k":  # q times it: infinite logits of either sign, or NaN
            if not math.isfinite(value):
                assert not torch.equal(after, clean[:, before:m])
        else:
            assert torch.equal(after[..., :5], clean[:, before:m, :, :5]) and torch.equal(after[..., 6:], clean[:, before:m, :, 6:])
            if math.isnan(value):
                assert torch.isnan(after[..., 5]).all()
            elif math.isinf(value):
                assert (after[..., 5] == value).all()
            else:
                assert torch.isfinite(after[..., 5]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logits_that_grow_along_the_keys(V, dtype):
    """Every key's logit above all before it, by 2 each: the running maximum moves with every tile, by far more than
    a weight could carry; and a far one at the start that outweighs all that follow."""
    n, D = 700, 64
    desc = V.CacheDesc(2, 1, 2, 1, D, n, dtype)
    c = fill(V, desc, [n, n], seed=3)
    c["k"].zero_()
    c["k"][0, 0, 0, :, 0] = torch.arange(n, device="cuda", dtype=F32).to(dtype)
    c["k"][1, 0, 0, 0, 0] = 500.0
    T = n + 2
    q = torch.zeros(1, 2 * T, 2, D, dtype=dtype, device="cuda")
    q[..., 0] = 2.0 * 8
    check_attention(V, desc, c, [300, 300], [n, n], q=q[:, :602])


@pytest.mark.parametrize("scale", [0.02, 1.7])
def test_scale(V, scale):
    for dtype in (BF16, F32):
        desc = V.CacheDesc(1, 1, 2, 1, 64, 200, dtype)
        check_attention(V, desc, fill(V, desc, [190]), [50], [190], scale=scale)


def test_a_length_outside_the_capacity_is_reported(V):
    for dtype in (BF16, F32):
        desc = V.CacheDesc(2, 1, 2, 1, 64, 64, dtype)
        c = fill(V, desc, [20, 30])
        for bad in (-1, 65):
            c["len"][0] = bad
            q, out = gen(0)(1, 8, 2, 64).to(dtype), torch.full((1, 8, 2, 64), 7.0, dtype=dtype, device="cuda")
            V.voxzip_prompt_attention(desc, 0, 1, q, offsets([4, 4]), c["k"], c["v"], c["len"], out)
            assert V.voxzip_get_status() == V.DEV_CAPACITY
            assert (out[:, :4] == 7).all() and not (out[:, 4:] == 7).any()


def test_attention_repeats_bit_for_bit_and_on_any_stream(V):
    for dtype in (BF16, F32):
        desc = V.CacheDesc(1, 1, 8, 2, 128, 3000, dtype)
        c = fill(V, desc, [2900])
        q = gen(5)(1, 11, 8, 128).to(dtype)
        outs = [torch.empty_like(q) for _ in range(4)]
        off = offsets([11])
        side = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for o, s in zip(outs, (None, side[0], side[1], side[0])):  # two at once on the two side streams
            V.voxzip_prompt_attention(desc, 0, 1, q, off, c["k"], c["v"], c["len"], o, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(outs[0], o) for o in outs[1:])


def test_a_turn_captured_and_replayed(V):
    """Append and attention of a turn in a CUDA graph, replayed on other rows and other lengths."""
    desc, r = V.CacheDesc(2, 1, 4, 2, 64, 512, BF16), V.RotaryDesc.make(64)
    rnd, ms = gen(4), [30, 21]
    c = fill(V, desc, [100, 170])
    qkv, pos = rnd(1, 51, 8, 64).to(BF16), torch.arange(51, dtype=I32, device="cuda")
    qo, out = torch.empty(1, 51, 4, 64, dtype=BF16, device="cuda"), torch.empty(1, 51, 4, 64, dtype=BF16, device="cuda")
    off = offsets(ms)

    def turn():
        append(V, desc, c, 0, 1, qkv[:, :, 4:6], qkv[:, :, 6:], pos, off, rotary=r, positions=pos, q=qkv[:, :, :4], q_out=qo)
        attend(V, desc, c, 0, 1, qo, off, out)

    start = {x: t.clone() for x, t in c.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        turn()
    for seed in (6, 7):
        for x in c:
            c[x].copy_(start[x])
        c["len"].copy_(torch.tensor([100 - seed, 170 - 20 * seed], dtype=I32, device="cuda")[:, None, None].expand(2, 1, 2))
        qkv.copy_(gen(seed)(1, 51, 8, 64))
        state = {x: t.clone() for x, t in c.items()}
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), {x: t.clone() for x, t in c.items()}
        for x in c:
            c[x].copy_(state[x])
        turn()
        assert torch.equal(got[0], out)
        for x in c:
            assert torch.equal(torch.nan_to_num(got[1][x].float()), torch.nan_to_num(c[x].float())), x


def test_caller_workspace_and_zero_tokens(V):
    desc = V.CacheDesc(1, 1, 8, 2, 128, 3000, BF16)
    c = fill(V, desc, [2900])
    q = gen(5)(1, 11, 8, 128).to(BF16)
    a, b = torch.empty_like(q), torch.empty_like(q)
    ws = torch.empty(V.voxzip_prompt_attention_workspace_size(desc, 1, 11), dtype=torch.uint8, device="cuda")
    V.voxzip_prompt_attention(desc, 0, 1, q, offsets([11]), c["k"], c["v"], c["len"], a, workspace=ws)
    V.voxzip_prompt_attention(desc, 0, 1, q, offsets([11]), c["k"], c["v"], c["len"], b)
    assert torch.equal(a, b)
    with pytest.raises(V.VoxZipError):
        V.voxzip_prompt_attention(desc, 0, 1, q, offsets([11]), c["k"], c["v"], c["len"], a, workspace=ws[:256])
    none = q[:, :0]
    V.voxzip_prompt_attention(desc, 0, 1, none, offsets([0]), c["k"], c["v"], c["len"], a[:, :0])
    V.voxzip_append(desc, 0, 1, none[:, :, :2], none[:, :, :2], torch.zeros(0, dtype=I32, device="cuda"), offsets([0]), c["k"], c["v"],
                    c["score"], c["pos"], c["len"])
    assert (c["len"] == 2900).all()


def test_binding_refuses(V):
    desc = V.CacheDesc(1, 1, 4, 2, 64, 64, BF16)
    c = fill(V, desc, [10])
    q, out, off = torch.zeros(1, 4, 4, 64, dtype=BF16, device="cuda"), torch.zeros(1, 4, 4, 64, dtype=BF16, device="cuda"), offsets([4])
    bad = [q[..., ::2].repeat(1, 1, 1, 2)[..., :63], q.transpose(1, 2), q.float(), q[0], torch.zeros(1, 4, 8, 64, dtype=BF16, device="cuda")[:, :, ::2],
           torch.zeros(1, 4, 4 * 64 + 4, dtype=BF16, device="cuda")[..., 4:].unflatten(-1, (4, 64)), q[:, :1].expand(1, 4, 4, 64),
           torch.zeros(2, 4, 4, 64, dtype=BF16, device="cuda")]
    for x in bad:
        with pytest.raises(ValueError):
            V.voxzip_prompt_attention(desc, 0, 1, x, off, c["k"], c["v"], c["len"], out)
    with pytest.raises(ValueError):
        V.voxzip_prompt_attention(desc, 0, 1, q, off[:1], c["k"], c["v"], c["len"], out)
    with pytest.raises(TypeError):  # positions are kept, but none are given
        V.voxzip_append(desc, 0, 1, q[:, :, :2], q[:, :, :2], None, off, c["k"], c["v"], c["score"], c["pos"], c["len"])
    with pytest.raises(ValueError):
        V.voxzip_rotary(desc, V.RotaryDesc.make(64, sections=(16, 16)), torch.zeros(1, 4, dtype=I32, device="cuda"), q=q, q_out=out)
    with pytest.raises(V.VoxZipError):
        V.voxzip_prompt_attention(desc, 1, 1, q, off, c["k"], c["v"], c["len"], out)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_several_layers_in_one_call(V, dtype):
    """Layers whose units differ in length (budgets per layer), queries at a stride of layers of their own."""
    ms, desc = [40, 3], V.CacheDesc(2, 4, 6, 2, 64, 200, dtype)
    c = fill(V, desc, [160, 90])
    c["len"][:, 2] -= 17
    c["len"][1, 3, 1] += 5
    c["k"].nan_to_num_(0.0)
    c["v"].nan_to_num_(0.0)
    for first, count in ((0, 4), (1, 3), (3, 1)):
        q = gen(2)(count, 2, 45, 6, 64).to(dtype)[:, 1]
        out = torch.empty(count, 45, 6, 64, dtype=dtype, device="cuda")
        V.voxzip_prompt_attention(desc, first, count, q, offsets(ms), c["k"], c["v"], c["len"], out)
        for b, t in enumerate((slice(0, 40), slice(40, 43))):
            for l in range(count):
                for h in range(2):
                    n = int(c["len"][b, first + l, h])
                    k, v = unit_rows(c, b, first + l, h, n)
                    want, mag, size = R.attention(q[l, t, 3 * h:3 * h + 3], k, v, n - ms[b] + 1, 0.125)
                    close(out[l, t, 3 * h:3 * h + 3], want, R.attention_bound(want, mag, size, n, 64, dtype), (b, l, h))


@pytest.mark.parametrize("dtype,paged", [(BF16, False), (BF16, True), (F32, False)])
def test_many_sequences(V, dtype, paged):
    """More sequences than a warp has lanes, most of a token or none."""
    ms = [i % 4 for i in range(75)] + [140]
    ns = [m + 3 * i % 60 for i, m in enumerate(ms)]
    desc = V.CacheDesc(len(ms), 1, 4, 2, 64, 256, dtype)
    check_attention(V, desc, fill(V, desc, ns, paged=paged), ms, ns, gap=1)


def test_a_wrong_hint_of_the_rows_appends_the_same(V):
    desc, r = V.CacheDesc(2, 1, 4, 2, 64, 400, BF16), V.RotaryDesc.make(64)
    qkv, pos, off = gen(1)(1, 310, 8, 64).to(BF16), torch.arange(310, dtype=I32, device="cuda"), offsets([300, 10])
    got = []
    for hint in (0, 1, 300, 10 ** 6):
        c, qo = fill(V, desc, [7, 90]), torch.empty(1, 310, 4, 64, dtype=BF16, device="cuda")
        append(V, desc, c, 0, 1, qkv[:, :, 4:6], qkv[:, :, 6:], pos, off, rotary=r, positions=pos, q=qkv[:, :, :4], q_out=qo, max_rows=hint)
        got.append({**c, "q": qo})
    for g in got[1:]:
        for x in g:
            assert torch.equal(torch.nan_to_num(g[x].float()), torch.nan_to_num(got[0][x].float())), x


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_cache_beyond_32_bit_offsets(V, dtype):
    """More than 2^32 bytes, and elements beyond 2^31, in front of the unit."""
    D, C = 128, 3_000_000
    desc = V.CacheDesc(1, 3, 4, 2, D, C, dtype)
    k, v = (torch.empty(1, 3, 2, C, D, dtype=dtype, device="cuda") for _ in range(2))
    assert k.numel() > 2 ** 31
    ln = torch.zeros(1, 3, 2, dtype=I32, device="cuda")
    n = C - 25
    for first in (n - 300, 0):  # the rows in front of the turn: the last ones of the unit, and the first ones
        rows = torch.arange(first, first + 300, device="cuda")
        rnd = gen(first % 97)
        kk, vv = rnd(2, 320, D).to(dtype), rnd(2, 320, D).to(dtype)
        k[0, 2, :, rows], v[0, 2, :, rows] = kk[:, :300], vv[:, :300]
        ln[0, 2] = first + 300
        V.voxzip_append(desc, 2, 1, kk[None, :, 300:].transpose(1, 2).contiguous(), vv[None, :, 300:].transpose(1, 2).contiguous(), None,
                        offsets([20]), k, v, None, None, ln)
        assert (ln[0, 2] == first + 320).all() and torch.equal(k[0, 2, :, first + 300:first + 320], kk[:, 300:])
        if first == 0:
            q, out = rnd(1, 20, 4, D).to(dtype), torch.empty(1, 20, 4, D, dtype=dtype, device="cuda")
            V.voxzip_prompt_attention(desc, 2, 1, q, offsets([20]), k, v, ln, out, max_len=320)
            for h in range(2):
                want, mag, size = R.attention(q[0, :, 2 * h:2 * h + 2], kk[h], vv[h], 301, D ** -0.5)
                close(out[0, :, 2 * h:2 * h + 2], want, R.attention_bound(want, mag, size, 320, D, dtype))


def test_another_device_is_refused(V, monkeypatch):
    desc = V.CacheDesc(1, 1, 4, 2, 64, 64, BF16)
    c, q = fill(V, desc, [10]), torch.zeros(1, 4, 4, 64, dtype=BF16, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        V.voxzip_prompt_attention(desc, 0, 1, q, offsets([4]), c["k"], c["v"], c["len"], q.clone())
    with pytest.raises(ValueError, match="current device"):
        V.voxzip_append(desc, 0, 1, q[:, :, :2], q[:, :, :2], torch.zeros(4, dtype=I32, device="cuda"), offsets([4]), c["k"], c["v"], c["score"],
                        c["pos"], c["len"])
    with pytest.raises(ValueError, match="current device"):
        V.voxzip_rotary(desc, V.RotaryDesc.make(64), torch.zeros(4, dtype=I32, device="cuda"), q=q, q_out=q)


# ----------------------------------------------------------------------------- all of it, as it is used

@pytest.mark.parametrize("dtype,paged", [(BF16, False), (BF16, True), (F32, False)])
def test_a_conversation(V, dtype, paged):
    """A prompt made into a slab, stage 1, decode steps on rotated rows, an eviction, a second turn, and steps after it:
    every attention against the plain one on the rows that the cache holds."""
    B, L, Hq, H, D, ms = 2, 2, 4, 2, 64, [90, 70]
    stride, cap = max(ms), 256
    rnd = gen(8)
    r = V.RotaryDesc.make(64, sections=(12, 10, 10), in_turns=True)
    slab = V.CacheDesc(B, L, Hq, H, D, stride, dtype)
    pre = dict(k=torch.full((B, L, H, stride, D), math.nan, dtype=dtype, device="cuda"), v=torch.zeros(B, L, H, stride, D, dtype=dtype, device="cuda"),
               len=torch.zeros(B, L, H, dtype=I32, device="cuda"))

    def rows(m):
        qkv = rnd(L, sum(m), (Hq + 2 * H) * D).to(dtype)
        return [x.unflatten(-1, (-1, D)) for x in qkv.split([Hq * D, H * D, H * D], -1)]

    # the prompt, layer by layer, as a model runs
    q, k, v = rows(ms)
    off, T = offsets(ms), sum(ms)
    pos = torch.cat([torch.arange(m) for m in ms]).to(I32).cuda().expand(3, T).contiguous()
    qo, out = torch.empty(L, T, Hq, D, dtype=dtype, device="cuda"), torch.empty(L, T, Hq, D, dtype=dtype, device="cuda")
    for l in range(L):
        V.voxzip_append(slab, l, 1, k[l:l + 1], v[l:l + 1], None, off, pre["k"], pre["v"], None, None, pre["len"], rotary=r,
                        positions=pos, q=q[l:l + 1], q_out=qo[l:l + 1], max_rows=stride)
        V.voxzip_prompt_attention(slab, l, 1, qo[l:l + 1], off, pre["k"], pre["v"], pre["len"], out[l:l + 1], max_rows=stride)
    want_k, size = R.rotate(k, pos, r)
    for b, m in enumerate(ms):
        t = slice(int(off[b]), int(off[b + 1]))
        for l in range(L):
            for h in range(H):
                close(pre["k"][b, l, h, :m], want_k[l, t, h], R.rotate_bound(want_k, size, dtype)[l, t, h])
                want, mag, big = R.attention(qo[l, t, 2 * h:2 * h + 2], pre["k"][b, l, h, :m], pre["v"][b, l, h, :m], 1, 0.125)
                close(out[l, t, 2 * h:2 * h + 2], want, R.attention_bound(want, mag, big, m, D, dtype))

    # stage 1: spans of four tokens to one row, from the tenth token on
    desc = V.CacheDesc(B, L, Hq, H, D, cap, dtype)
    from paper_2608_08569_gb300.session import Session
    s = Session(desc, [60, 50], 0.98, pages=64 if paged else None)
    starts = [torch.arange(10, m - 3, 4, dtype=I32) for m in ms]
    n = [len(x) for x in starts]
    i32 = lambda x: torch.as_tensor(x, dtype=I32).cuda()  # noqa: E731
    begin, length = [10, 10], [4 * x for x in n]
    s.prefill(pre["k"].nan_to_num(), pre["v"], i32(ms), i32(begin), i32(length), i32([0, n[0], n[0] + n[1]]), torch.cat(starts).cuda(),
              torch.cat(starts).cuda() + 4, i32([1] * sum(n)))
    kept = [m - 3 * x for m, x in zip(ms, n)]
    assert s.cache["len"][:, 0, 0].tolist() == kept

    def step(at):
        q, k, v = (x.view(L, B, -1, D) for x in rows([1, 1]))
        p = i32(at).expand(3, B).contiguous()
        qr, kr = torch.empty_like(q).contiguous(), torch.empty(L, B, H, D, dtype=dtype, device="cuda")
        V.voxzip_rotary(desc, r, p, q=q, k=k, q_out=qr, k_out=kr)
        out = torch.empty_like(qr)
        s.decode(qr, kr, v.contiguous(), p[0].contiguous(), out)
        for b in range(B):
            for l in range(L):
                for h in range(H):
                    m = int(s.cache["len"][b, l, h])
                    kk, vv = unit_rows(s.cache, b, l, h, m)
                    assert torch.equal(kk[-1], kr[l, b, h])
                    want, mag, big = R.attention(qr[l, b, 2 * h:2 * h + 2][None], kk, vv, m, 0.125)
                    # (the step adds its parts up in another order: twice the bound)
                    close(out[l, b, 2 * h:2 * h + 2][None], want, 2 * R.attention_bound(want, mag, big, m, D, dtype))

    at = list(ms)
    for _ in range(3):
        step(at)
        at = [x + 1 for x in at]
    before = s.cache["len"][:, 0, 0].tolist()
    s.evict()
    assert s.cache["len"][:, 0, 0].tolist() == [min(x, y) for x, y in zip(before, (60, 50))]

    # the second turn, and its answer
    turn = [33, 5]
    n0 = s.cache["len"][:, 0, 0].tolist()
    q, k, v = rows(turn)
    T = sum(turn)
    pos = torch.cat([torch.arange(m) + a for m, a in zip(turn, at)]).to(I32).cuda()
    out, qo = torch.empty(L, T, Hq, D, dtype=dtype, device="cuda"), torch.empty(L, T, Hq, D, dtype=dtype, device="cuda")
    for l in range(L):
        s.extend(q[l:l + 1], k[l:l + 1], v[l:l + 1], pos, offsets(turn), out[l:l + 1], max_rows=33, rotary=r,
                 positions=pos.expand(3, T).contiguous(), q_out=qo[l:l + 1], layer_begin=l, layer_count=1)
    assert s.n_max >= max(x + m for x, m in zip(n0, turn)) and (s.cache["len"][:, 1, 1].tolist() == [x + m for x, m in zip(n0, turn)])
    off = offsets(turn)
    for b, m in enumerate(turn):
        t = slice(int(off[b]), int(off[b + 1]))
        for l in range(L):
            for h in range(H):
                kk, vv = unit_rows(s.cache, b, l, h, n0[b] + m)
                assert torch.equal(vv[n0[b]:], v[l, t, h])
                want, mag, big = R.attention(qo[l, t, 2 * h:2 * h + 2], kk, vv, n0[b] + 1, 0.125)
                close(out[l, t, 2 * h:2 * h + 2], want, R.attention_bound(want, mag, big, n0[b] + m, D, dtype))
    assert (s.cache["score"][0, :, :, n0[0]:n0[0] + 33] == 0).all()
    step([a + m for a, m in zip(at, turn)])
    if paged:
        check_pages(desc, s.cache)
    # without a place for the rotated queries, and without a rotation
    again = torch.empty_like(out)
    s.extend(q, k, v, pos, offsets(turn), again, max_rows=33, rotary=r, positions=pos.expand(3, T).contiguous())
    s.extend(q, k, v, pos, offsets(turn), again, max_rows=33)
    assert s.cache["len"][:, 0, 0].tolist() == [x + 3 * m + 1 for x, m in zip(n0, turn)]


def test_a_packed_session_refuses_a_turn(V):
    from paper_2608_08569_gb300.session import Session
    s = Session(V.CacheDesc(1, 1, 2, 1, 64, 64, BF16), [32], 0.9, kv_bits=4)
    x = torch.zeros(1, 3, 2, 64, dtype=BF16, device="cuda")
    with pytest.raises(ValueError, match="kv_bits"):
        s.extend(x, x[:, :, :1], x[:, :, :1], torch.zeros(3, dtype=I32, device="cuda"), offsets([3]), x.clone(), max_rows=3)


@pytest.mark.skipif(os.environ.get("VOXZIP_CHECKED", "0") not in ("", "0"), reason="this is the checked run")
def test_checked_build(V):
    """The range-checked build gives the same results and no bit of VOXZIP_DEV_BOUNDS."""
    from paper_2608_08569_gb300.build import build_library
    build_library(checked=True)
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider"],
                       cwd=ROOT, env=dict(os.environ, VOXZIP_CHECKED="1"), capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
