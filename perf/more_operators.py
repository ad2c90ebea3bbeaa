"""Performance cases of a turn's prompt: its rows rotated, appended to a cache, and attending over it.

A request's prompt, and each later turn of its conversation, comes as packed rows of the model's
projections: sequence b's tokens are rows [off[b], off[b + 1]) of q, k and v, usually views of one
[tokens][(Hq + 2 Hkv) D] tensor. Per layer, positions are rotated into q and k, the k and v rows are
appended to the sequence's units (behind whatever compressed rows they hold), and the queries attend
over all of them, causally among their own rows.

kind "rotary"  q and k rows rotated by 1 to 3 position axes.
kind "append"  q and k rotated, k and v rows appended to a cache; each pass first drops what the last one
               appended, by copying the lengths back.
kind "attend"  the causal attention of the rows appended last, over the whole cache.
kind "turn"    an append and the attention behind it, on a dense or a paged cache.

The rotation turns the pair i of the first R channels by position[axis_i] * freq_i; a pair is channels
(i, i + R / 2) ("halves") or (2 i, 2 i + 1) ("adjacent"). Row i of a sequence's m rows in a unit of n rows
(its own included) sees slots [0, n - m + i].

Lengths belong to the case ("layout" seeds them); values come from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # True: the framework's operators, False: their plain forms

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
THINKER = dict(q_heads=32, kv_heads=4, head_dim=128, dtype="bf16")
# 64 pairs by time, height and width, taken in turn; one axis; the first 64 channels only, pairs side by side
AXES3 = dict(rotary_dim=128, theta=1e6, sections="24/20/20", turns=True, pairing="halves")
AXIS = dict(rotary_dim=64, theta=1e4, sections="32", turns=False, pairing="halves")
PARTIAL = dict(rotary_dim=64, theta=1e4, sections="16/8/8", turns=False, pairing="adjacent")
PAGE = 64


# ----------------------------------------------------------------------------- the cases

def _case(name, kind, *, batch, m, n0=0, ragged=False, layers=1, first=0, count=1, paged=False, far=0, layout=0, **shape):
    """m rows of every sequence (ragged: a quarter of it and up) behind n0 rows already cached (the same)."""
    return dict(name=name, kind=kind, batch=batch, m=m, n0=n0, ragged=ragged, layers=layers, first=first, count=count,
                paged=paged, far=far, layout=layout, **shape)


def listed():
    return [
        # One token of one sequence, all 48 layers, as the decode step takes them: the smallest call.
        _case("rotary_token", "rotary", batch=1, m=1, layers=48, count=48, far=46024, **THINKER, **AXES3),
        # A 10-min prompt in fp32, half of each head rotated, in pairs side by side.
        _case("rotary_prompt_f32", "rotary", batch=1, m=8012, **dict(THINKER, dtype="f32"), **PARTIAL),
        # A question of 57 tokens at most to four compressed 60-min recordings, one layer of four.
        _case("append_turn", "append", batch=4, m=57, n0=2301, ragged=True, layers=4, first=2, far=46024, layout=3,
              **THINKER, **AXES3),
        # A layer of a 60-min prompt.
        _case("append_60min", "append", batch=1, m=46024, **THINKER, **AXES3),
        # The question above on a paged cache, appended and attended.
        _case("turn_paged", "turn", batch=4, m=57, n0=2301, ragged=True, layers=4, first=2, paged=True, far=46024,
              layout=3, **THINKER, **AXES3),
        # 32 ragged prompts of 2-8 min, paged.
        _case("turn_batch32_paged", "turn", batch=32, m=6256, ragged=True, paged=True, layout=4, **THINKER, **AXES3),
        # The prompt of the smallest configuration, and of a 30-s clip, in fp32.
        _case("attend_tiny_f32", "attend", batch=1, m=632, q_heads=2, kv_heads=1, head_dim=64, dtype="f32", **AXIS),
        _case("attend_30s_f32", "attend", batch=1, m=631, **dict(THINKER, dtype="f32"), **AXES3),
        # Multi-head attention of D = 64, odd ragged lengths.
        _case("attend_mha64", "attend", batch=5, m=1237, ragged=True, layout=7, q_heads=16, kv_heads=16, head_dim=64,
              dtype="bf16", **AXIS),
        # 64 new tokens over an uncompressed 60-min cache: few rows, a long axis.
        _case("attend_long_cache", "attend", batch=1, m=64, n0=46024, **THINKER, **AXES3),
        # Prompts of 10 and of 60 minutes (the largest).
        _case("attend_10min", "attend", batch=1, m=8012, **THINKER, **AXES3),
        _case("attend_60min", "attend", batch=1, m=46024, **THINKER, **AXES3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(["rotary", "append", "attend", "attend", "attend", "turn"])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    heads, kv, dim = rng.choice([(32, 4, 128)] * 6 + [(16, 1, 64), (12, 4, 128), (16, 16, 64), (10, 2, 64), (32, 8, 128)])
    rot = AXES3 if dim == 128 and rng.random() < 0.7 else PARTIAL if rng.random() < 0.4 else AXIS
    batch = _log(rng, 1, 32)
    m = _log(rng, 1, 46024)
    n0 = 0 if rng.random() < 0.5 or kind == "rotary" else _log(rng, 1, 46024)
    layers = _log(rng, 1, 4) if kind in ("append", "turn") else 1
    count = layers
    if kind == "rotary" and m <= 8:
        layers = count = _log(rng, 1, 48)
    return _case("", kind, batch=batch, m=m, n0=n0, ragged=batch > 1 and rng.random() < 0.5, layers=layers, count=count,
                 paged=kind == "turn" and dtype == "bf16" and rng.random() < 0.7, far=rng.choice([0, 1000, 100000]),
                 layout=rng.randrange(1 << 20), q_heads=heads, kv_heads=kv, head_dim=dim, dtype=dtype, **rot)


def draw(rng):
    cases = listed()
    most = {k: max(_cost(c) for c in cases if c["kind"] == k) for k in ("rotary", "append", "attend", "turn")}
    f32 = max(_cost(c) for c in cases if c["kind"] == "attend" and c["dtype"] == "f32")
    while True:
        c = _draw_once(rng)
        cap = most[c["kind"]]
        if c["kind"] in ("attend", "turn") and c["dtype"] == "f32":
            cap = min(cap, 16 * f32)
        # what a pass holds on the card: rows of the packed tensors, the cache
        rows = c["batch"] * (c["m"] + c["n0"]) * c["layers"] * (c["q_heads"] + c["kv_heads"]) * c["head_dim"]
        if _cost(c) <= cap and rows < 2 ** 30:
            c.pop("name")
            return c


# ----------------------------------------------------------------------------- sizes of a case

def _lens(c):
    """Rows of every sequence, and rows cached before them."""
    if not c["ragged"]:
        return [c["m"]] * c["batch"], [c["n0"]] * c["batch"]
    rng = np.random.default_rng(c["layout"])
    m = rng.integers(max(1, c["m"] // 4), c["m"] + 1, c["batch"])
    n0 = rng.integers(c["n0"] // 2, c["n0"] + 1, c["batch"])
    m[0], n0[0] = c["m"], c["n0"]
    return [int(x) for x in m], [int(x) for x in n0]


def _capacity(c):
    return -(-(c["m"] + c["n0"] + 1) // PAGE) * PAGE


def work(case):
    c = case
    D, Hq, H, e = c["head_dim"], c["q_heads"], c["kv_heads"], 2 if c["dtype"] == "bf16" else 4
    m, n0 = _lens(c)
    T, axes = sum(m), len(c["sections"].split("/"))
    by = fl = 0
    if c["kind"] == "rotary":
        by, fl = T * (2 * (Hq + H) * D * e * c["count"] + 4 * axes), T * c["count"] * (Hq + H) * c["rotary_dim"] * 3
    if c["kind"] in ("append", "turn"):
        by += T * (c["count"] * (2 * (Hq + 2 * H) * D * e + 8 * H) + 4 * axes + 4)
        fl += T * c["count"] * (Hq + H) * c["rotary_dim"] * 3
    if c["kind"] in ("attend", "turn"):
        pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(m, n0))
        by += c["count"] * (2 * T * Hq * D * e + 2 * (T + sum(n0)) * H * D * e)
        fl += c["count"] * pairs * 4 * Hq * D
    return {"bytes": by, "flops": fl}


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 100)


# ----------------------------------------------------------------------------- inputs

class State:
    """What one case has in hand; fields by kind."""


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, g):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)


def _freqs(c):
    R = c["rotary_dim"]
    return [c["theta"] ** (-2.0 * i / R) for i in range(R // 2)]


def _axis_of_pairs(c):
    """The position axis of every pair: blocks of the sections' sizes, or the axes in turn while they last."""
    sec = [int(x) for x in c["sections"].split("/")]
    if not c["turns"]:
        return [a for a, k in enumerate(sec) for _ in range(k)]
    A = len(sec)
    return [i % A if i % A and i < A * sec[i % A] else 0 for i in range(sum(sec))]


def prepare(case, seed):
    c, s, g = case, State(), _generator(seed)
    B, L, n, Hq, H, D, dt = c["batch"], c["layers"], c["count"], c["q_heads"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]]
    s.case, s.kind, C = c, c["kind"], _capacity(c)
    m, n0 = _lens(c)
    T = sum(m)
    s.m, s.n0, s.T, s.shape = m, n0, T, (B, L, Hq, H, D, C, dt)
    off = np.concatenate([[0], np.cumsum(m)])
    s.off = torch.tensor(off, dtype=torch.int32, device="cuda")
    s.seq = torch.from_numpy(np.repeat(np.arange(B), m)).cuda()  # the sequence of every packed row
    s.row = torch.arange(T, device="cuda") - s.off.long()[s.seq]
    s.m_of, s.n0_of = torch.tensor(m, device="cuda"), torch.tensor(n0, device="cuda")
    s.freqs, s.axis, s.freq64 = _freqs(c), _axis_of_pairs(c), torch.tensor(_freqs(c), dtype=torch.float64, device="cuda")
    s.axis_t = torch.tensor(s.axis, device="cuda")
    # keys with 4 outlier channels per head, x8, as attention keys have
    scale = torch.ones(n, H, D)
    rng = np.random.default_rng(seed)
    for l in range(n):
        for h in range(H):
            scale[l, h, torch.from_numpy(rng.choice(D, 4, replace=False))] = 8.0
    scale = scale.to(dt).cuda()
    if s.kind != "attend":  # q, k and v: views of the projection's output
        s.qkv = _normal((n, T, (Hq + 2 * H) * D), dt, g)
        s.q, s.k, s.v = (x.unflatten(-1, (-1, D)) for x in s.qkv.split([Hq * D, H * D, H * D], -1))
        s.k.mul_(scale[:, None])
        # time runs on from where the conversation stands; the other axes are places in a frame
        A = len(c["sections"].split("/"))
        frame = torch.randint(0, 64, (A, T), generator=g, device="cuda")
        frame[0] = 0
        s.positions = (s.row + s.n0_of[s.seq] + c["far"] + frame).to(torch.int32)
        s.new_pos = s.positions[0].contiguous()
        s.q_out = torch.zeros((n, T, Hq, D), dtype=dt, device="cuda")
    else:
        s.q = _normal((n, T, Hq, D), dt, g)
    s.out = torch.zeros((n, T, Hq, D), dtype=dt, device="cuda")
    s.cache = s.desc = s.rot = None
    if s.kind == "rotary":
        s.k_out = torch.zeros((n, T, H, D), dtype=dt, device="cuda")
        return s
    len0 = torch.tensor(n0 if s.kind != "attend" else [a + b for a, b in zip(m, n0)], dtype=torch.int32, device="cuda")
    s.len0 = len0[:, None, None].expand(B, L, H).contiguous()
    score = torch.zeros((B, L, H, C), device="cuda").exponential_(1.0, generator=g)
    pos = torch.arange(C, dtype=torch.int32, device="cuda").expand(B, L, H, C).contiguous()
    if c["paged"]:
        # pages in a shuffled order, as after many requests; every unit holds the pages of slots [0, len]
        have = torch.div(s.len0.flatten().long(), PAGE, rounding_mode="floor") + 1
        most = -(-C // PAGE)
        pages = B * L * H * most + 3
        perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = torch.full((B * L * H, most), -1, dtype=torch.int32, device="cuda")
        live = torch.arange(most, device="cuda")[None] < have[:, None]
        used = int(sum(x // PAGE + 1 for x in n0)) * L * H
        table[live] = perm[:used]
        s.table0 = table.view(B, L, H, most)
        free = torch.zeros(pages, dtype=torch.int32, device="cuda")
        free[:pages - used] = perm[used:]
        s.free0, s.count0 = free, torch.tensor([pages - used], dtype=torch.int32, device="cuda")
        s.cache = dict(k_pool=_normal((pages, PAGE, D), dt, g), v_pool=_normal((pages, PAGE, D), dt, g),
                       page_table=s.table0.clone(), free_pages=free.clone(), free_count=s.count0.clone(), score=score, pos=pos,
                       len=s.len0.clone(), pages=pages, max_pages=most)
    else:
        s.cache = dict(k=_normal((B, L, H, C, D), dt, g), v=_normal((B, L, H, C, D), dt, g), score=score, pos=pos,
                       len=s.len0.clone())
        s.cache["k"][:, c["first"]:c["first"] + n].mul_(scale[None, :, :, None])
    return s


# ----------------------------------------------------------------------------- the plain forms

def _plain_rotate(s, x):
    """x [layers][T][heads][D], rotated, in fp32 (angles in 64 bits)."""
    half = len(s.freqs)
    angle = s.positions[s.axis_t].t().double() * s.freq64  # [T][R / 2]
    cos, sin = (f(angle).float()[None, :, None] for f in (torch.cos, torch.sin))
    x = x.float()
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    if s.case["pairing"] == "halves":
        lo, hi = r[..., :half], r[..., half:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin, rest], -1)
    lo, hi = r[..., 0::2], r[..., 1::2]
    return torch.cat([torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], -1).flatten(-2), rest], -1)


def _plain_append(s):
    c, cache = s.case, s.cache
    first, n, H = c["first"], c["count"], c["kv_heads"]
    s.q_out.copy_(_plain_rotate(s, s.q))
    k = _plain_rotate(s, s.k).to(s.q.dtype)
    b = s.seq[:, None, None]  # [T][layers][heads]
    l = torch.arange(first, first + n, device="cuda")[None, :, None]
    h = torch.arange(H, device="cuda")[None, None]
    slot = s.len0.long()[b, l, h] + s.row[:, None, None]
    if c["paged"]:
        # new pages come off the top of the stack, in the order of layers, sequences and heads
        len0 = s.len0[:, first:first + n].transpose(0, 1).long()  # [layers][B][H]
        had = torch.div(len0, PAGE, rounding_mode="floor") + 1
        new = torch.div(len0 + s.m_of[None, :, None], PAGE, rounding_mode="floor") + 1 - had
        before = (new.flatten().cumsum(0) - new.flatten()).view(new.shape)
        table = cache["page_table"][:, first:first + n].transpose(0, 1)  # a view
        i = torch.arange(table.shape[-1], device="cuda") - had[..., None]
        page = s.free0[(s.count0.long() - 1 - before[..., None] - i).clamp(0, cache["pages"] - 1)]
        table.copy_(torch.where((i >= 0) & (i < new[..., None]), page, table))
        cache["free_count"].copy_(s.count0 - new.sum())
        page = cache["page_table"].long()[b, l, h, torch.div(slot, PAGE, rounding_mode="floor")]
        cache["k_pool"][page, slot % PAGE] = k.transpose(0, 1)
        cache["v_pool"][page, slot % PAGE] = s.v.transpose(0, 1)
    else:
        cache["k"][b, l, h, slot] = k.transpose(0, 1)
        cache["v"][b, l, h, slot] = s.v.transpose(0, 1)
    cache["score"][b, l, h, slot] = 0.0
    cache["pos"][b, l, h, slot] = s.new_pos[:, None, None]
    cache["len"][:, first:first + n] = s.len0[:, first:first + n] + s.m_of.to(torch.int32)[:, None, None]


def _plain_attend(s, q):
    """Sequences padded to one length, a block of query rows at a time (their logits would not fit the card)."""
    c, cache = s.case, s.cache
    first, n, H, D, M = c["first"], c["count"], c["kv_heads"], c["head_dim"], c["m"]
    B, G, N = c["batch"], c["q_heads"] // c["kv_heads"], c["m"] + c["n0"]
    total = s.m_of + s.n0_of
    live = (torch.arange(N, device="cuda") < total[:, None])[:, None, None, :, None]  # [B][1][1][N][1]
    if c["paged"]:
        table = cache["page_table"][:, first:first + n].long()[..., :-(-N // PAGE)].clamp(min=0)
        k, v = (cache[x][table].flatten(3, 4)[:, :, :, :N].float() for x in ("k_pool", "v_pool"))
    else:
        k, v = (cache[x][:, first:first + n, :, :N].float() for x in ("k", "v"))  # [B][layers][H][N][D]
    k, v = torch.where(live, k, 0.0), torch.where(live, v, 0.0)
    rows = max(1, min(M, 2 ** 31 // (B * n * H * G * N)))
    for i0 in range(0, M, rows):
        i = torch.arange(i0, min(M, i0 + rows), device="cuda")
        keys = min(N, c["n0"] + int(i0) + rows)  # none of these rows sees more
        at = (s.off[:-1, None] + i).clamp(max=s.T - 1)  # [B][rows]
        x = q[:, at].float().unflatten(3, (H, G)).permute(1, 0, 3, 4, 2, 5)  # [B][layers][H][G][rows][D]
        x = x.flatten(3, 4) @ k[..., :keys, :].transpose(-1, -2)  # [B][layers][H][G rows][keys]
        x = x.unflatten(3, (G, -1)).mul_(1.0 / math.sqrt(D))
        seen = torch.arange(keys, device="cuda") <= (s.n0_of[:, None] + i)[..., None]  # [B][rows][keys]
        x.masked_fill_(~seen[:, None, None, None], -math.inf)
        x = x.sub_(x.amax(-1, keepdim=True)).exp_()
        x.div_(x.sum(-1, keepdim=True))
        o = (x.flatten(3, 4) @ v[..., :keys, :]).unflatten(3, (G, -1))  # [B][layers][H][G][rows][D]
        mine = i < s.m_of[:, None]  # [B][rows]
        s.out[:, at[mine]] = o.permute(1, 0, 4, 2, 3, 5).flatten(3, 4)[:, mine].to(s.out.dtype)


# ----------------------------------------------------------------------------- one pass

def run(s):
    c, cache = s.case, s.cache
    if own:
        import paper_2608_08569_gb300 as V
        if s.desc is None:
            s.desc = V.CacheDesc(*s.shape)
            s.rot = V.RotaryDesc(tuple(s.freqs), tuple(s.axis), c["pairing"])
        first, n, most = c["first"], c["count"], c["m"] + c["n0"]
    if s.kind == "rotary":
        if own:
            V.voxzip_rotary(s.desc, s.rot, s.positions, q=s.q, k=s.k, q_out=s.q_out, k_out=s.k_out)
        else:
            s.q_out.copy_(_plain_rotate(s, s.q))
            s.k_out.copy_(_plain_rotate(s, s.k))
        return dict(q=s.q_out, k=s.k_out)
    if s.kind == "attend":
        if own:
            V.voxzip_prompt_attention(s.desc, first, n, s.q, s.off, cache["k"], cache["v"], cache["len"], s.out,
                                      max_rows=c["m"], max_len=most)
        else:
            _plain_attend(s, s.q)
        return dict(out=s.out)
    cache["len"].copy_(s.len0)
    if c["paged"]:
        cache["page_table"].copy_(s.table0)
        cache["free_pages"].copy_(s.free0)
        cache["free_count"].copy_(s.count0)
    if not own:
        _plain_append(s)
    elif c["paged"]:
        V.voxzip_append_paged(s.desc, cache, first, n, s.k, s.v, s.new_pos, s.off, rotary=s.rot, positions=s.positions,
                              q=s.q, q_out=s.q_out, max_rows=c["m"])
    else:
        V.voxzip_append(s.desc, first, n, s.k, s.v, s.new_pos, s.off, cache["k"], cache["v"], cache["score"], cache["pos"],
                        cache["len"], rotary=s.rot, positions=s.positions, q=s.q, q_out=s.q_out, max_rows=c["m"])
    if s.kind == "append":
        return dict(q=s.q_out, k=cache["k"], v=cache["v"], score=cache["score"], pos=cache["pos"], len=cache["len"])
    if not own:
        _plain_attend(s, s.q_out)
    elif c["paged"]:
        V.voxzip_prompt_attention_paged(s.desc, cache, first, n, s.q_out, s.off, s.out, max_rows=c["m"], max_len=most)
    else:
        V.voxzip_prompt_attention(s.desc, first, n, s.q_out, s.off, cache["k"], cache["v"], cache["len"], s.out,
                                  max_rows=c["m"], max_len=most)
    if c["paged"]:  # which free page a unit gets is not part of the answer
        return dict(q=s.q_out, out=s.out, score=cache["score"], pos=cache["pos"], len=cache["len"], free=cache["free_count"])
    return dict(q=s.q_out, out=s.out, k=cache["k"], v=cache["v"], score=cache["score"], pos=cache["pos"], len=cache["len"])


# ----------------------------------------------------------------------------- what it should give

def _exact_rotate(s, x):
    x = x.double()
    y = x.clone()
    R = s.case["rotary_dim"]
    for i, (f, a) in enumerate(zip(s.freqs, s.axis)):
        th = (s.positions[a].double() * f)[None, :, None]
        lo, hi = (i, i + R // 2) if s.case["pairing"] == "halves" else (2 * i, 2 * i + 1)
        y[..., lo] = x[..., lo] * torch.cos(th) - x[..., hi] * torch.sin(th)
        y[..., hi] = x[..., lo] * torch.sin(th) + x[..., hi] * torch.cos(th)
    return y


def _exact_rows(cache, b, l, h, n, paged):
    if not paged:
        return cache["k"][b, l, h, :n], cache["v"][b, l, h, :n]
    at = cache["page_table"][b, l, h, :-(-n // PAGE)].long().clamp(min=0)
    return cache["k_pool"][at].flatten(0, 1)[:n], cache["v_pool"][at].flatten(0, 1)[:n]


def exact(case, seed):
    c = case
    w = work(c)
    if c["kind"] in ("attend", "turn") and w["flops"] > 6e12:
        return None  # over 20 seconds in 64 bits
    s = prepare(c, seed)
    if c["kind"] == "rotary":
        return dict(q=_exact_rotate(s, s.q), k=_exact_rotate(s, s.k))
    first, n, H, G, D = c["first"], c["count"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["head_dim"]
    got = dict(pos=None, len=None, free=None) if c["kind"] == "turn" and c["paged"] else dict(pos=None, len=None)
    off = [0] + [int(x) for x in np.cumsum(s.m)]
    q = s.q.double()
    if c["kind"] != "attend":
        got["q"] = q = _exact_rotate(s, s.q)
        knew, vnew = _exact_rotate(s, s.k), s.v.double()
        got["score"] = s.cache["score"].double()
        dense = not c["paged"]
        if dense:
            got["k"], got["v"] = s.cache["k"].double(), s.cache["v"].double()
        for b, (m, n0) in enumerate(zip(s.m, s.n0)):
            mine = slice(off[b], off[b + 1])
            got["score"][b, first:first + n, :, n0:n0 + m] = 0.0
            if dense:
                got["k"][b, first:first + n, :, n0:n0 + m] = knew[:, mine].transpose(1, 2)
                got["v"][b, first:first + n, :, n0:n0 + m] = vnew[:, mine].transpose(1, 2)
        if c["kind"] == "append":
            return got
        # what attends is what the cache and the packed queries hold, in their type
        q, knew = q.to(s.q.dtype).double(), knew.to(s.q.dtype).double()
    out = torch.zeros((n, s.T, H, G, D), dtype=torch.float64, device="cuda")
    for b, (m, n0) in enumerate(zip(s.m, s.n0)):
        for l in range(n):
            for h in range(H):
                if c["kind"] == "attend":
                    k, v = (x.double() for x in _exact_rows(s.cache, b, first + l, h, n0 + m, False))
                else:
                    k, v = (x.double() for x in _exact_rows(s.cache, b, first + l, h, n0, c["paged"]))
                    k = torch.cat([k, knew[l, off[b]:off[b + 1], h]])
                    v = torch.cat([v, vnew[l, off[b]:off[b + 1], h]])
                x = q[l, off[b]:off[b + 1]].unflatten(1, (H, G))[:, h]  # [m][G][D]
                for i in range(0, m, 512):
                    part = x[i:i + 512]
                    keys = n0 + min(m, i + 512)
                    z = part.flatten(0, 1) @ k[:keys].t() / math.sqrt(D)
                    last = n0 + i + torch.arange(len(part), device="cuda").repeat_interleave(G)
                    z[torch.arange(keys, device="cuda") > last[:, None]] = -math.inf
                    o = torch.softmax(z, -1) @ v[:keys]
                    out[l, off[b] + i:off[b] + i + len(part), h] = o.unflatten(0, (-1, G))
    out = out.flatten(2, 3)
    return dict(got, out=out) if c["kind"] == "turn" else dict(out=out)
