"""Performance cases of the cache held in 4 bits: packing it, decoding over it and evicting from it.

A cache of bf16 or fp32 K/V rows (what stage 1 leaves) is packed into 4 bits per element; each
generated token then appends a packed row, attends over the packed rows and updates their decayed
attention scores, and every 32 tokens the rows of least score leave. What is held in 4 bits comes
back as the values it stands for, through the call that reads a packed cache back.

kind "decode"  one token of every sequence, all layers in one call, then the appended rows read back
               (which rounding gave them is what a caller may want to know). Each pass first drops the
               token the last one appended, by copying the lengths back.
kind "evict"   one eviction of all layers, then the kept rows read back, as for a conversation that is
               set aside. Each pass first copies back the scores, positions and lengths.
kind "pack"    a cache packed and read back: a conversation is set aside, and returns.

The format, per row of a unit (a sequence, layer and kv-head), in groups of 32 channels:
  K      x = k * 2^-e with one exponent e per unit and channel: with a the channel's largest magnitude over
         the packed rows and m the lower median of the unit's a, e is the power of two nearest to a / m
         (floor(log2(a / m * sqrt 2)) in fp32, from -16 to 16; 0 where a or m is 0 or not finite). V: x = v.
  scale  s = x_m / -8 in bf16, x_m the group's element of largest magnitude (the positive one on a tie);
         0 if it is below the smallest normal number, NaN if x_m is not finite
  code   c = rint(x * (1 / s)) from -8 to 7, in fp32 (0 if s is 0 or NaN), stored as c + 8 in a nibble;
         it stands for c * s * 2^e (K) or c * s (V)
  K rows are 4-byte words: word q * (D / 32) + j holds channels 32 j + 8 q + i, i = 0 to 7, channel i at nibble
         i / 2 + 4 (i % 2). V rows are 2-byte words: word g * (D / 32) + j holds channels 32 j + 4 g + i, i = 0
         to 3, at nibble i.

Lengths belong to the case ("layout" seeds them); values come from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # True: the framework's operators, False: their plain forms

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
THINKER = dict(layers=48, q_heads=32, kv_heads=4, head_dim=128, dtype="bf16")
SINK, RECENT = 4, 0.2


# ----------------------------------------------------------------------------- the cases

def _decode(name, *, batch, n, ragged=False, gamma=0.99, layout=0, **shape):
    return dict(name=name, kind="decode", batch=batch, n=n, ragged=ragged, gamma=gamma, layout=layout, **shape)


def _evict(name, *, batch, budget, n, compaction="ordered", history=True, layout=0, **shape):
    return dict(name=name, kind="evict", batch=batch, budget=budget, n=n, compaction=compaction, history=history,
                layout=layout, **shape)


def _pack(name, *, batch, n, ragged=False, layout=0, **shape):
    return dict(name=name, kind="pack", batch=batch, n=n, ragged=ragged, layout=layout, **shape)


def listed():
    return [
        # The smallest call: one fp32 layer of one kv-head, 149 cached rows.
        _decode("decode_tiny_f32", batch=1, n=149, gamma=0.95, layers=1, q_heads=2, kv_heads=1, head_dim=64,
                dtype="f32"),
        # A token of a 10-min request at a 20x budget, fp32 activations, then bf16.
        _decode("decode_f32_10min", batch=1, n=416, **dict(THINKER, dtype="f32")),
        _decode("decode_10min", batch=1, n=416, **THINKER),
        # A token of 32 ragged sequences of 2-8 min at 4x.
        _decode("decode_batch32", batch=32, n=1564, ragged=True, gamma=0.98, layout=4, **THINKER),
        # A token of four 60-min requests at 20x, and at 4x (the largest).
        _decode("decode_60min", batch=4, n=2317, gamma=0.995, **THINKER),
        _decode("decode_60min_4x", batch=4, n=11522, gamma=0.995, **THINKER),
        # Multi-head attention (a group of one query head) of D = 64, an odd length.
        _decode("decode_mha64", batch=3, n=1237, ragged=True, layout=7, layers=24, q_heads=4, kv_heads=4, head_dim=64,
                dtype="bf16"),
        # The eviction after 32 tokens: a 30-s clip at 4x, four 60-min requests at 20x, the same with hole filling.
        _evict("evict_30s", batch=1, budget=157, n=189, **THINKER),
        _evict("evict_60min", batch=4, budget=2301, n=2333, **THINKER),
        _evict("evict_fill_60min", batch=4, budget=2301, n=2333, compaction="fill", **THINKER),
        # Packing what stage 1 left of a 30-s clip, and of four 60-min prompts cut to 20x.
        _pack("pack_30s", batch=1, n=157, **THINKER),
        _pack("pack_60min", batch=4, n=2301, **THINKER),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_shape(rng):
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if rng.random() < 0.6:
        return dict(THINKER, dtype=dtype)
    heads, kv, dim = rng.choice([(16, 1, 64), (12, 3, 128), (4, 4, 128), (2, 1, 64), (32, 8, 128), (4, 4, 64)])
    return dict(layers=_log(rng, 1, 48), q_heads=heads, kv_heads=kv, head_dim=dim, dtype=dtype)


def _draw_once(rng):
    kind = rng.choice(["decode", "decode", "decode", "evict", "evict", "pack"])
    batch, audio, text = _log(rng, 1, 32), _log(rng, 375, 45000), _log(rng, 32, 1024)
    rows = max(16, (audio + text) // rng.choice([4, 20]))
    common = dict(batch=batch, layout=rng.randrange(1 << 20), **_draw_shape(rng))
    ragged = batch > 1 and rng.random() < 0.5
    if kind == "decode":
        return _decode("", n=rows + rng.randrange(32), ragged=ragged, gamma=rng.choice([0.95, 0.98, 0.99, 0.995, 1.0]),
                       **common)
    if kind == "evict":
        return _evict("", budget=rows, n=rows + rng.choice([16, 32, 32, 32, 3 * rows]),
                      compaction=rng.choice(["ordered", "ordered", "fill"]), history=rng.random() < 0.85, **common)
    return _pack("", n=rows, ragged=ragged, **common)


def draw(rng):
    most = {k: max(work(c)["bytes"] for c in listed() if c["kind"] == k) for k in ("decode", "evict", "pack")}
    while True:
        c = _draw_once(rng)
        if work(c)["bytes"] <= most[c["kind"]]:
            c.pop("name")
            return c


# ----------------------------------------------------------------------------- sizes of a case

def _lens(c):
    """Rows of every sequence before the call."""
    if not c.get("ragged"):
        return [c["n"]] * c["batch"]
    lens = np.random.default_rng(c["layout"]).integers(c["n"] // 4, c["n"] + 1, c["batch"])
    lens[0] = c["n"]
    return [int(x) for x in lens]


def _capacity(c):
    return -(-(c["n"] + 32) // 8) * 8


def work(case):
    c = case
    D, G, units, e = c["head_dim"], c["q_heads"] // c["kv_heads"], c["layers"] * c["kv_heads"], 2 if c["dtype"] == "bf16" else 4
    packed, plain = D + D // 8, 2 * D * e  # a row's K and V
    if c["kind"] == "decode":
        rows = sum(_lens(c))
        # q, out, k_new, v_new, the channel exponents, the packed row written, read back as values, its position
        fixed = 2 * G * D * e + plain + D + packed + plain + 4
        return {"bytes": units * (rows * (packed + 8) + c["batch"] * fixed), "flops": units * rows * 4 * G * D}
    if c["kind"] == "pack":
        rows = sum(_lens(c))
        return {"bytes": units * rows * (2 * plain + packed), "flops": units * rows * 4 * D}
    m = int(RECENT * c["budget"])
    gone, hist = c["n"] - c["budget"], c["n"] - m - SINK
    first = SINK if not c["history"] else SINK + (hist - gone) // (gone + 1)  # the first row to leave, as expected
    moved = min(gone, c["budget"]) if c["compaction"] == "fill" else max(0, c["budget"] - first)
    by = 4 * c["n"] + c["budget"] * (packed + plain) + moved * (packed + 16)
    return {"bytes": units * c["batch"] * by, "flops": units * c["batch"] * 2 * c["budget"] * D}


# ----------------------------------------------------------------------------- the plain forms

def _group_scales(x):
    """[..., D] fp32 to the scales [..., D / 32] and, per element, codes from -8 to 7 as fp32."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    hi, lo = g.amax(-1), g.amin(-1)  # both NaN if one element is
    top = torch.where(hi >= -lo, hi, lo)
    s = (top * -0.125).to(torch.bfloat16).float()
    s = torch.where(s.abs() < 2.0 ** -126, torch.zeros_like(s), s)
    s = torch.where(torch.isfinite(hi) & torch.isfinite(lo), s, torch.full_like(s, math.nan))
    code = torch.round(g * (1.0 / s)[..., None]).clamp(-8, 7)
    code = torch.where(((s == 0) | torch.isnan(s))[..., None], torch.zeros_like(code), code)
    return s.to(torch.bfloat16), code.reshape(x.shape)


def _channel_exponents(top):
    """[..., D] largest magnitudes to exponents, int8."""
    mid = top.view(torch.int32).sort(-1).values[..., (top.shape[-1] - 1) // 2].view(torch.float32)[..., None]
    r = top / mid * np.float32(math.sqrt(2.0)).item()
    e = ((r.view(torch.int32) >> 23) - 127).clamp(-16, 16)
    known = (top > 0) & torch.isfinite(top) & (mid > 0) & torch.isfinite(mid)
    return torch.where(known, e, torch.zeros_like(e)).to(torch.int8)


def _power(e, sign=1):
    return ((sign * e.int() + 127) << 23).view(torch.float32)  # 2^e


def _pack_k(code):
    """Codes [..., D] to bytes [..., D / 2]."""
    J = code.shape[-1] // 32
    n = (code + 8).to(torch.int32).reshape(*code.shape[:-1], J, 4, 4, 2).transpose(-4, -3)  # [..., q, j, i / 2, i % 2]
    shift = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device=code.device, dtype=torch.int32)
    words = (n << shift).sum((-2, -1), dtype=torch.int32)  # disjoint bits: the top nibble may make it negative
    return words.reshape(*code.shape[:-1], -1).view(torch.uint8)


def _pack_v(code):
    J = code.shape[-1] // 32
    n = (code + 8).to(torch.int32).reshape(*code.shape[:-1], J, 8, 4).transpose(-3, -2)  # [..., g, j, i]
    shift = torch.tensor([0, 4, 8, 12], device=code.device, dtype=torch.int32)
    words = (n << shift).sum(-1, dtype=torch.int32)
    words = torch.where(words >= 2 ** 15, words - 2 ** 16, words).to(torch.int16)
    return words.reshape(*code.shape[:-1], -1).view(torch.uint8)


def _values(codes, scale, shifts, word):
    """The c * s that bytes [..., D / 2] and scales [..., J] stand for, [..., D] fp32; words of `word` hold len(shifts)."""
    J = scale.shape[-1]
    w = codes.view(word).reshape(*codes.shape[:-1], -1, J)
    shift = torch.tensor(shifts, device=codes.device, dtype=word)
    n = ((w[..., None] >> shift) & 15).transpose(-3, -2)  # [..., j, word, i]
    x = (n.float() - 8.0) * scale.float()[..., None, None]
    return x.reshape(*codes.shape[:-1], -1)


def _values_k(codes, scale, exp):
    return _values(codes, scale, [0, 16, 4, 20, 8, 24, 12, 28], torch.int32) * _power(exp)


def _values_v(codes, scale):
    return _values(codes, scale, [0, 4, 8, 12], torch.int16)


def _plain_decode(s):
    B, L, Hq, D = s.q.shape[1], s.q.shape[0], s.q.shape[2], s.q.shape[3]
    c, rows, n = s.cache, torch.arange(s.q.shape[1], device="cuda"), s.lens
    H = c["k_codes"].shape[2]
    knew, vnew = (x.float().transpose(0, 1) for x in (s.kn, s.vn))  # [B][L][Hkv][D]
    ks, kc = _group_scales(knew * _power(c["k_exp"], -1))
    vs, vc = _group_scales(vnew)
    for name, x in (("k_codes", _pack_k(kc)), ("k_scale", ks), ("v_codes", _pack_v(vc)), ("v_scale", vs)):
        c[name][rows, :, :, n] = x
    c["pos"][rows, :, :, n] = s.new_pos[:, None, None]
    c["len"].copy_(s.len0 + 1)
    q = s.q.float().view(L, B, H, Hq // H, D).transpose(0, 1)  # [B][L][Hkv][G][D]
    k = _values_k(c["k_codes"], c["k_scale"], c["k_exp"][:, :, :, None])
    slot = torch.arange(k.shape[3], device="cuda")
    live = (slot[None] <= n[:, None])[:, None, None]  # [B][1][1][C]
    x = (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(D))
    x = torch.where(live[..., None, :], x, torch.full_like(x, -math.inf))
    x = torch.exp(x - x.amax(-1, keepdim=True))
    p = x / x.sum(-1, keepdim=True)
    v = torch.where(live[..., None], _values_v(c["v_codes"], c["v_scale"]), 0.0)
    s.out.copy_((p @ v).reshape(B, L, Hq, D).transpose(0, 1))
    old = torch.where(slot == n[:, None], 0.0, s.gamma)[:, None, None] * c["score"]
    c["score"].copy_(torch.where(live, old + p.sum(-2), c["score"]))
    s.k_back.copy_((kc * ks.float().repeat_interleave(32, -1) * _power(c["k_exp"]))[:, :, :, None])
    s.v_back.copy_((vc * vs.float().repeat_interleave(32, -1))[:, :, :, None])


def _plain_evict(s):
    c, n, bud = s.cache, s.n, s.rows
    m = int(math.floor(float(np.float32(RECENT)) * bud)) if s.history else bud - SINK
    best = bud - SINK - m
    hist = c["score"][..., SINK:n - m]
    order = hist.sort(dim=-1, descending=True, stable=True).indices  # positions ascend with the slots
    keep = torch.ones(c["score"].shape[:3] + (n,), dtype=torch.bool, device="cuda")
    keep[..., SINK:n - m] = False
    keep.scatter_(-1, order[..., :best] + SINK, True)
    slot = torch.arange(n, device="cuda").expand(keep.shape)
    if s.compaction == "ordered":
        src = slot[keep].view(keep.shape[:3] + (bud,))
    else:
        movers = torch.where(keep[..., bud:], 0, 1).sort(dim=-1, stable=True).indices + bud
        hole = ~keep[..., :bud]
        src = torch.where(hole, movers.gather(-1, (hole.cumsum(-1) - 1).clamp(0, n - bud - 1)), slot[..., :bud])
    for name in ("k_codes", "k_scale", "v_codes", "v_scale"):
        at = src[..., None].expand(src.shape + c[name].shape[-1:])
        c[name][..., :bud, :] = c[name].gather(3, at)
    for name in ("score", "pos"):
        c[name][..., :bud] = c[name].gather(3, src)
    c["len"].fill_(bud)
    k = _values_k(c["k_codes"][..., :bud, :].contiguous(), c["k_scale"][..., :bud, :], c["k_exp"][:, :, :, None])
    s.k_back.copy_(k)
    s.v_back.copy_(_values_v(c["v_codes"][..., :bud, :].contiguous(), c["v_scale"][..., :bud, :]))


def _plain_pack(s):
    c = s.cache
    live = (torch.arange(s.k.shape[3], device="cuda") < c["len"][..., None])[..., None]  # [B][L][Hkv][C][1]
    k, v = (torch.where(live, x.float(), 0.0) for x in (s.k, s.v))
    c["k_exp"].copy_(_channel_exponents(k.abs().amax(-2)))
    ks, kc = _group_scales(k * _power(c["k_exp"], -1)[:, :, :, None])
    vs, vc = _group_scales(v)
    for name, x in (("k_codes", _pack_k(kc)), ("k_scale", ks), ("v_codes", _pack_v(vc)), ("v_scale", vs)):
        c[name].copy_(torch.where(live, x, c[name]))
    s.k_back.copy_(kc * ks.float().repeat_interleave(32, -1) * _power(c["k_exp"])[:, :, :, None])
    s.v_back.copy_(vc * vs.float().repeat_interleave(32, -1))


# ----------------------------------------------------------------------------- inputs

class State:
    """What one case has in hand; fields by kind."""


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, g):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)


def _key_scale(c, seed):
    """[L][Hkv][D]: 4 outlier channels per layer and kv-head, x16."""
    rng = np.random.default_rng(seed)
    s = np.ones((c["layers"], c["kv_heads"], c["head_dim"]), np.float32)
    for l in range(c["layers"]):
        for h in range(c["kv_heads"]):
            s[l, h, rng.choice(c["head_dim"], 4, replace=False)] = 16.0
    return torch.from_numpy(s).cuda()


def _packed_cache(c, capacity, scale, g):
    """A cache whose rows were packed from K (with its outlier channels) and V, layer by layer."""
    B, L, H, D, dt = c["batch"], c["layers"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]]
    new = lambda *shape, dtype: torch.empty((B, L, H) + shape, dtype=dtype, device="cuda")  # noqa: E731
    r = dict(k_codes=new(capacity, D // 2, dtype=torch.uint8), v_codes=new(capacity, D // 2, dtype=torch.uint8),
             k_scale=new(capacity, D // 32, dtype=torch.bfloat16), v_scale=new(capacity, D // 32, dtype=torch.bfloat16),
             k_exp=new(D, dtype=torch.int8))
    for l in range(L):
        k = _normal((B, H, capacity, D), dt, g).float() * scale[l][None, :, None]
        r["k_exp"][:, l] = e = _channel_exponents(k.abs().amax(-2))
        s, code = _group_scales(k * _power(e, -1)[:, :, None])
        r["k_scale"][:, l], r["k_codes"][:, l] = s, _pack_k(code)
        s, code = _group_scales(_normal((B, H, capacity, D), dt, g).float())
        r["v_scale"][:, l], r["v_codes"][:, l] = s, _pack_v(code)
    return r


def _state_tensors(c, capacity, g):
    """Scores, positions and lengths of one buffer, so that a pass restores them by one copy."""
    B, L, H = c["batch"], c["layers"], c["kv_heads"]
    slots, units = B * L * H * capacity, B * L * H
    live = torch.zeros(2 * slots + units, dtype=torch.int32, device="cuda")
    score = live[:slots].view(torch.float32).view(B, L, H, capacity)
    pos = live[slots:2 * slots].view(B, L, H, capacity)
    len_ = live[2 * slots:].view(B, L, H)
    score.exponential_(1.0, generator=g).mul_(c["q_heads"] / H / (max(1, c["n"]) * (1.005 - c.get("gamma", 0.99))))
    # ascending positions with gaps of 1 to 7 tokens
    pos.copy_(torch.randint(1, 8, pos.shape, generator=g, device="cuda", dtype=torch.int32).cumsum(-1, dtype=torch.int32))
    len_.copy_(torch.tensor(_lens(c), dtype=torch.int32, device="cuda")[:, None, None].expand(B, L, H))
    return live, dict(score=score, pos=pos, len=len_)


def prepare(case, seed):
    c, s, g = case, State(), _generator(seed)
    B, L, Hq, H, D, dt = c["batch"], c["layers"], c["q_heads"], c["kv_heads"], c["head_dim"], DTYPES[c["dtype"]]
    s.kind, s.case, capacity = c["kind"], c, _capacity(c)
    s.shape, s.desc = (B, L, Hq, H, D, capacity, dt), None
    s.n, scale = c["n"], _key_scale(c, seed)
    s.live, state = _state_tensors(c, capacity, g)
    s.before = s.live.clone()
    if s.kind == "pack":
        s.k = _normal((B, L, H, capacity, D), dt, g).mul_(scale[None, :, :, None, :])
        s.v = _normal((B, L, H, capacity, D), dt, g)
        new = lambda *shape, dtype: torch.zeros((B, L, H) + shape, dtype=dtype, device="cuda")  # noqa: E731
        s.cache = dict(k_codes=new(capacity, D // 2, dtype=torch.uint8), v_codes=new(capacity, D // 2, dtype=torch.uint8),
                       k_scale=new(capacity, D // 32, dtype=torch.bfloat16),
                       v_scale=new(capacity, D // 32, dtype=torch.bfloat16), k_exp=new(D, dtype=torch.int8), **state)
        s.rows = capacity
    else:
        s.cache = dict(_packed_cache(c, capacity, scale, g), **state)
        s.rows = 1 if s.kind == "decode" else c["budget"]
    s.k_back = torch.zeros((B, L, H, s.rows, D), dtype=dt, device="cuda")
    s.v_back = torch.zeros_like(s.k_back)
    if s.kind == "evict":
        s.budget = torch.full((B,), c["budget"], dtype=torch.int32, device="cuda")
        s.compaction, s.history = c["compaction"], c["history"]
    if s.kind == "decode":
        # queries: half noise, half a mix of 8 directions per layer and kv-head
        dirs = _normal((L, H, 8, D), torch.float32, g)
        mix = _normal((L, B, H, Hq // H, 8), torch.float32, g) / math.sqrt(8)
        q = 0.5 * _normal((L, B, H, Hq // H, D), torch.float32, g) + 0.5 * (mix @ dirs[:, None])
        s.q = q.reshape(L, B, Hq, D).to(dt)
        s.kn = (_normal((L, B, H, D), torch.float32, g) * scale[:, None]).to(dt)
        s.vn = _normal((L, B, H, D), dt, g)
        s.new_pos = (s.cache["pos"].amax() + 1).expand(B).contiguous()
        s.out = torch.empty_like(s.q)
        s.gamma, s.len0 = c["gamma"], s.cache["len"].clone()
        s.lens = torch.tensor(_lens(c), device="cuda")
    return s


# ----------------------------------------------------------------------------- one pass

def run(s):
    c = s.cache
    if own:
        from paper_2608_08569_gb300 import (CacheDesc, voxzip_decode_step_q4, voxzip_evict_q4, voxzip_q4_pack,
                                            voxzip_q4_unpack)
        desc, L = s.desc or CacheDesc(*s.shape), s.shape[1]
        s.desc = desc
    if s.kind == "decode":
        c["len"].copy_(s.len0)
        if own:
            voxzip_decode_step_q4(desc, c, 0, L, s.q, s.kn, s.vn, s.new_pos, s.gamma, s.out, max_len=s.n + 1)
            voxzip_q4_unpack(desc, c, 0, L, s.k_back, s.v_back, first=-1)
        else:
            _plain_decode(s)
        return dict(out=s.out, score=c["score"], pos=c["pos"], len=c["len"], k=s.k_back, v=s.v_back)
    if s.kind == "evict":
        s.live.copy_(s.before)
        if own:
            voxzip_evict_q4(desc, c, 0, L, s.budget, sink=SINK, recent_frac=RECENT, history=s.history,
                            compaction=s.compaction)
            voxzip_q4_unpack(desc, c, 0, L, s.k_back, s.v_back)
        else:
            _plain_evict(s)
        rows = lambda t: t[:, :, :, :s.rows]  # noqa: E731
        return dict(score=rows(c["score"]), pos=rows(c["pos"]), len=c["len"], k=s.k_back, v=s.v_back)
    if own:
        voxzip_q4_pack(desc, c, 0, L, s.k, s.v)
        voxzip_q4_unpack(desc, c, 0, L, s.k_back, s.v_back)
    else:
        _plain_pack(s)
    return dict(k=s.k_back, v=s.v_back, k_exp=c["k_exp"])


# ----------------------------------------------------------------------------- what it should give

def _exact_codes(x):
    """Values [..., D] that the format holds for x, in 64 bits (scales are bf16 by definition)."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    top = g.gather(-1, (g.abs() + (g > 0) * g.abs() * 1e-14).argmax(-1, keepdim=True))
    s = (top / -8).to(torch.bfloat16).double()
    return (torch.round(g / s).clamp(-8, 7) * s).reshape(x.shape)


def _exact_rows(codes, scale, per_word):
    """c * s of rows [..., D / 2], channel by channel from the format's definition, in 64 bits."""
    D, J = codes.shape[-1] * 2, scale.shape[-1]
    at = []
    for d in range(D):
        j, r = d // 32, d % 32
        nibble = (r // 8 * J + j) * 8 + r % 8 // 2 + 4 * (r % 2) if per_word == 8 else (r // 4 * J + j) * 4 + r % 4
        at.append(nibble)
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    c = both[..., torch.tensor(at, device=codes.device)].double() - 8
    return c * scale.double()[..., torch.arange(D, device=codes.device) // 32]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    B, L, Hq, H, D, C, dt = s.shape
    cache = s.cache
    if c["kind"] == "pack":
        k, v = (torch.zeros((B, L, H, C, D), dtype=torch.float64, device="cuda") for _ in range(2))
        for b, n in enumerate(_lens(c)):
            for l in range(L):
                x = s.k[b, l, :, :n].double()
                a = x.abs().amax(1)
                f = torch.exp2(torch.floor(torch.log2(a / a.sort(-1).values[:, (D - 1) // 2, None]) + 0.5).clamp(-16, 16))
                k[b, l, :, :n] = _exact_codes(x / f[:, None]) * f[:, None]
                v[b, l, :, :n] = _exact_codes(s.v[b, l, :, :n].double())
        return dict(k=k, v=v, k_exp=None)
    if c["kind"] == "evict":
        n, bud = c["n"], c["budget"]
        m = int(math.floor(float(np.float32(RECENT)) * bud)) if c["history"] else bud - SINK
        k, v = (torch.zeros((B, L, H, bud, D), dtype=torch.float64, device="cuda") for _ in range(2))
        score = torch.zeros((B, L, H, bud), dtype=torch.float64, device="cuda")
        for b in range(B):
            for l in range(L):
                for h in range(H):
                    sc = cache["score"][b, l, h, :n].double()
                    hist = torch.arange(SINK, n - m, device="cuda")
                    hist = hist.flip(0)  # of equal scores the highest position leaves first
                    gone = hist[sc[hist].argsort(stable=True)[: n - bud]]
                    src = torch.ones(n, dtype=torch.bool, device="cuda")
                    src[gone] = False
                    src = src.nonzero()[:, 0]
                    if c["compaction"] == "fill":
                        slots = torch.arange(bud, device="cuda")
                        slots[gone[gone < bud].sort().values] = src[src >= bud]
                        src = slots
                    score[b, l, h] = sc[src]
                    f = torch.exp2(cache["k_exp"][b, l, h].double())
                    k[b, l, h] = _exact_rows(cache["k_codes"][b, l, h, src], cache["k_scale"][b, l, h, src], 8) * f
                    v[b, l, h] = _exact_rows(cache["v_codes"][b, l, h, src], cache["v_scale"][b, l, h, src], 4)
        return dict(score=score, pos=None, len=None, k=k, v=v)
    out = torch.zeros((L, B, Hq, D), dtype=torch.float64, device="cuda")
    score = torch.zeros((B, L, H, C), dtype=torch.float64, device="cuda")
    kb, vb = (torch.zeros((B, L, H, 1, D), dtype=torch.float64, device="cuda") for _ in range(2))
    for b, n in enumerate(_lens(c)):
        for l in range(L):
            f = torch.exp2(cache["k_exp"][b, l].double())[:, None]
            kb[b, l] = _exact_codes(s.kn[l, b].double()[:, None] / f) * f
            vb[b, l] = _exact_codes(s.vn[l, b].double()[:, None])
            k = torch.cat([_exact_rows(cache["k_codes"][b, l, :, :n], cache["k_scale"][b, l, :, :n], 8) * f, kb[b, l]], 1)
            v = torch.cat([_exact_rows(cache["v_codes"][b, l, :, :n], cache["v_scale"][b, l, :, :n], 4), vb[b, l]], 1)
            p = torch.softmax(s.q[l, b].double().view(H, Hq // H, D) @ k.transpose(-1, -2) / math.sqrt(D), -1)
            out[l, b] = (p @ v).reshape(Hq, D)
            score[b, l] = cache["score"][b, l].double()
            score[b, l, :, :n] *= c["gamma"]
            score[b, l, :, n] = 0.0
            score[b, l, :, :n + 1] += p.sum(1)
    return dict(out=out, score=score, pos=None, len=None, k=kb, v=vb)
