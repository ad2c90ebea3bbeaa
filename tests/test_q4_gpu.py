"""The cache held in 4 bits on the GPU against the plain reference: packed bytes, scales and exponents bit for bit,
attention and scores within bounds that follow from the arithmetic, evictions exactly.

Bounds. Logits: products of codes and q are exact, their fp32 sums of D terms in some order and the D / 32 scaled
group sums are off by at most (D + 16) 2^-24 of the sum of |q k|; the code's offset of 8 is removed from the sums,
which at most doubles the terms' magnitude twice over (codes of up to 15 instead of 7.5 on average): 4 (D + 16)
2^-24. A softmax weight is then off by at most twice that, relatively, plus 2^-20 for the exponentials and sums.
Outputs: bf16 rounds weight times scale (2^-9) and the output (2^-9), relative to sum p |v|; fp32 neither.
"""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import q4_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def V():
    import paper_2608_08569_gb300 as V
    V.lib()
    return V


def _np(t):
    return t.float().cpu().numpy() if t.dtype == BF16 else t.cpu().numpy()


def make(V, *, B=1, L=1, Hq=2, H=1, D=64, C=64, dtype=BF16, lens=(0,), seed=0, outliers=True, layers=None,
         v_scale=1.0):
    """A packed cache with rows of N(0, 1) (K with outlier channels), lengths per sequence, and NaN scales and random
    codes in every slot from the length on."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    desc = V.CacheDesc(B, L, Hq, H, D, C, dtype)
    k = rnd(B, L, H, C, D)
    if outliers:
        k[..., ::29] *= 16.0
    k, v = k.to(dtype), (rnd(B, L, H, C, D) * v_scale).to(dtype)
    qc = V.allocate_q4_cache(desc)
    for name in ("k_codes", "v_codes"):
        qc[name].random_(0, 256, generator=g)
    for name in ("k_scale", "v_scale"):
        qc[name].fill_(math.nan)
    qc["len"].copy_(torch.tensor(lens, dtype=torch.int32, device="cuda")[:, None, None].expand(B, L, H))
    qc["score"].copy_(torch.rand(B, L, H, C, generator=g, device="cuda"))
    qc["pos"].copy_(torch.arange(C, device="cuda", dtype=torch.int32) * 3)
    V.voxzip_q4_pack(desc, qc, 0, L, k, v) if layers is None else V.voxzip_q4_pack(desc, qc, *layers, k, v)
    return desc, qc, k, v, rnd


def held(qc, D):
    """(K, V) values of every slot, fp64, from the packed bytes."""
    kc, vc = (R.from_bytes(_np(qc[n]), order) for n, order in (("k_codes", R.k_nibbles(D)), ("v_codes", R.v_nibbles(D))))
    return (R.values(kc, _np(qc["k_scale"]), _np(qc["k_exp"])[..., None, :].astype(np.float64)),
            R.values(vc, _np(qc["v_scale"])))


# ----------------------------------------------------------------------------- packing

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [(0,), (1,), (2, 0, 5), (31, 64, 33), (300, 17, 1, 299)])
def test_pack_holds_the_reference_bits(V, D, dtype, lens):
    C = max(4, -(-max(lens) // 4) * 4)
    desc, qc, k, v, _ = make(V, B=len(lens), L=2, Hq=6, H=3, D=D, C=C, dtype=dtype, lens=lens, seed=D + len(lens))
    kf, vf = k.float().cpu().numpy(), v.float().cpu().numpy()
    got = {n: _np(qc[n]) for n in ("k_codes", "v_codes", "k_scale", "v_scale", "k_exp")}
    for b, n in enumerate(lens):
        for l in range(2):
            for h in range(3):
                e = R.channel_exponents(kf[b, l, h, :n])
                assert (got["k_exp"][b, l, h] == e).all()
                ks, kc = R.quantise(kf[b, l, h, :n] * (np.float32(2.0) ** -e))
                vs, vc = R.quantise(vf[b, l, h, :n])
                assert (got["k_scale"][b, l, h, :n] == ks).all() and (got["v_scale"][b, l, h, :n] == vs).all()
                assert (got["k_codes"][b, l, h, :n] == R.to_bytes(kc, R.k_nibbles(D))).all()
                assert (got["v_codes"][b, l, h, :n] == R.to_bytes(vc, R.v_nibbles(D))).all()
                assert np.isnan(got["k_scale"][b, l, h, n:]).all() and np.isnan(got["v_scale"][b, l, h, n:]).all()
    assert V.voxzip_get_status() == 0


def test_pack_of_hard_rows(V):
    """Zeros, infinities, NaN, ties between a value and its negative, subnormal and huge magnitudes."""
    D, C = 128, 16
    desc = V.CacheDesc(1, 1, 1, 1, D, C, F32)
    k = torch.randn(1, 1, 1, C, D, generator=torch.Generator().manual_seed(1))
    k[..., 0, :] = 0.0
    k[..., 1, :32] = torch.tensor([-3.0, 3.0] * 16)
    k[..., 2, 32:64] = torch.tensor([2.0, -2.0] * 16)
    k[..., 3, :] = 1e-40
    k[..., 4, :32] = 3e38
    k[..., 4, 32:64] = -3e38
    k[..., 6, :] *= 1e-37
    v = k.clone()
    v[..., 5, 7] = math.inf
    v[..., 7, 70] = math.nan
    v[..., 8, 100] = -math.inf
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(C)
    V.voxzip_q4_pack(desc, qc, 0, 1, k.cuda(), v.cuda())
    kf, vf = k.numpy()[0, 0, 0], v.numpy()[0, 0, 0]
    e = R.channel_exponents(kf)
    ks, kc = R.quantise(kf * np.float32(2.0) ** -e)
    vs, vc = R.quantise(vf)
    np.testing.assert_array_equal(_np(qc["k_exp"])[0, 0, 0], e)
    np.testing.assert_array_equal(_np(qc["k_scale"])[0, 0, 0], ks)
    np.testing.assert_array_equal(_np(qc["v_scale"])[0, 0, 0], vs)
    np.testing.assert_array_equal(_np(qc["k_codes"])[0, 0, 0], R.to_bytes(kc, R.k_nibbles(D)))
    np.testing.assert_array_equal(_np(qc["v_codes"])[0, 0, 0], R.to_bytes(vc, R.v_nibbles(D)))
    ko, vo = (torch.empty(1, 1, 1, C, D, device="cuda") for _ in range(2))
    V.voxzip_q4_unpack(desc, qc, 0, 1, ko, vo)
    np.testing.assert_array_equal(_np(vo)[0, 0, 0], R.values(vc, vs).astype(np.float32))
    np.testing.assert_array_equal(_np(ko)[0, 0, 0], R.values(kc, ks, e).astype(np.float32))


def test_pack_with_channels_that_are_not_finite(V):
    """A channel with an infinity has no exponent; so has every channel when the median one is not finite or zero."""
    D, C = 64, 8
    desc = V.CacheDesc(1, 1, 3, 3, D, C, F32)
    k = torch.randn(1, 1, 3, C, D, generator=torch.Generator().manual_seed(2))
    k[0, 0, 0, 3, 5] = math.inf
    k[0, 0, 0, 4, 6] = math.nan
    k[0, 0, 0, :, 9] *= 64
    k[0, 0, 1, 2, :40] = math.nan
    k[0, 0, 2, :, :40] = 0.0
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(C)
    V.voxzip_q4_pack(desc, qc, 0, 1, k.cuda(), k.cuda())
    for h in range(3):
        kf = k.numpy()[0, 0, h]
        e = R.channel_exponents(kf)
        np.testing.assert_array_equal(_np(qc["k_exp"])[0, 0, h], e)
        np.testing.assert_array_equal(_np(qc["k_scale"])[0, 0, h], R.quantise(kf * np.float32(2.0) ** -e)[0])
    assert _np(qc["k_exp"])[0, 0, 0, 9] == 6 and not _np(qc["k_exp"])[0, 0, 1:].any()


def test_pack_of_a_layer_range_touches_no_other(V):
    desc, qc, k, v, _ = make(V, L=3, C=16, lens=(11,), layers=(1, 1))
    assert np.isnan(_np(qc["k_scale"])[:, [0, 2]]).all() and np.isfinite(_np(qc["k_scale"])[:, 1, :, :11]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("first,rows", [(0, 1), (0, 40), (5, 7), (30, 20), (-1, 1), (-3, 2), (-40, 50), (1 << 30, 2),
                                        (-(1 << 31), 2)])
def test_unpack_windows(V, D, dtype, first, rows):
    lens = (33, 0, 40)
    desc, qc, *_ = make(V, B=3, L=3, Hq=4, H=2, D=D, C=40, dtype=dtype, lens=lens)
    ko, vo = (torch.full((3, 2, 2, rows, D), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    V.voxzip_q4_unpack(desc, qc, 1, 2, ko, vo, first=first)
    for got, want in zip((ko, vo), held(qc, D)):
        for b, n in enumerate(lens):
            for r in range(rows):
                s = first + r + (n if first < 0 else 0)
                w = want[b, 1:, :, s] if 0 <= s < n else np.zeros((2, 2, D))
                w = torch.from_numpy(w).to(dtype)  # one rounding
                assert torch.equal(got[b, :, :, r].cpu(), w)
    assert V.voxzip_get_status() == 0


# ----------------------------------------------------------------------------- decode

def check_decode(V, *, B=1, L=1, Hq=2, H=1, D=64, C=64, dtype=BF16, lens=(0,), steps=1, gamma=0.97, max_len=0, sm_scale=0.0,
                 layers=None, seed=0, q_scale=1.0, v_scale=1.0, stream=None):
    desc, qc, _, _, rnd = make(V, B=B, L=L, Hq=Hq, H=H, D=D, C=C, dtype=dtype, lens=lens, seed=seed, v_scale=v_scale)
    l0, lc = layers or (0, L)
    G, scale = Hq // H, sm_scale if sm_scale > 0 else 1 / math.sqrt(D)
    for t in range(steps):
        q = (rnd(lc, B, Hq, D) * q_scale).to(dtype)
        kn, vn = rnd(lc, B, H, D), (rnd(lc, B, H, D) * v_scale).to(dtype)
        kn[..., ::29] *= 16.0
        kn = kn.to(dtype)
        npos = torch.arange(B, device="cuda", dtype=torch.int32) + 10000 + t
        out = torch.full((lc, B, Hq, D), 99.0, dtype=dtype, device="cuda")
        before = {n: _np(x).copy() for n, x in qc.items()}
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            V.voxzip_decode_step_q4(desc, qc, l0, lc, q, kn, vn, npos, gamma, out, max_len=max_len and max_len + t,
                                    sm_scale=sm_scale)
        torch.cuda.synchronize()
        assert V.voxzip_get_status() == 0
        after = {n: _np(x) for n, x in qc.items()}
        K, Vv = held(qc, D)
        for b in range(B):
            n = int(before["len"][b, 0, 0]) if lc == L else int(before["len"][b, l0, 0])
            for l in range(L):
                for h in range(H):
                    u = (b, l, h)
                    if not l0 <= l < l0 + lc:
                        assert all(np.array_equal(before[x][u], after[x][u], equal_nan=True) for x in before)
                        continue
                    assert after["len"][u] == n + 1 and after["pos"][u][n] == 10000 + t + b
                    e = before["k_exp"][u].astype(np.int32)
                    ks, kc = R.quantise(_np(kn)[l - l0, b, h] * np.float32(2.0) ** -e)
                    vs, vc = R.quantise(_np(vn)[l - l0, b, h])
                    assert (after["k_codes"][u][n] == R.to_bytes(kc, R.k_nibbles(D))).all() and (after["k_scale"][u][n] == ks).all()
                    assert (after["v_codes"][u][n] == R.to_bytes(vc, R.v_nibbles(D))).all() and (after["v_scale"][u][n] == vs).all()
                    for x in ("k_codes", "v_codes", "k_scale", "v_scale", "pos"):  # nothing else is written
                        same = np.delete(before[x][u], n, 0), np.delete(after[x][u], n, 0)
                        assert np.array_equal(*same, equal_nan=x.endswith("scale"))
                    assert np.array_equal(before["score"][u][n + 1:], after["score"][u][n + 1:])
                    qq = _np(q)[l - l0, b, h * G:(h + 1) * G].astype(np.float64)
                    o, sc, pv, qk, mass = R.decode_unit(qq, K[u][:n + 1], Vv[u][:n + 1], before["score"][u][:n].astype(np.float64),
                                                        np.float64(np.float32(gamma)), scale)
                    rel = 2 * 4 * (D + 16) * 2.0 ** -24 * qk + 2.0 ** -20
                    rel_out = rel + (2.0 ** -8 * 1.01 if dtype == BF16 else 2.0 ** -20)
                    got = _np(out)[l - l0, b, h * G:(h + 1) * G]
                    assert (np.abs(got - o) <= rel_out * pv + 1e-30).all(), (u, n, np.abs(got - o).max(), (rel_out * pv).max())
                    got = after["score"][u][:n + 1]
                    assert (np.abs(got - sc) <= rel * mass + 2.0 ** -22 * sc).all(), (u, n, np.abs(got - sc).max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [0, 1, 2, 3, 15, 16, 17, 30, 31, 32, 33, 47, 48, 63, 64, 65, 95, 127, 128, 129, 255, 257, 511, 600])
def test_decode_lengths(V, D, dtype, n):
    check_decode(V, D=D, dtype=dtype, lens=(n,), C=-(-(n + 3) // 4) * 4, Hq=8, H=1, steps=2, seed=n)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,H", [(1, 1), (4, 4), (2, 1), (9, 3), (7, 1), (24, 3), (9, 1), (12, 1), (32, 2)])
def test_decode_groups(V, D, dtype, Hq, H):
    check_decode(V, B=2, L=2, Hq=Hq, H=H, D=D, dtype=dtype, lens=(77, 130), C=136, seed=Hq)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,L,H,lens,max_len", [
    (1, 2, 2, (2500,), 2501), (1, 1, 1, (9001,), 0), (5, 24, 4, (700, 3, 0, 699, 350), 701),
    (3, 3, 4, (1237, 310, 64), 0), (40, 6, 4, tuple(range(0, 400, 10)), 392)])
def test_decode_shapes(V, dtype, B, L, H, lens, max_len):
    check_decode(V, B=B, L=L, Hq=8 * H, H=H, D=128, dtype=dtype, lens=lens, C=-(-(max(lens) + 5) // 4) * 4, max_len=max_len,
                 steps=2 if max(lens) < 3000 else 1)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [4, 16])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_decode_of_a_very_long_cache(V, D, G, dtype):
    """More rows than the CTAs of a cluster can hold the logits of."""
    check_decode(V, Hq=G, H=1, D=D, dtype=dtype, lens=(120001,), C=120008)


def test_decode_layer_ranges_and_scale(V):
    check_decode(V, L=4, Hq=4, H=2, lens=(100,), C=104, layers=(1, 2))
    check_decode(V, L=4, Hq=4, H=2, lens=(100,), C=104, layers=(3, 1), sm_scale=0.31, gamma=1.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_decode_sharp_and_flat_softmax(V, dtype):
    check_decode(V, D=128, Hq=8, lens=(333,), C=336, q_scale=12.0, dtype=dtype)
    check_decode(V, D=128, Hq=8, lens=(333,), C=336, q_scale=1e-6, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("v_scale", [1e10, 1e-12])
def test_decode_magnitudes_of_v(V, dtype, v_scale):
    """Within the range that the header states."""
    check_decode(V, D=128, Hq=8, lens=(200,), C=204, v_scale=v_scale, dtype=dtype)


def test_decode_on_another_stream(V):
    check_decode(V, D=128, Hq=8, lens=(333,), C=336, stream=torch.cuda.Stream())


def test_decode_is_deterministic(V):
    outs = []
    for _ in range(2):
        desc, qc, _, _, rnd = make(V, B=3, L=5, Hq=16, H=2, D=128, C=600, lens=(555, 100, 599), seed=4)
        q, kn, vn = (rnd(5, 3, x, 128).to(BF16) for x in (16, 2, 2))
        out = torch.empty_like(q)
        V.voxzip_decode_step_q4(desc, qc, 0, 5, q, kn, vn, torch.zeros(3, dtype=torch.int32, device="cuda"), 0.9, out)
        outs.append((out, qc["score"]))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_decode_a_row_that_is_not_finite_shows(V):
    """A NaN scale of a live K row reaches every output of its unit, of a V row every output of its group; other units
    stay clean."""
    for which, bad in (("k_scale", slice(None)), ("v_scale", slice(32, 64))):
        desc, qc, _, _, rnd = make(V, Hq=16, H=2, D=128, C=104, lens=(100,))
        qc[which][0, 0, 1, 41, 1] = math.nan
        q, kn, vn = (rnd(1, 1, x, 128).to(BF16) for x in (16, 2, 2))
        out = torch.empty_like(q)
        V.voxzip_decode_step_q4(desc, qc, 0, 1, q, kn, vn, torch.zeros(1, dtype=torch.int32, device="cuda"), 0.9, out)
        assert torch.isfinite(out[0, 0, :8]).all() and torch.isnan(out[0, 0, 8:, bad]).all()
        if which == "v_scale":
            rest = torch.ones(128, dtype=torch.bool, device="cuda")
            rest[32:64] = False
            assert torch.isfinite(out[0, 0, 8:, rest]).all()


def test_decode_device_errors_leave_the_unit_alone(V):
    desc, qc, _, _, rnd = make(V, B=3, Hq=4, H=1, D=64, C=8, lens=(8, 7, 3))
    q, kn, vn = (rnd(1, 3, x, 64).to(BF16) for x in (4, 1, 1))
    for max_len, bits, skipped in ((0, V.DEV_CAPACITY, (0,)), (5, V.DEV_CAPACITY | V.DEV_LEN_HINT, (0, 1))):
        qc["len"].copy_(torch.tensor([8, 7, 3], dtype=torch.int32, device="cuda")[:, None, None])
        before = {n: _np(x).copy() for n, x in qc.items()}
        out = torch.full((1, 3, 4, 64), 99.0, dtype=BF16, device="cuda")
        V.voxzip_decode_step_q4(desc, qc, 0, 1, q, kn, vn, torch.zeros(3, dtype=torch.int32, device="cuda"), 0.9, out,
                                max_len=max_len)
        assert V.voxzip_get_status() & bits == bits
        for b in range(3):
            assert bool((out[0, b] == 99.0).all()) == (b in skipped)
            if b in skipped:
                assert all(np.array_equal(before[n][b], _np(x)[b], equal_nan=True) for n, x in qc.items())
            else:
                assert _np(qc["len"])[b, 0, 0] == before["len"][b, 0, 0] + 1


def test_pack_and_unpack_device_errors(V):
    desc, qc, k, v, _ = make(V, B=2, D=64, C=8, lens=(8, 7))
    qc["len"][0] = 9
    before = _np(qc["k_codes"]).copy()
    V.voxzip_q4_pack(desc, qc, 0, 1, k, v)
    assert V.voxzip_get_status() == V.DEV_CAPACITY and (_np(qc["k_codes"])[0] == before[0]).all()
    qc["len"][0] = -1
    ko = torch.full((2, 1, 1, 8, 64), 5.0, dtype=BF16, device="cuda")
    V.voxzip_q4_unpack(desc, qc, 0, 1, ko, torch.empty_like(ko))
    assert V.voxzip_get_status() == V.DEV_CAPACITY and bool((ko[0] == 5.0).all()) and not bool((ko[1] == 5.0).all())


# ----------------------------------------------------------------------------- eviction

def check_evict(V, *, lens, budget, L=2, H=2, D=128, C=None, sink=4, recent_frac=0.2, history=True, compaction="ordered", layers=None,
                ties=None, shuffle=False, seed=0, status=0):
    B, C = len(lens), C or -(-max(lens) // 4) * 4
    desc, qc, _, _, _ = make(V, B=B, L=L, Hq=H, H=H, D=D, C=C, lens=lens, seed=seed)
    rng = np.random.default_rng(seed)
    if ties:
        qc["score"].copy_(torch.from_numpy(rng.integers(0, ties, (B, L, H, C)).astype(np.float32)))
    if shuffle:
        pos = np.argsort(rng.random((B, L, H, C)), -1).astype(np.int32) * 5
        qc["pos"].copy_(torch.from_numpy(pos))
    bud = torch.tensor(budget, dtype=torch.int32, device="cuda")
    l0, lc = layers or (0, L)
    before = {n: _np(x).copy() for n, x in qc.items()}
    V.voxzip_evict_q4(desc, qc, l0, lc, bud, sink=sink, recent_frac=recent_frac, history=history, compaction=compaction)
    assert V.voxzip_get_status() == status
    after = {n: _np(x) for n, x in qc.items()}
    for b, n in enumerate(lens):
        for l in range(L):
            bb = int(bud[b, l]) if bud.dim() == 2 else int(bud[b])
            for h in range(H):
                u = (b, l, h)
                if not l0 <= l < l0 + lc or n <= bb:
                    assert all(np.array_equal(before[x][u], after[x][u], equal_nan=True) for x in before)
                    continue
                _, src = R.kept_slots(before["score"][u], before["pos"][u], n, bb, sink, recent_frac, history, compaction == "fill")
                assert after["len"][u] == bb
                for x in ("k_codes", "v_codes", "k_scale", "v_scale", "score", "pos"):
                    assert np.array_equal(before[x][u][src], after[x][u][:bb]), (u, x)
                    assert np.array_equal(before[x][u][n:], after[x][u][n:], equal_nan=x.endswith("scale"))
                assert (before["k_exp"][u] == after["k_exp"][u]).all()


@pytest.mark.parametrize("compaction", ["ordered", "fill"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,budget", [((33, 20, 17), (16, 20, 16)), ((189,), (157,)), ((600, 257, 0), (300, 256, 5)),
                                         ((1500,), (40,)), ((2333,), (2301,)), ((5000,), (1250,))])
def test_evict_keeps_the_reference_rows(V, D, compaction, lens, budget):
    check_evict(V, D=D, lens=lens, budget=budget, compaction=compaction)


@pytest.mark.parametrize("compaction", ["ordered", "fill"])
@pytest.mark.parametrize("ties", [1, 2, 7])
def test_evict_ties_go_to_the_lower_position(V, compaction, ties):
    check_evict(V, lens=(700, 129), budget=(400, 100), compaction=compaction, ties=ties, shuffle=True)


@pytest.mark.parametrize("compaction", ["ordered", "fill"])
@pytest.mark.parametrize("kw", [dict(sink=0), dict(recent_frac=0.0), dict(sink=0, recent_frac=0.0), dict(recent_frac=1.0, sink=0),
                                dict(history=False), dict(history=False, sink=0), dict(sink=80, recent_frac=0.2)])
def test_evict_policies(V, compaction, kw):
    check_evict(V, lens=(333, 120), budget=(100, 100), compaction=compaction, shuffle=compaction == "fill", **kw)


@pytest.mark.parametrize("compaction", ["ordered", "fill"])
def test_evict_to_nothing_and_to_one(V, compaction):
    check_evict(V, lens=(333, 120), budget=(0, 1), sink=0, compaction=compaction)


@pytest.mark.parametrize("compaction", ["ordered", "fill"])
def test_evict_budgets_per_layer_and_layer_ranges(V, compaction):
    check_evict(V, L=3, lens=(200, 90), budget=((100, 50, 200), (40, 90, 89)), compaction=compaction)
    check_evict(V, L=3, lens=(200, 90), budget=(100, 50), layers=(1, 1), compaction=compaction)


def test_evict_device_errors(V):
    desc, qc, *_ = make(V, B=2, Hq=1, H=1, D=64, C=64, lens=(60, 60))
    before = {n: _np(x).copy() for n, x in qc.items()}
    V.voxzip_evict_q4(desc, qc, 0, 1, torch.tensor([3, 40], dtype=torch.int32, device="cuda"), sink=4)
    assert V.voxzip_get_status() == V.DEV_BAD_BUDGET
    assert np.array_equal(before["score"][0], _np(qc["score"])[0]) and _np(qc["len"]).ravel().tolist() == [60, 40]
    qc["len"].fill_(60)
    qc["pos"].fill_(7)
    V.voxzip_evict_q4(desc, qc, 0, 1, torch.tensor([40, 40], dtype=torch.int32, device="cuda"), compaction="fill")
    assert V.voxzip_get_status() == V.DEV_BAD_POSITIONS


def test_offsets_beyond_32_bits(V):
    """Units whose rows lie more than 2^32 bytes into the codes: packing, a decode step, reading back and an eviction of
    the last one (and its neighbours' bytes unchanged)."""
    L, D, C, n = 5, 128, 17_000_000, 150
    desc = V.CacheDesc(1, L, 8, 1, D, C, BF16)
    assert (L - 1) * C * (D // 2) > 2 ** 32
    e = lambda *shape, dtype: torch.empty((1, L, 1) + shape, dtype=dtype, device="cuda")
    qc = dict(k_codes=e(C, D // 2, dtype=torch.uint8), v_codes=e(C, D // 2, dtype=torch.uint8),
              k_scale=e(C, D // 32, dtype=BF16), v_scale=e(C, D // 32, dtype=BF16), k_exp=e(D, dtype=torch.int8),
              score=e(C, dtype=F32), pos=e(C, dtype=torch.int32), len=e(dtype=torch.int32))
    k, v = e(C, D, dtype=BF16), e(C, D, dtype=BF16)
    head = lambda t, m=n + 8: t[0, L - 1, 0, :m]
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    for t in (k, v):
        head(t).normal_(generator=g)
    head(qc["score"]).uniform_(generator=g)
    head(qc["pos"]).copy_(torch.arange(n + 8, device="cuda"))
    qc["len"].fill_(n)
    guard = qc["k_codes"][0, L - 2, 0, -64:].fill_(77)
    V.voxzip_q4_pack(desc, qc, L - 1, 1, k, v)
    q, kn, vn = (torch.randn(1, 1, x, D, generator=g, device="cuda").to(BF16) for x in (8, 1, 1))
    out = torch.empty_like(q)
    old = _np(head(qc["score"])).astype(np.float64)
    V.voxzip_decode_step_q4(desc, qc, L - 1, 1, q, kn, vn, torch.tensor([n], dtype=torch.int32, device="cuda"), 0.9, out,
                            max_len=n + 1)
    m = n + 1
    ko, vo = (torch.empty(1, 1, 1, m, D, dtype=BF16, device="cuda") for _ in range(2))
    V.voxzip_q4_unpack(desc, qc, L - 1, 1, ko, vo)
    kf = _np(head(k, n))
    ex = R.channel_exponents(kf)
    ks, kc = R.quantise(np.concatenate([kf, _np(kn)[0, 0]]) * np.float32(2.0) ** -ex)
    vs, vc = R.quantise(np.concatenate([_np(head(v, n)), _np(vn)[0, 0]]))
    K, Vv = R.values(kc, ks, ex), R.values(vc, vs)
    assert torch.equal(ko[0, 0, 0].cpu(), torch.from_numpy(K).to(BF16)) and torch.equal(vo[0, 0, 0].cpu(), torch.from_numpy(Vv).to(BF16))
    o, sc, pv, qk, mass = R.decode_unit(_np(q)[0, 0].astype(np.float64), K, Vv, old[:n], np.float64(np.float32(0.9)), 1 / math.sqrt(D))
    rel = 2 * 4 * (D + 16) * 2.0 ** -24 * qk + 2.0 ** -20
    assert (np.abs(_np(out)[0, 0] - o) <= (rel + 2.0 ** -8 * 1.01) * pv).all()
    assert (np.abs(_np(head(qc["score"], m)) - sc) <= rel * mass + 2.0 ** -22 * sc).all()
    before = {x: _np(head(qc[x], m)).copy() for x in ("k_codes", "v_codes", "k_scale", "v_scale", "score", "pos")}
    V.voxzip_evict_q4(desc, qc, L - 1, 1, torch.tensor([100], dtype=torch.int32, device="cuda"))
    _, src = R.kept_slots(before["score"], before["pos"], m, 100, 4, 0.2, True, False)
    for x, b in before.items():
        assert np.array_equal(b[src], _np(head(qc[x], 100))), x
    assert qc["len"].ravel().tolist() == [n] * (L - 1) + [100]
    assert bool((guard == 77).all()) and V.voxzip_get_status() == 0


# ----------------------------------------------------------------------------- a request

@pytest.mark.parametrize("compaction", ["ordered", "fill"])
def test_session_runs_a_request(V, compaction):
    """Session(kv_bits=4) is stage 1, packing, decode steps and evictions in turn; its loop replays from a graph; stage 1
    and lengths are those of the plain session, and the first outputs are near its own (keys and values are held to
    about a tenth of their spread: cosine above 0.9)."""
    from gpu_harness import make_inputs
    from paper_2608_08569_gb300 import workloads as W
    from paper_2608_08569_gb300.session import Session

    w = W.scaled(W.CONFIGS["short"], layers=3, steps=70, name="short_l3")
    inp = make_inputs(w, "cuda:0")
    B, L, Hq, H, D = w.batch, w.layers, w.q_heads, w.kv_heads, w.head_dim
    desc = V.CacheDesc(B, L, Hq, H, D, -(-w.capacity // 4) * 4, w.dtype)
    i32 = lambda a: torch.as_tensor(np.asarray(a), dtype=torch.int32, device="cuda")
    sp = inp["spans"]
    prompt = (inp["k_pre"], inp["v_pre"], i32(w.in_len), i32([w.audio_begin] * B), i32(w.audio_len), i32(sp.off),
              i32(sp.start), i32(sp.end), i32(sp.groups))
    plain = Session(desc, w.budget, w.gamma, compaction=compaction)
    s = Session(desc, w.budget, w.gamma, compaction=compaction, kv_bits=4)
    plain.prefill(*prompt)
    s.prefill(*prompt)
    assert torch.equal(plain.cache["len"], s.cache["len"]) and torch.equal(plain.cache["pos"], s.cache["pos"])
    by_hand = V.allocate_q4_cache(desc)
    for n in ("score", "pos", "len"):
        by_hand[n].copy_(s.cache[n])
    V.voxzip_q4_pack(desc, by_hand, 0, L, plain.cache["k"], plain.cache["v"])
    outs = [torch.empty(w.steps, L, B, Hq, D, dtype=w.dtype, device="cuda") for _ in range(3)]
    n = s.n_max
    for t in range(w.steps):
        args = (inp["q"][t], inp["kn"][t], inp["vn"][t], inp["new_pos"][t])
        s.decode(*args, outs[0][t])
        V.voxzip_decode_step_q4(desc, by_hand, 0, L, *args, w.gamma, outs[1][t], max_len=n + 1)
        n += 1
        if t == 0:
            plain.decode(*args, outs[2][t])
        if (t + 1) % 32 == 0:
            s.evict()
            V.voxzip_evict_q4(desc, by_hand, 0, L, s.budget, compaction=compaction)
            n = min(n, max(w.budget))
    assert torch.equal(outs[0], outs[1])
    assert all(torch.equal(by_hand[x], s.cache[x]) for x in ("score", "pos", "len", "k_codes", "v_codes", "k_exp"))
    assert torch.nn.functional.cosine_similarity(outs[0][0].float(), outs[2][0].float(), dim=-1).min() > 0.9
    s.prefill(*prompt)
    graph = s.capture_loop(inp["q"], inp["kn"], inp["vn"], inp["new_pos"], outs[2], 32)
    graph.replay()
    assert torch.equal(outs[0], outs[2]) and torch.equal(by_hand["score"], s.cache["score"])
    assert V.voxzip_get_status() == 0


# ----------------------------------------------------------------------------- the checked build

@pytest.mark.skipif(os.environ.get("VOXZIP_CHECKED", "0") not in ("", "0"), reason="this is the checked run")
def test_checked_build_passes_these_tests():
    """The range-checked build (its kernels skip and report an access outside its buffer) on this file."""
    from paper_2608_08569_gb300.build import build_library

    build_library(checked=True)
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), "-m", "gpu", "-x", "-q", "-p",
                        "no:cacheprovider"], cwd=ROOT, env=dict(os.environ, VOXZIP_CHECKED="1"), capture_output=True,
                       text=True, timeout=1500)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
