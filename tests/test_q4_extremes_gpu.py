"""The cache held in 4 bits at the ends of its types: what tests of ordinary rows do not reach."""
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


def _rounded(x, dtype):
    """fp64 values rounded once to the dtype, as fp32."""
    return torch.from_numpy(np.asarray(x, np.float64)).to(F32).to(dtype).float().numpy()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_read_back_of_every_code_scale_and_exponent(V, D, dtype):
    """Scales from the least to the greatest and zero, under exponents from -16 to 16: a code of 0 is 0 whatever they
    are, and all products above the least subnormal are exact in fp32."""
    C = 64
    rng = np.random.default_rng(D)
    desc = V.CacheDesc(1, 1, 1, 1, D, C, dtype)
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(C)
    for n in ("k_codes", "v_codes"):
        qc[n].copy_(torch.from_numpy(rng.integers(0, 256, qc[n].shape).astype(np.uint8)))
    zeros = 0x88 * np.ones(D // 2, np.uint8)
    for n in ("k_codes", "v_codes"):
        qc[n][0, 0, 0, 5] = torch.from_numpy(zeros)
    exponent = np.linspace(-126, 125, C).round()[:, None] * np.ones(D // 32)
    scales = R.bf16((rng.choice([-1, 1], exponent.shape) * rng.uniform(1, 1.99, exponent.shape) * 2.0 ** exponent).astype(np.float32))
    scales[5] = 2.0 ** 125
    scales[7] = 0.0
    for n in ("k_scale", "v_scale"):
        qc[n].copy_(torch.from_numpy(scales)[None, None, None])
    e = rng.integers(-16, 17, D)
    e[:4] = -16, 16, 16, -16
    qc["k_exp"].copy_(torch.from_numpy(e)[None, None, None])
    ko, vo = (torch.empty(1, 1, 1, C, D, dtype=dtype, device="cuda") for _ in range(2))
    V.voxzip_q4_unpack(desc, qc, 0, 1, ko, vo)
    kc, vc = (R.from_bytes(_np(qc[n]), order)[0, 0, 0] for n, order in (("k_codes", R.k_nibbles(D)), ("v_codes", R.v_nibbles(D))))
    with np.errstate(over="ignore"):
        np.testing.assert_array_equal(_np(ko)[0, 0, 0], _rounded(R.values(kc, scales, e.astype(np.float64)), dtype))
        np.testing.assert_array_equal(_np(vo)[0, 0, 0], _rounded(R.values(vc, scales), dtype))
    assert not _np(ko)[0, 0, 0, [5, 7]].any()


def _hard_rows(D, dtype):
    """[16][D]: zeros, ties of a value and its negative, subnormal, least normal and huge magnitudes, in a unit whose
    channels 3 and 40 are 16 times, and 7 and 50 a 1 000th of, the others'."""
    g = torch.Generator().manual_seed(D)
    x = torch.randn(16, D, generator=g)
    x[:, [3, 40]] *= 16.0
    x[:, [7, 50]] *= 2.0 ** -10
    spread = lambda lo, hi: torch.exp2(lo + (hi - lo) * torch.rand(D, generator=g)) * torch.where(torch.rand(D, generator=g) < 0.5, -1.0, 1.0)
    x[0] = 0.0
    x[1, :32] = torch.tensor([-3.0, 3.0] * 16)
    x[2, 32:64] = torch.tensor([2.0, -2.0] * 16)
    x[3] = 1e-40
    x[4, :32], x[4, 32:64] = 3e38, -3e38
    x[5] *= 1e-37
    # scales from 2^-126 on: the largest element from 2^-123, the others far into the subnormal numbers
    for r, hi in zip(range(6, 12), (-123.5, -122.0, -120.0, -118.0, -116.0, -113.0)):
        x[r] = spread(-133.0, hi)
        x[r, ::32] = 2.0 ** hi * (-1.0 if r % 2 else 1.0)
    x[12, ::2] = -x[12, 1::2].abs()  # each magnitude with both signs
    x[12, 1::2] = x[12, 1::2].abs()
    x[13, :32] = -0.0
    return x.to(dtype)


def _assert_packed(qc, h, k, v, D):
    """Unit h of a cache holds rows k and v (fp32 values of the dtype) bit for bit."""
    e = R.channel_exponents(k)
    np.testing.assert_array_equal(_np(qc["k_exp"])[0, 0, h], e)
    for rows, codes, scale, order in ((k * np.float32(2.0) ** -e, "k_codes", "k_scale", R.k_nibbles(D)),
                                      (v, "v_codes", "v_scale", R.v_nibbles(D))):
        s, c = R.quantise(rows)
        np.testing.assert_array_equal(_np(qc[scale])[0, 0, h], s)
        np.testing.assert_array_equal(_np(qc[codes])[0, 0, h], R.to_bytes(c, order))
    return e


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_pack_of_hard_rows_in_either_type(V, D, dtype):
    k = _hard_rows(D, dtype)
    v = k.clone()
    v[14, 7], v[15, 40], v[1, 40] = math.inf, math.nan, -math.inf
    desc = V.CacheDesc(1, 1, 1, 1, D, 16, dtype)
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(16)
    V.voxzip_q4_pack(desc, qc, 0, 1, k.cuda()[None, None, None], v.cuda()[None, None, None])
    kf, vf = k.float().numpy(), v.float().numpy()
    # the huge row makes every channel of its groups as large: exponents come from the others of the unit
    e = _assert_packed(qc, 0, kf, vf, D)
    ks, kc = R.quantise(kf * np.float32(2.0) ** -e)
    vs, vc = R.quantise(vf)
    ko, vo = (torch.empty(1, 1, 1, 16, D, dtype=dtype, device="cuda") for _ in range(2))
    V.voxzip_q4_unpack(desc, qc, 0, 1, ko, vo)
    np.testing.assert_array_equal(_np(ko)[0, 0, 0], _rounded(R.values(kc, ks, e), dtype))
    np.testing.assert_array_equal(_np(vo)[0, 0, 0], _rounded(R.values(vc, vs), dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shift", [-118, -110, -40, 100])
def test_pack_of_units_of_any_magnitude(V, D, dtype, shift):
    """Whole units near the ends of the type, with channels 16 and 2^-10 times the others': the exponents are those of
    ordinary units, and rows times 2^-e go below the least normal number."""
    k = _hard_rows(D, F32)
    k[0:7] = torch.randn(7, D, generator=torch.Generator().manual_seed(shift & 255))
    k[7:12] = k[0:5] * 2.0 ** torch.linspace(-9, -1, 5)[:, None]
    k[:, [3, 40]] = k[:, [3, 40]].sign() * (k[:, [3, 40]].abs().clamp(max=3.0) * 16)
    k[:, [7, 50]] = k[:, [7, 50]].clamp(-1, 1) * 2.0 ** -10
    k = (k * 2.0 ** shift).to(dtype)
    desc = V.CacheDesc(1, 1, 1, 1, D, 16, dtype)
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(16)
    V.voxzip_q4_pack(desc, qc, 0, 1, k.cuda()[None, None, None], k.cuda()[None, None, None])
    _assert_packed(qc, 0, k.float().numpy(), k.float().numpy(), D)


def _least_rows(D, dtype):
    """[256][D]: eight ordinary rows, which give channel d the exponent d % 5 - 2, and rows whose scales are 2^-126 to
    2^-125, with elements near the halves between codes: times 2^-e they lie below the least normal number."""
    g = torch.Generator().manual_seed(D + 1)
    pattern = torch.exp2((torch.arange(D) % 5 - 2).float())
    top = torch.exp2(-123 + torch.rand(256, D // 32, 1, generator=g))
    x = top / 8 * (torch.randint(-1, 2, (256, D // 32, 32), generator=g) + 0.48 + 0.04 * torch.rand(256, D // 32, 32, generator=g))
    x[:, :, :1] = top
    x = x.reshape(256, D)
    x[:8] = torch.randn(8, D, generator=g).clamp(-1, 1)
    x[0] = 1.0
    return (x * pattern).to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_pack_of_the_least_scales(V, D, dtype):
    k = _least_rows(D, dtype)
    kf = k.float().numpy()
    e = R.channel_exponents(kf)
    assert (e == np.arange(D) % 5 - 2).all()
    if dtype == BF16:  # products rounded to bf16 would give other codes
        x = kf * np.float32(2.0) ** -e
        s = np.repeat(R.quantise(x)[0], 32, -1)
        rounded = torch.from_numpy(x).to(BF16).float().numpy()
        assert (np.rint(rounded / s) != np.rint(x / s))[s != 0].sum() > 20
    desc = V.CacheDesc(1, 1, 1, 1, D, 256, dtype)
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(256)
    V.voxzip_q4_pack(desc, qc, 0, 1, k.cuda()[None, None, None], k.cuda()[None, None, None])
    _assert_packed(qc, 0, kf, kf, D)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_pack_of_channels_without_an_exponent_in_either_type(V, D, dtype):
    k = torch.randn(1, 1, 3, 8, D, generator=torch.Generator().manual_seed(2))
    k[0, 0, 0, 3, 5], k[0, 0, 0, 4, 6] = math.inf, math.nan
    k[0, 0, 0, :, 9] *= 64
    k[0, 0, 1, 2, :D // 2 + 8] = math.nan
    k[0, 0, 2, :, :D // 2 + 8] = 0.0
    k = k.to(dtype)
    desc = V.CacheDesc(1, 1, 3, 3, D, 8, dtype)
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(8)
    V.voxzip_q4_pack(desc, qc, 0, 1, k.cuda(), k.cuda())
    for h in range(3):
        e = _assert_packed(qc, h, k[0, 0, h].float().numpy(), k[0, 0, h].float().numpy(), D)
        assert (e[9] == 6) if h == 0 else not e.any()


# ----------------------------------------------------------------------------- appended rows unlike the packed ones

@pytest.mark.parametrize("dtype", [BF16, F32])
def test_an_appended_row_unlike_the_packed_ones(V, dtype):
    """Exponents stay as the last packing set them: a channel near zero then, and ordinary now, takes its group's scale
    (up to 2^16 times its value), and the group's other channels are held in its steps. Rows are as the format says."""
    D, C = 128, 8
    k = torch.randn(1, 1, 1, C, D, generator=torch.Generator().manual_seed(4))
    k[..., 5] *= 2.0 ** -20
    k[..., 70] = 0.0
    k = k.to(dtype).cuda()
    desc = V.CacheDesc(1, 1, 1, 1, D, C, dtype)
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(C - 1)
    V.voxzip_q4_pack(desc, qc, 0, 1, k, k)
    e = _np(qc["k_exp"])[0, 0, 0].astype(np.int32)
    assert e[5] == -16 and e[70] == 0
    kn = torch.randn(1, 1, 1, D, generator=torch.Generator().manual_seed(5)).to(dtype).cuda()
    q = torch.randn(1, 1, 1, D, generator=torch.Generator().manual_seed(6)).to(dtype).cuda()
    out = torch.empty_like(q)
    V.voxzip_decode_step_q4(desc, qc, 0, 1, q, kn, kn, torch.zeros(1, dtype=torch.int32, device="cuda"), 0.9, out)
    s, c = R.quantise(_np(kn)[0, 0, 0] * np.float32(2.0) ** -e)
    np.testing.assert_array_equal(_np(qc["k_scale"])[0, 0, 0, -1], s)
    np.testing.assert_array_equal(_np(qc["k_codes"])[0, 0, 0, -1], R.to_bytes(c, R.k_nibbles(D)))
    assert c[5] in (-8, 7) and not np.delete(c[:32], 5).any() and np.abs(c[32:]).max() == 8
    assert torch.isfinite(out).all() and V.voxzip_get_status() == 0


# ----------------------------------------------------------------------------- evictions of long units

def _evict(V, *, D, n, C, budget, compaction, shuffle, ties=None, seed=0):
    rng = np.random.default_rng(seed)
    desc = V.CacheDesc(1, 1, 1, 1, D, C, BF16)
    qc = V.allocate_q4_cache(desc)
    for name in ("k_codes", "v_codes"):
        qc[name].copy_(torch.from_numpy(rng.integers(0, 256, qc[name].shape).astype(np.uint8)))
    for name in ("k_scale", "v_scale"):
        qc[name].copy_(torch.from_numpy(rng.uniform(0.1, 0.5, qc[name].shape).astype(np.float32)))
    score = rng.integers(0, ties, C) if ties else rng.exponential(1.0, C)
    qc["score"].copy_(torch.from_numpy(score.astype(np.float32))[None, None, None])
    pos = (rng.permutation(C) if shuffle else np.arange(C)) * 5
    qc["pos"].copy_(torch.from_numpy(pos.astype(np.int32))[None, None, None])
    qc["len"].fill_(n)
    before = {x: _np(t).copy() for x, t in qc.items()}
    V.voxzip_evict_q4(desc, qc, 0, 1, torch.tensor([budget], dtype=torch.int32, device="cuda"), compaction=compaction)
    assert V.voxzip_get_status() == 0
    _, src = R.kept_slots(before["score"][0, 0, 0], before["pos"][0, 0, 0], n, budget, 4, 0.2, True, compaction == "fill")
    assert int(qc["len"]) == budget
    for x in ("k_codes", "v_codes", "k_scale", "v_scale", "score", "pos"):
        assert np.array_equal(before[x][0, 0, 0][src], _np(qc[x])[0, 0, 0, :budget]), x
        assert np.array_equal(before[x][0, 0, 0][n:], _np(qc[x])[0, 0, 0, n:]), x


@pytest.mark.parametrize("compaction", ["ordered", "fill"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,C", [(20479, 20480), (20480, 20480), (20484, 20484), (40959, 40960), (40961, 40964), (46001, 46004),
                                 (12000, 47048), (20300, 47048), (3000, 47048)])
@pytest.mark.parametrize("gone", [32, 0.5])
def test_evict_units_that_shared_memory_does_or_does_not_hold(V, D, compaction, n, C, gone):
    """160 KB hold 40 960 scores, or 20 480 with their positions, in caches of up to that capacity; above it what the
    compaction's ring takes does (20 to 72 KB), and longer units are read where they lie."""
    _evict(V, D=D, n=n, C=C, budget=n - gone if gone > 1 else int(n * gone), compaction=compaction, shuffle=compaction == "fill", seed=n)


@pytest.mark.parametrize("compaction", ["ordered", "fill"])
@pytest.mark.parametrize("ties", [1, 3])
def test_evict_ties_in_long_units(V, compaction, ties):
    _evict(V, D=128, n=46001, C=47048, budget=30000, compaction=compaction, shuffle=True, ties=ties)
    _evict(V, D=64, n=20484, C=20484, budget=20000, compaction=compaction, shuffle=True, ties=ties)


# ----------------------------------------------------------------------------- the checked build

@pytest.mark.skipif(os.environ.get("VOXZIP_CHECKED", "0") not in ("", "0"), reason="this is the checked run")
def test_checked_build_passes_these_tests():
    from paper_2608_08569_gb300.build import build_library

    build_library(checked=True)
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.abspath(__file__), os.path.join(here, "test_lengths.py"), "-m", "gpu",
                        "-x", "-q", "-p", "no:cacheprovider"], cwd=ROOT, env=dict(os.environ, VOXZIP_CHECKED="1"), capture_output=True,
                       text=True, timeout=1500)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
