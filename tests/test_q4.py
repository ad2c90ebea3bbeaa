"""The cache held in 4 bits without a GPU: the reference's own properties, argument checks of the C ABI (before any
CUDA call) and of the binding."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import q4_reference as R
from paper_2608_08569_gb300 import build as B

P = ctypes.c_void_p(256)  # a non-null, 256-byte aligned stand-in; never dereferenced on these paths


@pytest.fixture(scope="module")
def V():
    B.build_library()
    import paper_2608_08569_gb300 as V
    V.lib()
    return V


def _desc(V, **kw):
    base = dict(batch=1, layers=2, q_heads=8, kv_heads=2, head_dim=128, capacity=64, dtype=1)
    base.update(kw)
    return V._native._Desc(*[base[k] for k in ("batch", "layers", "q_heads", "kv_heads", "head_dim", "capacity", "dtype")])


def _q4(V, **kw):
    return V._native._Q4(*[kw.get(k, 256) for k in ("k_codes", "v_codes", "k_scale", "v_scale", "k_exp")])


def _calls(V, d, q, **o):
    """Status of each entry point with the given overrides."""
    L, r = V.lib(), ctypes.byref
    a = dict(lb=0, lc=1, p=P, len=P, gamma=0.9, scale=0.0, rows=4)
    a.update(o)
    pol = o.get("policy", V._native._EvictPolicy(4, 0.2, 1, 1, 0, 0))
    dd, qq = (None if x is None else r(x) for x in (d, q))
    return [L.voxzip_q4_pack(dd, qq, a["lb"], a["lc"], a["p"], P, a["len"], None),
            L.voxzip_q4_unpack(dd, qq, a["lb"], a["lc"], a["len"], 0, a["rows"], a["p"], P, None),
            L.voxzip_decode_step_q4(dd, qq, a["lb"], a["lc"], a["p"], P, P, P, P, P, a["len"], a["gamma"], a["scale"], 0,
                                    P, None),
            L.voxzip_evict_q4(dd, qq, a["lb"], a["lc"], P, a["p"], a["len"], P, None if pol is None else r(pol), None)]


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(head_dim=32), dict(q_heads=6, kv_heads=4), dict(batch=0),
                                dict(dtype=7), dict(capacity=0), dict(capacity=62), dict(capacity=63), dict(layers=-1)])
def test_bad_descriptors_are_einval(V, kw):
    assert _calls(V, _desc(V, **kw), _q4(V)) == [1] * 4


@pytest.mark.parametrize("kw", [dict(k_codes=0), dict(v_codes=0), dict(k_scale=0), dict(v_scale=0), dict(k_exp=0),
                                dict(k_codes=264), dict(v_codes=257), dict(k_scale=258), dict(v_scale=260), dict(k_exp=8)])
def test_bad_caches_are_einval(V, kw):
    assert _calls(V, _desc(V), _q4(V, **kw)) == [1] * 4


def test_bad_arguments_are_einval(V):
    d, q = _desc(V), _q4(V)
    assert _calls(V, None, q) == [1] * 4 and _calls(V, d, None) == [1] * 4
    assert _calls(V, d, q, lb=1, lc=2) == [1] * 4      # layers out of range
    assert _calls(V, d, q, lb=-1) == [1] * 4
    assert _calls(V, d, q, lc=0) == [1] * 4
    assert _calls(V, d, q, p=None) == [1] * 4
    assert _calls(V, d, q, len=None) == [1] * 4
    assert _calls(V, d, q, p=ctypes.c_void_p(260))[:3] == [1] * 3  # misaligned rows
    assert _calls(V, d, q, rows=0)[1] == 1
    assert V.lib().voxzip_decode_step_q4(ctypes.byref(d), ctypes.byref(q), 0, 1, P, P, P, P, ctypes.c_void_p(260), P, P, 0.9,
                                         0.0, 0, P, None) == 1  # misaligned scores
    for g in (0.0, -1.0, 1.5, float("nan")):
        assert _calls(V, d, q, gamma=g)[2] == 1
    for s in (float("nan"), float("inf")):
        assert _calls(V, d, q, scale=s)[2] == 1
    E = V._native._EvictPolicy
    for pol in (None, E(-1, 0.2, 1, 1, 0, 0), E(4, 1.5, 1, 1, 0, 0), E(4, float("nan"), 1, 1, 0, 0), E(4, 0.2, 2, 1, 0, 0),
                E(4, 0.2, 1, -1, 0, 0), E(4, 0.2, 1, 1, -1, 0), E(4, 0.2, 1, 1, 0, 2)):
        assert _calls(V, d, q, policy=pol)[3] == 1


def test_a_group_above_sixteen_is_unsupported(V):
    assert _calls(V, _desc(V, q_heads=34, kv_heads=2), _q4(V))[2] == 2


def test_the_binding_checks_tensors(V):
    desc = V.CacheDesc(1, 1, 2, 1, 64, 8)
    with pytest.raises(ValueError, match="multiple of 4"):
        V.allocate_q4_cache(V.CacheDesc(1, 1, 2, 1, 64, 10), device="cpu")
    qc = V.allocate_q4_cache(desc, device="cpu")
    assert qc["k_codes"].shape == (1, 1, 1, 8, 32) and qc["v_scale"].shape == (1, 1, 1, 8, 2)
    assert qc["k_exp"].shape == (1, 1, 1, 64) and qc["k_exp"].dtype == torch.int8
    k = torch.zeros(1, 1, 1, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        V.voxzip_q4_pack(desc, qc, 0, 1, k, k)
    with pytest.raises(ValueError, match=r"k_out must be"):
        V.voxzip_q4_unpack(desc, qc, 0, 1, k[0], k[0])
    with pytest.raises(ValueError, match="compaction|CUDA"):
        V.voxzip_evict_q4(desc, qc, 0, 1, torch.zeros(1, dtype=torch.int32), compaction="none")
    with pytest.raises(ValueError, match="dtype"):
        V.voxzip_q4_pack(desc, qc, 0, 1, k.float(), k)


def test_nibble_orders_are_permutations():
    for D in (64, 128):
        for order in (R.k_nibbles(D), R.v_nibbles(D)):
            assert sorted(order) == list(range(D))
            codes = np.arange(D) % 16 - 8
            assert (R.from_bytes(R.to_bytes(codes, order), order) == codes).all()


def test_the_reference_holds_what_the_format_promises():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((50, 128)).astype(np.float32)
    s, c = R.quantise(x)
    step = np.abs(np.repeat(s, 32, -1))
    assert (np.abs(R.values(c, s) - x) <= step * (1 + 2.0 ** -5)).all()   # a step at the clamped end
    inner = c < 7
    assert (np.abs(R.values(c, s) - x)[inner] <= 0.5 * step[inner] * (1 + 2.0 ** -5)).all()
    assert (np.abs(c).reshape(50, 4, 32).max(-1) == 8).all()              # the largest element is held at -8
    assert (R.quantise(np.zeros((1, 64), np.float32))[1] == 0).all()
    bad = x[:1].copy()
    bad[0, 40] = np.inf
    s, c = R.quantise(bad)
    assert np.isnan(s[0, 1]) and np.isfinite(s[0, [0, 2, 3]]).all() and (c[0, 32:64] == 0).all()


def test_outlier_channels_do_not_cost_the_others_their_codes():
    """Keys with 4 channels x16: without channel exponents an ordinary channel of an outlier's group keeps 1-2 codes."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((400, 128)).astype(np.float32)
    out = [3, 40, 77, 100]
    x[:, out] *= 16
    e = R.channel_exponents(x)
    assert (e[out] == 4).all() and np.abs(np.delete(e, out)).max() <= 1
    err = lambda y: np.linalg.norm(np.delete(y - x, out, 1)) / np.linalg.norm(np.delete(x, out, 1))
    s, c = R.quantise(x * np.float32(2.0) ** -e)
    s0, c0 = R.quantise(x)
    assert err(R.values(c, s, e)) < 0.12 < 0.5 < err(R.values(c0, s0))


def test_the_header_states_the_capacity_rule(V):
    text = open(os.path.join(B.ROOT, "include", "voxzip.h")).read()
    assert int(re.search(r"VOXZIP_Q4_CAPACITY_MULTIPLE (\d+)", text).group(1)) == V.Q4_CAPACITY_MULTIPLE


def test_the_session_checks_kv_bits(V):
    from paper_2608_08569_gb300.session import Session
    desc = V.CacheDesc(1, 1, 2, 1, 64, 64)
    with pytest.raises(ValueError, match="kv_bits"):
        Session(desc, (32,), 0.9, device="cpu", kv_bits=8)
    with pytest.raises(ValueError, match="paged"):
        Session(desc, (32,), 0.9, device="cpu", kv_bits=4, pages=4)
    s = Session(desc, (32,), 0.9, device="cpu", kv_bits=4)
    assert s.cache["k_codes"].shape == (1, 1, 1, 64, 32) and "k" not in s.cache
