"""A turn's prompt without a GPU: what the entry points refuse, how the rotation's tables are made, how launches are
planned."""
import copy
import ctypes
import math
import pickle

import pytest
import torch

P = ctypes.c_void_p(256)  # non-null and aligned; never dereferenced on these paths


@pytest.fixture(scope="module")
def V():
    from paper_2608_08569_gb300 import build as B
    B.build_library()
    import paper_2608_08569_gb300 as V
    V.lib()
    return V


@pytest.fixture(scope="module")
def N(V):
    return V._native


def _desc(N, **kw):
    base = dict(batch=2, layers=3, q_heads=8, kv_heads=2, head_dim=128, capacity=128, dtype=1)
    base.update(kw)
    return N._Desc(*[base[k] for k in ("batch", "layers", "q_heads", "kv_heads", "head_dim", "capacity", "dtype")])


def _rows(N, data=256, token=12 * 128, layer=0):
    return N._Rows(data, token, layer)


def _rot(N, **kw):
    n = kw.pop("n", 64)
    freq = (ctypes.c_double * n)(*kw.pop("freq", [1.0] * n))
    axis = kw.pop("axis", None)
    base = dict(rotary_dim=2 * n, axes=1, pairing=0)
    base.update(kw)
    r = N._RotaryDesc(base["rotary_dim"], base["axes"], base["pairing"], freq,
                      (ctypes.c_uint8 * n)(*axis) if axis is not None else None)
    r.keep = freq
    return r


def _append(N, L, desc=None, **o):
    d = desc if desc is not None else _desc(N)
    rows = {n: o.get(n, _rows(N)) for n in "qkv"}
    ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    g = o.get
    return L.voxzip_append(ref(d), ref(g("rotary", _rot(N))), g("begin", 0), g("count", 1), g("tokens", 500),
                           ref(rows["q"]), ref(rows["k"]), ref(rows["v"]), g("positions", P), g("new_pos", P),
                           g("off", P), 0, g("kc", P), g("vc", P), g("score", P), g("pos", P), g("len", P),
                           g("q_out", P), g("ws", P), g("bytes", 1 << 20), None)


def test_append_is_validated(N):
    L = N.lib()
    bad = [dict(begin=3), dict(count=0), dict(begin=2, count=2), dict(tokens=-1), dict(k=None), dict(v=None), dict(off=None),
           dict(len=None), dict(kc=None), dict(vc=None), dict(kc=ctypes.c_void_p(264)), dict(q_out=None),
           dict(q_out=ctypes.c_void_p(264)), dict(ws=None), dict(ws=ctypes.c_void_p(16)), dict(bytes=15), dict(positions=None),
           dict(new_pos=None), dict(k=_rows(N, data=264)), dict(k=_rows(N, token=255)), dict(k=_rows(N, token=260)),
           dict(q=_rows(N, token=8 * 128 - 8)), dict(v=_rows(N, data=0)), dict(count=2), dict(count=2, k=_rows(N, layer=12)),
           dict(rotary=_rot(N, rotary_dim=144)), dict(rotary=_rot(N, n=4)), dict(rotary=_rot(N, n=12)), dict(rotary=_rot(N, axes=0)),
           dict(rotary=_rot(N, pairing=2)), dict(rotary=_rot(N, axis=[1] * 64)), dict(rotary=_rot(N, freq=[math.nan] * 64)),
           dict(rotary=_rot(N, freq=[math.inf] * 64)), dict(rotary=_rot(N, freq=[2e6] * 64))]
    for o in bad:
        assert _append(N, L, **o) == 1, o
    for kw in (dict(head_dim=96), dict(q_heads=7), dict(batch=0), dict(dtype=2), dict(capacity=0)):
        assert _append(N, L, desc=_desc(N, **kw)) == 1, kw
        assert L.voxzip_append_workspace_size(ctypes.byref(_desc(N, **kw)), 1, 500, 0) == 0
    assert _append(N, L, tokens=0, k=None, v=None) == 0  # no rows: nothing to do
    size = lambda *a: L.voxzip_append_workspace_size(ctypes.byref(_desc(N)), *a)  # noqa: E731
    assert size(4, 500, 0) == 0 and size(3, 500, 0) == 256 == size(3, 500, 499)
    assert size(3, 500, 60) == 0 == size(3, 5, 0)  # short sequences need none
    # more tokens of layers than a grid has blocks for
    assert _append(N, L, desc=_desc(N, layers=2 ** 23), count=2 ** 23, bytes=1 << 40, **{n: _rows(N, layer=8) for n in "qkv"}) == 2


def test_rotary_is_validated(N):
    L, ref = N.lib(), ctypes.byref
    d, r, x = _desc(N), _rot(N), _rows(N)
    call = lambda d=d, r=r, L_=1, T=3, q=x, k=x, pos=P, qo=P, ko=P: L.voxzip_rotary(  # noqa: E731
        ref(d), r and ref(r), L_, T, q and ref(q), k and ref(k), pos, qo, ko, None)
    for kw in (dict(r=None), dict(L_=0), dict(T=-1), dict(q=None, k=None), dict(pos=None), dict(qo=None), dict(ko=None),
               dict(qo=ctypes.c_void_p(8)), dict(q=_rows(N, token=8)), dict(L_=2, k=_rows(N, layer=4)), dict(d=_desc(N, head_dim=64))):
        assert call(**kw) == 1, kw
    assert call(T=0, pos=None) == 0
    assert call(L_=2 ** 16, T=2 ** 16, q=_rows(N, layer=8), k=None) == 2


def test_attention_is_validated(N):
    L, ref = N.lib(), ctypes.byref
    x = _rows(N)
    call = lambda d=None, begin=0, count=1, T=5000, q=x, off=P, k=P, v=P, len=P, scale=0.0, out=P, ws=P, by=1 << 40: (  # noqa: E731
        L.voxzip_prompt_attention(ref(d if d is not None else _desc(N, capacity=4096)), begin, count, T, q and ref(q), off, k, v, len, scale, 0, 0,
                                  out, ws, by, None))
    for kw in (dict(begin=-1), dict(count=4), dict(T=-1), dict(q=None), dict(off=None), dict(k=None), dict(v=None), dict(len=None),
               dict(out=None), dict(out=ctypes.c_void_p(8)), dict(k=ctypes.c_void_p(8)), dict(scale=math.nan), dict(scale=math.inf),
               dict(q=_rows(N, token=100)), dict(T=9, ws=None), dict(T=9, by=0), dict(T=9, ws=ctypes.c_void_p(16))):
        assert call(**kw) == 1, kw
    assert call(T=0, q=None, out=None) == 0
    assert call(d=_desc(N, q_heads=34), q=_rows(N, token=34 * 128)) == 2  # a group of 17
    assert L.voxzip_prompt_attention_workspace_size(ref(_desc(N, q_heads=34)), 1, 5, 0, 0) == 0


def test_paged_forms_are_validated(N):
    L, ref = N.lib(), ctypes.byref
    make = lambda **kw: N._Paged(*[dict(dict(k_pool=256, v_pool=256, page_table=256, free_pages=256, free_count=256, pages=64,  # noqa: E731
                                            max_pages=2), **kw)[k] for k in ("k_pool", "v_pool", "page_table", "free_pages",
                                                                             "free_count", "pages", "max_pages")])
    d, x, r = _desc(N), _rows(N), _rot(N)
    for kw in (dict(max_pages=1), dict(pages=11), dict(k_pool=0), dict(v_pool=264), dict(page_table=0), dict(free_count=0)):
        pc = make(**kw)
        assert L.voxzip_append_paged(ref(d), ref(pc), ref(r), 0, 1, 5, None, ref(x), ref(x), P, P, P, 0, P, P, P, None, P, 4096,
                                     None) == 1, kw
        assert L.voxzip_prompt_attention_paged(ref(d), ref(pc), 0, 1, 5, ref(x), P, P, 0.0, 0, 0, P, P, 1 << 30, None) == 1, kw


def test_the_plan_fits_its_workspace(V):
    """Launches that fill the GPU need none; others a part of the keys each, a tile of them or more."""
    for dtype in (torch.bfloat16, torch.float32):
        d = V.CacheDesc(4, 2, 32, 4, 128, 46080, dtype)
        size = V.voxzip_prompt_attention_workspace_size
        assert size(d, 1, 46024) == 0
        small = size(d, 1, 1, 1, 46080)
        assert small > 0 and small % 256 == 0
        per_split = 32 * (128 * 4 + 8)
        assert 2 <= small // per_split <= 46080 // 64
        assert size(d, 1, 1, 1, 64) == 0  # too few keys to share out
        assert size(d, 1, 1, 1, 0) == small == size(d, 1, 1, 0, 0) == size(d, 1, 1, 7, 10 ** 9)


def test_rotary_desc(V):
    r = V.RotaryDesc.make(128, 1e6, (24, 20, 20), in_turns=True)
    assert r.rotary_dim == 128 and r.num_axes == 3
    assert [r.axes.count(a) for a in range(3)] == [24, 20, 20] and r.axes[:7] == (0, 1, 2, 0, 1, 2, 0) and r.axes[60:] == (0,) * 4
    assert V.RotaryDesc.make(64, sections=(16, 8, 8)).axes == (0,) * 16 + (1,) * 8 + (2,) * 8
    assert V.RotaryDesc.make(64).axes == () and V.RotaryDesc.make(64).num_axes == 1
    for kw in (dict(sections=(30,)), dict(sections=(40, -8)), dict(sections=(1, 31), in_turns=True)):
        with pytest.raises(ValueError):
            V.RotaryDesc.make(64, **kw)
    for bad in (V.RotaryDesc((1.0,) * 32, (), "thirds"), V.RotaryDesc((1.0,) * 32, (0,) * 31), V.RotaryDesc((1.0,) * 32, (-1,) * 32)):
        with pytest.raises(ValueError):
            bad._c
    r._c
    for same in (pickle.loads(pickle.dumps(r)), copy.deepcopy(r)):
        assert same == r and hash(same) == hash(r)


def test_binding_rejects_what_the_kernels_cannot_address(V):
    N = V._native
    d = V.CacheDesc(1, 1, 4, 2, 64, 64)
    t = torch.zeros(1, 3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA device"):
        N._rows(t, "k", d, 2)
    with pytest.raises(ValueError, match="dtype"):
        N._rows(t.float(), "k", d, 2)
    with pytest.raises(TypeError):
        N._rows([1], "k", d, 2)
    with pytest.raises(ValueError, match="needs q or k"):
        V.voxzip_rotary(d, V.RotaryDesc.make(64), torch.zeros(3, dtype=torch.int32))


def test_every_wait_of_the_tensor_core_kernel_is_bounded():
    """Barriers in shared memory are waited for by wait() and wait_warp() alone, which give up; there is no barrier of some
    warps that another's give-up would leave waiting."""
    import os
    from paper_2608_08569_gb300 import build as B
    s = open(os.path.join(B.CSRC, "prompt_attn_mma.cu")).read()
    assert s.count("mbar_try_wait(") == 1 and "for (uint32_t i = 0; i < kPolls; ++i)" in s
    assert "bar.sync" not in s and s.count("__syncthreads()") == 2
