"""Lengths that no cache holds: a unit whose length lies outside [0, capacity) is skipped by every decode step and
reported, up to the type's ends (a length of INT32_MAX plus one is negative: compared after the addition, it would pass
for an empty unit's)."""
import glob
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LENGTHS = [2 ** 31 - 1, -1, -2 ** 31, 1 << 30]


def test_no_decode_kernel_adds_to_a_length_before_it_is_checked():
    found = 0
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2608_08569_gb300", "csrc", "decode*.cu"))):
        s = open(path).read()
        sums, check = [m.start() for m in re.finditer(r"\bn_old \+ 1\b", s)], s.find("n_old < 0 || n_old >= ")
        assert sums and 0 <= check < min(sums), os.path.basename(path)
        assert not re.search(r"load_relaxed\(p\.len[^;]*\), 0\) \+ 1", s), os.path.basename(path)
        found += 1
    assert found >= 4


def _inputs(desc, L):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    rnd = lambda h: torch.randn(L, desc.batch, h, desc.head_dim, generator=g, device="cuda").to(desc.dtype)
    out = torch.full((L, desc.batch, desc.q_heads, desc.head_dim), 99.0, dtype=desc.dtype, device="cuda")
    return rnd(desc.q_heads), rnd(desc.kv_heads), rnd(desc.kv_heads), torch.zeros(desc.batch, dtype=torch.int32, device="cuda"), out


def _check(V, desc, c, step, bad):
    """`step` leaves the unit of sequence 1 alone, and takes the others'."""
    c["len"].fill_(5)
    c["len"][1, 0, 0] = bad
    before = {n: t.clone() for n, t in c.items() if isinstance(t, torch.Tensor)}
    q, kn, vn, npos, out = _inputs(desc, 1)
    step(q, kn, vn, npos, out)
    assert V.voxzip_get_status() == V.DEV_CAPACITY
    assert bool((out[0, 1] == 99.0).all()) and not bool((out[0, 0] == 99.0).any()) and not bool((out[0, 2] == 99.0).any())
    assert c["len"].ravel().tolist() == [6, bad, 6]
    for n in ("score", "pos"):
        assert torch.equal(before[n][1], c[n][1])
    for n in set(before) & {"k", "v", "k_codes", "v_codes", "k_scale", "v_scale"}:
        if before[n].shape[0] == 3:
            assert torch.equal(before[n][1], c[n][1])


@pytest.mark.gpu
@pytest.mark.parametrize("bad", LENGTHS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("capacity,max_len", [(64, 0), (64, 40), (120008, 0)])  # the last by the kernel of long caches
def test_q4_decode_skips_them(dtype, capacity, max_len, bad):
    import paper_2608_08569_gb300 as V
    desc = V.CacheDesc(3, 1, 2, 1, 64, capacity, dtype)
    c = V.allocate_q4_cache(desc)
    _check(V, desc, c, lambda q, kn, vn, npos, out: V.voxzip_decode_step_q4(desc, c, 0, 1, q, kn, vn, npos, 0.9, out,
                                                                            max_len=max_len), bad)


@pytest.mark.gpu
@pytest.mark.parametrize("bad", LENGTHS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_dense_decode_skips_them(dtype, bad):
    import paper_2608_08569_gb300 as V
    desc = V.CacheDesc(3, 1, 2, 1, 64, 64, dtype)
    c = V.allocate_cache(desc)
    _check(V, desc, c, lambda q, kn, vn, npos, out: V.voxzip_decode_step(
        desc, 0, 1, q, kn, vn, npos, c["k"], c["v"], c["score"], c["pos"], c["len"], 0.9, out), bad)


@pytest.mark.gpu
@pytest.mark.parametrize("bad", LENGTHS)
def test_paged_decode_skips_them(bad):
    import paper_2608_08569_gb300 as V
    desc = V.CacheDesc(3, 1, 2, 1, 64, 128, torch.bfloat16)
    c = V.allocate_paged_cache(desc, 6)
    _check(V, desc, c, lambda q, kn, vn, npos, out: V.voxzip_decode_step_paged(desc, c, 0, 1, q, kn, vn, npos, 0.9, out),
           bad)
