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
