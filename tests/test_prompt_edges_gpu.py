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
