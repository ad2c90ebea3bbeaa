"""A turn's prompt without a GPU, where it can go wrong: the order of its launches, the workspace of hints that do not fit."""
import re

import pytest
import torch

from test_kernel_sources import SOURCES
from test_prompt import N, V  # noqa: F401 (fixtures)


def test_no_warp_leaves_before_the_launch_in_front():
    """A launch's end implies its predecessor's only if each of its CTAs has waited for that one."""
    found = 0
    for f in ("rotary.cu", "prompt_attn.cu", "prompt_attn_mma.cu"):
        for m in re.finditer(r"__global__ void", SOURCES[f]):
            body = SOURCES[f][m.start():]
            before, wait, _ = body[body.index("{"):].partition("grid_dependency_wait()")
            assert wait and not re.search(r"\breturn\b", before), (f, SOURCES[f].count("\n", 0, m.start()) + 1)
            found += 1
    assert found >= 6
