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


def _parts_limit(D, dtype):
    """Pieces that are at work at once (bf16 one to an SM of 256 rows, fp32 three of 128), a row of fp32 sums and two
    statistics each; on as many SMs as a device of this kind may have."""
    rows = 256 if dtype is torch.bfloat16 else 3 * 128
    return 160 * rows * (D * 4 + 8) + 256


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
def test_no_hint_makes_the_workspace_large(V, dtype, D):
    """Padded rows with a right hint of the rows, and hints that are too low: a few tens of MB at most."""
    limit = _parts_limit(D, dtype)
    for Hq, H, L in ((32, 4, 1), (2, 1, 1), (5, 1, 1), (16, 16, 4), (32, 4, 48)):
        for B in (1, 4, 77):
            desc = V.CacheDesc(B, L, Hq, H, D, 46080, dtype)
            for T in (1, 57, 228, 4096, 8012, 46024, 10 ** 6):
                for max_rows in (0, 1, 2, 57, 300, 4000, T):
                    for max_len in (0, 64, 2358):
                        size = V.voxzip_prompt_attention_workspace_size(desc, L, T, max_rows, max_len)
                        assert size <= limit, (Hq, H, L, B, T, max_rows, max_len, size)


def test_the_workspace_does_not_grow_with_rows_of_no_sequence(V):
    desc = V.CacheDesc(4, 1, 32, 4, 128, 2368, torch.bfloat16)
    sizes = [V.voxzip_prompt_attention_workspace_size(desc, 1, T, 57, 2358) for T in (228, 4096, 46024)]
    assert sizes[0] > 0 and sizes[0] == sizes[1] == sizes[2]


def test_launches_are_sized_by_the_device():
    """As the row kernels' launches are: no number of SMs stands in the sources."""
    for f in ("rotary.cu", "prompt_attn.cu", "prompt_attn_mma.cu"):
        assert not re.search(r"\b1(48|52)\b(?! SM)", re.sub(r"//.*", "", SOURCES[f])), f


def test_no_pointer_in_front_of_an_array():
    """A unit's rows are found by its own length, not by an array that would begin at its first kv-head."""
    assert not re.search(r"\bstart - ", SOURCES["rotary.cu"])


def test_short_appends_of_many_units_are_planned_first(V):
    """One launch where all units' clusters start at once, a plan (4 bytes a unit) where they would wait for places."""
    desc = V.CacheDesc(4, 48, 32, 4, 128, 256, torch.bfloat16)
    size = lambda layers, rows: V.voxzip_append_workspace_size(desc, layers, 4 * rows, rows)  # noqa: E731
    assert size(1, 57) == 0 == size(1, 64) == size(12, 8) == size(2, 64)
    assert size(48, 57) == 48 * 16 * 4 == size(48, 64) and size(4, 64) == 256 == size(1, 65)
