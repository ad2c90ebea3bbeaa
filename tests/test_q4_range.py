"""The range that the header states for the 4-bit decode: inputs times powers of two, up to its ends, give the bits of
the unscaled call (K times 2^a and q times 2^-a leave every logit alone; V times 2^b scales the outputs)."""
import os
import re

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = torch.float32, torch.bfloat16
TEXT = re.sub(r"\s*\n \* ?", " ", open(os.path.join(ROOT, "include", "voxzip.h")).read())
STATED = re.search(r"\|q 2\^e\| and the scales of V must lie below 2\^(\d+) .{0,200}below 2\^-(\d+) may count as zero", TEXT)


def test_the_header_states_what_the_operands_carry():
    """q and weights times 2^84 stay below fp32's 2^128; products with codes of 2^-133 each, above 2^-126."""
    s = open(os.path.join(ROOT, "paper_2608_08569_gb300", "csrc", "decode_q4_mma.cu")).read()
    carry, uncarry = (int(re.search(rf"{n} = 0x1p(\d+)f", s).group(1)) for n in ("kCarry", "kUncarry"))
    assert STATED and uncarry == 133 - carry
    assert int(STATED.group(1)) == 128 - carry and int(STATED.group(2)) == 126 - uncarry


def _call(V, D, G, n, C, dtype, a, b, max_len):
    g = torch.Generator(device="cuda")
    g.manual_seed(D + n)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").clamp(-3.9, 3.9).to(dtype)
    desc = V.CacheDesc(2, 1, G, 1, D, C, dtype)
    qc = V.allocate_q4_cache(desc)
    qc["len"].fill_(n)
    V.voxzip_q4_pack(desc, qc, 0, 1, rnd(2, 1, 1, C, D) * 2.0 ** a, rnd(2, 1, 1, C, D) * 2.0 ** b)
    q, kn, vn = rnd(1, 2, G, D) * 2.0 ** -a, rnd(1, 2, 1, D) * 2.0 ** a, rnd(1, 2, 1, D) * 2.0 ** b
    assert float((q.float().abs() * 2.0 ** float(qc["k_exp"].max())).max()) < 2.0 ** int(STATED.group(1))
    out = torch.empty_like(q)
    V.voxzip_decode_step_q4(desc, qc, 0, 1, q, kn, vn, torch.zeros(2, dtype=torch.int32, device="cuda"), 0.9, out, max_len=max_len)
    assert V.voxzip_get_status() == 0
    return out.float().cpu().numpy(), qc["score"].cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,G,n,C,max_len", [(64, 2, 149, 152, 150), (128, 8, 600, 604, 601), (128, 16, 2000, 2004, 2001),
                                             (64, 4, 300, 120008, 0)])  # the last by the kernel of long caches
@pytest.mark.parametrize("a,b", [(-41, 45), (-41, -60), (60, 45), (60, -60)])
def test_powers_of_two_up_to_the_ends(D, G, n, C, max_len, dtype, a, b):
    """|q| up to 3.9 x 2^41 (2^43 and a channel exponent of 1 at most) down to 2^-60 and its lower bits; V's scales up to
    3.9 x 2^45 / 8 = 2^43.96, and down to 2^-61."""
    import paper_2608_08569_gb300 as V
    want, score = _call(V, D, G, n, C, dtype, 0, 0, max_len)
    got, sc = _call(V, D, G, n, C, dtype, a, b, max_len)
    assert np.array_equal(got, want * np.float32(2.0) ** b) and np.array_equal(sc, score)
