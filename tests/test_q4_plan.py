"""The choice of the 4-bit decode's launch, with a GPU's answers put in by hand: an error of the runtime is the call's
error and no slower kernel's, and the lengths above which that kernel runs are those that the header states."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_08569_gb300", "csrc")

PROGRAM = r"""
#include "decode_q4_plan.cuh"
#include <cstdio>
#include <cstdlib>
using namespace voxzip::q4;
template <int D, int NT, int kParts>
void run(int units, int nmax, int fails_at, int code) {  // the runtime's query number `fails_at` returns `code`
    Plan pl{9, 9, 9, 9};
    int asked = 0;
    const int err = choose_plan(
        Shape{D, kParts == 3, NT == 2}, 152, units, nmax, [](int rows, int S, int stages) { return Layout<D, NT, kParts>::bytes(rows, S, stages); },
        [&](int S, size_t bytes, int *n) {
            *n = 152 * (int)(kMaxSmem / bytes) / S;
            return ++asked == fails_at ? code : 0;
        },
        &pl);
    printf("%d %d %d %d %d %d\n", err, pl.S, pl.stages, pl.chunk_cap, pl.resident, asked);
}
int main(int argc, char **argv) {
    for (int i = 1; i + 6 < argc; i += 7) {
        const int D = atoi(argv[i]), NT = atoi(argv[i + 1]), parts = atoi(argv[i + 2]), units = atoi(argv[i + 3]), n = atoi(argv[i + 4]);
        const int at = atoi(argv[i + 5]), code = atoi(argv[i + 6]);
        if (D == 128) NT == 1 ? (parts == 1 ? run<128, 1, 1>(units, n, at, code) : run<128, 1, 3>(units, n, at, code))
                              : (parts == 1 ? run<128, 2, 1>(units, n, at, code) : run<128, 2, 3>(units, n, at, code));
        else NT == 1 ? (parts == 1 ? run<64, 1, 1>(units, n, at, code) : run<64, 1, 3>(units, n, at, code))
                     : (parts == 1 ? run<64, 2, 1>(units, n, at, code) : run<64, 2, 3>(units, n, at, code));
    }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, exe = d / "plan.cpp", d / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I" + CSRC, str(src), "-o",
                    str(exe)], check=True, capture_output=True, text=True)

    def run(*cases):
        """(error, S, stages, rows per CTA, resident clusters, queries) of (D, tiles of heads, parts, units, rows, failing
        query, its error) each."""
        out = subprocess.run([str(exe)] + [str(x) for c in cases for x in c], check=True, capture_output=True, text=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def test_a_failing_query_is_the_plans_error(plans):
    queries = plans((128, 1, 1, 768, 2317, 0, 0))[0][-1]
    assert queries > 6
    for i, got in enumerate(plans(*((128, 1, 1, 768, 2317, k + 1, 700 + k) for k in range(queries)))):
        assert got == (700 + i, 0, 0, 0, 0, i + 1)


def test_plans_hold_their_rows(plans):
    for D in (64, 128):
        for nt in (1, 2):
            for parts in (1, 3):
                cases = [(D, nt, parts, units, n, 0, 0) for units in (1, 192, 6144) for n in (1, 32, 33, 416, 2317, 40000)]
                for c, (err, S, stages, rows, resident, _) in zip(cases, plans(*cases)):
                    assert err == 0 and S >= 1 and stages in (2, 3) and resident >= 1 and rows % 32 == 0 and S * rows >= c[4]
    assert plans((128, 1, 1, 1, 2 ** 31 - 1, 0, 0))[0][:2] == (0, 0)


def test_the_header_states_the_lengths_that_a_cluster_holds(plans):
    text = open(os.path.join(ROOT, "include", "voxzip.h")).read()
    rows = re.findall(r"groups of (?:up to 8 heads|9 to 16) +D = 128: +(\d+) rows bf16, +(\d+) fp32; +D = 64: +(\d+) bf16, +(\d+) fp32", text)
    assert len(rows) == 2
    for nt, stated in zip((1, 2), rows):
        for (D, parts), n in zip(((128, 1), (128, 3), (64, 1), (64, 3)), map(int, stated)):
            at, above = plans((D, nt, parts, 4, n, 0, 0), (D, nt, parts, 4, n + 1, 0, 0))
            assert at[1] == 16 and above[:2] == (0, 0), (D, nt, parts, n)


def test_no_plan_is_kept_of_a_failure():
    s = open(os.path.join(CSRC, "decode_q4_mma.cu")).read()
    at = s.index("plan(d, units, nmax, &pl)")
    assert "return err" in s[at:s.index("cache[cache_next] =", at)]
