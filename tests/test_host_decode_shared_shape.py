"""Which kernel a decode behind shared prompts takes (csrc/decode_shared.h), in a host build, no GPU."""
import itertools
import subprocess

import pytest

from test_gpu_decode_shared import CASES as SMALL_CASES
from test_gpu_decode_shared import SMALL
from test_gpu_decode_shared_variants import CASES, RUNS
from test_host_work_share import host_program

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "decode_shared.h"
using namespace sepattn;
int sepattn::compute_units() { return 256; }
// lines  fp32 S G Hq Hkv d own_c prefix_c rope  of a file: rows of their own, column blocks, waves, chunks, slices of a prefix and of an own cache
int main(int, char **argv) {
    FILE *f = fopen(argv[1], "r");
    sepkv_params p = {}, q = {};
    int fp32, rope;
    while (fscanf(f, "%d %d %d %d %d %d %d %d %d", &fp32, &p.S, &q.S, &p.Hq, &p.Hkv, &p.d, &p.c, &q.c, &rope) == 9) {
        p.dtype = q.dtype = fp32 ? SEPATTN_FP32 : SEPATTN_BF16;
        q.Hq = p.Hq, q.Hkv = p.Hkv, q.d = p.d;
        const SharedShape s = shared_shape(p, q, rope);
        printf("%d %d %d %d %d %d\n", s.split_rows, s.nb, s.waves, s.chunks, s.n_prefix, s.n_own);
    }
}
"""


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    d = tmp_path_factory.mktemp("shared_shape")
    run = host_program(d, PROGRAM)

    def of(calls):
        (d / "calls").write_text("\n".join(" ".join(map(str, c)) for c in calls))
        return run(d / "calls")

    return of


def kernel(call, shape):
    """d, positions and what chooses among the kernels of a type"""
    return (call[0], call[5], call[8], *(shape[:1] if call[0] else shape[:3]))


def call_of(case, rope):
    dtype, S, Hq, Hkv, d, pc, n, _ = case[:8]
    return (int(dtype == "fp32"), S, len(n), Hq, Hkv, d, SMALL[3], pc, int(rope))


def test_the_cases_take_the_kernels_they_are_for(shapes):
    calls = [call_of(CASES[name], rope) for name, rope in RUNS]
    got = [tuple(s[:1] if c[0] else s[:3]) for c, s in zip(calls, shapes(calls))]
    assert got == [CASES[name][8 + rope] for name, rope in RUNS]
    # prompts of several slices, the last of them without an entry
    for (name, rope), shape in zip(RUNS, shapes(calls)):
        pc, entries = CASES[name][5], CASES[name][6][0]
        blocks = -(-pc // 32)
        per = -(-blocks // shape[4]) * 32
        assert shape[4] >= 2 and entries > per and entries % 32 != 0
        if pc > 1000:
            assert entries <= per * (shape[4] - 1)


def test_no_call_takes_another_kernel(shapes):
    calls = [call_of(CASES[name], rope) for name, rope in RUNS]
    tested = {kernel(c, s) for c, s in zip(calls, shapes(calls))}
    heads = [(8, 8), (32, 8), (28, 4), (8, 1), (64, 8), (71, 1)]
    sizes = [1, 2, 40, 300, 1000, 2500, 5000, 9000, 20000, 33333, 65536, 1 << 20]
    sweep = [(fp32, S, G, *h, d, c, pc, rope) for fp32, S, G, h, d, c, pc, rope in itertools.product(
        (0, 1), (1, 2, 5, 8, 17, 24, 33, 48, 100, 400), (1, 2, 5, 64), heads, (64, 128), (40, 800), sizes, (0, 1))]
    got = shapes(sweep)
    assert {kernel(c, s) for c, s in zip(sweep, got)} == tested
    for c, s in zip(sweep, got):
        gq = c[3] // c[4]
        rows = 64 * (1 if c[0] else s[1]) if s[0] else 16 * (1 if c[0] else s[1])
        # chunks enough for any division of the rows among the prefixes, slices that the chip and the caches can have
        assert s[3] >= -(-c[1] * gq // rows) and (c[2] == 1 or s[3] >= c[1] * gq // rows + min(c[1], c[2]))
        assert 1 <= s[4] <= 64 and 1 <= s[5] <= 64 and s[4] <= max(1, -(-c[7] // 32)) and s[5] <= max(1, -(-c[6] // 32))


def test_small_cases_stay_in_their_rows(shapes):
    """The cases of up to 32 rows have them in every wave, the others in waves of their own."""
    for name in ("two", "eight", "thirteen", "wide"):
        S, Hq, Hkv, d, own, prompts = SMALL_CASES[name][:6]
        (shape,) = shapes([(0, S, 1, Hq, Hkv, d, own[3], prompts[3], 0)])
        assert shape[0] == (S * Hq // Hkv > 32)
