"""How a decode over the cache in 4 bits is cut into slices (csrc/decode_fp4.h), in a host build, no GPU: whatever the lengths on the device are, the slices
are no more than what is launched and what the workspace has records for."""
import numpy as np
import pytest

from test_host_work_share import host_program

PROGRAM = r"""
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include "decode_fp4.h"
using namespace sepattn;
int sepattn::compute_units() { return 256; }
// blocks  S Hq Hkv d c units  of a file, S numbers of blocks behind each: slices launched, slices at most of a sequence, added by the kernel, slices of
// all sequences, the least and the most of one, wrong ones.  The reciprocal of the device is off by one unit in the last place: all three are tried.
int main(int, char **argv) {
    FILE *f = fopen(argv[1], "r");
    sepkv_params p = {};
    int units;
    while (fscanf(f, "%d %d %d %d %d %d", &p.S, &p.Hq, &p.Hkv, &p.d, &p.c, &units) == 6) {
        int *nb = (int *)malloc(p.S * sizeof(int)), total = 0;
        for (int i = 0; i < p.S; ++i) if (fscanf(f, "%d", nb + i) != 1) return 1; else total += nb[i];
        const MxShape x = mx_shape(p, units);
        int most_sum = 0, least = 1 << 30, most = 0, wrong = 0;
        for (int off = -1; off <= 1 && x.plan.most > 1; ++off) {
            const float r = 1.f / (float)mx_share(x.plan, total), per = off ? nextafterf(r, off * 10.f) : r;
            int sum = 0;
            for (int i = 0; i < p.S; ++i) {
                const int n = mx_slices(x.plan, nb[i], per);
                sum += n, least = n < least ? n : least, most = n > most ? n : most;
                // none without a block, all blocks in one, as the kernel deals them
                const float rn = 1.f / (float)n, pn = off ? nextafterf(rn, off * 10.f) : rn;
                const int each = n == 1 ? nb[i] : small_quotient(nb[i], pn), more = nb[i] - each * n;
                wrong += n > 1 && (each < 1 || more < 0 || more >= n);
            }
            most_sum = sum > most_sum ? sum : most_sum;
        }
        if (x.plan.most == 1) most_sum = p.S, least = most = 1;
        printf("%d %d %d %d %d %d %d %d\n", x.slices, x.plan.most, x.add, most_sum, least, most, wrong, (int)(mx_records(p, x) / p.Hq));
        free(nb);
    }
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    d = tmp_path_factory.mktemp("mx_slices")
    run = host_program(d, PROGRAM)

    def of(calls):
        (d / "calls").write_text("\n".join(" ".join(map(str, [*head, *blocks])) for head, blocks in calls))
        return run(d / "calls")

    return of


def lengths(rng, S, full):
    kind = rng.integers(5)
    if kind == 0:
        return rng.integers(0, full + 1, S)
    if kind == 1:
        return np.full(S, full)
    if kind == 2:  # few long ones among empty and short ones
        return np.where(rng.random(S) < 0.15, full, rng.integers(0, 3, S))
    if kind == 3:
        return rng.integers(0, min(full, 40) + 1, S)
    return np.full(S, int(rng.integers(0, full + 1)))


def test_slices_fit(cut):
    rng = np.random.default_rng(0)
    calls = [((140, 9, 9, 64, 800, 256), [25] * 20 + [1] * 120), ((152, 9, 9, 64, 5888, 256), [184] * 15 + [0] * 137), ((1, 1, 1, 64, 1 << 23, 256), [1 << 18])]
    for _ in range(6000):
        S, Hkv, G = int(rng.integers(1, 600 if rng.random() < 0.3 else 40)), int(rng.choice([1, 2, 3, 4, 5, 8, 9, 12, 16, 32, 96, 300])), int(rng.choice([1, 4, 7, 8, 17, 40]))
        c, d = int(2 ** rng.uniform(0, 20)), int(rng.choice([64, 128]))
        calls.append(((S, G * Hkv, Hkv, d, c, int(rng.choice([256, 256, 304, 64]))), lengths(rng, S, (c + 31) // 32)))
    cut_at_all = 0
    for (head, blocks), (launched, limit, add, total, least, most, wrong, records) in zip(calls, cut(calls)):
        S, Hq, Hkv, d, c, _ = head
        assert total <= launched, head
        assert 1 <= least and most <= limit and limit <= (16 if add else 64) and wrong == 0, head
        assert records == (launched if limit > 1 else 0), head
        assert launched <= 65535 or launched == S
        cut_at_all += most > 1
    assert cut_at_all > 1000
