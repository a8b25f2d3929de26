"""Every kernel that a decode behind shared prompts may take, over real prompts: which one a case takes is checked in
test_host_decode_shared_shape.py.  Needs an MI355X (256 compute units: the rule depends on their number)."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_decode_shared import SMALL, Case, slots_of, sp  # noqa: E402, F401

pytestmark = pytest.mark.gpu

# name: dtype, S, Hq, Hkv, d, capacity of the prompts, their entries, prefix of the sequences in turn; for calls without and with positions (None: not
# run) whether waves have rows of their own and, in bf16, column blocks of a wave and waves of a workgroup
CASES = {
    "64 shared 1": ("bf16", 1, 8, 1, 64, 1000, [837], [0], (0, 1, 4), (0, 1, 4)),
    "64 shared 2": ("bf16", 4, 8, 1, 64, 1000, [837], [0], (0, 2, 4), (0, 2, 4)),
    "64 own 1": ("bf16", 12, 8, 1, 64, 1000, [837], [0, 0, -1], (1, 1, 4), (1, 1, 4)),
    "64 own 2": ("bf16", 13, 16, 2, 64, 65536, [40011], [0], (1, 2, 4), (1, 2, 4)),
    "64 own 3": ("bf16", 23, 8, 1, 64, 65536, [40011], [0, 0, 0, -1], (1, 3, 4), (1, 3, 4)),
    "128 shared 1": ("bf16", 1, 8, 1, 128, 1000, [837], [0], (0, 1, 4), (0, 1, 4)),
    "128 shared 2": ("bf16", 4, 8, 1, 128, 1000, [837], [0], (0, 2, 4), (0, 2, 4)),
    "128 own 1": ("bf16", 12, 8, 1, 128, 1000, [837], [0, 0, -1], (1, 1, 4), (1, 1, 4)),
    "128 own 2": ("bf16", 48, 32, 8, 128, 2500, [2203], [0], (1, 2, 4), (1, 2, 4)),
    "128 own 2, two prompts": ("bf16", 24, 8, 1, 128, 65536, [40011, 33], [0, 0, 1], None, (1, 2, 4)),
    "128 own 3": ("bf16", 48, 32, 8, 128, 5000, [4441], [0], (1, 3, 4), None),
    "128 eight waves 2": ("bf16", 13, 16, 2, 128, 65536, [40011], [0], (1, 2, 8), None),          # slices of 46 blocks, the last one of nine: an odd
    "128 eight waves 3": ("bf16", 23, 8, 1, 128, 65536, [40011], [0, 0, 0, -1], (1, 3, 8), None),  # number for two groups of waves
    "64 fp32 shared": ("fp32", 2, 8, 1, 64, 1000, [837], [0], (0,), (0,)),
    "64 fp32 own": ("fp32", 12, 8, 1, 64, 1000, [837], [0, 0, -1], (1,), (1,)),
    "128 fp32 shared": ("fp32", 2, 8, 1, 128, 1000, [837], [0], (0,), (0,)),
    "128 fp32 own": ("fp32", 12, 8, 1, 128, 1000, [837], [0, 0, -1], (1,), (1,)),
}
OWN_N = [40, 7, 33]
RUNS = [(name, bool(rope)) for name, c in CASES.items() for rope in (0, 1) if c[8 + rope] is not None]


def make(name):
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the cases are sized for 256 compute units")
    dtype, S, Hq, Hkv, d, pc, n, of = CASES[name][:8]
    return Case(S, Hq, Hkv, d, dtype, SMALL, (0, 0, 1, pc), OWN_N, n, of, seed=len(name))


def wanted(case, rope):
    return tuple(t.cpu() for t in case.want(rope, "cuda"))


@pytest.mark.parametrize("factor", [1.0, 64.0])  # the second: maxima that rise again and again
@pytest.mark.parametrize("name,rope", RUNS)
def test_against_64_bits(sp, name, rope, factor):  # noqa: F811
    case = make(name)
    case.q.mul_(factor)
    out, lse = case.run(sp, rope)
    case.check(out, lse, rope, wanted(case, rope))
    again = case.run(sp, rope)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("name,rope", RUNS)
def test_values_not_finite(sp, name, rope):  # noqa: F811
    """An infinite value in the last entry (which fills up the last block) and in front of others, a query that is NaN: the sequences that see
    them show it, the others and the other columns are as accurate as without."""
    case = make(name)
    want, clean = wanted(case, rope), case.run(sp, rope)
    slots = slots_of(case.psizes[0], case.pa, case.ps, case.pc)
    case.Vp[0, :, slots[-1], 5], case.Vp[0, :, slots[100], 9] = float("inf"), float("-inf")
    behind = [i for i in range(case.S) if case.of[i] == 0]
    out, lse = case.run(sp, rope)
    assert (out[behind][..., 5] == float("inf")).all() and (out[behind][..., 9] == float("-inf")).all()
    for i in behind:
        out[i, :, 5], out[i, :, 9] = clean[0][i, :, 5], clean[0][i, :, 9]
    case.check(out, lse, rope, want)
    if len(behind) > 1:
        hit, head = behind[-2], case.Hq - 1
        case.q[hit, head, 3] = float("nan")
        out, lse = case.run(sp, rope)
        assert out[hit, head].isnan().all() and lse[hit, head].isnan()
        out[hit, head], lse[hit, head] = clean[0][hit, head], clean[1][hit, head]
        for i in behind:
            out[i, :, 5], out[i, :, 9] = clean[0][i, :, 5], clean[0][i, :, 9]
        case.check(out, lse, rope, want)


@pytest.mark.parametrize("name", [name for name, rope in RUNS if not rope])
@pytest.mark.parametrize("share", [0.45, 1.0])  # of the first prompt's entries: whole blocks and slices in front of the others, all of them
def test_scores_of_minus_infinity(sp, name, share):  # noqa: F811
    """Entries whose scores are minus infinity count with weight 0."""
    case = make(name)
    case.q[:, :, 0] = 1.0
    slots = slots_of(case.psizes[0], case.pa, case.ps, case.pc)
    none = int(share * len(slots))
    case.Kp[0][:, slots[:none], 0] = float("-inf")
    out, lse = case.run(sp, False)
    rest = len(slots) - none
    case.psizes[0] = [0, 0, max(rest - 1, 0), min(rest, 1), 0, (case.psizes[0][5] + none) % case.pc]
    case.check(out, lse, False, wanted(case, False))
