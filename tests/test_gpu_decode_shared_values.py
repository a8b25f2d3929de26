"""Decoding behind shared prompts: an infinite value comes out as the definition has it, wherever its entry lies.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_decode_shared import SMALL, Case, slots_of, sp  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("where", ["first", "last"])  # entry of the cache: the last one is the row that a block is filled up with
@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("S,Hq,Hkv,d,n,own_n", [
    (3, 8, 2, 64, 555, [40, 7, 33]),      # 12 rows of a KV head: every wave has all of them
    (8, 8, 2, 128, 555, [40, 7, 33]),     # 32
    (20, 8, 2, 128, 690, [40, 7, 33]),    # 80: each wave has its own
    (40, 16, 2, 64, 2500, [39]),          # 320
    (5, 8, 2, 128, 1, [1])])              # a block of one entry
def test_infinite_values(sp, S, Hq, Hkv, d, n, own_n, dtype, rope, where):  # noqa: F811
    """Every weight is positive, so a value of +inf (-inf) makes its column +inf (-inf) for the sequences that see it; the other columns
    and sequences are as accurate as without."""
    case = Case(S, Hq, Hkv, d, dtype, SMALL, (0, 0, 1, 2600), own_n, [n], [0, 0, -1], seed=S)
    want, clean = case.want(rope), case.run(sp, rope)
    entry = 0 if where == "first" else -1
    slot = slots_of(case.psizes[0], case.pa, case.ps, case.pc)[entry]
    case.Vp[0, :, slot, 5], case.Vp[0, :, slot, 9] = float("inf"), float("-inf")
    case.Vc[2, :, slots_of(case.sizes[2], case.a, case.s, case.c)[entry], 33] = float("inf")  # a sequence without a prompt
    case.Vc[1, :, slots_of(case.sizes[1], case.a, case.s, case.c)[entry], 33] = float("-inf")
    out, lse = case.run(sp, rope)
    behind = [i for i in range(S) if case.of[i] == 0]
    for rows, column, value in ((behind, 5, float("inf")), (behind, 9, float("-inf")), ([2], 33, float("inf")), ([1], 33, float("-inf"))):
        assert (out[rows][..., column] == value).all(), (column, out[rows][..., column])
        for i in rows:
            out[i, :, column] = clean[0][i, :, column]
    case.check(out, lse, rope, want)
