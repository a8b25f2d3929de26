"""Decoding behind shared prompts: an infinite value comes out as the definition has it, wherever its entry lies.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_decode_shared import BASE, SMALL, Case, slots_of, sp, turn  # noqa: E402, F401

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


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("S,Hq,Hkv,d,n,own_n", [
    (1, 1, 1, 64, 300, [40]), (2, 32, 8, 128, 600, [40, 1]), (8, 8, 2, 128, 700, [40, 33, 0]), (4, 32, 4, 64, 2500, [17]), (3, 8, 2, 64, 0, [40, 39, 2])])
def test_weights_of_16_bits(sp, S, Hq, Hkv, d, n, own_n, rope):  # noqa: F811
    """Up to 32 rows of a KV head, and in own caches: a weight is the sum of two bf16 numbers.  The first is off by 2^-7 of it at most (the last one
    below), the second, which is rounded, by 2^-8 of that.  The rest of the bound: Case.check."""
    case = Case(S, Hq, Hkv, d, "bf16", SMALL, (0, 0, 1, 2600), own_n, [n], [0], seed=S + d)
    out, lse = case.run(sp, rope)
    ref, _, size, reach = case.want(rope)
    score = reach * (d * 2.0 ** -24 + 2.0 ** -21 + (2.0 ** -20 + 2.0 ** -16 if rope else 0.0))
    err = (out.double().cpu() - ref).abs()
    bound = 2.0 ** -8 * ref.abs() + (2.0 ** -15 + 2.0 * score[..., None] + 2.0 ** -18) * size
    assert (err <= bound).all(), float((err / bound).max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("S,Hq,Hkv,d,n,own_n", [(4, 8, 2, 64, 700, [40, 7, 1]), (20, 8, 2, 128, 900, [33]), (3, 16, 2, 128, 2600, [40, 0]), (2, 4, 4, 64, 3, [1])])
def test_positions_from_keys_that_are_not_turned(sp, S, Hq, Hkv, d, n, own_n, dtype):  # noqa: F811
    """The whole chain, sepkv_rope_cache and the decode, against 64 bits from the keys as they were: a turned key of a prefix is stored in the
    cache's type, in bf16 off by 2^-8 of it at most (fp32: 2^-24, and the turn's 2^-20), and so is a score by that of its sum of magnitudes."""
    case = Case(S, Hq, Hkv, d, dtype, SMALL, (4, 30, 20, 2700), own_n, [n], [0], seed=n)
    table = sp.sepkv_rope_table(case.pc, d, BASE, "cuda")
    at = slots_of(case.psizes[0], case.pa, case.ps, case.pc)
    plain = case.Kp.clone()
    sp.sepkv_rope_cache(case.Kp, case.psz, table, case.pa, case.ps, case.pw)
    out, lse = case.run(sp, True)
    case.Kp = plain.double()
    case.Kp[0][:, at] = turn(case.Kp[0][:, at], torch.arange(n, device="cuda")[None])
    ref, ref_lse, size, reach = case.want(True)
    stored = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -20
    score = reach * (d * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -20 + (2.0 ** -16 if dtype == "bf16" else 0.0) + stored)
    err = (lse.double().cpu() - ref_lse).abs()
    print(f"lse off by {float(err.max()):.1e}, bound {float((score + 2.0 ** -22 * (ref_lse.abs() + 8.0)).min()):.1e}")
    assert (err <= score + 2.0 ** -22 * (ref_lse.abs() + 8.0)).all(), float(err.max())
    err = (out.double().cpu() - ref).abs()
    half = torch.finfo(case.dt).eps / 2
    assert (err <= half * ref.abs() + ((2.0 ** -8 if dtype == "bf16" else 0.0) + 2.0 * score[..., None] + 2.0 ** -18) * size).all(), float(err.max())
