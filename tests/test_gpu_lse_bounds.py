"""How far lse may be off where a decode keeps 16 bits or more of everything: over a cache in 4 bits, and behind shared prompts.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
import test_gpu_decode_shared as shared  # noqa: E402
import test_gpu_mx_decode as mx  # noqa: E402
from test_gpu_mx_decode import sp  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def check(case, lse, rope, dtype):
    """A: the largest scale * sum over the dimensions of |q| |k| of a row's entries (with positions, |k| with its partner's over a cache in 4 bits, of the
    turned rows behind shared prompts).  A score is a sum of at most 128 exact products in fp32 (each sum off by 2^-24 of A: 2^-17), scaled (2^-21), with
    positions turned by angles that are off by 2^-20, and in bf16 the turned rows are two numbers (2^-16): below 2^-16 A, or 2^-15 A for bf16 with
    positions.  The sum's and the logarithm's roundings follow: 2^-20 and 2^-22 of lse."""
    _, want, _, A = case.want(rope)
    off = 2.0 ** (-15 if rope and dtype == "bf16" else -16)
    there = ~torch.isinf(want)
    err = (lse.double().cpu() - want).abs()[there]
    assert (err <= (off * A + 2.0 ** -20 + 2.0 ** -22 * want.abs())[there]).all(), float(err.max())


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("larger", [1.0, 4.0, 30.0])
def test_cache_in_4_bits(sp, larger, dtype, rope):  # noqa: F811
    case = mx.Case(4, 32, 8, 128, dtype, mx.STREAM, [300, 100, 35, 3], seed=2)
    case.q *= larger
    check(case, case.run(sp, rope)[1], rope, dtype)


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("larger", [1.0, 4.0, 30.0])
def test_behind_shared_prompts(sp, larger, dtype, rope):  # noqa: F811
    case = shared.Case(8, 32, 8, 128, dtype, shared.SMALL, (0, 0, 1, 700), [0, 1, 31, 32, 33, 40], [700], [0], seed=2)
    case.q *= larger
    check(case, case.run(sp, rope)[1], rope, dtype)
