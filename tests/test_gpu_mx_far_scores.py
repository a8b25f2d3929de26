"""Decode over a cache in 4 bits with scores from 2^20 to 2^95, where neighbouring fp32 numbers lie up to 2^72 apart.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_mx_decode import DTYPES, sp, values  # noqa: E402, F401

pytestmark = pytest.mark.gpu

EXPONENTS = [20, 23, 24, 25, 27, 28, 29, 30, 31, 32, 33, 47, 63, 80, 95]
Hq, Hkv, SILENT = 8, 2, 5  # query head SILENT asks for nothing: its scores are 0
ASKED = 1.296875  # of dimension 0, in the others: a number of eight bits, so that its product with log2(e) has to be rounded


def decode(sp, q, cache, sizes, c, rope):  # noqa: F811
    args = (q, *cache, torch.tensor(sizes, dtype=torch.int32, device="cuda"))
    if rope:
        return sp.sepattn_decode_rope_mx(*args, sp.sepkv_rope_table(c, q.shape[-1], 10000.0, "cuda"), 0, 0, 1, 1.0)
    return sp.sepattn_decode_mx(*args, 0, 0, 1, 1.0)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64), ("fp32", 128)])
# (with positions keys at other places are turned away from the query)
@pytest.mark.parametrize("kind,n,rope", [("one ahead", n, rope) for n in (1, 32, 70, 1111) for rope in (False, True)]
                         + [(kind, n, False) for kind in ("one behind", "two ahead") for n in (32, 70, 1111)])
def test_far_scores(sp, dtype, d, n, kind, rope):  # noqa: F811
    """Sequence i has scores of ASKED 2^EXPONENTS[i] and the like, which every weight but the winners' vanishes behind: the output is the winner's value.  Where the
    largest score times log2(e) is 2^24 or more, bit for bit: weights 1 and 0, the mean of two exact in fp32 and rounded once.  Below that the winner's weight is
    2^x with x what the rounding of the maximum left, at most 1/2: cut into two numbers (bf16, off by 2^-16) or three (fp32, 2^-24), times the value and
    added (2^-24 each), over the sum of the weights (2^-24) by a division (2^-24), so off by 2^-22 of the values' magnitudes beside the cut, and rounded.
    lse is its score: off by the roundings of scale log2(e), of the product, of the
    sum with log2(1 or 2), of ln 2 and of the product with it, each 2^-24: less than 2^-21.  With positions the newest key's cos and sin are formed from two
    table rows (2^-20), and in bf16 the turned key is two numbers (2^-16)."""
    S, dt = len(EXPONENTS), DTYPES[dtype]
    g = torch.Generator().manual_seed(n)
    u8 = lambda low, high, *shape: torch.randint(low, high, shape, generator=g, dtype=torch.uint8)
    Vc, Vs = u8(0, 256, S, Hkv, n, d // 2), u8(124, 127, S, Hkv, n, d // 32)
    Kc, Ks = torch.zeros(S, Hkv, n, d // 2, dtype=torch.uint8), torch.full((S, Hkv, n, d // 32), 127, dtype=torch.uint8)
    Ks[..., 0] = torch.tensor([127 + e for e in EXPONENTS], dtype=torch.uint8)[:, None, None]
    one, minus_one, minus_two = 2, 10, 12  # codes of dimension 0
    if kind == "one behind":
        Kc[..., 0] = minus_two
    Kc[:, :, n - 1, 0] = minus_one if kind == "one behind" else one  # the newest entry: nothing turns its key
    other = n // 3
    if kind == "two ahead":
        Kc[:, :, other, 0] = one
    q = torch.zeros(S, Hq, d, dtype=dt)
    q[:, :, 0] = ASKED
    q[:, SILENT] = 0.0
    c = n + 1
    room = lambda t: torch.cat([t, torch.full((S, Hkv, 1, t.shape[-1]), 255, dtype=torch.uint8)], 2).cuda()
    cache, sizes = [room(t) for t in (Kc, Ks, Vc, Vs)], [[0, 0, n - 1, 1, 0, 0]] * S
    out, lse = decode(sp, q.cuda(), cache, sizes, c, rope)
    V = values(Vc, Vs)
    want = V[:, :, n - 1] if kind != "two ahead" else (V[:, :, n - 1] + V[:, :, other]) / 2
    want = want.repeat_interleave(Hq // Hkv, 1)
    score = torch.tensor([ASKED * 2.0 ** e for e in EXPONENTS], dtype=torch.float64)[:, None]
    score = -score if kind == "one behind" else score
    heard = [h for h in range(Hq) if h != SILENT]
    print("case", kind, dtype, d, n, rope, flush=True)
    got, want = out[:, heard].cpu().double(), want[:, heard]
    far = torch.tensor([ASKED * 2.0 ** e * 1.442695 >= 2.0 ** 24 for e in EXPONENTS])
    assert torch.equal(got[far], want[far].to(dt).double())
    size = (V[:, :, n - 1].abs() if kind != "two ahead" else (V[:, :, n - 1].abs() + V[:, :, other].abs()) / 2).repeat_interleave(Hq // Hkv, 1)[:, heard]
    assert ((got - want).abs() <= torch.finfo(dt).eps / 2 * want.abs() + ((2.0 ** -16 if dtype == "bf16" else 2.0 ** -24) + 2.0 ** -22) * size).all()
    off = 2.0 ** -21 + (2.0 ** -20 + (2.0 ** -16 if dtype == "bf16" else 0.0) if rope else 0.0)
    assert ((lse[:, heard].cpu().double() - score).abs() <= off * score.abs() + (1.0 if kind == "two ahead" else 0.0)).all()
    # the head beside them gives the bits that it gives alone
    alone = decode(sp, torch.zeros_like(q).cuda(), cache, sizes, c, rope)
    assert torch.equal(out[:, SILENT], alone[0][:, SILENT]) and torch.equal(lse[:, SILENT], alone[1][:, SILENT])
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
