"""The cache in 4 bits: every code with every scale byte, those included that the library itself does not write.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_mx_decode import DTYPES, LEVELS, STREAM, Case, slots_of, sp  # noqa: E402, F401

pytestmark = pytest.mark.gpu


def all_codes(d):
    """Codes of a row: every one of the sixteen in every block of 32, packed."""
    code = torch.arange(d).remainder(16)
    return code, (code[0::2] | (code[1::2] << 4)).to(torch.uint8)


def value_of(code, byte, dtype):
    """float64 of code times 2^(byte - 127) in dtype: beyond its range infinite; of byte 255 NaN."""
    v = (LEVELS[code] * torch.exp2(byte.double() - 127)[..., None]).to(dtype).double()
    return torch.where((byte == 255)[..., None], float("nan"), v)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_values(sp, d, dtype):  # noqa: F811
    """Slot j has scale byte j in block 0, 255 - j in block 1, and so on.  Exact, subnormal values included; magnitudes from 2^128 on are infinite."""
    c, dt = 256, DTYPES[dtype]
    code, row = all_codes(d)
    byte = torch.stack([torch.arange(256) if b % 2 == 0 else 255 - torch.arange(256) for b in range(d // 32)], -1)
    codes = row.expand(1, 1, c, d // 2).contiguous().cuda()
    scales = byte.to(torch.uint8)[None, None].contiguous().cuda()
    sizes = torch.tensor([[0, 0, c - 1, 1, 0, 0]], dtype=torch.int32, device="cuda")
    want = torch.stack([value_of(code[32 * b: 32 * b + 32], byte[:, b], dt) for b in range(d // 32)], 1).flatten(1)
    for got in sp.sepkv_expand_mx(codes, scales, codes.clone(), scales.clone(), sizes, 0, 0, 1, dtype=dt):
        got = got[0, 0].cpu().double()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        there = ~torch.isnan(want)
        assert torch.equal(got[there], want[there]) and torch.equal(torch.signbit(got[there]), torch.signbit(want[there]))


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_decode(sp, d, dtype, rope):  # noqa: F811
    """One entry a sequence, which has weight 1: the output is its value, exactly, for scale bytes 0 to 252; lse is its score for key scales from 0 up to
    2^95, off by four roundings of 2^-24 (and with positions 2^-20, in bf16 2^-16 more), below 2^-126 by that."""
    S, c, dt = 256, 8, DTYPES[dtype]
    code, row = all_codes(d)
    codes = row.expand(S, 1, c, d // 2).contiguous().cuda()
    byte = torch.arange(256, dtype=torch.uint8)[:, None, None, None].expand(S, 1, c, d // 32).contiguous().cuda()
    one = torch.full_like(byte, 127)
    sizes = torch.tensor([[0, 0, 0, 1, 0, 0]] * S, dtype=torch.int32, device="cuda")
    q = torch.zeros(S, 1, d, dtype=dt, device="cuda")
    q[:, :, 7] = 1.0  # of code 7: magnitude 6
    if rope:
        table = sp.sepkv_rope_table(c, d, 10000.0, "cuda")
        call = lambda Ks, Vs: sp.sepattn_decode_rope_mx(q, codes, Ks, codes, Vs, sizes, table, 0, 0, 1, 1.0)
    else:
        call = lambda Ks, Vs: sp.sepattn_decode_mx(q, codes, Ks, codes, Vs, sizes, 0, 0, 1, 1.0)
    out, lse = call(one, byte)
    assert torch.equal(out[:253, 0].cpu().double(), value_of(code, torch.arange(253), dt)) and torch.isnan(out[255]).all()
    finite = torch.isfinite(value_of(code, torch.tensor([253, 254]), dt))
    assert torch.equal(torch.isfinite(out[253:255, 0].cpu()), finite)  # magnitudes of 2^128 and more reach their own dimensions
    assert torch.equal(out[253:255, 0].cpu().double()[finite], value_of(code, torch.tensor([253, 254]), dt)[finite])
    out, lse = call(byte, one)
    score = (6.0 * torch.exp2(torch.arange(223).double() - 127))[:, None]
    off = 4 * 2.0 ** -24 + (2.0 ** -20 + (2.0 ** -16 if dtype == "bf16" else 0.0) if rope else 0.0)
    assert ((lse[:223].cpu().double() - score).abs() <= off * score + 2.0 ** -126).all()
    assert torch.equal(out[:223, 0].cpu().double(), value_of(code, torch.full((223,), 127), dt)) and torch.isnan(lse[255]).all()


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_infinite_magnitudes_stay_apart(sp, dtype, rope):  # noqa: F811
    """A key and a value with magnitudes past fp32: every query head that does not see them, and every other dimension, has the bits that it has without."""
    x = Case(3, 8, 2, 64, dtype, STREAM, [300, 100, 35], seed=3)
    out, lse = x.run(sp, rope)
    key, value = slots_of(x.sizes[1], x.a, x.s, x.c)[50], slots_of(x.sizes[2], x.a, x.s, x.c)[-1]
    x.cache[0][1, 1, key, :16] = 0x77  # code 7 in all dimensions of block 0
    x.cache[1][1, 1, key, 0] = 254
    x.cache[2][2, 0, value, 16:] = 0x77
    x.cache[3][2, 0, value, 1] = 253
    got, got_lse = x.run(sp, rope)
    same, same_lse = torch.ones_like(out, dtype=torch.bool), torch.ones_like(lse, dtype=torch.bool)
    same[1, 4:], same[2, :4, 32:], same_lse[1, 4:] = False, False, False
    assert torch.equal(got[same], out[same]) and torch.equal(got_lse[same_lse], lse[same_lse])
