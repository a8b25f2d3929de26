"""Rotary positions, calls whose rows are read with the non-temporal hint or cut into many chunks of heads (more than 128 MB read and written), on the
GPU against the definition in 64 bits.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_rope import DTYPES, members, projections, sp  # noqa: E402, F401

pytestmark = pytest.mark.gpu

CASES = [
    # B, L, Hq, Hkv, d, rotary, interleaved, layout, dtype; the first four with the hint (rows of 256 bytes and more)
    (1, 5501, 32, 8, 128, 128, False, "fused", "bf16"),
    (3, 2501, 28, 4, 128, 96, True, "fused", "bf16"),
    (2, 2805, 32, 8, 64, 64, False, "padded", "fp32"),
    (1, 3001, 37, 5, 128, 36, True, "dense", "fp32"),
    (1, 5701, 37, 5, 128, 20, False, "fused", "bf16"),      # value by value
    (8, 1855, 12, 12, 64, 16, False, "per_head", "bf16"),   # rows of 128 bytes
    (5, 4001, 13, 7, 64, 64, True, "fused", "bf16"),
]


def close(got, t, angle, interleaved):
    """The bounds of test_gpu_rope.close, head by head on the GPU; the other dimensions bit for bit."""
    rotary = 2 * angle.shape[-1]
    i, j = members(rotary, interleaved)
    half_step, cos, sin = torch.finfo(got.dtype).eps / 2, angle.cos(), angle.sin()
    for h in range(t.shape[1]):
        x, y = t[:, h], got[:, h]
        u, v = x[..., i].double(), x[..., j].double()
        size = 2.0 ** -20 * (u.abs() + v.abs())
        for part, want in ((y[..., i], u * cos - v * sin), (y[..., j], v * cos + u * sin)):
            err = (part.double() - want).abs()
            assert bool((err <= half_step * want.abs() + size).all()), (h, float(err.max()))
        assert torch.equal(y[..., rotary:], x[..., rotary:])


@pytest.mark.parametrize("B,L,Hq,Hkv,d,rotary,interleaved,layout,dtype", CASES)
@pytest.mark.parametrize("positions", ["index", "given"])
def test_large_calls(sp, B, L, Hq, Hkv, d, rotary, interleaved, layout, dtype, positions):  # noqa: F811
    dt = DTYPES[dtype]
    assert 2 * d * dt.itemsize * B * L * (Hq + 2 * Hkv) > 128 << 20
    freqs = sp.sepattn_rope_frequencies(rotary, 10000.0, device="cuda")
    pos, given = torch.arange(L, device="cuda").expand(B, L), None
    if positions == "given":
        pos = torch.randint(-(1 << 31), (1 << 31) - 1, (B, L), device="cuda", generator=torch.Generator(device="cuda").manual_seed(L))
        given = pos.to(torch.int32)
    angle = pos.double()[..., None] * freqs
    x, src = projections(layout, B, L, Hq, Hkv, d, dt)
    before = [t.clone() for t in src]
    kw = dict(positions=given, interleaved=interleaved)
    got = sp.sepattn_rope(*src, freqs, **kw)
    assert all(torch.equal(a, b) for a, b in zip(before, src))
    for y, t in zip(got[:2], src):
        close(y, t, angle, interleaved)
    assert torch.equal(got[2], src[2])
    # the gradient, into the projections' layout, whose other values stay
    dx, out = projections(layout, B, L, Hq, Hkv, d, dt, fill=7.0)
    sp.sepattn_rope_backward(*before, freqs, out=out, **kw)
    for y, t in zip(out[:2], before):
        close(y, t, -angle, interleaved)
    assert torch.equal(out[2], before[2])
    if layout == "padded":
        assert (dx[..., d:] == 7.0).all()
    # in place
    sp.sepattn_rope(*src, freqs, out=src, **kw)
    assert all(torch.equal(a, b) for a, b in zip(src, got))
    if layout == "padded":
        assert torch.equal(x[..., d:], projections(layout, B, L, Hq, Hkv, d, dt)[0][..., d:])
