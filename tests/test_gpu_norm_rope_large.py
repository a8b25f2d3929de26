"""Norms with rotary positions, calls of more than 128 MB: every form that reads its rows with the non-temporal hint, rows of 128 bytes, which are cut
into many chunks of heads, and pairs that are not whole pieces, against the definition in 64 bits on the GPU.  Needs an MI355X."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_norm_rope import DTYPES, EPS, members, projections, randn, sp, weight  # noqa: E402, F401

pytestmark = pytest.mark.gpu

CASES = [
    # B, L, Hq, Hkv, d, rotary, interleaved, layout, dtype; the first five with the hint (rows of 256 bytes and more)
    (1, 5501, 32, 8, 128, 128, False, "fused", "bf16"),
    (3, 2501, 28, 4, 128, 96, True, "fused", "bf16"),
    (2, 2805, 32, 8, 64, 64, False, "padded", "fp32"),
    (1, 3001, 37, 5, 128, 36, True, "dense", "fp32"),
    (2, 3003, 32, 8, 64, 0, True, "fused", "fp32"),
    (1, 5701, 37, 5, 128, 20, False, "fused", "bf16"),      # value by value
    (8, 1855, 12, 12, 64, 16, False, "per_head", "bf16"),   # rows of 128 bytes
    (5, 4001, 13, 7, 64, 64, True, "fused", "bf16"),
]


def turn(x, angle, interleaved):
    """float64 rows [B, L, d] turned, and the sum of the magnitudes that each value is made of."""
    x, size = x.clone(), x.abs()
    if angle is not None:
        i, j = members(2 * angle.shape[-1], interleaved)
        u, v, cos, sin = x[..., i].clone(), x[..., j].clone(), angle.cos(), angle.sin()
        x[..., i], x[..., j] = u * cos - v * sin, v * cos + u * sin
        size[..., i] = size[..., j] = u.abs() + v.abs()
    return x, size


@pytest.mark.parametrize("B,L,Hq,Hkv,d,rotary,interleaved,layout,dtype", CASES)
def test_large_calls(sp, B, L, Hq, Hkv, d, rotary, interleaved, layout, dtype):  # noqa: F811
    """The bounds of close(), close_gradient() and close_weight() in test_gpu_norm_rope.py, head by head; a thread adds at most 512 terms of a weight's gradient
    here: q and k are walked by a twelfth of 768 workgroups or more each, 16 rows and more at a time, and 37 * 5701 / (64 * 16) = 206."""
    dt = DTYPES[dtype]
    assert 2 * d * dt.itemsize * B * L * (Hq + 2 * Hkv) > 128 << 20
    freqs = sp.sepattn_rope_frequencies(rotary, 10000.0, device="cuda") if rotary else None
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (B, L), device="cuda", generator=torch.Generator(device="cuda").manual_seed(L))
    angle = pos.double()[..., None] * freqs if rotary else None
    kw = dict(positions=pos.to(torch.int32), interleaved=interleaved)
    w = [weight(d, dt, 1), weight(d, torch.float32 if dtype == "fp32" else dt, 2)]
    x, src = projections(layout, B, L, Hq, Hkv, d, dt)
    before = [t.clone() for t in src]
    half = torch.finfo(dt).eps / 2
    got = sp.sepattn_norm_rope(*src, *w, freqs, EPS, **kw)
    assert all(torch.equal(a, b) for a, b in zip(before, src)) and torch.equal(got[2], src[2])
    grads = [randn(B, h, L, d, dtype=dt, seed=5 + i) for i, h in enumerate((Hq, Hkv, Hkv))]
    dx, out = projections(layout, B, L, Hq, Hkv, d, dt, fill=7.0)
    *_, dwq, dwk = sp.sepattn_norm_rope_backward(*src[:2], *grads, *w, freqs, EPS, **kw, out=out)
    for y, t, gr, o, ww, dw in zip(got, src, grads, out, w, (dwq, dwk)):
        want_w, size_w = (torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(2))
        ww = ww.double()
        for h in range(t.shape[1]):
            row = t[:, h].double()
            r = 1.0 / ((row * row).mean(-1, keepdim=True) + EPS).sqrt()
            want, size = turn(row * r * ww, angle, interleaved)
            err = (y[:, h].double() - want).abs()
            assert bool((err <= half * want.abs() + 2.0 ** -18 * size).all()), (h, float(err.max()))
            g, gs = turn(gr[:, h].double(), None if angle is None else -angle, interleaved)
            want_w, size_w = want_w + (g * row * r).sum((0, 1)), size_w + (gs * (row * r).abs()).sum((0, 1))
            u, us = g * ww, gs * ww.abs()
            want = r * (u - row * r * r * (u * row).mean(-1, keepdim=True))
            size = r * (us + row.abs() * r * r * (us * row.abs()).mean(-1, keepdim=True))
            err = (o[:, h].double() - want).abs()
            assert bool((err <= half * want.abs() + 2.0 ** -16.5 * size).all()), (h, float(err.max()))
        err = (dw.double() - want_w).abs()
        assert bool((err <= (2.0 ** -18 + 518 * 2.0 ** -24) * size_w + 2.0 ** -24 * want_w.abs()).all()), float((err / size_w).max())
    assert torch.equal(out[2], grads[2])
    if layout == "padded":
        assert (dx[..., d:] == 7.0).all()
    # in place, both
    sp.sepattn_norm_rope_backward(*src[:2], *grads, *w, freqs, EPS, **kw, out=grads)
    assert all(torch.equal(a, b) for a, b in zip(grads, out))
    sp.sepattn_norm_rope(*src, *w, freqs, EPS, **kw, out=src)
    assert all(torch.equal(a, b) for a, b in zip(src, got))
    if layout == "padded":
        assert torch.equal(x[..., d:], projections(layout, B, L, Hq, Hkv, d, dt)[0][..., d:])
