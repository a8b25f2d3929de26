"""Norms of queries and keys with their rotary positions, against the definition in 64 bits.  Needs an MI355X."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2412_12094_amd as sp_

    sp_.load()
    return sp_


def randn(*shape, dtype, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def weight(d, dtype, seed):
    return (1.0 + 0.3 * torch.randn(d, generator=torch.Generator().manual_seed(seed))).to(dtype).cuda()


def f64(t):
    return t.detach().double().cpu()


def members(rotary, interleaved):
    n = rotary // 2
    return (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, n), slice(n, rotary))


def turn(x, pos, freqs, interleaved, sign=1.0):
    """float64 x [..., d] at positions [...], and the sum of the magnitudes that each value is made of."""
    x, size = x.clone(), x.abs()
    if freqs is None:
        return x, size
    angle = sign * pos.double()[..., None] * freqs.cpu()
    i, j = members(2 * freqs.numel(), interleaved)
    u, v = x[..., i].clone(), x[..., j].clone()
    x[..., i], x[..., j] = u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()
    size[..., i] = size[..., j] = u.abs() + v.abs()
    return x, size


def norm(x, w, eps):
    y = x / ((x * x).mean(-1, keepdim=True) + eps).sqrt()
    return y if w is None else y * f64(w)


def close(got, want, size):
    """One rounding to the output's type, and fp32 arithmetic.  The row's sum of squares is off by at most 2^-24 for each of the (at most 32) sums on a
    value's way, its root by half of that and rsqrt's 2^-22; two products; the turn adds 2^-20 of both members (cos and sin off by 2^-22, three
    roundings): 16 2^-24 + 2^-22 + 2^-23 + 2^-20 < 2^-18."""
    half_step = torch.finfo(got.dtype).eps / 2
    err = (f64(got) - want).abs()
    assert (err <= half_step * want.abs() + 2.0 ** -18 * size).all(), float((err - half_step * want.abs()).max())


def gradients(x, w, g, eps):
    """dx and the sum of magnitudes that its values are made of; dw and the sum over rows of magnitudes.  g float64, with the magnitudes that its values are made of."""
    g, gs = g
    r = 1.0 / ((x * x).mean(-1, keepdim=True) + eps).sqrt()
    ww = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else f64(w)
    u, us = g * ww, gs * ww.abs()
    dx = r * (u - x * r * r * (u * x).mean(-1, keepdim=True))
    dxs = r * (us + x.abs() * r * r * (us * x.abs()).mean(-1, keepdim=True))
    rows = tuple(range(x.dim() - 1))
    return dx, dxs, (g * x * r).sum(rows), (gs * (x * r).abs()).sum(rows)


def close_gradient(got, want, size):
    """As close(), with the row's r four times on the way and a second sum over the row: 4 (16 2^-24 + 2^-22) + 32 2^-24 + 2^-20 < 2^-16.5."""
    half_step = torch.finfo(got.dtype).eps / 2
    err = (f64(got) - want).abs()
    assert (err <= half_step * want.abs() + 2.0 ** -16.5 * size).all(), float((err - half_step * want.abs()).max())


def close_weight(got, want, size):
    """A term is off by 2^-18 (as in close()); a thread adds at most 128 of them in these tests and six levels follow in fp32, each sum off by
    2^-24 of the magnitudes in it; the rest is added in fp64, and the result rounded."""
    assert got.dtype == torch.float32
    err = (f64(got) - want).abs()
    assert (err <= (2.0 ** -18 + 134 * 2.0 ** -24) * size + 2.0 ** -24 * want.abs()).all(), float((err / size).max())


def projections(layout, B, L, Hq, Hkv, d, dtype, seed=0, fill=None):
    make = (lambda *s: randn(*s, dtype=dtype, seed=seed)) if fill is None else (lambda *s: torch.full(s, fill, dtype=dtype, device="cuda"))
    if layout == "fused":
        x = make(B, L, Hq + 2 * Hkv, d)
        parts = x.split([Hq, Hkv, Hkv], dim=2)
    elif layout == "per_head":
        x = make(B, L, Hq, 3, d)
        parts = x.unbind(3)
    elif layout == "padded":  # a row pitch of its own, tokens outermost
        x = make(L, B, Hq + 2 * Hkv, d + 16)
        parts = [t[..., :d].transpose(0, 1) for t in x.split([Hq, Hkv, Hkv], dim=2)]
    else:
        return None, [make(B, h, L, d) for h in (Hq, Hkv, Hkv)]
    return x, [t.transpose(1, 2) for t in parts]


CASES = [
    # B, L, Hq, Hkv, d, rotary, interleaved, layout, dtype, weights
    (1, 1, 1, 1, 64, 2, False, "dense", "bf16", "bf16"),
    (1, 1, 32, 8, 128, 128, False, "fused", "bf16", "bf16"),
    (2, 17, 5, 5, 64, 16, False, "per_head", "bf16", "fp32"),
    (3, 33, 7, 1, 128, 128, True, "fused", "bf16", "bf16"),
    (2, 31, 6, 3, 64, 38, False, "fused", "bf16", "none"),
    (2, 31, 6, 3, 64, 38, True, "padded", "bf16", "fp32"),
    (1, 130, 12, 4, 128, 126, False, "padded", "bf16", "bf16"),
    (2, 40, 4, 2, 128, 0, False, "fused", "bf16", "bf16"),
    (2, 40, 4, 2, 64, 0, True, "fused", "fp32", "none"),
    (5, 2, 3, 1, 128, 96, True, "fused", "fp32", "fp32"),
    (2, 65, 4, 2, 64, 64, False, "fused", "fp32", "bf16"),
    (1, 257, 28, 4, 128, 20, False, "fused", "fp32", "fp32"),
    (2, 9, 4, 4, 64, 36, True, "per_head", "fp32", "fp32"),
    (1, 2049, 2, 1, 128, 64, False, "dense", "bf16", "bf16"),
    (1, 16, 64, 8, 128, 128, False, "fused", "bf16", "bf16"),
]


@pytest.mark.parametrize("B,L,Hq,Hkv,d,rotary,interleaved,layout,dtype,weights", CASES)
@pytest.mark.parametrize("positions", ["index", "given", "documents"])
def test_forward_and_backward(sp, B, L, Hq, Hkv, d, rotary, interleaved, layout, dtype, weights, positions):
    dt = DTYPES[dtype]
    w = [None, None] if weights == "none" else [weight(d, DTYPES[weights], seed) for seed in (1, 2)]
    freqs = sp.sepattn_rope_frequencies(rotary, 10000.0, device="cuda") if rotary else None
    pos, given, doc = torch.arange(L).expand(B, L), None, None
    g = torch.Generator().manual_seed(1)
    if positions == "given":
        pos = torch.randint(-(1 << 31), (1 << 31) - 1, (B, L), generator=g)
        given = pos.to(torch.int32).cuda()
    elif positions == "documents":
        start = torch.where(torch.rand(B, L, generator=g) < 0.1, torch.arange(L), 0).cummax(1).values
        pos, doc = pos - start, start.to(torch.int32).cuda()
    kw = dict(positions=given, doc_start=doc, interleaved=interleaved)
    x, src = projections(layout, B, L, Hq, Hkv, d, dt)
    before = [t.clone() for t in src]
    Q, K, V = sp.sepattn_norm_rope(*src, *w, freqs, EPS, **kw)
    for got, t, ww in zip((Q, K), src, w):
        assert got.is_contiguous() and got.shape == t.shape
        close(got, *turn(norm(f64(t), ww, EPS), pos[:, None], freqs, interleaved))
    assert V.is_contiguous() and torch.equal(V, src[2])
    assert all(torch.equal(a, b) for a, b in zip(before, src))

    # the gradient, into a buffer of the projections' layout whose other values stay
    grads = [randn(B, h, L, d, dtype=dt, seed=5 + i) for i, h in enumerate((Hq, Hkv, Hkv))]
    dx, out = projections(layout, B, L, Hq, Hkv, d, dt, fill=7.0)
    *back, dwq, dwk = sp.sepattn_norm_rope_backward(*src[:2], *grads, *w, freqs, EPS, **kw, out=out)
    assert all(a is b for a, b in zip(back, out))
    for o, t, gr, ww, dw in zip(out, src, grads, w, (dwq, dwk)):
        want, size, want_w, size_w = gradients(f64(t), ww, turn(f64(gr), pos[:, None], freqs, interleaved, -1.0), EPS)
        close_gradient(o, want, size)
        close_weight(dw, want_w, size_w)
    assert torch.equal(out[2], grads[2])
    if layout == "padded":
        assert (dx[..., d:] == 7.0).all()
    # the same bits again, into buffers of the call's own, without values, without weights' gradients
    again = sp.sepattn_norm_rope_backward(*src[:2], *grads, *w, freqs, EPS, **kw)
    assert all(torch.equal(a, b) for a, b in zip(again, (*out, dwq, dwk)))
    less = sp.sepattn_norm_rope_backward(*src[:2], *grads[:2], None, *w, freqs, EPS, **kw, out_weights=(None, None))
    assert torch.equal(less[0], out[0]) and torch.equal(less[1], out[1]) and less[2:] == (None, None, None)
    one = torch.full((d,), 3.0, device="cuda")
    sp.sepattn_norm_rope_backward(*src[:2], *grads, *w, freqs, EPS, **kw, out_weights=(None, one))
    assert torch.equal(one, dwk)


def test_against_differences(sp):
    """The gradient of a sum of all outputs times fixed numbers, against central differences of the call itself in fp32."""
    B, L, Hq, Hkv, d = 1, 3, 2, 1, 64
    freqs = sp.sepattn_rope_frequencies(d, 10000.0, device="cuda")
    q, k = (randn(B, h, L, d, dtype=torch.float32, seed=h) for h in (Hq, Hkv))
    w = [weight(d, torch.float32, seed) for seed in (3, 4)]
    G = [randn(B, h, L, d, dtype=torch.float32, seed=7 + h) for h in (Hq, Hkv)]
    total = lambda q, k, w: sum((f64(a) * f64(b)).sum().item() for a, b in zip(sp.sepattn_norm_rope(q, k, None, *w, freqs, EPS), G))
    dq, dk, _, dwq, dwk = sp.sepattn_norm_rope_backward(q, k, *G, None, *w, freqs, EPS)
    rng = np.random.default_rng(0)
    # A difference over 2h = 2^-4: the outputs are off by 2^-18 of at most 2 (values up to 4, weights up to 2, both members) and there are 64 of them
    # that move, weighted by up to 4: by 64 2^-15 2^4 = 2^-5 at worst, 2^-5 / 8 with signs at random; third derivatives, below 8 a row, times h^2 / 6 add 2^-8
    h = 2.0 ** -5
    for t, dt in ((q, dq), (k, dk), (w[0], dwq), (w[1], dwk)):
        for i in rng.choice(t.numel(), 12, replace=False):
            at = t.view(-1)
            kept = at[i].item()
            at[i] = kept + h
            up = total(q, k, w)
            at[i] = kept - h
            down = total(q, k, w)
            at[i] = kept
            assert abs((up - down) / (2 * h) - dt.reshape(-1)[i].item()) < 2.0 ** -7 * (1 + abs(dt.reshape(-1)[i].item()))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_place_and_broadcast(sp, dtype):
    dt, B, L, Hq, Hkv, d = DTYPES[dtype], 2, 37, 8, 2, 128
    freqs = sp.sepattn_rope_frequencies(d, 10000.0, device="cuda")
    w = [weight(d, dt, 1), weight(d, dt, 2)]
    q, k = randn(B, Hq, L, d, dtype=dt), randn(B, Hkv, L, d, dtype=dt, seed=1)
    want = sp.sepattn_norm_rope(q, k, None, *w, freqs, EPS)
    a, b = q.clone(), k.clone()
    sp.sepattn_norm_rope(a, b, None, *w, freqs, EPS, out=(a, b, None))
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    grads = randn(B, Hq, L, d, dtype=dt, seed=2), randn(B, Hkv, L, d, dtype=dt, seed=3)
    back = sp.sepattn_norm_rope_backward(q, k, *grads, None, *w, freqs, EPS)
    a, b = (g.clone() for g in grads)
    sp.sepattn_norm_rope_backward(q, k, a, b, None, *w, freqs, EPS, out=(a, b, None))
    assert torch.equal(a, back[0]) and torch.equal(b, back[1])
    # one key head read as four, one row of q for all tokens
    k1, q1 = k[:, :1].expand(B, 4, L, d), q[:, :, :1].expand(B, Hq, L, d)
    got, dense = sp.sepattn_norm_rope(q1, k1, None, *w, freqs, EPS), sp.sepattn_norm_rope(q1.contiguous(), k1.contiguous(), None, *w, freqs, EPS)
    assert torch.equal(got[0], dense[0]) and torch.equal(got[1], dense[1])
    g1 = grads[1][:, :1].expand(B, 4, L, d)  # and so the gradients
    got = sp.sepattn_norm_rope_backward(q1, k1, grads[0], g1, None, *w, freqs, EPS)
    dense = sp.sepattn_norm_rope_backward(q1.contiguous(), k1.contiguous(), grads[0], g1.contiguous(), None, *w, freqs, EPS)
    assert all(torch.equal(x, y) for x, y in zip(got, dense) if x is not None)


def test_special_rows(sp):
    """Zeros with eps, small and large rows, infinities and NaN: each stays in its row."""
    B, L, H, d = 1, 9, 2, 64
    freqs = sp.sepattn_rope_frequencies(d, 10000.0, device="cuda")
    q, k = randn(B, H, L, d, dtype=torch.float32), randn(B, H, L, d, dtype=torch.float32, seed=1)
    grads = randn(B, H, L, d, dtype=torch.float32, seed=2), randn(B, H, L, d, dtype=torch.float32, seed=3)
    clean = sp.sepattn_norm_rope(q, k, None, None, None, freqs, EPS)
    clean_back = sp.sepattn_norm_rope_backward(q, k, *grads, None, None, None, freqs, EPS)
    x = q.clone()
    x[0, 0, 0] = 0.0
    x[0, 0, 2] *= 1e-12
    x[0, 0, 4] *= 1e17
    x[0, 0, 6, 5] = float("inf")
    x[0, 1, 8, 63] = float("nan")
    got = sp.sepattn_norm_rope(x, k, None, None, None, freqs, EPS)[0]
    back = sp.sepattn_norm_rope_backward(x, k, *grads, None, None, None, freqs, EPS)[0]
    assert (got[0, 0, 0] == 0).all()
    close(got[0, 0, :5], *turn(norm(f64(x[0, 0, :5]), None, EPS), torch.arange(5), freqs, False))
    rows = f64(x[0, 0, :5])
    want, size, _, _ = gradients(rows, None, turn(f64(grads[0][0, 0, :5]), torch.arange(5), freqs, False, -1.0), EPS)
    close_gradient(back[0, 0, :5], want, size)
    assert torch.isnan(got[0, 0, 6]).any() and torch.isnan(got[0, 1, 8]).all() and torch.isnan(back[0, 1, 8]).all()
    for l in (1, 3, 5, 7, 8):
        assert torch.equal(got[0, 0, l], clean[0][0, 0, l]) and torch.equal(back[0, 0, l], clean_back[0][0, 0, l])
    assert torch.equal(got[0, 1, :8], clean[0][0, 1, :8]) and torch.equal(back[0, 1, :8], clean_back[0][0, 1, :8])


def test_large(sp):
    """More than 128 MB, in tiles that do not fill a workgroup; sampled rows, and the weights' gradients from all."""
    B, L, Hq, Hkv, d = 3, 2731, 32, 8, 128
    freqs = sp.sepattn_rope_frequencies(d, 500000.0, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(B, L, Hq + 2 * Hkv, d, device="cuda", generator=g).to(torch.bfloat16)
    src = [t.transpose(1, 2) for t in x.split([Hq, Hkv, Hkv], dim=2)]
    w = [weight(d, torch.bfloat16, 1), weight(d, torch.bfloat16, 2)]
    Q, K, V = sp.sepattn_norm_rope(*src, *w, freqs, EPS)
    assert torch.equal(V, src[2])
    grads = [torch.randn(t.shape, device="cuda", generator=g).to(torch.bfloat16) for t in src]
    *dx, dwq, dwk = sp.sepattn_norm_rope_backward(*src[:2], *grads, *w, freqs, EPS)
    assert torch.equal(dx[2], grads[2])
    rows = torch.tensor([0, 1, 31, 32, 63, 64, 1000, 2700, 2729, 2730])
    for got, t, ww, d_, gr, dw in zip((Q, K), src, w, dx, grads, (dwq, dwk)):
        at = t[:, :, rows.cuda()]
        close(got[:, :, rows.cuda()], *turn(norm(f64(at), ww, EPS), rows, freqs, False))
        want, size, _, _ = gradients(f64(at), ww, turn(f64(gr[:, :, rows.cuda()]), rows, freqs, False, -1.0), EPS)
        close_gradient(d_[:, :, rows.cuda()], want, size)
        # all rows, on the GPU in float64
        xx, gg = t.double(), gr.double()
        r = 1.0 / ((xx * xx).mean(-1, keepdim=True) + EPS).sqrt()
        angle = torch.arange(L, device="cuda").double()[:, None] * freqs
        u, v = gg[..., :64], gg[..., 64:]
        y = torch.cat([u * angle.cos() + v * angle.sin(), v * angle.cos() - u * angle.sin()], -1)
        both = u.abs() + v.abs()
        close_weight(dw, (y * xx * r).sum((0, 1, 2)).cpu(), (torch.cat([both, both], -1) * (xx * r).abs()).sum((0, 1, 2)).cpu())


def test_streams_and_graph(sp):
    """Two calls at once on two streams, and a captured step (forward and backward) that is replayed with other inputs beside eager calls."""
    B, L, Hq, Hkv, d = 2, 300, 8, 2, 128
    freqs = sp.sepattn_rope_frequencies(d, 10000.0, device="cuda")
    w = [weight(d, torch.bfloat16, 1), weight(d, torch.bfloat16, 2)]
    make = lambda seed: [randn(B, h, L, d, dtype=torch.bfloat16, seed=seed + i) for i, h in enumerate((Hq, Hkv, Hkv))]
    step = lambda src, grads: (*sp.sepattn_norm_rope(*src, *w, freqs, EPS), *sp.sepattn_norm_rope_backward(*src[:2], *grads, *w, freqs, EPS))
    sets = [(make(10 * i), make(10 * i + 5)) for i in range(3)]
    want = [step(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got.append((i, step(*sets[i])))
    torch.cuda.synchronize()
    for i, r in got:
        assert all(torch.equal(a, b) for a, b in zip(r, want[i]))
    held = [[t.clone() for t in part] for part in sets[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*held)
    for i in (1, 2, 0, 1):
        for part, new in zip(held, sets[i]):
            for t, n in zip(part, new):
                t.copy_(n)
        graph.replay()
        eager = step(*sets[i])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i])) and all(torch.equal(a, b) for a, b in zip(eager, want[i]))


@pytest.mark.parametrize("dtype,d,rotary,interleaved", [("bf16", 128, 128, False), ("bf16", 64, 16, False), ("bf16", 128, 38, True), ("fp32", 128, 20, False),
                                                        ("fp32", 64, 64, True), ("bf16", 128, 0, False)])
@pytest.mark.parametrize("S,Hq,Hkv", [(1, 32, 8), (5, 7, 7), (3, 80, 40)])
def test_token_into_the_cache(sp, dtype, d, rotary, interleaved, S, Hq, Hkv):
    """The append with norm: the query and the key as sepattn_norm_rope gives them, the cache as sepkv_append leaves it."""
    dt, a, s, w, c = DTYPES[dtype], 2, 5, 4, 21
    freqs = sp.sepattn_rope_frequencies(rotary, 10000.0, device="cuda") if rotary else None
    wq, wk = weight(d, dt, 1), weight(d, dt, 2)
    q, k, v = randn(S, Hq, d, dtype=dt), randn(S, Hkv, d, dtype=dt, seed=1), randn(S, Hkv, d, dtype=dt, seed=2)
    pos = torch.arange(S, dtype=torch.int32, device="cuda") * 1000003
    rows = [[0, 0, 0, 0, 0, 0], [2, 3, 2, 4, 1, 7], [2, 5, 10, 4, 0, 3], [1, 0, 0, 0, 0, 0], [2, 0, 0, 3, 0, 13]]  # empty, in use, full, ...
    sizes = torch.tensor([rows[i % 5] for i in range(S)], dtype=torch.int32, device="cuda")
    sep = torch.ones(S, dtype=torch.uint8, device="cuda")
    cache = lambda: [randn(S, Hkv, c, d, dtype=dt, seed=3), randn(S, Hkv, c, d, dtype=dt, seed=4), torch.zeros(S, c - a - s, dtype=torch.uint8, device="cuda"), sizes.clone()]
    got, want = cache(), cache()
    out = sp.sepkv_append_norm_rope(q, k, v, sep, pos if rotary else None, wq, wk, freqs, EPS, *got, a, s, w, interleaved=interleaved)
    turned = sp.sepattn_norm_rope(q[:, :, None], k[:, :, None], None, wq, wk, freqs, EPS, positions=pos[:, None].contiguous(), interleaved=interleaved)
    sp.sepkv_append(turned[1][:, :, 0].contiguous(), v, sep, *want, Hq, a, s, w)
    assert torch.equal(out, turned[0][:, :, 0]) and all(torch.equal(x, y) for x, y in zip(got, want))
    got = cache()
    assert sp.sepkv_append_norm_rope(q, k, v, sep, pos if rotary else None, wq, wk, freqs, EPS, *got, a, s, w, interleaved=interleaved, out=q) is q
    assert torch.equal(q, out) and all(torch.equal(x, y) for x, y in zip(got, want))


def test_training_step(sp):
    """Norm and rotation, attention, and both gradients in one chain, against autograd of the chain in 64 bits."""
    B, Hq, Hkv, L, d, a, n = 1, 4, 2, 70, 64, 2, 16
    freqs = sp.sepattn_rope_frequencies(d, 10000.0, device="cuda")
    x = randn(B, L, Hq + 2 * Hkv, d, dtype=torch.float32)
    w = [weight(d, torch.float32, 1), weight(d, torch.float32, 2)]
    flags = (torch.rand(B, L, generator=torch.Generator().manual_seed(0)) < 0.1).to(torch.uint8)
    idx, cnt, pre = sp.sepattn_compact_indices(flags.cuda())
    src = [t.transpose(1, 2) for t in x.split([Hq, Hkv, Hkv], dim=2)]
    Q, K, V = sp.sepattn_norm_rope(*src, *w, freqs, EPS)
    scale = d ** -0.5
    O, LSE = sp.sepattn_forward(Q, K, V, idx, cnt, pre, a, n, scale)
    dO = randn(B, Hq, L, d, dtype=torch.float32, seed=9)
    dx = torch.empty_like(x)
    grads = sp.sepattn_backward(Q, K, V, O, LSE, dO, idx, cnt, pre, a, n, scale)
    *_, dwq, dwk = sp.sepattn_norm_rope_backward(*src[:2], *grads, *w, freqs, EPS, out=[t.transpose(1, 2) for t in dx.split([Hq, Hkv, Hkv], dim=2)])
    x64, w64 = f64(x).requires_grad_(), [f64(t).requires_grad_() for t in w]
    angle = torch.arange(L).double()[:, None] * freqs.cpu()

    def rows(t, weight_):
        t = t.transpose(1, 2)
        t = t / ((t * t).mean(-1, keepdim=True) + EPS).sqrt() * weight_
        u, v = t[..., : d // 2], t[..., d // 2:]
        return torch.cat([u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()], -1)

    q, k, v = x64.split([Hq, Hkv, Hkv], dim=2)
    q, k, v = rows(q, w64[0]), rows(k, w64[1]).repeat_interleave(Hq // Hkv, 1), v.transpose(1, 2).repeat_interleave(Hq // Hkv, 1)
    i, j = torch.arange(L)[:, None], torch.arange(L)[None]
    seen = (j <= i) & ((j < a) | (i - j < n) | (flags[0][None] > 0))
    o = torch.softmax((q @ k.transpose(-1, -2) * scale).masked_fill(~seen, float("-inf")), -1) @ v
    o.backward(f64(dO))
    # the attention's fp32 path holds 1e-4 (absolute, gradients of order one); the norm's gradient multiplies by w r, at most 2 here; a weight's
    # gradient is a sum over 4 * 70 rows of such errors times values up to 4, with signs at random (sqrt(280) 4 e-4 < 1e-2)
    assert (f64(O) - o.detach()).abs().max() < 1e-4
    assert (f64(dx) - x64.grad).abs().max() < 4e-4
    assert (f64(dwq) - w64[0].grad).abs().max() < 1e-2 and (f64(dwk) - w64[1].grad).abs().max() < 1e-2
