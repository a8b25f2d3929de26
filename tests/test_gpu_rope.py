"""Rotary positions in front of the attention and at the cache's door, against the definition in 64 bits.  Needs an MI355X."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2412_12094_amd as sp_

    sp_.load()
    return sp_


def members(rotary, interleaved):
    """The first and the second dimensions of the pairs."""
    n = rotary // 2
    return (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, n), slice(n, rotary))


def turned(x, pos, freqs, interleaved, sign=1.0):
    """x [..., d] (any type) at positions [...], in float64; and the sum of the magnitudes of what each value is made of."""
    x = x.detach().double().cpu().clone()
    angle = sign * pos.double().cpu()[..., None] * freqs.cpu()
    i, j = members(2 * freqs.numel(), interleaved)
    u, v = x[..., i].clone(), x[..., j].clone()
    size = torch.zeros_like(x)
    x[..., i], x[..., j] = u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()
    size[..., i] = size[..., j] = u.abs() + v.abs()
    return x, size


def close(got, want, size):
    """One rounding to the output's type (half a step), and fp32 arithmetic: cos and sin are off by 2^-22 (the angle's fraction of a turn
    rounded to fp32: pi 2^-24, sincospi: 2 steps), three roundings of 2^-24 of the products and their sum."""
    half_step = torch.finfo(got.dtype).eps / 2
    err = (got.double().cpu() - want).abs()
    assert (err <= half_step * want.abs() + 2.0 ** -20 * size).all(), float((err - half_step * want.abs()).max())


def randn(*shape, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(dtype).cuda()


def projections(layout, B, L, Hq, Hkv, d, dtype, fill=None):
    make = (lambda *s: randn(*s, dtype=dtype)) if fill is None else (lambda *s: torch.full(s, fill, dtype=dtype, device="cuda"))
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
        x = None
        return x, [make(B, h, L, d) for h in (Hq, Hkv, Hkv)]
    return x, [t.transpose(1, 2) for t in parts]


CASES = [
    # B, L, Hq, Hkv, d, rotary, interleaved, layout, dtype
    (1, 1, 1, 1, 64, 2, False, "dense", "bf16"),
    (1, 1, 32, 8, 128, 128, False, "fused", "bf16"),
    (2, 17, 5, 5, 64, 16, False, "per_head", "bf16"),
    (3, 33, 7, 1, 128, 128, True, "fused", "bf16"),
    (2, 31, 6, 3, 64, 38, False, "fused", "bf16"),
    (2, 31, 6, 3, 64, 38, True, "padded", "bf16"),
    (1, 130, 12, 4, 128, 126, False, "padded", "bf16"),
    (5, 2, 3, 1, 128, 96, True, "fused", "fp32"),
    (2, 65, 4, 2, 64, 64, False, "fused", "fp32"),
    (1, 257, 28, 4, 128, 20, False, "fused", "fp32"),
    (2, 9, 4, 4, 64, 36, True, "per_head", "fp32"),
    (1, 2049, 2, 1, 128, 64, False, "dense", "bf16"),
]


@pytest.mark.parametrize("B,L,Hq,Hkv,d,rotary,interleaved,layout,dtype", CASES)
@pytest.mark.parametrize("positions", ["index", "given", "documents"])
def test_forward_and_backward(sp, B, L, Hq, Hkv, d, rotary, interleaved, layout, dtype, positions):
    dt = DTYPES[dtype]
    freqs = sp.sepattn_rope_frequencies(rotary, 10000.0, device="cuda")
    pos, given, doc = torch.arange(L).expand(B, L), None, None
    g = torch.Generator().manual_seed(1)
    if positions == "given":
        pos = torch.randint(-(1 << 31), (1 << 31) - 1, (B, L), generator=g)
        pos[0, 0] = 4_000_000
        given = pos.to(torch.int32).cuda()
    elif positions == "documents":
        start = torch.where(torch.rand(B, L, generator=g) < 0.1, torch.arange(L), 0).cummax(1).values
        pos, doc = pos - start, start.to(torch.int32).cuda()
    x, src = projections(layout, B, L, Hq, Hkv, d, dt)
    before = [t.clone() for t in src]
    Q, K, V = sp.sepattn_rope(*src, freqs, positions=given, doc_start=doc, interleaved=interleaved)
    for got, t in zip((Q, K), src):
        assert got.is_contiguous() and got.shape == t.shape
        want, size = turned(t, pos[:, None], freqs, interleaved)
        close(got, want, size)
        assert torch.equal(got[..., rotary:], t[..., rotary:])
    assert V.is_contiguous() and torch.equal(V, src[2])
    assert all(torch.equal(a, b) for a, b in zip(before, src))

    # the gradient, into a buffer of the projections' layout whose other values stay
    grads = [randn(B, h, L, d, dtype=dt, seed=5 + i) for i, h in enumerate((Hq, Hkv, Hkv))]
    dx, out = projections(layout, B, L, Hq, Hkv, d, dt, fill=7.0)
    back = sp.sepattn_rope_backward(*grads, freqs, positions=given, doc_start=doc, interleaved=interleaved, out=out)
    for got, o, t in zip(back, out, grads):
        assert got is o
    for o, t in zip(out[:2], grads):
        want, size = turned(t, pos[:, None], freqs, interleaved, -1.0)
        close(o, want, size)
    assert torch.equal(out[2], grads[2])
    if layout == "padded":
        assert (dx[..., d:] == 7.0).all()
    # without `out`: views of one fused buffer
    free = sp.sepattn_rope_backward(*grads, freqs, positions=given, doc_start=doc, interleaved=interleaved)
    assert all(torch.equal(a, b) for a, b in zip(free, out))
    assert free[0].untyped_storage().data_ptr() == free[2].untyped_storage().data_ptr()
    assert free[0].transpose(1, 2).stride() == (L * (Hq + 2 * Hkv) * d, (Hq + 2 * Hkv) * d, d, 1) or B == 1


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [64, 22])
def test_gradient_against_differences(sp, interleaved, rotary):
    """The turn is linear: <dQ, (f(q + h e) - f(q - h e))> / 2h for directions e, and the adjoint identity, in fp32."""
    freqs = sp.sepattn_rope_frequencies(rotary, 10000.0, device="cuda")
    q, k = randn(1, 2, 5, 64, dtype=torch.float32), randn(1, 1, 5, 64, dtype=torch.float32, seed=1)
    dQ, dK = randn(1, 2, 5, 64, dtype=torch.float32, seed=2), randn(1, 1, 5, 64, dtype=torch.float32, seed=3)
    dq, dk, none = sp.sepattn_rope_backward(dQ, dK, None, freqs, interleaved=interleaved)
    assert none is None
    f = lambda a, b: sp.sepattn_rope(a, b, None, freqs, interleaved=interleaved)
    loss = lambda a, b: sum((x.double() * y.double()).sum().item() for x, y in zip(f(a, b)[:2], (dQ, dK)))
    h = 0.5  # any step: the function is linear; 640 terms of size about 1, each off by 2^-20 of it
    for seed in range(4):
        e = randn(1, 2, 5, 64, dtype=torch.float32, seed=10 + seed)
        slope = (loss(q + h * e, k) - loss(q - h * e, k)) / (2 * h)
        assert abs(slope - (dq.double() * e.double()).sum().item()) <= 640 * 4 * 2.0 ** -20
    assert abs(loss(q, k) - ((dq.double() * q.double()).sum() + (dk.double() * k.double()).sum()).item()) <= 960 * 4 * 2.0 ** -20


def test_in_place_broadcast_and_values_not_finite(sp):
    freqs = sp.sepattn_rope_frequencies(32, 10000.0, device="cuda")
    for interleaved in (False, True):
        q, k = randn(2, 4, 9, 64, dtype=torch.bfloat16), randn(2, 2, 9, 64, dtype=torch.bfloat16, seed=1)
        want = sp.sepattn_rope(q, k, None, freqs, interleaved=interleaved)
        a, b = q.clone(), k.clone()
        sp.sepattn_rope(a, b, None, freqs, interleaved=interleaved, out=(a, b, None))
        assert torch.equal(a, want[0]) and torch.equal(b, want[1])
        # one row of keys for all heads and sequences
        row = k[:1, :1].expand(2, 2, 9, 64)
        got = sp.sepattn_rope(q, row, row, freqs, interleaved=interleaved)
        assert torch.equal(got[1], sp.sepattn_rope(q, row.contiguous(), None, freqs, interleaved=interleaved)[1])
        assert torch.equal(got[2], row.contiguous())
        # dimensions that are not turned are copied whatever they hold, and reach nothing else
        q[0, 0, 0, 32:] = float("nan")
        q[0, 0, 1, 40] = float("inf")
        odd = sp.sepattn_rope(q, k, None, freqs, interleaved=interleaved)[0]
        assert torch.equal(odd[..., :32], want[0][..., :32])
        assert odd[0, 0, 0, 32:].isnan().all() and odd[0, 0, 1, 40].isinf() and odd[0, 0, 1, 41:].isfinite().all()


def test_frequencies_and_table(sp):
    n, d, base, factor, low, high, length = 513, 128, 500000.0, 8.0, 1.0, 4.0, 8192
    f = base ** (-2.0 * np.arange(d // 2) / d)
    turns = length * f / (2 * math.pi)
    keep = np.clip((turns - low) / (high - low), 0.0, 1.0)
    want = f * (keep + (1.0 - keep) / factor)
    got = sp.sepattn_rope_frequencies(d, base, factor, low, high, length, device="cuda")
    assert np.abs(got.cpu().numpy() / want - 1.0).max() < 1e-14
    assert (want < f).any() and (want == f).any() and ((want < f) & (want > f / factor)).any()
    table = sp.sepkv_rope_table_frequencies(n, got).cpu().double().numpy()
    angle = np.arange(n)[:, None] * want
    assert max(np.abs(table[:, 0] - np.cos(angle)).max(), np.abs(table[:, 1] - np.sin(angle)).max()) < 1.2e-7
    plain = sp.sepattn_rope_frequencies(d, base, device="cuda")
    assert torch.equal(sp.sepkv_rope_table(n, d, base, "cuda"), sp.sepkv_rope_table_frequencies(n, plain)) or \
        (sp.sepkv_rope_table(n, d, base, "cuda") - sp.sepkv_rope_table_frequencies(n, plain)).abs().max() < 1.2e-7


# ---- a token enters the cache --------------------------------------------------------------------
def cache(S, Hkv, d, a, s, w, c, dtype, seed=0):
    room = c - a - s
    Kc, Vc = randn(S, Hkv, c, d, dtype=dtype, seed=seed), randn(S, Hkv, c, d, dtype=dtype, seed=seed + 1)
    flags = torch.randint(0, 2, (S, room), generator=torch.Generator().manual_seed(seed)).to(torch.uint8).cuda()
    sizes = [[a, s // 2, 0, w - 1, 0, 0], [a, s, 3, w, max(s - 1, 0), room - 1], [max(a - 1, 0), 0, 0, 0, 0, 0], [a, 0, room - w, w, 0, 2]]
    return Kc, Vc, flags, torch.tensor([sizes[i % 4] for i in range(S)], dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("S,Hq,Hkv,d,rotary,interleaved,dtype", [
    (1, 32, 8, 128, 128, False, "bf16"), (6, 7, 1, 64, 22, False, "bf16"), (5, 3, 3, 64, 64, True, "fp32"), (4, 64, 64, 128, 50, True, "bf16"),
    (9, 40, 20, 128, 128, False, "fp32")])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_is_the_turn_and_then_the_append(sp, S, Hq, Hkv, d, rotary, interleaved, dtype, in_place):
    a, s, w, c = 3, 8, 5, 40
    dt = DTYPES[dtype]
    freqs = sp.sepattn_rope_frequencies(rotary, 10000.0, device="cuda")
    q, k, v = randn(S, Hq, d, dtype=dt), randn(S, Hkv, d, dtype=dt, seed=1), randn(S, Hkv, d, dtype=dt, seed=2)
    pos = torch.randint(0, 3_000_000, (S,), generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    sep = (torch.arange(S) % 2).to(torch.uint8).cuda()
    Kc, Vc, flags, sizes = cache(S, Hkv, d, a, s, w, c, dt)
    want = [t.clone() for t in (Kc, Vc, flags, sizes)]
    # the rows as [S, H, 1, d]: one token per sequence
    Q, K, _ = sp.sepattn_rope(q[:, :, None], k[:, :, None], None, freqs, positions=pos[:, None], interleaved=interleaved)
    exact, size = turned(q, pos[:, None], freqs, interleaved)
    sp.sepkv_append(K[:, :, 0].contiguous(), v, sep, *want, Hq, a, s, w)
    q0 = q.clone()
    got = sp.sepkv_append_rope(q, k, v, sep, pos, freqs, Kc, Vc, flags, sizes, a, s, w, interleaved=interleaved, out=q if in_place else None)
    assert (got is q) == in_place and (in_place or torch.equal(q, q0))
    assert torch.equal(got, Q[:, :, 0])
    close(got, exact, size)
    for x, y in zip((Kc, Vc, flags, sizes), want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("S,Hkv,d,a,s,w,c,dtype", [
    (1, 1, 64, 0, 0, 1, 2, "bf16"), (3, 5, 128, 4, 16, 8, 70, "bf16"), (2, 8, 64, 3, 9, 20, 333, "fp32"), (4, 2, 128, 0, 0, 1, 150, "fp32"),
    (5, 20, 128, 2, 0, 3, 30, "bf16")])
def test_keys_of_a_cache_are_turned_by_rank(sp, S, Hkv, d, a, s, w, c, dtype):
    room = c - a - s
    rng = np.random.default_rng(0)
    sizes = []
    for i in range(S):
        n = int(rng.integers(0, room + 1)) if i else room
        sizes.append([int(rng.integers(0, a + 1)), int(rng.integers(0, s + 1)), n - min(n, w), min(n, w), int(rng.integers(0, max(s, 1))), int(rng.integers(0, room))])
    if S > 1:
        sizes[1] = [0, 0, 0, 0, 0, 0]
    K = randn(S, Hkv, c, d, dtype=DTYPES[dtype])
    sz = torch.tensor(sizes, dtype=torch.int32, device="cuda")
    table = sp.sepkv_rope_table(c + 3, d, 10000.0, "cuda")
    freqs = sp.sepattn_rope_frequencies(d, 10000.0)
    out = torch.full_like(K, 7.0)
    kept = K.clone()
    assert sp.sepkv_rope_cache(K, sz, table, a, s, w, out=out) is out and torch.equal(K, kept)
    for i, row in enumerate(sizes):
        slots = list(range(row[0])) + [a + (row[4] + j) % s for j in range(row[1])] + [a + s + (row[5] + j) % room for j in range(row[2] + row[3])]
        if slots:
            want, size = turned(K[i][:, slots], torch.arange(len(slots))[None], freqs, False)
            close(out[i][:, slots], want, size)
        rest = [j for j in range(c) if j not in slots]
        assert (out[i][:, rest] == 7.0).all()
        kept[i][:, slots] = out[i][:, slots]
    assert sp.sepkv_rope_cache(K, sz, table, a, s, w) is K and torch.equal(K, kept)  # in place


def test_training_step_through_the_turn(sp):
    """Projections -> turn -> attention -> back, as a training step has them (fp32), against autograd of the definition in 64 bits."""
    B, L, Hq, Hkv, d, a, n, rotary = 2, 150, 4, 2, 64, 3, 24, 32
    freqs = sp.sepattn_rope_frequencies(rotary, 10000.0, device="cuda")
    x = randn(B, L, Hq + 2 * Hkv, d, dtype=torch.float32).mul_(0.5)
    src = [t.transpose(1, 2) for t in x.split([Hq, Hkv, Hkv], dim=2)]
    tok = torch.randint(0, 9, (B, L), generator=torch.Generator().manual_seed(4)).to(torch.int32).cuda()
    is_sep, idx, cnt, pre = sp.sepattn_mark_compact(tok, [1])
    scale = 1.0 / math.sqrt(d)
    Q, K, V = sp.sepattn_rope(*src, freqs)
    O, LSE = sp.sepattn_forward(Q, K, V, idx, cnt, pre, a, n, scale)
    dO = randn(B, Hq, L, d, dtype=torch.float32, seed=9)
    dx = torch.empty_like(x)
    sp.sepattn_rope_backward(*sp.sepattn_backward(Q, K, V, O, LSE, dO, idx, cnt, pre, a, n, scale), freqs,
                             out=[t.transpose(1, 2) for t in dx.split([Hq, Hkv, Hkv], dim=2)])

    y = x.double().cpu().requires_grad_(True)
    q, k, v = (t.transpose(1, 2) for t in y.split([Hq, Hkv, Hkv], dim=2))
    angle = torch.arange(L).double()[:, None] * freqs.cpu()

    def turn(t):
        u, w = t[..., : rotary // 2], t[..., rotary // 2: rotary]
        return torch.cat([u * angle.cos() - w * angle.sin(), w * angle.cos() + u * angle.sin(), t[..., rotary:]], -1)

    k, v = (t.repeat_interleave(Hq // Hkv, 1) for t in (turn(k), v))
    i, j = torch.arange(L)[:, None], torch.arange(L)[None]
    seen = (j <= i) & ((j < a) | (i - j < n) | (is_sep.cpu().bool()[:, None, None, :].expand(B, 1, L, L)))
    score = (turn(q) @ k.transpose(-1, -2) * scale).masked_fill(~seen, float("-inf"))
    out = torch.softmax(score, -1) @ v
    out.backward(dO.double().cpu())
    assert (O.double().cpu() - out).abs().max() < 1e-4 and (dx.double().cpu() - y.grad).abs().max() < 1e-4  # the fp32 path's tolerance


def test_step_in_a_graph(sp):
    """A captured step, replayed on new tokens between eager calls, gives what eager calls give."""
    S, Hq, Hkv, d, a, s, w, c = 3, 8, 2, 128, 2, 8, 16, 64
    freqs = sp.sepattn_rope_frequencies(d, 10000.0, device="cuda")
    state = cache(S, Hkv, d, a, s, w, c, torch.bfloat16)
    other = [t.clone() for t in state]
    q, k, v = (torch.empty(S, h, d, dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    pos, sep, out = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    call = lambda st: sp.sepkv_append_rope(q, k, v, sep, pos, freqs, *st, a, s, w, out=out)
    scratch = [t.clone() for t in state]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call(scratch)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(state)
    for step in range(4):
        for t, h in ((q, Hq), (k, Hkv), (v, Hkv)):
            t.copy_(randn(S, h, d, dtype=torch.bfloat16, seed=20 + 3 * step + h))
        pos.fill_(1000 + step)
        graph.replay()
        replayed = out.clone()
        call(other)
        torch.cuda.synchronize()
        assert torch.equal(replayed, out)
        for x, y in zip(state, other):
            assert torch.equal(x, y)


def test_rows_far_apart(sp):
    """Strides whose offsets pass 2^32 bytes, on both sides."""
    far = 2 ** 31 + 64
    x, y = (torch.empty(far + 2 ** 30 + 4096, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    view = lambda t: t.as_strided((2, 2, 5, 64), (far, 2 ** 30, 192, 1))
    q = randn(2, 2, 5, 64, dtype=torch.bfloat16)
    freqs = sp.sepattn_rope_frequencies(64, 10000.0, device="cuda")
    view(x).copy_(q)
    for fn in (sp.sepattn_rope, sp.sepattn_rope_backward):
        want = fn(q, q, q, freqs)
        y.fill_(7.0)
        k, v = torch.empty_like(q), torch.empty_like(q)
        fn(view(x), q, q, freqs, out=(view(y), k, v))
        assert torch.equal(view(y), want[0]) and torch.equal(k, want[1]) and torch.equal(v, q)
        assert int((y == 7.0).sum()) == y.numel() - q.numel()


def test_sizes_past_32_bits_are_refused(sp):
    freqs = sp.sepattn_rope_frequencies(64, 10000.0, device="cuda")
    q = torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16, device="cuda").expand(1, 1, 2 ** 32 + 5, 64)
    with pytest.raises(AssertionError):
        sp.sepattn_rope(q, q, None, freqs, out=(q, q, None))


def test_two_streams(sp):
    freqs = sp.sepattn_rope_frequencies(128, 10000.0, device="cuda")
    src = [[randn(1, h, 777, 128, dtype=torch.bfloat16, seed=h + i) for h in (8, 2, 2)] for i in (0, 1)]
    want = [sp.sepattn_rope(*x, freqs) for x in src]
    streams = [torch.cuda.Stream() for _ in src]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for x, st in zip(src, streams):
            with torch.cuda.stream(st):
                got.append(sp.sepattn_rope(*x, freqs))
    torch.cuda.synchronize()
    for i, out in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(out, want[i % 2]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_training_step_in_a_graph(sp, dtype):
    """Turn, attention and their gradients captured once, replayed on new inputs between eager steps: every replay gives the eager bits."""
    B, L, Hq, Hkv, d, a, n = 2, 200, 4, 2, 64, 2, 32
    freqs = sp.sepattn_rope_frequencies(d, 10000.0, device="cuda")
    x = torch.empty(B, L, Hq + 2 * Hkv, d, dtype=DTYPES[dtype], device="cuda")
    dO = torch.empty(B, Hq, L, d, dtype=DTYPES[dtype], device="cuda")
    tok = torch.randint(0, 9, (B, L), generator=torch.Generator().manual_seed(4)).to(torch.int32).cuda()
    _, idx, cnt, pre = sp.sepattn_mark_compact(tok, [1])
    scale = 1.0 / math.sqrt(d)
    split = lambda t: [u.transpose(1, 2) for u in t.split([Hq, Hkv, Hkv], dim=2)]

    def step():
        Q, K, V = sp.sepattn_rope(*split(x), freqs)
        O, LSE = sp.sepattn_forward(Q, K, V, idx, cnt, pre, a, n, scale)
        grads = sp.sepattn_backward(Q, K, V, O, LSE, dO, idx, cnt, pre, a, n, scale)
        return (O, *sp.sepattn_rope_backward(*grads, freqs))

    def fill(seed):
        x.copy_(randn(*x.shape, dtype=x.dtype, seed=seed))
        dO.copy_(randn(*dO.shape, dtype=x.dtype, seed=seed + 1))

    fill(0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        fill(10 + 2 * i)
        graph.replay()
        replayed = [t.clone() for t in captured]
        eager = step()
        torch.cuda.synchronize()
        for r, e in zip(replayed, eager):
            # fp32 sums of the gradient's slices: a captured call has two launches, whose slices are cut otherwise
            assert torch.equal(r, e) if dtype == "bf16" else (r - e).abs().max() < 1e-4
