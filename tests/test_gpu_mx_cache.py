"""The four-block cache in 4 bits: rounding, hand-over, tokens, compression and values, bit for bit.  Needs an MI355X."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2412_12094_amd as sp_

    sp_.load()
    return sp_


def randn(*shape, dtype, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def rounded(x):
    """codes [..., d] and scale bytes [..., d/32] (uint8, numpy) of rows x, from the definition: integers and exact comparisons in float64."""
    x = x.detach().double().cpu().numpy()
    y = x.reshape(*x.shape[:-1], -1, 32)
    big = np.abs(y).max(-1)
    bad = ~np.isfinite(y).all(-1)
    m, e = np.frexp(np.where(bad, 1.0, big))  # big = m 2^e, 1/2 <= m < 1
    e = np.where(m > 0.875, e + 1, e) - 3
    e = np.where(big > 0, np.clip(e, -125, 125), -125)
    size = np.abs(np.where(bad[..., None], 0.0, y)) / np.exp2(e.astype(np.float64))[..., None]
    code = np.zeros(y.shape, np.uint8)
    for i in range(1, 8):  # past the middle between two neighbours, or on it and the upper one is even
        middle = (LEVELS[i - 1] + LEVELS[i]) / 2
        code += (size > middle) | ((size == middle) & (i % 2 == 0))
    code |= np.where(np.signbit(y) & ~bad[..., None], 8, 0).astype(np.uint8)
    return code.reshape(x.shape), np.where(bad, 255, e + 127).astype(np.uint8)


def packed(code):
    return torch.from_numpy(code[..., 0::2] | (code[..., 1::2] << 4)).cuda()


def values(Kc, Ks):
    """float64 values of packed rows."""
    c, s = Kc.cpu().numpy(), Ks.cpu().numpy().astype(np.float64)
    code = np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], -1)
    v = np.array(LEVELS + tuple(-x for x in LEVELS))[code]
    return (v.reshape(*v.shape[:-1], -1, 32) * np.where(s == 255, np.nan, np.exp2(s - 127))[..., None]).reshape(v.shape)


def interesting(n, d, dtype):
    """Rows with ties, borders of the scale, zeros, all sizes that the type has, infinities and NaN."""
    g = torch.Generator().manual_seed(0)
    x = torch.randn(n, d, generator=g, dtype=torch.float64)
    levels = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 4.0, 0.5, 7.5], dtype=torch.float64)
    pick = lambda *s: levels[torch.randint(0, 12, s, generator=g)] * (1 - 2 * torch.randint(0, 2, s, generator=g))
    x[0::4] = pick(len(x[0::4]), d)
    x[1::4] = pick(len(x[1::4]), d) * (1 + 2.0 ** -7 * torch.randint(-1, 2, (len(x[1::4]), d), generator=g))
    exponent = torch.randint(-126, 126, (n, d // 32, 1), generator=g).double()
    exponent[: n // 2] = torch.randint(-3, 4, (n // 2, d // 32, 1), generator=g).double()
    x = (x.unflatten(-1, (-1, 32)) * torch.exp2(exponent)).flatten(-2)
    big = torch.finfo(dtype).max
    x = x.clamp(-big, big).to(dtype)
    x[2, :32] = 0.0
    x[3, :32], x[3, 5] = 0.0, -0.0
    x[5, 32:64], x[5, 40] = 0.0, 2.0 ** -133
    x[6, :32] = big
    x[7, 3], x[9, 33], x[10, 0] = float("inf"), float("nan"), float("-inf")
    return x


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_rounding(sp, d, dtype):
    """A prompt kept whole: codes and scales as defined, and the values read back."""
    dt, L = DTYPES[dtype], 601
    K, V = interesting(2 * L, d, dt).view(1, 2, L, d).cuda(), interesting(2 * L, d, dt).flip(0).view(1, 2, L, d).contiguous().cuda()
    none = torch.zeros((1, L), dtype=torch.uint8, device="cuda")
    idx, _, pre = sp.sepattn_compact_indices(none)
    Kc, Ks, Vc, Vs, flags, sizes = sp.sepkv_fill_from_prefill_mx(K, V, none, idx, pre, 4, 0, 0, 1, L, L)
    assert sizes.tolist() == [[0, 0, L - 1, 1, 0, 0]]
    for x, c, s in ((K, Kc, Ks), (V, Vc, Vs)):
        code, byte = rounded(x)
        bad = np.repeat(byte == 255, 32, -1)
        assert np.array_equal(s.cpu().numpy(), byte)
        assert torch.equal(c, packed(np.where(bad, 0, code)))
        v = values(c, s)
        err, x64 = np.abs(v - x.double().cpu().numpy()), x.double().cpu().numpy()
        scale = np.repeat(np.exp2(byte.astype(np.float64) - 127), 32, -1)
        size = np.abs(np.where(bad, 0, x64)) / scale
        # half a step: 1/4, 1/2 from 2 on, 1 from 4 to 7; beyond 7 only at the largest scale
        assert (err <= scale * np.where(size > 7, size - 6, np.where(size >= 4, 1, np.where(size >= 2, 0.5, 0.25))))[~bad].all()
        assert ((size <= 7) | (scale == 2.0 ** 125))[~bad].all()
    back = sp.sepkv_expand_mx(Kc, Ks, Vc, Vs, sizes, 0, 0, 1, dtype=dt)
    for got, c, s in zip(back, (Kc, Vc), (Ks, Vs)):
        assert got.dtype == dt and np.array_equal(got.double().cpu().numpy(), values(c, s), equal_nan=True)


def hand_over(sp, S, Hkv, L, d, dtype, blocks, nw, density, seed=0):
    a, s, w, c = blocks
    K, V = randn(S, Hkv, L, d, dtype=dtype, seed=seed), randn(S, Hkv, L, d, dtype=dtype, seed=seed + 1)
    sep = (torch.rand(S, L, generator=torch.Generator().manual_seed(seed)) < density).to(torch.uint8).cuda()
    idx, _, pre = sp.sepattn_compact_indices(sep)
    return K, V, sep, idx, pre


FILL = [
    # S, Hkv, L, d, dtype, (a, s, w, c), nw, density
    (1, 1, 1, 64, "bf16", (0, 0, 1, 2), 1, 0.5),
    (1, 1, 1, 128, "bf16", (4, 2, 1, 9), 0, 0.5),
    (2, 3, 200, 128, "bf16", (4, 16, 20, 100), 50, 0.2),
    (3, 2, 333, 64, "fp32", (3, 100, 7, 180), 70, 0.4),
    (2, 8, 1000, 128, "fp32", (4, 0, 30, 300), 250, 0.3),
    (2, 5, 700, 64, "bf16", (1, 500, 30, 700), 10, 0.1),
    (1, 2, 50, 128, "bf16", (60, 8, 8, 100), 0, 0.1),
    (5, 4, 260, 128, "bf16", (0, 7, 16, 280), 256, 0.9),
]


@pytest.mark.parametrize("S,Hkv,L,d,dtype,blocks,nw,density", FILL)
def test_hand_over_and_compression(sp, S, Hkv, L, d, dtype, blocks, nw, density):
    """The same rows in the same slots as the plain cache's calls keep, rounded; compressed twice, with tokens between."""
    a, s, w, c = blocks
    dt = DTYPES[dtype]
    args = hand_over(sp, S, Hkv, L, d, dt, blocks, nw, density)
    Kp, Vp, flags_p, sizes_p = sp.sepkv_fill_from_prefill(*args, Hkv, a, s, w, c, nw)
    *mx, flags, sizes = sp.sepkv_fill_from_prefill_mx(*args, Hkv, a, s, w, c, nw)

    def same():
        assert torch.equal(flags, flags_p) and torch.equal(sizes, sizes_p)
        K, V = sp.sepkv_expand_mx(*mx, sizes, a, s, w, dtype=dt)
        for got, plain in ((K, Kp), (V, Vp)):
            code, byte = rounded(plain)
            want = values(packed(code), torch.from_numpy(byte))
            for i, row in enumerate(sizes.tolist()):
                room = c - a - s
                at = list(range(row[0])) + [a + (row[4] + j) % s for j in range(row[1])] + [a + s + (row[5] + j) % room for j in range(row[2] + row[3])]
                rest = [j for j in range(c) if j not in set(at)]
                assert np.array_equal(got[i][:, at].double().cpu().numpy(), want[i][:, at])
                assert (got[i][:, rest] == 0).all()

    same()
    # fresh buffers hold zeros beyond the sizes; a caller's keep what they held there
    used = (sp.sepkv_expand_mx(*mx, sizes, a, s, w, dtype=torch.float32)[0] != 0).any(-1)
    assert (mx[0][~used].view(-1) % 128 % 8 == 0).all()
    own = [torch.full_like(t, 0xA5) for t in (*mx, flags)] + [torch.zeros_like(sizes)]
    got = sp.sepkv_fill_from_prefill_mx(*args, Hkv, a, s, w, c, nw, out=own)
    assert all(x is y for x, y in zip(got, own)) and torch.equal(own[5], sizes)
    inside = torch.zeros(S, c, dtype=torch.bool)
    for i, row in enumerate(sizes.tolist()):
        inside[i, list(range(row[0])) + list(range(a, a + row[1])) + list(range(a + s, a + s + row[2] + row[3]))] = True
    for x, y in zip(own[:4], mx):
        x, y, keep = x.transpose(1, 2), y.transpose(1, 2), inside.cuda()
        assert torch.equal(x[keep], y[keep]) and (x[~keep] == 0xA5).all()
    for step in range(2):
        sp.sepkv_evict_window(Kp, Vp, flags_p, sizes_p, Hkv, a, s, w)
        sp.sepkv_evict_window_mx(*mx, flags, sizes, Hkv, a, s, w)
        same()
        for t in range(w + 5):  # more than the local window holds; a full window keeps its rows
            k, v = randn(S, Hkv, d, dtype=dt, seed=100 + t), randn(S, Hkv, d, dtype=dt, seed=200 + t)
            sep = torch.full((S,), t % 3 == 0, dtype=torch.uint8, device="cuda")
            sp.sepkv_append(k, v, sep, Kp, Vp, flags_p, sizes_p, Hkv, a, s, w)
            sp.sepkv_append_mx(k, v, sep, *mx, flags, sizes, Hkv, a, s, w)
        same()


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype,d,rotary,interleaved", [("bf16", 128, 128, False), ("bf16", 64, 16, False), ("bf16", 128, 38, True), ("bf16", 128, 38, False),
                                                        ("fp32", 128, 20, False), ("fp32", 64, 64, True), ("fp32", 128, 128, False)])
@pytest.mark.parametrize("S,Hq,Hkv", [(1, 32, 8), (5, 7, 7), (3, 70, 35)])
def test_turned_token(sp, norm, dtype, d, rotary, interleaved, S, Hq, Hkv):
    """What the separate calls would leave: the turned query and key in the rows' type, then the append."""
    dt, a, s, w, c = DTYPES[dtype], 2, 5, 4, 21
    freqs = sp.sepattn_rope_frequencies(rotary, 10000.0, device="cuda")
    weights = [(1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(i))).to(dt).cuda() for i in range(2)]
    q, k, v = randn(S, Hq, d, dtype=dt), randn(S, Hkv, d, dtype=dt, seed=1), randn(S, Hkv, d, dtype=dt, seed=2)
    pos = torch.arange(S, dtype=torch.int32, device="cuda") * 1000003
    rows = [[0, 0, 0, 0, 0, 0], [2, 3, 2, 4, 1, 7], [2, 5, 10, 4, 0, 3], [1, 0, 0, 0, 0, 0], [2, 0, 0, 3, 0, 13]]  # empty, in use, full, ...
    sep = torch.ones(S, dtype=torch.uint8, device="cuda")

    def cache():
        g = torch.Generator().manual_seed(3)
        u8 = lambda *shape: torch.randint(0, 255, shape, generator=g, dtype=torch.uint8).cuda()
        return [u8(S, Hkv, c, d // 2), u8(S, Hkv, c, d // 32), u8(S, Hkv, c, d // 2), u8(S, Hkv, c, d // 32), u8(S, c - a - s),
                torch.tensor([rows[i % 5] for i in range(S)], dtype=torch.int32, device="cuda")]

    got, want = cache(), cache()
    kw = dict(positions=pos[:, None].contiguous(), interleaved=interleaved)
    if norm:
        out = sp.sepkv_append_norm_rope_mx(q, k, v, sep, pos, *weights, freqs, 1e-6, *got, a, s, w, interleaved=interleaved)
        tq, tk, _ = sp.sepattn_norm_rope(q[:, :, None], k[:, :, None], None, *weights, freqs, 1e-6, **kw)
    else:
        out = sp.sepkv_append_rope_mx(q, k, v, sep, pos, freqs, *got, a, s, w, interleaved=interleaved)
        tq, tk, _ = sp.sepattn_rope(q[:, :, None], k[:, :, None], None, freqs, **kw)
    sp.sepkv_append_mx(tk[:, :, 0].contiguous(), v, sep, *want, Hq, a, s, w)
    assert torch.equal(out, tq[:, :, 0]) and all(torch.equal(x, y) for x, y in zip(got, want))
    # and the append writes the rounded rows: into the first empty slot of sequence 0
    for c_, s_, x in ((want[0], want[1], tk[0, :, 0]), (want[2], want[3], v[0])):
        code, byte = rounded(x)
        assert torch.equal(c_[0][:, 0], packed(code)) and np.array_equal(s_[0][:, 0].cpu().numpy(), byte)


def test_normed_token_that_is_not_turned(sp):
    S, H, d, dt = 2, 3, 64, torch.bfloat16
    q, k, v = (randn(S, H, d, dtype=dt, seed=i) for i in range(3))
    cache = lambda: [torch.zeros(S, H, 4, n, dtype=torch.uint8, device="cuda") for n in (32, 2, 32, 2)] + [
        torch.zeros(S, 4, dtype=torch.uint8, device="cuda"), torch.zeros(S, 6, dtype=torch.int32, device="cuda")]
    sep, got, want = torch.zeros(S, dtype=torch.uint8, device="cuda"), cache(), cache()
    out = sp.sepkv_append_norm_rope_mx(q, k, v, sep, None, None, None, None, 1e-6, *got, 0, 0, 1)
    tq, tk, _ = sp.sepattn_norm_rope(q[:, :, None], k[:, :, None], None, None, None, None, 1e-6)
    sp.sepkv_append_mx(tk[:, :, 0].contiguous(), v, sep, *want, H, 0, 0, 1)
    assert torch.equal(out, tq[:, :, 0]) and all(torch.equal(x, y) for x, y in zip(got, want)) and got[5][:, 3].tolist() == [1, 1]


def test_sizes_outside_their_ranges(sp):
    """Clamped on the device, as in the plain calls: nothing is read or written out of bounds, the neighbours stay."""
    S, H, d, a, s, w, c = 3, 2, 64, 2, 4, 3, 16
    big = 1 << 30
    sizes = torch.tensor([[big, big, big, big, big, big], [-5, -5, -5, -5, -5, -5], [2, 4, 3, 3, 1, 2]], dtype=torch.int32, device="cuda")
    mx = [torch.randint(1, 250, (S + 2, H, c, n), dtype=torch.uint8, generator=torch.Generator().manual_seed(n)).cuda() for n in (32, 2, 32, 2)]
    before = [t.clone() for t in mx]
    inner = [t[1:-1] for t in mx]
    flags = torch.ones(S, c - a - s, dtype=torch.uint8, device="cuda")
    sp.sepkv_expand_mx(*inner, sizes, a, s, w)
    sp.sepkv_evict_window_mx(*inner, flags, sizes.clone(), H, a, s, w)
    row = randn(S, H, d, dtype=torch.bfloat16)
    sp.sepkv_append_mx(row, row, flags[:, 0].contiguous(), *inner, flags, sizes.clone(), H, a, s, w)
    torch.cuda.synchronize()
    for t, b in zip(mx, before):
        assert torch.equal(t[0], b[0]) and torch.equal(t[-1], b[-1])
