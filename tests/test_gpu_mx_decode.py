"""Decode over a cache in 4 bits against softmax attention in 64 bits.  Needs an MI355X."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BASE = 10000.0
LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], dtype=torch.float64)


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2412_12094_amd as sp_

    sp_.load()
    return sp_


def values(codes, scales):
    """float64 values of packed rows."""
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    s = scales.double()
    s = torch.where(s == 255, float("nan"), torch.exp2(s - 127))
    return (LEVELS.to(codes.device)[code].unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def slots_of(row, a, s, c):
    room = c - a - s
    return list(range(row[0])) + [a + (row[4] + j) % s for j in range(row[1])] + [a + s + (row[5] + j) % room for j in range(row[2] + row[3])]


def sizes_of(n, rng, a, s, w, c):
    """A row of sizes with n entries: the window first, then separators, then initial entries are what is missing; random ring heads."""
    room = c - a - s
    init = min(n, a)
    sep = min(n - init, int(rng.integers(0, s + 1))) if s else 0
    win = n - init - sep
    if win > room:
        sep, win = sep + win - room, room
    assert 0 <= sep <= s and 0 <= win <= room
    local = min(win, w)
    return [init, sep, win - local, local, int(rng.integers(0, max(s, 1))), int(rng.integers(0, room))]


def turn(x, pos):
    h = x.shape[-1] // 2
    f = BASE ** (-torch.arange(h, dtype=torch.float64, device=pos.device) / h)
    angle = pos.double()[..., None] * f
    u, v = x[..., :h], x[..., h:]
    return torch.cat([u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()], -1)


class Case:
    def __init__(self, S, Hq, Hkv, d, dtype, blocks, entries, seed=0, spread=2):
        self.a, self.s, self.w, self.c = blocks
        self.S, self.Hq, self.Hkv, self.d, self.dt = S, Hq, Hkv, d, DTYPES[dtype]
        rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        self.sizes = [sizes_of(entries[i % len(entries)], rng, *blocks) for i in range(S)]
        self.q = torch.randn(S, Hq, d, generator=g).to(self.dt).cuda()
        # all codes; scales around 1/4 .. 1/2 so that values are of order one; a slot without an entry is NaN: nothing may read one
        self.cache = []
        for _ in range(2):
            codes = torch.randint(0, 256, (S, Hkv, self.c, d // 2), generator=g, dtype=torch.uint8)
            scales = torch.randint(126 - spread, 126 + 1, (S, Hkv, self.c, d // 32), generator=g, dtype=torch.uint8)
            for i, row in enumerate(self.sizes):
                used = set(slots_of(row, self.a, self.s, self.c))
                scales[i][:, [j for j in range(self.c) if j not in used]] = 255
            self.cache += [codes.cuda(), scales.cuda()]
        self.scale = 1.0 / math.sqrt(d)
        self.sz = torch.tensor(self.sizes, dtype=torch.int32, device="cuda")

    def run(self, sp, rope, **kw):
        if not rope:
            return sp.sepattn_decode_mx(self.q, *self.cache, self.sz, self.a, self.s, self.w, self.scale, **kw)
        table = sp.sepkv_rope_table(self.c, self.d, BASE, "cuda")
        return sp.sepattn_decode_rope_mx(self.q, *self.cache, self.sz, table, self.a, self.s, self.w, self.scale, **kw)

    def want(self, rope, where="cpu"):
        """out, lse, mean of |V| under the weights, largest sum of the magnitudes in a score; in float64."""
        out, lse, size, reach = (torch.zeros(self.S, self.Hq, self.d, dtype=torch.float64), torch.full((self.S, self.Hq), float("-inf"), dtype=torch.float64),
                                 torch.zeros(self.S, self.Hq, self.d, dtype=torch.float64), torch.zeros(self.S, self.Hq, dtype=torch.float64))
        Kc, Ks, Vc, Vs = self.cache
        for i in range(self.S):
            at = slots_of(self.sizes[i], self.a, self.s, self.c)
            if not at:
                continue
            K, V = values(Kc[i][:, at].to(where), Ks[i][:, at].to(where)), values(Vc[i][:, at].to(where), Vs[i][:, at].to(where))
            q = self.q[i].to(where).double()
            both = K.abs()
            if rope:
                h = self.d // 2
                both = (both[..., :h] + both[..., h:]).repeat(1, 1, 2)  # what a turned value is made of
                # (a rotation of both is one by the difference)
                K = turn(K, (torch.arange(len(at), device=where) - (len(at) - 1))[None])
            K, V, both = (t.repeat_interleave(self.Hq // self.Hkv, 0) for t in (K, V, both))
            x = (K @ q[..., None])[..., 0] * self.scale
            p = torch.softmax(x, -1)
            out[i], size[i] = (p[:, None] @ V)[:, 0], (p[:, None] @ V.abs())[:, 0]
            lse[i], reach[i] = torch.logsumexp(x, -1), (both @ q.abs()[..., None])[..., 0].amax(-1) * self.scale
        return out, lse, size, reach

    def check(self, out, lse, rope, want=None):
        """A score: d products of exact operands added in fp32 (each sum off by 2^-24 of what it holds, at most d of them), then scaled (2^-21); with positions
        cos and sin, formed from two table rows, and the turn: 2^-20; in bf16 the turned key as two numbers, cut at 2^-7 and rounded at 2^-9 of
        that.  lse: the score's error, the sum's (2^-20) and the logarithm's.  An output: its rounding; the weights (two numbers: 2^-16; three: 2^-24); the
        scores' errors twice (weight and sum); sums and exponentials in fp32 (2^-18).  Below 2^-126 steps are fixed: 2^-133 in bf16, of which a rounding is
        off by half; 2^-149 in fp32, where the sums of at most 2^14 entries with three products each are off by less than 2^16 halves of it: 2^-134 too."""
        ref, ref_lse, size, reach = want or self.want(rope)
        bf16 = self.dt == torch.bfloat16
        score = reach * (self.d * 2.0 ** -24 + 2.0 ** -21 + (2.0 ** -20 + (2.0 ** -16 if bf16 else 0.0) if rope else 0.0))
        none = torch.isinf(ref_lse)
        got = lse.double().cpu()
        assert torch.equal(torch.isinf(got) & (got < 0), none)
        err = (got - ref_lse).abs()[~none]
        assert (err <= (score + 2.0 ** -20 + 2.0 ** -22 * ref_lse.abs())[~none]).all(), float(err.max())
        half = torch.finfo(self.dt).eps / 2
        fixed = 2.0 ** -134
        err = (out.double().cpu() - ref).abs()
        assert (err <= fixed + half * ref.abs() + ((2.0 ** -16 if bf16 else 2.0 ** -24) + 2.0 * score[..., None] + 2.0 ** -18) * size).all(), float(err.max())
        assert (out[none.cuda()] == 0).all()


BARE = (0, 0, 1, 70)
SMALL = (3, 8, 6, 40)
STREAM = (4, 100, 30, 300)
CASES = {
    # S, Hq, Hkv, d, blocks, entries
    "one entry": (1, 1, 1, 64, BARE, [1]),
    "one head of 128": (1, 1, 1, 128, BARE, [70]),
    "borders of a block": (7, 4, 2, 128, BARE, [31, 32, 33, 63, 64, 65, 0]),
    "borders of a block, 64": (7, 4, 4, 64, BARE, [31, 32, 33, 63, 64, 65, 0]),
    "small": (8, 32, 8, 128, SMALL, [0, 1, 2, 17, 39, 40]),
    "capacity of two": (2, 8, 8, 64, (0, 0, 1, 2), [2, 1]),
    "stream": (3, 28, 4, 128, STREAM, [300, 211, 7]),
    "stream, 64": (5, 12, 12, 64, STREAM, [300, 150, 33, 0]),
    "sixteen heads": (2, 16, 1, 128, STREAM, [300, 90]),
    "seventeen heads": (2, 17, 1, 128, STREAM, [300, 90]),
    "forty heads": (2, 40, 1, 64, STREAM, [255, 290]),
    "many sequences": (70, 8, 2, 128, SMALL, [40, 13, 0, 27, 1]),
    "long": (1, 4, 2, 128, (4, 2000, 300, 5000), [4999]),
    "long, 64": (2, 8, 8, 64, (0, 0, 1, 9000), [9000, 4321]),
    "full chip": (20, 32, 32, 64, STREAM, [300, 201]),
}


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", CASES)
def test_decode(sp, name, dtype, rope):
    S, Hq, Hkv, d, blocks, entries = CASES[name]
    x = Case(S, Hq, Hkv, d, dtype, blocks, entries, seed=len(name))
    out, lse = x.run(sp, rope)
    x.check(out, lse, rope)
    # outputs of the caller's, no lse, a workspace that holds anything and is one byte as large as it has to be; the same bits
    need = sp.sepattn_decode_mx_workspace_bytes(x.q, x.cache[0], x.a, x.s, x.w)
    ws, o = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda"), torch.full_like(out, 9.0)
    got = x.run(sp, rope, out=(o, None), ws=ws)
    assert got[0] is o and got[1] is None and torch.equal(o, out)
    with pytest.raises(sp.SepattnError):
        x.run(sp, rope, ws=ws[: need - 1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_random_shapes(sp, dtype):
    rng = np.random.default_rng(11)
    for case in range(12):
        Hkv, G, d = int(rng.integers(1, 9)), int(rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 20])), int(rng.choice([64, 128]))
        a, s, w = int(rng.integers(0, 6)), int(rng.integers(0, 200)), int(rng.integers(1, 60))
        c = a + s + w + int(rng.integers(1, 900))
        S = int(rng.integers(1, 9))
        x = Case(S, G * Hkv, Hkv, d, dtype, (a, s, w, c), [int(n) for n in rng.integers(0, c + 1, 4)], seed=case, spread=6)
        for rope in (False, True):
            print("case", case, S, G, Hkv, d, (a, s, w, c), rope, flush=True)
            x.check(*x.run(sp, rope), rope)


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128)])
def test_scores_far_apart(sp, dtype, d, rope):
    """Large queries: scores in the hundreds, the largest at the end, in the middle, everywhere; the maximum is raised again and again."""
    x = Case(3, 8, 2, d, dtype, STREAM, [300, 299, 64], seed=5)
    x.q *= 30.0
    x.check(*x.run(sp, rope), rope)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_extreme_scales(sp, dtype):
    """Blocks far out in the scales' range: values up to 6 2^100 (V; unnormalised sums of them fit fp32) and down to 2^-126 (K, V)."""
    x = Case(2, 4, 2, 64, dtype, BARE, [70, 33], seed=1)
    small, large = x.cache[1], x.cache[3]
    small[small != 255] = 2
    large[..., 0][large[..., 0] != 255] = 227
    large[..., 1][large[..., 1] != 255] = 2
    x.check(*x.run(sp, False), False)


def test_not_finite(sp):
    """A NaN in a query, in a key and in a value reaches the results that see it, and no others."""
    for dtype, rope in (("bf16", False), ("fp32", False), ("bf16", True), ("fp32", True)):
        x = Case(4, 8, 2, 64, dtype, STREAM, [300, 100, 35, 9], seed=3)
        out, lse = x.run(sp, rope)
        x.q[0, 3, 7] = float("nan")
        first = slots_of(x.sizes[1], x.a, x.s, x.c)
        x.cache[1][1, 1, first[50], 0] = 255   # a block of a key: query heads 4 .. 7 of sequence 1
        last = slots_of(x.sizes[2], x.a, x.s, x.c)[-1]
        x.cache[3][2, 0, last, 1] = 255        # a block of a value: dimensions 32 .. 63 of heads 0 .. 3 of sequence 2
        got, got_lse = x.run(sp, rope)
        bad, bad_lse = torch.zeros_like(out, dtype=torch.bool), torch.zeros_like(lse, dtype=torch.bool)
        bad[0, 3], bad[1, 4:], bad[2, :4, 32:] = True, True, True
        bad_lse[0, 3], bad_lse[1, 4:] = True, True
        assert torch.equal(torch.isnan(got), bad) and torch.equal(torch.isnan(got_lse), bad_lse)
        assert torch.equal(got[~bad], out[~bad]) and torch.equal(got_lse[~bad_lse], lse[~bad_lse])
        x.q[3, 0, 0] = float("inf")
        assert torch.isnan(x.run(sp, rope)[0][3, 0]).all()


def test_far_offsets(sp):
    """Codes of more than 4 GiB: the rows of the last sequences."""
    S, H, d, c = 9, 8, 128, 1 << 20
    codes = [torch.zeros(S, H, c, d // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((S, H, c, d // 32), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert codes[0].numel() > 1 << 32
    x = Case(S, 2 * H, H, d, "bf16", BARE, [70, 45], seed=2)
    # the same entries at the end of the long cache, in the window's ring
    sizes = []
    for i, row in enumerate(x.sizes):
        at, n = slots_of(row, 0, 0, 70), row[2] + row[3]
        to = [(c - 20 + j) % c for j in range(n)]
        for long, short in zip((codes[0], scales[0], codes[1], scales[1]), x.cache):
            long[i][:, to] = short[i][:, at]
        sizes.append([0, 0, n - 1, 1, 0, c - 20])
    sz = torch.tensor(sizes, dtype=torch.int32, device="cuda")
    for rope in (False, True):
        args = (x.q, codes[0], scales[0], codes[1], scales[1], sz)
        if rope:
            out = sp.sepattn_decode_rope_mx(*args, sp.sepkv_rope_table(c, d, BASE, "cuda"), 0, 0, 1, x.scale)
        else:
            out = sp.sepattn_decode_mx(*args, 0, 0, 1, x.scale)
        x.check(*out, rope)


@pytest.mark.parametrize("rope", [False, True])
def test_streams_and_graphs(sp, rope):
    """Calls at once on two streams with workspaces of their own; two captured graphs that share one workspace, replayed in turn beside eager calls."""
    xs = [Case(4, 32, 8, 128, "bf16", STREAM, [300, 100, 0, 35], seed=i) for i in range(2)]
    want = [x.run(sp, rope) for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got.append((i, xs[i].run(sp, rope)))
    torch.cuda.synchronize()
    for i, r in got:
        assert all(torch.equal(a, b) for a, b in zip(r, want[i]))
    need = sp.sepattn_decode_mx_workspace_bytes(xs[0].q, xs[0].cache[0], xs[0].a, xs[0].s, xs[0].w)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    table = sp.sepkv_rope_table(xs[0].c, 128, BASE, "cuda")
    for x in xs:
        out = (torch.empty_like(x.q), torch.empty(4, 32, device="cuda"))
        call = (lambda x=x, out=out: sp.sepattn_decode_rope_mx(x.q, *x.cache, x.sz, table, x.a, x.s, x.w, x.scale, out=out, ws=ws)) if rope else (
            lambda x=x, out=out: sp.sepattn_decode_mx(x.q, *x.cache, x.sz, x.a, x.s, x.w, x.scale, out=out, ws=ws))
        call()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
        outs.append(out)
    for i in (0, 1, 1, 0, 1, 0):
        outs[i][0].fill_(5.0)
        graphs[i].replay()
        eager = xs[1 - i].run(sp, rope, ws=ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i])) and all(torch.equal(a, b) for a, b in zip(eager, want[1 - i]))


def test_agrees_with_the_plain_cache(sp):
    """The same values in a plain cache: the two decodes differ by what the plain one rounds (its weights, once: 2^-8; with positions its turned rows)."""
    x = Case(4, 32, 8, 128, "bf16", STREAM, [300, 100, 35, 1], seed=8)
    K, V = sp.sepkv_expand_mx(*x.cache, x.sz, x.a, x.s, x.w)
    out, lse = x.run(sp, False)
    plain, plain_lse = sp.sepattn_decode(x.q, K, V, x.sz, x.a, x.s, x.w, x.scale)
    ref, _, size, reach = x.want(False)
    score = reach * (128 * 2.0 ** -24 + 2.0 ** -21)
    assert ((out.double() - plain.double()).abs().cpu() <= 2 * 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -15 + 4 * score[..., None]) * size).all()
    assert ((lse - plain_lse).abs().cpu() <= 2 * score + 2.0 ** -18).all()


@pytest.mark.parametrize("positions", ["text", "cache"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_generation(sp, dtype, positions):
    """A prompt enters the cache, tokens follow through norm, rotation, append, compression and attention; every step against softmax attention in
    64 bits over the values that the cache holds."""
    S, Hq, Hkv, L, d, dt = 3, 8, 2, 90, 128, DTYPES[dtype]
    a, s, w, c = 2, 6, 8, 40
    g = torch.Generator().manual_seed(0)
    randn = lambda *shape: torch.randn(*shape, generator=g).to(dt).cuda()
    freqs = sp.sepattn_rope_frequencies(d, BASE, device="cuda")
    weights = [(1 + 0.2 * torch.randn(d, generator=g)).to(dt).cuda() for _ in range(2)]
    q, k, v = randn(S, Hq, L, d), randn(S, Hkv, L, d), randn(S, Hkv, L, d)
    text = positions == "text"
    _, K, V = sp.sepattn_norm_rope(q, k, v, *weights, freqs if text else None, 1e-6)
    sep = (torch.rand(S, L, generator=g) < 0.2).to(torch.uint8).cuda()
    idx, _, pre = sp.sepattn_compact_indices(sep)
    *mx, flags, sizes = sp.sepkv_fill_from_prefill_mx(K, V, sep, idx, pre, Hq, a, s, w, c, 25)
    x = Case(S, Hq, Hkv, d, dtype, (a, s, w, c), [1])
    x.cache, x.sz = mx, sizes
    for t in range(30):
        if t % 7 == 0:
            sp.sepkv_evict_window_mx(*mx, flags, sizes, Hq, a, s, w)
        before = sizes[:, :4].sum(1).tolist()
        pos = torch.full((S,), L + t, dtype=torch.int32, device="cuda")
        new = torch.full((S,), int(t % 4 == 0), dtype=torch.uint8, device="cuda")
        x.q = sp.sepkv_append_norm_rope_mx(randn(S, Hq, d), randn(S, Hkv, d), randn(S, Hkv, d), new, pos if text else None, *weights, freqs if text else None, 1e-6,
                                           *mx, flags, sizes, a, s, w)
        x.sizes = sizes.tolist()
        assert [sum(r[:4]) for r in x.sizes] == [n + 1 for n in before]
        x.check(*x.run(sp, not text), not text)


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("S,d,entries", [(2, 128, 600), (33, 128, 600), (70, 64, 600), (130, 64, 300), (512, 64, 200), (513, 64, 200)])
def test_uneven_lengths(sp, rope, S, d, entries):
    """Sequences of every length in one call, which are cut into slices by their lengths; a captured call (whose slices another launch adds) gives the same
    bits, also for lengths that the device learns after the capture."""
    rng = np.random.default_rng(S)
    lengths = [entries, 0, 1] + [int(n) for n in rng.integers(0, entries + 1, S)]
    x = Case(S, 3, 1, d, "bf16", (2, 40, 30, entries), lengths, seed=S)
    want = x.run(sp, rope)
    x.check(*want, rope)
    table = sp.sepkv_rope_table(x.c, d, BASE, "cuda")
    ws = torch.zeros(sp.sepattn_decode_mx_workspace_bytes(x.q, x.cache[0], x.a, x.s, x.w), dtype=torch.uint8, device="cuda")
    out = (torch.empty_like(x.q), torch.empty(S, 3, device="cuda"))

    def call():
        if rope:
            sp.sepattn_decode_rope_mx(x.q, *x.cache, x.sz, table, x.a, x.s, x.w, x.scale, out=out, ws=ws)
        else:
            sp.sepattn_decode_mx(x.q, *x.cache, x.sz, x.a, x.s, x.w, x.scale, out=out, ws=ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    full = x.sz.clone()
    for keep in (1.0, 0.4, 0.0, 0.7, 1.0):
        x.sz.copy_(full)
        x.sz[1::2, 2] = (full[1::2, 2] * keep).int()  # (of every second sequence; a shorter window holds no slot that was empty)
        eager = [t.clone() for t in x.run(sp, rope, ws=ws)]
        out[0].fill_(5.0), out[1].fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
        if keep == 1.0:
            assert all(torch.equal(a, b) for a, b in zip(eager, want))
        else:
            y = x.__class__.__new__(x.__class__)
            y.__dict__.update(x.__dict__, sizes=x.sz.tolist())
            y.check(*eager, rope)


@pytest.mark.parametrize("rope", [False, True])
def test_few_long_among_many_short(sp, rope):
    """More sequences than there are workgroups to spare: the slices of the long ones fit what is launched and the workspace."""
    x = Case(140, 9, 9, 64, "bf16", (2, 40, 30, 800), [800, 1, 30, 0, 20, 9, 31], seed=4)
    need = sp.sepattn_decode_mx_workspace_bytes(x.q, x.cache[0], x.a, x.s, x.w)
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    x.check(*x.run(sp, rope, ws=ws[:need]), rope)
    assert (ws[need:] == 0xA5).all()


@pytest.mark.parametrize("rope", [False, True])
def test_sizes_outside_their_ranges(sp, rope):
    """Clamped on the device before sequences are cut into slices: the bits of the clamped sizes."""
    a, s, w, c = 4, 100, 30, 500
    x = Case(5, 8, 2, 64, "bf16", (a, s, w, c), [1], seed=9)
    for scales in (x.cache[1], x.cache[3]):
        scales.fill_(126)
    big, room = 1 << 30, c - a - s
    x.sz.copy_(torch.tensor([[big] * 6, [-5] * 6, [2, 40, 100, 30, 7, 9], [big, -1, 3, big, -1, big], [a, s, room, 5, s, room]], dtype=torch.int32))
    got = [t.clone() for t in x.run(sp, rope)]
    x.sz.copy_(torch.tensor([[a, s, room, 0, s - 1, room - 1], [0] * 6, [2, 40, 100, 30, 7, 9], [a, 0, 3, room - 3, 0, room - 1], [a, s, room, 0, s - 1, room - 1]],
                            dtype=torch.int32))
    want = x.run(sp, rope)
    assert all(torch.equal(i, j) for i, j in zip(got, want)) and torch.isfinite(got[1][[0, 2, 3, 4]]).all() and (got[0][1] == 0).all()


@pytest.mark.parametrize("rope", [False, True])
def test_captured_generation(sp, rope):
    """A step (compression, token through norm and rotation, attention) captured once and replayed with the program's own eager calls between, against
    the same steps one by one: the same bits, in the cache too."""
    S, Hq, Hkv, L, d = 3, 8, 2, 400, 128
    a, s, w, c = 2, 60, 40, 600
    g = torch.Generator().manual_seed(3)
    randn = lambda *shape: torch.randn(*shape, generator=g).to(torch.bfloat16).cuda()
    freqs, table = sp.sepattn_rope_frequencies(d, BASE, device="cuda"), sp.sepkv_rope_table(c, d, BASE, "cuda")
    weights = [(1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in range(2)]
    sep = (torch.rand(S, L, generator=g) < 0.2).to(torch.uint8).cuda()
    idx, _, pre = sp.sepattn_compact_indices(sep)
    state = sp.sepkv_fill_from_prefill_mx(randn(S, Hkv, L, d), randn(S, Hkv, L, d), sep, idx, pre, Hq, a, s, w, c, 200)
    tokens = [(randn(S, Hq, d), randn(S, Hkv, d), randn(S, Hkv, d)) for _ in range(8)]
    q, k, v = (t.clone() for t in tokens[0])
    pos, new = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.ones(S, dtype=torch.uint8, device="cuda")
    out, turned = (torch.empty_like(q), torch.empty(S, Hq, device="cuda")), torch.empty_like(q)
    ws = torch.zeros(sp.sepattn_decode_mx_workspace_bytes(q, state[0], a, s, w), dtype=torch.uint8, device="cuda")

    def step(cache, flags, sizes):
        sp.sepkv_evict_window_mx(*cache, flags, sizes, Hq, a, s, w)
        sp.sepkv_append_norm_rope_mx(q, k, v, new, None if rope else pos, *weights, None if rope else freqs, 1e-6, *cache, flags, sizes, a, s, w, out=turned)
        if rope:
            sp.sepattn_decode_rope_mx(turned, *cache, sizes, table, a, s, w, 0.1, out=out, ws=ws)
        else:
            sp.sepattn_decode_mx(turned, *cache, sizes, a, s, w, 0.1, out=out, ws=ws)

    def enter(t):
        for x, y in zip((q, k, v), tokens[t]):
            x.copy_(y)
        pos.fill_(L + t)

    mine, eager = [t.clone() for t in state], [t.clone() for t in state]
    step(mine[:4], *mine[4:])
    for x, y in zip(mine, state):
        x.copy_(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(mine[:4], *mine[4:])
    for t in range(len(tokens)):
        enter(t)
        step(eager[:4], *eager[4:])
        want = [x.clone() for x in (*out, turned)]
        for x in (*out, turned):
            x.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((*out, turned), want)), t
        assert all(torch.equal(x, y) for x, y in zip(mine, eager)), t


def test_one_workspace_for_calls_of_other_shapes(sp):
    """What one call leaves in a workspace is where the next one counts its slices: every call gives the bits of one with a workspace of its own."""
    xs = [Case(2, 8, 2, 128, "bf16", (2, 40, 30, 900), [900, 333], seed=1), Case(70, 3, 1, 64, "bf16", (2, 40, 30, 600), [600, 0, 1, 77, 410], seed=2),
          Case(4, 12, 12, 64, "fp32", STREAM, [300, 211, 7, 150], seed=3)]
    want = [x.run(sp, rope) for x in xs for rope in (False, True)]
    need = max(sp.sepattn_decode_mx_workspace_bytes(x.q, x.cache[0], x.a, x.s, x.w) for x in xs)
    ws = torch.randint(0, 256, (need,), dtype=torch.uint8, generator=torch.Generator().manual_seed(0)).cuda()
    for _ in range(5):
        got = [x.run(sp, rope, ws=ws) for x in xs for rope in (False, True)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for i, j in zip(got, want) for a, b in zip(i, j))
