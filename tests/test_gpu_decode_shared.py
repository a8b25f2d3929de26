"""Decoding behind shared prompts against softmax attention in 64 bits.  Needs an MI355X."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BASE = 10000.0


@pytest.fixture(scope="module")
def sp():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2412_12094_amd as sp_

    sp_.load()
    return sp_


def randn(*shape, dtype, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


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


def blank(x, sizes, a, s, c):
    """NaN in every slot without an entry: nothing may read one."""
    for i, row in enumerate(sizes):
        used = set(slots_of(row, a, s, c))
        x[i][:, [j for j in range(c) if j not in used]] = float("nan")
    return x


def turn(x, pos):
    """float64 [..., d] turned by pos [...]; dimension i with i + d/2."""
    h = x.shape[-1] // 2
    f = BASE ** (-torch.arange(h, dtype=torch.float64, device=pos.device) / h)
    angle = pos.double()[..., None] * f
    u, v = x[..., :h], x[..., h:]
    return torch.cat([u * angle.cos() - v * angle.sin(), v * angle.cos() + u * angle.sin()], -1)


class Case:
    def __init__(self, S, Hq, Hkv, d, dtype, own, prompts, own_n, prompt_n, prefix_of, seed=0):
        self.a, self.s, self.w, self.c = own
        self.pa, self.ps, self.pw, self.pc = prompts
        self.S, self.G, self.Hq, self.Hkv, self.d, self.dt = S, len(prompt_n), Hq, Hkv, d, DTYPES[dtype]
        rng = np.random.default_rng(seed)
        self.sizes = [sizes_of(own_n[i % len(own_n)], rng, *own) for i in range(S)]
        self.psizes = [sizes_of(n, rng, *prompts) for n in prompt_n]
        self.of = [prefix_of[i % len(prefix_of)] for i in range(S)]
        self.q = randn(S, Hq, d, dtype=self.dt, seed=seed)
        self.Kc, self.Vc = (blank(randn(S, Hkv, self.c, d, dtype=self.dt, seed=seed + i), self.sizes, self.a, self.s, self.c) for i in (1, 2))
        self.Kp, self.Vp = (blank(randn(self.G, Hkv, self.pc, d, dtype=self.dt, seed=seed + i), self.psizes, self.pa, self.ps, self.pc) for i in (3, 4))
        self.scale = 1.0 / math.sqrt(d)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        self.sz, self.psz, self.prefix_of = i32(self.sizes), i32(self.psizes), i32(self.of)

    def run(self, sp, rope, **kw):
        start, seq = sp.sepkv_group_sequences(self.prefix_of, self.G)
        args = (self.q, self.Kc, self.Vc, self.sz, self.a, self.s, self.w, self.Kp, self.Vp, self.psz, self.pa, self.ps, self.pw,
                self.prefix_of, start, seq)
        if not rope:
            return sp.sepattn_decode_shared(*args, self.scale, **kw)
        return sp.sepattn_decode_shared_rope(*args, sp.sepkv_rope_table(self.pc + self.c, self.d, BASE, "cuda"), self.scale, **kw)

    def want(self, rope, where="cpu"):
        """out, lse, mean of |V| under the weights, largest sum of |q_i k_i| scale over the keys of a row; in float64."""
        f = lambda t: t.detach().to(where).double()
        out, lse, size, reach = (torch.zeros(self.S, self.Hq, self.d, dtype=torch.float64), torch.full((self.S, self.Hq), float("-inf"), dtype=torch.float64),
                                 torch.zeros(self.S, self.Hq, self.d, dtype=torch.float64), torch.zeros(self.S, self.Hq, dtype=torch.float64))
        for i in range(self.S):
            at = slots_of(self.sizes[i], self.a, self.s, self.c)
            K, V, q = f(self.Kc[i][:, at]), f(self.Vc[i][:, at]), f(self.q[i])
            g = self.of[i]
            shared = slots_of(self.psizes[g], self.pa, self.ps, self.pc) if 0 <= g < self.G else []
            if rope and len(at) + len(shared):
                K = turn(K, len(shared) + torch.arange(len(at), device=where)[None])
                q = turn(q, torch.tensor(len(shared) + len(at) - 1, device=where))
            if shared:
                K, V = torch.cat([f(self.Kp[g][:, shared]), K], 1), torch.cat([f(self.Vp[g][:, shared]), V], 1)
            if K.shape[1] == 0:
                continue
            K, V = (t.repeat_interleave(self.Hq // self.Hkv, 0) for t in (K, V))
            x = (K @ q[..., None])[..., 0] * self.scale
            p = torch.softmax(x, -1)
            out[i], size[i] = (p[:, None] @ V)[:, 0], (p[:, None] @ V.abs())[:, 0]
            lse[i], reach[i] = torch.logsumexp(x, -1), (K.abs() @ q.abs()[..., None])[..., 0].amax(-1) * self.scale
        return out, lse, size, reach

    def check(self, out, lse, rope, want=None):
        ref, ref_lse, size, reach = want or self.want(rope)
        # a score: d products added in fp32 (each sum off by 2^-24 of what it holds, at most d of them), and scaled; with positions the angles'
        # 2^-20 and, in bf16, the turned one of key and query as two numbers (2^-8 of 2^-8)
        score = reach * (self.d * 2.0 ** -24 + 2.0 ** -21 + (2.0 ** -20 + (2.0 ** -16 if self.dt == torch.bfloat16 else 0.0) if rope else 0.0))
        none = torch.isinf(ref_lse)
        got = lse.double().cpu()
        assert torch.equal(torch.isinf(got) & (got < 0), none)
        err = (got - ref_lse).abs()[~none]
        assert (err <= (score + 2.0 ** -22 * (ref_lse.abs() + 8.0))[~none]).all(), float(err.max())
        # an output: its rounding, that of the weights (bf16), the scores' errors twice (weight and sum), sums in fp32
        half = torch.finfo(self.dt).eps / 2
        weights = 2.0 ** -8 if self.dt == torch.bfloat16 else 0.0
        err = (out.double().cpu() - ref).abs()
        assert (err <= half * ref.abs() + (weights + 2.0 * score[..., None] + 2.0 ** -18) * size).all(), float(err.max())
        assert (out[none.cuda()] == 0).all()


SMALL = (3, 8, 6, 40)   # a, s, w, c of an own cache
BARE = (0, 0, 1, 70)    # ... of a sequence that keeps everything
CASES = {
    # S, Hq, Hkv, d, own, prompts, entries of the own caches, entries of the prompts, prefix_of
    "one": (1, 1, 1, 64, BARE, (0, 0, 1, 2), [1], [1], [0]),
    "one of many heads": (1, 40, 1, 128, BARE, (0, 0, 1, 200), [5], [199], [0]),
    "two": (2, 32, 8, 128, SMALL, (4, 16, 8, 100), [40, 1], [100], [0]),
    "eight": (8, 32, 8, 128, SMALL, (0, 0, 1, 700), [0, 1, 31, 32, 33, 40], [700], [0]),          # 32 rows per KV head
    "thirteen": (13, 28, 4, 64, SMALL, (4, 30, 20, 600), [40, 7], [555], [0]),                    # 91 rows
    "spread": (37, 12, 4, 128, SMALL, (0, 0, 1, 333), [17, 0, 40], [333, 1, 0, 64, 65], [4, -1, 0, 0, 3, 2, 1, 7, 0]),
    "nobody": (5, 8, 2, 64, SMALL, (0, 0, 1, 64), [40, 0], [64, 10], [-1]),
    "nothing": (4, 6, 2, 128, SMALL, (0, 0, 1, 64), [0], [0, 12], [0, -1]),
    "many prompts": (70, 4, 2, 64, SMALL, (2, 6, 4, 50), [9, 40], [(7 * i) % 51 for i in range(66)], [(5 * i) % 67 - 1 for i in range(67)]),
    "long": (3, 16, 2, 128, SMALL, (4, 512, 64, 9001), [40], [8990], [0]),
    "wide": (40, 16, 2, 64, SMALL, (0, 0, 1, 2500), [3, 38], [2500], [0]),                        # 320 rows
    "one wide KV head": (9, 71, 1, 64, SMALL, (0, 0, 1, 130), [12], [129], [0]),
}


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("name", CASES)
def test_against_64_bits(sp, name, dtype, rope):
    S, Hq, Hkv, d, own, prompts, own_n, prompt_n, of = CASES[name]
    case = Case(S, Hq, Hkv, d, dtype, own, prompts, own_n, prompt_n, of, seed=len(name))
    out, lse = case.run(sp, rope)
    case.check(out, lse, rope)
    again = case.run(sp, rope)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_large_scores(sp):
    """Scores of some thousand: a row's maximum decides, and slices without it count with weight 0."""
    case = Case(6, 8, 2, 64, "bf16", SMALL, (0, 0, 1, 900), [40, 3], [900], [0])
    case.q.mul_(256.0)  # a power of two: exact
    out, lse = case.run(sp, False)
    case.check(out, lse, False)


def test_plan_and_sizes_out_of_range(sp):
    """Values outside their ranges: the results of the sequences they concern are unspecified, nothing else is."""
    case = Case(12, 8, 2, 64, "bf16", SMALL, (0, 0, 1, 200), [20, 40], [150, 90], [0, 1, -1])
    start, seq = sp.sepkv_group_sequences(case.prefix_of, 2)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    args = lambda sz, psz, of, st, sq: (case.q, case.Kc.nan_to_num(), case.Vc.nan_to_num(), sz, *SMALL[:3], case.Kp.nan_to_num(), case.Vp.nan_to_num(), psz,
                                        0, 0, 1, of, st, sq, case.scale)
    big = 1 << 30
    for st in ([0, big, -big], [-5, 3, 2], [big, big, big], [0, 0, 0]):
        sp.sepattn_decode_shared(*args(case.sz, case.psz, case.prefix_of, i32(st), seq))
    sp.sepattn_decode_shared(*args(case.sz, case.psz, case.prefix_of, start, seq * big - 1))
    sp.sepattn_decode_shared(*args(case.sz, case.psz, case.prefix_of * big, start, seq))
    sp.sepattn_decode_shared(*args(case.sz + big, case.psz - big, case.prefix_of, start, seq))
    torch.cuda.synchronize()
    out, lse = case.run(sp, False)
    case.check(out, lse, False)


def test_outputs_and_workspace_of_the_caller(sp):
    case = Case(5, 8, 2, 128, "bf16", SMALL, (0, 0, 1, 300), [20, 40], [300], [0, -1])
    want = case.run(sp, False)
    ws = torch.full((sp.sepattn_decode_shared_workspace_bytes(case.q, case.Kc, *SMALL[:3], case.Kp, 0, 0, 1),), 255, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(case.q)
    got = case.run(sp, False, out=(out, None), ws=ws)
    assert got[0] is out and got[1] is None and torch.equal(out, want[0])
    with pytest.raises(sp.SepattnError) as err:
        case.run(sp, False, ws=ws[:-256])
    assert err.value.status == 5
    # on a stream of its own
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = case.run(sp, False)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("S,G", [(1, 1), (64, 1), (65, 3), (1000, 12), (130, 200), (5000, 7)])
def test_sequences_are_listed_in_order(sp, S, G):
    rng = np.random.default_rng(S)
    of = rng.integers(-2, G + 2, size=S).astype(np.int32)
    of[0] = np.iinfo(np.int32).min
    start, seq = (t.cpu().numpy() for t in sp.sepkv_group_sequences(torch.from_numpy(of).cuda(), G))
    members = [np.flatnonzero(of == g) for g in range(G)]
    assert np.array_equal(start, np.concatenate([[0], np.cumsum([len(m) for m in members])]))
    listed = np.concatenate(members)
    assert np.array_equal(seq, np.concatenate([listed, np.zeros(S - len(listed), np.int32)]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_generation_behind_a_shared_prompt(sp, dtype):
    """A prompt is prefilled, handed over to a prefix cache and turned once; three sequences then append tokens of their own.  Every step
    equals the decode with positions over caches of their own that hold the prompt as well, within what that one rounds."""
    dt = DTYPES[dtype]
    S, Hq, Hkv, d, L, scale = 3, 8, 2, 64, 300, 0.125
    K, V = randn(1, Hkv, L, d, dtype=dt, seed=1), randn(1, Hkv, L, d, dtype=dt, seed=2)
    tok = torch.randint(0, 9, (1, L), generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    is_sep, idx, cnt, pre = sp.sepattn_mark_compact(tok, [1])
    pa, ps, pw, pc = 4, 64, 50, 130
    Kp, Vp, _, psz = sp.sepkv_fill_from_prefill(K, V, is_sep, idx, pre, Hq, pa, ps, pw, pc, 60)
    row = psz[0].tolist()
    at = slots_of(row, pa, ps, pc)
    a, s, w, c = 0, 4, 8, 32
    table = sp.sepkv_rope_table(pc + c, d, BASE, "cuda")
    whole_c = len(at) + c
    whole = [torch.zeros(S, Hkv, whole_c, d, dtype=dt, device="cuda") for _ in range(2)]
    whole[0][:, :, : len(at)], whole[1][:, :, : len(at)] = Kp[:, :, at], Vp[:, :, at]
    whole_sizes = torch.tensor([[0, 0, len(at) - 1, 1, 0, 0]] * S, dtype=torch.int32, device="cuda")
    sp.sepkv_rope_cache(Kp, psz, table, pa, ps, pw)
    of = torch.tensor([0, 0, 0], dtype=torch.int32, device="cuda")
    start, seq = sp.sepkv_group_sequences(of, 1)
    Kc, Vc = (torch.zeros(S, Hkv, c, d, dtype=dt, device="cuda") for _ in range(2))
    flags, sizes = torch.zeros(S, c - s, dtype=torch.uint8, device="cuda"), torch.zeros(S, 6, dtype=torch.int32, device="cuda")
    wflags = torch.zeros(S, whole_c, dtype=torch.uint8, device="cuda")
    for step in range(12):
        q, k, v = (randn(S, h, d, dtype=dt, seed=100 + 3 * step + i) for i, h in enumerate((Hq, Hkv, Hkv)))
        sep = torch.zeros(S, dtype=torch.uint8, device="cuda")
        sp.sepkv_append(k, v, sep, Kc, Vc, flags, sizes, Hq, a, s, w)
        sp.sepkv_append(k, v, sep, *whole, wflags, whole_sizes, Hq, 0, 0, 1)
        out, lse = sp.sepattn_decode_shared_rope(q, Kc, Vc, sizes, a, s, w, Kp, Vp, psz, pa, ps, pw, of, start, seq, table, scale)
        ref, ref_lse = sp.sepattn_decode_rope(q, *whole, whole_sizes, table, 0, 0, 1, scale)
        # what the library states for the decode with positions
        assert (out.float() - ref.float()).abs().max() <= (2e-2 if dtype == "bf16" else 1e-4)
        assert (lse - ref_lse).abs().max() <= (1e-2 if dtype == "bf16" else 1e-4)


@pytest.mark.parametrize("rope", [False, True])
def test_in_a_graph(sp, rope):
    """Two captured calls on one workspace, replayed after new queries and with eager calls between: every replay gives the eager bits."""
    case = Case(7, 8, 2, 128, "bf16", SMALL, (0, 0, 1, 900), [20, 40], [900, 77], [0, 1, -1])
    start, seq = sp.sepkv_group_sequences(case.prefix_of, case.G)
    table = sp.sepkv_rope_table(case.pc + case.c, case.d, BASE, "cuda")
    ws = torch.empty(sp.sepattn_decode_shared_workspace_bytes(case.q, case.Kc, *SMALL[:3], case.Kp, 0, 0, 1), dtype=torch.uint8, device="cuda")
    q2 = case.q.clone()

    def call(q, out=None):
        args = (q, case.Kc, case.Vc, case.sz, *SMALL[:3], case.Kp, case.Vp, case.psz, 0, 0, 1, case.prefix_of, start, seq)
        return sp.sepattn_decode_shared_rope(*args, table, case.scale, out=out, ws=ws) if rope else sp.sepattn_decode_shared(*args, case.scale, out=out, ws=ws)

    outs = [(torch.empty_like(case.q), torch.empty(7, 8, dtype=torch.float32, device="cuda")) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(case.q, outs[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(case.q, outs[0])
        call(q2, outs[1])
    for step in range(4):
        case.q.copy_(randn(7, 8, 128, dtype=torch.bfloat16, seed=50 + step))
        q2.copy_(randn(7, 8, 128, dtype=torch.bfloat16, seed=60 + step))
        graph.replay()
        torch.cuda.synchronize()
        for q, out in zip((case.q, q2), outs):
            want = call(q)
            assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("S,own_n,prompt_n,of", [
    (13, [40, 1], [33100], [0]),                 # 104 rows of a KV head
    (24, [40, 0, 33], [33333], [0]),             # 192
    (24, [40], [31], [0]),                       # nearly every slice is empty
    (40, [7, 40], [33333, 1500, 0], [0, 1, 0, 2, 0, -1])])
def test_many_slices(sp, S, own_n, prompt_n, of, rope):
    case = Case(S, 8, 1, 128, "bf16", SMALL, (4, 700, 64, 33333), own_n, prompt_n, of, seed=S)
    out, lse = case.run(sp, rope)
    case.check(out, lse, rope, tuple(t.cpu() for t in case.want(rope, "cuda")))


@pytest.mark.parametrize("S,Hq,Hkv,G", [(1500, 2, 1, 3000), (2047, 32, 4, 2), (65535, 1, 1, 1)])
def test_many_sequences_and_prompts(sp, S, Hq, Hkv, G):
    """As many rows and prompts as the calls take; a few of the sequences are looked at."""
    case = Case(min(S, 64), Hq, Hkv, 64, "bf16", (1, 1, 1, 4), (0, 0, 1, 3), [0, 1, 4], [3, 0, 2], [0], seed=5)
    at = sorted({(i * 997) % S for i in range(64)} | {0, S - 1})[: case.S]
    small, (K, V, Kp, Vp) = case, (case.Kc, case.Vc, case.Kp, case.Vp)
    full = Case.__new__(Case)
    full.__dict__.update(small.__dict__)
    index = torch.zeros(S, dtype=torch.long, device="cuda")
    index[at] = torch.arange(len(at), device="cuda")
    which = torch.arange(G, device="cuda") % 3
    full.S, full.G = S, G
    full.q, full.Kc, full.Vc, full.sz = small.q[index], K[index], V[index], small.sz[index]
    full.Kp, full.Vp, full.psz = Kp[which], Vp[which], small.psz[which]
    full.prefix_of = ((torch.arange(S, device="cuda") * 7) % (G + 1)).to(torch.int32)  # G: none
    out, lse = full.run(sp, False)
    small.S, small.G = len(at), G
    small.q, small.Kc, small.Vc = full.q[at], full.Kc[at], full.Vc[at]
    small.sizes = [full.sz[i].tolist() for i in at]
    small.Kp, small.Vp, small.psizes = full.Kp, full.Vp, full.psz.tolist()
    small.of = full.prefix_of[at].tolist()
    small.check(out[at], lse[at], False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_slots_far_apart(sp, dtype):
    """The longest caches that are taken (rows up to 2^32 bytes into a head), entries in their last and first slots."""
    c = (2 ** 32 - 1) // (4 * 128)
    case = Case(2, 4, 1, 128, dtype, SMALL, SMALL, [40, 37], [40], [0], seed=3)
    a, s, w, small = SMALL
    room = c - a - s
    rows = [[3, 5, 10, 6, 7, room - 9], [0, 8, 20, 6, 1, room - 1]]

    def spread(x, sizes):
        big = torch.full((x.shape[0], 1, c, 128), float("nan"), dtype=x.dtype, device="cuda")
        for i, row in enumerate(sizes):
            at = slots_of(row, a, s, c)
            big[i][:, at] = randn(1, len(at), 128, dtype=x.dtype, seed=11 + i)
        return big

    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    case.c = case.pc = c
    case.sizes, case.psizes = rows, rows[:1]
    case.sz, case.psz = i32(rows), i32(rows[:1])
    case.Kc, case.Vc, case.Kp, case.Vp = spread(case.Kc, rows), spread(case.Vc, rows), spread(case.Kp, rows[:1]), spread(case.Vp, rows[:1])
    for rope in (False, True):
        out, lse = case.run(sp, rope)
        case.check(out, lse, rope)


def test_two_streams(sp):
    """Calls on two streams at once, a workspace each."""
    cases = [Case(6, 16, 2, 128, "bf16", SMALL, (0, 0, 1, 4000), [40, 3], [4000], [0], seed=i) for i in (1, 2)]
    want = [c.run(sp, True) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for c, st in zip(cases, streams):
            with torch.cuda.stream(st):
                got.append(c.run(sp, True))
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(got):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_values_not_finite_stay_with_the_sequences_that_see_them(sp, dtype, rope, value):
    """A query, an own value, a prefix's value: other sequences, also of the same prefix and product, are as accurate as without."""
    case = Case(23, 8, 2, 64, dtype, SMALL, (4, 30, 20, 600), [40, 7, 30], [555, 90], [0, 1, 0, -1], seed=8)
    want = case.want(rope)
    clean = case.run(sp, rope)
    case.q[4, 3, 5] = value                                                            # sequence 4 shares prefix 0
    case.Vc[2, :, slots_of(case.sizes[2], case.a, case.s, case.c)[3], 7] = value       # sequence 2: prefix 0
    for hit in (lambda i: i in (2, 4), lambda i: i in (2, 4) or case.of[i] == 1):
        out, lse = case.run(sp, rope)
        rows = [i for i in range(case.S) if hit(i)]
        assert all(not out[i].isfinite().all() for i in rows)
        out[rows], lse[rows] = clean[0][rows], clean[1][rows]
        case.check(out, lse, rope, want)
        case.Vp[1, :, slots_of(case.psizes[1], case.pa, case.ps, case.pc)[50]] = value  # everyone's behind prefix 1


@pytest.mark.parametrize("S", [3, 20])  # a wave has all rows, or its own
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scores_of_minus_infinity(sp, dtype, S):
    """Entries whose scores are minus infinity count with weight 0, whole blocks and slices of them, and in front of the others."""
    case = Case(S, 8, 2, 64, dtype, SMALL, (0, 0, 1, 700), [40, 7, 0], [700], [0], seed=S)
    case.q[:, :, 0] = 1.0
    case.psizes = [[0, 0, 699, 1, 0, 0]]
    case.psz = torch.tensor(case.psizes, dtype=torch.int32, device="cuda")
    case.Kp[:, :, :300, 0] = float("-inf")
    got = case.run(sp, False)
    case.psizes = [[0, 0, 399, 1, 0, 300]]
    want = case.want(False)
    case.check(*got, False, want)
    case.Kp[:, :, :, 0] = float("-inf")
    out, lse = case.run(sp, False)
    case.of = [-1] * S
    case.check(out, lse, False)
