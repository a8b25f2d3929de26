"""Rotary positions and decoding behind a shared prompt, as cases that can be timed and compared.

Kinds of call, each as a training loop or a server makes it:

  rotate    Q, K, V of a batch leave the projections token by token; Q and K are turned by their positions and
            all three are laid out head by head, as the attention calls take them
  gradient  dQ, dK, dV of the attention go back to what the projections put out
  step      one new token per sequence: its query is turned, its key is turned and enters the cache with its value
  admit     a prompt that many sequences share is taken in: its cached keys are turned by their positions within
            the cache, and the sequences of the batch are listed by the prompt they share
  shared    one token per sequence over the cache of the prompt that it shares with others, read once for all of
            them, and its own cache

With `own` false every kind is computed from elementary torch operations in 32 bits, with `own` true by the
package's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}

ROTATE = dict(kind="rotate", dtype="bf16", layout="fused", pairs="half", positions="index", base=500000.0, factor=1.0)
CACHE = dict(a=0, s=64, w=256, c=800)                      # a sequence's own part: what follows the shared prompt
KEPT = dict(prefix="kept", pa=4, ps=1024, pw=256, pc=1536)  # a prompt of which initial, separator and last tokens are kept
WHOLE = dict(prefix="whole", pa=0, ps=0, pw=1)              # a prompt kept whole, in the window of its cache


def listed():
    return [
        # the training step at 8K context: one fused projection, every pair turned
        dict(ROTATE, name="rotate_8k", B=1, Hq=32, Hkv=8, L=8192, d=128, rotary=128),
        # the training shape of many short sequences: a quarter of the head turned, q, k, v side by side in every head
        dict(ROTATE, name="rotate_2k", B=8, Hq=12, Hkv=12, L=2048, d=64, rotary=16, layout="per_head", base=10000.0),
        # gradients of the 8K step
        dict(ROTATE, name="gradient_8k", kind="gradient", B=1, Hq=32, Hkv=8, L=8192, d=128, rotary=128),
        # a fp32 run that a bf16 run is checked against, odd sizes: neighbouring pairs, packed documents, stretched frequencies
        dict(ROTATE, name="gradient_ragged", kind="gradient", dtype="fp32", layout="split", pairs="neighbours", positions="documents",
             factor=8.0, B=3, Hq=28, Hkv=4, L=1531, d=128, rotary=96),
        # one conversation, one token: latency
        dict(kind="step", name="step_one", dtype="bf16", S=1, Hq=32, Hkv=8, d=128, rotary=128, pairs="half", base=500000.0, far=3000, **CACHE),
        # a serving batch far into its streams, neighbouring pairs
        dict(kind="step", name="step_batch", dtype="bf16", S=64, Hq=32, Hkv=8, d=128, rotary=64, pairs="neighbours", base=10000.0,
             far=4000000, **CACHE),
        # one prompt kept whole, one batch
        dict(kind="admit", name="admit_8k", dtype="bf16", S=32, G=1, Hkv=8, d=128, base=500000.0, pc=8192, **WHOLE),
        # several compressed prompts, a batch that is spread over them and over none, in no order
        dict(kind="admit", name="admit_groups", dtype="bf16", S=1000, G=12, Hkv=8, d=128, base=500000.0, **KEPT),
        # two conversations that share a short prompt: latency
        dict(kind="shared", name="shared_two", dtype="bf16", S=2, G=1, alone=0, Hq=32, Hkv=8, d=128, rope=False, pc=600, **WHOLE, **CACHE),
        # a serving batch behind an instruction of 8K tokens, positions within the caches
        dict(kind="shared", name="shared_8k", dtype="bf16", S=32, G=1, alone=0, Hq=32, Hkv=8, d=128, rope=True, pc=8192, **WHOLE, **CACHE),
        # the same behind a document of 64K tokens: the largest call
        dict(kind="shared", name="shared_64k", dtype="bf16", S=48, G=1, alone=0, Hq=32, Hkv=8, d=128, rope=False, pc=65536, **WHOLE, **CACHE),
        # the fp32 path at the size it is used for: checking; one query head per KV head, three prompts, sequences without one
        dict(kind="shared", name="shared_check", dtype="fp32", S=11, G=3, alone=2, Hq=12, Hkv=12, d=64, rope=True, prefix="kept", pa=3, ps=100,
             pw=50, pc=300, a=0, s=16, w=64, c=150),
    ]


def _logint(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(8, 8), (12, 12), (32, 8), (16, 4), (28, 4), (8, 2), (16, 8), (32, 32), (6, 3), (8, 1), (64, 8)]


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "gradient", "step", "admit", "shared", "shared", "shared"])
    (Hq, Hkv), d = rng.choice(HEADS), rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    base = rng.choice([10000.0, 500000.0])
    rotary = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)])
    pairs = rng.choice(["half", "half", "neighbours"])
    if kind in ("rotate", "gradient"):
        layout = rng.choice(["fused", "split", "per_head"])
        if layout == "per_head":
            Hkv = Hq
        c = dict(ROTATE, kind=kind, dtype=dtype, layout=layout, pairs=pairs, positions=rng.choice(["index", "given", "documents"]), base=base,
                 factor=rng.choice([1.0, 1.0, 4.0, 32.0]), Hq=Hq, Hkv=Hkv, d=d, rotary=rotary)
        while True:
            c.update(B=rng.choice([1, 1, 2, 3, 8]), L=_logint(rng, 1, 16384))
            if c["B"] * c["L"] * (Hq + 2 * Hkv) * d <= 8192 * 48 * 128:
                return c
    cache = dict(a=rng.choice([0, 0, 4]), s=_logint(rng, 16, 512), w=_logint(rng, 16, 512))
    cache["c"] = cache["a"] + cache["s"] + cache["w"] + _logint(rng, 16, 512)
    if kind == "step":
        while True:
            S = _logint(rng, 1, 128)
            if S * Hkv * cache["c"] * d <= 64 * 8 * 800 * 128:
                return dict(kind=kind, dtype=dtype, S=S, Hq=Hq, Hkv=Hkv, d=d, rotary=rotary, pairs=pairs, base=base, far=_logint(rng, 1000, 4000000),
                            **cache)
    while True:
        G, S = rng.choice([1, 1, 2, 3, 5]), _logint(rng, 1, 200)
        if rng.random() < 0.6:
            prefix = dict(WHOLE, pc=_logint(rng, 2, 65536))
        else:
            prefix = dict(prefix="kept", pa=rng.choice([0, 3, 4]), ps=_logint(rng, 16, 2048), pw=_logint(rng, 16, 512))
            prefix["pc"] = prefix["pa"] + prefix["ps"] + prefix["pw"] + _logint(rng, 16, 512)
        rows = G * Hkv * prefix["pc"] * d
        if kind == "admit" and rows <= 8 * 65536 * 128:
            return dict(kind=kind, dtype=dtype, S=S, G=G, Hkv=Hkv, d=d, base=base, **prefix)
        # (the plain form looks at every prompt for every sequence)
        if kind == "shared" and rows + S * Hkv * cache["c"] * d <= 8 * 65536 * 128 and S * Hq * G * prefix["pc"] <= 48 * 32 * 65536:
            return dict(kind=kind, dtype=dtype, S=S, G=G, alone=rng.choice([0, 0, min(S, 2)]), Hq=Hq, Hkv=Hkv, d=d, rope=rng.random() < 0.5,
                        **prefix, **cache)


# ------------------------------------------------------------------------------------------------
def _normal(g, shape, dtype, scale=1.0):
    return torch.randn(shape, device="cuda", generator=g, dtype=torch.float32).mul_(scale).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _frequencies(c):
    """float64: radians per position of every pair, base^(-2i/rotary); with a factor, slow ones (less than one turn in
    8192 positions) divided by it, fast ones (more than four) kept, between them a blend."""
    f = [c["base"] ** (-2.0 * i / c["rotary"]) for i in range(c["rotary"] // 2)]
    factor = c.get("factor", 1.0)
    if factor != 1.0:
        blend = [min(1.0, max(0.0, (8192 * x / (2 * math.pi) - 1.0) / 3.0)) for x in f]
        f = [x * b + x / factor * (1.0 - b) for x, b in zip(f, blend)]
    return torch.tensor(f, dtype=torch.float64, device="cuda")


def _outside_layout(c, x):
    """q, k, v [B, H, L, d] as views of what the projections put out."""
    Hq, Hkv = c["Hq"], c["Hkv"]
    if c["layout"] == "per_head":
        q, k, v = x.unbind(3)
    elif c["layout"] == "fused":
        q, k, v = x.split([Hq, Hkv, Hkv], dim=2)
    else:
        q, k, v = x
    return tuple(t.transpose(1, 2) for t in (q, k, v))


def _prepare_rotate(c, g):
    B, Hq, Hkv, L, d, dtype = c["B"], c["Hq"], c["Hkv"], c["L"], c["d"], DTYPES[c["dtype"]]
    st = dict(c, freqs=_frequencies(c), pos=None, doc_start=None)
    if c["positions"] == "given":  # prompts that continue behind different histories
        first = torch.randint(0, 1 << 20, (B, 1), device="cuda", generator=g)
        st["pos"] = (first + torch.arange(L, device="cuda")).to(torch.int32)
    if c["positions"] == "documents":
        starts = torch.rand((B, L), device="cuda", generator=g) < 4.0 / max(L, 4)
        starts[:, 0] = True
        st["doc_start"] = torch.where(starts, torch.arange(L, device="cuda"), 0).cummax(1).values.to(torch.int32)
    if c["kind"] == "gradient":
        st["grads"] = tuple(_normal(g, (B, h, L, d), dtype) for h in (Hq, Hkv, Hkv))
        return st
    if c["layout"] == "per_head":
        st["x"] = _normal(g, (B, L, Hq, 3, d), dtype)
    elif c["layout"] == "fused":
        st["x"] = _normal(g, (B, L, Hq + 2 * Hkv, d), dtype)
    else:
        st["x"] = tuple(_normal(g, (B, L, h, d), dtype) for h in (Hq, Hkv, Hkv))
    return st


def _spread(i, n):
    """0 <= x < 1, evenly spread over i = 0 .. n-1, in no order."""
    return (i * 0.6180339887498949) % 1.0 if n > 1 else 0.5


def _own_sizes(c):
    """Valid entries of every sequence's own cache: between half full and full; one holds a single token."""
    a, s, w, room = c["a"], c["s"], c["w"], c["c"] - c["a"] - c["s"]
    out = []
    for i in range(c["S"]):
        x = _spread(i, c["S"])
        past = int(x * (room - w))
        out.append([a, int((0.5 + 0.5 * x) * s), past, w, 0, 0] if i % 7 != 3 else [min(a, 1), 0, 0, 0 if a else 1, 0, 0])
    return out


def _prefix_sizes(c):
    pa, ps, pw, pc = (c[k] for k in ("pa", "ps", "pw", "pc"))
    room = pc - pa - ps
    out = []
    for i in range(c["G"]):
        x = 1.0 - 0.4 * i / c["G"]  # the first one fills its cache
        if c["prefix"] == "whole":
            n = max(1, int(x * pc))
            out.append([0, 0, n - 1, 1, 0, 0])
        else:
            out.append([pa, int(x * ps), int(x * (room - pw)), pw, 0, 0])
    return out


def _prefix_of(c):
    """The prompt of every sequence, -1 for none: the first prompt has the most sequences."""
    S, G = c["S"], c["G"]
    none = c.get("alone", S // 10 if G > 1 else 0)
    return [-1 if i < none else min(int(G * _spread(i, S) ** 1.5), G - 1) for i in range(S)]


def _heads(g, sizes, s, room):
    """Ring heads of caches that have dropped entries before."""
    n = sizes.shape[0]
    sizes[:, 4] = torch.randint(0, max(s, 1), (n,), device="cuda", generator=g)
    sizes[:, 5] = torch.randint(0, room, (n,), device="cuda", generator=g)
    return sizes


def _prepare_step(c, g):
    S, Hq, Hkv, d, a, s, cc, dtype = c["S"], c["Hq"], c["Hkv"], c["d"], c["a"], c["s"], c["c"], DTYPES[c["dtype"]]
    room = cc - a - s
    st = dict(c, freqs=_frequencies(c), Kc=_normal(g, (S, Hkv, cc, d), dtype), Vc=_normal(g, (S, Hkv, cc, d), dtype))
    st.update(q=_normal(g, (S, Hq, d), dtype), k=_normal(g, (S, Hkv, d), dtype), v=_normal(g, (S, Hkv, d), dtype))
    st["sep"] = (torch.rand((S,), device="cuda", generator=g) < 0.08).to(torch.uint8)
    st["flags"] = (torch.rand((S, room), device="cuda", generator=g) < 0.08).to(torch.uint8)
    st["pos"] = torch.randint(cc, max(cc + 1, c["far"]), (S,), device="cuda", generator=g).to(torch.int32)
    st["sizes"] = _heads(g, _ints(_own_sizes(c)), s, room)
    return st


def _table(n_pos, d, base):
    """fp32 [n_pos, 2, d/2]: cos, then sin, of position * base^(-2i/d)."""
    f = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    angle = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack([angle.cos(), angle.sin()], dim=1).float().contiguous()


def _prepare_admit(c, g):
    G, Hkv, d, pc = c["G"], c["Hkv"], c["d"], c["pc"]
    st = dict(c, K=_normal(g, (G, Hkv, pc, d), DTYPES[c["dtype"]]), psizes=_ints(_prefix_sizes(c)), table=_table(pc, d, c["base"]))
    st["K_out"] = torch.zeros_like(st["K"])
    st["prefix_of"] = _ints(_prefix_of(c))[torch.randperm(c["S"], device="cuda", generator=g)].contiguous()
    if c["prefix"] == "kept":
        _heads(g, st["psizes"], c["ps"], pc - c["pa"] - c["ps"])
    return st


def _prepare_shared(c, g):
    S, G, Hq, Hkv, d, a, s, cc, pc, dtype = c["S"], c["G"], c["Hq"], c["Hkv"], c["d"], c["a"], c["s"], c["c"], c["pc"], DTYPES[c["dtype"]]
    st = dict(c, scale=1.0 / math.sqrt(d), q=_normal(g, (S, Hq, d), dtype))
    st.update(Kc=_normal(g, (S, Hkv, cc, d), dtype), Vc=_normal(g, (S, Hkv, cc, d), dtype))
    st.update(Kp=_normal(g, (G, Hkv, pc, d), dtype), Vp=_normal(g, (G, Hkv, pc, d), dtype))
    st["sizes"], st["psizes"] = _heads(g, _ints(_own_sizes(c)), s, cc - a - s), _ints(_prefix_sizes(c))
    if c["prefix"] == "kept":
        _heads(g, st["psizes"], c["ps"], pc - c["pa"] - c["ps"])
    st["table"] = _table(pc + cc, d, 500000.0) if c["rope"] else None
    of = _prefix_of(c)
    st["prefix_of"] = _ints(of)[torch.randperm(S, device="cuda", generator=g)].contiguous()
    # the plan that a program makes when its batch changes: the sequences listed by prompt
    alone = of.count(-1)
    order = torch.argsort(st["prefix_of"], stable=True)[alone:]
    st["group_seq"] = torch.cat([order, order.new_zeros(alone)]).to(torch.int32)
    counts = [of.count(i) for i in range(G)]
    st["group_start"] = _ints([sum(counts[:i]) for i in range(G + 1)])
    return st


PREPARE = dict(rotate=_prepare_rotate, gradient=_prepare_rotate, step=_prepare_step, admit=_prepare_admit, shared=_prepare_shared)


def prepare(case, seed):
    return PREPARE[case["kind"]](case, torch.Generator(device="cuda").manual_seed(seed))


# ---- the package's calls ------------------------------------------------------------------------
def _own_rotate(st):
    import paper_2412_12094_amd as sp

    q, k, v = _outside_layout(st, st["x"])
    return sp.sepattn_rope(q, k, v, st["freqs"], positions=st["pos"], doc_start=st["doc_start"], interleaved=st["pairs"] == "neighbours")


def _own_gradient(st):
    import paper_2412_12094_amd as sp

    B, Hq, Hkv, L, d, dtype = st["B"], st["Hq"], st["Hkv"], st["L"], st["d"], DTYPES[st["dtype"]]
    if st["layout"] == "per_head":
        dx = torch.empty((B, L, Hq, 3, d), dtype=dtype, device="cuda")
    elif st["layout"] == "fused":
        dx = torch.empty((B, L, Hq + 2 * Hkv, d), dtype=dtype, device="cuda")
    else:
        dx = tuple(torch.empty((B, L, h, d), dtype=dtype, device="cuda") for h in (Hq, Hkv, Hkv))
    sp.sepattn_rope_backward(*st["grads"], st["freqs"], positions=st["pos"], doc_start=st["doc_start"], interleaved=st["pairs"] == "neighbours",
                             out=_outside_layout(st, dx))
    return dx


def _own_step(st):
    import paper_2412_12094_amd as sp

    sizes = st["sizes"].clone()  # (a pass leaves the state as it found it)
    q = sp.sepkv_append_rope(st["q"], st["k"], st["v"], st["sep"], st["pos"], st["freqs"], st["Kc"], st["Vc"], st["flags"], sizes, st["a"],
                             st["s"], st["w"], interleaved=st["pairs"] == "neighbours")
    return dict(q=q, Kc=st["Kc"], Vc=st["Vc"], flags=st["flags"], sizes=sizes)


def _own_admit(st):
    import paper_2412_12094_amd as sp

    start, seq = sp.sepkv_group_sequences(st["prefix_of"], st["G"])
    K = sp.sepkv_rope_cache(st["K"], st["psizes"], st["table"], st["pa"], st["ps"], st["pw"], out=st["K_out"])
    return dict(K=K, start=start, seq=seq)


def _own_shared(st):
    import paper_2412_12094_amd as sp

    args = (st["q"], st["Kc"], st["Vc"], st["sizes"], st["a"], st["s"], st["w"], st["Kp"], st["Vp"], st["psizes"], st["pa"], st["ps"], st["pw"],
            st["prefix_of"], st["group_start"], st["group_seq"])
    if st["rope"]:
        return sp.sepattn_decode_shared_rope(*args, st["table"], st["scale"])
    return sp.sepattn_decode_shared(*args, st["scale"])


# ---- the plain forms ------------------------------------------------------------------------------
def _turn(x, cos, sin, pairs, back=False):
    """The first 2 * cos.shape[-1] values of x's last dimension turned by the angles, the rest as they are; fp32."""
    r = 2 * cos.shape[-1]
    x = x.float()
    if back:
        sin = -sin
    if pairs == "half":
        u, v = x[..., : r // 2], x[..., r // 2: r]
        return torch.cat([u * cos - v * sin, v * cos + u * sin, x[..., r:]], dim=-1)
    u, v = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([u * cos - v * sin, v * cos + u * sin], dim=-1).flatten(-2), x[..., r:]], dim=-1)


def _angles(st, pos):
    angle = pos.double()[..., None] * st["freqs"]
    return angle.cos().float(), angle.sin().float()


def _positions(st):
    if st["pos"] is not None:
        return st["pos"]
    index = torch.arange(st["L"], device="cuda").expand(st["B"], -1)
    return index if st["doc_start"] is None else index - st["doc_start"]


def _plain_rotate(st):
    cos, sin = (t[:, None] for t in _angles(st, _positions(st)))
    q, k, v = _outside_layout(st, st["x"])
    return _turn(q, cos, sin, st["pairs"]).to(q.dtype), _turn(k, cos, sin, st["pairs"]).to(k.dtype), v.contiguous()


def _plain_gradient(st):
    cos, sin = (t[:, None] for t in _angles(st, _positions(st)))
    dQ, dK, dV = st["grads"]
    parts = [t.to(dV.dtype).transpose(1, 2) for t in (_turn(dQ, cos, sin, st["pairs"], True), _turn(dK, cos, sin, st["pairs"], True), dV)]
    if st["layout"] == "per_head":
        return torch.stack(parts, dim=3)
    if st["layout"] == "fused":
        return torch.cat(parts, dim=2)
    return tuple(t.contiguous() for t in parts)


def _plain_step(st):
    a, s, w, cc = st["a"], st["s"], st["w"], st["c"]
    room, sizes = cc - a - s, st["sizes"].clone()
    cos, sin = (t[:, None] for t in _angles(st, st["pos"]))
    q = _turn(st["q"], cos, sin, st["pairs"]).to(st["q"].dtype)
    k = _turn(st["k"], cos, sin, st["pairs"]).to(st["k"].dtype)
    used = sizes[:, 2] + sizes[:, 3]
    initial = sizes[:, 0] < a
    enters = initial | (used < room)
    window = (sizes[:, 5] + used) % room
    slot = torch.where(initial, sizes[:, 0], a + s + window).long()
    row = torch.arange(st["S"], device="cuda")
    st["Kc"][row, :, slot] = torch.where(enters[:, None, None], k, st["Kc"][row, :, slot])
    st["Vc"][row, :, slot] = torch.where(enters[:, None, None], st["v"], st["Vc"][row, :, slot])
    flagged = enters & ~initial
    st["flags"][row, window.long()] = torch.where(flagged, st["sep"], st["flags"][row, window.long()])
    sizes[:, 0] += initial
    over = flagged & (sizes[:, 3] + 1 > w)
    sizes[:, 2] += over
    sizes[:, 3] += flagged & ~over
    return dict(q=q, Kc=st["Kc"], Vc=st["Vc"], flags=st["flags"], sizes=sizes)


def _slots(sizes, a, s, c):
    """valid [S, c], rank [S, c]: whether a slot holds an entry, and which one, oldest first."""
    j, room = torch.arange(c, device="cuda"), c - a - s
    n_init, n_sep, n_win, head_sep, head_win = (t[:, None] for t in (sizes[:, 0], sizes[:, 1], sizes[:, 2] + sizes[:, 3], sizes[:, 4], sizes[:, 5]))
    k, u = (j - a - head_sep) % max(s, 1), (j - a - s - head_win) % room
    valid = torch.where(j < a, j < n_init, torch.where(j < a + s, k < n_sep, u < n_win))
    return valid, torch.where(j < a, j, torch.where(j < a + s, n_init + k, n_init + n_sep + u))


def _plain_admit(st):
    valid, rank = _slots(st["psizes"], st["pa"], st["ps"], st["pc"])
    table = st["table"][torch.where(valid, rank, 0).long()]  # [G, pc, 2, d/2]
    K = _turn(st["K"], table[:, None, :, 0], table[:, None, :, 1], "half").to(st["K"].dtype)
    of, G = st["prefix_of"], st["G"]
    start = (of[None] < torch.arange(G + 1, device="cuda")[:, None]).sum(1) - (of < 0).sum()
    member = of >= 0
    order = torch.argsort(torch.where(member, of, G), stable=True)
    seq = torch.where(member[order], order, 0)
    return dict(K=torch.where(valid[:, None, :, None], K, st["K_out"]), start=start.to(torch.int32), seq=seq.to(torch.int32))


def _plain_shared(st):
    S, G, Hq, Hkv, d, scale = st["S"], st["G"], st["Hq"], st["Hkv"], st["d"], st["scale"]
    heads = Hq // Hkv
    valid, rank = _slots(st["sizes"], st["a"], st["s"], st["c"])
    pvalid, _ = _slots(st["psizes"], st["pa"], st["ps"], st["pc"])
    of = st["prefix_of"]
    q = st["q"].float().view(S, Hkv, heads, d)
    Kc = torch.where(valid[:, None, :, None], st["Kc"].float(), 0.0)
    if st["rope"]:
        before = torch.where(of >= 0, pvalid.sum(1)[of.clamp(min=0).long()], 0)  # positions taken by the prompt
        at = (before + valid.sum(1) - 1).clamp(min=0)
        turn = st["table"][at]
        q = _turn(q, turn[:, None, None, 0], turn[:, None, None, 1], "half")
        turn = st["table"][(before[:, None] + torch.where(valid, rank, 0)).long()]
        Kc = _turn(Kc, turn[:, None, :, 0], turn[:, None, :, 1], "half")
    # the own entries' scores, then those of every prompt's entries; what a sequence does not see is left out
    P = pvalid.shape[1]
    rows = q.transpose(0, 1).reshape(1, Hkv, S * heads, d)
    Kp = torch.where(pvalid[:, None, :, None], st["Kp"].float(), 0.0)
    x = torch.matmul(rows, Kp.transpose(-1, -2)).view(G, Hkv, S, heads, P).permute(2, 1, 3, 0, 4).reshape(S, Hkv, heads, G * P)
    x = torch.cat([torch.matmul(q, Kc.transpose(-1, -2)), x], dim=-1).mul_(scale)
    shared = (pvalid & (of[:, None] == torch.arange(G, device="cuda"))[..., None]).view(S, G * P)
    x.masked_fill_(~torch.cat([valid, shared], dim=1)[:, None, None], float("-inf"))
    m = x.amax(-1)
    p = x.sub_(torch.where(torch.isinf(m), 0.0, m)[..., None]).exp_()
    total = p.sum(-1)
    out = torch.matmul(p[..., : st["c"]], torch.where(valid[:, None, :, None], st["Vc"].float(), 0.0))
    p = p[..., st["c"]:].view(S, Hkv, heads, G, P).permute(3, 1, 0, 2, 4).reshape(G, Hkv, S * heads, P)
    Vp = torch.where(pvalid[:, None, :, None], st["Vp"].float(), 0.0)
    out += torch.matmul(p, Vp).sum(0).view(Hkv, S, heads, d).transpose(0, 1)
    out = torch.where((total > 0)[..., None], out / total[..., None], 0.0)
    return out.reshape(S, Hq, d).to(st["q"].dtype), (m + total.log()).view(S, Hq)


RUN = {True: dict(rotate=_own_rotate, gradient=_own_gradient, step=_own_step, admit=_own_admit, shared=_own_shared),
       False: dict(rotate=_plain_rotate, gradient=_plain_gradient, step=_plain_step, admit=_plain_admit, shared=_plain_shared)}


def run(state):
    return RUN[bool(own)][state["kind"]](state)


# ------------------------------------------------------------------------------------------------
def work(case):
    """Bytes: every input once, every output once; of the caches the valid entries only."""
    c, es = case, 4 if case["dtype"] == "fp32" else 2
    d = c["d"]
    if c["kind"] in ("rotate", "gradient"):
        tokens = c["B"] * c["L"]
        return {"bytes": 2 * es * tokens * (c["Hq"] + 2 * c["Hkv"]) * d + (0 if c["positions"] == "index" else 4 * tokens),
                "flops": 3.0 * tokens * (c["Hq"] + c["Hkv"]) * c["rotary"]}
    if c["kind"] == "step":
        S = c["S"]
        return {"bytes": 2 * es * S * (c["Hq"] + 2 * c["Hkv"]) * d + S * (4 + 1 + 1 + 48), "flops": 3.0 * S * (c["Hq"] + c["Hkv"]) * c["rotary"]}
    prompts = [sum(x[:4]) for x in _prefix_sizes(c)]
    S, G, Hkv = c["S"], c["G"], c["Hkv"]
    if c["kind"] == "admit":
        rows = sum(prompts)
        return {"bytes": 2 * es * Hkv * rows * d + 4 * max(prompts) * d + 24 * G + 4 * S + 4 * (G + 1) + 4 * S, "flops": 3.0 * Hkv * rows * d}
    mine = sum(sum(x[:4]) for x in _own_sizes(c))
    of = _prefix_of(c)
    read = sum(n for i, n in enumerate(prompts) if i in of)
    pairs = mine + sum(prompts[i] for i in of if i >= 0)
    return {"bytes": 2 * es * Hkv * d * (mine + read) + S * c["Hq"] * (2 * es * d + 4) + 24 * (S + G) + 8 * S,
            "flops": 4.0 * d * c["Hq"] * pairs}


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _rotation(x, pos, freqs, pairs):
    """x [..., d] turned by pos [...] as complex numbers."""
    n = freqs.numel()
    x = x.double().clone()
    first = slice(0, n) if pairs == "half" else slice(0, 2 * n, 2)
    second = slice(n, 2 * n) if pairs == "half" else slice(1, 2 * n, 2)
    z = torch.complex(x[..., first], x[..., second]) * torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                                                                   pos.double()[..., None] * freqs.to("cuda"))
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _entries(row, a, s, c):
    """The slots of a cache's entries, oldest first."""
    n_init, n_sep, past, local, head_sep, head_win = row
    room = c - a - s
    return list(range(n_init)) + [a + (head_sep + i) % s for i in range(n_sep)] + [a + s + (head_win + i) % room for i in range(past + local)]


def _exact_rotate(st):
    index = torch.arange(st["L"], device="cuda")[None].repeat(st["B"], 1)
    pos = (st["pos"] if st["pos"] is not None else index - (0 if st["doc_start"] is None else st["doc_start"]))[:, None]
    if st["kind"] == "rotate":
        q, k, v = _outside_layout(st, st["x"])
        return _rotation(q, pos, st["freqs"], st["pairs"]), _rotation(k, pos, st["freqs"], st["pairs"]), v.double().contiguous()
    dQ, dK, dV = st["grads"]
    parts = _rotation(dQ, -pos, st["freqs"], st["pairs"]), _rotation(dK, -pos, st["freqs"], st["pairs"]), dV.double()
    B, Hq, Hkv, L, d = st["B"], st["Hq"], st["Hkv"], st["L"], st["d"]
    if st["layout"] == "split":
        return tuple(t.permute(0, 2, 1, 3).contiguous() for t in parts)
    shape = (B, L, Hq, 3, d) if st["layout"] == "per_head" else (B, L, Hq + 2 * Hkv, d)
    dx = torch.empty(shape, dtype=torch.float64, device="cuda")
    for t, to in zip(parts, _outside_layout(st, dx)):
        to.copy_(t)
    return dx


def _exact_step(st):
    a, s, w, cc = st["a"], st["s"], st["w"], st["c"]
    q = _rotation(st["q"], st["pos"][:, None], st["freqs"], st["pairs"])
    k = _rotation(st["k"], st["pos"][:, None], st["freqs"], st["pairs"])
    Kc, Vc, flags, sizes = st["Kc"].double(), st["Vc"].double(), st["flags"].clone(), st["sizes"].tolist()
    for i, row in enumerate(sizes):
        count = row[2] + row[3]
        if row[0] < a:
            slot, row[0] = row[0], row[0] + 1
        elif count < cc - a - s:
            place = (row[5] + count) % (cc - a - s)
            slot = a + s + place
            flags[i, place] = st["sep"][i]
            row[2 if row[3] == w else 3] += 1
        else:
            continue
        Kc[i, :, slot], Vc[i, :, slot] = k[i], st["v"][i].double()
    return dict(q=q, Kc=Kc, Vc=Vc, flags=flags, sizes=_ints(sizes))


def _exact_admit(st):
    K = torch.zeros(st["K"].shape, dtype=torch.float64, device="cuda")
    f = st["base"] ** (-2.0 * torch.arange(st["d"] // 2, dtype=torch.float64) / st["d"])
    for i, row in enumerate(st["psizes"].tolist()):
        at = _entries(row, st["pa"], st["ps"], st["pc"])
        K[i, :, at] = _rotation(st["K"][i, :, at], torch.arange(len(at), device="cuda")[None], f, "half")
    of = st["prefix_of"].tolist()
    members = [[i for i, x in enumerate(of) if x == n] for n in range(st["G"])]
    seq = [i for m in members for i in m]
    start = [sum(len(m) for m in members[:n]) for n in range(st["G"] + 1)]
    return dict(K=K, start=_ints(start), seq=_ints(seq + [0] * (st["S"] - len(seq))))


def _exact_shared(st):
    S, Hq, Hkv, d = st["S"], st["Hq"], st["Hkv"], st["d"]
    f = 500000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    prompts = []
    for i, row in enumerate(st["psizes"].tolist()):
        at = torch.tensor(_entries(row, st["pa"], st["ps"], st["pc"]), device="cuda")
        prompts.append((st["Kp"][i][:, at].double(), st["Vp"][i][:, at].double()))
    out = torch.zeros((S, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((S, Hq), float("-inf"), dtype=torch.float64, device="cuda")
    of = st["prefix_of"].tolist()
    for i, row in enumerate(st["sizes"].tolist()):
        at = torch.tensor(_entries(row, st["a"], st["s"], st["c"]), device="cuda", dtype=torch.long)
        K, V, q = st["Kc"][i][:, at].double(), st["Vc"][i][:, at].double(), st["q"][i].double()
        before = prompts[of[i]][0].shape[1] if of[i] >= 0 else 0
        if st["rope"]:
            K = _rotation(K, before + torch.arange(len(at), device="cuda")[None], f, "half")
            q = _rotation(q, torch.full((1,), before + len(at) - 1, device="cuda"), f, "half")
        if of[i] >= 0:
            K, V = torch.cat([prompts[of[i]][0], K], dim=1), torch.cat([prompts[of[i]][1], V], dim=1)
        if K.shape[1] == 0:
            continue
        x = torch.bmm(q.view(Hkv, Hq // Hkv, d), K.transpose(1, 2).contiguous()) * st["scale"]
        out[i] = torch.bmm(torch.softmax(x, dim=-1), V).view(Hq, d)
        lse[i] = torch.logsumexp(x, dim=-1).view(Hq)
    return out, lse


EXACT = dict(rotate=_exact_rotate, gradient=_exact_rotate, step=_exact_step, admit=_exact_admit, shared=_exact_shared)


def exact(case, seed):
    return EXACT[case["kind"]](prepare(case, seed))
