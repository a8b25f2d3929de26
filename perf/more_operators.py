"""Norms of queries and keys with their rotary positions, and a KV cache held in 4 bits, as cases that can be timed and compared.

Kinds of call, each as a training loop or a server makes it:

  norm      q, k, v of a batch leave the projections token by token; the rows of q and k are divided by their root mean square,
            multiplied by a weight per dimension and turned by their positions, and all three are laid out head by head
  gradient  dQ, dK, dV of the attention go back to what the projections put out, and to the two weights
  token     one new token per sequence: its query and key are normed and turned, the key enters the cache with its value
  admit     a prompt is taken into a 4-bit cache: its kept keys and values are rounded to 4 bits on the way, the separators of
            the past window move to their block, and the cache is read back as values
  step      one new token per sequence, normed and turned, enters a 4-bit cache, and attends to it
  decode    one query per sequence over a 4-bit cache

A cache in 4 bits holds E2M1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign; dimension 2i in the low half of byte i) with a scale
2^(byte - 127) for every 32 dimensions of a row.

With `own` false every kind is computed from elementary torch operations in 32 bits, with `own` true by the package's calls.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}

NORM = dict(kind="norm", dtype="bf16", layout="fused", pairs="half", positions="index", base=500000.0)
STREAM = dict(a=4, s=1024, w=256, c=3332)  # what a stream keeps: initial tokens, separators, a window
SHORT = dict(a=4, s=64, w=256, c=800)      # a conversation


def listed():
    return [
        # the training step at 8K context: one fused projection, every pair turned
        dict(NORM, name="norm_8k", B=1, Hq=32, Hkv=8, L=8192, d=128, rotary=128),
        # a fp32 run that a bf16 run is checked against, odd sizes: neighbouring pairs, packed documents, a part of the head turned
        dict(NORM, name="norm_ragged", dtype="fp32", layout="split", pairs="neighbours", positions="documents", B=3, Hq=28, Hkv=4, L=1531,
             d=128, rotary=96),
        # gradients of the 8K step
        dict(NORM, name="gradient_8k", kind="gradient", B=1, Hq=32, Hkv=8, L=8192, d=128, rotary=128),
        # gradients of many short sequences: a quarter of the head turned, q, k, v side by side in every head
        dict(NORM, name="gradient_2k", kind="gradient", B=8, Hq=12, Hkv=12, L=2048, d=64, rotary=16, layout="per_head", base=10000.0),
        # one conversation, one token: latency
        dict(kind="token", name="token_one", dtype="bf16", S=1, Hq=32, Hkv=8, d=128, rotary=128, pairs="half", base=500000.0, far=3000, **SHORT),
        # a serving batch far into its streams, neighbouring pairs
        dict(kind="token", name="token_batch", dtype="bf16", S=64, Hq=32, Hkv=8, d=128, rotary=64, pairs="neighbours", base=10000.0,
             far=4000000, **SHORT),
        # prompts of 8K tokens enter the caches of their streams
        dict(kind="admit", name="admit_8k", dtype="bf16", S=8, Hq=32, Hkv=8, d=128, L=8192, nw=1500, density=0.08, **STREAM),
        # odd sizes in fp32, more separators than the cache keeps
        dict(kind="admit", name="admit_ragged", dtype="fp32", S=3, Hq=12, Hkv=12, d=64, L=2311, nw=333, density=0.3, a=3, s=150, w=100, c=601),
        # one conversation, one token through norm, rotation, cache and attention: latency
        dict(kind="step", name="step_one", dtype="bf16", S=1, Hq=32, Hkv=8, d=128, rotary=128, pairs="half", base=500000.0, far=3000, **SHORT),
        # a serving batch of compressed streams, positions within the cache
        dict(kind="decode", name="decode_stream", dtype="bf16", S=32, Hq=32, Hkv=8, d=128, rope=True, **STREAM),
        # few sequences that keep everything: the largest call
        dict(kind="decode", name="decode_64k", dtype="bf16", S=4, Hq=32, Hkv=8, d=128, rope=False, a=0, s=0, w=1, c=65536),
        # the fp32 path at the size it is used for: checking; one query head per KV head
        dict(kind="decode", name="decode_check", dtype="fp32", S=11, Hq=12, Hkv=12, d=64, rope=True, a=3, s=100, w=50, c=300),
    ]


def _logint(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(8, 8), (12, 12), (32, 8), (16, 4), (28, 4), (8, 2), (16, 8), (32, 32), (6, 3), (8, 1), (64, 8), (20, 1)]


def draw(rng):
    kind = rng.choice(["norm", "gradient", "token", "admit", "step", "decode", "decode", "decode"])
    (Hq, Hkv), d = rng.choice(HEADS), rng.choice([64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    base = rng.choice([10000.0, 500000.0])
    rotary = rng.choice([d, d, d // 2, d // 4, 2 * rng.randint(1, d // 2)])
    pairs = rng.choice(["half", "half", "neighbours"])
    if kind in ("norm", "gradient"):
        layout = rng.choice(["fused", "split", "per_head"])
        if layout == "per_head":
            Hkv = Hq
        c = dict(NORM, kind=kind, dtype=dtype, layout=layout, pairs=pairs, positions=rng.choice(["index", "given", "documents"]), base=base,
                 Hq=Hq, Hkv=Hkv, d=d, rotary=rotary)
        while True:
            c.update(B=rng.choice([1, 1, 2, 3, 8]), L=_logint(rng, 1, 16384))
            if c["B"] * c["L"] * (Hq + 2 * Hkv) * d <= 8192 * 48 * 128:
                return c
    while True:
        cache = dict(a=rng.choice([0, 0, 4]), s=_logint(rng, 16, 2048), w=_logint(rng, 16, 512))
        cache["c"] = cache["a"] + cache["s"] + cache["w"] + _logint(rng, 16, 1024)
        if kind == "decode" and rng.random() < 0.4:  # everything is kept, in the window
            cache = dict(a=0, s=0, w=1, c=_logint(rng, 2, 65536))
        S = _logint(rng, 1, 128)
        values = S * Hkv * cache["c"] * d
        if kind == "admit":
            L = _logint(rng, 1, 16384)
            nw = rng.randint(0, min(cache["c"] - cache["a"] - cache["s"], L - min(cache["a"], L)))
            if values <= 8 * 8 * 3332 * 128 and S * Hkv * L * d <= 8 * 8 * 8192 * 128:
                return dict(kind=kind, dtype=dtype, S=S, Hq=Hq, Hkv=Hkv, d=d, L=L, nw=nw, density=rng.choice([0.08, 0.02, 0.3]), **cache)
        elif kind == "decode":
            if values <= 4 * 8 * 65536 * 128 and S * Hq * cache["c"] <= 4 * 32 * 65536:
                return dict(kind=kind, dtype=dtype, S=S, Hq=Hq, Hkv=Hkv, d=d, rope=rng.random() < 0.5, **cache)
        elif values <= 64 * 8 * 800 * 128:
            return dict(kind=kind, dtype=dtype, S=S, Hq=Hq, Hkv=Hkv, d=d, rotary=rotary, pairs=pairs, base=base, far=_logint(rng, 1000, 4000000),
                        **cache)


# ------------------------------------------------------------------------------------------------
def _normal(g, shape, dtype, scale=1.0):
    return torch.randn(shape, device="cuda", generator=g, dtype=torch.float32).mul_(scale).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _frequencies(c):
    """float64: radians per position of every pair."""
    return torch.tensor([c["base"] ** (-2.0 * i / c["rotary"]) for i in range(c["rotary"] // 2)], dtype=torch.float64, device="cuda")


def _weights(c, g):
    return tuple((1.0 + 0.2 * torch.randn((c["d"],), device="cuda", generator=g)).to(DTYPES[c["dtype"]]) for _ in range(2))


EPS = 1e-6


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


def _prepare_norm(c, g):
    B, Hq, Hkv, L, d, dtype = c["B"], c["Hq"], c["Hkv"], c["L"], c["d"], DTYPES[c["dtype"]]
    st = dict(c, freqs=_frequencies(c), pos=None, doc_start=None, weights=_weights(c, g))
    if c["positions"] == "given":  # prompts that continue behind different histories
        first = torch.randint(0, 1 << 20, (B, 1), device="cuda", generator=g)
        st["pos"] = (first + torch.arange(L, device="cuda")).to(torch.int32)
    if c["positions"] == "documents":
        starts = torch.rand((B, L), device="cuda", generator=g) < 4.0 / max(L, 4)
        starts[:, 0] = True
        st["doc_start"] = torch.where(starts, torch.arange(L, device="cuda"), 0).cummax(1).values.to(torch.int32)
    if c["layout"] == "per_head":
        st["x"] = _normal(g, (B, L, Hq, 3, d), dtype)
    elif c["layout"] == "fused":
        st["x"] = _normal(g, (B, L, Hq + 2 * Hkv, d), dtype)
    else:
        st["x"] = tuple(_normal(g, (B, L, h, d), dtype) for h in (Hq, Hkv, Hkv))
    if c["kind"] == "gradient":
        st["grads"] = tuple(_normal(g, (B, h, L, d), dtype) for h in (Hq, Hkv, Hkv))
    return st


def _spread(i, n):
    """0 <= x < 1, evenly spread over i = 0 .. n-1, in no order."""
    return (i * 0.6180339887498949) % 1.0 if n > 1 else 0.5


def _cache_sizes(c):
    """Valid entries of every sequence's cache: between half full and full, with room for a token; of a batch one holds a single token."""
    a, s, w, room = c["a"], c["s"], c["w"], c["c"] - c["a"] - c["s"]
    out = []
    for i in range(c["S"]):
        x = _spread(i, c["S"])
        past = int((0.5 + 0.5 * x) * (room - w)) if s == 0 else int(x * (room - w))
        if past + w == room and c["kind"] != "decode":
            past -= 1
        out.append([a, int((0.5 + 0.5 * x) * s), past, w, 0, 0] if i % 7 != 3 else [min(a, 1), 0, 0, 0 if a else 1, 0, 0])
    return out


def _ring_heads(g, c):
    """int32 [S, 6]: the sizes, with ring heads of caches that have dropped entries before."""
    sizes, S = _ints(_cache_sizes(c)), c["S"]
    sizes[:, 4] = torch.randint(0, max(c["s"], 1), (S,), device="cuda", generator=g)
    sizes[:, 5] = torch.randint(0, c["c"] - c["a"] - c["s"], (S,), device="cuda", generator=g)
    return sizes


def _to_fp4(x):
    """x [..., d] -> codes 0 .. 15 as int32 [..., d] and scale bytes int32 [..., d/32]."""
    y = x.float().unflatten(-1, (-1, 32))
    big = y.abs().amax(-1)
    m, e = torch.frexp(big)  # big = m 2^e, 1/2 <= m < 1; the largest two-bit value below 2^e is 7/8 2^e
    byte = torch.where(big > 0, e - 1 + (m > 0.875) - 2, -125).clamp(-125, 125) + 127
    t = torch.ldexp(y, (127 - byte)[..., None])
    size = t.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    size = ((size / step).round() * step).clamp(max=6.0)
    code = torch.where(size < 2, 2 * size, torch.where(size < 4, size + 2, size / 2 + 4)).to(torch.int32) + 8 * torch.signbit(t)
    return code.flatten(-2), byte


def _from_fp4(code, byte):
    """float32: the values that codes [..., d] and scale bytes [..., d/32] stand for."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    return (table[code.long()].unflatten(-1, (-1, 32)) * torch.exp2(byte.float() - 127)[..., None]).flatten(-2)


def _packed(code):
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)


def _unpacked(x):
    return torch.stack([x & 15, x >> 4], dim=-1).flatten(-2)


def _normal_fp4(g, shape):
    """Normal values in 4 bits, made a slice at a time."""
    code = torch.empty((*shape[:-1], shape[-1] // 2), dtype=torch.uint8, device="cuda")
    byte = torch.empty((*shape[:-1], shape[-1] // 32), dtype=torch.uint8, device="cuda")
    for i in range(shape[0]):
        n, b = _to_fp4(_normal(g, shape[1:], torch.float32))
        code[i], byte[i] = _packed(n), b
    return code, byte


def _prepare_token(c, g):
    S, Hq, Hkv, d, cc, dtype = c["S"], c["Hq"], c["Hkv"], c["d"], c["c"], DTYPES[c["dtype"]]
    st = dict(c, freqs=_frequencies(c), weights=_weights(c, g), scale=1.0 / math.sqrt(d))
    if c["kind"] == "token":
        st.update(Kc=_normal(g, (S, Hkv, cc, d), dtype), Vc=_normal(g, (S, Hkv, cc, d), dtype))
    else:
        (st["Kc"], st["Ks"]), (st["Vc"], st["Vs"]) = _normal_fp4(g, (S, Hkv, cc, d)), _normal_fp4(g, (S, Hkv, cc, d))
    st.update(q=_normal(g, (S, Hq, d), dtype), k=_normal(g, (S, Hkv, d), dtype), v=_normal(g, (S, Hkv, d), dtype))
    st["sep"] = (torch.rand((S,), device="cuda", generator=g) < 0.08).to(torch.uint8)
    st["flags"] = (torch.rand((S, cc - c["a"] - c["s"]), device="cuda", generator=g) < 0.08).to(torch.uint8)
    st["pos"] = torch.randint(cc, max(cc + 1, c["far"]), (S,), device="cuda", generator=g).to(torch.int32)
    st["sizes"] = _ring_heads(g, c)
    return st


def _prepare_admit(c, g):
    S, Hkv, L, d, dtype = c["S"], c["Hkv"], c["L"], c["d"], DTYPES[c["dtype"]]
    st = dict(c, K=_normal(g, (S, Hkv, L, d), dtype), V=_normal(g, (S, Hkv, L, d), dtype))
    sep = torch.rand((S, L), device="cuda", generator=g) < c["density"]
    # as marking and compaction leave them: the separators' positions in ascending order, and how many stand before each position
    at = torch.where(sep, torch.arange(L, device="cuda"), L).sort(1).values
    st.update(is_sep=sep.to(torch.uint8), sep_idx=torch.where(at < L, at, -1).to(torch.int32))
    st["sep_prefix"] = torch.cat([torch.zeros((S, 1), device="cuda"), sep.cumsum(1)], dim=1).to(torch.int32)
    return st


def _table(n_pos, d, base):
    """fp32 [n_pos, 2, d/2]: cos, then sin, of position * base^(-2i/d)."""
    f = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    angle = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack([angle.cos(), angle.sin()], dim=1).float().contiguous()


def _prepare_decode(c, g):
    S, Hq, Hkv, d, cc = c["S"], c["Hq"], c["Hkv"], c["d"], c["c"]
    st = dict(c, scale=1.0 / math.sqrt(d), q=_normal(g, (S, Hq, d), DTYPES[c["dtype"]]), table=_table(cc, d, 500000.0) if c["rope"] else None)
    (st["Kc"], st["Ks"]), (st["Vc"], st["Vs"]) = _normal_fp4(g, (S, Hkv, cc, d)), _normal_fp4(g, (S, Hkv, cc, d))
    st["sizes"] = _ring_heads(g, c)
    return st


PREPARE = dict(norm=_prepare_norm, gradient=_prepare_norm, token=_prepare_token, step=_prepare_token, admit=_prepare_admit, decode=_prepare_decode)


def prepare(case, seed):
    return PREPARE[case["kind"]](case, torch.Generator(device="cuda").manual_seed(seed))


# ---- the package's calls ------------------------------------------------------------------------
def _own_norm(st):
    import paper_2412_12094_amd as sp

    q, k, v = _outside_layout(st, st["x"])
    return sp.sepattn_norm_rope(q, k, v, *st["weights"], st["freqs"], EPS, positions=st["pos"], doc_start=st["doc_start"],
                                interleaved=st["pairs"] == "neighbours")


def _own_gradient(st):
    import paper_2412_12094_amd as sp

    B, Hq, Hkv, L, d, dtype = st["B"], st["Hq"], st["Hkv"], st["L"], st["d"], DTYPES[st["dtype"]]
    if st["layout"] == "per_head":
        dx = torch.empty((B, L, Hq, 3, d), dtype=dtype, device="cuda")
    elif st["layout"] == "fused":
        dx = torch.empty((B, L, Hq + 2 * Hkv, d), dtype=dtype, device="cuda")
    else:
        dx = tuple(torch.empty((B, L, h, d), dtype=dtype, device="cuda") for h in (Hq, Hkv, Hkv))
    q, k, _ = _outside_layout(st, st["x"])
    _, _, _, dq_weight, dk_weight = sp.sepattn_norm_rope_backward(
        q, k, *st["grads"], *st["weights"], st["freqs"], EPS, positions=st["pos"], doc_start=st["doc_start"],
        interleaved=st["pairs"] == "neighbours", out=_outside_layout(st, dx))
    return dict(dx=dx, dq_weight=dq_weight, dk_weight=dk_weight)


def _own_token(st):
    import paper_2412_12094_amd as sp

    sizes = st["sizes"].clone()  # (a pass leaves the state as it found it)
    q = sp.sepkv_append_norm_rope(st["q"], st["k"], st["v"], st["sep"], st["pos"], *st["weights"], st["freqs"], EPS, st["Kc"], st["Vc"],
                                  st["flags"], sizes, st["a"], st["s"], st["w"], interleaved=st["pairs"] == "neighbours")
    return dict(q=q, Kc=st["Kc"], Vc=st["Vc"], flags=st["flags"], sizes=sizes)


def _own_step(st):
    import paper_2412_12094_amd as sp

    sizes, cache, blocks = st["sizes"].clone(), (st["Kc"], st["Ks"], st["Vc"], st["Vs"]), (st["a"], st["s"], st["w"])
    q = sp.sepkv_append_norm_rope_mx(st["q"], st["k"], st["v"], st["sep"], st["pos"], *st["weights"], st["freqs"], EPS, *cache, st["flags"],
                                      sizes, *blocks, interleaved=st["pairs"] == "neighbours")
    out, lse = sp.sepattn_decode_mx(q, *cache, sizes, *blocks, st["scale"])
    return dict(q=q, out=out, lse=lse, flags=st["flags"], sizes=sizes)


def _own_admit(st):
    import paper_2412_12094_amd as sp

    blocks = (st["a"], st["s"], st["w"])
    *cache, flags, sizes = sp.sepkv_fill_from_prefill_mx(st["K"], st["V"], st["is_sep"], st["sep_idx"], st["sep_prefix"], st["Hq"], *blocks,
                                                          st["c"], st["nw"])
    sp.sepkv_evict_window_mx(*cache, flags, sizes, st["Hq"], *blocks)
    K, V = sp.sepkv_expand_mx(*cache, sizes, *blocks, dtype=DTYPES[st["dtype"]])
    return dict(K=K, V=V, flags=flags, sizes=sizes)


def _own_decode(st):
    import paper_2412_12094_amd as sp

    args = (st["q"], st["Kc"], st["Ks"], st["Vc"], st["Vs"], st["sizes"])
    if st["rope"]:
        return sp.sepattn_decode_rope_mx(*args, st["table"], st["a"], st["s"], st["w"], st["scale"])
    return sp.sepattn_decode_mx(*args, st["a"], st["s"], st["w"], st["scale"])


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


def _normed(x, weight):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()


def _plain_norm(st):
    cos, sin = (t[:, None] for t in _angles(st, _positions(st)))
    q, k, v = _outside_layout(st, st["x"])
    q, k = (_turn(_normed(x, w), cos, sin, st["pairs"]).to(v.dtype) for x, w in zip((q, k), st["weights"]))
    return q, k, v.contiguous()


def _normed_gradient(x, weight, g):
    """g: the gradient of the normed row -> those of the row and of the weight."""
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    u = g * weight.float()
    return r * (u - x * (r * r * (u * x).mean(-1, keepdim=True))), (g * x * r).sum((0, 1, 2), dtype=torch.float64).float()


def _plain_gradient(st):
    cos, sin = (t[:, None] for t in _angles(st, _positions(st)))
    q, k, _ = _outside_layout(st, st["x"])
    dQ, dK, dV = st["grads"]
    dq, dq_weight = _normed_gradient(q, st["weights"][0], _turn(dQ, cos, sin, st["pairs"], True))
    dk, dk_weight = _normed_gradient(k, st["weights"][1], _turn(dK, cos, sin, st["pairs"], True))
    parts = [t.to(dV.dtype).transpose(1, 2) for t in (dq, dk, dV)]
    if st["layout"] == "per_head":
        dx = torch.stack(parts, dim=3)
    elif st["layout"] == "fused":
        dx = torch.cat(parts, dim=2)
    else:
        dx = tuple(t.contiguous() for t in parts)
    return dict(dx=dx, dq_weight=dq_weight, dk_weight=dk_weight)


def _enter(st, sizes, q, k, v, parts):
    """The rows of `parts`' (cache, new row) pairs enter the caches; sizes and flags follow."""
    a, s, w = st["a"], st["s"], st["w"]
    room = st["c"] - a - s
    used = sizes[:, 2] + sizes[:, 3]
    initial = sizes[:, 0] < a
    enters = initial | (used < room)
    window = (sizes[:, 5] + used) % room
    slot = torch.where(initial, sizes[:, 0], a + s + window).long()
    row = torch.arange(st["S"], device="cuda")
    for cache, new in parts:
        cache[row, :, slot] = torch.where(enters[:, None, None], new, cache[row, :, slot])
    flagged = enters & ~initial
    st["flags"][row, window.long()] = torch.where(flagged, st["sep"], st["flags"][row, window.long()])
    sizes[:, 0] += initial
    over = flagged & (sizes[:, 3] + 1 > w)
    sizes[:, 2] += over
    sizes[:, 3] += flagged & ~over


def _turned_token(st):
    cos, sin = (t[:, None] for t in _angles(st, st["pos"]))
    return tuple(_turn(_normed(st[n], w), cos, sin, st["pairs"]).to(st[n].dtype) for n, w in zip(("q", "k"), st["weights"]))


def _plain_token(st):
    sizes = st["sizes"].clone()
    q, k = _turned_token(st)
    _enter(st, sizes, q, k, st["v"], [(st["Kc"], k), (st["Vc"], st["v"])])
    return dict(q=q, Kc=st["Kc"], Vc=st["Vc"], flags=st["flags"], sizes=sizes)


def _slots(sizes, a, s, c):
    """valid [S, c], rank [S, c]: whether a slot holds an entry, and which one, oldest first."""
    j, room = torch.arange(c, device="cuda"), c - a - s
    n_init, n_sep, n_win, head_sep, head_win = (t[:, None] for t in (sizes[:, 0], sizes[:, 1], sizes[:, 2] + sizes[:, 3], sizes[:, 4], sizes[:, 5]))
    k, u = (j - a - head_sep) % max(s, 1), (j - a - s - head_win) % room
    valid = torch.where(j < a, j < n_init, torch.where(j < a + s, k < n_sep, u < n_win))
    return valid, torch.where(j < a, j, torch.where(j < a + s, n_init + k, n_init + n_sep + u))


def _attend(st, q, sizes):
    S, Hq, Hkv, d = st["S"], st["Hq"], st["Hkv"], st["d"]
    valid, rank = _slots(sizes, st["a"], st["s"], st["c"])
    q = q.float().view(S, Hkv, Hq // Hkv, d)
    K = torch.where(valid[:, None, :, None], _from_fp4(_unpacked(st["Kc"]), st["Ks"]), 0.0)
    if st.get("rope"):
        at = st["table"][(valid.sum(1) - 1).clamp(min=0)]
        q = _turn(q, at[:, None, None, 0], at[:, None, None, 1], "half")
        at = st["table"][torch.where(valid, rank, 0).long()]
        K = _turn(K, at[:, None, :, 0], at[:, None, :, 1], "half")
    x = torch.matmul(q, K.transpose(-1, -2)).mul_(st["scale"])
    x.masked_fill_(~valid[:, None, None], float("-inf"))
    m = x.amax(-1)
    p = x.sub_(torch.where(torch.isinf(m), 0.0, m)[..., None]).exp_()
    total = p.sum(-1)
    out = torch.matmul(p, torch.where(valid[:, None, :, None], _from_fp4(_unpacked(st["Vc"]), st["Vs"]), 0.0))
    out = torch.where((total > 0)[..., None], out / total[..., None], 0.0)
    return out.reshape(S, Hq, d).to(st["q"].dtype), (m + total.log()).view(S, Hq)


def _plain_step(st):
    sizes = st["sizes"].clone()
    q, k = _turned_token(st)
    (kn, kb), (vn, vb) = _to_fp4(k), _to_fp4(st["v"])
    _enter(st, sizes, q, k, st["v"], [(st["Kc"], _packed(kn)), (st["Ks"], kb.to(torch.uint8)), (st["Vc"], _packed(vn)), (st["Vs"], vb.to(torch.uint8))])
    out, lse = _attend(st, q, sizes)
    return dict(q=q, out=out, lse=lse, flags=st["flags"], sizes=sizes)


def _plain_admit(st):
    S, L, a, s, w, c, nw = (st[n] for n in ("S", "L", "a", "s", "w", "c", "nw"))
    room, n_init, start, local = c - a - s, min(a, L), L - nw, min(w, nw)
    past = nw - local
    before = st["sep_prefix"][:, start] - st["sep_prefix"][:, n_init]        # separators that are older than the window
    kept = before.clamp(max=s)
    moved = st["sep_prefix"][:, start + past] - st["sep_prefix"][:, start]  # those of the past window
    total = kept + moved
    drop = (total - s).clamp(min=0)
    j = torch.arange(c, device="cuda")
    # entry number k of the separators that have entered stands at k mod s; window entry u stands at u
    k = drop[:, None] + (j - a - drop[:, None]) % max(s, 1)
    listed_at = (st["sep_prefix"][:, start] - kept)[:, None] + k
    sep_from = st["sep_idx"].gather(1, listed_at.clamp(0, L - 1).long())
    u = j - a - s
    source = torch.where(j < a, j, torch.where(j < a + s, sep_from, start + u))
    valid = torch.where(j < a, j < n_init, torch.where(j < a + s, k < total[:, None], (u >= past) & (u < nw)))
    source = torch.where(valid, source, 0).long()

    def take(x):
        rows = x.gather(2, source[:, None, :, None].expand(-1, x.shape[1], -1, x.shape[3]))
        return torch.where(valid[:, None, :, None], _from_fp4(*_to_fp4(rows)), 0.0).to(x.dtype)

    flags = torch.zeros((S, room), dtype=torch.uint8, device="cuda")
    flags[:, :nw] = st["is_sep"][:, start:]
    fixed = torch.ones((S,), dtype=torch.int32, device="cuda")
    sizes = torch.stack([n_init * fixed, total - drop, 0 * fixed, local * fixed, drop % max(s, 1), (past % room) * fixed], dim=1).to(torch.int32)
    return dict(K=take(st["K"]), V=take(st["V"]), flags=flags, sizes=sizes)


def _plain_decode(st):
    return _attend(st, st["q"], st["sizes"])


RUN = {True: dict(norm=_own_norm, gradient=_own_gradient, token=_own_token, step=_own_step, admit=_own_admit, decode=_own_decode),
       False: dict(norm=_plain_norm, gradient=_plain_gradient, token=_plain_token, step=_plain_step, admit=_plain_admit, decode=_plain_decode)}


def run(state):
    return RUN[bool(own)][state["kind"]](state)


# ------------------------------------------------------------------------------------------------
def work(case):
    """Bytes: every input once, every output once; of the caches the valid entries only, in 4 bits 17/32 bytes a value."""
    c, es = case, 4 if case["dtype"] == "fp32" else 2
    d, Hq, Hkv = c["d"], c["Hq"], c["Hkv"]
    if c["kind"] in ("norm", "gradient"):
        tokens, turned = c["B"] * c["L"], c["B"] * c["L"] * (Hq + Hkv)
        given = 0 if c["positions"] == "index" else 4 * tokens
        if c["kind"] == "norm":
            return {"bytes": 2 * es * tokens * (Hq + 2 * Hkv) * d + given + 2 * es * d, "flops": turned * (4.0 * d + 3.0 * c["rotary"])}
        return {"bytes": es * d * (3 * turned + 2 * tokens * Hkv) + given + 2 * (es + 4) * d, "flops": turned * (11.0 * d + 3.0 * c["rotary"])}
    S = c["S"]
    entries = sum(sum(x[:4]) for x in _cache_sizes(c)) if c["kind"] != "admit" else 0
    turn = S * (Hq + Hkv) * (4.0 * d + 3.0 * c.get("rotary", 0))
    if c["kind"] == "token":
        return {"bytes": 2 * es * S * (Hq + 2 * Hkv) * d + S * (4 + 1 + 1 + 48), "flops": turn}
    if c["kind"] == "admit":
        L, n_init, local = c["L"], min(c["a"], c["L"]), min(c["w"], c["nw"])
        rows = n_init + local + min(c["s"], int(c["density"] * max(0, L - n_init - local)))
        return {"bytes": 2 * S * Hkv * d * es * (rows + c["c"]) + S * (L + 24), "flops": 4.0 * S * Hkv * d * rows}
    held, attend = 17 * 2 * Hkv * d * entries // 32, 4.0 * d * Hq * entries
    if c["kind"] == "step":
        return {"bytes": held + es * S * (3 * Hq + 2 * Hkv) * d + S * (4 * Hq + 4 + 1 + 1 + 48), "flops": attend + turn}
    return {"bytes": held + S * Hq * (2 * es * d + 4) + 24 * S + (4 * d * max(sum(x[:4]) for x in _cache_sizes(c)) if c["rope"] else 0),
            "flops": attend + (3.0 * Hkv * d * entries if c["rope"] else 0.0)}


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


def _unit(x, weight):
    """Rows scaled to a root mean square of 1 (but for EPS), by the norm."""
    x = x.double()
    return x * weight.double() / (torch.linalg.vector_norm(x, dim=-1, keepdim=True).square() / x.shape[-1] + EPS).sqrt()


def _exact_norm(st):
    index = torch.arange(st["L"], device="cuda")[None].repeat(st["B"], 1)
    pos = (st["pos"] if st["pos"] is not None else index - (0 if st["doc_start"] is None else st["doc_start"]))[:, None]
    q, k, v = _outside_layout(st, st["x"])
    if st["kind"] == "norm":
        return tuple(_rotation(_unit(x, w), pos, st["freqs"], st["pairs"]) for x, w in zip((q, k), st["weights"])) + (v.double().contiguous(),)
    dQ, dK, dV = st["grads"]
    parts, weights = [], []
    for x, w, g in ((q, st["weights"][0], dQ), (k, st["weights"][1], dK)):
        x, w = x.double().requires_grad_(), w.double().requires_grad_()
        dx, dw = torch.autograd.grad(_unit(x, w), (x, w), _rotation(g, -pos, st["freqs"], st["pairs"]))
        parts.append(dx.detach())
        weights.append(dw)
    parts.append(dV.double())
    B, Hq, Hkv, L, d = st["B"], st["Hq"], st["Hkv"], st["L"], st["d"]
    if st["layout"] == "split":
        dx = tuple(t.permute(0, 2, 1, 3).contiguous() for t in parts)
    else:
        dx = torch.empty((B, L, Hq, 3, d) if st["layout"] == "per_head" else (B, L, Hq + 2 * Hkv, d), dtype=torch.float64, device="cuda")
        for t, to in zip(parts, _outside_layout(st, dx)):
            to.copy_(t)
    return dict(dx=dx, dq_weight=weights[0], dk_weight=weights[1])


def _entries(row, a, s, c):
    """The slots of a cache's entries, oldest first."""
    n_init, n_sep, past, local, head_sep, head_win = row
    room = c - a - s
    return list(range(n_init)) + [a + (head_sep + i) % s for i in range(n_sep)] + [a + s + (head_win + i) % room for i in range(past + local)]


def _place(st):
    """Per sequence the slot that a token enters, or None; the new sizes and flags."""
    a, s, w, room = st["a"], st["s"], st["w"], st["c"] - st["a"] - st["s"]
    sizes, flags, slots = st["sizes"].tolist(), st["flags"].clone(), []
    for i, row in enumerate(sizes):
        count = row[2] + row[3]
        slots.append(None)
        if row[0] < a:
            slots[i], row[0] = row[0], row[0] + 1
        elif count < room:
            place = (row[5] + count) % room
            slots[i] = a + s + place
            flags[i, place] = st["sep"][i]
            row[2 if row[3] == w else 3] += 1
    return slots, _ints(sizes), flags


def _exact_token(st):
    q, k = (_rotation(_unit(st[n], w), st["pos"][:, None], st["freqs"], st["pairs"]) for n, w in zip(("q", "k"), st["weights"]))
    slots, sizes, flags = _place(st)
    Kc, Vc = st["Kc"].double(), st["Vc"].double()
    for i, slot in enumerate(slots):
        if slot is not None:
            Kc[i, :, slot], Vc[i, :, slot] = k[i], st["v"][i].double()
    return dict(q=q, Kc=Kc, Vc=Vc, flags=flags, sizes=sizes)


_EDGES = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)  # between neighbouring magnitudes; a value on the 2nd, 4th, 6th goes up, on the others down


def _rounded(x):
    """float64: what 4 bits leave of rows x."""
    y = x.double().unflatten(-1, (-1, 32))
    big = y.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(big.clamp(min=1e-300)))
    e = torch.where(big > 1.75 * 2.0 ** e, e + 1, e)
    scale = 2.0 ** (e - 2).clamp(-125, 125)
    size = y.abs() / scale
    n = sum((size >= t if i % 2 else size > t).long() for i, t in enumerate(_EDGES))
    at = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")[n]
    return (torch.where(y < 0, -at, at) * scale).flatten(-2)


def _values(code, byte):
    """float64: the values of a cache's packed rows, from the bits of their codes."""
    out = torch.empty((*code.shape[:-1], 2 * code.shape[-1]), dtype=torch.float64, device="cuda")
    for half in range(2):
        n = (code >> (4 * half)) & 15
        e, m = (n >> 1) & 3, (n & 1).double()
        out[..., half::2] = torch.where(e > 0, (1 + m / 2) * 2.0 ** (e.double() - 1), m / 2) * (1 - 2 * (n >> 3).double())
    return (out.unflatten(-1, (-1, 32)) * 2.0 ** (byte.double()[..., None] - 127)).flatten(-2)


def _softmax_over(st, q, sizes, token=None):
    S, Hq, Hkv, d = st["S"], st["Hq"], st["Hkv"], st["d"]
    f = 500000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    out = torch.zeros((S, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((S, Hq), float("-inf"), dtype=torch.float64, device="cuda")
    for i, row in enumerate(sizes.tolist()):
        at = _entries(row, st["a"], st["s"], st["c"])
        if not at:
            continue
        K, V = (_values(st[n][i][:, at], st[b][i][:, at]) for n, b in (("Kc", "Ks"), ("Vc", "Vs")))
        x = q[i].double()
        if token is not None and token[0][i] in at:
            K[:, at.index(token[0][i])], V[:, at.index(token[0][i])] = token[1][i], token[2][i]
        if st.get("rope"):
            K = _rotation(K, torch.arange(len(at), device="cuda")[None], f, "half")
            x = _rotation(x, torch.full((1,), len(at) - 1, device="cuda"), f, "half")
        x = torch.bmm(x.view(Hkv, Hq // Hkv, d), K.transpose(1, 2).contiguous()) * st["scale"]
        out[i] = torch.bmm(torch.softmax(x, dim=-1), V).view(Hq, d)
        lse[i] = torch.logsumexp(x, dim=-1).view(Hq)
    return out, lse


def _exact_step(st):
    turned = [_rotation(_unit(st[n], w), st["pos"][:, None], st["freqs"], st["pairs"]) for n, w in zip(("q", "k"), st["weights"])]
    slots, sizes, flags = _place(st)
    q, k = (t.to(st["q"].dtype) for t in turned)  # what the attention reads, and what is rounded to 4 bits
    out, lse = _softmax_over(st, q, sizes, (slots, _rounded(k), _rounded(st["v"])))
    return dict(q=turned[0], out=out, lse=lse, flags=flags, sizes=sizes)


def _exact_admit(st):
    S, Hkv, L, d, a, s, w, c, nw = (st[n] for n in ("S", "Hkv", "L", "d", "a", "s", "w", "c", "nw"))
    K, V = (torch.zeros((S, Hkv, c, d), dtype=torch.float64, device="cuda") for _ in range(2))
    room, flags, rows = c - a - s, torch.zeros((S, c - a - s), dtype=torch.uint8), []
    for i, sep in enumerate(st["is_sep"].tolist()):
        held = {p: p for p in range(min(a, L))}
        old = [p for p in range(min(a, L), L - nw) if sep[p]]
        old = old[len(old) - min(s, len(old)):]
        window = list(range(L - nw, L))
        for u, p in enumerate(window):
            flags[i, u] = sep[p]
        past = len(window) - min(w, nw)
        entered = old + [p for p in window[:past] if sep[p]]
        gone = max(0, len(entered) - s)
        held.update({a + n % s: p for n, p in enumerate(entered) if n >= gone})
        held.update({a + s + u: p for u, p in enumerate(window) if u >= past})
        rows.append([min(a, L), len(entered) - gone, 0, nw - past, gone % s if s else 0, past % room])
        if held:
            to, at = list(held.keys()), list(held.values())
            K[i, :, to], V[i, :, to] = _rounded(st["K"][i][:, at]), _rounded(st["V"][i][:, at])
    return dict(K=K, V=V, flags=flags.cuda(), sizes=_ints(rows))


def _exact_decode(st):
    return _softmax_over(st, st["q"], st["sizes"])


EXACT = dict(norm=_exact_norm, gradient=_exact_norm, token=_exact_token, step=_exact_step, admit=_exact_admit, decode=_exact_decode)


def exact(case, seed):
    return EXACT[case["kind"]](prepare(case, seed))
