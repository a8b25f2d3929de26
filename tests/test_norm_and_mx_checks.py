"""What the calls for normed rows and for the cache in 4 bits refuse before anything is allocated or launched.  Needs no GPU."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
from torch._subclasses.fake_tensor import FakeTensorMode  # noqa: E402

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced
ODD = ctypes.c_void_p(0x1008)   # 8-byte aligned only
NULL, SHAPE, PARAM, DTYPE, WORKSPACE = 1, 2, 3, 4, 5
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def sp():
    import os

    import paper_2412_12094_amd as sp_

    if not os.path.exists(sp_.LIB_PATH):
        from paper_2412_12094_amd import build

        build.build()
    sp_.load()
    from paper_2412_12094_amd import binding

    binding._native()
    return sp_


def fake(*shape, dtype=torch.bfloat16, device="cuda"):
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device=device)


# ---- the C entry points --------------------------------------------------------------------------
def norm_params(sp, **kw):
    v = dict(B=2, Hq=8, Hkv=2, L=16, d=128, rotary_dim=128, interleaved=0, dtype=0, weight_dtype=0, eps=1e-6)
    v.update(kw)
    return sp.SepattnNormRopeParams(*v.values())


def strided(sp, tensors, strides):
    ref = lambda s: None if s is None else ctypes.byref(sp.SepattnStrides(*s))
    return [x for t, s in zip(tensors, strides) for x in (t, ref(s))]


def norm_rope(sp, weights=(FAKE, FAKE), freqs=FAKE, positions=None, doc=None, src=(FAKE,) * 3, dst=(FAKE,) * 3, frm=(None,) * 3, to=(None,) * 3, **kw):
    return sp.load().sepattn_norm_rope(ctypes.byref(norm_params(sp, **kw)), *weights, freqs, positions, doc, *strided(sp, src + dst, frm + to), None)


def backward(sp, weights=(FAKE, FAKE), freqs=FAKE, positions=None, doc=None, x=(FAKE,) * 2, src=(FAKE,) * 3, dst=(FAKE,) * 3, xs=(None,) * 2,
             frm=(None,) * 3, to=(None,) * 3, dw=(FAKE, FAKE), ws=FAKE, n=None, **kw):
    lib, p = sp.load(), norm_params(sp, **kw)
    n = lib.sepattn_norm_rope_backward_workspace_bytes(ctypes.byref(norm_params(sp))) if n is None else n
    return lib.sepattn_norm_rope_backward(ctypes.byref(p), *weights, freqs, positions, doc, *strided(sp, x + src + dst, xs + frm + to), *dw, ws, n, None)


@pytest.mark.parametrize("call", [norm_rope, backward])
def test_norm_rope_arguments(sp, call):
    r = lambda **kw: call(sp, **kw)
    assert r(freqs=None) == NULL and r(src=(None, FAKE, FAKE)) == NULL and r(dst=(FAKE, None, FAKE)) == NULL
    assert r(src=(FAKE, FAKE, None)) == NULL and r(dst=(FAKE, FAKE, None)) == NULL  # values on one side only
    assert r(B=0) == SHAPE and r(L=0) == SHAPE and r(Hq=0) == SHAPE and r(Hkv=-1) == SHAPE and r(B=65536) == SHAPE and r(Hq=65535) == SHAPE
    assert r(B=65535, L=1 << 20, Hq=1, Hkv=1) == SHAPE
    assert r(d=96) == DTYPE and r(dtype=2) == DTYPE and r(weight_dtype=2) == DTYPE and r(weight_dtype=-1) == DTYPE
    assert r(rotary_dim=-2) == PARAM and r(rotary_dim=130) == PARAM and r(rotary_dim=33) == PARAM
    assert r(eps=-1e-6) == PARAM and r(eps=NAN) == PARAM and r(eps=INF) == PARAM
    assert r(positions=FAKE, doc=FAKE) == PARAM
    assert r(src=(ODD, FAKE, FAKE)) == PARAM and r(dst=(FAKE, FAKE, ODD)) == PARAM and r(freqs=ctypes.c_void_p(0x1004)) == PARAM
    assert r(weights=(ctypes.c_void_p(0x1001), FAKE)) == PARAM and r(weights=(FAKE, ctypes.c_void_p(0x1002)), weight_dtype=1) == PARAM
    for s in ((-2048, 128, 1024), (1, 128, 1024), (16384, 132, 1024), (16384, 128, 1028)):  # negative, not a multiple of 8
        assert r(frm=(s, None, None)) == PARAM
    for s in ((0, 2048, 128), (16 * 8 * 128, 0, 128), (16 * 8 * 128 - 8, 2048, 128)):  # outputs whose rows overlap
        assert r(to=(s, None, None)) == PARAM, s


def test_norm_rope_backward_alone(sp):
    r = lambda **kw: backward(sp, **kw)
    lib = sp.load()
    need = lib.sepattn_norm_rope_backward_workspace_bytes(ctypes.byref(norm_params(sp)))
    assert need > 0 and need % 256 == 0
    assert lib.sepattn_norm_rope_backward_workspace_bytes(ctypes.byref(norm_params(sp, rotary_dim=0))) == need
    assert lib.sepattn_norm_rope_backward_workspace_bytes(ctypes.byref(norm_params(sp, d=96))) == 0
    assert lib.sepattn_norm_rope_backward_workspace_bytes(None) == 0
    assert r(x=(None, FAKE)) == NULL and r(x=(FAKE, None)) == NULL and r(x=(ODD, FAKE)) == PARAM and r(xs=((1, 128, 1024), None)) == PARAM
    assert r(ws=None) == WORKSPACE and r(n=need - 1) == WORKSPACE and r(ws=ctypes.c_void_p(0x1010)) == WORKSPACE
    assert r(dw=(ctypes.c_void_p(0x1002), FAKE)) == PARAM and r(dw=(None, FAKE), ws=None) == WORKSPACE


def kv(sp, **kw):
    v = dict(S=2, Hq=8, Hkv=2, d=128, a=4, s=64, w=32, c=200, scale=0.1, dtype=0)
    v.update(kw)
    return sp.SepkvParams(*v.values())


@pytest.mark.parametrize("norm,mx", [(True, False), (False, True), (True, True)])
def test_tokens(sp, norm, mx):
    fn = getattr(sp.load(), "sepkv_append_" + ("norm_" if norm else "") + "rope" + ("_mx" if mx else ""))

    def r(p=None, rotary=64, eps=1e-6, wt=0, wq=FAKE, wk=FAKE, f=FAKE, pos=FAKE, q=FAKE, k=FAKE, v=FAKE, sep=FAKE, o=FAKE, cache=None, win=FAKE, sizes=FAKE):
        head = (ctypes.byref(p or kv(sp)), rotary, 0) + ((eps, wt, wq, wk) if norm else ())
        return fn(*head, f, pos, q, k, v, sep, o, *(cache or (FAKE,) * (4 if mx else 2)), win, sizes, None)

    for name in ("f", "pos", "q", "k", "v", "sep", "o", "win", "sizes"):
        assert r(**{name: None}) == NULL, name
    for name in ("q", "k", "v", "o"):
        assert r(**{name: ODD}) == PARAM, name
    assert r(rotary=130) == PARAM and r(rotary=31) == PARAM and r(rotary=-2) == PARAM and r(p=kv(sp, w=0)) == PARAM and r(p=kv(sp, d=80)) == DTYPE
    n = 4 if mx else 2
    for i in range(n):
        assert r(cache=tuple(None if j == i else FAKE for j in range(n))) == NULL
    assert r(cache=(ODD,) + (FAKE,) * (n - 1)) == PARAM
    if mx:
        assert r(cache=(FAKE, ctypes.c_void_p(0x1002), FAKE, FAKE)) == PARAM  # scales of d = 128: words
    if norm:
        assert r(eps=-1.0) == PARAM and r(eps=NAN) == PARAM and r(wt=3) == DTYPE and r(wq=ctypes.c_void_p(0x1001)) == PARAM
        assert r(rotary=0, f=None, pos=None, q=None) == NULL  # no frequencies are needed, a query is
    else:
        assert r(rotary=0) == PARAM


def test_mx_cache_calls(sp):
    lib = sp.load()
    word = ctypes.c_void_p(0x1002)

    def over(fn, args, **special):
        """Each argument NULL in turn."""
        for i, a in enumerate(args):
            if a is FAKE:
                assert fn(ctypes.byref(kv(sp)), *(None if j == i else x for j, x in enumerate(args))) == NULL, (fn, i)
        assert fn(None, *args) == NULL
        assert fn(ctypes.byref(kv(sp, c=100)), *args) == PARAM and fn(ctypes.byref(kv(sp, d=32)), *args) == DTYPE and fn(ctypes.byref(kv(sp, S=0)), *args) == SHAPE

    over(lib.sepkv_append_mx, (FAKE,) * 9 + (None,))
    over(lib.sepkv_evict_window_mx, (FAKE,) * 6 + (None,))
    over(lib.sepkv_expand_mx, (FAKE,) * 7 + (None,))
    app = lambda *a: lib.sepkv_append_mx(ctypes.byref(kv(sp)), *a, None)
    assert app(ODD, *[FAKE] * 8) == PARAM and app(FAKE, FAKE, FAKE, ODD, *[FAKE] * 5) == PARAM and app(FAKE, FAKE, FAKE, FAKE, word, *[FAKE] * 4) == PARAM
    assert lib.sepkv_evict_window_mx(ctypes.byref(kv(sp)), FAKE, FAKE, ODD, FAKE, FAKE, FAKE, None) == PARAM
    big = kv(sp, S=16384, Hq=2, Hkv=2)
    assert lib.sepkv_expand_mx(ctypes.byref(big), *[FAKE] * 7, None) == SHAPE
    assert lib.sepkv_expand_mx(ctypes.byref(kv(sp)), *[FAKE] * 5, ODD, FAKE, None) == PARAM
    for fn in (lib.sepkv_fill_from_prefill_mx, lib.sepkv_fill_from_prefill_mx_zeroed):
        f = lambda p=None, L=300, nw=100, K=FAKE, sep=FAKE, cap=300, cache=(FAKE,) * 4, win=FAKE, sizes=FAKE: fn(
            ctypes.byref(p or kv(sp)), L, nw, K, FAKE, sep, FAKE, cap, FAKE, *cache, win, sizes, None)
        assert f(K=None) == NULL and f(sep=None) == NULL and f(win=None) == NULL and f(sizes=None) == NULL
        for i in range(4):
            assert f(cache=tuple(None if j == i else FAKE for j in range(4))) == NULL
        assert f(K=ODD) == PARAM and f(cache=(ODD, FAKE, FAKE, FAKE)) == PARAM and f(cache=(FAKE, FAKE, FAKE, word)) == PARAM
        assert f(L=0) == SHAPE and f(cap=0) == 6 and f(nw=-1) == PARAM and f(nw=133) == PARAM and f(L=50, nw=47) == PARAM and f(p=big) == SHAPE


@pytest.mark.parametrize("rope", [False, True])
def test_mx_decode(sp, rope):
    lib = sp.load()
    need = lib.sepattn_decode_mx_workspace_bytes(ctypes.byref(kv(sp)))
    assert need > 0 and need % 256 == 0 and lib.sepattn_decode_mx_workspace_bytes(ctypes.byref(kv(sp, d=32))) == 0

    def r(p=None, q=FAKE, cache=(FAKE,) * 4, sizes=FAKE, table=(FAKE, 200), out=FAKE, ws=FAKE, n=need):
        p = ctypes.byref(p or kv(sp))
        if rope:
            return lib.sepattn_decode_rope_mx(p, q, *cache, sizes, *table, out, None, ws, n, None)
        return lib.sepattn_decode_mx(p, q, *cache, sizes, out, None, ws, n, None)

    assert r(q=None) == NULL and r(sizes=None) == NULL and r(out=None) == NULL and r(q=ODD) == PARAM and r(out=ODD) == PARAM
    for i in range(4):
        assert r(cache=tuple(None if j == i else FAKE for j in range(4))) == NULL
    assert r(cache=(FAKE, FAKE, ODD, FAKE)) == PARAM and r(cache=(FAKE, FAKE, FAKE, ctypes.c_void_p(0x1002))) == PARAM
    assert r(p=kv(sp, S=0)) == SHAPE and r(p=kv(sp, scale=NAN)) == PARAM and r(p=kv(sp, dtype=2)) == DTYPE and r(p=kv(sp, Hq=9)) == SHAPE
    assert r(ws=None) == WORKSPACE and r(n=need - 1) == WORKSPACE and r(ws=ctypes.c_void_p(0x1010)) == WORKSPACE
    if rope:
        assert r(table=(None, 200)) == NULL and r(table=(FAKE, 199)) == SHAPE and r(table=(ODD, 200)) == PARAM


# ---- the binding ---------------------------------------------------------------------------------------
ERRORS = (AssertionError, ValueError, TypeError)
F64, F32, U8, I32 = torch.float64, torch.float32, torch.uint8, torch.int32


def test_binding_of_norm_rope(sp):
    f, q, k, w = fake(32, dtype=F64), fake(2, 8, 16, 64), fake(2, 2, 16, 64), fake(64)
    base = dict(q=q, k=k, v=None, wq=w, wk=w, f=f, eps=1e-6)
    bad = [("k", k[:, :, :15]), ("k", fake(2, 2, 16, 128)), ("v", fake(2, 4, 16, 64)), ("k", fake(2, 2, 16, 64, dtype=F32)), ("q", q[0]), ("f", fake(32, dtype=F32)),
           ("f", fake(2, 16, dtype=F64)), ("f", fake(32, dtype=F64, device="cpu")), ("q", fake(2, 8, 16, 64, device="cpu")), ("wq", fake(128)), ("wk", fake(1, 64)),
           ("wq", fake(64, dtype=F32)), ("wk", fake(64, dtype=F64)), ("wq", fake(64, device="cpu")), ("eps", "x")]
    for name, value in bad:
        with pytest.raises(ERRORS):
            sp.sepattn_norm_rope(*{**base, name: value}.values())
        b = {**base, name: value}
        with pytest.raises(ERRORS):
            sp.sepattn_norm_rope_backward(q, k, *b.values())
    for kw in [dict(positions=fake(16, dtype=I32)), dict(positions=fake(2, 16, dtype=torch.int64)), dict(doc_start=fake(2, 15, dtype=I32)), dict(out=(q, k)),
               dict(out=(q, k, k)), dict(out=(k, q, None))]:
        with pytest.raises(ERRORS):
            sp.sepattn_norm_rope(*base.values(), **kw)
        with pytest.raises(ERRORS):
            sp.sepattn_norm_rope_backward(q, k, *base.values(), **kw)
    for args, kw in [((q[:, :7], k), {}), ((q, k.float()), {}), ((q, fake(2, 2, 16, 64, device="cpu")), {}), ((q, k), dict(out_weights=(w, w))),
                     ((q, k), dict(out_weights=(fake(64, dtype=F32),))), ((q, k), dict(out_weights=(fake(32, dtype=F32), None))), ((q, k), dict(ws=fake(4, dtype=U8, device="cpu")))]:
        with pytest.raises(ERRORS):
            sp.sepattn_norm_rope_backward(*args, *base.values(), out=(q, k, None), **kw)
    with pytest.raises(ValueError, match="different devices"):
        sp.sepattn_norm_rope(q, fake(2, 2, 16, 64, device="cuda:1"), None, w, w, f, 1e-6, out=(q, k, None))


def test_binding_of_the_mx_cache(sp):
    S, Hq, Hkv, d, c = 3, 8, 2, 64, 40
    row = dict(q=fake(S, Hq, d), k=fake(S, Hkv, d), v=fake(S, Hkv, d), sep=fake(S, dtype=U8))
    turn, norm = dict(pos=fake(S, dtype=I32)), dict(wq=fake(d), wk=fake(d))
    f = dict(f=fake(16, dtype=F64))
    cache = dict(Kc=fake(S, Hkv, c, 32, dtype=U8), Ks=fake(S, Hkv, c, 2, dtype=U8), Vc=fake(S, Hkv, c, 32, dtype=U8), Vs=fake(S, Hkv, c, 2, dtype=U8))
    state = dict(flags=fake(S, 28, dtype=U8), sizes=fake(S, 6, dtype=I32))
    wrong_cache = [("Kc", fake(S, Hkv, c, 32)), ("Kc", fake(S, Hkv, c + 1, 32, dtype=U8)), ("Kc", fake(S, Hkv, c, 64, dtype=U8)), ("Ks", fake(S, Hkv, c, 4, dtype=U8)),
                   ("Vs", fake(S, Hkv, c, 2, dtype=torch.int8)), ("Vc", fake(S, Hkv, c, 32, dtype=U8, device="cpu")), ("Vc", fake(S, Hkv, c, 32, dtype=U8, device="cuda:1"))]
    wrong_state = [("flags", fake(S, 27, dtype=U8)), ("sizes", fake(S - 1, 6, dtype=I32)), ("sizes", fake(S, 4, dtype=I32))]
    wrong_row = [("k", fake(S, Hkv + 1, d)), ("v", fake(S, Hkv, d, dtype=F32)), ("sep", fake(S + 1, dtype=U8))]
    wrong_q = [("q", fake(S, Hq, 128)), ("q", fake(S, Hq * d)), ("q", fake(S + 1, Hq, d)), ("pos", fake(S, 1, dtype=I32)), ("f", fake(16))]
    wrong_norm = [("wq", fake(d + 1)), ("wk", fake(d, dtype=F32)), ("wk", fake(d, dtype=F64))]
    calls = [
        (lambda v: sp.sepkv_append_rope_mx(*v, 4, 8, 8, out=row["q"]), {**row, **turn, **f, **cache, **state}, wrong_cache + wrong_state + wrong_row + wrong_q),
        (lambda v: sp.sepkv_append_norm_rope_mx(*v, 4, 8, 8, out=row["q"]), {**row, **turn, **norm, **f, "eps": 1e-6, **cache, **state},
         wrong_cache + wrong_state + wrong_row + wrong_q + wrong_norm),
        (lambda v: sp.sepkv_append_mx(*v, Hq, 4, 8, 8), {**{n: row[n] for n in ("k", "v", "sep")}, **cache, **state}, wrong_cache + wrong_state + wrong_row),
        (lambda v: sp.sepkv_evict_window_mx(*v, Hq, 4, 8, 8), {**cache, **state}, wrong_cache + wrong_state),
        (lambda v: sp.sepkv_expand_mx(*v, 4, 8, 8), {**cache, "sizes": state["sizes"]}, wrong_cache + wrong_state[1:]),
        (lambda v: sp.sepattn_decode_mx(*v, 4, 8, 8, 0.1), {"q": row["q"], **cache, "sizes": state["sizes"]}, wrong_cache + wrong_state[1:] + wrong_q[:3]),
    ]
    plain = dict(Kc=fake(S, Hkv, c, d), Vc=fake(S, Hkv, c, d))
    calls.append((lambda v: sp.sepkv_append_norm_rope(*v, 4, 8, 8, out=row["q"]), {**row, **turn, **norm, **f, "eps": 1e-6, **plain, **state},
                  wrong_state + wrong_row + wrong_q + wrong_norm + [("Kc", fake(S + 1, Hkv, c, d)), ("Vc", fake(S, Hkv, c + 1, d))]))
    for call, base, wrong in calls:
        for name, value in wrong:
            with pytest.raises(ERRORS):
                call({**base, name: value}.values())
    with pytest.raises(AssertionError, match="rope_table"):
        sp.sepattn_decode_rope_mx(row["q"], *cache.values(), state["sizes"], fake(c, 2, d, dtype=F32), 4, 8, 8, 0.1)
    with pytest.raises(AssertionError, match="lse"):
        sp.sepattn_decode_mx(row["q"], *cache.values(), state["sizes"], 4, 8, 8, 0.1, out=(row["q"], fake(S, Hq - 1, dtype=F32)))
    with pytest.raises(TypeError):
        sp.sepkv_expand_mx(*cache.values(), state["sizes"], 4, 8, 8, dtype=torch.float16)
    with pytest.raises(AssertionError, match="out"):
        sp.sepkv_expand_mx(*cache.values(), state["sizes"], 4, 8, 8, out=(fake(S, Hkv, c, d), fake(S, Hkv, c, d, dtype=F32)))


def test_binding_of_the_mx_hand_over(sp):
    S, Hkv, L, d = 2, 2, 50, 64
    base = dict(K=fake(S, Hkv, L, d), V=fake(S, Hkv, L, d), sep=fake(S, L, dtype=U8), idx=fake(S, L, dtype=I32), pre=fake(S, L + 1, dtype=I32))
    for name, value in [("V", fake(S, Hkv, L, 128)), ("V", fake(S, Hkv, L, d, dtype=F32)), ("sep", fake(S, L + 1, dtype=U8)), ("idx", fake(L, dtype=I32)), ("pre", fake(S, L, dtype=I32)),
                        ("K", fake(Hkv, L, d)), ("K", fake(S, Hkv, L, 96)), ("pre", fake(S, L + 1, dtype=torch.int64))]:
        with pytest.raises(ERRORS):
            sp.sepkv_fill_from_prefill_mx(*{**base, name: value}.values(), 8, 4, 8, 8, 40, 20)
    u8 = lambda *s: fake(*s, dtype=U8)
    good = (u8(S, Hkv, 40, 32), u8(S, Hkv, 40, 2), u8(S, Hkv, 40, 32), u8(S, Hkv, 40, 2), u8(S, 28), fake(S, 6, dtype=I32))
    for i, value in [(0, u8(S, Hkv, 41, 32)), (1, u8(S, Hkv, 40, 4)), (4, u8(S, 27)), (5, fake(S, 4, dtype=I32)), (2, fake(S, Hkv, 40, 32))]:
        with pytest.raises(ERRORS):
            sp.sepkv_fill_from_prefill_mx(*base.values(), 8, 4, 8, 8, 40, 20, out=good[:i] + (value,) + good[i + 1:])
    with pytest.raises(AssertionError, match="out"):  # a cache of another shape than the call's
        sp.sepkv_fill_from_prefill_mx(*base.values(), 8, 4, 8, 8, 41, 20, out=good)
    with pytest.raises(AssertionError, match="blocks"):
        sp.sepkv_fill_from_prefill_mx(*base.values(), 8, 4, 36, 8, 40, 20)
