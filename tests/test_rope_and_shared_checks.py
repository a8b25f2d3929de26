"""What the calls for rotary positions and shared prompts refuse before anything is allocated or launched.  Needs no GPU."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")
from torch._subclasses.fake_tensor import FakeTensorMode  # noqa: E402

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced
ODD = ctypes.c_void_p(0x1008)   # 8-byte aligned only


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
def rope(sp, freqs=FAKE, positions=None, doc=None, src=(FAKE, FAKE, FAKE), dst=(FAKE, FAKE, FAKE), to=(None, None, None), frm=(None, None, None), fn="sepattn_rope", **kw):
    v = dict(B=2, Hq=8, Hkv=2, L=16, d=128, rotary_dim=128, interleaved=0, dtype=0)
    v.update(kw)
    p = sp.SepattnRopeParams(*v.values())
    ref = lambda s: None if s is None else ctypes.byref(sp.SepattnStrides(*s))
    pairs = [x for t, s in zip(src + dst, frm + to) for x in (t, ref(s))]
    return getattr(sp.load(), fn)(ctypes.byref(p), freqs, positions, doc, *pairs, None)


@pytest.mark.parametrize("fn", ["sepattn_rope", "sepattn_rope_backward"])
def test_rope_arguments(sp, fn):
    r = lambda **kw: rope(sp, fn=fn, **kw)
    assert r(freqs=None) == 1 and r(src=(None, FAKE, FAKE)) == 1 and r(dst=(FAKE, None, FAKE)) == 1
    assert r(src=(FAKE, FAKE, None)) == 1 and r(dst=(FAKE, FAKE, None)) == 1  # values on one side only
    assert r(B=0) == 2 and r(L=0) == 2 and r(Hq=0) == 2 and r(Hkv=-1) == 2 and r(B=65536) == 2 and r(Hq=65535) == 2
    assert r(d=96) == 4 and r(dtype=2) == 4
    assert r(rotary_dim=0) == 3 and r(rotary_dim=130) == 3 and r(rotary_dim=33) == 3
    assert r(positions=FAKE, doc=FAKE) == 3
    assert r(src=(ODD, FAKE, FAKE)) == 3 and r(dst=(FAKE, FAKE, ODD)) == 3 and r(freqs=ctypes.c_void_p(0x1004)) == 3
    for s in ((-2048, 128, 1024), (1, 128, 1024), (16384, 132, 1024), (16384, 128, 1028)):  # negative, not a multiple of 8
        assert r(frm=(s, None, None)) == 3
    assert r(frm=((1 << 41, 128, 1024), None, None)) == 2
    assert r(frm=((128, 128, 1 << 40), None, None), L=1 << 30, B=1, Hq=1) == 2  # a span that 64 bits do not hold
    # outputs whose rows overlap
    for s in ((0, 2048, 128), (16 * 8 * 128, 0, 128), (16 * 8 * 128, 2048, 120), (16 * 8 * 128 - 8, 2048, 128), (128, 128, 2048), (16384, 1024, 128)):
        assert r(to=(s, None, None)) == 3, s
    assert sp.load().sepattn_rope(None, FAKE, None, None, *[FAKE, None] * 6, None) == 1


def test_rope_frequencies(sp):
    f = sp.sepattn_rope_frequencies(6, 10000.0)
    assert f.dtype == torch.float64 and all(abs(float(x) / 10000.0 ** (-i / 3) - 1) < 1e-15 for i, x in enumerate(f))
    half = sp.sepattn_rope_frequencies(6, 10000.0, factor=2.0)
    assert torch.equal(half * 2.0, f)
    parts = sp.sepattn_rope_frequencies(64, 10000.0, 4.0, 1.0, 32.0, 4096)
    plain = sp.sepattn_rope_frequencies(64, 10000.0)
    turns = 4096 * plain / (2 * math.pi)
    assert torch.equal(parts[turns >= 32], plain[turns >= 32]) and torch.equal(parts[turns <= 1] * 4, plain[turns <= 1])
    between = (turns > 1) & (turns < 32)
    assert between.any() and (parts[between] < plain[between]).all() and (parts[between] > plain[between] / 4).all()
    lib, out = sp.load(), (ctypes.c_double * 64)()
    call = lambda *a: lib.sepattn_rope_frequencies(*a, out)
    assert call(0, 1e4, 1.0, 1.0, 4.0, 0) == 3 and call(7, 1e4, 1.0, 1.0, 4.0, 0) == 3 and call(130, 1e4, 1.0, 1.0, 4.0, 0) == 3
    assert call(8, 1.0, 1.0, 1.0, 4.0, 0) == 3 and call(8, float("nan"), 1.0, 1.0, 4.0, 0) == 3
    assert call(8, 1e4, 0.5, 1.0, 4.0, 0) == 3 and call(8, 1e4, float("nan"), 1.0, 4.0, 0) == 3 and call(8, 1e4, 1.0, 1.0, 4.0, -1) == 3
    assert call(8, 1e4, 2.0, 4.0, 4.0, 100) == 3 and call(8, 1e4, 2.0, -1.0, 4.0, 100) == 3 and call(8, 1e4, 2.0, 4.0, 4.0, 0) == 0
    assert lib.sepattn_rope_frequencies(8, 1e4, 1.0, 1.0, 4.0, 0, None) == 1
    with pytest.raises(sp.SepattnError):
        sp.sepattn_rope_frequencies(9, 1e4)
    table = lambda n=4, d=64, f=FAKE, t=FAKE: lib.sepkv_rope_table_frequencies(n, d, f, t, None)
    assert table(f=None) == 1 and table(t=None) == 1 and table(n=0) == 2 and table(d=32) == 4 and table(t=ODD) == 3


def kv(sp, **kw):
    v = dict(S=2, Hq=8, Hkv=2, d=128, a=4, s=64, w=32, c=200, scale=0.1, dtype=0)
    v.update(kw)
    return sp.SepkvParams(*v.values())


def test_cache_calls(sp):
    lib = sp.load()
    app = lambda p=None, rotary=64, f=FAKE, q=FAKE, o=FAKE: lib.sepkv_append_rope(
        ctypes.byref(p or kv(sp)), rotary, 0, f, FAKE, q, FAKE, FAKE, FAKE, o, FAKE, FAKE, FAKE, FAKE, None)
    assert app(f=None) == 1 and app(q=None) == 1 and app(o=None) == 1 and app(q=ODD) == 3 and app(o=ODD) == 3
    assert app(rotary=0) == 3 and app(rotary=130) == 3 and app(rotary=31) == 3 and app(kv(sp, w=0)) == 3 and app(kv(sp, d=80)) == 4
    grp = lambda of=FAKE, S=4, G=2: lib.sepkv_group_sequences(of, S, G, FAKE, FAKE, None)
    assert grp(of=None) == 1 and grp(S=0) == 2 and grp(G=0) == 2 and grp(S=65536) == 2 and grp(G=65536) == 2
    enc = lambda p=None, n=200, k=FAKE, o=FAKE: lib.sepkv_rope_cache(ctypes.byref(p or kv(sp)), FAKE, FAKE, n, k, o, None)
    assert enc(k=None) == 1 and enc(o=None) == 1 and enc(n=199) == 2 and enc(o=ODD) == 3 and enc(kv(sp, S=0)) == 2


def test_shared_decode(sp):
    lib = sp.load()
    need = lib.sepattn_decode_shared_workspace_bytes(ctypes.byref(kv(sp)), ctypes.byref(kv(sp, S=3)))
    assert need > 0 and need % 256 == 0

    def call(p=None, pp=None, q=FAKE, kp=FAKE, of=FAKE, ws=FAKE, n=need, rope=None):
        p, pp = ctypes.byref(p or kv(sp)), ctypes.byref(pp or kv(sp, S=3))
        args = (p, pp, q, FAKE, FAKE, FAKE, kp, FAKE, FAKE, of, FAKE, FAKE)
        if rope is None:
            return lib.sepattn_decode_shared(*args, FAKE, None, ws, n, None)
        return lib.sepattn_decode_shared_rope(*args, *rope, FAKE, None, ws, n, None)

    assert call(q=None) == 1 and call(kp=None) == 1 and call(of=None) == 1 and call(kp=ODD) == 3
    assert call(pp=kv(sp, Hkv=4)) == 2 and call(pp=kv(sp, Hq=16)) == 2 and call(pp=kv(sp, d=64)) == 4 and call(pp=kv(sp, dtype=1)) == 4
    assert call(pp=kv(sp, c=100)) == 3 and call(p=kv(sp, S=0)) == 2 and call(p=kv(sp, scale=float("nan"))) == 3
    assert call(ws=None) == 5 and call(n=need - 1) == 5 and call(ws=ctypes.c_void_p(0x1010)) == 5
    assert call(rope=(None, 400)) == 1 and call(rope=(FAKE, 399)) == 2 and call(rope=(ODD, 400)) == 3
    assert lib.sepattn_decode_shared_workspace_bytes(ctypes.byref(kv(sp)), ctypes.byref(kv(sp, d=64))) == 0
    assert lib.sepattn_decode_shared(None, ctypes.byref(kv(sp)), *[FAKE] * 11, None, FAKE, need, None) == 1


# ---- the binding ---------------------------------------------------------------------------------------
def test_binding_of_rope(sp):
    f, q, k = fake(32, dtype=torch.float64), fake(2, 8, 16, 64), fake(2, 2, 16, 64)
    for args, kw in [
        ((q, k[:, :, :15], None, f), {}), ((q, fake(2, 2, 16, 128), None, f), {}), ((q, k, fake(2, 4, 16, 64), f), {}),
        ((q, fake(2, 2, 16, 64, dtype=torch.float32), None, f), {}), ((q[0], k, None, f), {}), ((q, k, None, fake(32, dtype=torch.float32)), {}),
        ((q, k, None, fake(2, 16, dtype=torch.float64)), {}), ((q, k, None, fake(32, dtype=torch.float64, device="cpu")), {}),
        ((q.transpose(2, 3), k.transpose(2, 3), None, f), {}), ((fake(2, 8, 16, 64, device="cpu"), k, None, f), {}),
        ((q, k, None, f), dict(positions=fake(16, dtype=torch.int32))), ((q, k, None, f), dict(positions=fake(2, 16, dtype=torch.int64))),
        ((q, k, None, f), dict(doc_start=fake(2, 15, dtype=torch.int32))), ((q, k, None, f), dict(out=(q, k))), ((q, k, None, f), dict(out=(q, k, k))),
        ((q, k, k, f), dict(out=(q, k, None))), ((q, k, None, f), dict(out=(k, q, None))),
        ((fake(2, 8, 16, 64, dtype=torch.float16), fake(2, 2, 16, 64, dtype=torch.float16), None, f), {}),
    ]:
        for call in (sp.sepattn_rope, sp.sepattn_rope_backward):
            with pytest.raises((AssertionError, ValueError, TypeError)):
                call(*args, **kw)
    with pytest.raises(ValueError, match="different devices"):
        sp.sepattn_rope(q, fake(2, 2, 16, 64, device="cuda:1"), None, f, out=(q, k, None))


def test_binding_of_the_cache_calls(sp):
    i32, u8 = torch.int32, torch.uint8
    S, Hq, Hkv, d, c = 3, 8, 2, 64, 40
    base = dict(q=fake(S, Hq, d), k=fake(S, Hkv, d), v=fake(S, Hkv, d), sep=fake(S, dtype=u8), pos=fake(S, dtype=i32), f=fake(16, dtype=torch.float64),
                Kc=fake(S, Hkv, c, d), Vc=fake(S, Hkv, c, d), flags=fake(S, 28, dtype=u8), sizes=fake(S, 6, dtype=i32))
    for name, value in [("q", fake(S, Hq, 128)), ("q", fake(S, Hq * d)), ("k", fake(S, Hkv + 1, d)), ("v", fake(S, Hkv, d, dtype=torch.float32)), ("sep", fake(S + 1, dtype=u8)),
                        ("pos", fake(S, 1, dtype=i32)), ("pos", fake(S, dtype=torch.int64)), ("f", fake(16)), ("Kc", fake(S + 1, Hkv, c, d)), ("Vc", fake(S, Hkv, c + 1, d)),
                        ("flags", fake(S, 27, dtype=u8)), ("sizes", fake(S - 1, 6, dtype=i32)), ("sizes", fake(S, 4, dtype=i32)), ("k", fake(S, Hkv, d, device="cuda:1"))]:
        with pytest.raises((AssertionError, ValueError, TypeError)):
            sp.sepkv_append_rope(*{**base, name: value}.values(), 4, 8, 8, out=base["q"])
    with pytest.raises(AssertionError, match="out"):
        sp.sepkv_append_rope(*base.values(), 4, 8, 8, out=fake(S, Hq, d, dtype=torch.float32))
    for of, out in [(fake(4, dtype=torch.int64), None), (fake(2, 2, dtype=i32), None), (fake(4, dtype=i32), (fake(3, dtype=i32), fake(4, dtype=i32))),
                    (fake(4, dtype=i32), (fake(4, dtype=i32), fake(3, dtype=i32)))]:
        with pytest.raises(AssertionError):
            sp.sepkv_group_sequences(of, 3, out=out)
    table = fake(c, 2, d // 2, dtype=torch.float32)
    for args, kw in [((base["Kc"], base["sizes"][:2], table), {}), ((base["Kc"], base["sizes"], fake(c, d, dtype=torch.float32)), {}),
                     ((base["Kc"], base["sizes"], fake(c, 2, d, dtype=torch.float32)), {}), ((base["Kc"], base["sizes"], table), dict(out=fake(S, Hkv, c + 1, d)))]:
        with pytest.raises((AssertionError, ValueError)):
            sp.sepkv_rope_cache(*args, 4, 8, 8, **kw)


def test_binding_of_the_shared_decode(sp):
    i32 = torch.int32
    S, G, Hq, Hkv, d, c, pc = 3, 2, 8, 2, 64, 40, 100
    base = dict(q=fake(S, Hq, d), Kc=fake(S, Hkv, c, d), Vc=fake(S, Hkv, c, d), sizes=fake(S, 6, dtype=i32), a=4, s=8, w=8, Kp=fake(G, Hkv, pc, d),
                Vp=fake(G, Hkv, pc, d), psizes=fake(G, 6, dtype=i32), pa=0, ps=0, pw=1, of=fake(S, dtype=i32), start=fake(G + 1, dtype=i32), seq=fake(S, dtype=i32))
    for name, value in [("q", fake(S, Hq, 128)), ("q", fake(S + 1, Hq, d)), ("Kc", fake(S, Hkv, c, d, dtype=torch.float32)), ("Vc", fake(S, Hkv, c - 1, d)),
                        ("sizes", fake(S + 1, 6, dtype=i32)), ("Kp", fake(G, Hkv + 1, pc, d)), ("Kp", fake(G, Hkv, pc, 128)), ("Vp", fake(G, Hkv, pc, d, dtype=torch.float32)),
                        ("psizes", fake(G + 1, 6, dtype=i32)), ("of", fake(S + 1, dtype=i32)), ("of", fake(S, dtype=torch.int64)), ("start", fake(G, dtype=i32)),
                        ("seq", fake(S - 1, dtype=i32)), ("Vp", fake(G, Hkv, pc, d, device="cuda:1"))]:
        with pytest.raises((AssertionError, ValueError, TypeError)):
            sp.sepattn_decode_shared(*{**base, name: value}.values(), 0.1, out=(base["q"], None))
    with pytest.raises(AssertionError, match="rope_table"):
        sp.sepattn_decode_shared_rope(*base.values(), fake(200, 2, d, dtype=torch.float32), 0.1)
    with pytest.raises(AssertionError, match="lse"):
        sp.sepattn_decode_shared(*base.values(), 0.1, out=(base["q"], fake(S, Hq - 1, dtype=torch.float32)))
    with pytest.raises(ValueError, match="number of tensors"):
        sp.sepattn_decode_shared(*base.values(), 0.1, out=(base["q"],))
