"""The hand-over into a cache in 4 bits that writes the whole of its buffers: what the plain form writes, bit for bit, and 0 everywhere else, over memory
that holds something else; the plain form leaves what it does not use.  Needs an MI355X."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
from test_gpu_mx_cache import DTYPES, FILL, hand_over, sp  # noqa: E402, F401

pytestmark = pytest.mark.gpu

GUARD = 64  # bytes behind a buffer that nothing may touch
HELD = 0xA5


def ptr(t):
    return ctypes.c_void_p(t.data_ptr())


@pytest.mark.parametrize("S,Hkv,L,d,dtype,blocks,nw,density", FILL)
def test_caches_are_zero_beyond_their_sizes(sp, S, Hkv, L, d, dtype, blocks, nw, density):  # noqa: F811
    a, s, w, c = blocks
    K, V, sep, idx, pre = hand_over(sp, S, Hkv, L, d, DTYPES[dtype], blocks, nw, density)
    params = sp.SepkvParams(S, Hkv, Hkv, d, a, s, w, c, 1.0, sp.SEPATTN_BF16 if dtype == "bf16" else sp.SEPATTN_FP32)
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    lib, room = sp.load(), c - a - s
    sizes_of = (S * Hkv * c * d // 2, S * Hkv * c * d // 32) * 2 + (S * room,)  # Kc, Ks, Vc, Vs, flags

    def run(fn, held):
        x = [torch.full((n + GUARD,), held, dtype=torch.uint8, device="cuda") for n in sizes_of]
        sizes = torch.full((S * 6,), -1, dtype=torch.int32, device="cuda")
        assert fn(ctypes.byref(params), L, nw, ptr(K), ptr(V), ptr(sep), ptr(idx), idx.shape[1], ptr(pre), *[ptr(t) for t in x], ptr(sizes), st) == 0
        return x, sizes.view(S, 6).tolist()

    (zeroed, sizes), (plain, plain_sizes) = run(lib.sepkv_fill_from_prefill_mx_zeroed, HELD), run(lib.sepkv_fill_from_prefill_mx, HELD)
    assert sizes == plain_sizes and all(min(row) >= 0 for row in sizes)
    used, flagged = torch.zeros(S, c, dtype=torch.bool), torch.zeros(S, room, dtype=torch.bool)
    for i, row in enumerate(sizes):
        assert row[4:] == [0, 0]
        n = row[2] + row[3]
        used[i, list(range(row[0])) + list(range(a, a + row[1])) + list(range(a + s, a + s + n))] = True
        flagged[i, :n] = True
    used = used[:, None].expand(S, Hkv, c).cuda()
    for x, y, n, where in zip(zeroed, plain, sizes_of, [used] * 4 + [flagged.cuda()]):
        assert (x[n:] == HELD).all() and (y[n:] == HELD).all()
        x, y = x[:n].view(*where.shape, -1), y[:n].view(*where.shape, -1)
        assert torch.equal(x[where], y[where]) and (x[~where] == 0).all() and (y[~where] == HELD).all()
    # rows of which something was written: over another filling the plain form writes the same
    other, _ = run(lib.sepkv_fill_from_prefill_mx, 0x5A)
    for y, z, n, where in zip(plain, other, sizes_of, [used] * 4 + [flagged.cuda()]):
        assert torch.equal(y[:n].view(*where.shape, -1)[where], z[:n].view(*where.shape, -1)[where])
