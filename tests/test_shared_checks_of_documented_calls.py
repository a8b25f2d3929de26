"""Calls for shared prompts and frequencies that the documentation allows, and arguments that it does not, up to the last check in front of
a launch.  Needs no GPU."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
from test_rope_and_shared_checks import FAKE, kv, sp  # noqa: E402, F401


@pytest.mark.parametrize("scale", [0.0, -1.0, float("nan")])
def test_scale_of_the_prefix_caches_is_not_looked_at(sp, scale):  # noqa: F811
    lib, p = sp.load(), ctypes.byref(kv(sp))
    want = lib.sepattn_decode_shared_workspace_bytes(p, ctypes.byref(kv(sp, S=3)))
    pp = ctypes.byref(kv(sp, S=3, scale=scale))
    assert want > 0 and lib.sepattn_decode_shared_workspace_bytes(p, pp) == want
    # everything but the workspace is in order
    assert lib.sepattn_decode_shared(p, pp, *[FAKE] * 11, None, None, 0, None) == 5
    assert lib.sepattn_decode_shared_rope(p, pp, *[FAKE] * 10, FAKE, 400, FAKE, None, None, 0, None) == 5


def test_frequencies_take_sizes_of_32_bits(sp):  # noqa: F811
    """A size past 32 bits is refused, not taken for what its lower bits say."""
    for size in (2 ** 32, 2 ** 32 + 8192, 2 ** 31):
        with pytest.raises(OverflowError):
            sp.sepattn_rope_frequencies(64, 10000.0, 4.0, 1.0, 4.0, size)
        with pytest.raises(OverflowError):
            sp.sepattn_rope_frequencies(size + 64, 10000.0)
    assert torch.equal(sp.sepattn_rope_frequencies(64, 10000.0, 1.0, 1.0, 4.0, 2 ** 31 - 1), sp.sepattn_rope_frequencies(64, 10000.0))
