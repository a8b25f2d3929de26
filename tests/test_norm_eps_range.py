"""Which eps the calls for normed rows take: 0 to 1e30.  Needs no GPU."""
import ctypes

import pytest

pytest.importorskip("torch")
from test_norm_and_mx_checks import FAKE, NULL, PARAM, kv, norm_params, sp  # noqa: E402, F401


@pytest.mark.parametrize("eps,taken", [(0.0, True), (1e-45, True), (1.0, True), (1e30, True), (1.0001e30, False), (3e38, False), (-1e-45, False)])
def test_eps(sp, eps, taken):  # noqa: F811
    lib = sp.load()
    assert (lib.sepattn_norm_rope_backward_workspace_bytes(ctypes.byref(norm_params(sp, eps=eps))) > 0) == taken
    for name, cache in (("sepkv_append_norm_rope", (None, FAKE)), ("sepkv_append_norm_rope_mx", (None, FAKE, FAKE, FAKE))):  # a NULL that is looked at later
        rc = getattr(lib, name)(ctypes.byref(kv(sp)), 64, 0, eps, 0, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, *cache, FAKE, FAKE, None)
        assert rc == (NULL if taken else PARAM), name
