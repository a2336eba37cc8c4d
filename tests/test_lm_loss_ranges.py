"""Ranges of the loss's ids (no GPU needed): every call returns before any launch."""
import ctypes as C
import os

import pytest

import paper_2411_06465_amd as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libl4d.so not built")


def test_a_shard_beyond_the_last_id_is_refused():
    """vocab_start + vocab_shard, the id behind the shard, has to be one."""
    p = [C.c_void_p((1 << 40) + (i << 30)) for i in range(6)]
    ar = C.c_void_p()
    assert L.lib().l4d_arena_create(p[0], 256, C.byref(ar)) == L.L4D_OK
    last = (1 << 63) - 1
    for v0, want in ((last, L.L4D_EINVAL), (last - 99, L.L4D_EINVAL), (last - 100, L.L4D_ENOMEM)):   # 256 bytes hold no workspace
        assert L.lib().lm_loss_fwd(64, 64, 100, v0, *p[:3], None, None, p[3], p[4], None, ar, None) == want, v0
        assert L.lib().lm_loss_bwd(64, 64, 100, v0, *p[:4], None, 1.0, p[4], p[5], ar, None) == want, v0
    L.lib().l4d_arena_destroy(ar)
