"""More that the training calls refuse: host code only, no GPU (nothing is enqueued for a call that is refused)."""
import ctypes as C
import os

import pytest

from paper_2301_06051_amd import binding as b

if not os.path.exists(b.LIB_PATH):
    pytest.skip("library not built", allow_module_level=True)

P = 1 << 30                                        # an aligned address that no call reaches
N, W = 100, 192                                    # voxels, channels


def _cfg(dtype=b.DSVT_BF16):
    return b.MhaCfg(W, 8, dtype, b.I32x3(12, 12, 1), 0, P, None, 529)


def _maps():
    return b.Maps(N, 10, 36, P, None, P, b.TileList(0, None, None, None, None))


@pytest.mark.parametrize("dtype,e", [(b.DSVT_BF16, 2), (b.DSVT_F32, 4)])
def test_set_mha_refuses_rows_over_rows(dtype, e):
    L, cfg, maps = b.lib(), _cfg(dtype), _maps()
    far = P + (1 << 28)
    # (row length, stride) in elements, and where the written rows begin, in elements behind the others
    for ld_r, ld_w, at in ((3 * W, 3 * W, 0), (4 * W, 4 * W, 0), (4 * W, 4 * W, 3 * W - 8), (4 * W, 4 * W, 4 * W * 99 + 8), (4 * W, 4 * W, -4 * W * 99 + 8),
                           (3 * W, 4 * W, 16), (4 * W, 3 * W, 3 * W * 100 - 8)):
        at *= e
        assert L.dsvt_set_mha(C.byref(cfg), C.byref(maps), P, P, ld_r, P + at, ld_w, None) == b.DSVT_EINVAL, (ld_r, ld_w, at)
        assert L.dsvt_set_mha_backward(C.byref(cfg), C.byref(maps), P, P, ld_r, far, W, P + at, ld_w, P, P, 1 << 30, None) == b.DSVT_EINVAL
        assert L.dsvt_set_mha_backward(C.byref(cfg), C.byref(maps), P, far, 3 * W, P, ld_r, P + at, ld_w, P, P, 1 << 30, None) == (
            b.DSVT_EINVAL), (ld_r, ld_w, at)
