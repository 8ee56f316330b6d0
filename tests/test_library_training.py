"""What the training calls refuse, and the bucket function: host code only, no GPU (nothing is enqueued for a call that is refused)."""
import ctypes as C
import math
import os

import numpy as np
import pytest

from paper_2301_06051_amd import binding as b

if not os.path.exists(b.LIB_PATH):
    pytest.skip("library not built", allow_module_level=True)

OK, EINVAL, ENOSPC, EUNSUPPORTED = b.DSVT_OK, b.DSVT_EINVAL, b.DSVT_ENOSPC, b.DSVT_EUNSUPPORTED
P = 1 << 20                                        # an aligned address that no call reaches


def _mha(**kw):
    v = dict(C=192, heads=8, dtype=b.DSVT_BF16, win=(12, 12, 1), dup_mode=0, rel_bias=P, rel_bucket=None, n_rel=529) | kw
    return b.MhaCfg(v["C"], v["heads"], v["dtype"], b.I32x3(*v["win"]), v["dup_mode"], v["rel_bias"], v["rel_bucket"], v["n_rel"])


def _maps(**kw):
    v = dict(n_voxels=100, max_sets=10, tau=36, set_inds=P, n_sets=P) | kw
    return b.Maps(v["n_voxels"], v["max_sets"], v["tau"], v["set_inds"], None, v["n_sets"], b.TileList(0, None, None, None, None))


def _forward(cfg=None, maps=None, coords=P, qkv=P, ld=576, out=P, ld_out=192):
    return b.lib().dsvt_set_mha(C.byref(cfg or _mha()), C.byref(maps or _maps()), coords, qkv, ld, out, ld_out, None)


def _backward(cfg=None, maps=None, coords=P, qkv=P, ld=576, g=P, ld_g=192, d=P, ld_d=576, rel=P, ws=P, ws_bytes=1 << 30):
    return b.lib().dsvt_set_mha_backward(C.byref(cfg or _mha()), C.byref(maps or _maps()), coords, qkv, ld, g, ld_g, d, ld_d, rel, ws, ws_bytes, None)


@pytest.mark.parametrize("cfg,rc", [
    (dict(C=0), EINVAL), (dict(heads=0), EINVAL), (dict(heads=7), EINVAL), (dict(dtype=2), EINVAL), (dict(dup_mode=2), EINVAL), (dict(win=(12, 0, 1)), EINVAL),
    (dict(win=(5000, 1, 1), n_rel=9999), EINVAL), (dict(n_rel=0), EINVAL), (dict(n_rel=528), EINVAL), (dict(heads=16), EUNSUPPORTED), (dict(heads=2), EUNSUPPORTED),
    (dict(win=(4096, 4096, 1), rel_bucket=P, n_rel=8), EUNSUPPORTED)])
def test_set_mha_refuses_configurations(cfg, rc):
    assert _forward(_mha(**cfg)) == rc and _backward(_mha(**cfg)) == rc
    size = C.c_size_t(0)
    assert b.lib().dsvt_set_mha_backward_workspace_size(C.byref(_mha(**cfg)), C.byref(_maps()), C.byref(size)) == rc


@pytest.mark.parametrize("maps,rc", [(dict(n_voxels=-1), EINVAL), (dict(max_sets=-1), EINVAL), (dict(max_sets=2 ** 30 + 1), EINVAL), (dict(tau=0), EINVAL), (dict(tau=97), EUNSUPPORTED),
                                     (dict(set_inds=None), EINVAL), (dict(n_sets=None), EINVAL)])
def test_set_mha_refuses_maps(maps, rc):
    assert _forward(maps=_maps(**maps)) == rc and _backward(maps=_maps(**maps)) == rc


@pytest.mark.parametrize("kw", [dict(coords=None), dict(coords=P + 4), dict(qkv=None), dict(qkv=P + 8), dict(ld=575), dict(ld=580), dict(ld=2 ** 32)])
def test_set_mha_refuses_arrays(kw):
    assert _forward(**kw) == EINVAL and _backward(**kw) == EINVAL


def test_set_mha_refuses_its_own_arrays_and_scratch():
    for kw in (dict(out=None), dict(out=P + 2), dict(ld_out=191), dict(ld_out=196)):
        assert _forward(**kw) == EINVAL
    for kw in (dict(g=None), dict(g=P + 8), dict(ld_g=184), dict(d=None), dict(d=P + 8), dict(ld_d=192), dict(ws=None), dict(ws=P + 4)):
        assert _backward(**kw) == EINVAL
    need = C.c_size_t(0)
    assert b.lib().dsvt_set_mha_backward_workspace_size(C.byref(_mha()), C.byref(_maps()), C.byref(need)) == OK and need.value > 0
    assert _backward(ws_bytes=need.value - 1) == ENOSPC
    assert _backward(_mha(rel_bias=None), rel=P) == EINVAL                                      # a gradient of no table
    none = C.c_size_t(1)
    assert b.lib().dsvt_set_mha_backward_workspace_size(C.byref(_mha(rel_bias=None)), C.byref(_maps()), C.byref(none)) == OK and none.value == 0
    # no voxels: nothing to do, whatever the pointers
    assert _forward(maps=_maps(n_voxels=0, set_inds=None, n_sets=None), coords=None, qkv=None, out=None) == OK
    assert b.lib().dsvt_set_mha(None, C.byref(_maps()), P, P, 576, P, 192, None) == EINVAL
    assert b.lib().dsvt_set_mha(C.byref(_mha()), None, P, P, 576, P, 192, None) == EINVAL


def test_layer_norm_refusals():
    L = b.lib()
    cfg = lambda **kw: b.LnCfg(*(dict(C=192, dtype=b.DSVT_BF16, gamma=P, beta=P, eps=1e-5) | kw).values())  # noqa: E731
    fwd = lambda c=None, x=P, ldx=192, r=P, ldr=192, n=10, y=P, ldy=192: L.dsvt_layer_norm(  # noqa: E731
        C.byref(c or cfg()), x, ldx, r, ldr, n, y, ldy, None)
    back = lambda c=None, dy=P, ldd=192, x=P, ldx=192, r=P, ldr=192, n=10, dx=P, ld=192, dg=P, db=P, ws=P, size=1 << 30: (  # noqa: E731
        L.dsvt_layer_norm_backward(C.byref(c or cfg()), dy, ldd, x, ldx, r, ldr, n, dx, ld, dg, db, ws, size, None))
    for kw in (dict(C=0), dict(C=-1), dict(dtype=5), dict(gamma=None), dict(eps=-1.0), dict(eps=math.nan)):
        assert fwd(cfg(**kw)) == EINVAL and back(cfg(**kw)) == EINVAL
    assert fwd(cfg(C=65537), ldx=65537, ldr=65537, ldy=65537) == EUNSUPPORTED
    assert fwd(cfg(beta=None)) == EINVAL
    for kw in (dict(x=None), dict(x=P + 1), dict(ldx=191), dict(ldr=0), dict(r=P + 1), dict(n=-1)):
        assert fwd(**kw) == EINVAL and back(**kw) == EINVAL
    for kw in (dict(y=None), dict(y=P + 1), dict(ldy=10)):
        assert fwd(**kw) == EINVAL
    for kw in (dict(dy=None), dict(ldd=0), dict(dx=None), dict(ld=0), dict(dg=None), dict(db=None), dict(ws=None), dict(ws=P + 8)):
        assert back(**kw) == EINVAL
    size = C.c_size_t(0)
    assert L.dsvt_layer_norm_backward_workspace_size(C.byref(cfg()), 10, C.byref(size)) == OK and size.value >= 10 * 192 * 8
    assert back(size=size.value - 1) == ENOSPC
    assert fwd(n=0, x=None, r=None, y=None) == OK
    assert L.dsvt_layer_norm_backward_workspace_size(C.byref(cfg()), -1, C.byref(size)) == EINVAL
    last = 0
    for n in (0, 1, 2, 100, 512, 513, 10 ** 6):
        assert L.dsvt_layer_norm_backward_workspace_size(C.byref(cfg()), n, C.byref(size)) == OK and size.value >= last
        last = size.value


def test_buckets_by_their_definition():
    for win, exact, side in (((12, 12, 8), 4, 6), ((12, 12, 1), 3, 5), ((12, 12, 32), 4, 7), ((30, 30, 1), 1, 30), ((5, 7, 2), 2, 2), ((1, 1, 1), 1, 1)):
        got, n_rel = b.dsvt_rel_buckets(win, exact, side)
        axes = []
        for w in win:
            most, axis = min(side, w), []
            for d in range(1 - w, w):
                a = abs(d)
                k = a
                if a >= exact and w > exact:
                    k = exact + math.floor((most - exact) * (math.log(a / exact) / math.log(w / exact)))
                axis.append((most, math.copysign(min(k, most - 1), d)))
            axes.append(axis)
        want = [((x + m0 - 1) * (2 * m1 - 1) + y + m1 - 1) * (2 * m2 - 1) + z + m2 - 1 for m0, x in axes[0] for m1, y in axes[1] for m2, z in axes[2]]
        assert np.array_equal(got, np.array(want).astype(np.int32)) and got.min() == 0 and got.max() == n_rel - 1
    full, n_rel = b.dsvt_rel_buckets((12, 12, 1), 12, 12)                                       # as many buckets as offsets: one each
    assert n_rel == 529 and np.array_equal(full, np.arange(529))


def test_buckets_refusals():
    for win, exact, side in (((0, 1, 1), 1, 1), ((12, 12, 1), 0, 3), ((12, 12, 1), 4, 3), ((5000, 1, 1), 2, 3), ((1000, 1000, 5), 2, 3)):
        with pytest.raises(b.DsvtError):
            b.dsvt_rel_buckets(win, exact, side)
