"""More that the training calls refuse: host code only, no GPU (nothing is enqueued for a call that is refused)."""
import ctypes as C
import os
import subprocess
import sys
from types import SimpleNamespace

import pytest
import torch

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


def test_tensors_that_require_gradients_are_refused():
    """By every call, for every tensor of it, before anything else is looked at; not without gradients enabled."""
    def tensors(names, needing):
        return {k: torch.zeros((4, 4), requires_grad=k == needing) for k in names}

    def calls(t):
        mha, ln = SimpleNamespace(rel_bias=t["rel_bias"]), SimpleNamespace(gamma=t["gamma"], beta=t["beta"])
        return {"qkv rel_bias out": lambda: b.dsvt_set_mha(mha, None, None, t["qkv"], out=t["out"]),
                "qkv d_out rel_bias d_qkv d_rel_bias": lambda: b.dsvt_set_mha_backward(mha, None, None, t["qkv"], t["d_out"], t["d_qkv"], t["d_rel_bias"]),
                "x res gamma beta y": lambda: b.dsvt_layer_norm(ln, t["x"], t["res"], y=t["y"]),
                "dy x res gamma dx d_gamma d_beta": lambda: b.dsvt_layer_norm_backward(ln, t["dy"], t["x"], t["res"], t["dx"], t["d_gamma"], t["d_beta"])}

    names = {k for args in calls(dict.fromkeys("qkv rel_bias out d_out d_qkv d_rel_bias x res gamma beta y dy dx d_gamma d_beta".split())) for k in args.split()}
    for needing in names:
        for args, call in calls(tensors(names, needing)).items():
            if needing in args.split():
                with pytest.raises(RuntimeError, match="records no graph"):
                    call()
                with torch.no_grad(), pytest.raises(Exception) as e:      # of the next check: the arguments are no call's
                    call()
                assert "records no graph" not in str(e.value)


class _Elsewhere:
    """A tensor on another device than the current one."""

    device, shape = "cuda:3", (4,)

    def get_device(self):
        return 3

    def is_contiguous(self):
        return True

    def stride(self):
        return (1,)


class _NoLibrary:
    """Fails the test if a call goes on to the library; sizes are asked for."""

    def __getattr__(self, name):
        if name.endswith("workspace_size"):
            return getattr(self.library, name)
        raise AssertionError(f"{name} was called")


def test_scratch_and_maps_that_kernels_cannot_use_are_refused(monkeypatch):
    """Host memory, memory of another device, and an expanded tensor, whose elements are more than its memory holds.  The current device is
    taken to be that of the host's tensors (-1), so that everything else fits."""
    no = _NoLibrary()
    no.library = b.lib()
    monkeypatch.setattr(b, "_current_device", lambda: -1)
    monkeypatch.setattr(b, "_current_stream", lambda device: 0)
    monkeypatch.setattr(b, "lib", lambda: no)
    n, c, heads = 3, 64, 4
    i32 = dict(dtype=torch.int32)
    mha = b.SetMha(c, heads, "f32", (3, 3, 1), torch.zeros((heads, 25)))
    ln = b.LayerNorm(torch.zeros(c), torch.zeros(c), "f32")
    coords, qkv, d_out = torch.zeros((n, 4), **i32), torch.zeros((n, 3 * c)), torch.zeros((n, c))

    def maps(device=-1):
        return SimpleNamespace(n_voxels=n, max_sets=2, tau=4, device=device, struct=b.Maps(n, 2, 4, P, None, P, b.TileList(0, None, None, None, None)))

    for bad in (_Elsewhere(), torch.zeros(1, dtype=torch.uint8).expand(1 << 20)):
        with pytest.raises(ValueError, match="ws"):
            b.dsvt_set_mha_backward(mha, maps(), coords, qkv, d_out, ws=bad)
        with pytest.raises(ValueError, match="ws"):
            b.dsvt_layer_norm_backward(ln, d_out, d_out, ws=bad)
    with pytest.raises(ValueError, match="SimpleNamespace was made on cuda:3"):
        b.dsvt_set_mha(mha, maps(3), coords, qkv)
    with pytest.raises(ValueError, match="SimpleNamespace was made on cuda:3"):
        b.dsvt_set_mha_backward(mha, maps(3), coords, qkv, d_out)
    with pytest.raises(AssertionError):
        b.SetMaps.of(torch.zeros((2, 4), **i32), torch.zeros((1,), **i32), n)                  # of the host
    with pytest.raises(AssertionError, match="dsvt_set_mha was called"):                       # and nothing else was wrong
        b.dsvt_set_mha(mha, maps(), coords, qkv)
    with pytest.raises(AssertionError, match="dsvt_layer_norm_backward was called"):
        b.dsvt_layer_norm_backward(ln, d_out, d_out, ws=torch.zeros(1 << 16, dtype=torch.uint8))


def test_import_with_a_torch_for_the_cpu():
    """Which has no torch._C._cuda_* functions: the package, its size queries and its refusals work all the same."""
    code = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_")]:
    delattr(torch._C, name)
import paper_2301_06051_amd as dsvt
assert dsvt.dsvt_rel_buckets((12, 12, 1), 3, 5)[1] == 81
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


def test_operators_keep_nothing_of_every_shape(monkeypatch):
    """A training run has another number of rows and sets in every step; sizes are right in any order of them."""
    monkeypatch.setattr(b, "_current_device", lambda: -1)
    mha, ln = b.SetMha(64, 4, "f32", (3, 3, 1), torch.zeros((4, 25))), b.LayerNorm(torch.zeros(64), torch.zeros(64), "f32")

    def held(o):
        return sum(len(v) for v in vars(o).values() if isinstance(v, (dict, list, tuple, set)))

    def maps(sets, tau):
        return SimpleNamespace(max_sets=sets, tau=tau, struct=b.Maps(9, sets, tau, P, None, P, b.TileList(0, None, None, None, None)))

    first = [(b.dsvt_layer_norm_backward_workspace_size(ln, n), b.dsvt_set_mha_backward_workspace_size(mha, maps(n, 4))) for n in range(2, 600)]
    before = held(mha), held(ln)
    again = [(b.dsvt_layer_norm_backward_workspace_size(ln, n), b.dsvt_set_mha_backward_workspace_size(mha, maps(n, 4))) for n in range(599, 1, -1)]
    assert first == again[::-1] and first[0][0] == 2 * 2 * 64 * 4 and first[-1][0] == 512 * 2 * 64 * 4
    assert (held(mha), held(ln)) == before and max(before) < 10
    assert b.dsvt_set_mha_backward_workspace_size(mha, maps(8, 4)) == b.dsvt_set_mha_backward_workspace_size(mha, maps(8, 96))


def test_one_row_has_no_stride():
    """The first row of rows that lie 579 elements apart begins on 16 bytes, which is all that one row needs."""
    for stride in (579, 3, 0, 1 << 40):
        row = torch.empty_strided((1, 576), (stride, 1), dtype=torch.bfloat16, device="meta")
        assert row.stride(0) == stride and b._rows(row, (1, 576), torch.bfloat16, row.get_device(), "qkv") == 576
    assert b._rows(torch.empty((2, 579))[:, :576], (2, 576), torch.float32, -1, "qkv") == 579
    assert b._rows(torch.empty((0, 192)), (0, 192), torch.float32, -1, "x") == 192


@pytest.mark.parametrize("heads,side_by_side", [(8, 8), (24, 8), (40, 8), (12, 6), (7, 7), (11, 1), (33, 3), (264, 8)])
def test_backward_workgroups_fit_the_chip_at_once(heads, side_by_side):
    """A row of partial sums for every part of the sets; a part has a workgroup for every group of heads, all parts together at most one a
    compute unit (256), and at least eight parts."""
    cfg, size = b.MhaCfg(8 * heads, heads, b.DSVT_BF16, b.I32x3(12, 12, 1), 0, P, None, 529), C.c_size_t(0)
    for sets in (0, 1, 8, 9, 50, 100, 1 << 20):
        assert b.lib().dsvt_set_mha_backward_workspace_size(C.byref(cfg), C.byref(b.Maps(N, sets, 36, P, None, P, b.TileList(0, None, None, None, None))), C.byref(size)) == 0
        parts, rest = divmod(size.value, heads * 529 * 4)
        groups = heads // side_by_side
        assert rest == 0 and parts % 8 == 0 and parts == min(max(256 // groups // 8 * 8, 8), max((sets + 7) // 8 * 8, 8)), (sets, parts)
