"""ctypes binding of libdsvt.so: argument marshalling only.

Every step of the path runs inside the HIP library; PyTorch supplies device memory and the
stream.  There is no CPU fallback: a missing library raises.
"""
import ctypes as C
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdsvt.so")

DSVT_OK, DSVT_EINVAL, DSVT_ENOSPC, DSVT_EHIP, DSVT_EUNSUPPORTED = 0, -1, -2, -3, -4
DSVT_F32, DSVT_BF16 = 0, 1
ST_COORD_RANGE, ST_COORD_REPEAT, ST_SET_OVERFLOW, ST_WS_STATE, ST_VOXEL_OVERFLOW, ST_TILE_OVERFLOW = 1, 2, 4, 8, 16, 32
_ERR = {-1: "DSVT_EINVAL", -2: "DSVT_ENOSPC", -3: "DSVT_EHIP", -4: "DSVT_EUNSUPPORTED"}
_DT = {"f32": (DSVT_F32, torch.float32), "bf16": (DSVT_BF16, torch.bfloat16)}

I32x3 = C.c_int32 * 3
F32x3 = C.c_float * 3


class PartCfg(C.Structure):
    _fields_ = [("grid", I32x3), ("win", I32x3), ("shift", I32x3), ("tau", C.c_int32), ("batch", C.c_int32),
                ("axis", C.c_int32)]


class TileList(C.Structure):
    _fields_ = [("max_tiles", C.c_int32), ("tile_first", C.c_void_p), ("n_tiles", C.c_void_p),
                ("tile_order", C.c_void_p), ("tile_desc", C.c_void_p)]


class XyJob(C.Structure):
    _fields_ = [("cfg", PartCfg), ("set_inds_x", C.c_void_p), ("set_inds_y", C.c_void_p), ("voxel_slot_x", C.c_void_p),
                ("voxel_slot_y", C.c_void_p), ("n_sets", C.c_void_p), ("set_win", C.c_void_p), ("max_sets", C.c_int32),
                ("tiles", C.POINTER(TileList)), ("tile_desc_y", C.c_void_p), ("ws", C.c_void_p), ("ws_bytes", C.c_size_t),
                ("status", C.c_void_p)]


class Maps(C.Structure):
    _fields_ = [("n_voxels", C.c_int32), ("max_sets", C.c_int32), ("tau", C.c_int32), ("set_inds", C.c_void_p),
                ("voxel_slot", C.c_void_p), ("n_sets", C.c_void_p), ("tiles", TileList)]


class LayerW(C.Structure):
    _fields_ = [("C", C.c_int32), ("heads", C.c_int32), ("hidden", C.c_int32), ("dtype", C.c_int32),
                ("w_qkv", C.c_void_p), ("w_o", C.c_void_p), ("w_1", C.c_void_p), ("w_2", C.c_void_p),
                ("b_qkv", C.c_void_p), ("b_o", C.c_void_p), ("b_1", C.c_void_p), ("b_2", C.c_void_p),
                ("ln1_g", C.c_void_p), ("ln1_b", C.c_void_p), ("ln2_g", C.c_void_p), ("ln2_b", C.c_void_p),
                ("ln_eps", C.c_float), ("rel_bias", C.c_void_p), ("win", I32x3), ("dup_mode", C.c_int32),
                ("packed", C.c_void_p)]


class VfeCfg(C.Structure):
    _fields_ = [("grid", I32x3), ("batch", C.c_int32), ("range_min", F32x3), ("voxel_size", F32x3), ("f_in", C.c_int32),
                ("C", C.c_int32), ("dtype", C.c_int32), ("w", C.c_void_p), ("b", C.c_void_p), ("relu", C.c_int32)]


class PoolCfg(C.Structure):
    _fields_ = [("grid", I32x3), ("pool", I32x3), ("batch", C.c_int32), ("C", C.c_int32), ("heads", C.c_int32),
                ("dtype", C.c_int32), ("w_q", C.c_void_p), ("w_k", C.c_void_p), ("w_v", C.c_void_p),
                ("w_o", C.c_void_p), ("b_q", C.c_void_p), ("b_k", C.c_void_p), ("b_v", C.c_void_p),
                ("b_o", C.c_void_p), ("ln_g", C.c_void_p), ("ln_b", C.c_void_p), ("ln_eps", C.c_float),
                ("mask_empty", C.c_int32), ("packed", C.c_void_p)]


class MhaCfg(C.Structure):
    _fields_ = [("C", C.c_int32), ("heads", C.c_int32), ("dtype", C.c_int32), ("win", I32x3), ("dup_mode", C.c_int32),
                ("rel_bias", C.c_void_p), ("rel_bucket", C.c_void_p), ("n_rel", C.c_int32)]


class LnCfg(C.Structure):
    _fields_ = [("C", C.c_int32), ("dtype", C.c_int32), ("gamma", C.c_void_p), ("beta", C.c_void_p), ("eps", C.c_float)]


_lib = None


def lib():
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                               "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
        L.dsvt_partition_bound.argtypes = [C.POINTER(PartCfg), i32, C.POINTER(i32), C.POINTER(i32), C.POINTER(sz)]
        L.dsvt_partition.argtypes = [C.POINTER(PartCfg), vp, i32, vp, vp, vp, i32, vp, C.POINTER(TileList), vp, sz, vp, vp]
        L.dsvt_partition_ws_init.argtypes = [C.POINTER(PartCfg), i32, vp, sz, vp]
        L.dsvt_partition_xy.argtypes = [C.POINTER(PartCfg), vp, i32, vp, vp, vp, vp, vp, i32, vp, C.POINTER(TileList), vp,
                                        vp, sz, vp, vp]
        L.dsvt_partition_xy_multi.argtypes = [C.POINTER(XyJob), i32, vp, i32, vp]
        L.dsvt_layer_packed_size.argtypes = [C.POINTER(LayerW), C.POINTER(sz)]
        L.dsvt_layer_pack.argtypes = [C.POINTER(LayerW), vp, sz, vp]
        L.dsvt_block_workspace_size.argtypes = [C.POINTER(LayerW), i32, C.POINTER(sz)]
        L.dsvt_set_attention_workspace_size.argtypes = [C.POINTER(LayerW), i32, C.POINTER(sz)]
        L.dsvt_set_attention.argtypes = [C.POINTER(LayerW), C.POINTER(Maps), vp, vp, vp, vp, sz, vp]
        L.dsvt_block.argtypes = [C.POINTER(LayerW), C.POINTER(Maps), vp, vp, vp, vp, sz, vp]
        L.dsvt_pool_packed_size.argtypes = [C.POINTER(PoolCfg), C.POINTER(sz)]
        L.dsvt_pool_pack.argtypes = [C.POINTER(PoolCfg), vp, sz, vp]
        L.dsvt_attn_pool_workspace_size.argtypes = [C.POINTER(PoolCfg), i32, C.POINTER(sz)]
        L.dsvt_attn_pool.argtypes = [C.POINTER(PoolCfg), vp, vp, i32, vp, vp, vp, vp, sz, vp, vp]
        L.dsvt_attn_pool_static.argtypes = [C.POINTER(PoolCfg), vp, vp, i32, vp, vp, vp, vp, vp]
        L.dsvt_bev_scatter.argtypes = [vp, vp, i32, i32, i32, i32, C.POINTER(I32x3), vp, vp, vp]
        L.dsvt_vfe_workspace_size.argtypes = [C.POINTER(VfeCfg), i32, i32, C.POINTER(sz)]
        L.dsvt_vfe.argtypes = [C.POINTER(VfeCfg), vp, vp, i32, vp, vp, vp, i32, vp, sz, vp, vp]
        i64 = C.c_int64
        L.dsvt_rel_buckets.argtypes = [C.POINTER(I32x3), i32, i32, vp, C.POINTER(i32)]
        L.dsvt_set_mha.argtypes = [C.POINTER(MhaCfg), C.POINTER(Maps), vp, vp, i64, vp, i64, vp]
        L.dsvt_set_mha_backward_workspace_size.argtypes = [C.POINTER(MhaCfg), C.POINTER(Maps), C.POINTER(sz)]
        L.dsvt_set_mha_backward.argtypes = [C.POINTER(MhaCfg), C.POINTER(Maps), vp, vp, i64, vp, i64, vp, i64, vp, vp, sz, vp]
        L.dsvt_layer_norm.argtypes = [C.POINTER(LnCfg), vp, i64, vp, i64, i32, vp, i64, vp]
        L.dsvt_layer_norm_backward_workspace_size.argtypes = [C.POINTER(LnCfg), i32, C.POINTER(sz)]
        L.dsvt_layer_norm_backward.argtypes = [C.POINTER(LnCfg), vp, i64, vp, i64, vp, i64, i32, vp, i64, vp, vp, vp, sz, vp]
        L.dsvt_prof_enable.argtypes = [i32]
        L.dsvt_prof_collect.argtypes = [C.POINTER(C.c_float), C.POINTER(i32), i32]
        L.dsvt_prof_kernel_count.restype = i32
        L.dsvt_prof_kernel_name.argtypes = [i32]
        L.dsvt_prof_kernel_name.restype = C.c_char_p
        _lib = L
    return _lib


class DsvtError(RuntimeError):
    def __init__(self, where, rc):
        super().__init__(f"{where} returned {_ERR.get(rc, rc)}")
        self.rc = rc


def _check(where, rc):
    if rc != DSVT_OK:
        raise DsvtError(where, rc)


def _stream(stream):
    return C.c_void_p(torch.cuda.current_stream().cuda_stream if stream is None else stream)


def _ptr(t):
    return C.c_void_p(0 if t is None else t.data_ptr())


def _dev(a, dtype):
    return torch.as_tensor(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype).contiguous()


def part_cfg(grid, win, shift, tau, batch, axis):
    return PartCfg(I32x3(*grid), I32x3(*win), I32x3(*shift), tau, batch, axis)


def dsvt_partition_bound(cfg, n_voxels):
    ms, mt, ws = C.c_int32(0), C.c_int32(0), C.c_size_t(0)
    _check("dsvt_partition_bound",
           lib().dsvt_partition_bound(C.byref(cfg), n_voxels, C.byref(ms), C.byref(mt), C.byref(ws)))
    return ms.value, mt.value, ws.value


class SetMaps:
    """Device buffers of one (window configuration, axis) and the struct the kernels read."""

    def __init__(self, cfg, n_voxels, max_sets=None, tiles=True, common=None, max_tiles=None):
        """common: the SetMaps of the other axis of the same dsvt_partition_xy call, whose n_sets, set_win,
        status, scratch and tile boundaries this one shares.  max_tiles: a work list shorter than the bound."""
        bound, tile_bound, ws_bytes = dsvt_partition_bound(cfg, n_voxels)
        self.cfg, self.n_voxels, self.tau = cfg, n_voxels, cfg.tau
        self.max_sets = bound if max_sets is None else max_sets
        i32 = dict(dtype=torch.int32, device="cuda")
        self.set_inds = torch.full((self.max_sets, cfg.tau), -1, **i32)
        self.voxel_slot = torch.full((n_voxels,), -1, **i32)
        if common is None:
            self.set_win = torch.full((self.max_sets,), -1, **i32)
            self.n_sets = torch.zeros((1,), **i32)
            self.status = torch.zeros((1,), **i32)
            self.ws = torch.empty((ws_bytes,), dtype=torch.uint8, device="cuda")
            _check("dsvt_partition_ws_init",
                   lib().dsvt_partition_ws_init(C.byref(cfg), n_voxels, _ptr(self.ws), ws_bytes, _stream(None)))
            torch.cuda.current_stream().synchronize()     # the maps may first be used on any stream
        else:
            assert common.max_sets == self.max_sets and common.n_voxels == n_voxels
            self.set_win, self.n_sets, self.status, self.ws = common.set_win, common.n_sets, common.status, common.ws
        self.max_tiles = tile_bound if (tiles and tile_bound > 0 and cfg.tau <= 96) else 0
        if self.max_tiles and max_tiles is not None:
            self.max_tiles = min(self.max_tiles, max_tiles)
        if self.max_tiles:
            if common is None:
                self.tile_first = torch.full((self.max_tiles + 1,), -1, **i32)
                self.n_tiles = torch.zeros((1,), **i32)
                self.tile_order = torch.full((self.max_tiles,), -1, **i32)
            else:
                self.tile_first, self.n_tiles, self.tile_order = common.tile_first, common.n_tiles, common.tile_order
            self.tile_desc = torch.full((self.max_tiles, 256), -1, **i32)
            self.tile_list = TileList(self.max_tiles, self.tile_first.data_ptr(), self.n_tiles.data_ptr(),
                                      self.tile_order.data_ptr(), self.tile_desc.data_ptr())
        else:
            self.tile_first = self.n_tiles = self.tile_order = self.tile_desc = None
            self.tile_list = TileList(0, None, None, None, None)
        self.struct = Maps(n_voxels, self.max_sets, cfg.tau, self.set_inds.data_ptr(), self.voxel_slot.data_ptr(),
                           self.n_sets.data_ptr(), self.tile_list)
        self.device = self.set_inds.get_device()

    @classmethod
    def of(cls, set_inds, n_sets, n_voxels):
        """Maps from slot maps the caller has: set_inds int32 [max_sets, tau], n_sets int32 [1] (both on the GPU), as
        dsvt_partition writes them.  For dsvt_set_mha and its backward call: there is no work list and no voxel_slot."""
        assert set_inds.is_cuda and set_inds.dtype == torch.int32 and set_inds.is_contiguous() and set_inds.dim() == 2
        assert n_sets.device == set_inds.device and n_sets.dtype == torch.int32 and n_sets.numel() == 1
        m = cls.__new__(cls)
        m.cfg, m.n_voxels, m.tau, m.max_sets, m.max_tiles = None, n_voxels, set_inds.shape[1], set_inds.shape[0], 0
        m.set_inds, m.n_sets, m.voxel_slot = set_inds, n_sets, None
        m.tile_list = TileList(0, None, None, None, None)
        m.struct = Maps(n_voxels, m.max_sets, m.tau, set_inds.data_ptr(), None, n_sets.data_ptr(), m.tile_list)
        m.device = set_inds.get_device()
        return m


def dsvt_partition(cfg, coords, out=None, stream=None):
    """coords: int32 cuda tensor [N,4].  Returns the SetMaps it filled (allocated here unless given)."""
    assert coords.is_cuda and coords.dtype == torch.int32 and coords.is_contiguous() and coords.shape[1] == 4
    n = coords.shape[0]
    out = SetMaps(cfg, n) if out is None else out
    assert out.n_voxels == n
    rc = lib().dsvt_partition(C.byref(cfg), _ptr(coords), n, _ptr(out.set_inds), _ptr(out.voxel_slot),
                              _ptr(out.n_sets), out.max_sets, _ptr(out.set_win),
                              C.byref(out.tile_list) if out.max_tiles else None, _ptr(out.ws), out.ws.numel(),
                              _ptr(out.status),
                              _stream(stream))
    _check("dsvt_partition", rc)
    return out


class SetMapsXY:
    """The maps of both axes of one window configuration, filled by one dsvt_partition_xy call; indexes
    and iterates like the pair [X-axis maps, Y-axis maps]."""

    def __init__(self, cfg, n_voxels, max_sets=None, tiles=True, max_tiles=None):
        self.x = SetMaps(cfg, n_voxels, max_sets, tiles, max_tiles=max_tiles)
        self.y = SetMaps(cfg, n_voxels, max_sets, tiles, common=self.x, max_tiles=max_tiles)
        self.n_voxels = n_voxels

    def __getitem__(self, k):
        return (self.x, self.y)[k]

    def __iter__(self):
        return iter((self.x, self.y))

    def __len__(self):
        return 2


def dsvt_partition_xy(cfg, coords, out=None, stream=None):
    """Both rotated partitions of one window configuration.  Returns the SetMapsXY it filled."""
    assert coords.is_cuda and coords.dtype == torch.int32 and coords.is_contiguous() and coords.shape[1] == 4
    n = coords.shape[0]
    out = SetMapsXY(cfg, n) if out is None else out
    assert out.n_voxels == n
    x, y = out.x, out.y
    rc = lib().dsvt_partition_xy(C.byref(cfg), _ptr(coords), n, _ptr(x.set_inds), _ptr(y.set_inds), _ptr(x.voxel_slot),
                                 _ptr(y.voxel_slot), _ptr(x.n_sets), x.max_sets, _ptr(x.set_win),
                                 C.byref(x.tile_list) if x.max_tiles else None, _ptr(y.tile_desc) if x.max_tiles else None,
                                 _ptr(x.ws), x.ws.numel(), _ptr(x.status), _stream(stream))
    _check("dsvt_partition_xy", rc)
    return out


def dsvt_partition_xy_multi(cfgs, coords, outs, stream=None):
    """The partitions of several window configurations (cfgs[k] into the SetMapsXY outs[k]) in one pass."""
    assert coords.is_cuda and coords.dtype == torch.int32 and coords.is_contiguous() and coords.shape[1] == 4
    n = coords.shape[0]
    assert len(cfgs) == len(outs) and all(o.n_voxels == n for o in outs)
    jobs = (XyJob * len(cfgs))()
    for j, cfg, o in zip(jobs, cfgs, outs):
        x, y = o.x, o.y
        j.cfg = cfg
        j.set_inds_x, j.set_inds_y = x.set_inds.data_ptr(), y.set_inds.data_ptr()
        j.voxel_slot_x, j.voxel_slot_y = x.voxel_slot.data_ptr(), y.voxel_slot.data_ptr()
        j.n_sets, j.set_win, j.max_sets = x.n_sets.data_ptr(), x.set_win.data_ptr(), x.max_sets
        j.tiles = C.pointer(x.tile_list) if x.max_tiles else None
        j.tile_desc_y = y.tile_desc.data_ptr() if x.max_tiles else None
        j.ws, j.ws_bytes, j.status = x.ws.data_ptr(), x.ws.numel(), x.status.data_ptr()
    _check("dsvt_partition_xy_multi", lib().dsvt_partition_xy_multi(jobs, len(cfgs), _ptr(coords), n, _stream(stream)))
    return outs


class LayerWeights:
    """Device copy of one DSVT layer's parameters (from a synth-style dict of numpy arrays)."""

    def __init__(self, w, dup_mode=0):
        code, tdt = _DT[w["dtype"]]
        f32 = torch.float32
        self.t = {k: _dev(w[k], tdt) for k in ("w_qkv", "w_o", "w_1", "w_2")}
        self.t.update({k: _dev(w[k], f32) for k in ("b_qkv", "b_o", "b_1", "b_2", "ln1_g", "ln1_b", "ln2_g", "ln2_b")})
        self.t["rel_bias"] = None if w.get("rel_bias") is None else _dev(w["rel_bias"], f32)
        self.dtype, self.C = tdt, w["C"]
        p = lambda k: self.t[k].data_ptr() if self.t[k] is not None else None
        self.struct = LayerW(w["C"], w["heads"], w["hidden"], code, p("w_qkv"), p("w_o"), p("w_1"), p("w_2"),
                             p("b_qkv"), p("b_o"), p("b_1"), p("b_2"), p("ln1_g"), p("ln1_b"), p("ln2_g"), p("ln2_b"),
                             w["ln_eps"], p("rel_bias"), I32x3(*w["win"]), dup_mode, None)
        nbytes = C.c_size_t(0)
        _check("dsvt_layer_packed_size", lib().dsvt_layer_packed_size(C.byref(self.struct), C.byref(nbytes)))
        self.packed = torch.empty((nbytes.value,), dtype=torch.uint8, device="cuda")
        _check("dsvt_layer_pack", lib().dsvt_layer_pack(C.byref(self.struct), _ptr(self.packed), nbytes.value, _stream(None)))
        self.struct.packed = self.packed.data_ptr()


def dsvt_set_attention_workspace_size(layer, n_voxels):
    sz = C.c_size_t(0)
    _check("dsvt_set_attention_workspace_size",
           lib().dsvt_set_attention_workspace_size(C.byref(layer.struct), n_voxels, C.byref(sz)))
    return sz.value


def dsvt_block_workspace_size(layer, n_voxels):
    sz = C.c_size_t(0)
    _check("dsvt_block_workspace_size", lib().dsvt_block_workspace_size(C.byref(layer.struct), n_voxels, C.byref(sz)))
    return sz.value


def _ws(nbytes, ws):
    if ws is None:
        ws = torch.empty((max(nbytes, 1),), dtype=torch.uint8, device="cuda")
    return ws


def dsvt_set_attention(layer, maps, coords, x, y=None, ws=None, stream=None):
    assert x.is_cuda and x.dtype == layer.dtype and x.is_contiguous() and x.shape == (maps.n_voxels, layer.C)
    y = torch.empty_like(x) if y is None else y
    ws = _ws(dsvt_block_workspace_size(layer, maps.n_voxels), ws)
    rc = lib().dsvt_set_attention(C.byref(layer.struct), C.byref(maps.struct), _ptr(coords), _ptr(x), _ptr(y),
                                  _ptr(ws), ws.numel(), _stream(stream))
    _check("dsvt_set_attention", rc)
    return y


def dsvt_block(layers, maps, coords, x_in, x_out=None, ws=None, stream=None):
    """layers: (X-axis LayerWeights, Y-axis LayerWeights); maps: (X-axis SetMaps, Y-axis SetMaps)."""
    assert x_in.is_cuda and x_in.dtype == layers[0].dtype and x_in.is_contiguous()
    x_out = torch.empty_like(x_in) if x_out is None else x_out
    ws = _ws(dsvt_block_workspace_size(layers[0], maps[0].n_voxels), ws)
    lw = (LayerW * 2)(layers[0].struct, layers[1].struct)
    mp = (Maps * 2)(maps[0].struct, maps[1].struct)
    rc = lib().dsvt_block(lw, mp, _ptr(coords), _ptr(x_in), _ptr(x_out), _ptr(ws), ws.numel(), _stream(stream))
    _check("dsvt_block", rc)
    return x_out


class PoolWeights:
    def __init__(self, w, grid, pool, batch, mask_empty=1):
        code, tdt = _DT[w["dtype"]]
        self.t = {k: _dev(w[k], tdt) for k in ("w_q", "w_k", "w_v", "w_o")}
        self.t.update({k: _dev(w[k], torch.float32) for k in ("b_q", "b_k", "b_v", "b_o", "ln_g", "ln_b")})
        self.dtype, self.C = tdt, w["C"]
        p = lambda k: self.t[k].data_ptr()
        self.struct = PoolCfg(I32x3(*grid), I32x3(*pool), batch, w["C"], w["heads"], code, p("w_q"), p("w_k"),
                              p("w_v"), p("w_o"), p("b_q"), p("b_k"), p("b_v"), p("b_o"), p("ln_g"), p("ln_b"),
                              w["ln_eps"], mask_empty, None)
        nbytes = C.c_size_t(0)
        _check("dsvt_pool_packed_size", lib().dsvt_pool_packed_size(C.byref(self.struct), C.byref(nbytes)))
        self.packed = torch.empty((nbytes.value,), dtype=torch.uint8, device="cuda")
        _check("dsvt_pool_pack", lib().dsvt_pool_pack(C.byref(self.struct), _ptr(self.packed), nbytes.value, _stream(None)))
        self.struct.packed = self.packed.data_ptr()


def dsvt_attn_pool_workspace_size(pool, n_voxels):
    sz = C.c_size_t(0)
    _check("dsvt_attn_pool_workspace_size",
           lib().dsvt_attn_pool_workspace_size(C.byref(pool.struct), n_voxels, C.byref(sz)))
    return sz.value


def dsvt_attn_pool(pool, coords, x, out=None, ws=None, stream=None):
    """Returns (out_coords [N,4], out [N,C], n_out device scalar, status); the first n_out rows are valid."""
    n = coords.shape[0]
    assert x.is_cuda and x.dtype == pool.dtype and x.is_contiguous() and x.shape == (n, pool.C)
    if out is None:
        out = (torch.zeros((n, 4), dtype=torch.int32, device="cuda"), torch.zeros_like(x),
               torch.zeros((1,), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda"))
    ws = _ws(dsvt_attn_pool_workspace_size(pool, n), ws)
    rc = lib().dsvt_attn_pool(C.byref(pool.struct), _ptr(coords), _ptr(x), n, _ptr(out[0]), _ptr(out[1]), _ptr(out[2]),
                              _ptr(ws), ws.numel(), _ptr(out[3]), _stream(stream))
    _check("dsvt_attn_pool", rc)
    return out


def dsvt_attn_pool_static(pool, coords, x, out, stream=None):
    """dsvt_attn_pool on the library's built-in scratch: no workspace, nothing allocated.  `out` = the caller's
    (out_coords [N,4] int32, out [N,C], n_out, status) tensors."""
    n = coords.shape[0]
    assert x.is_cuda and x.dtype == pool.dtype and x.is_contiguous() and x.shape == (n, pool.C)
    rc = lib().dsvt_attn_pool_static(C.byref(pool.struct), _ptr(coords), _ptr(x), n, _ptr(out[0]), _ptr(out[1]), _ptr(out[2]),
                                     _ptr(out[3]), _stream(stream))
    _check("dsvt_attn_pool_static", rc)
    return out


def dsvt_bev_scatter(coords, x, batch, grid, out=None, stream=None):
    """Dense channels-last map [batch, X, Y, Z, C] with every voxel's row at its cell, zeros elsewhere.
    Returns (out, status)."""
    n, c = x.shape
    assert x.is_cuda and x.is_contiguous() and coords.shape == (n, 4) and x.dtype in (torch.float32, torch.bfloat16)
    if out is None:
        out = torch.empty((batch, *grid, c), dtype=x.dtype, device="cuda")
    status = torch.zeros((1,), dtype=torch.int32, device="cuda")
    rc = lib().dsvt_bev_scatter(_ptr(coords), _ptr(x), n, c, DSVT_F32 if x.dtype == torch.float32 else DSVT_BF16, batch,
                                C.byref(I32x3(*grid)), _ptr(out), _ptr(status), _stream(stream))
    _check("dsvt_bev_scatter", rc)
    return out, status


def dsvt_vfe_workspace_size(cfg, n_points, max_voxels):
    b = C.c_size_t(0)
    _check("dsvt_vfe_workspace_size", lib().dsvt_vfe_workspace_size(C.byref(cfg), n_points, max_voxels, C.byref(b)))
    return b.value


class Vfe:
    """Configuration, weights and buffers of one dsvt_vfe call site: `max_points` points in, at most
    `max_voxels` voxels out.  w [C, f_in] and b [C] are float32 device tensors or None."""

    def __init__(self, grid, batch, range_min, voxel_size, f_in, C_out, dtype, max_points, max_voxels, w=None, b=None,
                 relu=False):
        self.w, self.b = w, b
        self.cfg = VfeCfg(I32x3(*grid), batch, F32x3(*range_min), F32x3(*voxel_size), f_in, C_out, _DT[dtype][0],
                          None if w is None else w.data_ptr(), None if b is None else b.data_ptr(), int(relu))
        self.max_points, self.max_voxels = max_points, max_voxels
        self.ws = torch.empty((dsvt_vfe_workspace_size(self.cfg, max_points, max_voxels),), dtype=torch.uint8, device="cuda")
        self.coords = torch.empty((max_voxels, 4), dtype=torch.int32, device="cuda")
        self.x = torch.empty((max_voxels, C_out), dtype=_DT[dtype][1], device="cuda")
        self.n_voxels = torch.zeros((1,), dtype=torch.int32, device="cuda")
        self.status = torch.zeros((1,), dtype=torch.int32, device="cuda")


def dsvt_vfe(vfe, points, point_batch=None, stream=None):
    """Encodes `points` [P, f_in] float32 (device) into vfe.coords / vfe.x / vfe.n_voxels."""
    n = points.shape[0]
    assert points.is_cuda and points.is_contiguous() and points.dtype == torch.float32 and n <= vfe.max_points
    assert points.shape[1] == vfe.cfg.f_in
    assert point_batch is None or (point_batch.is_cuda and point_batch.dtype == torch.int32 and point_batch.shape == (n,))
    rc = lib().dsvt_vfe(C.byref(vfe.cfg), _ptr(points), None if point_batch is None else _ptr(point_batch), n,
                        _ptr(vfe.coords), _ptr(vfe.x), _ptr(vfe.n_voxels), vfe.max_voxels, _ptr(vfe.ws), vfe.ws.numel(),
                        _ptr(vfe.status), _stream(stream))
    _check("dsvt_vfe", rc)
    return vfe


# A call of a small operator is mostly host time: the current device and the handle of its current stream come without the objects that
# torch.cuda puts around them (a torch built for the CPU has neither function), and a workspace's size is asked for only if the shape is not
# that of the call before.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda device: torch.cuda.current_stream(device).cuda_stream)


def _rows(t, shape, dtype, device, what):
    """The row stride of a [rows, columns] tensor of the current device (`device`) whose columns are neighbours; of one row, whatever its tensor
    says, the row's length."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or (shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what}: a {dtype} tensor of shape {tuple(shape)} with neighbouring columns on the current device, cuda:{device}, is wanted; "
                         f"got {t.dtype} {tuple(t.shape)}, strides {tuple(t.stride())}, on {t.device}")
    return t.stride(0) if shape[0] > 1 else shape[1]


def _elsewhere(device, *owners):
    for owner in owners:
        if owner.device != device:
            raise ValueError(f"the {type(owner).__name__} was made on cuda:{owner.device}, the current device is cuda:{device}")


def _scratch(ws, device):
    """Address and bytes of the caller's scratch."""
    if ws.get_device() != device or not ws.is_contiguous():
        raise ValueError(f"ws: contiguous memory on the current device, cuda:{device}, is wanted; got {tuple(ws.shape)}, strides {tuple(ws.stride())}, "
                         f"on {ws.device}")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _vector(t, shape, dtype, device, what):
    if t.shape != shape or t.dtype is not dtype or t.get_device() != device or not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {tuple(shape)} on the current device, cuda:{device}, is wanted; got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")


# The calls record no graph: with gradients enabled, tensors that one is to pass through are refused, where it would be lost without a word.
_recording = torch.is_grad_enabled


def _no_graph(call, *tensors):
    for t in tensors:
        if t is not None and t.requires_grad:
            raise RuntimeError(f"{call} records no graph for automatic differentiation, and a tensor of it requires gradients: call it under "
                               "torch.no_grad(), or within a torch.autograd.Function whose backward makes the backward call")


def _new_on(stream, device, like, shape, dtype):
    """An uninitialised tensor for kernels that run on the stream of that handle (0: the default stream).  It is a block of that stream's, whose
    earlier users are so ordered before them: a block of the current stream may be in use there still."""
    if stream == _current_stream(device):
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)):
        t = like.new_empty(shape, dtype=dtype)
    t.record_stream(torch.cuda.current_stream())       # where the caller goes on with it
    return t


def dsvt_rel_buckets(win, n_exact, n_side):
    """(int32 numpy array of every offset's bucket, number of buckets) for SetMha's rel_bucket and table; see dsvt.h."""
    n = C.c_int32(0)
    _check("dsvt_rel_buckets", lib().dsvt_rel_buckets(C.byref(I32x3(*win)), n_exact, n_side, None, C.byref(n)))
    bucket = np.zeros(((2 * win[0] - 1) * (2 * win[1] - 1) * (2 * win[2] - 1),), np.int32)
    _check("dsvt_rel_buckets", lib().dsvt_rel_buckets(C.byref(I32x3(*win)), n_exact, n_side, bucket.ctypes.data_as(C.c_void_p), C.byref(n)))
    return bucket, n.value


class SetMha:
    """Shape and relative position bias of one set attention on projected rows.  rel_bias: float32 [heads, n_rel] or None;
    rel_bucket: int32 [(2L-1)(2W-1)(2H-1)] or None (an entry for every offset).  Both stay the caller's: the tensors
    are read at every call."""

    def __init__(self, channels, heads, dtype, win, rel_bias=None, rel_bucket=None, dup_mode=0):
        code, self.dtype = _DT[dtype]
        self.C, self.heads, self.rel_bias, self.rel_bucket = channels, heads, rel_bias, rel_bucket
        offsets = (2 * win[0] - 1) * (2 * win[1] - 1) * (2 * win[2] - 1)
        n_rel = 0
        if rel_bias is not None:
            n_rel = rel_bias.shape[-1]
            _vector(rel_bias, (heads, n_rel), torch.float32, _current_device(), "rel_bias")
        if rel_bucket is not None:
            _vector(rel_bucket, (offsets,), torch.int32, _current_device(), "rel_bucket")
        self.struct = MhaCfg(channels, heads, code, I32x3(*win), dup_mode, None if rel_bias is None else rel_bias.data_ptr(),
                             None if rel_bucket is None else rel_bucket.data_ptr(), n_rel)
        self.ref, self.size, self.device = C.byref(self.struct), (None, 0), _current_device()     # size: the last shape and its workspace bytes


def dsvt_set_mha(mha, maps, coords, qkv, out=None, stream=None):
    """Attention inside every set of `maps` on projected rows qkv [N, 3C]; returns out [N, C]."""
    if _recording():
        _no_graph("dsvt_set_mha", qkv, mha.rel_bias, out)
    n, c, dtype, dev = maps.n_voxels, mha.C, mha.dtype, _current_device()
    if mha.device != dev or maps.device != dev:
        _elsewhere(dev, mha, maps)
    ld = _rows(qkv, (n, 3 * c), dtype, dev, "qkv")
    _vector(coords, (n, 4), torch.int32, dev, "coords")
    if out is None:
        out, ld_out = qkv.new_empty((n, c)) if stream is None else _new_on(stream, dev, qkv, (n, c), dtype), c
    else:
        ld_out = _rows(out, (n, c), dtype, dev, "out")
    rc = lib().dsvt_set_mha(mha.ref, C.byref(maps.struct), coords.data_ptr(), qkv.data_ptr(), ld, out.data_ptr(), ld_out,
                            _current_stream(dev) if stream is None else stream)
    if rc:
        _check("dsvt_set_mha", rc)
    return out


def dsvt_set_mha_backward_workspace_size(mha, maps):
    shape = (maps.max_sets, maps.tau)
    last, size = mha.size
    if shape != last:
        b = C.c_size_t(0)
        _check("dsvt_set_mha_backward_workspace_size", lib().dsvt_set_mha_backward_workspace_size(mha.ref, C.byref(maps.struct), C.byref(b)))
        size = b.value
        mha.size = shape, size
    return size


def dsvt_set_mha_backward(mha, maps, coords, qkv, d_out, d_qkv=None, d_rel_bias=None, want_rel_bias=True, ws=None, stream=None):
    """Gradients of dsvt_set_mha: returns (d_qkv [N, 3C], d_rel_bias [heads, n_rel] float32, or None without a table or if not
    wanted)."""
    if _recording():
        _no_graph("dsvt_set_mha_backward", qkv, d_out, mha.rel_bias, d_qkv, d_rel_bias)
    n, c, dtype, dev = maps.n_voxels, mha.C, mha.dtype, _current_device()
    if mha.device != dev or maps.device != dev:
        _elsewhere(dev, mha, maps)
    ld, ld_out = _rows(qkv, (n, 3 * c), dtype, dev, "qkv"), _rows(d_out, (n, c), dtype, dev, "d_out")
    _vector(coords, (n, 4), torch.int32, dev, "coords")
    if d_qkv is None:
        d_qkv, ld_d = qkv.new_empty((n, 3 * c)) if stream is None else _new_on(stream, dev, qkv, (n, 3 * c), dtype), 3 * c
    else:
        ld_d = _rows(d_qkv, (n, 3 * c), dtype, dev, "d_qkv")
    if d_rel_bias is not None:
        _vector(d_rel_bias, mha.rel_bias.shape if mha.rel_bias is not None else (), torch.float32, dev, "d_rel_bias")
    elif want_rel_bias and mha.rel_bias is not None:
        d_rel_bias = torch.empty_like(mha.rel_bias) if stream is None else _new_on(stream, dev, qkv, mha.rel_bias.shape, torch.float32)
    p_ws, ws_bytes, p_rel = None, 0, None
    if d_rel_bias is not None:
        p_rel = d_rel_bias.data_ptr()
        if ws is None:
            ws_bytes = dsvt_set_mha_backward_workspace_size(mha, maps)
            ws = qkv.new_empty(ws_bytes, dtype=torch.uint8) if stream is None else _new_on(stream, dev, qkv, ws_bytes, torch.uint8)
            p_ws = ws.data_ptr()
        else:
            p_ws, ws_bytes = _scratch(ws, dev)
    rc = lib().dsvt_set_mha_backward(mha.ref, C.byref(maps.struct), coords.data_ptr(), qkv.data_ptr(), ld, d_out.data_ptr(), ld_out,
                                     d_qkv.data_ptr(), ld_d, p_rel, p_ws, ws_bytes, _current_stream(dev) if stream is None else stream)
    if rc:
        _check("dsvt_set_mha_backward", rc)
    return d_qkv, d_rel_bias


class LayerNorm:
    """Parameters of one LayerNorm of a residual sum.  gamma, beta: float32 [C]; both stay the caller's: they are read at every call."""

    def __init__(self, gamma, beta, dtype, eps=1e-5):
        code, self.dtype = _DT[dtype]
        self.C, self.gamma, self.beta = gamma.shape[0], gamma, beta
        _vector(gamma, (self.C,), torch.float32, _current_device(), "gamma")
        _vector(beta, (self.C,), torch.float32, _current_device(), "beta")
        self.struct = LnCfg(self.C, code, gamma.data_ptr(), beta.data_ptr(), eps)
        self.ref, self.size, self.device = C.byref(self.struct), (None, 0), _current_device()     # size: the last shape and its workspace bytes


def dsvt_layer_norm(ln, x, res=None, y=None, stream=None):
    """LayerNorm of x + res (of x without res), rows [N, C]; returns y."""
    if _recording():
        _no_graph("dsvt_layer_norm", x, res, ln.gamma, ln.beta, y)
    n, c, dtype, dev = x.shape[0], ln.C, ln.dtype, _current_device()
    if ln.device != dev:
        _elsewhere(dev, ln)
    ld_x = _rows(x, (n, c), dtype, dev, "x")
    ld_res, p_res = (0, None) if res is None else (_rows(res, (n, c), dtype, dev, "res"), res.data_ptr())
    if y is None:
        y, ld_y = x.new_empty((n, c)) if stream is None else _new_on(stream, dev, x, (n, c), dtype), c
    else:
        ld_y = _rows(y, (n, c), dtype, dev, "y")
    rc = lib().dsvt_layer_norm(ln.ref, x.data_ptr(), ld_x, p_res, ld_res, n, y.data_ptr(), ld_y, _current_stream(dev) if stream is None else stream)
    if rc:
        _check("dsvt_layer_norm", rc)
    return y


def dsvt_layer_norm_backward_workspace_size(ln, n_rows):
    last, size = ln.size
    if n_rows != last:
        b = C.c_size_t(0)
        _check("dsvt_layer_norm_backward_workspace_size", lib().dsvt_layer_norm_backward_workspace_size(ln.ref, n_rows, C.byref(b)))
        size = b.value
        ln.size = n_rows, size
    return size


def dsvt_layer_norm_backward(ln, dy, x, res=None, dx=None, d_gamma=None, d_beta=None, ws=None, stream=None):
    """Gradients of dsvt_layer_norm: returns (dx, which is that of x and of res, d_gamma [C], d_beta [C])."""
    if _recording():
        _no_graph("dsvt_layer_norm_backward", dy, x, res, ln.gamma, dx, d_gamma, d_beta)
    n, c, dtype, dev = x.shape[0], ln.C, ln.dtype, _current_device()
    if ln.device != dev:
        _elsewhere(dev, ln)
    ld_dy, ld_x = _rows(dy, (n, c), dtype, dev, "dy"), _rows(x, (n, c), dtype, dev, "x")
    ld_res, p_res = (0, None) if res is None else (_rows(res, (n, c), dtype, dev, "res"), res.data_ptr())
    if dx is None:
        dx, ld_dx = x.new_empty((n, c)) if stream is None else _new_on(stream, dev, x, (n, c), dtype), c
    else:
        ld_dx = _rows(dx, (n, c), dtype, dev, "dx")
    if d_gamma is None:
        d_gamma = torch.empty_like(ln.gamma) if stream is None else _new_on(stream, dev, x, (c,), torch.float32)
    else:
        _vector(d_gamma, (c,), torch.float32, dev, "d_gamma")
    if d_beta is None:
        d_beta = torch.empty_like(ln.gamma) if stream is None else _new_on(stream, dev, x, (c,), torch.float32)
    else:
        _vector(d_beta, (c,), torch.float32, dev, "d_beta")
    if ws is None:
        ws_bytes = dsvt_layer_norm_backward_workspace_size(ln, n)
        ws = x.new_empty(ws_bytes, dtype=torch.uint8) if stream is None else _new_on(stream, dev, x, ws_bytes, torch.uint8)
        p_ws = ws.data_ptr()
    else:
        p_ws, ws_bytes = _scratch(ws, dev)
    rc = lib().dsvt_layer_norm_backward(ln.ref, dy.data_ptr(), ld_dy, x.data_ptr(), ld_x, p_res, ld_res, n, dx.data_ptr(), ld_dx, d_gamma.data_ptr(),
                                        d_beta.data_ptr(), p_ws, ws_bytes, _current_stream(dev) if stream is None else stream)
    if rc:
        _check("dsvt_layer_norm_backward", rc)
    return dx, d_gamma, d_beta


def prof_enable(max_launches):
    _check("dsvt_prof_enable", lib().dsvt_prof_enable(max_launches))


def prof_collect():
    """{kernel name: (total ms, launches)} for the launches recorded since prof_enable."""
    n = lib().dsvt_prof_kernel_count()
    ms, cnt = (C.c_float * n)(), (C.c_int32 * n)()
    _check("dsvt_prof_collect", lib().dsvt_prof_collect(ms, cnt, n))
    return {lib().dsvt_prof_kernel_name(k).decode(): (float(ms[k]), int(cnt[k])) for k in range(n)}
