"""dsvt_set_mha, dsvt_layer_norm and their backward calls against plain 64-bit references, element by element."""
import math

import numpy as np
import pytest
import torch

import synth

pytestmark = pytest.mark.gpu
dsvt = pytest.importorskip("paper_2301_06051_amd")
import train_ref as ref  # noqa: E402
from gpu_util import TOL, dev_coords, dev_feats, gpu_maps, rel_err  # noqa: E402

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _inputs(seed, n, c, dtype, heads, n_rel, bias_scale=0.5):
    g = _gen(seed)
    qkv, d_out = torch.randn((n, 3 * c), generator=g).to(DT[dtype]), torch.randn((n, c), generator=g).to(DT[dtype])
    table = None if n_rel is None else bias_scale * torch.randn((heads, n_rel), generator=g)
    return qkv, d_out, table


def _run(coords, maps, win, c, heads, dtype, qkv, d_out, table, bucket=None, dup=0, case=""):
    """Both directions on the GPU against the reference; returns the GPU results."""
    cd, xd, gd = coords.cuda(), qkv.cuda(), d_out.cuda()
    td, bd = None if table is None else table.cuda(), None if bucket is None else bucket.cuda()
    mha = dsvt.SetMha(c, heads, dtype, win, td, bd, dup)
    out = dsvt.dsvt_set_mha(mha, maps, cd, xd)
    d_qkv, d_rel = dsvt.dsvt_set_mha_backward(mha, maps, cd, xd, gd)
    torch.cuda.synchronize()
    inds = maps.set_inds[:int(maps.n_sets.item())].cpu()
    r = ref.mha(qkv, ref.members(inds, maps.n_voxels, dup), coords, win, heads, table, bucket, d_out)
    ref.check("out", out, r, case)
    ref.check("d_qkv", d_qkv, r, case)
    if table is not None:
        ref.check("d_rel_bias", d_rel, r, case)
    else:
        assert d_rel is None
    return out, d_qkv, d_rel


def _frame(seed, grid, n, batch=1):
    rng = np.random.default_rng(seed)
    rows = []
    for b in range(batch):
        cell = rng.permutation(grid[0] * grid[1] * grid[2])[:n]
        rows.append(np.stack([np.full(n, b), cell // (grid[1] * grid[2]), cell // grid[2] % grid[1], cell % grid[2]], 1))
    return torch.from_numpy(np.concatenate(rows).astype(np.int32))


CASES = [
    # C, heads, dtype, grid, voxels a frame, batch, window, tau, repeats are keys, buckets (exact, side)
    (64, 4, "f32", (48, 48, 1), 700, 1, (12, 12, 1), 36, 0, None),
    (64, 4, "f32", (30, 20, 1), 400, 2, (12, 12, 1), 36, 1, (3, 5)),
    (64, 4, "bf16", (30, 20, 1), 1, 1, (12, 12, 1), 36, 0, None),
    (192, 8, "bf16", (40, 40, 1), 900, 1, (12, 12, 1), 36, 0, None),
    (192, 8, "bf16", (25, 25, 8), 900, 1, (12, 12, 8), 48, 1, (4, 6)),
    (128, 8, "bf16", (60, 60, 1), 1800, 1, (30, 30, 1), 90, 0, None),
    (128, 8, "bf16", (31, 31, 1), 500, 1, (30, 30, 1), 96, 1, (2, 6)),
    (96, 4, "f32", (24, 24, 2), 500, 1, (8, 8, 2), 65, 0, None),
    (128, 2, "bf16", (24, 24, 2), 300, 1, (8, 8, 2), 24, 0, (2, 4)),
    (128, 2, "f32", (24, 24, 2), 300, 1, (8, 8, 2), 64, 1, None),
    (40, 1, "bf16", (24, 24, 1), 200, 1, (9, 7, 1), 1, 0, None),
    (56, 7, "bf16", (24, 24, 1), 200, 1, (9, 7, 1), 17, 1, None),
    (264, 11, "bf16", (20, 20, 1), 150, 1, (12, 12, 1), 33, 0, (1, 3)),
    (192, 12, "f32", (20, 20, 1), 150, 1, (12, 12, 1), 32, 1, (1, 1)),
    (256, 8, "bf16", (20, 20, 1), 250, 1, (12, 12, 1), 48, 0, (3, 4)),
    (144, 3, "bf16", (24, 24, 1), 300, 1, (12, 12, 1), 60, 1, None),
    (96, 3, "f32", (24, 24, 1), 300, 1, (12, 12, 1), 48, 0, None),
    (128, 4, "bf16", (24, 24, 1), 400, 1, (20, 20, 1), 96, 0, None),
    (48, 3, "f32", (24, 24, 1), 400, 1, (20, 20, 1), 96, 1, (4, 8)),
    (16, 2, "bf16", (30, 30, 1), 700, 1, (12, 12, 1), 16, 0, None),
]


@pytest.mark.parametrize("c,heads,dtype,grid,n,batch,win,tau,dup,buckets", CASES)
def test_set_mha_and_gradients(c, heads, dtype, grid, n, batch, win, tau, dup, buckets):
    case = f"C{c} h{heads} {dtype} {grid} n{n}x{batch} win{win} tau{tau} dup{dup} {buckets}"
    print("[case]", case, flush=True)
    coords = _frame(n + c, grid, n, batch)
    maps = gpu_maps(coords.cuda(), grid, win, tuple(w // 2 for w in win), tau, batch, 0)
    if buckets:
        b, n_rel = dsvt.dsvt_rel_buckets(win, *buckets)
        bucket = torch.from_numpy(b)
    else:
        bucket, n_rel = None, synth.weights.rel_table_size(win)
    qkv, d_out, table = _inputs(c + n, n * batch, c, dtype, heads, n_rel)
    _run(coords, maps, win, c, heads, dtype, qkv, d_out, table, bucket, dup, case)


@pytest.mark.parametrize("dtype,c,heads", [("bf16", 192, 8), ("f32", 64, 4)])
def test_set_mha_without_a_positional_term(dtype, c, heads):
    coords = _frame(5, (40, 40, 1), 300)
    maps = gpu_maps(coords.cuda(), (40, 40, 1), (12, 12, 1), (0, 0, 0), 36, 1, 1)
    qkv, d_out, _ = _inputs(6, 300, c, dtype, heads, None)
    print("[case] no table", dtype, flush=True)
    _run(coords, maps, (12, 12, 1), c, heads, dtype, qkv, d_out, None, case="no table " + dtype)


@pytest.mark.parametrize("win,buckets", [((12, 12, 32), None), ((12, 12, 32), (4, 7)), ((24, 24, 1), None), ((12, 12, 8), None), ((30, 30, 20), None),
                                         ((30, 30, 32), (2, 4))])
def test_set_mha_large_tables(win, buckets):
    """Tables that LDS holds for all heads, for a few, for one, or not at all (their sums then shared out over workgroups)."""
    grid = (30, 30, win[2])
    n = 700
    coords = _frame(7, grid, n)
    maps = gpu_maps(coords.cuda(), grid, win, (6, 6, 0), 36, 1, 0)
    b, n_rel = dsvt.dsvt_rel_buckets(win, *buckets) if buckets else (None, synth.weights.rel_table_size(win))
    qkv, d_out, table = _inputs(8, n, 192, "bf16", 8, n_rel)
    print("[case] table", win, buckets, n_rel, flush=True)
    _run(coords, maps, win, 192, 8, "bf16", qkv, d_out, table, None if b is None else torch.from_numpy(b), case=f"table {win} {buckets}")


def _one_window(sets, n, tau, slots):
    """Maps by hand: rows of `slots` (padded with -1), with rows of rubbish past n_sets."""
    inds = torch.full((sets + 3, tau), 2 ** 31 - 1, dtype=torch.int32)
    for i, row in enumerate(slots):
        inds[i] = torch.tensor(list(row) + [-1] * (tau - len(row)), dtype=torch.int32)
    return dsvt.SetMaps.of(inds.cuda(), torch.tensor([sets], dtype=torch.int32, device="cuda"), n)


@pytest.mark.parametrize("dup", [0, 1])
@pytest.mark.parametrize("dtype,c,heads", [("bf16", 192, 8), ("f32", 64, 4), ("bf16", 128, 2)])
def test_set_mha_empty_slots_sets_and_rows(dtype, c, heads, dup):
    """Slots that hold no voxel (-1 or out of range, in front, between and behind), a set of none, sets of 1, 16, 17 and 64 voxels, voxels in
    no set whose rows hold NaN: neither read nor written."""
    n, tau, win = 130, 70, (16, 16, 1)
    coords = torch.stack([torch.zeros(n), torch.arange(n) // 16, torch.arange(n) % 16, torch.zeros(n)], 1).to(torch.int32)
    slots = [[-1, 3, 3, 3, -1, 130, 4, 4, 5], [], [6], [v for v in range(10, 26) for _ in range(3)], list(range(30, 47)),
             [-7] + list(range(50, 114)) + [113, 113]]
    maps = _one_window(len(slots), n, tau, slots)
    qkv, d_out, table = _inputs(9, n, c, dtype, heads, synth.weights.rel_table_size(win))
    used = torch.zeros(n, dtype=torch.bool)
    for row in slots:
        used[[v for v in row if 0 <= v < n]] = True
    qkv[~used] = math.nan
    d_out[~used] = math.inf
    mha = dsvt.SetMha(c, heads, dtype, win, table.cuda(), None, dup)
    out = torch.full((n, c), 7.0, dtype=DT[dtype], device="cuda")
    d_qkv = torch.full((n, 3 * c), 7.0, dtype=DT[dtype], device="cuda")
    print("[case] empty slots", dtype, c, dup, flush=True)
    dsvt.dsvt_set_mha(mha, maps, coords.cuda(), qkv.cuda(), out=out)
    _, d_rel = dsvt.dsvt_set_mha_backward(mha, maps, coords.cuda(), qkv.cuda(), d_out.cuda(), d_qkv=d_qkv)
    torch.cuda.synchronize()
    r = ref.mha(qkv, ref.members(maps.set_inds[:len(slots)].cpu(), n, dup), coords, win, heads, table, None, d_out)
    for name, got in (("out", out), ("d_qkv", d_qkv), ("d_rel_bias", d_rel)):
        ref.check(name, got, r, "empty slots")
    assert bool((out.cpu()[~used] == 7).all()) and bool((d_qkv.cpu()[~used] == 7).all())


@pytest.mark.parametrize("low", [-math.inf, float(torch.finfo(torch.float32).min)])
@pytest.mark.parametrize("dtype,c,heads,tau", [("bf16", 192, 8, 36), ("f32", 64, 4, 36), ("bf16", 128, 8, 90)])
def test_set_mha_biases_that_mask(dtype, c, heads, tau, low):
    """Head 0: every pair masked; head 1: all but a voxel's own cell; head 2: cells to one side.  -inf everywhere leaves a row of zeros
    without a gradient, the lowest finite value everywhere is the same for all keys and masks none."""
    win, n = (12, 12, 1), 250
    coords = _frame(10, (20, 20, 1), n)
    maps = gpu_maps(coords.cuda(), (20, 20, 1), win, (0, 0, 0), tau, 1, 0)
    qkv, d_out, table = _inputs(11, n, c, dtype, heads, synth.weights.rel_table_size(win))
    centre = table.shape[1] // 2
    table[0] = low
    table[1] = low
    table[1, centre] = 0.3
    table[2, :centre] = low
    print("[case] masking biases", dtype, tau, low, flush=True)
    if math.isinf(low):
        out, d_qkv, d_rel = _run(coords, maps, win, c, heads, dtype, qkv, d_out, table, case=f"masks {low}")
        d = c // heads
        assert bool((out[:, :d] == 0).all()) and bool((d_qkv[:, :d] == 0).all()) and bool((d_rel[0] == 0).all())
    else:
        # a logit next to the lowest value has no digits left for q.k: all keys of head 0 weigh the same, in 64 bits they are that only
        # after the logits' rounding, which the zeroed queries do in the reference
        d = c // heads
        qkv[:, :d] = 0
        _run(coords, maps, win, c, heads, dtype, qkv, d_out, table, case=f"masks {low}")


@pytest.mark.parametrize("dtype,tau", [("bf16", 36), ("f32", 36), ("bf16", 90)])
def test_set_mha_logits_of_any_size(dtype, tau):
    """Logits of up to 1e11: the probabilities are one key's alone wherever the largest logit stands out, and everything is finite."""
    win, n, c, heads = (12, 12, 1), 250, 64, 4
    coords = _frame(61, (20, 20, 1), n)
    maps = gpu_maps(coords.cuda(), (20, 20, 1), win, (0, 0, 0), tau, 1, 0)
    qkv, d_out, table = _inputs(62, n, c, dtype, heads, synth.weights.rel_table_size(win))
    qkv[:, :2 * c] *= 2.0 ** 17
    print("[case] large logits", dtype, tau, flush=True)
    mha = dsvt.SetMha(c, heads, dtype, win, table.cuda())
    out = dsvt.dsvt_set_mha(mha, maps, coords.cuda(), qkv.cuda()).cpu()
    d_qkv, d_rel = dsvt.dsvt_set_mha_backward(mha, maps, coords.cuda(), qkv.cuda(), d_out.cuda())
    assert all(bool(t.isfinite().all()) for t in (out, d_qkv, d_rel))
    x, d, clear = qkv.double().reshape(n, 3, heads, c // heads), c // heads, 0
    for vox, _ in ref.members(maps.set_inds[:int(maps.n_sets)].cpu(), n, 0):
        s = torch.einsum("qhd,khd->hqk", x[vox, 0], x[vox, 1])
        best = s.topk(min(2, len(vox)), dim=2).values
        # sums of 16 products in 32 bits are off by 2^-20 of their sizes at most: 1e5 of a logit here
        stands_out = (best[..., 0] - best[..., -1] > 1e6) | (len(vox) == 1)
        want = x[vox, 2].permute(1, 0, 2).gather(1, s.argmax(2)[..., None].expand(-1, -1, d))
        got = out.double().reshape(n, heads, d)[vox].permute(1, 0, 2)
        assert torch.equal(got[stands_out], want[stands_out])
        clear += int(stands_out.sum())
    assert clear > n * heads * 0.9


def test_set_mha_backward_without_the_tables_gradient():
    win, n, c, heads = (12, 12, 1), 250, 192, 8
    coords = _frame(63, (20, 20, 1), n)
    maps = gpu_maps(coords.cuda(), (20, 20, 1), win, (0, 0, 0), 36, 1, 0)
    qkv, d_out, table = (t.cuda() for t in _inputs(64, n, c, "bf16", heads, 529))
    mha = dsvt.SetMha(c, heads, "bf16", win, table)
    both, rel = dsvt.dsvt_set_mha_backward(mha, maps, coords.cuda(), qkv, d_out)
    alone, none = dsvt.dsvt_set_mha_backward(mha, maps, coords.cuda(), qkv, d_out, want_rel_bias=False)
    assert none is None and rel is not None and torch.equal(alone, both)


def test_calls_refuse_tensors_that_do_not_fit():
    coords = _frame(65, (20, 20, 1), 50).cuda()
    maps = gpu_maps(coords, (20, 20, 1), (12, 12, 1), (0, 0, 0), 36, 1, 0)
    qkv, d_out, table = (t.cuda() for t in _inputs(66, 50, 64, "bf16", 4, 529))
    mha = dsvt.SetMha(64, 4, "bf16", (12, 12, 1), table)
    ln = dsvt.LayerNorm(torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), "bf16")
    for bad in (qkv.float(), qkv[:49], qkv[:, :128], qkv.cpu(), qkv.t().contiguous().t()):
        with pytest.raises(ValueError):
            dsvt.dsvt_set_mha(mha, maps, coords, bad)
        with pytest.raises(ValueError):
            dsvt.dsvt_set_mha_backward(mha, maps, coords, bad, d_out)
    for bad in (d_out.float(), d_out[:3], d_out.cpu()):
        with pytest.raises(ValueError):
            dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, bad)
        with pytest.raises(ValueError):
            dsvt.dsvt_layer_norm_backward(ln, bad, d_out)
    with pytest.raises(dsvt.DsvtError):                       # a broadcast gradient: rows of stride 0
        dsvt.dsvt_layer_norm_backward(ln, d_out[:1].expand(50, 64), d_out)
    with pytest.raises(dsvt.DsvtError):                       # rows that do not start on 16 bytes
        dsvt.dsvt_set_mha(mha, maps, coords, torch.zeros((50, 200), dtype=torch.bfloat16, device="cuda")[:, 4:196])
    with pytest.raises(ValueError):
        dsvt.SetMha(64, 4, "bf16", (12, 12, 1), table, torch.zeros(528, dtype=torch.int32, device="cuda"))


def test_set_mha_buckets_outside_the_table_are_no_term():
    win, n, c, heads = (12, 12, 1), 250, 192, 8
    coords = _frame(12, (30, 30, 1), n)
    maps = gpu_maps(coords.cuda(), (30, 30, 1), win, (0, 0, 0), 36, 1, 0)
    qkv, d_out, table = _inputs(13, n, c, "bf16", heads, 7)
    bucket = torch.randint(-2, 10, (23 * 23,), generator=_gen(14), dtype=torch.int32)
    bucket[5] = 2 ** 31 - 1
    print("[case] buckets out of range", flush=True)
    _run(coords, maps, win, c, heads, "bf16", qkv, d_out, table, bucket, case="buckets out of range")


def test_set_mha_sets_that_fit_no_window_take_the_term_of_offset_0():
    """Maps built with another window than the table's: nothing is read or added outside it."""
    n, c, heads, win = 200, 64, 4, (3, 3, 1)
    coords = _frame(15, (60, 60, 1), n)
    maps = gpu_maps(coords.cuda(), (60, 60, 1), (30, 30, 1), (0, 0, 0), 36, 1, 0)
    qkv, d_out, table = _inputs(16, n, c, "f32", heads, 25)
    print("[case] far voxels", flush=True)
    _run(coords, maps, win, c, heads, "f32", qkv, d_out, table, case="far voxels")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_set_mha_strided_rows(dtype):
    """Slices of wider arrays on both sides; what lies between the rows stays as it is."""
    c, heads, n, win = 64, 4, 220, (12, 12, 1)
    coords = _frame(17, (24, 24, 1), n)
    maps = gpu_maps(coords.cuda(), (24, 24, 1), win, (6, 6, 0), 36, 1, 0)
    qkv, d_out, table = _inputs(18, n, c, dtype, heads, 529)
    wide = lambda t, w: torch.full((n, t + w), 5.0, dtype=DT[dtype], device="cuda")[:, 8:8 + t]  # noqa: E731
    xs, gs, os_, ds = wide(3 * c, 24), wide(c, 16), wide(c, 40), wide(3 * c, 16)
    xs.copy_(qkv)
    gs.copy_(d_out)
    mha = dsvt.SetMha(c, heads, dtype, win, table.cuda())
    print("[case] strided", dtype, flush=True)
    assert dsvt.dsvt_set_mha(mha, maps, coords.cuda(), xs, out=os_) is os_
    _, d_rel = dsvt.dsvt_set_mha_backward(mha, maps, coords.cuda(), xs, gs, d_qkv=ds)
    r = ref.mha(qkv, ref.members(maps.set_inds[:int(maps.n_sets)].cpu(), n, 0), coords, win, heads, table, None, d_out)
    for name, got in (("out", os_), ("d_qkv", ds), ("d_rel_bias", d_rel)):
        ref.check(name, got, r, "strided")
    for t in (os_, ds):
        assert bool((t._base[:, :8] == 5).all()) and bool((t._base[:, 8 + t.shape[1]:] == 5).all())


def test_set_mha_offsets_past_32_bits():
    """Row strides that put the last rows of every array past 2^31 elements."""
    c, heads, n, win = 64, 4, 40, (12, 12, 1)
    coords = _frame(19, (12, 12, 1), n)
    maps = gpu_maps(coords.cuda(), (12, 12, 1), win, (0, 0, 0), 36, 1, 0)
    qkv, d_out, table = _inputs(20, n, c, "bf16", heads, 529)
    ld = 2 ** 26 + 64
    buf = torch.empty((n * ld,), dtype=torch.bfloat16, device="cuda")
    view = lambda at, w: buf.as_strided((n, w), (ld, 1), at)  # noqa: E731
    xs, gs, os_, ds = view(0, 3 * c), view(1024, c), view(2048, c), view(4096, 3 * c)
    xs.copy_(qkv)
    gs.copy_(d_out)
    mha = dsvt.SetMha(c, heads, "bf16", win, table.cuda())
    print("[case] far rows", flush=True)
    dsvt.dsvt_set_mha(mha, maps, coords.cuda(), xs, out=os_)
    dsvt.dsvt_set_mha_backward(mha, maps, coords.cuda(), xs, gs, d_qkv=ds)
    r = ref.mha(qkv, ref.members(maps.set_inds[:int(maps.n_sets)].cpu(), n, 0), coords, win, heads, table, None, d_out)
    ref.check("out", os_, r, "far rows")
    ref.check("d_qkv", ds, r, "far rows")


def test_set_mha_gradients_against_differences():
    """Central differences of sum(out * d_out) in the kernel's own fp32 results, along random directions of q, k, v and the table."""
    c, heads, n, win = 64, 4, 90, (12, 12, 1)
    coords = _frame(21, (12, 12, 1), n)
    maps = gpu_maps(coords.cuda(), (12, 12, 1), win, (0, 0, 0), 36, 1, 0)
    qkv, d_out, table = (t.cuda() for t in _inputs(22, n, c, "f32", heads, 529))
    cd = coords.cuda()
    value = lambda x, t: float((dsvt.dsvt_set_mha(dsvt.SetMha(c, heads, "f32", win, t), maps, cd, x).double() * d_out.double()).sum())  # noqa: E731
    d_qkv, d_rel = dsvt.dsvt_set_mha_backward(dsvt.SetMha(c, heads, "f32", win, table), maps, cd, qkv, d_out)
    g = torch.Generator(device="cuda").manual_seed(23)
    step = 2.0 ** -7
    for part in ("q", "k", "v", "table"):
        dirx, dirt = torch.zeros_like(qkv), torch.zeros_like(table)
        if part == "table":
            dirt.normal_(generator=g)
        else:
            i = "qkv".index(part)
            dirx[:, i * c:(i + 1) * c].normal_(generator=g)
        slope = float((d_qkv.double() * dirx.double()).sum() + (d_rel.double() * dirt.double()).sum())
        diff = (value(qkv + step * dirx, table + step * dirt) - value(qkv - step * dirx, table - step * dirt)) / (2 * step)
        # the third derivative's term, step^2 / 6 of a sum of n * c values whose third derivatives are of order |direction of a logit|^3 ~ 8, adding up like
        # random ones, and the fp32 roundings of the values, 2^-22 sqrt(n c) / step: together under 2e-3 of sqrt(n c) * 8
        bound = (step ** 2 / 6 * 8 * 8 + 2.0 ** -22 / step) * math.sqrt(n * c)
        print(f"[err] differences {part}: {slope:.6g} against {diff:.6g}, bound {bound:.3g}", flush=True)
        assert abs(slope - diff) <= bound


@pytest.mark.parametrize("win,c,heads,buckets", [((12, 12, 1), 192, 8, None), ((12, 12, 32), 192, 8, (4, 7)), ((12, 12, 32), 128, 8, None), ((12, 12, 8), 64, 4, None)])
def test_set_mha_backward_repeats_bit_for_bit(win, c, heads, buckets):
    grid, n = (60, 60, win[2]), 3000
    coords = _frame(24, grid, n)
    maps = gpu_maps(coords.cuda(), grid, win, (0, 0, 0), 36, 1, 0)
    b, n_rel = dsvt.dsvt_rel_buckets(win, *buckets) if buckets else (None, synth.weights.rel_table_size(win))
    qkv, d_out, table = (t.cuda() for t in _inputs(25, n, c, "bf16", heads, n_rel))
    mha = dsvt.SetMha(c, heads, "bf16", win, table, None if b is None else torch.from_numpy(b).cuda())
    print("[case] repeats", win, buckets, flush=True)
    cd = coords.cuda()
    want = dsvt.dsvt_set_mha_backward(mha, maps, cd, qkv, d_out)
    for _ in range(10):
        got = dsvt.dsvt_set_mha_backward(mha, maps, cd, qkv, d_out)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


LN_CASES = [(1, 192, "bf16", True), (2000, 64, "f32", True), (333, 192, "bf16", True), (777, 128, "bf16", False), (513, 256, "f32", False),
            (100, 99, "f32", True), (100, 99, "bf16", False), (33, 1, "f32", True), (65, 7, "bf16", True), (40, 320, "bf16", True),
            (40, 600, "f32", True), (20, 1000, "bf16", False), (19, 2048, "bf16", True), (9, 2056, "bf16", True), (9, 1500, "f32", True),
            (600, 257, "f32", True), (5, 5001, "bf16", True), (3, 65536, "f32", False), (40000, 64, "bf16", True), (16, 48, "f32", True), (700, 24, "bf16", True), (70, 700, "bf16", True),
            (70, 701, "bf16", False), (70, 401, "bf16", True), (50, 1023, "f32", True), (30, 1900, "bf16", True), (30, 4096, "bf16", True), (30, 8192, "bf16", True),
            (30, 4096, "f32", False), (700, 2056, "f32", True), (600, 1025, "bf16", True)]


@pytest.mark.parametrize("n,c,dtype,with_res", LN_CASES)
def test_layer_norm_and_gradients(n, c, dtype, with_res):
    case = f"ln {n}x{c} {dtype} res{int(with_res)}"
    print("[case]", case, flush=True)
    g = _gen(n + c)
    x = (torch.randn((n, c), generator=g) + 0.5).to(DT[dtype])
    r = (0.5 * torch.randn((n, c), generator=g)).to(DT[dtype]) if with_res else None
    gamma, beta = 1 + 0.1 * torch.randn(c, generator=g), 0.1 * torch.randn(c, generator=g)
    dy = torch.randn((n, c), generator=g).to(DT[dtype])
    ln = dsvt.LayerNorm(gamma.cuda(), beta.cuda(), dtype, 1e-5)
    rd = None if r is None else r.cuda()
    y = dsvt.dsvt_layer_norm(ln, x.cuda(), rd)
    dx, dg, db = dsvt.dsvt_layer_norm_backward(ln, dy.cuda(), x.cuda(), rd)
    want = ref.layer_norm(x, r, gamma, beta, 1e-5, dy)
    for name, got in (("y", y), ("dx", dx), ("d_gamma", dg), ("d_beta", db)):
        ref.check(name, got, want, case)
    again = dsvt.dsvt_layer_norm_backward(ln, dy.cuda(), x.cuda(), rd)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dg, db)))


@pytest.mark.parametrize("dtype,c,off,pad", [("bf16", 192, 8, 24), ("bf16", 192, 3, 5), ("f32", 64, 1, 2), ("f32", 100, 4, 4), ("bf16", 2050, 1, 1)])
def test_layer_norm_strided_and_unaligned_rows(dtype, c, off, pad):
    n = 77
    g = _gen(c + off)
    gamma, beta = 1 + 0.1 * torch.randn(c, generator=g), 0.1 * torch.randn(c, generator=g)
    t = lambda: torch.full((n, off + c + pad), 3.0, dtype=DT[dtype], device="cuda")[:, off:off + c]  # noqa: E731
    host = [torch.randn((n, c), generator=g).to(DT[dtype]) for _ in range(3)]
    x, r, dy, y, dx = (t() for _ in range(5))
    for a, b in zip((x, r, dy), host):
        a.copy_(b)
    ln = dsvt.LayerNorm(gamma.cuda(), beta.cuda(), dtype, 1e-5)
    print("[case] ln strided", dtype, c, off, flush=True)
    dsvt.dsvt_layer_norm(ln, x, r, y=y)
    _, dg, db = dsvt.dsvt_layer_norm_backward(ln, dy, x, r, dx=dx)
    want = ref.layer_norm(host[0], host[1], gamma, beta, 1e-5, host[2])
    for name, got in (("y", y), ("dx", dx), ("d_gamma", dg), ("d_beta", db)):
        ref.check(name, got, want, "ln strided")
    for a in (y, dx):
        assert bool((a._base[:, :off] == 3).all()) and bool((a._base[:, off + c:] == 3).all())


@pytest.mark.parametrize("c", [192, 2100])
def test_layer_norm_in_place(c):
    n, g = 130, _gen(c)
    x, r, dy = (torch.randn((n, c), generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    ln = dsvt.LayerNorm(torch.randn(c, generator=g).cuda(), torch.randn(c, generator=g).cuda(), "bf16")
    y, (dx, dg, db) = dsvt.dsvt_layer_norm(ln, x, r), dsvt.dsvt_layer_norm_backward(ln, dy, x, r)
    dy2 = dy.clone()
    got = dsvt.dsvt_layer_norm_backward(ln, dy2, x, r, dx=dy2)
    assert torch.equal(dy2, dx) and torch.equal(got[1], dg) and torch.equal(got[2], db)
    for k in (0, 1):
        a = [x.clone(), r.clone()]
        dsvt.dsvt_layer_norm(ln, *a, y=a[k])
        assert torch.equal(a[k], y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_norm_rows_without_variance_and_with_large_means(dtype):
    """Constant rows (only eps keeps the division finite), rows of zeros, a mean a thousand times the deviation, an infinity and a NaN (which stay in their rows)."""
    c = 192
    g = _gen(31)
    x = torch.randn((8, c), generator=g)
    x[0], x[1], x[2] = 2.0, 0.0, 1000.0 + x[2]
    x = x.to(DT[dtype])
    gamma, beta, dy = torch.randn(c, generator=g), torch.randn(c, generator=g), torch.randn((8, c), generator=g).to(DT[dtype])
    ln = dsvt.LayerNorm(gamma.cuda(), beta.cuda(), dtype, 1e-5)
    want = ref.layer_norm(x, None, gamma, beta, 1e-5, dy)
    dx, dg, db = dsvt.dsvt_layer_norm_backward(ln, dy.cuda(), x.cuda())
    for name, got in (("y", dsvt.dsvt_layer_norm(ln, x.cuda())), ("dx", dx), ("d_gamma", dg), ("d_beta", db)):
        ref.check(name, got, want, "ln special rows")
    bad = x.clone()
    bad[3, 5], bad[4, 6] = math.inf, math.nan
    y = dsvt.dsvt_layer_norm(ln, bad.cuda()).cpu()
    dx2 = dsvt.dsvt_layer_norm_backward(ln, dy.cuda(), bad.cuda())[0].cpu()
    keep = [0, 1, 2, 5, 6, 7]
    assert bool(y[3:5].isnan().all()) and torch.equal(y[keep], dsvt.dsvt_layer_norm(ln, x.cuda()).cpu()[keep])
    assert bool(dx2[3:5].isnan().all()) and torch.equal(dx2[keep], dx.cpu()[keep])


def test_layer_norm_offsets_past_32_bits():
    n, c = 11_200_001, 192
    x = torch.zeros((n, c), dtype=torch.bfloat16, device="cuda")
    g = _gen(32)
    rows = torch.randn((5, c), generator=g).to(torch.bfloat16)
    x[-5:] = rows.cuda()
    gamma, beta = torch.randn(c, generator=g), torch.randn(c, generator=g)
    ln = dsvt.LayerNorm(gamma.cuda(), beta.cuda(), "bf16")
    print("[case] ln far rows", flush=True)
    y = dsvt.dsvt_layer_norm(ln, x)
    ref.check("y", y[-5:], ref.layer_norm(rows, None, gamma, beta, 1e-5), "ln far rows")
    del y
    dx, dg, _ = dsvt.dsvt_layer_norm_backward(ln, x, x)
    want = ref.layer_norm(rows, None, gamma, beta, 1e-5, rows)
    ref.check("dx", dx[-5:], want, "ln far rows")
    ref.check("d_gamma", dg, want, "ln far rows")            # the other rows' gradients are zeros


def test_calls_without_rows():
    ln = dsvt.LayerNorm(torch.ones(192, device="cuda"), torch.ones(192, device="cuda"), "bf16")
    none = torch.empty((0, 192), dtype=torch.bfloat16, device="cuda")
    assert dsvt.dsvt_layer_norm(ln, none, none).shape == (0, 192)
    dx, dg, db = dsvt.dsvt_layer_norm_backward(ln, none, none, d_gamma=torch.ones(192, device="cuda"), d_beta=torch.ones(192, device="cuda"))
    assert dx.shape == (0, 192) and not dg.any() and not db.any()
    mha = dsvt.SetMha(192, 8, "bf16", (12, 12, 1), torch.ones((8, 529), device="cuda"))
    maps = dsvt.SetMaps.of(torch.empty((0, 36), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda"), 0)
    coords, rows = torch.empty((0, 4), dtype=torch.int32, device="cuda"), torch.empty((0, 576), dtype=torch.bfloat16, device="cuda")
    assert dsvt.dsvt_set_mha(mha, maps, coords, rows).shape == (0, 192)
    d_qkv, d_rel = dsvt.dsvt_set_mha_backward(mha, maps, coords, rows, none, d_rel_bias=torch.ones((8, 529), device="cuda"))
    assert d_qkv.shape == (0, 576) and not d_rel.any()
    # voxels, but no sets (n_sets = 0)
    maps = dsvt.SetMaps.of(torch.zeros((4, 36), dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda"), 9)
    coords, rows = torch.zeros((9, 4), dtype=torch.int32, device="cuda"), torch.ones((9, 576), dtype=torch.bfloat16, device="cuda")
    out = dsvt.dsvt_set_mha(mha, maps, coords, rows, out=torch.full((9, 192), 7.0, dtype=torch.bfloat16, device="cuda"))
    _, d_rel = dsvt.dsvt_set_mha_backward(mha, maps, coords, rows, rows[:, :192], d_rel_bias=torch.ones((8, 529), device="cuda"))
    assert bool((out == 7).all()) and not d_rel.any()


class _Step:
    """One DSVT layer's training step out of the library's operators and matrix products, as a training program has it (weights of
    the rows' type; post-norm: y = LN2(h + W2 gelu(W1 h)), h = LN1(x + Wo attention(Wqkv x)))."""

    def __init__(self, w, win, maps, coords):
        t = dsvt.LayerWeights(w).t
        self.t, self.maps, self.coords = t, maps, coords
        self.mha = dsvt.SetMha(w["C"], w["heads"], w["dtype"], win, t["rel_bias"])
        self.ln1 = dsvt.LayerNorm(t["ln1_g"], t["ln1_b"], w["dtype"], w["ln_eps"])
        self.ln2 = dsvt.LayerNorm(t["ln2_g"], t["ln2_b"], w["dtype"], w["ln_eps"])

    def linear(self, x, name):
        return torch.addmm(self.t["b_" + name].to(x.dtype), x, self.t["w_" + name].t())

    def forward(self, x):
        qkv = self.linear(x, "qkv")
        o = dsvt.dsvt_set_mha(self.mha, self.maps, self.coords, qkv)
        r1 = self.linear(o, "o")
        h = dsvt.dsvt_layer_norm(self.ln1, x, r1)
        u = self.linear(h, "1")
        a = torch.nn.functional.gelu(u)
        r2 = self.linear(a, "2")
        return dsvt.dsvt_layer_norm(self.ln2, h, r2), (qkv, o, r1, h, u, a, r2)

    def backward(self, x, kept, dy):
        qkv, o, r1, h, u, a, r2 = kept
        grads = {}

        def linear_back(d, inp, name):
            grads["w_" + name], grads["b_" + name] = d.t() @ inp, d.float().sum(0)
            return d @ self.t["w_" + name]

        dz2, grads["ln2_g"], grads["ln2_b"] = dsvt.dsvt_layer_norm_backward(self.ln2, dy, h, r2)
        da = linear_back(dz2, a, "2")
        du = torch.ops.aten.gelu_backward(da, u)
        dh = dz2 + linear_back(du, h, "1")
        dz1, grads["ln1_g"], grads["ln1_b"] = dsvt.dsvt_layer_norm_backward(self.ln1, dh, x, r1)
        do = linear_back(dz1, o, "o")
        d_qkv, grads["rel_bias"] = dsvt.dsvt_set_mha_backward(self.mha, self.maps, self.coords, qkv, do)
        grads["x"] = dz1 + linear_back(d_qkv, x, "qkv")
        return grads


def _layer_reference(w, sets, coords, x, dy):
    """The same layer in 64 bits on the CPU, with gradients by automatic differentiation."""
    p = {k: torch.as_tensor(v).double().requires_grad_() for k, v in w.items() if isinstance(v, np.ndarray)}
    xd = x.double().requires_grad_()
    n, c = x.shape
    h, d = w["heads"], c // w["heads"]
    qkv = (xd @ p["w_qkv"].t() + p["b_qkv"]).reshape(n, 3, h, d)
    parts, order = [], []
    for vox, _ in sets:
        v = torch.tensor(vox)
        q, k, val = (qkv[v, i].transpose(0, 1) for i in range(3))
        xyz = coords[v][:, 1:].long()
        at = torch.zeros((len(vox), len(vox)), dtype=torch.long)
        for a, win in enumerate(w["win"]):
            at = at * (2 * win - 1) + xyz[:, None, a] - xyz[None, :, a] + win - 1
        s = torch.softmax(q @ k.transpose(1, 2) / math.sqrt(d) + p["rel_bias"][:, at], -1)
        parts.append((s @ val).transpose(0, 1).reshape(len(vox), c))
        order += vox
    o = torch.cat(parts)[torch.tensor(order).argsort()]
    norm = torch.nn.functional.layer_norm
    hh = norm(xd + o @ p["w_o"].t() + p["b_o"], (c,), p["ln1_g"], p["ln1_b"], w["ln_eps"])
    m = torch.nn.functional.gelu(hh @ p["w_1"].t() + p["b_1"]) @ p["w_2"].t() + p["b_2"]
    y = norm(hh + m, (c,), p["ln2_g"], p["ln2_b"], w["ln_eps"])
    names = list(p)
    grads = torch.autograd.grad(y, [xd] + [p[k] for k in names], dy.double())
    return y.detach(), dict(zip(["x"] + names, grads))


@pytest.mark.parametrize("c,heads,hidden,dtype", [(64, 4, 128, "f32"), (192, 8, 384, "bf16")])
def test_layer_training_step(c, heads, hidden, dtype):
    """A whole layer's forward and backward pass out of these operators: the output is that of the fused inference layer within its
    bar, the gradients are those of the 64-bit layer."""
    grid, win, tau, n = (40, 40, 1), (12, 12, 1), 36, 800
    coords = _frame(41, grid, n)
    cd = coords.cuda()
    maps = gpu_maps(cd, grid, win, (6, 6, 0), tau, 1, 0)
    w = synth.make_layer_weights(42, c, heads, hidden, win, dtype)
    x = torch.randn((n, c), generator=_gen(43)).to(DT[dtype])
    dy = torch.randn((n, c), generator=_gen(44)).to(DT[dtype])
    print("[case] layer step", dtype, flush=True)
    step = _Step(w, win, maps, cd)
    y, kept = step.forward(x.cuda())
    grads = step.backward(x.cuda(), kept, dy.cuda())
    sets = ref.members(maps.set_inds[:int(maps.n_sets)].cpu(), n, 0)
    want, wgrads = _layer_reference(w, sets, coords, x, dy)
    assert rel_err(y, want.numpy()) < TOL[dtype]
    # A gradient has passed through about ten tensors of the rows' type on its way (each off by half a step of its size, independently, most by a
    # part of it): ten half steps of bf16 are 4 %, of the gradient's root mean square; in fp32 sums of up to n terms count too
    bound = 10 * ref.half_step(DT[dtype]) if dtype == "bf16" else 1e-4
    for name, g in grads.items():
        a, b = g.detach().cpu().double(), wgrads[name]
        off = float((a - b).norm() / b.norm())
        print(f"[err] layer step {dtype} d {name}: {off:.3g}", flush=True)
        assert off < bound, name
    # and as a block beside the fused inference path: both layers of it
    layers = [dsvt.LayerWeights(w), dsvt.LayerWeights(w)]
    fused = dsvt.dsvt_block(layers, [maps, maps], cd, x.cuda())
    twice, _ = step.forward(y)
    assert rel_err(twice, fused.double().cpu().numpy()) < 2 * TOL[dtype]


def test_training_step_in_a_graph_and_on_other_streams():
    """Captured once, replayed with eager work in between (on the same scratch too); two eager steps on streams of their own at once."""
    grid, win, n = (60, 60, 1), (12, 12, 1), 2000
    coords = _frame(51, grid, n).cuda()
    maps = gpu_maps(coords, grid, win, (0, 0, 0), 36, 1, 0)
    b, n_rel = dsvt.dsvt_rel_buckets(win, 3, 5)
    qkv, d_out, table = (t.cuda() for t in _inputs(52, n, 192, "bf16", 8, n_rel))
    mha = dsvt.SetMha(192, 8, "bf16", win, table, torch.from_numpy(b).cuda())
    ln = dsvt.LayerNorm(torch.randn(192, device="cuda"), torch.randn(192, device="cuda"), "bf16")

    def step():
        o = dsvt.dsvt_set_mha(mha, maps, coords, qkv)
        y = dsvt.dsvt_layer_norm(ln, qkv[:, :192], o)
        dz, dg, db = dsvt.dsvt_layer_norm_backward(ln, d_out, qkv[:, :192], o)
        return (y, dg, db, *dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, dz))

    print("[case] graph and streams", flush=True)
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    keep = qkv.clone()
    for rep in range(4):
        for t in got:
            t.fill_(9)
        qkv.neg_()
        step()                                                   # eager work between the replays, on other values
        qkv.copy_(keep)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), rep
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            results.append(step())
    torch.cuda.synchronize()
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(r, want))
    # the stream given by its handle: scratch that the call allocates itself stays until that stream is done with it
    s = streams[0]
    s.wait_stream(torch.cuda.current_stream())
    outs = [dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, d_out, stream=s.cuda_stream) for _ in range(3)]
    junk = [torch.full((1 << 22,), 77, dtype=torch.uint8, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    plain = dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, d_out)
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, plain)) and len(junk) == 8
