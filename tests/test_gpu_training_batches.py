"""dsvt_set_mha and its backward call where a workgroup goes through many sets: look-ups of later sets beside earlier ones, rows fetched ahead, turns
over several rounds, a last batch that is not full.  Element by element against the 64-bit reference."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
dsvt = pytest.importorskip("paper_2301_06051_amd")
import train_ref as ref  # noqa: E402

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _sets(seed, n_sets, tau, win, sizes, repeats):
    """(set_inds [n_sets, tau], coords [N, 4]): sets of random ones of `sizes` voxels at random cells of a window of their own, each voxel in one set.
    repeats: slots left over repeat voxels, else they are empty."""
    rng = np.random.default_rng(seed)
    of = rng.choice(sizes, n_sets)
    n = int(of.sum())
    order = rng.permutation(n)                       # rows of a set lie anywhere
    inds, coords, at = np.full((n_sets, tau), -1, np.int32), np.zeros((n, 4), np.int32), 0
    for s, m in enumerate(of):
        vox = order[at:at + m]
        at += m
        cell = rng.choice(win[0] * win[1] * win[2], m, replace=False)
        coords[vox, 1] = s % 512 * win[0] + cell // (win[1] * win[2])
        coords[vox, 2] = s // 512 * win[1] + cell // win[2] % win[1]
        coords[vox, 3] = cell % win[2]
        if m and repeats:
            inds[s] = vox[np.arange(tau) * m // tau]
        else:
            inds[s, :m] = vox
    return torch.from_numpy(inds), torch.from_numpy(coords)


# C, heads, dtype, window, tau, repeats are keys, buckets (exact, side), sets, their sizes.  A backward workgroup takes as many sets a batch as it has
# wavefronts (eight, or four); a forward call has up to twice as many workgroups.
CASES = {
    # eight heads a workgroup: one set at a time, rows held in registers and the next set's fetched ahead
    "one_slot": (256, 32, "bf16", (8, 8, 1), 48, 0, None, 3300, (0, 1, 2, 16, 17, 33, 48)),
    "one_slot_repeats_f32": (256, 32, "f32", (8, 8, 1), 40, 1, (2, 4), 2900, (0, 1, 3, 16, 17, 40)),
    # two heads a workgroup: four sets side by side, which take turns at the table's sums
    "four_slots": (32, 2, "bf16", (7, 7, 1), 33, 1, None, 9200, (0, 1, 2, 3, 17, 33)),
    "buckets_slots": (128, 16, "bf16", (12, 12, 32), 36, 0, (4, 7), 4700, (0, 1, 2, 16, 36)),
    "tiny_sets": (64, 8, "bf16", (3, 3, 1), 4, 0, (1, 2), 13001, (0, 1, 2, 3, 4)),
    # tables and sums that LDS does not hold: several workgroups go through the same sets
    "in_memory": (256, 32, "bf16", (30, 30, 20), 20, 0, None, 2300, (0, 1, 2, 3, 20)),
    "in_memory_f32": (64, 2, "f32", (30, 30, 20), 40, 1, None, 500, (0, 1, 17, 40)),
    # sets above 48 voxels: rows read again for each query tile, look-ups after a batch's sets
    "large_sets": (256, 32, "bf16", (10, 10, 1), 96, 0, None, 1200, (0, 1, 16, 17, 49, 65, 96)),
    "large_sets_slots": (48, 2, "bf16", (10, 10, 1), 64, 1, (2, 4), 4500, (0, 1, 2, 17, 64)),
    # four wavefronts a workgroup
    "wide_heads_f32": (256, 4, "f32", (6, 6, 1), 20, 0, None, 4300, (0, 1, 2, 16, 20)),
}


@pytest.mark.parametrize("name", CASES)
def test_set_mha_over_many_batches(name):
    c, heads, dtype, win, tau, dup, buckets, n_sets, sizes = CASES[name]
    inds, coords = _sets(len(name) + tau, n_sets, tau, win, sizes, dup or tau % 2)
    n = coords.shape[0]
    print("[case]", name, n_sets, "sets", n, "voxels", flush=True)
    bucket, n_rel = dsvt.dsvt_rel_buckets(win, *buckets) if buckets else (None, (2 * win[0] - 1) * (2 * win[1] - 1) * (2 * win[2] - 1))
    bucket = None if bucket is None else torch.from_numpy(bucket)
    g = torch.Generator().manual_seed(n_sets)
    qkv, d_out = torch.randn((n, 3 * c), generator=g).to(DT[dtype]), torch.randn((n, c), generator=g).to(DT[dtype])
    table = 0.5 * torch.randn((heads, n_rel), generator=g)
    # the number of sets says more than there is room for: what has room is computed
    maps = dsvt.SetMaps.of(inds.cuda(), torch.tensor([n_sets + (100 if name == "tiny_sets" else 0)], dtype=torch.int32, device="cuda"), n)
    mha = dsvt.SetMha(c, heads, dtype, win, table.cuda(), None if bucket is None else bucket.cuda(), dup)
    parts = dsvt.dsvt_set_mha_backward_workspace_size(mha, maps) // (4 * heads * (n_rel + (bucket is not None)))
    assert n_sets > 2 * 8 * parts                    # three batches at least, the last not full
    out = dsvt.dsvt_set_mha(mha, maps, coords.cuda(), qkv.cuda())
    d_qkv, d_rel = dsvt.dsvt_set_mha_backward(mha, maps, coords.cuda(), qkv.cuda(), d_out.cuda())
    torch.cuda.synchronize()
    r = ref.mha(qkv, ref.members(inds, n, dup), coords, win, heads, table, bucket, d_out)
    for key, got in (("out", out), ("d_qkv", d_qkv), ("d_rel_bias", d_rel)):
        ref.check(key, got, r, name)
