"""The operators a DSVT layer's training step needs beside matrix products, as cases that can be timed: set attention on
projected rows with a learned relative position bias (one entry an offset, or by buckets), and layer norm of a residual
sum; each forward and backward.

Set attention takes the slot maps of a partition, the voxel coordinates and the projected rows qkv [N, 3C]; backward takes
the gradient of its output and gives that of qkv and of the bias table.  Layer norm takes x and the branch r that is added
to it; backward gives the gradient of the sum (which is both x's and r's) and of gamma and beta.
"""
import math

import torch

own = False

EPS = 1e-5


def _ln(name, n, c, dtype, res, back):
    return {"name": name, "op": "ln_bwd" if back else "ln", "n": n, "c": c, "dtype": dtype, "res": res}


def _mha(name, x, y, z, win, win_z, shift, tau, n, batch, c, heads, dtype, dist, exact, side, repeats, order, back):
    """exact / side: offsets up to exact - 1 cells along an axis have buckets of their own, longer ones share the other
    side - exact by their logarithm; side = 0: one entry an offset.  repeats: repeated slots stay keys."""
    return {"name": name, "op": "mha_bwd" if back else "mha", "gx": x, "gy": y, "gz": z, "win": win, "win_z": win_z, "shift": shift, "tau": tau,
            "n": n, "batch": batch, "c": c, "heads": heads, "dtype": dtype, "dist": dist, "exact": exact, "side": side, "repeats": repeats,
            "order": order}


def listed():
    return [
        # one row: the smallest call there is, launch and host time
        _ln("ln_one_row", 1, 192, "bf16", True, False),
        # the norm after the attention of a pillar frame
        _ln("ln_pillar", 30000, 192, "bf16", True, False),
        # training step of the small fp32 model
        _ln("ln_bwd_small_f32", 2000, 64, "f32", True, True),
        # a width that is no multiple of a vector, no residual
        _ln("ln_bwd_odd", 9973, 99, "f32", False, True),
        # the largest: a batch of four crowded frames
        _ln("ln_bwd_batch4", 800000, 192, "bf16", True, True),
        # the small fp32 model on a small grid
        _mha("mha_small_f32", 48, 48, 1, 12, 1, 0, 36, 2000, 1, 64, 4, "f32", "uniform", 0, 0, False, "key", False),
        # the ordinary pillar frame
        _mha("mha_pillar", 468, 468, 1, 12, 1, 0, 36, 30000, 1, 192, 8, "bf16", "radial", 0, 0, False, "key", False),
        # the 3D voxel frame, 15 x 15 x 11 buckets for 23 x 23 x 15 offsets, rows in no order
        _mha("mha_voxel_buckets", 468, 468, 32, 12, 8, 6, 48, 120000, 1, 192, 8, "bf16", "radial", 4, 6, False, "random", False),
        # training step of the ordinary pillar frame
        _mha("mha_bwd_pillar", 468, 468, 1, 12, 1, 6, 36, 30000, 1, 192, 8, "bf16", "radial", 0, 0, False, "key", True),
        # the wide-window pillar model: 30 x 30 windows, sets of 90, repeated slots kept as keys
        _mha("mha_bwd_wide", 360, 360, 1, 30, 1, 15, 90, 20000, 1, 128, 8, "bf16", "radial", 0, 0, True, "key", True),
        # fp32 training of the small model, with buckets
        _mha("mha_bwd_small_f32", 48, 48, 1, 12, 1, 6, 36, 2000, 1, 64, 4, "f32", "uniform", 3, 5, False, "random", True),
        # the largest: four frames whose voxels crowd into few tall windows
        _mha("mha_bwd_skewed4", 468, 468, 32, 12, 32, 0, 36, 200000, 4, 192, 8, "bf16", "skewed", 4, 7, False, "key", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    back = rng.random() < 0.6
    if rng.random() < 0.4:
        c = rng.choice([64, 128, 192, 192, 256, _log(rng, 32, 768)])
        n = _log(rng, 1, 800000 * 192 // max(c, 192))
        dtype = rng.choice(["bf16", "bf16", "f32"])
        case = _ln("", n // 2 + 1 if dtype == "f32" else n, c, dtype, rng.random() < 0.7, back)
    else:
        form = rng.choice(["small", "pillar", "pillar", "wide", "voxel", "voxel"])
        c, heads = rng.choice([(64, 4), (128, 8), (192, 8), (192, 8), (96, 4), (128, 2), (256, 8)])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"]) if form in ("small", "pillar") else "bf16"
        dist, order, repeats = rng.choice(["radial", "uniform"]), rng.choice(["key", "random"]), rng.random() < 0.3
        exact = rng.randint(2, 4)
        side = rng.choice([0, exact + rng.randint(1, 4)])
        if form == "small":
            g, w = rng.randint(24, 120), rng.randint(8, 16)
            case = _mha("", g, g + rng.randint(0, 9), 1, w, 1, rng.choice([0, w // 2]), rng.choice([24, 36, 48]), _log(rng, 1, 500), 1, c, heads,
                        dtype, dist, exact, side, repeats, order, back)
        elif form == "voxel":
            wz = rng.choice([8, 32])
            case = _mha("", 468, 468, 32, 12, wz, rng.choice([0, 6]), rng.choice([36, 48]), _log(rng, 20000, 150000), rng.choice([1, 2]), c,
                        heads, dtype, rng.choice(["radial", "skewed"]), exact, side, repeats, order, back)
        elif form == "wide":
            case = _mha("", 360, 360, 1, 30, 1, rng.choice([0, 15]), rng.choice([60, 90]), _log(rng, 1500, 30000), rng.choice([1, 2]), c, heads,
                        dtype, dist, exact, side, repeats, order, back)
        else:
            w = rng.choice([12, 12, 24])
            case = _mha("", 468, 468, 1, w, 1, rng.choice([0, w // 2]), rng.choice([36, 36, 48]), _log(rng, 1500, 50000), rng.choice([1, 2, 4]), c,
                        heads, dtype, dist, exact, side, repeats, order, back)
    del case["name"]
    return case


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _windows(case):
    return (case["win"], case["win"], case["win_z"]), (case["shift"], case["shift"], 0)


def _frames(case, gen):
    """int32 [batch * n, 4] distinct cells (b, x, y, z): n of a frame's cells are drawn without repetition, each with a weight
    (1/r around the middle with a height profile near the ground and uniform clutter; or a twentieth of the windows holding
    most of the weight)."""
    gx, gy, gz, b, n = case["gx"], case["gy"], case["gz"], case["batch"], case["n"]
    f = dict(device="cuda", dtype=torch.float32)
    x, y, z = (torch.arange(g, **f) for g in (gx, gy, gz))
    w = torch.ones((gx, gy, gz), **f)
    if case["dist"] == "radial":
        r = ((x[:, None] - gx / 2 + 0.5) ** 2 + (y[None, :] - gy / 2 + 0.5) ** 2).sqrt().clamp(min=1.0)
        high = 0.1 / gz + torch.softmax(-((z - 5.0) / 3.0) ** 2 / 2, 0)
        w = 0.2 / (gx * gy * gz) + 0.8 * ((1 / r) / (1 / r).sum())[:, :, None] * high
    elif case["dist"] == "skewed":
        (l, k, h), _ = _windows(case)
        nw = (-(-gx // l), -(-gy // k), -(-gz // h))
        hot = torch.rand(nw, device="cuda", generator=gen) < 0.05
        share = torch.where(hot, 0.7 / hot.sum().clamp(min=1), 0.3 / (~hot).sum().clamp(min=1))
        w = share[(x // l).long()][:, (y // k).long()][:, :, (z // h).long()]
    u = torch.rand((b, gx * gy * gz), device="cuda", generator=gen)
    cells = (w.reshape(1, -1).log() - (-(u.clamp(min=1e-30).log())).clamp(min=1e-30).log()).topk(n, dim=1).indices.sort(dim=1).values
    cells = (cells + torch.arange(b, device="cuda")[:, None] * (gx * gy * gz)).reshape(-1)
    if case["order"] == "random":
        cells = cells[torch.randperm(cells.numel(), device="cuda", generator=gen)]
    return torch.stack([cells // (gx * gy * gz), cells // (gy * gz) % gx, cells // gz % gy, cells % gz], 1).to(torch.int32)


def _maps(case, coords):
    """Slot maps of the X-axis partition: a window of N voxels has S = ceil(N / tau) sets, slot k of its j-th set holds the voxel
    of inner rank floor((j tau + k) N / (S tau)).  Returns set_inds [bound, tau] (-1 past the sets) and their number."""
    win, shift = _windows(case)
    tau, n = case["tau"], coords.shape[0]
    c = coords.long()
    key = c[:, 0]
    for a, g in enumerate((case["gx"], case["gy"], case["gz"])):
        key = key * (-(-(g + shift[a]) // win[a])) + (c[:, a + 1] + shift[a]) // win[a]
    inner = torch.zeros_like(key)
    for a in range(3):
        inner = inner * win[a] + (c[:, a + 1] + shift[a]) % win[a]
    rank = (key * (win[0] * win[1] * win[2]) + inner).argsort()
    _, count = key[rank].unique_consecutive(return_counts=True)
    sets = (count + tau - 1) // tau
    first = count.cumsum(0) - count
    of = torch.repeat_interleave(torch.arange(len(sets), device="cuda"), sets)
    j = torch.arange(len(of), device="cuda") - (sets.cumsum(0) - sets)[of]
    slot = (j[:, None] * tau + torch.arange(tau, device="cuda")) * count[of][:, None] // (sets[of] * tau)[:, None]
    windows = case["batch"] * math.prod(-(-(g + s) // w) for g, s, w in zip((case["gx"], case["gy"], case["gz"]), shift, win))
    inds = torch.full((n // tau + min(n, windows), tau), -1, dtype=torch.int32, device="cuda")
    inds[:len(of)] = rank[first[of][:, None] + slot].to(torch.int32)
    return inds, len(of)


def _buckets(case):
    """Bucket of every offset (x most significant), signed along each axis, and the number of buckets."""
    win, _ = _windows(case)
    e, b, index, total = case["exact"], case["side"], torch.zeros(1, dtype=torch.int64), 1
    for w in win:
        d = torch.arange(1 - w, w)
        most = min(b, w)
        far = e + ((d.abs().clamp(min=1).double() / e).log() / math.log(max(w, e + 1) / e) * (most - e)).floor().long()
        near = torch.where(d.abs() < e, d.abs(), far.clamp(max=most - 1)).clamp(max=most - 1)
        index = (index[:, None] * (2 * most - 1) + (near * d.sign() + most - 1)).reshape(-1)
        total *= 2 * most - 1
    return index.to(torch.int32).cuda(), total


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, c = _type(case), case["c"]
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    if case["op"].startswith("ln"):
        n = case["n"]
        # rows as a layer has them: x left by the norm before, r out of a projection, a gradient of small values
        s = {"op": case["op"], "x": normal(n, c).to(t), "r": (0.5 * normal(n, c) + 0.1).to(t) if case["res"] else None,
             "gamma": 1 + 0.1 * normal(c), "beta": 0.1 * normal(c), "dy": (1e-2 * normal(n, c)).to(t)}
        if own:
            import paper_2301_06051_amd as dsvt
            s["ln"] = dsvt.LayerNorm(s["gamma"], s["beta"], case["dtype"], EPS)
        return s
    coords = _frames(case, gen)
    n, win = coords.shape[0], _windows(case)[0]
    inds, n_sets = _maps(case, coords)
    offsets = math.prod(2 * w - 1 for w in win)
    bucket, n_rel = _buckets(case) if case["side"] else (None, offsets)
    s = {"op": case["op"], "heads": case["heads"], "win": win, "repeats": case["repeats"], "coords": coords, "set_inds": inds, "sets": n_sets,
         "n_sets": torch.tensor([n_sets], dtype=torch.int32, device="cuda"), "bucket": bucket, "rel_bias": 0.5 * normal(case["heads"], n_rel),
         "qkv": normal(n, 3 * c).to(t), "d_out": (1e-2 * normal(n, c)).to(t)}
    if own:
        import paper_2301_06051_amd as dsvt
        s["mha"] = dsvt.SetMha(c, case["heads"], case["dtype"], win, s["rel_bias"], bucket, int(case["repeats"]))
        s["maps"] = dsvt.SetMaps.of(inds, s["n_sets"], n)
    return s


def _sum(s):
    return s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()


def _normed(z):
    m = z - z.mean(1, keepdim=True)
    r = torch.rsqrt((m * m).mean(1, keepdim=True) + EPS)
    return m * r, r


def _attend(s):
    """Gathered rows and probabilities of every set: (voxels [S, tau], first slots of a voxel [S, tau], q, k, v [S, heads, tau, d],
    buckets [S, tau, tau], P [S, heads, tau, tau])."""
    vox = s["set_inds"][:s["sets"]].long()
    first = torch.ones_like(vox, dtype=torch.bool)
    first[:, 1:] = vox[:, 1:] != vox[:, :-1]
    n, c3 = s["qkv"].shape
    h = s["heads"]
    q, k, v = s["qkv"].float()[vox].reshape(*vox.shape, 3, h, c3 // 3 // h).permute(2, 0, 3, 1, 4)
    at = s["coords"].long()[vox][:, :, 1:]
    l, w, d = s["win"]
    code = (at[..., 0] * (2 * w - 1) + at[..., 1]) * (2 * d - 1) + at[..., 2]
    offset = code[:, :, None] - code[:, None, :] + ((l - 1) * (2 * w - 1) + w - 1) * (2 * d - 1) + d - 1
    rel = offset if s["bucket"] is None else s["bucket"].long()[offset]
    logits = (q @ k.transpose(2, 3)) * (1 / math.sqrt(q.shape[-1])) + s["rel_bias"][:, rel].transpose(0, 1)
    if not s["repeats"]:
        logits = logits.masked_fill(~first[:, None, None, :], -math.inf)
    e = (logits - logits.amax(3, keepdim=True)).exp()
    return vox, first, q, k, v, rel, e / e.sum(3, keepdim=True)


def _rows(slots, vox, first, like):
    """The values at the first slots [S, heads, tau, d], as rows of their voxels [N, heads * d]."""
    out = torch.empty((like.shape[0], slots.shape[1] * slots.shape[3]), dtype=like.dtype, device=like.device)
    out[vox[first]] = slots.transpose(1, 2).flatten(2)[first].to(like.dtype)
    return out


def run(s):
    op = s["op"]
    if own:
        import paper_2301_06051_amd as dsvt
        if op == "ln":
            return {"y": dsvt.dsvt_layer_norm(s["ln"], s["x"], s["r"])}
        if op == "ln_bwd":
            dx, dg, db = dsvt.dsvt_layer_norm_backward(s["ln"], s["dy"], s["x"], s["r"])
            return {"dx": dx, "d_gamma": dg, "d_beta": db}
        if op == "mha":
            return {"out": dsvt.dsvt_set_mha(s["mha"], s["maps"], s["coords"], s["qkv"])}
        d_qkv, d_rel = dsvt.dsvt_set_mha_backward(s["mha"], s["maps"], s["coords"], s["qkv"], s["d_out"])
        return {"d_qkv": d_qkv, "d_rel_bias": d_rel}
    if op == "ln":
        n, _ = _normed(_sum(s))
        return {"y": (n * s["gamma"] + s["beta"]).to(s["x"].dtype)}
    if op == "ln_bwd":
        n, r = _normed(_sum(s))
        dy = s["dy"].float()
        w = dy * s["gamma"]
        dx = r * (w - w.mean(1, keepdim=True) - n * (w * n).mean(1, keepdim=True))
        # sums over all rows are long: in 64 bits
        return {"dx": dx.to(s["x"].dtype), "d_gamma": (dy * n).sum(0, dtype=torch.float64).float(), "d_beta": dy.sum(0, dtype=torch.float64).float()}
    vox, first, q, k, v, rel, p = _attend(s)
    if op == "mha":
        return {"out": _rows(p @ v, vox, first, s["qkv"])}
    g = s["d_out"].float()[vox].reshape(*vox.shape, s["heads"], -1).transpose(1, 2) * first[:, None, :, None]
    dv = p.transpose(2, 3) @ g
    t = g @ v.transpose(2, 3)
    ds = p * (t - (p * t).sum(3, keepdim=True))
    scale = 1 / math.sqrt(q.shape[-1])
    dq, dk = (ds @ k) * scale, (ds.transpose(2, 3) @ q) * scale
    if s["repeats"]:        # slots of one voxel are one row: their gradients add up
        rows = s["qkv"].shape[0]
        d_qkv = torch.zeros((rows, s["qkv"].shape[1]), device="cuda")
        d_qkv.index_add_(0, vox.reshape(-1), torch.cat([a.transpose(1, 2).flatten(2) for a in (dq, dk, dv)], 2).flatten(0, 1))
        d_qkv = d_qkv.to(s["qkv"].dtype)
    else:
        d_qkv = torch.cat([_rows(a, vox, first, s["qkv"]) for a in (dq, dk, dv)], 1)
    # a bucket's sum runs over every set: in 64 bits, as differences of the running sum over the pairs in the buckets' order
    bucket, order = rel.reshape(-1).sort()
    sums = torch.nn.functional.pad(ds.transpose(0, 1).flatten(1)[:, order].double().cumsum(1), (1, 0))
    ends = torch.searchsorted(bucket, torch.arange(s["rel_bias"].shape[1] + 1, device="cuda"))
    return {"d_qkv": d_qkv, "d_rel_bias": sums[:, ends].diff(dim=1).float()}


def work(case):
    e, c = (2 if case["dtype"] == "bf16" else 4), case["c"]
    if case["op"].startswith("ln"):
        rows = 2 + int(case["res"]) + int(case["op"] == "ln_bwd")
        return {"bytes": rows * case["n"] * c * e + (4 if case["op"] == "ln_bwd" else 2) * c * 4,
                "flops": (16 if case["op"] == "ln_bwd" else 8) * case["n"] * c}
    n, back = case["n"] * case["batch"], case["op"] == "mha_bwd"
    win, _ = _windows(case)
    entries = math.prod(2 * (min(case["side"], w) if case["side"] else w) - 1 for w in win)
    # a set holds about half as many voxels as it has slots
    pairs = n * max(1, case["tau"] // 2)
    return {"bytes": (7 if back else 4) * n * c * e + 20 * n + (2 if back else 1) * case["heads"] * entries * 4,
            "flops": (10 if back else 4) * c * pairs}


def exact(case, seed):
    """The same outputs in 64 bits: every voxel's row taken once a set with the number of its slots as its weight (or 1), and
    gradients by automatic differentiation of the definition."""
    s = prepare(case, seed)
    dbl = lambda a: None if a is None else a.detach().double().requires_grad_()  # noqa: E731
    if case["op"].startswith("ln"):
        x, r, g, b = dbl(s["x"]), dbl(s["r"]), dbl(s["gamma"]), dbl(s["beta"])
        z = x if r is None else x + r
        var, mean = torch.var_mean(z, 1, correction=0, keepdim=True)
        y = (z - mean) / (var + EPS).sqrt() * g + b
        if case["op"] == "ln":
            return {"y": y.detach()}
        dx, dg, db = torch.autograd.grad(y, (x, g, b), s["dy"].double())
        return {"dx": dx, "d_gamma": dg, "d_beta": db}
    inds = s["set_inds"][:s["sets"]].long()
    run_start = torch.cat([torch.ones_like(inds[:, :1], dtype=torch.bool), inds.diff(dim=1) != 0], 1)
    place = run_start.long().cumsum(1) - 1                                   # place of a slot's voxel among the set's voxels
    most = int(place.max()) + 1
    weight = torch.zeros((len(inds), most), dtype=torch.float64, device="cuda").scatter_add_(1, place, torch.ones_like(inds, dtype=torch.float64))
    member = torch.zeros((len(inds), most), dtype=torch.int64, device="cuda").scatter_(1, place, inds)
    there = weight > 0
    qkv = dbl(s["qkv"])
    n, h = qkv.shape[0], case["heads"]
    d = case["c"] // h
    rows = qkv.reshape(n, 3, h, d)[member]                                   # [S, m, 3, h, d]
    q, k, v = (rows[:, :, i].permute(0, 2, 1, 3).contiguous() for i in range(3))
    xyz = s["coords"].long()[member][..., 1:]
    step = xyz[:, :, None] - xyz[:, None, :]
    win = _windows(case)[0]
    both = there[:, :, None] & there[:, None, :]
    index = torch.zeros_like(step[..., 0])
    for a in range(3):
        index = index * (2 * win[a] - 1) + torch.where(both, step[..., a], 0) + win[a] - 1
    if s["bucket"] is not None:
        index = s["bucket"].long()[index]
    bias = dbl(s["rel_bias"][:, index])                                      # [h, S, m, m]
    logit = torch.matmul(q, k.transpose(2, 3).contiguous()) / math.sqrt(d) + bias.transpose(0, 1)
    keys = (weight if case["repeats"] else there.double()).clamp(min=1e-300).log()
    logit = (logit + keys[:, None, None, :]).masked_fill(~there[:, None, None, :], -math.inf)
    slots = torch.matmul(torch.softmax(logit, 3), v).transpose(1, 2).flatten(2)
    where = torch.zeros(n, dtype=torch.int64, device="cuda")
    where[member[there]] = torch.arange(there.numel(), device="cuda").reshape(there.shape)[there]
    out = slots.flatten(0, 1)[where]
    if case["op"] == "mha":
        return {"out": out.detach()}
    d_qkv, d_bias = torch.autograd.grad(out, (qkv, bias), s["d_out"].double())
    index, order = index.flatten().sort()
    entry, count = index.unique_consecutive(return_counts=True)
    d_table = torch.zeros(s["rel_bias"].shape, dtype=torch.float64, device="cuda")
    d_table[:, entry] = torch.segment_reduce(d_bias.flatten(1)[:, order].t().contiguous(), "sum", lengths=count, axis=0).t()
    return {"d_qkv": d_qkv, "d_rel_bias": d_table}
