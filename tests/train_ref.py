"""Plain 64-bit references of the training operators, and how far a result may be from them.

The bounds count roundings.  u = 2^-24 is half a step of float32, h = eps / 2 of the rows' type (bf16 2^-8, fp32 2^-24).  A sum of n terms
is off by at most n u times the sum of their sizes; what is stored in the rows' type, and the operands P and ds of
the products in bf16, by h times their size.
"""
import math

import numpy as np
import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def members(set_inds, n_voxels, dup):
    """Per set: (voxels, weights as keys), the first slot of every run of equal valid slots."""
    out = []
    for row in set_inds.tolist():
        vox, weight, prev = [], [], None
        for v in row:
            v = v if 0 <= v < n_voxels else -1
            if v >= 0 and v != prev:
                vox.append(v)
                weight.append(1)
            elif v >= 0:
                weight[-1] += 1 if dup else 0
            prev = v
        out.append((vox, weight))
    return out


def mha(qkv, sets, coords, win, heads, table, bucket, d_out=None):
    """Double reference: dict of out, and with d_out of d_qkv and d_rel_bias, each with its bound under "<name>_bound".  Rows of
    voxels in no set are NaN in the results (no value).  qkv, d_out: CPU tensors of the rows' type; table: float32 or None."""
    h_step = half_step(qkv.dtype)
    narrow = h_step if qkv.dtype == torch.bfloat16 else 0.0
    n, c3 = qkv.shape
    c = c3 // 3
    d = c // heads
    sig = 1 / math.sqrt(d)
    x = qkv.double().numpy().reshape(n, 3, heads, d)
    g_all = None if d_out is None else d_out.double().numpy().reshape(n, heads, d)
    b_all = None if table is None else table.double().numpy()
    xyz = coords.numpy()[:, 1:]
    out, ob = np.full((n, heads, d), np.nan), np.zeros((n, heads, d))
    dx, db = np.full((n, 3, heads, d), np.nan), np.zeros((n, 3, heads, d))
    dt, dtb, terms = (None, None, None) if table is None else (np.zeros(b_all.shape), np.zeros(b_all.shape), np.zeros(b_all.shape[1]))
    dts = None if table is None else np.zeros(b_all.shape)
    for vox, weight in sets:
        if not vox:
            continue
        m, vi = len(vox), np.array(vox)
        q, k, v = (x[vi, i].transpose(1, 0, 2) for i in range(3))                  # [heads, m, d]
        bias, index = np.zeros((heads, m, m)), np.full((m, m), -1)
        if table is not None:
            p = xyz[vi].astype(np.int64)
            lin, count = np.zeros((m, m), np.int64), 1
            for axis, w in enumerate(win):
                lin = lin * (2 * w - 1) + (p[:, None, axis] - p[None, :, axis]) + w - 1
                count *= 2 * w - 1
            if any(np.ptp(p[:, axis]) >= w for axis, w in enumerate(win)):
                lin[:] = count // 2                 # not one window's voxels: the term of offset 0 for all pairs
            index = lin
            if bucket is not None:
                e = bucket.numpy()[np.clip(index, 0, None)]
                index = np.where((index >= 0) & (e >= 0) & (e < b_all.shape[1]), e, -1)
            bias = np.where(index >= 0, b_all[:, np.clip(index, 0, None)], 0.0)
        dot, size = q @ k.transpose(0, 2, 1) * sig, np.abs(q) @ np.abs(k).transpose(0, 2, 1) * sig
        s = dot + bias
        top = s.max(2, keepdims=True)
        with np.errstate(invalid="ignore"):
            e = np.where(np.isneginf(top), 0.0, np.exp(s - np.where(np.isneginf(top), 0.0, top))) * np.array(weight, float)
        total = e.sum(2, keepdims=True)
        pr = np.divide(e, total, out=np.zeros_like(e), where=total != 0)
        # a logit is off by (d + 6) roundings of its parts (products' sum, scale, table, sum, difference to the largest), P relatively by
        # twice the largest such error among the pair and the rest of the sum, and by m + 8 roundings of exp, weight, sum and division
        # (a bias next to the lowest float leaves no digits of q.k: comparable only where all keys have the same one, and then exact)
        fin = np.where(np.abs(bias) < 1e30, np.abs(bias), 0.0)
        es = (d + 6) * U * (size + fin) + 2 * U * np.where(np.abs(s) < 1e30, np.abs(s), 0.0)
        es = np.where(pr > 0, es, 0.0)
        rel = es + es.max(2, keepdims=True) + (m + 8) * U
        rel = np.expm1(rel)
        out[vi] = (pr @ v).transpose(1, 0, 2)
        av = np.abs(v)
        ob[vi] = (((rel + narrow + (m + 2) * U) * pr) @ av).transpose(1, 0, 2) * (1 + h_step) + h_step * np.abs(out[vi])
        if g_all is None:
            continue
        g = g_all[vi].transpose(1, 0, 2)
        ag = np.abs(g)
        t, ts = g @ v.transpose(0, 2, 1), ag @ av.transpose(0, 2, 1)
        D = (pr * t).sum(2, keepdims=True)
        et = d * U * ts
        eD = (pr * (rel * np.abs(t) + et)).sum(2, keepdims=True) + (m + 2) * U * (pr * np.abs(t)).sum(2, keepdims=True)
        ds = pr * (t - D)
        eds = pr * ((rel + 2 * U) * np.abs(t - D) + et + eD + U * (np.abs(t) + np.abs(D)))
        dv = pr.transpose(0, 2, 1) @ g
        dq, dk = sig * (ds @ k), sig * (ds.transpose(0, 2, 1) @ q)
        wide = eds + (narrow + (m + 4) * U) * np.abs(ds)                            # as operands of products of m terms
        wide_p = (rel + narrow + (m + 4) * U) * pr
        for i, val, err in ((0, dq, sig * (wide @ np.abs(k))), (1, dk, sig * (wide.transpose(0, 2, 1) @ np.abs(q))),
                            (2, dv, wide_p.transpose(0, 2, 1) @ ag)):
            dx[vi, i] = val.transpose(1, 0, 2)
            db[vi, i] = (err * (1 + h_step) + h_step * np.abs(val)).transpose(1, 0, 2)
        if table is not None:
            for hh in range(heads):
                np.add.at(dt[hh], index[index >= 0], ds[hh][index >= 0])
                np.add.at(dtb[hh], index[index >= 0], eds[hh][index >= 0])
                np.add.at(dts[hh], index[index >= 0], np.abs(ds[hh])[index >= 0])
            np.add.at(terms, index[index >= 0], 1)
    r = {"out": out.reshape(n, c), "out_bound": ob.reshape(n, c)}
    if g_all is not None:
        r |= {"d_qkv": dx.reshape(n, c3), "d_qkv_bound": db.reshape(n, c3)}
        if table is not None:
            r |= {"d_rel_bias": dt, "d_rel_bias_bound": dtb + (terms + 8) * U * dts}
    return r


def layer_norm(x, res, gamma, beta, eps, dy=None):
    """Double reference of LayerNorm of x + res and of its gradients, with bounds; CPU tensors."""
    hs = half_step(x.dtype)
    c, rows = x.shape[1], x.shape[0]
    depth = max(40, c // 256 + 12)                  # additions behind one sum over a row
    z = x.double() + (0 if res is None else res.double())
    g, b = gamma.double(), beta.double()
    mean = z.mean(1, keepdim=True)
    dev = z - mean
    rs = 1 / (dev.pow(2).mean(1, keepdim=True) + eps).sqrt()
    n = dev * rs
    e_dev = U * (z.abs() + dev.abs()) + depth * U * z.abs().mean(1, keepdim=True)
    rel_rs = rs * e_dev.pow(2).mean(1, keepdim=True).sqrt() + (depth + 6) * U
    e_n = rs * e_dev + n.abs() * (rel_rs + 2 * U)
    y = n * g + b
    r = {"y": y, "y_bound": e_n * g.abs() + 2 * U * ((n * g).abs() + b.abs()) + hs * y.abs() * (1 + U) + 1e-38}
    if dy is not None:
        d = dy.double()
        w = d * g
        mw, mwn = w.mean(1, keepdim=True), (w * n).mean(1, keepdim=True)
        dx = rs * (w - mw - n * mwn)
        e_mw = (depth + 2) * U * w.abs().mean(1, keepdim=True)
        e_mwn = (depth + 3) * U * (w * n).abs().mean(1, keepdim=True) + (w.abs() * e_n).mean(1, keepdim=True)
        e = rs * (4 * U * (w.abs() + mw.abs() + (n * mwn).abs()) + e_mw + e_n * mwn.abs() + n.abs() * e_mwn) + (rel_rs + 2 * U) * dx.abs()
        long = rows / 512 + 64                      # additions behind one sum over the rows: a workgroup's, and over the workgroups
        r |= {"dx": dx, "dx_bound": e * (1 + hs) + hs * dx.abs() + 1e-38,
              "d_gamma": (d * n).sum(0), "d_gamma_bound": (d.abs() * e_n).sum(0) + long * U * (d * n).abs().sum(0) + 1e-38,
              "d_beta": d.sum(0), "d_beta_bound": long * U * d.abs().sum(0) + 1e-38}
    return r


def check(name, got, ref, case=""):
    """got (a tensor) against ref[name] within ref[name + "_bound"]; values that the reference does not have are not compared."""
    want, bound = (torch.as_tensor(ref[k]).double() for k in (name, name + "_bound"))
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (case, name, got.shape, want.shape)
    there = ~want.isnan()
    off = (got - want).abs()
    assert bool(got[there].isfinite().all()), f"{case} {name}: not finite"
    worst = float((off[there] / bound[there].clamp(min=1e-300)).max()) if bool(there.any()) else 0.0
    print(f"[err] {case} {name}: largest error {float(off[there].max()) if bool(there.any()) else 0.0:.3g}, {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{case} {name}: {worst:.3g} times its bound"
