"""Operators for layers whose rows are kept in 8 bits, as cases that can be timed: the root-mean-square norm of a residual sum
(forward, backward, and forward into 8 bits with the projection that reads them), the matrix product of rows and weights in 8 bits,
GELU into 8 bits with its input kept in 8 bits, and what the backward pass makes of kept rows: GELU's gradient, and the
gradients of a projection's weights and bias.

A row in 8 bits is C whole numbers from -127 to 127, its codes, and a scale s in 32 bits: with m the largest size in the row
s = m / 127, and a value v has the code that is nearest to v * (127 / m) (ties to the even one).
"""
import math

import torch

own = False

EPS = 1e-5


def _rms(name, op, n, c, dtype, res):
    """op: rms, rms_bwd."""
    return {"name": name, "op": op, "n": n, "c": c, "dtype": dtype, "res": res}


def _product(name, op, n, c, o, dtype, bias, gelu):
    """op: rms_linear, linear, wgrad.  Rows of c values, o outputs a row."""
    return {"name": name, "op": op, "n": n, "c": c, "o": o, "dtype": dtype, "bias": bias, "gelu": gelu}


def _gelu(name, op, n, c, dtype):
    """op: gelu, gelu_bwd."""
    return {"name": name, "op": op, "n": n, "c": c, "dtype": dtype}


def listed():
    return [
        # one row: the smallest call there is, launch and host time
        _rms("rms_one_row", "rms", 1, 192, "bf16", True),
        # the norm before a branch, with the sum that the next branch is added to: four crowded frames
        _rms("rms_batch4", "rms", 800000, 192, "bf16", True),
        # training step of a pillar frame, the gradient of the sum joining that of the norm
        _rms("rms_bwd_pillar", "rms_bwd", 30000, 192, "bf16", True),
        # a width that is no multiple of a vector, no residual
        _rms("rms_bwd_odd", "rms_bwd", 9973, 99, "f32", False),
        # norm and the projection to q, k and v of a pillar frame, served in 8 bits
        _product("rms_linear_pillar", "rms_linear", 30000, 192, 576, "bf16", True, False),
        # one token through a wide layer: the weights are all there is to read
        _product("linear_one_row", "linear", 1, 4096, 4096, "bf16", True, False),
        # a small odd layer with its activation, in 32 bits
        _product("linear_odd", "linear", 1000, 99, 130, "f32", True, True),
        # the largest product: a batch through a wide layer
        _product("linear_large", "linear", 8192, 4096, 4096, "bf16", True, False),
        # the MLP's activation of a pillar frame, input kept for the backward pass
        _gelu("gelu_pillar", "gelu", 30000, 384, "bf16"),
        # its gradient over four crowded frames
        _gelu("gelu_bwd_batch4", "gelu_bwd", 800000, 384, "bf16"),
        # weight gradient of the projection to q, k and v of a pillar frame
        _product("wgrad_pillar", "wgrad", 30000, 192, 576, "bf16", True, False),
        # weight gradient of a wide layer over a long batch
        _product("wgrad_large", "wgrad", 65536, 1024, 2048, "bf16", True, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    return rng.choice([64, 128, 192, 192, 256, 384, 576, 1024, _log(rng, lo, hi), _log(rng, lo, hi) | 1])


def draw(rng):
    op = rng.choice(["rms", "rms_bwd", "rms_linear", "linear", "linear", "gelu", "gelu_bwd", "wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op in ("rms", "rms_bwd"):
        c = _width(rng, 16, 8192)
        most = 800000 * 192 // (c * (2 if dtype == "f32" else 1))
        case = _rms("", op, _log(rng, 1, most), c, dtype, rng.random() < 0.7)
    elif op in ("gelu", "gelu_bwd"):
        c = _width(rng, 16, 8192)
        dtype = "bf16" if op == "gelu" else dtype
        most = (200000 if op == "gelu" else 800000) * 384 // (c * (2 if dtype == "f32" else 1))
        case = _gelu("", op, _log(rng, 1, most), c, dtype)
    else:
        dtype = "bf16" if op == "rms_linear" else dtype
        c, o = _width(rng, 16, 6000), _width(rng, 8, 6000)
        # at most the large products' work (in 32 bits a quarter of it), and half a gigabyte of rows
        most = min((4096 * 8192 * 4096 if op != "wgrad" else 65536 * 1024 * 2048) // (c * o * (4 if dtype == "f32" else 1)), (1 << 29) // (4 * (c + o)), 200000)
        case = _product("", op, _log(rng, 1, max(most, 2)), c, o, dtype, rng.random() < 0.8, op == "linear" and rng.random() < 0.3)
    del case["name"]
    return case


def _codes(v):
    """Codes and scales of rows of 32 bits, in operations of 32 bits; 64 bits stay 64."""
    top = v.abs().amax(1, keepdim=True)
    return (v * (torch.full_like(top, 127) / top)).round(), (top / 127).squeeze(1)


def _padded(codes):
    """int8 rows that begin on 16 bytes."""
    n, c = codes.shape
    t = torch.zeros((n, (c + 15) // 16 * 16), dtype=torch.int8, device="cuda")[:, :c]
    return t.copy_(codes)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    op, n, c = case["op"], case["n"], case["c"]
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
    # rows as a layer has them: channels of several sizes
    rows = lambda: normal(n, c) * (0.4 * normal(c)).exp()  # noqa: E731
    s = {"op": op, "type": t}
    if op in ("rms", "rms_bwd", "rms_linear"):
        s |= {"x": rows().to(t), "r": (0.5 * normal(n, c) + 0.1).to(t) if case.get("res", True) else None, "gamma": 1 + 0.1 * normal(c)}
        if op == "rms_bwd":
            s |= {"dy": (1e-2 * normal(n, c)).to(t), "d_sum": (1e-2 * normal(n, c)).to(t) if case["res"] else None}
    if op in ("linear", "wgrad"):
        codes, s["scale"] = _codes(rows().to(t).float())
        s["codes"] = _padded(codes)
    if op in ("linear", "rms_linear"):
        w, s["w_scale"] = _codes(normal(case["o"], c) / math.sqrt(c))
        s |= {"w_codes": _padded(w), "bias": 0.1 * normal(case["o"]) if case["bias"] else None, "gelu": case["gelu"]}
    if op == "wgrad":
        s |= {"dy": (1e-2 * normal(n, case["o"])).to(t), "bias": case["bias"]}
    if op in ("gelu", "gelu_bwd"):
        h = (1.5 * rows()).to(t)
        if op == "gelu":
            s["h"] = h
        else:
            codes, s["scale"] = _codes(h.float())
            s |= {"codes": _padded(codes), "dy": (1e-2 * normal(n, c)).to(t)}
    if own:
        import paper_2301_06051_amd as dsvt
        if "gamma" in s:
            s["rms"] = dsvt.RmsNorm(s["gamma"], case["dtype"], EPS)
        if "codes" in s:
            s["rows"] = dsvt.Rows8.of(s["codes"], s["scale"])
        if "w_codes" in s:
            s["linear"] = dsvt.Linear8(dsvt.Rows8.of(s["w_codes"], s["w_scale"]), case["dtype"], s["bias"], s["gelu"])
    return s


def _own(s):
    import paper_2301_06051_amd as dsvt
    op = s["op"]
    if op == "rms":
        y, z = dsvt.dsvt_rms_norm(s["rms"], s["x"], s["r"], want_sum=True)
        return {"y": y, "z": z}
    if op == "rms_bwd":
        dx, dg = dsvt.dsvt_rms_norm_backward(s["rms"], s["dy"], s["x"], s["r"], s["d_sum"])
        return {"dx": dx, "d_gamma": dg}
    if op == "rms_linear":
        rows, z = dsvt.dsvt_rms_norm_rows8(s["rms"], s["x"], s["r"], want_sum=True)
        return {"y": dsvt.dsvt_linear_rows8(s["linear"], rows), "z": z}
    if op == "linear":
        return {"y": dsvt.dsvt_linear_rows8(s["linear"], s["rows"])}
    if op == "gelu":
        out, kept = dsvt.dsvt_gelu_rows8(s["h"])
        return {"out": dsvt.dsvt_read_rows8(out, "bf16"), "kept": dsvt.dsvt_read_rows8(kept, "bf16")}
    if op == "gelu_bwd":
        return {"dh": dsvt.dsvt_gelu_rows8_backward(s["rows"], s["dy"])}
    dw, db = dsvt.dsvt_linear_rows8_weight_grad(s["rows"], s["dy"], want_bias=s["bias"])
    return {"d_w": dw, "d_b": db} if s["bias"] else {"d_w": dw}


def _sum(s):
    return s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()


def _phi(h):
    """Distribution of the normal law, without losing the digits of its lower end."""
    return 0.5 * torch.erfc(h * -math.sqrt(0.5))


def _linear(s, codes, scale):
    """Rows in 8 bits times weights in 8 bits."""
    y = (codes @ s["w_codes"].float().t()) * scale[:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return (y * _phi(y) if s["gelu"] else y).to(s["type"])


def run(s):
    if own:
        return _own(s)
    op, t = s["op"], s["type"]
    if op in ("rms", "rms_bwd", "rms_linear"):
        z = _sum(s)
        r = torch.rsqrt((z * z).mean(1, keepdim=True) + EPS)
        n = z * r
        if op == "rms":
            return {"y": (n * s["gamma"]).to(t), "z": z.to(t)}
        if op == "rms_linear":
            return {"y": _linear(s, *_codes(n * s["gamma"])), "z": z.to(t)}
        dy = s["dy"].float()
        w = dy * s["gamma"]
        dx = r * (w - n * (w * n).mean(1, keepdim=True))
        dx = dx if s["d_sum"] is None else dx + s["d_sum"].float()
        # sums over all rows are long: in 64 bits
        return {"dx": dx.to(t), "d_gamma": (dy * n).sum(0, dtype=torch.float64).float()}
    if op == "linear":
        return {"y": _linear(s, s["codes"].float(), s["scale"])}
    if op == "gelu":
        h = s["h"].float()
        (out, a), (kept, b) = _codes(h * _phi(h)), _codes(h)
        return {"out": (out * a[:, None]).to(t), "kept": (kept * b[:, None]).to(t)}
    x = s["codes"].float() * s["scale"][:, None]
    dy = s["dy"].float()
    if op == "gelu_bwd":
        return {"dh": (dy * (_phi(x) + x * (x * x * -0.5).exp() * (1 / math.sqrt(2 * math.pi)))).to(t)}
    d_w = (dy.t() @ x).to(t)
    return {"d_w": d_w, "d_b": dy.sum(0, dtype=torch.float64).float()} if s["bias"] else {"d_w": d_w}


def work(case):
    e, op, n, c = (2 if case["dtype"] == "bf16" else 4), case["op"], case["n"], case["c"]
    if op == "rms":
        return {"bytes": (3 + int(case["res"])) * n * c * e + 4 * c, "flops": 6 * n * c}
    if op == "rms_bwd":
        return {"bytes": (3 + 2 * int(case["res"])) * n * c * e + 8 * c, "flops": 13 * n * c}
    if op == "gelu":
        return {"bytes": 3 * n * c * e, "flops": 40 * n * c}
    if op == "gelu_bwd":
        return {"bytes": n * c * (2 * e + 1) + 4 * n, "flops": 40 * n * c}
    o = case["o"]
    flops = 2 * n * c * o
    if op == "wgrad":
        return {"bytes": n * o * e + n * (c + 4) + o * c * e + 4 * o, "flops": flops}
    rows = 3 * n * c * e + 4 * c if op == "rms_linear" else n * (c + 4)
    return {"bytes": rows + o * (c + 8) + n * o * e, "flops": flops}


def exact(case, seed):
    """The same outputs in 64 bits, from the definitions; gradients by automatic differentiation."""
    s = prepare(case, seed)
    op = case["op"]
    d = lambda a: None if a is None else a.detach().double()  # noqa: E731

    def activation(v):
        return v * 0.5 * (1 + torch.erf(v / math.sqrt(2)))

    def in_8_bits(v):
        unit = v.abs().amax(1, keepdim=True) / 127
        return (v / unit).round() * unit

    def project(rows):
        y = torch.nn.functional.pad(rows, (0, 1), value=1.0) @ torch.cat([d(s["w_codes"]) * d(s["w_scale"])[:, None],
                                                                           (torch.zeros_like(s["w_scale"]) if s["bias"] is None else s["bias"]).double()[:, None]], 1).t().contiguous()
        return activation(y) if s["gelu"] else y

    if op in ("rms", "rms_bwd", "rms_linear"):
        z = d(s["x"]) if s["r"] is None else d(s["x"]) + d(s["r"])
        gamma = d(s["gamma"])
        if op == "rms_bwd":
            z.requires_grad_()
            gamma.requires_grad_()
        y = z / (z.square().sum(1, keepdim=True) / z.shape[1] + EPS).sqrt() * gamma
        if op == "rms":
            return {"y": y, "z": z}
        if op == "rms_linear":
            return {"y": project(in_8_bits(y)), "z": z}
        dz, dg = torch.autograd.grad(y, (z, gamma), d(s["dy"]))
        return {"dx": dz if s["d_sum"] is None else dz + d(s["d_sum"]), "d_gamma": dg}
    if op == "gelu":
        h = d(s["h"])
        return {"out": in_8_bits(activation(h)), "kept": in_8_bits(h)}
    x = d(s["codes"]) * d(s["scale"])[:, None]
    if op == "linear":
        return {"y": project(x)}
    if op == "gelu_bwd":
        x.requires_grad_()
        return {"dh": torch.autograd.grad(activation(x), x, d(s["dy"]))[0]}
    weights, bias = torch.zeros((case["o"], case["c"]), dtype=torch.float64, device="cuda", requires_grad=True), None
    y = x @ weights.t()
    if s["bias"]:
        bias = torch.zeros(case["o"], dtype=torch.float64, device="cuda", requires_grad=True)
        y = y + bias
    grads = torch.autograd.grad(y, [weights] + ([bias] if s["bias"] else []), d(s["dy"]))
    return dict(zip(("d_w", "d_b"), grads))
