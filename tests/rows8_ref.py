"""Plain 64-bit references of the operators on rows in 8 bits, and how far a result may be from them.

The bounds count roundings.  U = 2^-24 is half a step of float32, h = eps / 2 of the rows' type (bf16 2^-8, fp32 2^-24).  A sum of n terms is off by
at most n U times the sum of their sizes.  PHI bounds the error of the normal distribution: 7.5e-8 of its formula, and five roundings of
a polynomial of at most 0.75 (5 * 0.75 U = 2.2e-7).
"""
import torch

from train_ref import U, half_step

PHI = 3.0e-7
SMALLEST = 2.0 ** -118


def quantise(x):
    """Codes and scales of rows x by the definition, in float32 operations of the CPU (each rounded once)."""
    x = x.detach().cpu().float()
    top = x.abs().amax(1, keepdim=True)                       # (NaN in it: NaN)
    numbers = x.isfinite().all(1, keepdim=True)
    plain = numbers & (top >= SMALLEST)
    safe = torch.where(plain, top, torch.ones_like(top))
    by = torch.full_like(safe, 127) / safe
    codes = torch.where(plain, (torch.where(plain, x, torch.zeros_like(x)) * by).round(), torch.zeros_like(x))
    by127 = safe / 127
    by127 = torch.where((by127 * 127).isinf(), by127.nextafter(torch.zeros_like(by127)), by127)
    scale = torch.where(plain, by127, torch.where(numbers, torch.zeros_like(top), torch.full_like(top, float("nan"))))
    return codes.to(torch.int8), scale.squeeze(1)


def check_codes(got, want, err, case=""):
    """Rows8 against values `want` (64 bits) that the call knew up to `err`: the scale is that of the largest value, every code the nearest, each
    as far as the errors leave it open."""
    codes, scale = got.codes.cpu().double(), got.scale.cpu().double()
    top, e_top = want.abs().amax(1, keepdim=True), err.amax(1, keepdim=True)
    assert bool(((scale[:, None] - top / 127).abs() <= e_top / 127 + 2 * U * top / 127 + 1e-40).all()), f"{case}: scale"
    assert bool((codes.abs() <= 127).all())
    # half a step, what the value was off, and the roundings of the quotient and the product (127 / m, v * that: 2 U of at most 127 steps) and of the scale
    room = scale[:, None] * (0.5 + 127 * 4 * U) + err + e_top * (codes.abs() / 127)
    off = ((codes * scale[:, None] - want).abs() / room.clamp(min=1e-300)).max() if codes.numel() else torch.zeros(())
    print(f"[err] {case} codes: {float(off):.4f} of the bound", flush=True)
    assert float(off) <= 1.0, case


def check(name, got, want, bound, case=""):
    got, want, bound = got.detach().cpu().double(), want.double(), bound.double()
    assert got.shape == want.shape, (case, name, got.shape, want.shape)
    assert bool(got.isfinite().all()), f"{case} {name}: not finite"
    worst = float(((got - want).abs() / bound.clamp(min=1e-300)).max()) if got.numel() else 0.0
    print(f"[err] {case} {name}: {worst:.3f} of its bound", flush=True)
    assert worst <= 1.0, f"{case} {name}: {worst:.3g} times its bound"


def cdf(x):
    return 0.5 * torch.erfc(x * -(0.5 ** 0.5))


def gelu(x):
    return x * cdf(x)


def gelu_slope(x):
    return cdf(x) + x * torch.exp(-0.5 * x * x) / (2 * torch.pi) ** 0.5


def gelu_error(x, e=0.0):
    """How far a gelu in 32 bits of a value that is off by e may be: the slope is at most 1.13."""
    return x.abs() * PHI + 2 * U * gelu(x).abs() + 1.13 * e


def rms(x, res, gamma, eps, dy=None, d_sum=None):
    """dict of (value, bound): y (as it is before it is rounded to the type, and "y_rows" after it), z; with dy dx and d_gamma."""
    hs, c, rows = half_step(x.dtype), x.shape[1], x.shape[0]
    depth = max(40, c // 256 + 12)                            # additions behind one sum over a row
    z = x.double() + (0 if res is None else res.double())
    g = gamma.double()
    ez = U * z.abs() if res is not None else torch.zeros_like(z)
    mean = z.pow(2).mean(1, keepdim=True)
    rs = 1 / (mean + eps).sqrt()
    rel_rs = (depth + 8) * U + U
    n = z * rs
    e_n = n.abs() * (rel_rs + 2 * U) + rs * ez
    y = n * g
    e_y = e_n * g.abs() + 2 * U * y.abs() + 1e-44
    r = {"y": (y, e_y), "y_rows": (y, e_y + hs * (y.abs() + e_y) + 1e-38), "z": (z, ez + hs * z.abs() * (1 + U) + 1e-38)}
    if dy is None:
        return r
    d = dy.double()
    w = d * g
    mwn = (w * n).mean(1, keepdim=True)
    e_mwn = (depth + 4) * U * (w * n).abs().mean(1, keepdim=True) + (w.abs() * e_n).mean(1, keepdim=True)
    dx = rs * (w - n * mwn)
    e = rs * (4 * U * (w.abs() + (n * mwn).abs()) + e_n * mwn.abs() + n.abs() * e_mwn) + (rel_rs + 2 * U) * dx.abs()
    if d_sum is not None:
        dx = dx + d_sum.double()
        e = e + U * dx.abs()
    long = rows / 512 + 64                                    # additions behind one sum over the rows: a workgroup's, and over the workgroups
    return r | {"dx": (dx, e * (1 + hs) + hs * dx.abs() + 1e-38),
                "d_gamma": ((d * n).sum(0), (d.abs() * e_n).sum(0) + long * U * (d * n).abs().sum(0) + 1e-38)}


def linear(codes, scale, w_codes, w_scale, bias, dtype, act):
    """(value, bound) of the product; the sum of codes is exact, and three roundings of a product follow it, one of the bias's addition."""
    whole = codes.cpu().double() @ w_codes.cpu().double().t()
    p = whole * scale.cpu().double()[:, None] * w_scale.cpu().double()
    y = p if bias is None else p + bias.cpu().double()
    e = 3.5 * U * p.abs() + U * y.abs() + 1e-44
    if act:
        y, e = gelu(y), gelu_error(y, e)
    hs = half_step(dtype)
    return y, e + hs * (y.abs() + e) + 1e-38


def weight_grad(codes, scale, dy):
    """dict of (value, bound).  Rows of bf16: the kept values are rounded to bf16 as operands of the products."""
    hs = half_step(dy.dtype)
    narrow = hs if dy.dtype == torch.bfloat16 else 0.0
    x, d = codes.cpu().double() * scale.cpu().double()[:, None], dy.cpu().double()
    n = x.shape[0]
    dw, size = d.t() @ x, d.abs().t() @ x.abs()
    db, db_size = d.sum(0), d.abs().sum(0)
    return {"d_w": (dw, (narrow + (n + 8) * U) * size * (1 + hs) + hs * dw.abs() + 1e-38), "d_b": (db, (n + 8) * U * db_size + 1e-38)}
