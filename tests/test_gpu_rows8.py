"""The operators on rows in 8 bits against plain 64-bit references, element by element."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
dsvt = pytest.importorskip("paper_2301_06051_amd")
import rows8_ref as ref  # noqa: E402

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rows(g, n, c, dtype, spread=0.4):
    """Rows with channels of several sizes."""
    return (torch.randn((n, c), generator=g) * (spread * torch.randn((c,), generator=g)).exp()).to(DT[dtype])


def _placed(t, form):
    """The same rows on the GPU as columns of a wider array: "tight" none, "wide" rows on 16 bytes, "odd" rows that begin anywhere."""
    if form == "tight":
        return t.cuda()
    extra, at = {"wide": (32, 16), "odd": (3, 1)}[form]
    wide = torch.full((t.shape[0], t.shape[1] + extra), 7.0, dtype=t.dtype, device="cuda")
    wide[:, at:at + t.shape[1]].copy_(t)
    return wide[:, at:at + t.shape[1]]


def _codes(codes, scale, fill=127):
    """Rows8 of given codes; what lies past a row's end is `fill`."""
    n, c = codes.shape
    wide = torch.full((n, (c + 15) // 16 * 16), fill, dtype=torch.int8, device="cuda")
    wide[:, :c].copy_(codes)
    return dsvt.Rows8.of(wide[:, :c], scale.cuda())


def _random_codes(g, n, c, fill=127):
    codes = torch.randint(-127, 128, (n, c), generator=g).to(torch.int8)
    return _codes(codes, 0.01 * torch.rand((n,), generator=g) + 1e-3, fill)


SHAPES = [(1, 1), (1, 192), (3, 7), (17, 16), (300, 64), (257, 99), (130, 192), (65, 300), (33, 700), (20, 1025), (9, 2056), (5, 4100), (5, 8192), (3, 8200), (2, 9001),
          (700, 24), (2500, 192), (2, 65536)]


@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", ["tight", "wide", "odd"])
def test_keep_and_read(n, c, dtype, form):
    x = _rows(_gen(n + c), n, c, dtype)
    print("[case] keep", n, c, dtype, form, flush=True)
    kept = dsvt.dsvt_keep_rows8(_placed(x, form))
    back = dsvt.dsvt_read_rows8(kept, dtype)
    codes, scale = ref.quantise(x)
    assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.scale.cpu(), scale)
    assert torch.equal(back.cpu(), (codes.float() * scale[:, None]).to(DT[dtype]))
    placed = _placed(torch.zeros_like(x), form)
    assert dsvt.dsvt_read_rows8(kept, dtype, x=placed) is placed and torch.equal(placed, back)
    if form != "tight":
        wide = placed._base
        assert bool((wide[:, c + (16 if form == "wide" else 1):] == 7).all()) and bool((wide[:, :(16 if form == "wide" else 1)] == 7).all())


@pytest.mark.parametrize("c", [5, 192, 700, 9000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_special_values(c, dtype):
    """Zeros, values next to zero, next to the largest number, ties, infinities and NaN: each row by itself."""
    top = torch.finfo(DT[dtype]).max
    x = torch.randn((12, c), generator=_gen(c)).to(DT[dtype])
    x[0] = 0
    x[1] = 1e-38
    x[2] = (torch.arange(c) % 2 * 2 - 1) * top
    x[3, c // 2] = math.inf
    x[4, c - 1] = -math.inf
    x[5, 0] = math.nan
    x[6] = 2.0 ** -118
    x[7] = 2.0 ** -118 * (1 - 2.0 ** -8)
    x[8] = 127
    x[8, 1:] = (torch.arange(c - 1) % 253 - 126.5).to(DT[dtype])            # halves between codes, as far as the type has them
    x[9] = -0.0
    x[10] = -x[10].abs()
    x[11] = math.nan
    print("[case] special rows", c, dtype, flush=True)
    kept = dsvt.dsvt_keep_rows8(x.cuda())
    codes, scale = ref.quantise(x)
    assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.scale.cpu().nan_to_num(-1), scale.nan_to_num(-1))
    assert scale[[3, 4, 5, 11]].isnan().all() and not scale[[0, 1, 7, 9]].any() and bool((scale[[2, 6]] > 0).all())
    back = dsvt.dsvt_read_rows8(kept, dtype).cpu()
    assert back[[3, 4, 5, 11]].isnan().all() and not back[[0, 1, 7, 9]].any()
    good = [0, 1, 2, 6, 7, 8, 9, 10]
    w = _random_codes(_gen(1), 20, c)
    y = dsvt.dsvt_linear_rows8(dsvt.Linear8(w, dtype), kept).cpu()
    assert y[[3, 4, 5, 11]].isnan().all() and not y[good].isnan().any()
    out, again = dsvt.dsvt_gelu_rows8(x.cuda())
    assert torch.equal(again.codes, kept.codes) and out.scale.cpu()[[3, 4, 5, 11]].isnan().all() and out.scale.cpu()[good].isfinite().all()
    dh = dsvt.dsvt_gelu_rows8_backward(kept, torch.ones((12, c), dtype=DT[dtype], device="cuda")).cpu()
    assert dh[[3, 4, 5, 11]].isnan().all() and dh[good].isfinite().all() and bool(((dh[[0, 9]].double() - 0.5).abs() <= ref.PHI).all()) and bool((dh[8, 0] == 1).all())
    dw, db = dsvt.dsvt_linear_rows8_weight_grad(kept, torch.ones((12, 3), dtype=DT[dtype], device="cuda"))
    assert dw.isnan().all() and bool((db == 12).all())


@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form,res", [("tight", True), ("tight", False), ("wide", True), ("odd", True)])
def test_rms_norm(n, c, dtype, form, res):
    """Both directions, all outputs; codes and rows of one call each."""
    g = _gen(n * 3 + c)
    x, r, dy, ds = _rows(g, n, c, dtype), torch.randn((n, c), generator=g).to(DT[dtype]), torch.randn((n, c), generator=g).to(DT[dtype]), torch.randn((n, c), generator=g).to(DT[dtype])
    gamma = 1 + 0.3 * torch.randn((c,), generator=g)
    r, ds = (r, ds) if res else (None, None)
    case = f"rms {n} {c} {dtype} {form} {res}"
    print("[case]", case, flush=True)
    norm = dsvt.RmsNorm(gamma.cuda(), dtype, EPS)
    xd, rd, dyd, dsd = (None if t is None else _placed(t, form) for t in (x, r, dy, ds))
    want = ref.rms(x, r, gamma, EPS, dy, ds)
    y, z = dsvt.dsvt_rms_norm(norm, xd, rd, want_sum=True)
    ref.check("y", y, *want["y_rows"], case)
    ref.check("z", z, *want["z"], case)
    assert torch.equal(dsvt.dsvt_rms_norm(norm, xd, rd), y)
    out, z2 = dsvt.dsvt_rms_norm_rows8(norm, xd, rd, want_sum=True)
    ref.check_codes(out, *want["y"], case)
    assert torch.equal(z2, z) and torch.equal(dsvt.dsvt_rms_norm_rows8(norm, xd, rd).codes, out.codes)
    dx, dg = dsvt.dsvt_rms_norm_backward(norm, dyd, xd, rd, dsd)
    ref.check("dx", dx, *want["dx"], case)
    ref.check("d_gamma", dg, *want["d_gamma"], case)
    # in place: the sum and the norm over the branch and the input, the gradient over that of the sum
    a, b = xd.clone(), dyd.clone()
    y3, z3 = dsvt.dsvt_rms_norm(norm, a, rd, y=None if rd is None else rd, z=a)
    assert z3 is a and torch.equal(z3, z) and torch.equal(y3, y)
    rd = None if r is None else _placed(r, form)
    assert torch.equal(dsvt.dsvt_rms_norm_backward(norm, b, xd, rd, dsd, dx=b)[0], dx)
    if dsd is not None:
        assert torch.equal(dsvt.dsvt_rms_norm_backward(norm, dyd, xd, rd, dsd, dx=dsd)[0], dx)


@pytest.mark.parametrize("c", [5, 192, 700, 9000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rms_norm_of_special_values(c, dtype):
    """Rows of zeros, with an infinity, a NaN, and of numbers whose squares are not: each by itself, in rows and in 8 bits."""
    x = torch.randn((6, c), generator=_gen(c)).to(DT[dtype])
    x[0] = 0
    x[1, c // 2] = math.inf
    x[2, 0] = math.nan
    x[3] = 1e30
    x[4, c - 1] = -math.inf
    print("[case] special norms", c, dtype, flush=True)
    norm = dsvt.RmsNorm(torch.ones(c, device="cuda"), dtype, EPS)
    y, z = dsvt.dsvt_rms_norm(norm, x.cuda(), want_sum=True)
    rows = dsvt.dsvt_rms_norm_rows8(norm, x.cuda())
    assert torch.equal(z.cpu().nan_to_num(7), x.nan_to_num(7)) and not y[[0, 3]].any() and y[5].isfinite().all()
    assert y[2].isnan().all() and y[1, c // 2].isnan() and y[4, c - 1].isnan()               # (infinity by infinity)
    assert rows.scale[[1, 2, 4]].isnan().all() and not rows.codes[:5].any() and not rows.scale[[0, 3]].any() and bool(rows.scale[5] > 0)
    dx, dg = dsvt.dsvt_rms_norm_backward(norm, torch.ones_like(x).cuda(), x.cuda())
    assert dx[2].isnan().all() and dx[5].isfinite().all() and dg.isnan().any()


def test_rms_norm_by_differences():
    """The gradient against quotients of differences of the forward call, in fp32."""
    g, n, c = _gen(5), 6, 48
    x, dy, gamma = torch.randn((n, c), generator=g).cuda(), torch.randn((n, c), generator=g).cuda(), (1 + 0.3 * torch.randn((c,), generator=g)).cuda()
    dx, dg = dsvt.dsvt_rms_norm_backward(dsvt.RmsNorm(gamma, "f32", EPS), dy, x)
    for seed in range(4):
        v, u = torch.randn((n, c), generator=_gen(10 + seed)).cuda(), torch.randn((c,), generator=_gen(20 + seed)).cuda()
        t = 2.0 ** -7
        f = lambda s: float((dsvt.dsvt_rms_norm(dsvt.RmsNorm(gamma + s * u, "f32", EPS), x + s * v).double() * dy.double()).sum())  # noqa: E731
        quotient, slope = (f(t) - f(-t)) / (2 * t), float((dx.double() * v).sum() + (dg.double() * u).sum())
        # the third derivative along (v, u) is at most some tens per value, |dy| about 1: t^2 / 6 of it over n c values that add up with random
        # signs, sqrt(n c) 50 t^2 / 6; and roundings of 2^-23 a value over 2 t
        assert abs(quotient - slope) < math.sqrt(n * c) * (50 * t * t / 6 + 2.0 ** -23 / t), (quotient, slope)


@pytest.mark.parametrize("n,c", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", ["tight", "odd"])
def test_gelu(n, c, dtype, form):
    g = _gen(n * 5 + c)
    h, dy = 1.5 * _rows(g, n, c, dtype), torch.randn((n, c), generator=g).to(DT[dtype])
    if n > 2:
        h[1] = torch.linspace(-9, 9, c).to(DT[dtype])
    case = f"gelu {n} {c} {dtype} {form}"
    print("[case]", case, flush=True)
    hd, dyd = _placed(h, form), _placed(dy, form)
    out, kept = dsvt.dsvt_gelu_rows8(hd)
    codes, scale = ref.quantise(h)
    assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.scale.cpu(), scale)
    ref.check_codes(out, ref.gelu(h.double()), ref.gelu_error(h.double()), case)
    only, none = dsvt.dsvt_gelu_rows8(hd, want_kept=False)
    assert none is None and torch.equal(only.codes, out.codes) and torch.equal(only.scale, out.scale)
    k = codes.double() * scale.double()[:, None]
    want = dy.double() * ref.gelu_slope(k)
    hs, u = ref.half_step(DT[dtype]), ref.U
    # Phi, the density's part (six roundings of at most 0.3), and the kept value's own rounding where the slope changes by at most 0.8 of it
    err = dy.double().abs() * (ref.PHI + 6 * 0.3 * u + 0.8 * u * k.abs() + 2 * u * 1.13)
    dh = dsvt.dsvt_gelu_rows8_backward(kept, dyd)
    ref.check("dh", dh, want, err * (1 + hs) + hs * want.abs() + 1e-38, case)
    again = dyd.clone()
    assert dsvt.dsvt_gelu_rows8_backward(kept, again, dh=again) is again and torch.equal(again, dh)


LINEAR = [(1, 1, 1), (1, 192, 576), (1, 4096, 300), (2, 15, 3), (5, 16, 17), (15, 17, 16), (16, 63, 64), (17, 64, 130), (33, 65, 192), (64, 99, 130), (100, 192, 384),
          (128, 128, 128), (129, 200, 129), (257, 384, 192), (300, 1000, 257), (1000, 99, 130), (513, 64, 1000), (2000, 192, 576), (700, 576, 520), (260, 1040, 516), (70, 1100, 130), (500, 2064, 100), (64, 300, 200)]


@pytest.mark.parametrize("n,c,o", LINEAR)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form,bias,act", [("tight", True, False), ("odd", False, False), ("wide", True, True)])
def test_linear(n, c, o, dtype, form, bias, act):
    g = _gen(n + 7 * c + o)
    x, w = _random_codes(g, n, c), _random_codes(g, o, c, fill=-127)
    b = torch.randn((o,), generator=g) if bias else None
    case = f"linear {n} {c} {o} {dtype} {form} {bias} {act}"
    print("[case]", case, flush=True)
    layer = dsvt.Linear8(w, dtype, None if b is None else b.cuda(), act)
    want = ref.linear(x.codes, x.scale, w.codes, w.scale, b, DT[dtype], act)
    y = _placed(torch.zeros((n + 2, o), dtype=DT[dtype]), form)
    y[n:] = 3
    dsvt.dsvt_linear_rows8(layer, x, y=y[:n])
    ref.check("y", y[:n], *want, case)
    assert bool((y[n:] == 3).all()) and (form == "tight" or bool((y._base[:, -1] == 7).all()))
    assert torch.equal(dsvt.dsvt_linear_rows8(layer, x), y[:n])


@pytest.mark.parametrize("n", [1, 300])
def test_linear_longest_sum(n):
    """65,536 columns of the largest codes: the sum of 1.06e9 is exact."""
    c = 65536
    x = _codes(torch.full((n, c), 127, dtype=torch.int8), torch.ones((n,)))
    w = _codes(torch.tensor([[127], [-127], [1]], dtype=torch.int8).expand(3, c), torch.ones((3,)))
    print("[case] longest sum", n, flush=True)
    y = dsvt.dsvt_linear_rows8(dsvt.Linear8(w, "f32"), x)
    assert torch.equal(y.cpu(), torch.tensor([[127. * 127 * c, -127. * 127 * c, 127. * c]]).expand(n, 3))


GRADS = [(0, 5, 3), (1, 1, 1), (1, 192, 576), (7, 15, 3), (31, 17, 16), (32, 64, 64), (33, 65, 63), (65, 99, 130), (200, 192, 384), (257, 128, 129), (1000, 64, 192), (3000, 40, 72),
         (513, 300, 520), (5000, 192, 100), (20000, 16, 24)]


@pytest.mark.parametrize("n,c,o", GRADS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", ["tight", "wide", "odd"])
def test_weight_grad(n, c, o, dtype, form):
    g = _gen(n + 3 * c + o)
    x, dy = _random_codes(g, n, c), torch.randn((n, o), generator=g).to(DT[dtype])
    case = f"wgrad {n} {c} {o} {dtype} {form}"
    print("[case]", case, flush=True)
    want = ref.weight_grad(x.codes, x.scale, dy)
    dyd, d_w = _placed(dy, form), _placed(torch.zeros((o, c), dtype=DT[dtype]), form)
    got, d_b = dsvt.dsvt_linear_rows8_weight_grad(x, dyd, d_w=d_w)
    assert got is d_w
    ref.check("d_w", d_w, *want["d_w"], case)
    ref.check("d_b", d_b, *want["d_b"], case)
    assert form == "tight" or bool((d_w._base[:, -1] == 7).all())
    plain, none = dsvt.dsvt_linear_rows8_weight_grad(x, dyd, want_bias=False)
    assert none is None and torch.equal(plain, d_w)


@pytest.mark.parametrize("n,c,o", [(30001, 190, 575), (30000, 192, 576), (40000, 130, 570), (100003, 127, 191)])
@pytest.mark.parametrize("form", ["tight", "odd"])
def test_weight_grad_of_many_rows(n, c, o, form):
    """Many slices of few columns, whose partial sums are joined."""
    g = _gen(n + 3 * c + o)
    x, dy = _random_codes(g, n, c), torch.randn((n, o), generator=g).to(torch.bfloat16)
    case = f"wgrad of many rows {n} {c} {o} {form}"
    print("[case]", case, flush=True)
    want = ref.weight_grad(x.codes, x.scale, dy)
    dyd, d_w = _placed(dy, form), _placed(torch.zeros((o, c), dtype=torch.bfloat16), form)
    _, d_b = dsvt.dsvt_linear_rows8_weight_grad(x, dyd, d_w=d_w)
    ref.check("d_w", d_w, *want["d_w"], case)
    ref.check("d_b", d_b, *want["d_b"], case)
    assert form == "tight" or bool((d_w._base[:, -1] == 7).all())
    plain, _ = dsvt.dsvt_linear_rows8_weight_grad(x, dyd, want_bias=False)
    assert torch.equal(plain, d_w)


def test_rows_past_31_bits():
    """Arrays of more than 2^31 bytes and values: the last rows are those of a call on them alone."""
    n, c = 12_000_000, 192
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((n, c), dtype=torch.bfloat16, device="cuda", generator=g)
    print("[case] long arrays", flush=True)
    last = x[-1000:].contiguous()
    norm = dsvt.RmsNorm(torch.ones(c, device="cuda"), "bf16")
    kept, tail = dsvt.dsvt_keep_rows8(x), dsvt.dsvt_keep_rows8(last)
    assert torch.equal(kept.codes[-1000:], tail.codes) and torch.equal(kept.scale[-1000:], tail.scale)
    assert torch.equal(dsvt.dsvt_read_rows8(kept, "bf16")[-1000:], dsvt.dsvt_read_rows8(tail, "bf16"))
    assert torch.equal(dsvt.dsvt_gelu_rows8_backward(kept, x)[-1000:], dsvt.dsvt_gelu_rows8_backward(tail, last))
    y, z = dsvt.dsvt_rms_norm(norm, x, x, want_sum=True)
    y1, z1 = dsvt.dsvt_rms_norm(norm, last, last, want_sum=True)
    assert torch.equal(y[-1000:], y1) and torch.equal(z[-1000:], z1)
    del y, z
    dx = dsvt.dsvt_rms_norm_backward(norm, x, x, x, x)[0]
    assert torch.equal(dx[-1000:], dsvt.dsvt_rms_norm_backward(norm, last, last, last, last)[0])
    del dx
    layer = dsvt.Linear8(_random_codes(_gen(1), c, c), "bf16")
    assert torch.equal(dsvt.dsvt_linear_rows8(layer, kept)[-1000:], dsvt.dsvt_linear_rows8(layer, tail))
    # only the last rows have a gradient: theirs alone
    dy = torch.zeros((n, c), dtype=torch.bfloat16, device="cuda")
    dy[-1000:] = last
    dw, db = dsvt.dsvt_linear_rows8_weight_grad(kept, dy)
    want = ref.weight_grad(tail.codes, tail.scale, last)
    ref.check("d_w", dw, *want["d_w"], "long arrays")
    ref.check("d_b", db, *want["d_b"], "long arrays")


class _Mlp:
    """x1 = rms(x + branch), y = x1 + W2 gelu(W1 x1): the MLP of a layer, its activations kept in 8 bits only."""

    def __init__(self, g, c, hidden):
        mk = lambda o, i: (torch.randn((o, i), generator=g) / math.sqrt(i)).to(torch.bfloat16).cuda()  # noqa: E731
        self.w1, self.w2 = mk(hidden, c), mk(c, hidden)
        self.b1, self.b2 = (0.1 * torch.randn((k,), generator=g).cuda() for k in (hidden, c))
        self.gamma = (1 + 0.1 * torch.randn((c,), generator=g)).cuda()
        self.norm = dsvt.RmsNorm(self.gamma, "bf16", EPS)
        self.l1, self.l2 = (dsvt.Linear8(dsvt.dsvt_keep_rows8(w), "bf16", b) for w, b in ((self.w1, self.b1), (self.w2, self.b2)))

    def forward(self, x, branch):
        x1, z = dsvt.dsvt_rms_norm_rows8(self.norm, x, branch, want_sum=True)
        h = dsvt.dsvt_linear_rows8(self.l1, x1)
        a, k = dsvt.dsvt_gelu_rows8(h)
        return z + dsvt.dsvt_linear_rows8(self.l2, a), (z, x1, a, k)

    def backward(self, dy, saved):
        z, x1, a, k = saved
        dw2, db2 = dsvt.dsvt_linear_rows8_weight_grad(a, dy)
        dh = dsvt.dsvt_gelu_rows8_backward(k, dy @ self.w2)
        dw1, db1 = dsvt.dsvt_linear_rows8_weight_grad(x1, dh)
        dx, dg = dsvt.dsvt_rms_norm_backward(self.norm, dh @ self.w1, z, None, dy)
        return {"dx": dx, "gamma": dg, "w1": dw1, "b1": db1, "w2": dw2, "b2": db2}


def test_mlp_step():
    """The operators as a layer's MLP uses them, forward and backward, against the 64-bit layer without 8 bits."""
    n, c, hidden = 2000, 192, 384
    g = _gen(8)
    x, branch, dy = (torch.randn((n, c), generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    mlp = _Mlp(g, c, hidden)
    print("[case] mlp step", flush=True)
    y, saved = mlp.forward(x, branch)
    got = mlp.backward(dy, saved)
    leaves = {"dx": x.double() + branch.double(), "gamma": mlp.gamma.double(), "w1": mlp.w1.double(), "b1": mlp.b1.double(), "w2": mlp.w2.double(), "b2": mlp.b2.double()}
    for t in leaves.values():
        t.requires_grad_()
    z = leaves["dx"]
    x1 = z / (z.pow(2).mean(1, keepdim=True) + EPS).sqrt() * leaves["gamma"]
    want = z + ref.gelu(x1 @ leaves["w1"].t() + leaves["b1"]) @ leaves["w2"].t() + leaves["b2"]
    grads = dict(zip(leaves, torch.autograd.grad(want, list(leaves.values()), dy.double())))
    # A value in 8 bits is off by up to m / 254, at random, so sqrt(1/3) of it in the mean square; with the largest of a row below 4.5 times its mean
    # square that is 1.0 % a tensor.  Behind an output are at most x1, w1, a, w2, and behind a gradient x1, w1, k and one of x1, a: four tensors,
    # 2.1 % of the branch, and 4 bf16 roundings of 0.4 % each at most.
    for name, a, b in [("y", y, want), *((k, got[k], grads[k]) for k in got)]:
        off = float((a.double() - b).norm() / b.norm())
        print(f"[err] mlp {name}: {off:.4g}", flush=True)
        assert off < 0.021 + 4 * 2.0 ** -8, name


def test_mlp_step_in_a_graph_and_on_other_streams():
    """Captured once, replayed with eager work between; two eager steps on streams of their own at once; a stream given by its handle."""
    n, c, hidden = 3000, 192, 384
    g = _gen(9)
    x, branch, dy = (torch.randn((n, c), generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    mlp = _Mlp(g, c, hidden)

    def step(**kw):
        rows, z = dsvt.dsvt_rms_norm_rows8(mlp.norm, x, branch, want_sum=True, **kw)
        h = dsvt.dsvt_linear_rows8(mlp.l1, rows, **kw)
        a, k = dsvt.dsvt_gelu_rows8(h, **kw)
        y = dsvt.dsvt_linear_rows8(mlp.l2, a, **kw)
        dw2, db2 = dsvt.dsvt_linear_rows8_weight_grad(a, dy, **kw)
        dh = dsvt.dsvt_gelu_rows8_backward(k, h, **kw)
        dw1, db1 = dsvt.dsvt_linear_rows8_weight_grad(rows, dh, **kw)
        dx, dg = dsvt.dsvt_rms_norm_backward(mlp.norm, dy, z, None, y, **kw)
        n1 = dsvt.dsvt_rms_norm(mlp.norm, dx, y, **kw)
        return [rows.codes, rows.scale, z, h, a.codes, k.codes, y, dw2, db2, dh, dw1, db1, dx, dg, n1, dsvt.dsvt_read_rows8(dsvt.dsvt_keep_rows8(n1, **kw), "bf16", **kw)]

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
    keep = x.clone()
    for rep in range(4):
        for t in got:
            t.fill_(9)
        x.neg_()
        step()                                                   # eager work between the replays, on other values
        x.copy_(keep)
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
    s = streams[0]
    s.wait_stream(torch.cuda.current_stream())
    outs = step(stream=s.cuda_stream)
    junk = [torch.full((1 << 22,), 77, dtype=torch.uint8, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want)) and len(junk) == 8


def test_arguments():
    """Scratch and outputs of the caller; what does not fit is refused."""
    n, c, o = 3000, 192, 130
    g = _gen(2)
    x, dy = _rows(g, n, c, "bf16").cuda(), torch.randn((n, o), generator=g).to(torch.bfloat16).cuda()
    norm = dsvt.RmsNorm(torch.ones(c, device="cuda"), "bf16")
    kept = dsvt.dsvt_keep_rows8(x)
    mine = dsvt.Rows8.empty(n, c)
    assert dsvt.dsvt_keep_rows8(x, out=mine) is mine and torch.equal(mine.codes, kept.codes)
    want, size = dsvt.dsvt_linear_rows8_weight_grad(kept, dy), dsvt.dsvt_linear_rows8_weight_grad_workspace_size(c, o, "bf16", n)
    ws = torch.full((size + 16,), 3, dtype=torch.uint8, device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(dsvt.dsvt_linear_rows8_weight_grad(kept, dy, ws=ws), want)) and bool((ws[size:] == 3).all())
    rms_want, rms_size = dsvt.dsvt_rms_norm_backward(norm, x, x), dsvt.dsvt_rms_norm_backward_workspace_size(norm, n)
    ws = torch.full((rms_size + 16,), 3, dtype=torch.uint8, device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(dsvt.dsvt_rms_norm_backward(norm, x, x, ws=ws), rms_want)) and bool((ws[rms_size:] == 3).all())
    small = torch.zeros((size - 1,), dtype=torch.uint8, device="cuda")
    with pytest.raises(dsvt.DsvtError, match="ENOSPC"):
        dsvt.dsvt_linear_rows8_weight_grad(kept, dy, ws=small)
    with pytest.raises(dsvt.DsvtError, match="ENOSPC"):
        dsvt.dsvt_rms_norm_backward(norm, x, x, ws=small[:rms_size - 1])
    layer = dsvt.Linear8(dsvt.dsvt_keep_rows8(x[:o]), "bf16")
    for call in (lambda: dsvt.dsvt_keep_rows8(x.half()), lambda: dsvt.dsvt_keep_rows8(x.t()), lambda: dsvt.dsvt_keep_rows8(x.cpu()), lambda: dsvt.dsvt_keep_rows8(x[0]),
                 lambda: dsvt.dsvt_keep_rows8(x, out=dsvt.Rows8.empty(n, c - 1)), lambda: dsvt.dsvt_keep_rows8(x, out=dsvt.Rows8.empty(n, c, "cpu")),
                 lambda: dsvt.dsvt_rms_norm(norm, x[:, :64]), lambda: dsvt.dsvt_rms_norm(norm, x.float()), lambda: dsvt.dsvt_rms_norm(norm, x, x[:-1]),
                 lambda: dsvt.dsvt_rms_norm_backward(norm, x, x, None, x[:, :-1]), lambda: dsvt.dsvt_rms_norm_rows8(norm, x, out=dsvt.Rows8.empty(n + 1, c)),
                 lambda: dsvt.dsvt_gelu_rows8(x, kept=dsvt.Rows8.empty(n, 2 * c)), lambda: dsvt.dsvt_gelu_rows8_backward(kept, x[1:]),
                 lambda: dsvt.dsvt_linear_rows8(layer, dsvt.Rows8.empty(n, c + 1)), lambda: dsvt.dsvt_linear_rows8(layer, kept, y=torch.empty((n, o), device="cuda")),
                 lambda: dsvt.dsvt_linear_rows8_weight_grad(kept, dy[1:]), lambda: dsvt.dsvt_linear_rows8_weight_grad(kept, dy, d_w=x[:o].float()),
                 lambda: dsvt.Linear8(kept, "bf16", torch.zeros(n - 1, device="cuda")), lambda: dsvt.Linear8(kept, "bf16", torch.zeros(n))):
        with pytest.raises(ValueError):
            call()


def test_no_rows():
    c, o = 192, 64
    x = torch.empty((0, c), dtype=torch.bfloat16, device="cuda")
    norm = dsvt.RmsNorm(torch.ones(c, device="cuda"), "bf16")
    kept = dsvt.dsvt_keep_rows8(x)
    assert kept.codes.shape == (0, c) and dsvt.dsvt_read_rows8(kept, "f32").shape == (0, c)
    assert dsvt.dsvt_rms_norm(norm, x, x, want_sum=True)[1].shape == (0, c)
    dx, dg = dsvt.dsvt_rms_norm_backward(norm, x, x)
    assert dx.shape == (0, c) and not dg.any() and dg.shape == (c,)
    assert dsvt.dsvt_gelu_rows8(x)[0].scale.shape == (0,) and dsvt.dsvt_gelu_rows8_backward(kept, x).shape == (0, c)
    layer = dsvt.Linear8(dsvt.dsvt_keep_rows8(torch.ones((o, c), device="cuda")), "bf16")
    assert dsvt.dsvt_linear_rows8(layer, kept).shape == (0, o)
    dw, db = dsvt.dsvt_linear_rows8_weight_grad(kept, torch.empty((0, o), dtype=torch.bfloat16, device="cuda"))
    assert dw.shape == (o, c) and not dw.any() and not db.any()


@pytest.mark.parametrize("n,c,o,dtype,act", [(70001, 64, 130, "bf16", False), (66000, 192, 576, "f32", False), (40000, 99, 520, "bf16", True), (30000, 192, 576, "bf16", False),
                                             (33001, 300, 641, "f32", True), (33000, 520, 1040, "bf16", False), (140000, 16, 136, "bf16", False)])
def test_linear_in_parts(n, c, o, dtype, act):
    """Many rows, where workgroups go from tile to tile: every row is that of a call on 1,000 rows, where each has one."""
    g = _gen(n + c)
    x, w = _random_codes(g, n, c), _random_codes(g, o, c)
    layer = dsvt.Linear8(w, dtype, torch.randn((o,), generator=g).cuda(), act)
    print("[case] linear in parts", n, c, o, dtype, flush=True)
    y = dsvt.dsvt_linear_rows8(layer, x)
    for at in range(0, n, 1000):
        part = dsvt.Rows8.of(x.codes[at:at + 1000], x.scale[at:at + 1000])
        assert torch.equal(y[at:at + 1000], dsvt.dsvt_linear_rows8(layer, part)), at
    assert torch.equal(dsvt.dsvt_linear_rows8(layer, x), y)


@pytest.mark.parametrize("n,c,o", [(70001, 64, 64), (33000, 16, 130), (25000, 33, 170), (40000, 192, 300), (33010, 1, 200), (30001, 250, 257), (9000, 100, 1000),
                                   (140000, 99, 7), (300000, 65, 5), (70016, 129, 96)])
@pytest.mark.parametrize("dtype,form,bias,act", [("bf16", "tight", True, False), ("bf16", "odd", False, True), ("bf16", "wide", True, True),
                                                 ("f32", "tight", True, True), ("f32", "odd", True, False)])
def test_linear_of_short_rows(n, c, o, dtype, form, bias, act):
    """Many short rows, which wavefronts go through on their own."""
    g = _gen(n + 7 * c + o)
    x, w = _random_codes(g, n, c), _random_codes(g, o, c, fill=-127)
    b = torch.randn((o,), generator=g) if bias else None
    case = f"short rows {n} {c} {o} {dtype} {form} {bias} {act}"
    print("[case]", case, flush=True)
    layer = dsvt.Linear8(w, dtype, None if b is None else b.cuda(), act)
    want = ref.linear(x.codes, x.scale, w.codes, w.scale, b, DT[dtype], act)
    y = _placed(torch.zeros((n + 2, o), dtype=DT[dtype]), form)
    y[n:] = 3
    dsvt.dsvt_linear_rows8(layer, x, y=y[:n])
    ref.check("y", y[:n], *want, case)
    assert bool((y[n:] == 3).all()) and (form == "tight" or bool((y._base[:, -1] == 7).all()))


@pytest.mark.parametrize("n,c,o,dtype,act", [(60000, 260, 250, "bf16", False), (120000, 272, 251, "bf16", False), (60001, 520, 253, "f32", True), (66001, 300, 200, "bf16", True),
                                             (66000, 257, 130, "f32", False), (26000, 2100, 401, "bf16", False), (7000, 2053, 1000, "bf16", True), (7001, 2048, 999, "f32", False)])
@pytest.mark.parametrize("form", ["tight", "odd"])
def test_linear_of_large_tiles(n, c, o, dtype, act, form):
    """Many rows, of which workgroups take large tiles, several of them each or as many as the chip has room for."""
    g = _gen(n + 7 * c + o)
    x, w, b = _random_codes(g, n, c), _random_codes(g, o, c, fill=-127), torch.randn((o,), generator=g)
    case = f"large tiles {n} {c} {o} {dtype} {act} {form}"
    print("[case]", case, flush=True)
    y = _placed(torch.zeros((n + 2, o), dtype=DT[dtype]), form)
    y[n:] = 3
    dsvt.dsvt_linear_rows8(dsvt.Linear8(w, dtype, b.cuda(), act), x, y=y[:n])
    ref.check("y", y[:n], *ref.linear(x.codes, x.scale, w.codes, w.scale, b, DT[dtype], act), case)
    assert bool((y[n:] == 3).all()) and (form == "tight" or bool((y._base[:, -1] == 7).all()))


@pytest.mark.parametrize("c", [3, 7, 9, 99, 191, 300, 1025, 2057, 4100, 6001, 8189, 9001])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_lies_beside_rows(c, dtype):
    """Rows that begin and end on any value: what lies before and behind them stays as it is, in rows and in codes."""
    n, g, ld = 13, _gen(c), (c + 15) // 16 * 16 + 16
    print("[case] beside rows", c, dtype, flush=True)
    x, r, dy = (_placed(torch.randn((n, c), generator=g).to(DT[dtype]), "odd") for _ in range(3))
    norm = dsvt.RmsNorm((1 + 0.1 * torch.randn((c,), generator=g)).cuda(), dtype)

    def rows():
        return torch.full((n, c + 3), 5.0, dtype=DT[dtype], device="cuda")

    def codes():
        wide = torch.full((n, ld), 77, dtype=torch.int8, device="cuda")
        return wide, dsvt.Rows8.of(wide[:, :c], torch.zeros((n,), device="cuda"))

    (a, b, d, e, f), (p, k8), (q, o8), (w, r8) = (rows() for _ in range(5)), codes(), codes(), codes()
    inner = slice(1, 1 + c)
    dsvt.dsvt_rms_norm(norm, x, r, y=a[:, inner], z=b[:, inner])
    dsvt.dsvt_rms_norm_rows8(norm, x, r, out=r8)
    dsvt.dsvt_rms_norm_backward(norm, dy, x, r, dx=d[:, inner])
    dsvt.dsvt_gelu_rows8(x, out=o8, kept=k8)
    dsvt.dsvt_read_rows8(k8, dtype, x=e[:, inner])
    dsvt.dsvt_gelu_rows8_backward(k8, dy, dh=f[:, inner])
    y, z = dsvt.dsvt_rms_norm(norm, x.contiguous(), r.contiguous(), want_sum=True)
    kept = dsvt.dsvt_keep_rows8(x.contiguous())
    assert torch.equal(k8.codes, kept.codes) and torch.equal(k8.scale, kept.scale)
    assert torch.equal(a[:, inner], y) and torch.equal(b[:, inner], z) and torch.equal(e[:, inner], dsvt.dsvt_read_rows8(kept, dtype))
    assert torch.equal(f[:, inner], dsvt.dsvt_gelu_rows8_backward(kept, dy.contiguous()))
    assert all(bool((t[:, 0] == 5).all()) and bool((t[:, 1 + c:] == 5).all()) for t in (a, b, d, e, f))
    assert all(bool((t[:, c:] == 77).all()) for t in (p, q, w))


@pytest.mark.parametrize("n,c,dtype", [(360000, 192, "bf16"), (90000, 385, "f32"), (90000, 384, "f32")])
def test_large_results(n, c, dtype):
    """Results of more than 128 MB, whose stores are marked: as in parts of 1 / 9."""
    g = torch.Generator(device="cuda").manual_seed(9)
    x, r, dy = (torch.randn((n, c), device="cuda", generator=g).to(DT[dtype]) for _ in range(3))
    norm, part = dsvt.RmsNorm(1 + 0.1 * torch.randn(c, device="cuda", generator=g), dtype), n // 9
    print("[case] large results", n, c, dtype, flush=True)
    kept = dsvt.dsvt_keep_rows8(x)
    (y, z), dx = dsvt.dsvt_rms_norm(norm, x, r, want_sum=True), dsvt.dsvt_rms_norm_backward(norm, dy, x, r)[0]
    back, dh = dsvt.dsvt_read_rows8(kept, dtype), dsvt.dsvt_gelu_rows8_backward(kept, dy)
    for at in range(0, n, part):
        rows = slice(at, at + part)
        some = dsvt.Rows8.of(kept.codes[rows], kept.scale[rows])
        y1, z1 = dsvt.dsvt_rms_norm(norm, x[rows], r[rows], want_sum=True)
        assert torch.equal(y[rows], y1) and torch.equal(z[rows], z1), at
        assert torch.equal(dx[rows], dsvt.dsvt_rms_norm_backward(norm, dy[rows], x[rows], r[rows])[0]), at
        assert torch.equal(back[rows], dsvt.dsvt_read_rows8(some, dtype)) and torch.equal(dh[rows], dsvt.dsvt_gelu_rows8_backward(some, dy[rows])), at


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 100])
def test_linear_of_infinities(n, dtype):
    """Through a bias: an infinity stays one, GELU has its limits, a NaN stays one."""
    g = _gen(4)
    x, w = _random_codes(g, n, 64), _random_codes(g, 5, 64)
    bias = torch.tensor([math.inf, -math.inf, math.nan, 3e38, -3e38]).cuda()
    plain, act = (dsvt.dsvt_linear_rows8(dsvt.Linear8(w, dtype, bias, k), x).float().cpu() for k in (False, True))
    assert bool((plain[:, 0] == math.inf).all()) and bool((plain[:, 1] == -math.inf).all()) and plain[:, 2].isnan().all()
    assert bool((act[:, 0] == math.inf).all()) and not act[:, 1].any() and act[:, 2].isnan().all()
    assert torch.equal(act[:, 3], plain[:, 3]) and not act[:, 4].any()


def test_rows_far_apart():
    """Rows 8 MiB apart, as columns of a very wide array."""
    n, c, o, ld = 70, 200, 130, 1 << 23
    g = _gen(6)
    x, w = _random_codes(g, n, c), _random_codes(g, o, c)
    wide = torch.zeros((n, ld), dtype=torch.int8, device="cuda")
    wide[:, 64:64 + c] = x.codes
    far = dsvt.Rows8.of(wide[:, 64:64 + c], x.scale)
    layer = dsvt.Linear8(w, "bf16")
    print("[case] rows far apart", flush=True)
    assert torch.equal(dsvt.dsvt_linear_rows8(layer, far), dsvt.dsvt_linear_rows8(layer, x))
    assert torch.equal(dsvt.dsvt_linear_rows8(dsvt.Linear8(far, "f32"), x), dsvt.dsvt_linear_rows8(dsvt.Linear8(x, "f32"), x))
    assert torch.equal(dsvt.dsvt_read_rows8(far, "f32"), dsvt.dsvt_read_rows8(x, "f32"))
    dy = torch.randn((n, o), generator=g).to(torch.bfloat16).cuda()
    assert all(torch.equal(a, b) for a, b in zip(dsvt.dsvt_linear_rows8_weight_grad(far, dy), dsvt.dsvt_linear_rows8_weight_grad(x, dy)))
