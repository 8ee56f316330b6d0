"""The weight gradient from rows in 8 bits where sums are of whole numbers that 32 bits hold, so that a lost row, step or slice, one that counts
twice, or a rounding of an operand shows: the results are the exact sums, rounded once to their type."""
import pytest
import torch

pytestmark = pytest.mark.gpu
dsvt = pytest.importorskip("paper_2301_06051_amd")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# outputs and columns of the tiles that a call takes; calls of few slices and of one, sizes that are whole tiles and that are not
SQUARE_64, SQUARE_128, SQUARE_192, SQUARE_256, LONG = (64, 64), (128, 128), (192, 192), (256, 256), (192, 64)
CASES = [("bf16", 1000, 16, 5, SQUARE_64), ("bf16", 2011, 383, 390, SQUARE_64), ("bf16", 130, 70, 9, SQUARE_64), ("bf16", 900, 1, 1, SQUARE_64), ("bf16", 8000, 192, 192, SQUARE_64),
         ("bf16", 333, 3001, 2003, SQUARE_128), ("bf16", 20011, 603, 701, SQUARE_128), ("bf16", 20000, 640, 768, SQUARE_128),
         ("bf16", 700001, 190, 191, SQUARE_192), ("bf16", 800000, 192, 192, SQUARE_192), ("bf16", 600003, 131, 573, SQUARE_192),
         ("bf16", 301, 4001, 4003, SQUARE_256), ("bf16", 16000, 1021, 1000, SQUARE_256), ("bf16", 16384, 1024, 1024, SQUARE_256), ("bf16", 9001, 2050, 1999, SQUARE_256),
         ("bf16", 30001, 190, 575, LONG), ("bf16", 30000, 192, 576, LONG), ("bf16", 100003, 127, 191, LONG), ("bf16", 40000, 130, 570, LONG),
         ("f32", 1000, 16, 3, SQUARE_64), ("f32", 20003, 63, 130, SQUARE_64), ("f32", 300, 385, 390, SQUARE_64), ("f32", 30000, 192, 576, SQUARE_64),
         ("f32", 8001, 1001, 1003, SQUARE_128), ("f32", 20000, 1024, 1024, SQUARE_128), ("f32", 70, 4099, 4001, SQUARE_128)]


def _inputs(n, c, o, dtype, seed, large=False):
    """Codes of all sizes, scales that are whole numbers up to 31, so that values have up to 12 bits, dy of -1, 0 and 1: sums stay below 2^24.
    large: values are 0 or at least 256."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    whole = lambda lo, hi, *shape: torch.randint(lo, hi, shape, device="cuda", generator=g)  # noqa: E731
    wide = torch.full((n, (c + 15) // 16 * 16), 127, dtype=torch.int8, device="cuda")
    wide[:, :c] = (whole(16, 128, n, c) * whole(-1, 2, n, c) if large else whole(-127, 128, n, c)).to(torch.int8)
    rows = dsvt.Rows8.of(wide[:, :c], whole(16 if large else 1, 32, n).float())
    return rows, whole(-1, 2, n, o).to(DT[dtype])


def _sums(rows, dy):
    x, d = rows.codes.double() * rows.scale.double()[:, None], dy.double()
    return d.t().contiguous() @ x, d.sum(0)


def _odd(t):
    """The same values as columns of a wider array, rows begin anywhere; everything beside them is 7."""
    wide = torch.full((t.shape[0], t.shape[1] + 5), 7, dtype=t.dtype, device="cuda")
    wide[:, 3:-2] = t
    return wide[:, 3:-2]


def _tiles(c, o, dtype, n, tile):
    """Whether scratch of the call is of slices of such tiles (of one slice there is none)."""
    size = dsvt.dsvt_linear_rows8_weight_grad_workspace_size(c, o, dtype, n)
    squares = -(-o // tile[0]) * -(-c // tile[1])
    return size % (4 * (squares * tile[0] * tile[1] + o)) == 0


@pytest.mark.parametrize("dtype,n,c,o,tile", CASES)
@pytest.mark.parametrize("large", [False, True])
def test_weight_grad_is_exact(dtype, n, c, o, tile, large):
    """Two bf16 operands that make a value of 256 or more are whole numbers (their steps are 1 at least): nothing is rounded but the result.  Those of smaller
    ones may have fractions, down to 2^-8 of 1, which the sums round away: n / 8 matrix instructions add to one (16 rows each, for either operand), each
    with an error below 2^-24 of a sum, which is below twice the largest result; together, of signs without an order, below 8 sqrt(n / 8) times that.  A
    result with the error e is rounded to what is nearest, and so off by at most 2 |e| more than without."""
    print("[case] exact weight grad", dtype, n, c, o, tile, large, flush=True)
    rows, dy = _inputs(n, c, o, dtype, n + c + o, large)
    assert _tiles(c, o, dtype, n, tile)
    d_w, d_b = _sums(rows, dy)
    top = float(d_w.abs().max())
    assert top < 2 ** 23                                      # (and so are partial sums below 2^24)
    want = d_w.float().to(DT[dtype])
    rounded, e = (want.double() - d_w).abs(), 8 * (n / 8) ** 0.5 * 2.0 ** -24 * 2 * top

    def good(got):
        return torch.equal(got, want) if large or dtype == "f32" else bool(((got.double() - d_w).abs() <= rounded + 2 * e).all())

    got, bias = dsvt.dsvt_linear_rows8_weight_grad(rows, dy)
    assert good(got) and torch.equal(bias, d_b.float())
    placed = _odd(torch.zeros_like(want))
    again, bias = dsvt.dsvt_linear_rows8_weight_grad(rows, _odd(dy), d_w=placed)
    assert good(again) and torch.equal(bias, d_b.float())
    assert bool((placed._base[:, :3] == 7).all()) and bool((placed._base[:, -2:] == 7).all())
    assert torch.equal(dsvt.dsvt_linear_rows8_weight_grad(rows, dy, want_bias=False)[0], got)


@pytest.mark.parametrize("dtype,n,c,o,tile", [case for case in CASES if case[1] <= 100003])
def test_weight_grad_of_any_scale(dtype, n, c, o, tile):
    """Scales of 24 bits.  A result v + e is rounded to what is nearest to it, so it is off by at most twice |e| more than v rounded.  e has the errors of n
    terms and of 2 n additions, whose signs have no order.  A term of bf16 operands is off by 2^-15 of it: a value is taken as its first 8 bits and the rest,
    below 2^-7 of it, which is rounded by at most 2^-8 of that; of 32 bits 2^-23.  An addition is off by 2^-24 of a sum, and that is the root of the sum of the
    terms' squares, `size`, in the mean.  So e is size (2^-15 + sqrt(2 n) 2^-24) or less in the mean square, and one of millions below 8 times that; all
    together, in the norm, below 2 times it.  (One 8-bit operand would be off by 2^-8 a term.)"""
    print("[case] weight grad of any scale", dtype, n, c, o, flush=True)
    g = torch.Generator(device="cuda").manual_seed(n + o)
    rows, dy = _inputs(n, c, o, dtype, n + c + o)
    rows.scale.copy_(torch.rand((n,), device="cuda", generator=g) + 0.5)
    dy.copy_(torch.randn((n, o), device="cuda", generator=g))
    d_w, d_b = _sums(rows, dy)
    x, d = rows.codes.double() * rows.scale.double()[:, None], dy.double()
    size, size_b = (d.square().t().contiguous() @ x.square()).sqrt(), d.square().sum(0).sqrt()
    got, bias = dsvt.dsvt_linear_rows8_weight_grad(rows, dy)
    u = 2.0 ** -24
    e = size * ((2.0 ** -15 if dtype == "bf16" else 2.0 ** -23) + (2 * n) ** 0.5 * u)
    rounded = (d_w.float().to(DT[dtype]).double() - d_w).abs() + u * d_w.abs()           # (by way of 32 bits)
    err = (got.double() - d_w).abs()
    worst, off, may = float((err / (rounded + 2 * 8 * e).clamp(min=1e-30)).max()), float(err.norm()), float(rounded.norm() + 2 * 2 * e.norm())
    print(f"[err] {worst:.3f} of the bound, norm {off / float(d_w.norm()):.3e}, may be {may / float(d_w.norm()):.3e}", flush=True)
    assert worst <= 1.0 and (off <= may or got.numel() < 64)
    assert bool(((bias.double() - d_b).abs() <= u * d_b.abs() + 8 * n ** 0.5 * u * size_b).all())


def test_weight_grad_of_the_smallest_and_largest_rows():
    """Rows next to the smallest a row may be and to the largest number, an output a row: as far as bf16 and the smallest steps of it, 2^-133, go."""
    print("[case] weight grad of extreme rows", flush=True)
    n, c = 64, 40
    codes = torch.zeros((n, 48), dtype=torch.int8, device="cuda")
    codes[:, :c] = torch.randint(-127, 128, (n, c), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.int8)
    codes[:, 0] = 127
    for scale, by in ((2.0 ** -125 * 1.99, 2.0 ** 60), (2.0 ** -110 * 1.37, 2.0 ** 60), (float.fromhex("0x1.020406p+121"), 2.0 ** -60)):
        rows = dsvt.Rows8.of(codes[:, :c], torch.full((n,), scale, device="cuda"))
        got, bias = dsvt.dsvt_linear_rows8_weight_grad(rows, (by * torch.eye(n, device="cuda")).to(torch.bfloat16))
        want = codes[:, :c].double() * rows.scale[:, None].double() * by
        assert bool(((got.double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -15) + 2.0 ** -134 * by).all()) and bool((bias == by).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,c,o", [(40, 192, 64), (9000, 70, 200), (16384, 1024, 1024)])
def test_weight_grad_of_infinities(dtype, n, c, o):
    """An infinity in dy makes infinities of its output's sums, by the sign of the kept value, where that is not zero; a NaN makes NaN of them all;
    other outputs are what they are without.  Scales are powers of two, of whose values one term of 8 bits would be enough."""
    print("[case] weight grad of infinities", dtype, n, c, o, flush=True)
    rows, dy = _inputs(n, c, o, dtype, n)
    rows.scale.copy_(2.0 ** torch.randint(-20, 20, (n,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)))
    rows.codes[n - 3, :3] = torch.tensor([0, 1, -127], dtype=torch.int8, device="cuda")
    plain, bias = dsvt.dsvt_linear_rows8_weight_grad(rows, dy)
    dy[n - 3, 1], dy[5, 3] = float("-inf"), float("nan")
    got, got_bias = dsvt.dsvt_linear_rows8_weight_grad(rows, dy)
    want = plain.clone()
    want[1] = (rows.codes[n - 3].to(want.dtype) * float("-inf"))
    want[3] = float("nan")
    same = lambda a, b: torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7, 1e30, -1e30), b.nan_to_num(7, 1e30, -1e30))  # noqa: E731
    bias[1], bias[3] = float("-inf"), float("nan")
    assert bool(got[1, 0].isnan()) and same(got, want) and same(got_bias, bias)


@pytest.mark.parametrize("dtype,n,c,o", [("f32", 300007, 63, 130), ("f32", 200001, 1001, 900), ("bf16", 400007, 63, 130), ("bf16", 150001, 2049, 4097)])
def test_weight_grad_joins_slices_in_64_bits(dtype, n, c, o):
    """Positive whole numbers: a slice's sums (of at most 16,384 rows of fp32, 65,536 of bf16) are below 2^24, those over all rows above; they are added as
    64 bits hold them and rounded once.  bf16: the bias, and of the weights, whose slices' sums pass 2^24, the first bits."""
    print("[case] weight grad of long sums", dtype, n, c, o, flush=True)
    g = torch.Generator(device="cuda").manual_seed(n)
    wide = torch.randint(50, 128, (n, (c + 15) // 16 * 16), device="cuda", dtype=torch.int8, generator=g)
    rows = dsvt.Rows8.of(wide[:, :c], torch.ones(n, device="cuda"))
    dy = torch.randint(*((1, 5) if dtype == "f32" else (100, 128)), (n, o), device="cuda", generator=g, dtype=torch.int32).to(DT[dtype])
    d_w, d_b = _sums(rows, dy)
    assert float((d_w if dtype == "f32" else d_b).min()) > 2 ** 24
    got, bias = dsvt.dsvt_linear_rows8_weight_grad(rows, dy)
    assert torch.equal(bias, d_b.float())
    if dtype == "f32":
        assert torch.equal(got, d_w.float())
    else:
        assert bool(((got.double() - d_w).abs() <= d_w * (2.0 ** -8 + 2.0 ** -14)).all())
