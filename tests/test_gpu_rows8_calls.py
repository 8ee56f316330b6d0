"""Calls on rows in 8 bits that the documentation allows: as many rows as a call can have, all results of a norm at once, what lies around results."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
dsvt = pytest.importorskip("paper_2301_06051_amd")

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def test_as_many_rows_as_a_call_can_have():
    """2^31 - 1 rows of one bf16 value: kept, read back and multiplied by one they are what they were.  (The value is 127 times its scale, two
    roundings of 32 bits off, so the same in bf16.)"""
    n = (1 << 31) - 1
    print("[case] 2^31 - 1 rows", flush=True)
    torch.cuda.empty_cache()
    x = torch.randn((n, 1), dtype=torch.bfloat16, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    kept = dsvt.dsvt_keep_rows8(x)
    back = torch.full_like(x, 7)
    assert torch.equal(dsvt.dsvt_read_rows8(kept, "bf16", x=back), x)
    one = dsvt.dsvt_keep_rows8(torch.ones((1, 1), device="cuda"))
    y = back.fill_(7)
    assert torch.equal(dsvt.dsvt_linear_rows8(dsvt.Linear8(one, "bf16"), kept, y=y), x)
    del x, kept, back, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,c,o", [(3, 64, 20), (100, 64, 70), (100, 4096, 20), (70000, 64, 64), (40000, 192, 200), (60000, 260, 250), (120000, 272, 251), (26000, 2100, 401), (200, 300, 130)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", [False, True])
def test_linear_of_huge_rows_and_tiny_weights(n, c, o, dtype, act):
    """Sums times a scale next to the largest pass 32 bits; times the other scale they are ordinary numbers.  Huge rows beside plain ones, in every kernel."""
    print("[case] huge rows", n, c, o, dtype, act, flush=True)
    g = torch.Generator(device="cuda").manual_seed(n + c)
    codes = lambda k: torch.randint(-127, 128, (k, (c + 15) // 16 * 16), device="cuda", generator=g).to(torch.int8)[:, :c]  # noqa: E731
    x, w, s = codes(n), codes(o), torch.rand(n, device="cuda", generator=g) + 0.5
    huge = torch.arange(n, device="cuda") % 7 == 2
    by = torch.where(huge, torch.full_like(s, 2.0 ** 120), torch.full_like(s, 2.0 ** 80))
    t = (torch.rand(o, device="cuda", generator=g) + 0.5) * 2.0 ** -100
    bias = 1e6 * torch.randn(o, device="cuda", generator=g)
    got = dsvt.dsvt_linear_rows8(dsvt.Linear8(dsvt.Rows8.of(w, t), dtype, bias, act), dsvt.Rows8.of(x, s * by)).double()
    p = (x.double() @ w.double().t().contiguous()) * (s * by).double()[:, None] * t.double()
    want = p + bias.double()
    # roundings: the sum's to 32 bits, of two products, of the bias's addition; then the type's; GELU is the value or next to nothing, but near zero
    e = 2.0 ** -24 * (3.5 * p.abs() + want.abs())
    if act:
        want, e = torch.where(want > 0, want, torch.zeros_like(want)), e + 0.2
    half = torch.finfo(DT[dtype]).eps / 2
    assert bool(got.isfinite().all()) and float(got[huge].abs().max()) > 2.0 ** 20
    assert bool(((got - want).abs() <= e + half * (want.abs() + e) + 1e-30).all())
