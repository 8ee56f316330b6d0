"""What the calls on rows in 8 bits refuse, and their references: host code only, no GPU (nothing is enqueued for a call that is refused)."""
import ctypes as C
import os
from types import SimpleNamespace

import pytest
import torch

import rows8_ref as ref
from paper_2301_06051_amd import binding as b

if not os.path.exists(b.LIB_PATH):
    pytest.skip("library not built", allow_module_level=True)

P = 1 << 30                                        # an aligned address that no call reaches
N, W, O = 100, 192, 130


def _r8(codes=P, ld=W, scale=P):
    return C.byref(b.Rows8S(codes, ld, scale))


BAD_ROWS8 = [None, _r8(codes=None), _r8(scale=None), _r8(codes=P + 8), _r8(ld=W - 16), _r8(ld=W + 8), _r8(scale=P + 2)]


def _rms(c=W, dtype=b.DSVT_BF16, gamma=P, eps=1e-5):
    return C.byref(b.RmsCfg(c, dtype, gamma, eps))


def _linear(c=W, o=O, dtype=b.DSVT_BF16, act=0, codes=P, ld=W, scale=P):
    return C.byref(b.Linear8Cfg(c, o, dtype, act, b.Rows8S(codes, ld, scale), None))


BF, E, U = b.DSVT_BF16, b.DSVT_EINVAL, b.DSVT_EUNSUPPORTED


def test_rows_are_refused():
    L = b.lib()
    for bad in BAD_ROWS8:
        assert L.dsvt_keep_rows8(W, BF, P, W, N, bad, None) == E
        assert L.dsvt_read_rows8(W, BF, bad, N, P, W, None) == E
        assert L.dsvt_gelu_rows8_backward(W, BF, bad, P, W, N, P, W, None) == E
        assert L.dsvt_linear_rows8(_linear(), bad, N, P, O, None) == E
        assert L.dsvt_linear_rows8_weight_grad(W, O, BF, bad, P, O, N, P, W, None, P, 1 << 40, None) == E
        if bad is not None:
            assert L.dsvt_gelu_rows8(W, BF, P, W, N, bad, None, None) == E and L.dsvt_gelu_rows8(W, BF, P, W, N, None, bad, None) == E
            assert L.dsvt_rms_norm(_rms(), P, W, None, 0, N, None, 0, P, W, bad, None) == E
    assert L.dsvt_gelu_rows8(W, BF, P, W, N, None, None, None) == E
    far = P + (1 << 24)                            # two results in one place
    assert L.dsvt_gelu_rows8(W, BF, far, W, N, _r8(scale=far), _r8(), None) == E and L.dsvt_gelu_rows8(W, BF, far, W, N, _r8(codes=far), _r8(), None) == E
    assert L.dsvt_rms_norm(_rms(), far, W, None, 0, N, P, W, P, W, None, None) == E
    # rows too far apart for a step of the weight gradient
    assert L.dsvt_linear_rows8_weight_grad(W, O, BF, _r8(ld=1 << 24), P, O, N, P, W, None, P, 1 << 40, None) == U
    assert L.dsvt_linear_rows8_weight_grad(W, O, BF, _r8(), P, 1 << 24, N, P, W, None, P, 1 << 40, None) == U
    # addresses that are no multiple of an element, strides below a row, no address
    for at, ld in ((P + 1, W), (P, W - 1), (None, W)):
        assert L.dsvt_keep_rows8(W, BF, at, ld, N, _r8(), None) == E
        assert L.dsvt_read_rows8(W, BF, _r8(), N, at, ld, None) == E
        assert L.dsvt_gelu_rows8(W, BF, at, ld, N, _r8(), None, None) == E
        assert L.dsvt_gelu_rows8_backward(W, BF, _r8(), at, ld, N, P, W, None) == E
        assert L.dsvt_gelu_rows8_backward(W, BF, _r8(), P, W, N, at, ld, None) == E
        assert L.dsvt_linear_rows8(_linear(o=W), _r8(), N, at, ld, None) == E
        assert L.dsvt_linear_rows8_weight_grad(W, W, BF, _r8(), at, ld, N, P, W, None, P, 1 << 40, None) == E
        assert L.dsvt_linear_rows8_weight_grad(W, W, BF, _r8(), P, W, N, at, ld, None, P, 1 << 40, None) == E
        assert L.dsvt_rms_norm(_rms(), at, ld, None, 0, N, None, 0, P, W, None, None) == E
        assert L.dsvt_rms_norm(_rms(), P, W, None, 0, N, None, 0, at, ld, None, None) == E
        assert L.dsvt_rms_norm_backward(_rms(), at, ld, P, W, None, 0, None, 0, N, P, W, P, P, 1 << 40, None) == E
        assert L.dsvt_rms_norm_backward(_rms(), P, W, P, W, None, 0, None, 0, N, at, ld, P, P, 1 << 40, None) == E
        if at is not None:
            assert L.dsvt_rms_norm(_rms(), P, W, at, ld, N, None, 0, P, W, None, None) == E
            assert L.dsvt_rms_norm(_rms(), P, W, None, 0, N, at, ld, P, W, None, None) == E
            assert L.dsvt_rms_norm_backward(_rms(), P, W, P, W, None, 0, at, ld, N, P, W, P, P, 1 << 40, None) == E


def test_shapes_and_types_are_refused():
    L, size = b.lib(), C.c_size_t(0)
    for c, dtype, n, want in ((0, BF, N, E), (-1, BF, N, E), (W, 2, N, E), (W, -1, N, E), (W, BF, -1, E), (65537, BF, N, U)):
        r8 = _r8(ld=1 << 20)
        assert L.dsvt_keep_rows8(c, dtype, P, 1 << 20, n, r8, None) == want
        assert L.dsvt_read_rows8(c, dtype, r8, n, P, 1 << 20, None) == want
        assert L.dsvt_gelu_rows8(c, dtype, P, 1 << 20, n, r8, r8, None) == want
        assert L.dsvt_gelu_rows8_backward(c, dtype, r8, P, 1 << 20, n, P, 1 << 20, None) == want
        assert L.dsvt_linear_rows8(_linear(c=c, dtype=dtype, ld=1 << 20), r8, n, P, 1 << 20, None) == want
        assert L.dsvt_linear_rows8(_linear(o=c, dtype=dtype), _r8(), n, P, 1 << 20, None) == want
        for shape in ((c, O), (W, c)):
            assert L.dsvt_linear_rows8_weight_grad_workspace_size(*shape, dtype, n, C.byref(size)) == want
            assert L.dsvt_linear_rows8_weight_grad(*shape, dtype, r8, P, 1 << 20, n, P, 1 << 20, None, P, 1 << 40, None) == want
        assert L.dsvt_rms_norm(_rms(c, dtype), P, 1 << 20, None, 0, n, None, 0, P, 1 << 20, None, None) == want
        assert L.dsvt_rms_norm_backward_workspace_size(_rms(c, dtype), n, C.byref(size)) == want
    for cfg in (_rms(gamma=None), _rms(eps=-1.0), _rms(eps=float("nan"))):
        assert L.dsvt_rms_norm(cfg, P, W, None, 0, N, None, 0, P, W, None, None) == E
    assert L.dsvt_rms_norm(_rms(), P, W, None, 0, N, P, W, None, 0, None, None) == E                  # neither rows nor codes wanted
    for act in (-1, 2):
        assert L.dsvt_linear_rows8(_linear(act=act), _r8(), N, P, O, None) == E
    for w in (dict(codes=None), dict(scale=None), dict(ld=W - 16), dict(codes=P + 4)):
        assert L.dsvt_linear_rows8(_linear(**w), _r8(), N, P, O, None) == E


def test_scratch_is_refused():
    L, size = b.lib(), C.c_size_t(0)
    assert L.dsvt_rms_norm_backward_workspace_size(_rms(), N, None) == E and L.dsvt_linear_rows8_weight_grad_workspace_size(W, O, BF, N, None) == E
    assert L.dsvt_rms_norm_backward_workspace_size(_rms(), N, C.byref(size)) == 0 and size.value > 0
    for ws, nbytes, want in ((None, size.value, E), (P + 8, size.value, E), (P, size.value - 1, b.DSVT_ENOSPC)):
        assert L.dsvt_rms_norm_backward(_rms(), P, W, P, W, None, 0, None, 0, N, P, W, P, ws, nbytes, None) == want
    assert L.dsvt_rms_norm_backward(_rms(), P, W, P, W, None, 0, None, 0, N, P, W, None, P, 1 << 40, None) == E
    assert L.dsvt_linear_rows8_weight_grad_workspace_size(W, O, BF, 100 * N, C.byref(size)) == 0 and size.value > 0
    for ws, nbytes, want in ((None, size.value, E), (P + 8, size.value, E), (P, size.value - 1, b.DSVT_ENOSPC)):
        assert L.dsvt_linear_rows8_weight_grad(W, O, BF, _r8(), P, O, 100 * N, P, W, None, ws, nbytes, None) == want


def test_rows8_of_tensors():
    i8 = dict(dtype=torch.int8)
    good = torch.zeros((5, 112), **i8)[:, :99]
    r = b.Rows8.of(good, torch.zeros(5))
    assert (r.n, r.C, r.struct.ld, r.device) == (5, 99, 112, -1)
    assert b.Rows8.of(torch.zeros((1, 112), **i8)[:, :99], torch.zeros(1)).struct.ld == 112
    assert b.Rows8.empty(3, 100, "cpu").struct.ld == 112 and b.Rows8.empty(3, 64, "cpu").struct.ld == 64
    for codes, scale in ((torch.zeros((5, 99), **i8), torch.zeros(5)), (good, torch.zeros(4)), (good, torch.zeros(5).double()), (good.float(), torch.zeros(5)),
                         (torch.zeros((5, 128), **i8)[:, 8:107], torch.zeros(5)), (torch.zeros((112, 5), **i8).t(), torch.zeros(5)), (good[0], torch.zeros(5)),
                         (torch.zeros((5, 0), **i8), torch.zeros(5)), (torch.zeros(5 * 112 - 13, **i8).as_strided((5, 99), (112, 1)), torch.zeros(5)),
                         (torch.zeros((1, 99), **i8), torch.zeros(1)), (torch.zeros((1, 112), **i8).expand(5, 112), torch.zeros(5))):
        with pytest.raises(ValueError):
            b.Rows8.of(codes, scale)


def test_tensors_that_require_gradients_are_refused():
    def needing(name, k):
        return torch.zeros((4, 16), requires_grad=name == k)

    def calls(k):
        rows = SimpleNamespace(given=needing("scale", k), n=4, C=16, device=-1)
        rms = SimpleNamespace(gamma=needing("gamma", k))
        lin = SimpleNamespace(weight=SimpleNamespace(given=needing("w_scale", k)), bias=needing("bias", k), device=-1)
        t = lambda name: needing(name, k)  # noqa: E731
        return {"x": lambda: b.dsvt_keep_rows8(t("x")), "h": lambda: b.dsvt_gelu_rows8(t("h")),
                "scale xx": lambda: b.dsvt_read_rows8(rows, "f32", x=t("xx")),
                "x res gamma y z": lambda: b.dsvt_rms_norm(rms, t("x"), t("res"), t("y"), t("z")),
                "x res gamma z out": lambda: b.dsvt_rms_norm_rows8(rms, t("x"), t("res"), None, t("z")),
                "dy x res d_sum gamma dx d_gamma": lambda: b.dsvt_rms_norm_backward(rms, t("dy"), t("x"), t("res"), t("d_sum"), t("dx"), t("d_gamma")),
                "scale dy dh": lambda: b.dsvt_gelu_rows8_backward(rows, t("dy"), t("dh")),
                "scale w_scale bias y": lambda: b.dsvt_linear_rows8(lin, rows, t("y")),
                "scale dy d_w d_b": lambda: b.dsvt_linear_rows8_weight_grad(rows, t("dy"), t("d_w"), t("d_b"))}

    for k in {n for names in calls(None) for n in names.split()} - {"out"}:
        for names, call in calls(k).items():
            if k in names.split():
                with pytest.raises(RuntimeError, match="records no graph"):
                    call()


def test_reference_gradients_by_differences():
    """The references' gradients against quotients of differences of their own forward values."""
    g = torch.Generator().manual_seed(1)
    n, c = 4, 24
    x, dy, gamma = torch.randn((n, c), generator=g), torch.randn((n, c), generator=g), 1 + 0.2 * torch.randn((c,), generator=g)
    r = ref.rms(x, None, gamma, 1e-5, dy)

    def f(x, gamma):
        z = x.double()
        return float((z / (z.pow(2).mean(1, keepdim=True) + 1e-5).sqrt() * gamma.double() * dy.double()).sum())

    t = 1e-4                                       # third derivatives of some tens a value: 1e-8 times them, times sqrt(n c)
    for k in range(3):
        v, u = torch.randn((n, c), generator=g).double(), torch.randn((c,), generator=g).double()
        got = float((r["dx"][0] * v).sum() + (r["d_gamma"][0] * u).sum())
        assert abs((f(x + t * v, gamma + t * u) - f(x - t * v, gamma - t * u)) / (2 * t) - got) < 1e-5
    h = torch.linspace(-8, 8, 1001).double()
    assert float(((ref.gelu(h + t) - ref.gelu(h - t)) / (2 * t) - ref.gelu_slope(h)).abs().max()) < 1e-7
    assert bool((ref.gelu_slope(h) < 1.13).all())


def test_reference_codes():
    """Of halves: to the even one; of rows that have no scale."""
    codes, scale = ref.quantise(torch.tensor([[127., 0.5, 1.5, 2.5, -0.5, -1.5, -126.5], [0.] * 7, [1e-36] * 7, [float("inf")] + [1.] * 6]))
    assert codes.tolist() == [[127, 0, 2, 2, 0, -2, -126], [0] * 7, [0] * 7, [0] * 7]
    assert scale[:3].tolist() == [1., 0., 0.] and bool(scale[3].isnan())
