"""More that the calls on rows in 8 bits, and the norms', refuse: host code only, no GPU (nothing is enqueued for a call that is refused)."""
import os
from types import SimpleNamespace

import pytest
import torch

from paper_2301_06051_amd import binding as b

if not os.path.exists(b.LIB_PATH):
    pytest.skip("library not built", allow_module_level=True)

MANY = [(1 << 31, 16), ((1 << 32) + 5, 16), (3, (1 << 32) + 16)]


@pytest.mark.parametrize("n,c", MANY)
def test_more_rows_and_columns_than_31_bits_are_refused(n, c, monkeypatch):
    """(2^32 + 5 rows would be 5 in the library, and nothing said about it.)  Tensors without memory, of a device that counts as the current one."""
    monkeypatch.setattr(b, "_current_device", lambda: -1)
    empty = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device="meta")  # noqa: E731
    x, dy, vector = empty(n, c), empty(n, 16), empty(c, dtype=torch.float32)
    calls = [lambda: b.dsvt_keep_rows8(x), lambda: b.dsvt_gelu_rows8(x), lambda: b.Rows8.empty(n, c, "meta"),
             lambda: b.Rows8.of(empty(n, c, dtype=torch.int8), empty(n, dtype=torch.float32)),
             lambda: b.dsvt_linear_rows8_weight_grad_workspace_size(c, 64, "bf16", n), lambda: b.dsvt_linear_rows8_weight_grad_workspace_size(64, c, "bf16", n)]
    if n > c:
        few = SimpleNamespace(C=c, gamma=vector, beta=vector, dtype=torch.bfloat16, device=-1, size=(None, 0), ref=None)
        rows = SimpleNamespace(given=None, n=n, C=c, device=-1, ref=None)
        calls += [lambda: b.dsvt_rms_norm(few, x), lambda: b.dsvt_rms_norm_rows8(few, x), lambda: b.dsvt_rms_norm_backward(few, x, x), lambda: b.dsvt_layer_norm(few, x),
                  lambda: b.dsvt_layer_norm_backward(few, x, x), lambda: b.dsvt_gelu_rows8_backward(rows, x), lambda: b.dsvt_linear_rows8_weight_grad(rows, dy),
                  lambda: b.dsvt_rms_norm_backward_workspace_size(few, n), lambda: b.dsvt_layer_norm_backward_workspace_size(few, n)]
    else:
        calls += [lambda: b.RmsNorm(vector, "bf16"), lambda: b.LayerNorm(vector, vector, "bf16"),
                  lambda: b.dsvt_linear_rows8_weight_grad(SimpleNamespace(given=None, n=n, C=16, device=-1, ref=None), x)]
    for call in calls:
        with pytest.raises(ValueError, match="at most"):
            call()
