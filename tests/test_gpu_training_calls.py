"""How the training calls treat streams, memory and arguments on the GPU."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu
dsvt = pytest.importorskip("paper_2301_06051_amd")
from gpu_util import gpu_maps  # noqa: E402
from paper_2301_06051_amd import binding  # noqa: E402

N, C, HEADS, WIN = 300, 64, 4, (12, 12, 1)


def _problem():
    g = torch.Generator().manual_seed(1)
    cell = torch.randperm(400, generator=g)[:N]
    coords = torch.stack([torch.zeros_like(cell), cell // 20, cell % 20, torch.zeros_like(cell)], 1).to(torch.int32).cuda()
    maps = gpu_maps(coords, (20, 20, 1), WIN, (0, 0, 0), 36, 1, 0)
    qkv, d_out = (torch.randn((N, k * C), generator=g).to(torch.bfloat16).cuda() for k in (3, 1))
    mha = dsvt.SetMha(C, HEADS, "bf16", WIN, torch.randn((HEADS, 529), generator=g).cuda())
    ln = dsvt.LayerNorm(torch.ones(C, device="cuda"), torch.zeros(C, device="cuda"), "bf16")
    return coords, maps, qkv, d_out, mha, ln


def _calls(problem, **kw):
    coords, maps, qkv, d_out, mha, ln = problem
    return [dsvt.dsvt_set_mha(mha, maps, coords, qkv, **kw), *dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, d_out, **kw),
            dsvt.dsvt_layer_norm(ln, d_out, **kw), *dsvt.dsvt_layer_norm_backward(ln, d_out, d_out, **kw)]


class _Recorder:
    """The library, keeping the arguments of its calls."""

    def __init__(self, library):
        self.library, self.calls = library, []

    def __getattr__(self, name):
        f = getattr(self.library, name)
        return lambda *args: self.calls.append((name, args)) or f(*args)


def _stream_of(pointer):
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= pointer < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("no block of the allocator's")


@pytest.mark.parametrize("handle", ["other", "default", "current"])
def test_memory_of_a_call_on_another_stream_is_that_streams(handle, monkeypatch):
    """Outputs and scratch that a call allocates are blocks of the stream its kernels run on: one of the current stream's may be in use there."""
    problem = _problem()
    want = _calls(problem)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    current = side if handle == "default" else torch.cuda.current_stream()
    run_on = {"other": side, "default": torch.cuda.default_stream(), "current": current}[handle].cuda_stream
    recorder = _Recorder(binding.lib())
    monkeypatch.setattr(binding, "lib", lambda: recorder)
    with torch.cuda.stream(current):
        got = _calls(problem, stream=run_on)
    torch.cuda.synchronize()
    scratch = [args[-3] for name, args in recorder.calls if name in ("dsvt_set_mha_backward", "dsvt_layer_norm_backward")]
    assert len(scratch) == 2 and all(scratch)
    assert all(args[-1] == run_on for name, args in recorder.calls if not name.endswith("size"))
    assert all(_stream_of(p) == run_on for p in scratch + [t.data_ptr() for t in got])
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_set_mha_slices_of_one_array_lie_beside_each_other():
    """All arrays of a call as columns of one; over each other they are refused."""
    coords, maps, qkv, d_out, mha, _ = _problem()
    wide = torch.full((N, 8 * C + 16), 5.0, dtype=torch.bfloat16, device="cuda")
    x, o, g, d = (wide[:, a * C:b * C] for a, b in ((0, 3), (3, 4), (4, 5), (5, 8)))
    x.copy_(qkv)
    g.copy_(d_out)
    want = dsvt.dsvt_set_mha(mha, maps, coords, qkv), dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, d_out)[0]
    dsvt.dsvt_set_mha(mha, maps, coords, x, out=o)
    dsvt.dsvt_set_mha_backward(mha, maps, coords, x, g, d_qkv=d)
    assert torch.equal(o, want[0]) and torch.equal(d, want[1]) and torch.equal(x, qkv) and bool((wide[:, 8 * C:] == 5).all())
    # row by row one behind the other: of the same array, N rows on
    both = torch.empty((2 * N, 3 * C), dtype=torch.bfloat16, device="cuda")
    both[:N].copy_(qkv)
    dsvt.dsvt_set_mha_backward(mha, maps, coords, both[:N], d_out, d_qkv=both[N:])
    assert torch.equal(both[:N], qkv) and torch.equal(both[N:], want[1])
    for out in (x[:, :C], x[:, 2 * C:], wide[:, 2 * C + 8:3 * C + 8]):
        with pytest.raises(dsvt.DsvtError):
            dsvt.dsvt_set_mha(mha, maps, coords, x, out=out)
    for grad in (x, wide[:, 2 * C:5 * C], wide[:, 4 * C - 8:7 * C - 8], both[1:N + 1]):
        with pytest.raises(dsvt.DsvtError):
            dsvt.dsvt_set_mha_backward(mha, maps, coords, x if grad._base is wide else both[:N], g, d_qkv=grad)


def test_calls_within_an_autograd_function():
    """As part of a graph: in a Function, whose gradients are those of the calls made by hand; not twice differentiable, which is refused."""
    coords, maps, qkv, d_out, mha, ln = _problem()

    class Attention(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, table):
            ctx.save_for_backward(x, table)
            return dsvt.dsvt_set_mha(dsvt.SetMha(C, HEADS, "bf16", WIN, table), maps, coords, x)

        @staticmethod
        def backward(ctx, g):
            x, table = ctx.saved_tensors
            return dsvt.dsvt_set_mha_backward(dsvt.SetMha(C, HEADS, "bf16", WIN, table), maps, coords, x, g.contiguous())

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, branch, gamma, beta):
            ctx.save_for_backward(x, branch, gamma, beta)
            return dsvt.dsvt_layer_norm(dsvt.LayerNorm(gamma, beta, "bf16"), x, branch)

        @staticmethod
        def backward(ctx, dy):
            x, branch, gamma, beta = ctx.saved_tensors
            dz, dg, db = dsvt.dsvt_layer_norm_backward(dsvt.LayerNorm(gamma, beta, "bf16"), dy.contiguous(), x, branch)
            return dz, dz, dg, db

    x, t, gamma, beta = (a.detach().clone().requires_grad_() for a in (qkv, mha.rel_bias, ln.gamma, ln.beta))
    with pytest.raises(RuntimeError, match="records no graph"):
        dsvt.dsvt_set_mha(mha, maps, coords, x)
    o = Attention.apply(x, t)
    y = Norm.apply(d_out, o, gamma, beta)
    got = torch.autograd.grad(y, (x, t, gamma, beta), d_out, retain_graph=True)
    plain = dsvt.dsvt_set_mha(mha, maps, coords, qkv)
    dz, dg, db = dsvt.dsvt_layer_norm_backward(ln, d_out, d_out, plain)
    assert torch.equal(y, dsvt.dsvt_layer_norm(ln, d_out, plain))
    assert all(torch.equal(a, b) for a, b in zip(got, (*dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, dz), dg, db)))
    with pytest.raises(RuntimeError, match="records no graph"):
        torch.autograd.grad(y, (x, t), d_out, create_graph=True)


def test_scratch_of_the_caller():
    """Of any type and of more bytes than needed; on the host, expanded or too small it is refused."""
    coords, maps, qkv, d_out, mha, ln = _problem()
    want = dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, d_out), dsvt.dsvt_layer_norm_backward(ln, d_out, d_out)
    sizes = dsvt.dsvt_set_mha_backward_workspace_size(mha, maps), dsvt.dsvt_layer_norm_backward_workspace_size(ln, N)
    for t in (torch.uint8, torch.float32):
        a, b = (torch.full((s // t.itemsize + 5,), 3, dtype=t, device="cuda") for s in sizes)
        assert all(torch.equal(x, y) for x, y in zip(dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, d_out, ws=a), want[0]))
        assert all(torch.equal(x, y) for x, y in zip(dsvt.dsvt_layer_norm_backward(ln, d_out, d_out, ws=b), want[1]))
        assert bool((a[-5:] == 3).all()) and bool((b[-5:] == 3).all())
    for bad in (torch.zeros(max(sizes), dtype=torch.uint8), torch.zeros(1, dtype=torch.uint8, device="cuda").expand(max(sizes))):
        with pytest.raises(ValueError):
            dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, d_out, ws=bad)
        with pytest.raises(ValueError):
            dsvt.dsvt_layer_norm_backward(ln, d_out, d_out, ws=bad)
    with pytest.raises(dsvt.DsvtError):
        dsvt.dsvt_set_mha_backward(mha, maps, coords, qkv, d_out, ws=torch.zeros(sizes[0] - 1, dtype=torch.uint8, device="cuda"))
    with pytest.raises(dsvt.DsvtError):
        dsvt.dsvt_layer_norm_backward(ln, d_out, d_out, ws=torch.zeros(sizes[1] - 1, dtype=torch.uint8, device="cuda"))


def test_one_voxel_out_of_odd_rows():
    """A tensor of one row has a stride that nothing goes by."""
    coords, _, qkv, d_out, mha, ln = _problem()
    maps = dsvt.SetMaps.of(torch.zeros((1, 4), dtype=torch.int32, device="cuda"), torch.ones((1,), dtype=torch.int32, device="cuda"), 1)
    odd = torch.zeros((2, 3 * C + 1), dtype=torch.bfloat16, device="cuda")
    odd[:1, :3 * C] = qkv[:1]
    x, g = odd[:1, :3 * C], d_out[:1]
    assert torch.equal(dsvt.dsvt_set_mha(mha, maps, coords[:1].clone(), x), qkv[:1, 2 * C:])       # one key: its value
    d_qkv, d_rel = dsvt.dsvt_set_mha_backward(mha, maps, coords[:1].clone(), x, g)
    assert torch.equal(d_qkv[:, 2 * C:], g) and not d_qkv[:, :2 * C].any() and not d_rel.any()


def _launches(call):
    """(workgroups, bytes of dynamic LDS) of the kernels that a call launches, from its captured graph, which is never run."""
    class Params(ctypes.Structure):                  # hipKernelNodeParams
        _fields_ = [("block", ctypes.c_uint32 * 3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", ctypes.c_uint32 * 3),
                    ("args", ctypes.c_void_p), ("lds", ctypes.c_uint32)]

    with open("/proc/self/maps") as f:
        hip = ctypes.CDLL(next(line.split()[-1] for line in f if "libamdhip64" in line))
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw, count, kind, out = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0), ctypes.c_int(0), []
    assert hip.hipGraphGetNodes(raw, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert hip.hipGraphGetNodes(raw, nodes, ctypes.byref(count)) == 0
    for node in nodes:
        assert hip.hipGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        if kind.value == 0:                          # hipGraphNodeTypeKernel
            p = Params()
            assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(p)) == 0
            out.append((p.grid[0], p.lds))
    return out


@pytest.mark.parametrize("win,heads,tau,most", [((12, 12, 1), 8, 36, 512), ((12, 12, 8), 8, 48, 512), ((12, 12, 32), 8, 36, 256), ((30, 30, 20), 8, 36, 512),
                                                ((12, 12, 32), 24, 48, 256), ((12, 12, 1), 24, 36, 512), ((12, 12, 1), 8, 90, 256)])
def test_set_mha_workgroups_fit_the_chip_at_once(win, heads, tau, most):
    """A forward call fills 256 compute units once: with two workgroups each where half of the LDS and of the registers is enough, else with one."""
    n, sets = 40, 5000
    maps = dsvt.SetMaps.of(torch.full((sets, tau), -1, dtype=torch.int32, device="cuda"), torch.zeros((1,), dtype=torch.int32, device="cuda"), n)
    coords, qkv = torch.zeros((n, 4), dtype=torch.int32, device="cuda"), torch.zeros((n, 24 * heads), dtype=torch.bfloat16, device="cuda")
    mha = dsvt.SetMha(8 * heads, heads, "bf16", win, torch.zeros((heads, (2 * win[0] - 1) * (2 * win[1] - 1) * (2 * win[2] - 1)), device="cuda"))
    out = torch.empty((n, 8 * heads), dtype=torch.bfloat16, device="cuda")
    (grid, lds), = _launches(lambda: dsvt.dsvt_set_mha(mha, maps, coords, qkv, out=out))
    print("[case]", win, heads, tau, grid, "workgroups", lds, "bytes", flush=True)
    assert most * 3 // 4 <= grid <= most and lds <= (65 << 10 if most == 512 else 146 << 10)


def test_layer_norm_adds_workgroups_in_64_bits():
    """Gradients in rows 64 apart, each in another workgroup's sum and so alone in it: what is left of large ones that cancel is exact."""
    n, c = 16384, 64
    g = torch.Generator().manual_seed(5)
    dy = torch.zeros((n, c))
    few = torch.randint(1 << 19, 1 << 20, (256, c), generator=g).float()
    few[1::2] = 1 / 8 - few[::2]                     # (20 bits and three behind the point)
    dy[::64] = few
    ln = dsvt.LayerNorm(torch.ones(c, device="cuda"), torch.zeros(c, device="cuda"), "f32")
    x = torch.randn((n, c), generator=g)
    _, _, d_beta = dsvt.dsvt_layer_norm_backward(ln, dy.cuda(), x.cuda())
    want = dy.double().sum(0)
    assert bool((want.abs() < 64).all()) and torch.equal(d_beta.cpu(), want.float())
