"""Gradients of the norm in captured graphs: the scratch memory of a replay is nobody else's."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mx():
    from paper_2310_10537_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.lib()
    return binding


def operands(rows, cols, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dy, h = (torch.randn((rows, cols), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    return dy, h, torch.randn((cols,), device="cuda", generator=g), torch.rand((rows,), device="cuda", generator=g) + 0.5


@pytest.mark.parametrize("given", [False, True], ids=["current_stream", "given_stream"])
@pytest.mark.parametrize("rows,cols", [(700, 1000), (40, 20000)], ids=str)
def test_graph_captured_without_torch(mx, rows, cols, given):
    """A capture that torch's allocator knows nothing of: the replays leave memory alone that torch has handed out since, and give the eager result."""
    with open("/proc/self/maps") as f:
        hip = ctypes.CDLL(next(line.split()[-1] for line in f if "libamdhip64" in line))
    dy, h, w, rstd = operands(rows, cols, rows)
    want = mx.mx_rmsnorm_bwd(dy, h, w, rstd)
    dx = torch.empty_like(dy)
    need = mx.lib().mx_rmsnorm_bwd_workspace_bytes(rows, cols)
    stream, graph, run = torch.cuda.Stream(), ctypes.c_void_p(), ctypes.c_void_p()
    raw = ctypes.c_void_p(stream.cuda_stream)
    torch.cuda.synchronize()

    def call():
        if given:
            return mx.mx_rmsnorm_bwd(dy, h, w, rstd, dx_out=dx, stream=stream)[1]
        with torch.cuda.stream(stream):
            return mx.mx_rmsnorm_bwd(dy, h, w, rstd, dx_out=dx)[1]

    eager = call()                                      # the pools hold blocks of these sizes now
    stream.synchronize()
    assert torch.equal(eager, want[1])
    del eager
    assert hip.hipStreamBeginCapture(raw, 2) == 0       # relaxed
    dw = call()
    assert hip.hipStreamEndCapture(raw, ctypes.byref(graph)) == 0 and graph.value
    assert hip.hipGraphInstantiate(ctypes.byref(run), graph, None, None, ctypes.c_size_t(0)) == 0
    later = []
    for st in (stream, torch.cuda.current_stream()):
        with torch.cuda.stream(st):
            later += [torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda") for n in (need, need, 4 * cols, 4 * cols)]
    torch.cuda.synchronize()
    for k in range(4):
        dx.zero_()
        dw.zero_()
        torch.cuda.synchronize()
        assert hip.hipGraphLaunch(run, raw) == 0
        stream.synchronize()
        assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]), k
        assert all(bool((t == 0xA5).all()) for t in later), k
        assert torch.equal(mx.mx_rmsnorm_bwd(dy, h, w, rstd)[1], want[1])        # eager work between the replays
        torch.cuda.synchronize()
    assert hip.hipGraphExecDestroy(run) == 0 and hip.hipGraphDestroy(graph) == 0


def test_two_graphs_at_once_with_a_workspace_each(mx):
    """The C entry that takes a workspace, captured twice and replayed on two streams at the same time."""
    rows, cols = 2500, 1024
    need = mx.lib().mx_rmsnorm_bwd_workspace_bytes(rows, cols)
    sets, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(2):
        dy, h, w, rstd = operands(rows, cols, 50 + k)
        want = mx.mx_rmsnorm_bwd(dy, h, w, rstd)
        dx, dw = torch.zeros_like(dy), torch.zeros((cols,), device="cuda")
        ws = torch.full((need,), 0xA5, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            status = mx.lib().mx_rmsnorm_bwd_ws(dy.data_ptr(), cols, h.data_ptr(), cols, w.data_ptr(), mx.DT_F32, rstd.data_ptr(), None, 0, mx.DT_BF16, rows, cols,
                                                dx.data_ptr(), cols, dw.data_ptr(), ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
        assert status == mx.MX_OK
        sets.append((graph, want, dx, dw, (dy, h, w, rstd, ws)))
    for _ in range(4):
        for _, _, dx, dw, _ in sets:
            dx.zero_()
            dw.zero_()
        torch.cuda.synchronize()
        for _ in range(5):
            for st, (graph, *_) in zip(streams, sets):
                with torch.cuda.stream(st):
                    graph.replay()
        torch.cuda.synchronize()
        for _, want, dx, dw, _ in sets:
            assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
