"""The RMS norm with its casts, and its gradients."""
import numpy as np
import pytest
import torch

import b128_model as model
from gpu_util import to_dev, to_host
from paper_2310_10537_amd import inputs

pytestmark = pytest.mark.gpu
EPS = 1e-5
B128 = 6                                                        # output kinds: the six MX formats, then the two with a scale per 128


@pytest.fixture(scope="module")
def mx():
    from paper_2310_10537_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.lib()
    return binding


def matrix(rows, cols, dt, seed, extra=8):
    """Seeded rows of different sizes with longer rows in memory, and their Float32 values."""
    g = np.random.default_rng(seed)
    x = (g.standard_normal((rows, cols)) * np.exp(g.standard_normal((rows, 1)))).astype(np.float32)
    per16 = 8 if dt == torch.bfloat16 else 4
    dev = torch.full((rows, -(-cols // per16) * per16 + extra), 77.0, dtype=dt, device="cuda")[:, :cols]
    dev.copy_(torch.from_numpy(x))
    return dev, dev.float().cpu().numpy()


def like(x):
    """Another matrix of the same pitch (which empty_like does not keep)."""
    return torch.full_like(x._base, -1.0)[:, :x.shape[1]]


def long_sum(cols):
    """Additions that a thread makes one after the other, and those that join the threads."""
    return 8 * max(8, -(-cols // 2048)) + 10


def check_rstd(rstd, h, eps):
    want = 1 / np.sqrt((h.astype(np.float64) ** 2).mean(1) + eps)
    # half the relative error of the sum; two roundings before the root, one unit of the root
    assert (np.abs(rstd - want) <= want * (long_sum(h.shape[1]) / 2 + 1 + 2) * 2.0 ** -24).all()


def cast(mx, y, kind, rnd):
    """The stand-alone cast of the Float32 y (with a row more, so that rows of any length have an aligned pitch)."""
    rows, cols = y.shape
    d = torch.full((rows + 1, -(-cols // 4) * 4), 5.0, device="cuda")[:, :cols]
    d[:rows].copy_(torch.from_numpy(y))
    e, s = mx.mx_quantize_b128(d, 1, kind - B128) if kind >= B128 else mx.mx_quantize(d, 1, kind, rnd)
    return e[:rows], s[:rows]


SHAPES = [(1, 1), (1, 4096), (3, 33), (5, 1000), (2, 2050), (1025, 130), (1030, 1000), (1024, 2056), (1100, 4096), (4, 4104), (3, 8200), (2, 16384), (2, 16392), (1, 40000)]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES, ids=str)
def test_norm_and_casts(mx, rows, cols, dt):
    """h, rstd and y against their definitions, and every cast equal to that of y."""
    x, xf = matrix(rows, cols, dt, rows + cols)
    r, rf = matrix(rows, cols, dt, rows + cols + 1)
    w, wf = matrix(1, cols, torch.float32 if rows % 2 else dt, 9, 0)
    w, wf = w.reshape(-1), wf[0]
    for residual in (False, True):
        hf = xf
        if residual:
            hf = xf + rf
            hf = inputs.bf16_bits_to_f32(inputs.f32_to_bf16_bits(hf)) if dt == torch.bfloat16 else hf
        h = like(x)
        rstd = torch.empty((rows,), device="cuda")
        y = mx.mx_rmsnorm(x, w, EPS, residual=r if residual else None, h_out=h, rstd_out=rstd)
        rs = to_host(rstd)
        check_rstd(rs, hf, EPS)
        assert np.array_equal(h.float().cpu().numpy(), hf)
        yf = (hf * wf) * rs[:, None]
        assert np.array_equal(y.float().cpu().numpy(), yf if dt == torch.float32 else inputs.bf16_bits_to_f32(inputs.f32_to_bf16_bits(yf)))
        for kind in range(8):
            for rnd in (0, 1, 2) if kind < B128 and rows * cols < 20000 else (0,):
                h = like(x)
                kw = {"residual": r if residual else None, "h_out": h, "rstd_out": rstd.zero_()}
                got = mx.mx_rmsnorm_b128(x, w, EPS, kind - B128, **kw) if kind >= B128 else mx.mx_rmsnorm_q(x, w, EPS, kind, rnd, **kw)
                assert np.array_equal(to_host(rstd), rs) and np.array_equal(h.float().cpu().numpy(), hf), kind
                want = cast(mx, yf, kind, rnd)
                assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (residual, kind, rnd)


@pytest.mark.parametrize("rows,cols", [(1, 129), (3, 1000), (1030, 520), (2, 16392)], ids=str)
def test_rows_of_zeros_nan_and_infinity(mx, rows, cols):
    """A row of zeros stays zero, a NaN takes its row, an infinity makes rstd zero; the other rows do not notice."""
    for dt in (torch.float32, torch.bfloat16):
        x, xf = matrix(rows, cols, dt, cols)
        bad = x.clone()
        if rows > 2:
            bad[1, cols // 2] = float("nan")
            bad[2, cols - 1] = float("inf")
        bad[0] = 0
        for kind in range(8):
            f = (lambda t: mx.mx_rmsnorm_b128(t, None, EPS, kind - B128)) if kind >= B128 else (lambda t: mx.mx_rmsnorm_q(t, None, EPS, kind))
            good, got = f(x), f(bad)
            y = mx.mx_rmsnorm(bad, None, EPS).float().cpu().numpy()
            assert not y[0].any() and (rows < 3 or (np.isnan(y[1]).all() and np.isnan(y[2, -1]) and not y[2, :-1].any()))
            assert torch.equal(good[0][3:], got[0][3:]) and torch.equal(good[1][3:], got[1][3:])
            assert not (got[0][0] & 127).any()
            if rows > 2 and dt == torch.float32:
                want = cast(mx, y, kind, 0)
                if kind >= B128:
                    assert model.same_codes(to_host(want[0]), to_host(got[0]), kind - B128)
                else:
                    assert torch.equal(got[0][2:], want[0][2:]) or kind < 2
                assert torch.equal(got[1].view(torch.uint8), want[1].view(torch.uint8))


def test_in_place_and_all_outputs(mx):
    """h over x or over the residual, y over x, nothing written beside the rows."""
    for rows, cols in ((3, 1000), (1030, 1000), (2, 20000)):
        x, _ = matrix(rows, cols, torch.bfloat16, 1)
        r, _ = matrix(rows, cols, torch.bfloat16, 2)
        w, _ = matrix(1, cols, torch.bfloat16, 3, 0)
        w = w.reshape(-1)
        h, y = like(x), like(x)
        want = mx.mx_rmsnorm_q(x, w, EPS, 0, residual=r, h_out=h, y_out=y)
        for target in ("x", "r"):
            a, b = x._base.clone()[:, :cols], r._base.clone()[:, :cols]
            into = a if target == "x" else b
            got = mx.mx_rmsnorm_q(a, w, EPS, 0, residual=b, h_out=into)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(into, h)
            assert bool((into._base[:, cols:] == 77).all())
        a = x._base.clone()[:, :cols]
        assert torch.equal(mx.mx_rmsnorm(a, w, EPS, residual=r, y_out=a), y) and torch.equal(a, y)
        assert bool((a._base[:, cols:] == 77).all())


BWD = [(1, 1), (1, 4096), (7, 33), (3, 129), (600, 512), (2100, 520), (2500, 1000), (2049, 2048), (700, 2056), (515, 4100), (600, 8192), (5, 8200), (70, 20000)]


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", BWD, ids=str)
def test_gradients(mx, rows, cols, dt):
    dy, dyf = matrix(rows, cols, dt, 1)
    h, hf = matrix(rows, cols, dt, 2)
    dh, dhf = matrix(rows, cols, dt, 3)
    for weighted in (True, False):
        w = to_dev(inputs.gaussian_f32((cols,), seed=4)) if weighted else None
        wf = w.cpu().numpy() if weighted else None
        rstd = torch.empty((rows,), device="cuda")
        mx.mx_rmsnorm(h, w, EPS, rstd_out=rstd)
        for past in (False, True):
            dx, dw = mx.mx_rmsnorm_bwd(dy, h, w, rstd, dh=dh if past else None)
            rs = to_host(rstd)
            want, want_w = model.norm_backward(dyf, hf, wf, rs, dhf if past else None)
            # roundings: four in a term of the mean, its sum; four more, each at most the size of what it rounds
            g, x = np.abs(dyf * (wf if weighted else 1.0)).astype(np.float64), np.abs(hf * rs[:, None]).astype(np.float64)
            mean = (g * x).mean(1, keepdims=True)
            size = rs[:, None] * (g + x * mean)
            bound = size * (long_sum(cols) + 8) * 2.0 ** -24 + (np.abs(dhf) + np.abs(want) if past else 0) * 2.0 ** -24 + 2.0 ** -140
            if dt == torch.bfloat16:
                bound = bound + (np.abs(want) + bound) * 2.0 ** -8
            got = dx.float().cpu().numpy()
            assert (np.abs(got - want) <= bound).all(), (weighted, past)
            # dweight: xhat rounded once, a thread's rows one after the other, then the lines: never more than rows of them
            total = (np.abs(dyf) * x).astype(np.float64).sum(0)
            chain = min(rows, -(-rows // 64) + 64 + 20)
            assert (np.abs(to_host(dw) - want_w) <= total * (chain + 2) * 2.0 ** -24 + 2.0 ** -140).all(), (weighted, past)
        only, none = mx.mx_rmsnorm_bwd(dy, h, w, rstd, dh=dh, want_dweight=False)
        assert none is None and torch.equal(only, dx)
        for target in ("dy", "h", "dh"):
            t = {"dy": dy, "h": h, "dh": dh}
            t = {k: v._base.clone()[:, :cols] for k, v in t.items()}
            got, dw2 = mx.mx_rmsnorm_bwd(t["dy"], t["h"], w, rstd, dh=t["dh"], dx_out=t[target])
            assert torch.equal(got, dx) and torch.equal(dw2, dw) and bool((got._base[:, cols:] == 77).all()), target


def test_gradients_against_differences(mx):
    """(f(h + d) - f(h - d)) / 2d of f = sum dy y in 64 bits."""
    rows, cols, d = 3, 40, 1e-5
    dy, dyf = matrix(rows, cols, torch.float32, 1)
    h, hf = matrix(rows, cols, torch.float32, 2)
    w = inputs.gaussian_f32((cols,), seed=4)
    rstd = torch.empty((rows,), device="cuda")
    mx.mx_rmsnorm(h, to_dev(w), EPS, rstd_out=rstd)
    dx, dw = mx.mx_rmsnorm_bwd(dy, h, to_dev(w), rstd)

    def f(hh, ww):
        return (dyf * (hh * ww / np.sqrt((hh * hh).mean(1, keepdims=True) + EPS))).sum()

    for r in range(rows):
        for c in range(0, cols, 3):
            e = np.zeros((rows, cols))
            e[r, c] = d
            want = (f(hf + e, w) - f(hf - e, w)) / (2 * d)
            assert abs(float(dx[r, c]) - want) <= 1e-4 * max(1.0, abs(want))      # d^2 f''' / 6, far below
    for c in range(cols):
        e = np.zeros(cols)
        e[c] = d
        want = (f(hf.astype(np.float64), w + e) - f(hf.astype(np.float64), w - e)) / (2 * d)
        assert abs(float(dw[c]) - want) <= 1e-4 * max(1.0, abs(want))


def test_empty_sizes(mx):
    x = torch.empty((0, 64), device="cuda")
    assert mx.mx_rmsnorm(x, None, EPS).shape == (0, 64)
    dx, dw = mx.mx_rmsnorm_bwd(x, x, None, torch.empty((0,), device="cuda"))
    assert dx.shape == (0, 64) and not dw.any() and dw.shape == (64,)
    e, s = mx.mx_rmsnorm_b128(torch.empty((4, 0), device="cuda"), None, EPS, 0)
    assert e.shape == (4, 0) and s.shape == (4, 0)


def test_stream_and_captured_graph(mx):
    """On another stream, with the scratch memory from the library or a workspace, and captured with both passes."""
    g = torch.Generator(device="cuda").manual_seed(1)
    rows, cols = 700, 1000
    x, r, dy = (torch.randn((rows, cols), device="cuda", generator=g).to(torch.bfloat16) for _ in range(3))
    w = torch.randn((cols,), device="cuda", generator=g)
    h, rstd, dx = torch.empty_like(x), torch.empty((rows,), device="cuda"), torch.empty_like(x)

    def both(stream=None):
        e, s = mx.mx_rmsnorm_q(x, w, EPS, 0, residual=r, h_out=h, rstd_out=rstd, stream=stream)
        return e, s, *mx.mx_rmsnorm_bwd(dy, h, w, rstd, dx_out=dx, stream=stream)

    want = [t.clone() for t in both()]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = both(st)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ws = torch.empty(mx.lib().mx_rmsnorm_bwd_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    e = torch.empty((rows, 1024), dtype=torch.uint8, device="cuda")
    s = torch.empty((rows, 32), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mx.mx_rmsnorm_q(x, w, EPS, 0, residual=r, h_out=h, rstd_out=rstd, elems_out=e, scales_out=s)
        dx2, dw2 = mx.mx_rmsnorm_bwd(dy, h, w, rstd)
    for k in range(3):
        for t in (x, r, dy):
            t.copy_(torch.randn((rows, cols), device="cuda", generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (e, s, dx2, dw2)]
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
    del ws


def test_two_captured_graphs_at_once(mx):
    """Gradients captured in two graphs, replayed on two streams at the same time: each has its scratch memory."""
    g = torch.Generator(device="cuda").manual_seed(3)
    w = torch.randn((2048,), device="cuda", generator=g)
    sets, graphs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(2):
        dy, h = (torch.randn((3000, 2048), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
        rstd = torch.rand((3000,), device="cuda", generator=g) + 0.5
        sets.append((dy, h, rstd, [t.clone() for t in mx.mx_rmsnorm_bwd(dy, h, w, rstd)]))
    torch.cuda.synchronize()
    for dy, h, rstd, _ in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, mx.mx_rmsnorm_bwd(dy, h, w, rstd)))
    for _ in range(4):
        for graph, (dx, dw) in graphs:
            dx.zero_()
            dw.zero_()
        torch.cuda.synchronize()
        for _ in range(5):
            for st, (graph, _) in zip(streams, graphs):
                with torch.cuda.stream(st):
                    graph.replay()
        torch.cuda.synchronize()
        for (_, got), (*_, want) in zip(graphs, sets):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_binding_refuses_tensors_that_do_not_fit(mx):
    x = torch.zeros((32, 256), device="cuda")
    w, rstd = torch.ones((256,), device="cuda"), torch.ones((32,), device="cuda")
    e, s = mx.mx_quantize_b128(x, 1, 0)
    half = x.to(torch.bfloat16)
    for call in (lambda: mx.mx_rmsnorm(x[0], w, EPS), lambda: mx.mx_rmsnorm(x.t(), w[:32].contiguous(), EPS), lambda: mx.mx_rmsnorm(x, w[:128], EPS),
                 lambda: mx.mx_rmsnorm(x, w, EPS, residual=half), lambda: mx.mx_rmsnorm(x, w, EPS, residual=x[:31]), lambda: mx.mx_rmsnorm(x, w, EPS, h_out=x.cpu()),
                 lambda: mx.mx_rmsnorm(x, w.cpu(), EPS), lambda: mx.mx_rmsnorm(x, w, EPS, rstd_out=rstd.double()), lambda: mx.mx_rmsnorm_q(x, w, EPS, 0, elems_out=e[:, :128]),
                 lambda: mx.mx_rmsnorm_b128(x, w, EPS, 0, scales_out=s.t()), lambda: mx.mx_rmsnorm_bwd(x, half, w, rstd), lambda: mx.mx_rmsnorm_bwd(x, x, w, rstd[:31]),
                 lambda: mx.mx_rmsnorm_bwd(x, x, w, rstd, dx_out=x[:, :128]), lambda: mx.mx_dequantize_b128(e, s, 0, 32, 384, 1), lambda: mx.mx_dequantize_b128(e, s, 0, 33, 256, 1),
                 lambda: mx.mx_dequantize_b128(e, s, 0, 32, 256, 1, out=x[:31]), lambda: mx.mx_gemm_b128(e, s, 0, e, s[:7], 0, 256), lambda: mx.mx_gemm_b128(e, s, 0, e, s, 0, 128),
                 lambda: mx.mx_gemm_b128(e, s, 0, e.cpu(), s.cpu(), 0, 256), lambda: mx.mx_gemm_b128(e, s, 0, e, s, 0, 256, out=x)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: mx.mx_rmsnorm(x.half(), None, EPS), lambda: mx.mx_rmsnorm(x, w.half(), EPS), lambda: mx.mx_quantize_b128(x.double(), 1, 0),
                 lambda: mx.mx_gemm_b128(e, s, 0, e, s, 0, 256, dtype=torch.float16)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: mx.mx_quantize_b128(x, 1, 2), lambda: mx.mx_quantize_b128(x, 2, 0), lambda: mx.mx_rmsnorm(x, w, -1.0), lambda: mx.mx_rmsnorm_q(x, w, EPS, 6),
                 lambda: mx.mx_rmsnorm_q(x, w, EPS, 0, rnd=3), lambda: mx.mx_quantize_b128(torch.zeros((32, 250), device="cuda"), 1, 0)):
        with pytest.raises(mx.MxError):
            call()
