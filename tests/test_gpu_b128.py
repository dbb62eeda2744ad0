"""The cast to 8 bits with a Float32 scale per 128 and its inverse, bit for bit, and the product of such operands."""
import numpy as np
import pytest
import torch

import b128_model as model
from gpu_util import same_floats, to_dev, to_host
from paper_2310_10537_amd import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mx():
    from paper_2310_10537_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.lib()
    return binding


def awkward(rows, cols, seed):
    """Float32 data whose blocks hold zeros, outliers, infinities, NaN, subnormals, values near either end of the range, and ties."""
    wide = -(-cols // 32) * 32
    x = inputs.adversarial_f32(rows, wide, seed)[:, :cols].copy()
    g = np.random.default_rng(seed)
    for r in range(0, rows, 7):
        x[r] = (g.integers(-64, 65, cols) / 16).astype(np.float32)           # finite throughout, many of them half way
    for r in range(1, rows, 7):
        x[r] = g.standard_normal(cols).astype(np.float32)
    for r in range(2, rows, 7):
        x[r] = 0
    for r in range(3, rows, 7):
        x[r] = (g.standard_normal(cols) * 2.0 ** -127).astype(np.float32)
    return x


def padded(t, extra):
    """The same matrix with rows that are longer in memory, filled with a value that would show."""
    rows, cols = t.shape
    per16 = 16 // t.element_size()
    ld = -(-cols // per16) * per16 + extra
    out = torch.full((rows, ld), 3.0e30, dtype=t.dtype, device=t.device)[:, :cols]
    out.copy_(t)
    return out


SHAPES = [(1, 1), (1, 129), (3, 128), (130, 7), (127, 255), (128, 256), (260, 392), (33, 1000)]


@pytest.mark.parametrize("tile", [False, True], ids=["1x128", "128x128"])
@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("bf16", [False, True], ids=["f32", "bf16"])
def test_cast_and_back(mx, bf16, fmt, axis, tile):
    for rows, cols in SHAPES:
        for data in (awkward(rows, cols, rows + cols), inputs.gaussian_f32((rows, cols), seed=rows, std=0.02)):
            if bf16:
                bits = inputs.f32_to_bf16_bits(data)
                x, dev = inputs.bf16_bits_to_f32(bits), to_dev(bits)
            else:
                x, dev = data, to_dev(data)
            want_e, want_s = model.quantize(x, axis, fmt, tile)
            e, s = mx.mx_quantize_b128(padded(dev, 16), axis, fmt, tile=tile)
            what = (rows, cols)
            assert e.shape == want_e.shape and s.shape == want_s.shape, what
            assert np.array_equal(to_host(s).view(np.uint32), want_s.view(np.uint32)), what
            assert model.same_codes(to_host(e), want_e, fmt), what
            v = model.values(want_e, want_s, fmt, tile, np.float32)
            v = v[:, :cols] if axis == 1 else v[:, :rows].T
            v = np.ascontiguousarray(v)
            for dt in (torch.float32, torch.bfloat16):
                out = padded(torch.zeros((rows, cols), dtype=dt, device="cuda"), 16)
                whole = out._base if out._base is not None else out
                mx.mx_dequantize_b128(e, s, fmt, rows, cols, axis, tile=tile, out=out)
                want = v if dt == torch.float32 else inputs.f32_to_bf16_bits(v)
                assert same_floats(to_host(out), want), (what, dt)
                assert bool((whole[:, cols:] == torch.tensor(3.0e30, dtype=dt)).all()), what


def test_tile_cast_of_the_transpose_is_the_transpose(mx):
    w = to_dev(inputs.gaussian_f32((300, 520), seed=5))
    e, s = mx.mx_quantize_b128(w, 1, 0, tile=True)
    et, st = mx.mx_quantize_b128(w, 0, 0, tile=True)
    assert torch.equal(et[:, :300], e[:, :520].T) and torch.equal(st, s.T)


def test_largest_and_smallest_magnitudes(mx):
    """Scales at both ends of Float32's range."""
    big, tiny = np.finfo(np.float32).max, np.float32(2.0 ** -149)
    x = np.zeros((6, 128), dtype=np.float32)
    x[0, 3], x[1, 5], x[2, 7], x[3, 9], x[4, :2] = big, tiny, 2.0 ** -126, -2.0 ** -120, (np.inf, tiny)
    x[5, 0] = np.nan
    for fmt in (0, 1):
        want_e, want_s = model.quantize(x, 1, fmt, False)
        e, s = mx.mx_quantize_b128(to_dev(x), 1, fmt)
        assert np.array_equal(to_host(s), want_s) and model.same_codes(to_host(e), want_e, fmt)
        assert np.isfinite(want_s).all() and (want_s >= np.float32(2.0 ** -126)).all()


# ---------------------------------------------------------------------------------------------
# The product
# ---------------------------------------------------------------------------------------------
def integer_operand(rows, K, fmt, tile, g):
    """Codes of whole numbers -4 .. 4 and power-of-two scales: every sum of the product is exact in Float32 in any order."""
    codes = np.array([np.flatnonzero(model.table(fmt)[:124] == v)[0] for v in range(5)], dtype=np.uint8)
    v = g.integers(-4, 5, (rows, K), dtype=np.int8)
    e = codes[np.abs(v)] | np.where(v < 0, 128, 0).astype(np.uint8)
    shape = (-(-rows // 128) if tile else rows, K // 128)
    s = (2.0 ** g.integers(-2, 3, shape)).astype(np.float32)
    return e, s


GEMMS = [(1, 1, 128), (1, 200, 384), (2, 33, 1152), (15, 130, 1024), (16, 16, 2176), (17, 31, 640), (33, 129, 1280), (64, 300, 256), (65, 64, 128),
         (100, 257, 896), (128, 128, 512), (130, 70, 640), (300, 515, 384), (9, 16500, 256), (20, 8200, 384), (30, 8192, 1152), (64, 8200, 1024), (70, 130, 2048),
         (65, 257, 512), (200, 33000, 640), (257, 129, 1408), (1030, 8200, 768), (520, 530, 1024), (545, 1030, 1152), (530, 520, 384), (1030, 300, 640),
         (128, 1024, 256), (250, 510, 512)]


def product_operands(rows_a, rows_b, K, fa, fb, tiles, seed):
    g = np.random.default_rng(seed)
    return integer_operand(rows_a, K, fa, tiles[0], g), integer_operand(rows_b, K, fb, tiles[1], g)


@pytest.mark.parametrize("tiles", [(False, True), (False, False), (True, False), (True, True)], ids=lambda t: "x".join("tile" if v else "rows" for v in t))
@pytest.mark.parametrize("fa,fb", [(0, 0), (0, 1), (1, 0), (1, 1)])
def test_product_exactly(mx, fa, fb, tiles):
    """Where no sum rounds, every entry is exact whatever the kernel, and nothing beside C is written."""
    for M, N, K in GEMMS:
        (ea, sa), (eb, sb) = product_operands(M, N, K, fa, fb, tiles, M + N + K)
        va, vb = (torch.from_numpy(model.values(*o, np.float32)).cuda() for o in ((ea, sa, fa, tiles[0]), (eb, sb, fb, tiles[1])))
        want = (va.double() @ vb.double().T.contiguous()).cpu()
        a, b = (to_dev(ea), to_dev(sa)), (to_dev(eb), to_dev(sb))
        for dt in (torch.float32, torch.bfloat16):
            for pad in (0, 3, 8):
                buf = torch.full((M + 1, N + pad), 7.0, dtype=dt, device="cuda")
                mx.mx_gemm_b128(*a, fa, *b, fb, K, out=buf[:M, :N])
                assert torch.equal(buf[:M, :N].cpu(), want.float().to(dt)), (M, N, K, dt, pad)
                assert bool((buf[M:] == 7).all()) and bool((buf[:, N:] == 7).all()), (M, N, K, dt, pad)


def check_product(mx, a, sa, fa, b, sb, fb, tiles, K):
    """Against 64 bits.  Error of an entry: the matrix instruction cuts each run of 8 products at 14 bits below the largest (14 steps a
    run), Float32 rounds once per run and block, twice in a block's scale: K / 8 + 3 K / 128 roundings at most."""
    va = torch.from_numpy(model.values(a, sa, fa, tiles[0])).cuda()
    vb = torch.from_numpy(model.values(b, sb, fb, tiles[1])).cuda()
    C = mx.mx_gemm_b128(to_dev(a), to_dev(sa), fa, to_dev(b), to_dev(sb), fb, K).double()
    want, size = va @ vb.T.contiguous(), va.abs() @ vb.abs().T.contiguous()
    worst = torch.zeros_like(size)                      # sum over the runs of 8 of the largest product: at most |a| largest times |b| largest
    ma, mb = va.abs().view(va.shape[0], -1, 8).amax(2), vb.abs().view(vb.shape[0], -1, 8).amax(2)
    worst = ma @ mb.T.contiguous()
    bound = 14 * 2.0 ** -14 * worst + (K / 8 + 3 * K / 128) * 2.0 ** -24 * size
    err = (C - want).abs()
    assert bool((err <= bound).all()), float((err / bound).max())
    # and the errors, of either sign, are far below that together (cuts towards one side: a mean of half a step for 8 products)
    return float(err.norm() / want.norm())


@pytest.mark.parametrize("M,N,K", [(1, 300, 4096), (7, 129, 11008), (40, 260, 2048), (64, 96, 8192), (200, 333, 1152), (513, 700, 1024), (300, 300, 4096), (530, 520, 4096), (520, 530, 1152)], ids=str)
@pytest.mark.parametrize("fa,fb,tiles", [(0, 0, (False, True)), (1, 0, (False, True)), (0, 1, (False, False)), (0, 0, (True, True))], ids=str)
def test_product_of_cast_data(mx, M, N, K, fa, fb, tiles):
    a, sa = model.quantize(inputs.student_t_f32((M, K), seed=M), 1, fa, tiles[0])
    b, sb = model.quantize(inputs.gaussian_f32((N, K), seed=N, std=0.02), 1, fb, tiles[1])
    check_product(mx, a, sa, fa, b, sb, fb, tiles, K)


@pytest.mark.parametrize("M,N", [(3, 40), (70, 260), (300, 130), (600, 530)])
def test_nan_and_infinity_reach_their_entries_only(mx, M, N):
    K = 512
    x, w = np.ones((M, K), np.float32), np.ones((N, K), np.float32)
    x[1, 200], w[5, 300] = np.nan, np.inf
    a = mx.mx_quantize_b128(to_dev(x), 1, 0)
    b = mx.mx_quantize_b128(to_dev(w), 1, 1)
    C = mx.mx_gemm_b128(*a, 0, *b, 1, K)
    rows = torch.zeros((M, N), dtype=torch.bool)
    rows[1] = True
    assert torch.equal(C.isnan().cpu(), rows)
    rows[1] = False
    rows[:, 5] = True
    rows[1, 5] = False
    assert torch.equal(C.isinf().cpu(), rows)
    # the scales are fl(1 / 448) and fl(1 / 57344), so a value is 1 to within a rounding: both scales, their product, and four
    # multiply-adds of 128 * 448 * 57344 = 2^7 * 7^2 * 2^19, which is exact: seven roundings
    assert bool(((C[0, :5] - 512.0).abs() <= 512.0 * 7 * 2.0 ** -24).all())


def test_empty_k_and_empty_sizes(mx):
    e = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
    f = lambda *s: torch.empty(s, dtype=torch.float32, device="cuda")  # noqa: E731
    for M, N in ((3, 5), (200, 300)):
        C = mx.mx_gemm_b128(e(M, 0), f(M, 0), 0, e(N, 0), f(N, 0), 0, 0, out=torch.full((M, N), 9.0, device="cuda"))
        assert bool((C == 0).all())
    assert mx.mx_gemm_b128(e(0, 256), f(0, 2), 0, e(4, 256), f(4, 2), 0, 256).shape == (0, 4)
    assert mx.mx_gemm_b128(e(4, 256), f(4, 2), 0, e(0, 256), f(0, 2), 0, 256).shape == (4, 0)
    x = torch.empty((0, 256), device="cuda")
    codes, scales = mx.mx_quantize_b128(x, 1, 0)
    assert codes.shape == (0, 256) and scales.shape == (0, 2)
    assert mx.mx_dequantize_b128(codes, scales, 0, 0, 256, 1).shape == (0, 256)


def test_other_stream_and_captured_graph(mx):
    """Calls on a stream that is not the current one, and a captured cast and product replayed on new data."""
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((70, 640), device="cuda", generator=g)
    w = torch.randn((260, 640), device="cuda", generator=g) * 0.02
    we, ws = mx.mx_quantize_b128(w, 1, 0, tile=True)
    want = mx.mx_gemm_b128(*mx.mx_quantize_b128(x, 1, 0), 0, we, ws, 0, 640)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    e, s = mx.mx_quantize_b128(x, 1, 0, stream=st)
    out = torch.empty((70, 260), device="cuda")
    mx.mx_gemm_b128(e, s, 0, we, ws, 0, 640, out=out, stream=st)
    st.synchronize()
    assert torch.equal(out, want)
    for t in (e, s, out):
        t.record_stream(st)
    out.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mx.mx_quantize_b128(x, 1, 0, elems_out=e, scales_out=s)
        mx.mx_gemm_b128(e, s, 0, we, ws, 0, 640, out=out)
    for k in range(3):
        x.copy_(torch.randn((70, 640), device="cuda", generator=g))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, mx.mx_gemm_b128(*mx.mx_quantize_b128(x, 1, 0), 0, we, ws, 0, 640)), k
