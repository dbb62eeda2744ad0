"""The norms, the 128-element forms and the products together, as a layer uses them: forward, gradient of the input, gradient of the weight."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 1e-5
E4M3, E5M2 = 0, 1


@pytest.fixture(scope="module")
def mx():
    from paper_2310_10537_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.lib()
    return binding


def near(got, want, cut, what):
    """A product of bf16 output against 64 bits: half a unit of the output's significand, and what the matrix instruction cuts off (`cut`)."""
    assert bool(((got.double() - want).abs() <= want.abs() * 2.0 ** -8 + cut * (1 + 2.0 ** -8)).all()), what


def cut_of(a, b):
    """14 steps of 2^-14 of the largest product of each run of 8, and a Float32 rounding for each run and three for each block."""
    K = a.shape[1]
    ma, mb = a.abs().view(a.shape[0], -1, 8).amax(2), b.abs().view(b.shape[0], -1, 8).amax(2)
    return 14 * 2.0 ** -14 * (ma @ mb.T.contiguous()) + (K / 8 + 3 * K / 128) * 2.0 ** -24 * (a.abs() @ b.abs().T.contiguous())


@pytest.mark.parametrize("M,K,N", [(1, 256, 384), (40, 640, 1000), (300, 520, 257), (1030, 1024, 768)], ids=str)
def test_projection_forward_and_backward(mx, M, K, N):
    g = torch.Generator(device="cuda").manual_seed(M)
    rows = lambda m, n, std=1.0: mx._empty_rows(m, n, torch.bfloat16, torch.device("cuda", 0)).copy_(torch.randn((m, n), device="cuda", generator=g) * std)  # noqa: E731
    x, r, dy, dh = rows(M, K), rows(M, K), rows(M, N), rows(M, K)
    w = mx._empty_rows(N, K, torch.float32, x.device).copy_(torch.randn((N, K), device="cuda", generator=g) * 0.05)
    gain = (1 + 0.1 * torch.randn((K,), device="cuda", generator=g)).to(torch.bfloat16)
    h, y, rstd = rows(M, K), rows(M, K), torch.empty((M,), device="cuda")
    up = lambda n: -(-n // 128) * 128  # noqa: E731

    # forward: norm and cast in one call, product with the weight's tiles
    xe, xs = mx.mx_rmsnorm_b128(x, gain, EPS, E4M3, residual=r, h_out=h, y_out=y, rstd_out=rstd)
    we, ws = mx.mx_quantize_b128(w, 1, E4M3, tile=True)
    out = mx.mx_gemm_b128(xe, xs, E4M3, we, ws, E4M3, up(K), dtype=torch.bfloat16)
    whole = lambda e, s, fmt, tile=False: mx.mx_dequantize_b128(e, s, fmt, e.shape[0], e.shape[1], 1, tile=tile).double()  # noqa: E731  (with the fill)
    a, b = whole(xe, xs, E4M3), whole(we, ws, E4M3, True)
    near(out, a @ b.T.contiguous(), cut_of(a, b), "forward")

    # the gradient that reaches the norm, through the transposed weight's tiles, and the norm's own
    ge, gs = mx.mx_quantize_b128(dy, 1, E5M2)
    te, ts = mx.mx_quantize_b128(w, 0, E4M3, tile=True)
    dn = mx.mx_gemm_b128(ge, gs, E5M2, te, ts, E4M3, up(N), dtype=torch.bfloat16, out=rows(M, K))
    a, b = whole(ge, gs, E5M2), whole(te, ts, E4M3, True)
    near(dn, a @ b.T.contiguous(), cut_of(a, b), "gradient of the input")
    dx, dgain = mx.mx_rmsnorm_bwd(dn, h, gain, rstd, dh=dh)
    hd = h.double().requires_grad_(True)
    gd = gain.double().requires_grad_(True)
    yd = hd * gd / (hd.square().mean(1, keepdim=True) + EPS).sqrt()
    yd.backward(dn.double())
    want = hd.grad + dh.double()
    scale = (dn.double() * gain.double()).abs().amax(1, keepdim=True) * rstd.double()[:, None] * 2 + want.abs()
    assert bool(((dx.double() - want).abs() <= want.abs() * 2.0 ** -8 + scale * 2.0 ** -16).all())
    assert float((dgain.double() - gd.grad).norm() / gd.grad.norm()) <= 2.0 ** -18
    assert bool(((y.double() - yd.detach()).abs() <= yd.detach().abs() * (2.0 ** -8 + 2.0 ** -18) + 2.0 ** -120).all())

    # the weight's gradient: both operands along the tokens
    ce, cs = mx.mx_quantize_b128(dy, 0, E5M2)
    ye, ys = mx.mx_quantize_b128(y, 0, E4M3)
    dw = mx.mx_gemm_b128(ce, cs, E5M2, ye, ys, E4M3, up(M))
    a, b = whole(ce, cs, E5M2), whole(ye, ys, E4M3)
    want = a @ b.T.contiguous()
    assert bool(((dw.double() - want).abs() <= cut_of(a, b) + want.abs() * 2.0 ** -24).all())


def test_decoding_step_captured(mx):
    """Norm, MX product and 128-element product of a few tokens, captured once and replayed on new tokens, the stream updated in place."""
    g = torch.Generator(device="cuda").manual_seed(5)
    M, K, N = 3, 512, 768
    wm = mx.mx_quantize(torch.randn((N, K), device="cuda", generator=g), 1, 0)
    wb = mx.mx_quantize_b128(torch.randn((N, K), device="cuda", generator=g), 1, 0, tile=True)
    gain = torch.ones((K,), device="cuda", dtype=torch.bfloat16)
    stream, add = (torch.randn((M, K), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))

    def step(h, dx):
        e, s = mx.mx_rmsnorm_q(dx, gain, EPS, 0, residual=h, h_out=h)
        a = mx.mx_gemm(e, s, 0, *wm, 0, K, dtype=torch.bfloat16)
        e, s = mx.mx_rmsnorm_b128(h, gain, EPS, 0)
        return a, mx.mx_gemm_b128(e, s, 0, *wb, 0, K, dtype=torch.bfloat16)

    step(stream.clone(), add)
    torch.cuda.synchronize()
    held = stream.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(held, add)
    held.copy_(stream)
    eager = stream.clone()
    for k in range(4):
        add.copy_(torch.randn((M, K), device="cuda", generator=g).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        want = step(eager, add)
        assert torch.equal(held, eager) and all(torch.equal(a, b) for a, b in zip(outs, want)), k


@pytest.mark.parametrize("axis,tile", [(1, False), (1, True), (0, False), (0, True)])
def test_casts_beyond_32_bits(mx, axis, tile):
    """More than 2^32 bytes: the last blocks as those of a tensor of their own."""
    rows, cols = 70016, 33024
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda").normal_()
    e, s = mx.mx_quantize_b128(x, axis, E4M3, tile=tile)
    r0, c0 = rows - 384, cols - 384
    part = x[r0:, c0:].contiguous()
    pe, ps = mx.mx_quantize_b128(part, axis, E4M3, tile=tile)
    l0, b0 = (r0, c0) if axis == 1 else (c0, r0)
    assert torch.equal(e[l0:, b0:], pe) and torch.equal(s[l0 // (128 if tile else 1):, b0 // 128:], ps)
    v = mx.mx_dequantize_b128(e, s, E4M3, rows, cols, axis, tile=tile, dtype=torch.bfloat16)
    assert torch.equal(v[r0:, c0:], mx.mx_dequantize_b128(pe, ps, E4M3, 384, 384, axis, tile=tile, dtype=torch.bfloat16))
    assert torch.equal(v[:64, :128], mx.mx_dequantize_b128(*mx.mx_quantize_b128(x[:128, :128].contiguous(), axis, E4M3, tile=tile), E4M3, 128, 128, axis, tile=tile, dtype=torch.bfloat16)[:64])


def test_norms_beyond_32_bits(mx):
    rows, cols = 300000, 8192
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda").normal_()
    w = torch.randn((cols,), device="cuda")
    h, rstd = torch.empty_like(x), torch.empty((rows,), device="cuda")
    e, s = mx.mx_rmsnorm_b128(x, w, EPS, E4M3, residual=x, h_out=h, rstd_out=rstd)
    part = x[-50:].clone()                            # (the gradient below is written over x)
    ph, pr = torch.empty_like(part), torch.empty((50,), device="cuda")
    pe, ps = mx.mx_rmsnorm_b128(part, w, EPS, E4M3, residual=part, h_out=ph, rstd_out=pr)
    assert torch.equal(e[-50:], pe) and torch.equal(s[-50:], ps) and torch.equal(h[-50:], ph) and torch.equal(rstd[-50:], pr)
    dx, _ = mx.mx_rmsnorm_bwd(x, h, w, rstd, dx_out=x)
    want, _ = mx.mx_rmsnorm_bwd(part, ph, w, pr)
    assert torch.equal(dx[-50:], want)


@pytest.mark.parametrize("M,N,K", [(70016, 33000, 512), (8, 70016, 65536), (24, 70016, 65536), (100, 70016, 65536), (70016, 200, 65536), (3, 200, 1 << 25), (100, 200, 1 << 25), (520, 530, 1 << 24)], ids=str)
def test_products_beyond_32_bits(mx, M, N, K):
    """C or an operand beyond 2^32 bytes, K beyond the tiles' offsets: the last entries, of numbers whose sums are exact."""
    g = torch.Generator(device="cuda").manual_seed(K)
    codes = torch.tensor([0, 0, 0, 0x38, 0xB8, 0x40], dtype=torch.uint8, device="cuda")          # 0, 1, -1, 2

    def operand(rows):
        e = torch.randint(0, 6, (rows, K // 64), generator=g, device="cuda", dtype=torch.int32)
        e = codes[e].repeat_interleave(64, 1)
        e[-1, -1] = 0x38
        return e, torch.ones((rows, K // 128), device="cuda")

    a, b = operand(M), operand(N)
    out = mx.mx_gemm_b128(*a, E4M3, *b, E4M3, K, dtype=torch.bfloat16)
    ra, rb = max(0, M - 30), max(0, N - 40)
    fa, fb = (t.view(torch.float8_e4m3fn).float().double() for t in (a[0][ra:], b[0][rb:]))
    assert torch.equal(out[ra:, rb:], (fa @ fb.T.contiguous()).float().to(torch.bfloat16))
