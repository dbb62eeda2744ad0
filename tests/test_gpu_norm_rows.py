"""Norms of rows with NaN, infinities and zeros, code for code; the gradients' C entry with a workspace; the weight's gradient beyond 32-bit offsets."""
import numpy as np
import pytest
import torch

import b128_model as model
from gpu_util import to_host

pytestmark = pytest.mark.gpu
EPS = 1e-5
B128 = 6


@pytest.fixture(scope="module")
def mx():
    from paper_2310_10537_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.lib()
    return binding


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(5, 129), (7, 1000), (1030, 520), (4, 8200), (4, 16392)], ids=str)
def test_casts_of_rows_with_nan_and_infinity(mx, rows, cols, dt):
    """Every code and scale is that of the stand-alone cast of h * rstd in Float32 (NaN codes may differ in their sign)."""
    g = np.random.default_rng(cols)
    x = torch.from_numpy((g.standard_normal((rows, cols)) * np.exp(g.standard_normal((rows, 1)))).astype(np.float32))
    x[0] = 0
    x[1, cols // 2] = float("nan")
    x[2, cols - 1] = float("inf")
    x[2, 0] = float("-inf")
    x[3, 0], x[3, 1] = float("inf"), float("nan")
    wide = torch.full((rows, -(-cols // 8) * 8), 9.0, dtype=dt, device="cuda")[:, :cols]
    wide.copy_(x)
    rstd = torch.empty((rows,), device="cuda")
    mx.mx_rmsnorm(wide, None, EPS, rstd_out=rstd)
    rs = to_host(rstd)
    assert rs[0] == np.float32(1 / np.sqrt(np.float32(EPS))) or abs(rs[0] * np.sqrt(EPS) - 1) <= 2.0 ** -22
    assert np.isnan(rs[1]) and rs[2] == 0 and np.isnan(rs[3])
    with np.errstate(invalid="ignore"):
        y = wide.float().cpu().numpy() * rs[:, None]
    assert np.isnan(y[2, [0, cols - 1]]).all() and not y[2, 1:-1].any()
    plain = torch.zeros((rows, -(-cols // 4) * 4), device="cuda")[:, :cols]
    plain.copy_(torch.from_numpy(y))
    for kind in range(8):
        for rnd in (0, 1, 2) if kind < B128 else (0,):
            if kind >= B128:
                e, s = mx.mx_rmsnorm_b128(wide, None, EPS, kind - B128)
                we, ws = mx.mx_quantize_b128(plain, 1, kind - B128)
            else:
                e, s = mx.mx_rmsnorm_q(wide, None, EPS, kind, rnd)
                we, ws = mx.mx_quantize(plain, 1, kind, rnd)
            assert torch.equal(s.view(torch.uint8), ws.view(torch.uint8)), (kind, rnd)
            if kind in (0, 1, B128, B128 + 1):
                assert model.same_codes(to_host(e), to_host(we), kind % B128), (kind, rnd)
            else:
                assert torch.equal(e, we), (kind, rnd)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(1, 8), (70, 512), (700, 1000), (300, 8200), (20, 20000)], ids=str)
def test_gradients_with_a_workspace_on_another_stream(mx, rows, cols, dt):
    """The same bits as without one, from a workspace of exactly the size asked for that holds garbage; a smaller one is refused."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    dy, h, dh = (torch.randn((rows, cols), device="cuda", generator=g).to(dt) for _ in range(3))
    w, rstd = torch.randn((cols,), device="cuda", generator=g), torch.rand((rows,), device="cuda", generator=g) + 0.5
    want = mx.mx_rmsnorm_bwd(dy, h, w, rstd, dh=dh)
    need = mx.lib().mx_rmsnorm_bwd_workspace_bytes(rows, cols)
    room = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    dx, dw = torch.full_like(dy, 7.0), torch.full((cols,), 7.0, device="cuda")
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())

    def call(size):
        return mx.lib().mx_rmsnorm_bwd_ws(dy.data_ptr(), cols, h.data_ptr(), cols, w.data_ptr(), mx.DT_F32, rstd.data_ptr(), dh.data_ptr(), cols, mx._dt(dy), rows, cols,
                                          dx.data_ptr(), cols, dw.data_ptr(), room.data_ptr(), size, st.cuda_stream)

    assert call(need - 1) == mx.MX_ERR_WORKSPACE
    st.synchronize()
    assert bool((dx == 7).all()) and bool((dw == 7).all())
    assert call(need) == mx.MX_OK
    st.synchronize()
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and bool((room[need:] == 0xA5).all())


def test_gradient_of_the_weight_beyond_32_bits(mx):
    """300000 rows of 8192: 256 lines of 1172 rows each at most, one after the other, then four lines and ten joins; xhat and its product rounded once each."""
    rows, cols = 300000, 8192
    g = torch.Generator(device="cuda").manual_seed(2)
    dy, h = (torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    rstd = torch.rand((rows,), device="cuda", generator=g) + 0.5
    _, dw = mx.mx_rmsnorm_bwd(dy, h, None, rstd)
    want, size = torch.zeros((cols,), dtype=torch.float64, device="cuda"), torch.zeros((cols,), dtype=torch.float64, device="cuda")
    for r in range(0, rows, 20000):
        term = dy[r:r + 20000].double() * (h[r:r + 20000].double() * rstd[r:r + 20000, None].double())
        want += term.sum(0)
        size += term.abs().sum(0)
    assert bool(((dw.double() - want).abs() <= size * (1172 + 14 + 2) * 2.0 ** -24).all())
    # the roundings are independent: a chain of n of them adds up to the square root of n / 2 (its sums grow with the square root of their length)
    assert float((dw.double() - want).norm() / want.norm()) <= (1172 / 2 + 16) ** 0.5 * 2.0 ** -24
