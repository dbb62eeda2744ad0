"""The sums of dweight: how many roundings an entry passes through."""
import numpy as np
import pytest
import torch

import b128_model as model
from gpu_util import to_dev, to_host

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mx():
    from paper_2310_10537_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    binding.lib()
    return binding


# a row for each line of partial sums (or four, of rows that a wave holds), and a line or two for each of the sums that are joined last: powers of two
@pytest.mark.parametrize("rows,cols", [(64, 1000), (128, 520), (64, 8200), (64, 20000), (256, 512), (512, 40), (64, 16384)], ids=str)
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_equal_parts_are_joined_in_pairs(mx, rows, cols, dt):
    """Sums of 2, 4, 8 ... equal numbers do not round: the result is rows times one product.  (Added one after the other, three of them would.)"""
    g = np.random.default_rng(rows + cols)
    h = torch.from_numpy(g.standard_normal((1, cols)).astype(np.float32)).to(dt)
    rstd = np.float32(0.7)
    x = h.float().numpy()[0] * rstd                               # rounded to Float32
    h = h.cuda().expand(rows, cols).contiguous()
    dy = torch.ones((rows, cols), dtype=dt, device="cuda")
    _, dw = mx.mx_rmsnorm_bwd(dy, h, None, torch.full((rows,), float(rstd), device="cuda"))
    assert np.array_equal(to_host(dw), x * np.float32(rows))


def test_error_of_independent_terms(mx):
    """333 x 1000: 333 lines, six at most for each of 64 sums, which meet two by two.  The roundings are independent, each at most half a unit of what it
    rounds (mean square a third of that), and with T terms of variance v the squares of all rounded numbers add up to, in units of T v: products and
    xhat 2, the runs of up to six lines 64 (2 + 3 + 4 + 5 + 6) / 333 = 3.9 at most (in pairs less), six levels of pairs 6."""
    rows, cols = 333, 1000
    g = np.random.default_rng(7)
    dy, h = (g.standard_normal((rows, cols)).astype(np.float32) for _ in range(2))
    rstd = (0.5 + g.random(rows)).astype(np.float32)
    _, dw = mx.mx_rmsnorm_bwd(to_dev(dy), to_dev(h), None, to_dev(rstd))
    _, want = model.norm_backward(dy, h, None, rstd, None)
    error = np.linalg.norm(to_host(dw) - want) / np.linalg.norm(want)
    print("error", error)
    assert error <= np.sqrt((2 + 3.9 + 6) / 3) * 2.0 ** -24
