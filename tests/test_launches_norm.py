"""The kernels that the norms and the 128-element forms take at the borders of their rules, and the scratch memory they ask for (no GPU)."""
import pytest

import launches

P = 0x1000                                    # any aligned address
F32, BF16 = 0, 1
E4M3, E5M2 = 0, 1


@pytest.fixture(scope="module")
def trace(tmp_path_factory):
    so = launches.build(str(tmp_path_factory.mktemp("runtime")))
    return lambda calls: launches.trace(so, [(n, a, 0) for n, a in calls])


def one(trace, *call):
    (status, seen), = trace([call])
    assert status == 0, status
    return seen


def grids_fit(seen):
    return all(k[0] == "alloc" or (k[2][0] * k[3] < 1 << 32 and k[2][1] <= 65535) for k in seen)


def product(M, N, K, tb=1, fa=E4M3, fb=E4M3, dt=BF16):
    return "mx_gemm_b128", (M, N, K, P, P, 0, fa, P, P, tb, fb, P, dt, N, 0)


def form(trace, *args, **kw):
    seen = one(trace, *product(*args, **kw))
    assert len(seen) == 1 and grids_fit(seen)
    name, t = seen[0][:2]
    return (name, *[int(v) for v in t[4:]])


FEW, TILE, PLAIN = "gemm128_few_kernel", "gemm128_tile_kernel", "gemm128_kernel"
T256, T2X1, T128 = (TILE, 4, 8, 4, 2, 1), (TILE, 4, 4, 4, 2, 1), (TILE, 4, 4, 2, 2, 2)


def test_forms_of_the_product(trace):
    assert form(trace, 1, 4096, 4096) == form(trace, 16, 16383, 4096) == form(trace, 16, 1, 128) == (FEW, 1, 1, 4)
    assert form(trace, 16, 16384, 4096) == (FEW, 1, 4, 2)
    # one round of work-groups over 256 compute units, of the smallest that give one
    assert form(trace, 17, 2048, 4096) == form(trace, 64, 1024, 128) == form(trace, 256, 256, 1 << 24) == form(trace, 4096, 16, 4096) == (FEW, 1, 1, 4)
    assert form(trace, 17, 2049, 4096) == form(trace, 17, 4096, 4096) == form(trace, 128, 1024, 128) == form(trace, 4096, 32, 4096) == (FEW, 2, 1, 4)
    assert form(trace, 17, 4097, 4096) == form(trace, 32, 8192, 4096) == form(trace, 64, 4096, 128) == form(trace, 512, 512, 4096) == form(trace, 8192, 32, 4096) == (FEW, 2, 2, 2)
    assert form(trace, 17, 8193, 4096) == form(trace, 32, 1 << 20, 128) == (FEW, 2, 4, 2)
    for tb in (0, 1):
        assert form(trace, 33, 8191, 4096, tb) == form(trace, 512, 513, 4096, tb) == form(trace, 65, 4096, 4096, tb) == form(trace, 1000, 4096, 4096, tb) == T128
        assert form(trace, 512, 11008, 4096, tb) == form(trace, 2048, 4096, 4096, tb) == T2X1
        assert form(trace, 8192, 11008, 4096, tb) == form(trace, 4096, 4096, 4096, tb) == form(trace, 1000, 11008, 4096, tb) == T256
    # halves of K want at least four blocks each, and as many in the one as in the other
    assert form(trace, 128, 4096, 1024) == T128
    assert form(trace, 128, 4096, 1024 - 128) == form(trace, 128, 4096, 1024 + 128) == form(trace, 128, 4096, 512) == T2X1
    # less than four blocks, or a K that 32-bit offsets of 256 rows do not reach
    assert form(trace, 128, 4096, 384) == form(trace, 4096, 4096, 128) == form(trace, 128, 4096, 1 << 24) == (PLAIN, 4, 4, 2, 2)
    assert form(trace, 128, 4096, (1 << 24) - 256) == T128


def test_formats_and_types_of_the_product(trace):
    for fa in (E4M3, E5M2):
        for fb in (E4M3, E5M2):
            for dt in (F32, BF16):
                for tb in (0, 1):
                    seen = one(trace, *product(600, 500, 1024, tb, fa, fb, dt))
                    assert seen[0][1][:4] == (str(fa), str(fb), str(dt), "false" if tb else "true")


def test_largest_grids(trace):
    for M, N in ((1 << 19, 1 << 18), (1, (1 << 27) - 16), (64, 8191), (1 << 22, 128)):
        assert grids_fit(one(trace, *product(M, N, 512)))
    for rows, cols, axis, tile in ((1 << 20, 1 << 14, 0, 0), (1 << 20, 1 << 14, 1, 1), (1 << 22, 1 << 14, 1, 0), (1, 1 << 33, 1, 0)):
        assert grids_fit(one(trace, "mx_quantize_b128", (P, BF16, rows, cols, cols, axis, tile, E4M3, P, P, 0)))
        assert grids_fit(one(trace, "mx_dequantize_b128", (P, P, E4M3, rows, cols, axis, tile, P, BF16, cols, 0)))


def test_long_runs_of_rows_take_several_launches(trace):
    units = 1 << 31                                     # a launch numbers 16-byte pieces with 31 bits
    rows, cols = 1 << 20, 1 << 15
    seen = one(trace, "mx_quantize_b128", (P, F32, rows, cols, cols, 1, 0, E4M3, P, P, 0))
    assert {k[0] for k in seen} == {"cast128_row_kernel"} and len(seen) == -(-rows * cols // 4 // units) + 1
    assert sum(k[2][0] for k in seen) * 1024 >= rows * cols // 4


@pytest.fixture(scope="module")
def norm_calls():
    """The norm takes a Float32 argument, which the stand-alone process cannot pass: the gradients, which have none, stand for both."""
    def bwd(rows, cols, dt=BF16, dw=P, ws=0, wb=0):
        return "mx_rmsnorm_bwd_ws", (P, cols, P, cols, P, F32, P, P, cols, dt, rows, cols, P, cols, dw, ws, wb, 0)
    return bwd


def test_gradients(trace, norm_calls):
    def names(seen):
        return [k[0] if k[0] == "alloc" else (k[0], *k[1][1:]) for k in seen]
    one_vector, two, wave = ("norm_bwd_kernel", "1", "false"), ("norm_bwd_kernel", "2", "false"), ("norm_bwd_kernel", "1", "true")
    for cols, kernel, threads in ((8, wave, 256), (512, wave, 256), (520, one_vector, 128), (4096, one_vector, 512), (8192, one_vector, 1024), (8200, two, 576), (16384, two, 1024)):
        seen = one(trace, *norm_calls(5000, cols))
        assert names(seen) == ["alloc", kernel, ("norm_bwd_weight_kernel",)] and seen[1][3] == threads, cols
        lines = seen[1][2][0]
        assert seen[0][1] >= lines * cols * 4 and lines <= 1024
        assert names(one(trace, *norm_calls(5000, cols, dw=0))) == [kernel]
        need = seen[0][1]
        assert names(one(trace, *norm_calls(5000, cols, ws=P, wb=need))) == [kernel, ("norm_bwd_weight_kernel",)]
    seen = one(trace, *norm_calls(70, 16392))
    assert names(seen) == ["alloc", ("norm_bwd_long_weight_kernel",), ("norm_bwd_long_kernel",), ("norm_bwd_weight_kernel",)]
    assert names(one(trace, *norm_calls(0, 64))) == [("norm_bwd_weight_kernel",)]
    seen = one(trace, *norm_calls((1 << 24) + 5, 16392, dw=0))
    assert len(seen) == 2 and grids_fit(seen) and sum(k[2][0] for k in seen) == (1 << 24) + 5


def test_gradients_of_very_wide_rows(trace, norm_calls):
    for cols in ((1 << 26) - 8, 1 << 26, (1 << 30) + 8):
        for rows in (0, 3):
            seen = one(trace, *norm_calls(rows, cols))
            assert grids_fit(seen)
            assert sum(k[2][0] for k in seen if k[0] == "norm_bwd_weight_kernel") * 16 >= cols
