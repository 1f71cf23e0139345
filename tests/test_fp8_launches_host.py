"""Host-only checks of what the 8-bit operators and the block norms launch at the ends of the extents that they take: a grid
dimension of 2^32 threads or more is cut short without an error, so none may be launched."""
import ctypes

import pytest

import paper_2511_03586_amd as perf
from tests import launches as L
from tests.fp8_helpers import up

FAKE = 1 << 40  # a 16-byte aligned device address; never dereferenced
F32, BF16, E4M3, E5M2 = perf.PERF_F32, perf.PERF_BF16, perf.PERF_E4M3, perf.PERF_E5M2
MOST = 1 << 30  # rows and columns


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    return L.build_recorder(str(tmp_path_factory.mktemp("recorder")))


def _check_grids(results):
    for r in results:
        assert r["status"] == perf.PERF_OK and r["launches"]
        for l in r["launches"]:
            for n, threads in zip(l["grid"], l["block"]):
                assert 0 < n * threads < 1 << 32, l
            assert l["grid"][1] <= 65535 and l["grid"][2] <= 65535, l


def _quantize(rows, cols, row, transposed, block_rows=1, x_dt=BF16, q_dt=E4M3):
    return ("perf_quantize_fp8", dict(x=FAKE, q=FAKE if row else None, scales=FAKE if row else None, qt=FAKE if transposed else None,
                                      scales_t=FAKE if transposed else None, rows=rows, cols=cols, ldx=cols, ldq=cols, lds=up(cols),
                                      ldqt=rows, ldst=up(rows), block_rows=block_rows, x_dt=x_dt, q_dt=q_dt))


# x of at most 2^37 elements; around the numbers of blocks that a launch holds, and at the ends
QUANTIZE = [(rows, cols) for cols in (1, 128, 129, 300, 3000, 3968, 3969, 1 << 16, 1 << 23, MOST)
            for rows in sorted({1, 127, 128, *(min(MOST, max(1, ((1 << 29) - d) // up(cols))) for d in (65, 33, 32, 31, 1, 0, -1, -33)),
                                min(MOST, (1 << 37) // cols)}) if rows * cols <= 1 << 37]


def test_quantize_grids(recorder):
    for row, transposed, block_rows in ((True, False, 1), (False, True, 1), (True, True, 1), (True, False, 128), (True, True, 128)):
        _check_grids(L.record(recorder, [_quantize(r, c, row, transposed, block_rows) for r, c in QUANTIZE]))


def test_quantize_rows_are_all_launched(recorder):
    """The launches of a call take up each other's rows, and every block of a row has its eight lanes."""
    for (rows, cols), r in zip(QUANTIZE, L.record(recorder, [_quantize(r, c, True, False) for r, c in QUANTIZE], "quantize_rows_kernel", 4)):
        done = 0
        for l in r["launches"]:
            x, q, scales, items = l["args"]
            assert x == FAKE + done * cols * 2 and q == FAKE + done * cols and scales == FAKE + done * up(cols) * 4
            assert items % (8 * up(cols)) == 0 and l["grid"][0] * l["block"][0] >= items > 0
            done += items // (8 * up(cols))
        assert done == rows, (rows, cols)


def _norm(rows, cols, gate_rows, x_dt, y_dt):
    return ("perf_residual_norm", dict(u=FAKE, x=FAKE, gate=FAKE if gate_rows else None, gamma_post=FAKE, gamma_pre=FAKE, h=FAKE, y=FAKE,
                                       y_scales=FAKE, rrms_post=FAKE, rrms_pre=FAKE, rows=rows, cols=cols, ldu=cols, ldx=cols, ldg=cols,
                                       gate_rows=gate_rows, ldh=cols, ldy=cols, lds=up(cols), residual_scale=1.0, eps=1e-5, x_dt=x_dt,
                                       y_dt=y_dt))


def _norm_gradient(rows, cols, gate_rows, x_dt):
    gate = FAKE if gate_rows else None
    return ("perf_residual_norm_backward", dict(dy=FAKE, dh=FAKE, h=FAKE, u=FAKE, gate=gate, gamma_post=FAKE, gamma_pre=FAKE, rrms_post=FAKE,
                                                rrms_pre=FAKE, dx=FAKE, du=FAKE, dgate=gate, dgamma_post=FAKE, dgamma_pre=FAKE,
                                                workspace=FAKE, rows=rows, cols=cols, lddy=cols, lddh=cols, ldh=cols, ldu=cols, ldg=cols,
                                                gate_rows=gate_rows, lddx=cols, lddu=cols, lddg=cols, residual_scale=1.0, x_dt=x_dt))


# rows of every number of waves, and those that are not held in registers, to the ends
NORMS = [(rows, cols) for cols in (1, 7, 8, 512, 513, 4096, 16384, 16385, 1 << 20, (1 << 28) - 64, (1 << 28) - 63, 1 << 28, MOST)
         for rows in (1, 2, 255, 256, 257, 4097, 1 << 20, MOST) if rows * cols <= 1 << 37]


def test_norm_grids(recorder):
    _check_grids(L.record(recorder, [_norm(r, c, g, dt, y) for r, c in NORMS for g in (0, 1, 16, 1000, r)
                                     for dt, y in ((BF16, E4M3), (F32, F32))]))


def test_norm_gradient_grids(recorder):
    _check_grids(L.record(recorder, [_norm_gradient(r, c, g, dt) for r, c in NORMS for g in (0, 1, 16, 1000, r) for dt in (BF16, F32)]))


def test_norm_gradient_sums_of_all_columns_are_launched(recorder):
    """64 columns to a workgroup; a launch takes up where the one before it ends."""
    for (rows, cols), r in zip(NORMS, L.record(recorder, [_norm_gradient(r, c, 0, BF16) for r, c in NORMS], "residual_norm_sums_kernel", 5)):
        done = 0
        for l in r["launches"]:
            if "residual_norm_sums_kernel" in l["name"]:
                assert ctypes.c_int32(l["args"][4]).value == done
                done += l["grid"][0] * 64
        assert done == up(cols, 64) * 64 or (done == 0 and len(r["launches"]) == 1), (rows, cols)


def _gemm(m, n, k, batch, b_rows, a_dt, c_dt):
    return ("perf_gemm_fp8", dict(A=FAKE, scaleA=FAKE, B=FAKE, scaleB=FAKE, C=FAKE, M=m, N=n, K=k, lda=up(k, 16) * 16, ldsa=up(k),
                                  ldb=up(k, 16) * 16, ldsb=up(k), ldc=n, b_block_rows=b_rows, batch=batch, strideC=m * n, a_dt=a_dt,
                                  c_dt=c_dt))


def test_gemm_grids(recorder):
    """Every product is launched, unless its tiles of 128 x 128 are more than a launch holds: then none is."""
    extents = (1, 16, 17, 33, 65, 128, 129, 300, 4096, 1 << 16, 1 << 23, (1 << 27) + 1, MOST)
    calls = [_gemm(m, n, k, batch, b_rows, a_dt, c_dt) for m in extents for n in extents for k in (1, 300, 1500, 8000)
             for batch in (1, 70000) if m * n * batch <= 1 << 56 for b_rows, a_dt, c_dt in ((1, E4M3, F32), (128, E5M2, BF16), (128, E4M3, F32))]
    refused = 0
    for (_, a), r in zip(calls, L.record(recorder, calls)):
        if r["status"] == perf.PERF_ERR_UNSUPPORTED:
            assert up(a["M"], 128) * up(a["N"], 128) * 256 >= 1 << 32 and not r["launches"], a
            refused += 1
        else:
            _check_grids([r])
    assert refused < len(calls) // 4
