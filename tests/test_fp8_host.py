"""Host-only checks of the 8-bit operators' and the block norms' arguments: what the header refuses is refused before a device
is touched (no call here gets as far), and the workspace's size is that of its documentation."""
import os

import pytest

import paper_2511_03586_amd as perf

FAKE = 0x10000  # a non-null, 16-byte aligned device address; never dereferenced
NULL, SHAPE, DTYPE, ALIGN, UNSUPPORTED = (perf.PERF_ERR_NULL, perf.PERF_ERR_SHAPE, perf.PERF_ERR_DTYPE, perf.PERF_ERR_ALIGN,
                                          perf.PERF_ERR_UNSUPPORTED)
F32, BF16, E4M3, E5M2 = perf.PERF_F32, perf.PERF_BF16, perf.PERF_E4M3, perf.PERF_E5M2
HUGE = 1 << 60  # a row stride whose second row has no offset of 63 bits


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(perf.LIB_PATH):
        from paper_2511_03586_amd import build
        build.build(verbose=False)


def _refuses(call, base, cases):
    for changes, status in cases:
        assert call(**{**base, **changes}, check=False) == status, changes


def test_quantize_refuses():
    base = dict(x=FAKE, q=FAKE, scales=FAKE, qt=FAKE, scales_t=FAKE, rows=300, cols=200, ldx=200, ldq=208, lds=2, ldqt=304, ldst=3,
                block_rows=1, x_dt=BF16, q_dt=E4M3)
    _refuses(perf.perf_quantize_fp8, base, [
        (dict(x=None), NULL), (dict(q=None), NULL), (dict(scales=None), NULL), (dict(qt=None), NULL), (dict(scales_t=None), NULL),
        (dict(q=None, scales=None, qt=None, scales_t=None), NULL),
        (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(rows=-1), SHAPE), (dict(rows=(1 << 30) + 1, ldqt=1 << 31, ldst=1 << 31), SHAPE),
        (dict(cols=(1 << 30) + 1, ldx=1 << 31, ldq=1 << 31, lds=1 << 31), SHAPE),
        (dict(ldx=199), SHAPE), (dict(ldq=199), SHAPE), (dict(lds=1), SHAPE), (dict(ldqt=299), SHAPE), (dict(ldst=2), SHAPE),
        (dict(ldx=HUGE), SHAPE), (dict(ldq=HUGE), SHAPE), (dict(ldqt=HUGE), SHAPE), (dict(lds=HUGE), SHAPE), (dict(ldst=HUGE), SHAPE),
        (dict(block_rows=0), SHAPE), (dict(block_rows=64), SHAPE),
        (dict(x_dt=E4M3), DTYPE), (dict(x_dt=9), DTYPE), (dict(q_dt=BF16), DTYPE), (dict(q_dt=-1), DTYPE),
        (dict(x=FAKE + 1), ALIGN), (dict(x=FAKE + 2, x_dt=F32), ALIGN), (dict(scales=FAKE + 2), ALIGN), (dict(scales_t=FAKE + 1), ALIGN),
    ])
    with pytest.raises(perf.PerfError):
        perf.perf_quantize_fp8(**{**base, "x": None})


def test_gemm_refuses():
    base = dict(A=FAKE, scaleA=FAKE, B=FAKE, scaleB=FAKE, C=FAKE, M=40, N=70, K=300, lda=304, ldsa=3, ldb=304, ldsb=3, ldc=70,
                b_block_rows=1, a_dt=E4M3, b_dt=E4M3, c_dt=BF16)
    two = dict(batch=2, strideA=40 * 304, strideSA=120, strideB=70 * 304, strideSB=210, strideC=2800)
    _refuses(perf.perf_gemm_fp8, base, [
        *((dict([(k, None)]), NULL) for k in ("A", "scaleA", "B", "scaleB", "C")),
        *((dict([(k, v)]), SHAPE) for k in ("M", "N", "K") for v in (0, -3, (1 << 30) + 1)),
        (dict(batch=0), SHAPE), (dict(lda=288), SHAPE), (dict(ldb=288), SHAPE), (dict(ldsa=2), SHAPE), (dict(ldsb=2), SHAPE),
        (dict(ldc=69), SHAPE), (dict(ldc=HUGE), SHAPE), (dict(lda=HUGE), SHAPE), (dict(ldsb=HUGE), SHAPE), (dict(b_block_rows=2), SHAPE),
        (dict(alpha=float("nan")), SHAPE), (dict(alpha=float("inf")), SHAPE),
        ({**two, "strideA": -16}, SHAPE), ({**two, "strideSB": -1}, SHAPE), ({**two, "strideC": 2799}, SHAPE),
        ({**two, "strideC": 1 << 61}, SHAPE), ({**two, "strideB": 1 << 60}, SHAPE),
        (dict(a_dt=BF16), DTYPE), (dict(b_dt=F32), DTYPE), (dict(c_dt=E4M3), DTYPE), (dict(c_dt=4), DTYPE),
        (dict(A=FAKE + 8), ALIGN), (dict(B=FAKE + 1), ALIGN), (dict(scaleA=FAKE + 2), ALIGN), (dict(scaleB=FAKE + 1), ALIGN),
        (dict(C=FAKE + 1), ALIGN), (dict(C=FAKE + 2, c_dt=F32), ALIGN),
        (dict(b_dt=E5M2), UNSUPPORTED), (dict(lda=300), UNSUPPORTED), (dict(ldb=312), UNSUPPORTED), (dict(lda=1 << 23), UNSUPPORTED),
        (dict(ldb=1 << 23), UNSUPPORTED), (dict(ldsa=1 << 23), UNSUPPORTED), (dict(ldsb=1 << 23), UNSUPPORTED),
        ({**two, "strideA": 40 * 304 + 8}, UNSUPPORTED), ({**two, "strideB": 4}, UNSUPPORTED),
        (dict(M=1 << 30, N=1 << 29, ldc=1 << 29), UNSUPPORTED),
    ])


def test_norm_refuses():
    base = dict(u=FAKE, x=FAKE, gate=FAKE, gamma_post=FAKE, gamma_pre=FAKE, h=FAKE, y=FAKE, y_scales=FAKE, rrms_post=FAKE,
                rrms_pre=FAKE, rows=10, cols=200, ldu=200, ldx=200, ldg=200, gate_rows=10, ldh=200, ldy=208, lds=2,
                residual_scale=1.0, eps=1e-5, x_dt=BF16, gate_dt=F32, param_dt=F32, y_dt=E4M3)
    _refuses(perf.perf_residual_norm, base, [
        (dict(u=None), NULL), (dict(x=None), NULL), (dict(h=None, y=None), NULL), (dict(gamma_pre=None), NULL), (dict(y_scales=None), NULL),
        (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(rows=(1 << 30) + 1), SHAPE), (dict(cols=(1 << 30) + 1), SHAPE),
        *((dict([(k, 199)]), SHAPE) for k in ("ldu", "ldx", "ldg", "ldh", "ldy")), (dict(lds=1), SHAPE),
        *((dict([(k, HUGE)]), SHAPE) for k in ("ldu", "ldx", "ldg", "ldh", "ldy", "lds")),
        (dict(gate_rows=0), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE),
        (dict(residual_scale=float("inf")), SHAPE), (dict(residual_scale=float("nan")), SHAPE),
        (dict(x_dt=E4M3), DTYPE), (dict(gate_dt=E5M2), DTYPE), (dict(param_dt=7), DTYPE), (dict(y_dt=-2), DTYPE),
        (dict(u=FAKE + 1), ALIGN), (dict(x=FAKE + 1), ALIGN), (dict(h=FAKE + 1), ALIGN), (dict(gate=FAKE + 2), ALIGN),
        (dict(gamma_post=FAKE + 2), ALIGN), (dict(gamma_pre=FAKE + 2), ALIGN), (dict(rrms_post=FAKE + 2), ALIGN),
        (dict(rrms_pre=FAKE + 2), ALIGN), (dict(y_scales=FAKE + 2), ALIGN), (dict(y_dt=BF16, y=FAKE + 1), ALIGN),
        (dict(y_dt=F32), UNSUPPORTED), (dict(y_dt=E5M2), UNSUPPORTED),
    ])


def test_norm_gradient_refuses():
    ld = dict((k, 200) for k in ("lddy", "lddh", "ldh", "ldu", "ldg", "lddx", "lddu", "lddg"))
    base = dict(dy=FAKE, dh=FAKE, h=FAKE, u=FAKE, gate=FAKE, gamma_post=FAKE, gamma_pre=FAKE, rrms_post=FAKE, rrms_pre=FAKE, dx=FAKE,
                du=FAKE, dgate=FAKE, dgamma_post=FAKE, dgamma_pre=FAKE, workspace=FAKE, rows=10, cols=200, gate_rows=10, **ld,
                residual_scale=1.0, x_dt=BF16, gate_dt=F32, param_dt=F32)
    _refuses(perf.perf_residual_norm_backward, base, [
        (dict(dy=None, dh=None), NULL), *((dict([(k, None)]), NULL) for k in ("u", "dx", "du", "workspace", "h", "gamma_pre", "rrms_pre",
                                                                             "rrms_post", "gate", "gamma_post", "dy")),
        (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(rows=(1 << 30) + 1), SHAPE), (dict(cols=(1 << 30) + 1), SHAPE),
        *((dict([(k, v)]), SHAPE) for k in ld for v in (199, HUGE)),
        (dict(gate_rows=0), SHAPE), (dict(residual_scale=float("nan")), SHAPE),
        (dict(x_dt=E4M3), DTYPE), (dict(gate_dt=2), DTYPE), (dict(param_dt=3), DTYPE),
        *((dict([(k, FAKE + 1)]), ALIGN) for k in ("dy", "dh", "h", "u", "dx", "du")),
        *((dict([(k, FAKE + 2)]), ALIGN) for k in ("gate", "dgate", "gamma_post", "gamma_pre", "rrms_post", "rrms_pre", "dgamma_post",
                                                   "dgamma_pre", "workspace")),
    ])


def test_workspace_of_the_gradient():
    size = perf.perf_residual_norm_backward_workspace_bytes
    assert size(0, 8) == size(8, 0) == size(-1, 8) == size((1 << 30) + 1, 8) == size(8, (1 << 30) + 1) == -1
    for rows in (1, 15, 16, 255, 256, 257, 4000, 8192, 16384, 1 << 20, 1 << 30):
        for cols in (1, 7, 8, 512, 513, 4096, 8192, 8193, 16384, 16385, 1 << 20):
            need = size(rows, cols)
            # four rows of sums for each of up to 256 runs of rows; a mean for each row where a row is not held in registers
            assert 16 * cols <= need <= 16 * 256 * cols + (4 * rows if cols < 8 or cols > 16384 else 0)
            assert rows > 16384 or need <= size(16384, cols)  # no smaller for more rows
