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
