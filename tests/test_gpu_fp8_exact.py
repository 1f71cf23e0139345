"""GPU: the block-scaled 8-bit product with sums that no kernel may round, so that one lost or misplaced product shows, also in a
bf16 C."""
import numpy as np
import pytest
import torch

import paper_2511_03586_amd as perf
from tests import fp8_helpers as F

pytestmark = pytest.mark.gpu

F32, BF16, E4M3, E5M2 = perf.PERF_F32, perf.PERF_BF16, perf.PERF_E4M3, perf.PERF_E5M2
F8 = F.F8

# one row, a few and a tile's (waves that divide K, of each height and width); four stages; two; 256 x 256 (bf16 C); K from less
# than a block to more than the stages hold
SIZES = [(1, 40, 384), (1, 20000, 1100), (20, 9000, 1500), (50, 70, 257), (64, 11000, 2049), (300, 260, 4097), (700, 1500, 300),
         (1500, 1700, 2049), (513, 4100, 130), (2049, 2100, 515), (130, 16300, 700), (3700, 3601, 700), (2305, 4096, 77)]


def _check(a, sa, b, sb, b_rows, a_dt):
    ref, _ = F.gemm_ref(a.to(F8[a_dt]), sa, b.to(torch.float8_e4m3fn), sb, b_rows)
    for c_dt in (BF16, F32):
        c = F.run_gemm(a.to(F8[a_dt]), sa, b.to(torch.float8_e4m3fn), sb, b_rows, c_dt, a_dt=a_dt)
        assert np.array_equal(c, ref if c_dt == F32 else torch.from_numpy(ref).to(torch.bfloat16).double().numpy())


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("b_rows,a_dt", [(1, E5M2), (128, E4M3)])
def test_sums_that_fit_bf16(m, n, k, b_rows, a_dt):
    """Products of -1, 0 and 1, scales that are powers of two, one for a row: results are whole numbers of magnitude up to 256 times
    a power of two, which bf16 holds."""
    g = np.random.default_rng(m + n + k)
    a, b = (torch.from_numpy(g.integers(-1, 2, (rows, k)).astype(np.float32)) for rows in (m, n))
    whole = (a @ b.T).abs().max()
    assert whole <= 256
    sa = torch.from_numpy(2.0 ** g.integers(-8, 9, (m, 1))).float().repeat(1, F.up(k))
    sb = torch.from_numpy(2.0 ** g.integers(-8, 9, (F.up(n, b_rows), 1))).float().repeat(1, F.up(k))
    _check(a, sa, b, sb, b_rows, a_dt)


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("b_rows,a_dt", [(1, E4M3), (128, E5M2)])
def test_sums_that_fit_fp32(m, n, k, b_rows, a_dt):
    """Products of up to 16, scales of 2^-2 to 2^2 for each block: multiples of 2^-4 of magnitude up to 2^8 K <= 2^20.1, in any order;
    rounded once to bf16.  (Of eight products at once the instruction for bf16 C drops what lies below 2^-13 of the largest, which
    products of 1 to 16 do not.)"""
    g = np.random.default_rng(m + n + k + 1)
    a, b = (torch.from_numpy(g.integers(-4, 5, (rows, k)).astype(np.float32)) for rows in (m, n))
    sa = torch.from_numpy(2.0 ** g.integers(-2, 3, (m, F.up(k)))).float()
    sb = torch.from_numpy(2.0 ** g.integers(-2, 3, (F.up(n, b_rows), F.up(k)))).float()
    _check(a, sa, b, sb, b_rows, a_dt)
