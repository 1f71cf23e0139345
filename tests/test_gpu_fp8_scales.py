"""GPU: the block-scaled 8-bit product with scales over the range that its documentation allows, in every kernel."""
import numpy as np
import pytest
import torch

import paper_2511_03586_amd as perf
from tests import fp8_helpers as F
from tests import parity as P

pytestmark = pytest.mark.gpu

F32, BF16, E4M3, E5M2 = perf.PERF_F32, perf.PERF_BF16, perf.PERF_E4M3, perf.PERF_E5M2

# a few rows and few tiles (waves that divide K), 168 tiles (four stages), 289 tiles (two; of 128 x 96 for fp32 C with scales by
# rows) and 841 (256 x 256 for bf16 C)
SIZES = [(3, 200, 300), (200, 300, 256), (1500, 1700, 513), (2049, 2100, 300), (3700, 3601, 300)]


def _signed(g, shape, least):
    """least * [1, 2), either sign"""
    return torch.from_numpy((least * g.uniform(1, 2, shape) * g.choice([-1.0, 1.0], shape)).astype(np.float32))


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("b_rows", [1, 128])
@pytest.mark.parametrize("c_dt", [F32, BF16])
@pytest.mark.parametrize("large", [False, True])
def test_two_scales_whose_product_leaves_fp32(m, n, k, b_rows, c_dt, large):
    """Two scales of 2^-70, whose product is no normal number, with large operands; of 2^70 and 2^60, whose product is none of
    fp32's, with small ones.  The results are ordinary numbers.  A block of zeros in between has scales of 2^95 and 2^120: it adds
    nothing."""
    g = np.random.default_rng(m + k)
    ea, eb, alpha = (70, 60, 2.0 ** -20) if large else (-70, -70, 2.0 ** 20)
    a = _signed(g, (m, k), 2.0 ** -13 if large else 2.0 ** 12).to(torch.float8_e5m2)
    b = _signed(g, (n, k), 2.0 ** -6 if large else 2.0 ** 6).to(torch.float8_e4m3fn)
    sa = _signed(g, (m, F.up(k)), 2.0 ** ea).abs()
    sb = _signed(g, (F.up(n, b_rows), F.up(k)), 2.0 ** eb).abs()
    a[:, 128:256] = 0
    sa[:, 1], sb[:, 1] = 2.0 ** 95, 2.0 ** 120
    ref, absdot = F.gemm_ref(a, sa, b, sb, b_rows, alpha)
    assert 2.0 ** -100 < absdot.min() and absdot.max() < 2.0 ** 107  # (ordinary numbers, also before alpha)
    c = F.run_gemm(a, sa, b, sb, b_rows, c_dt, alpha, a_dt=E5M2)
    P.assert_contraction_close(c, ref, absdot, k + 3 + (2 ** 13 if c_dt == BF16 else 0), out_bf16=c_dt == BF16)


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("b_rows", [1, 128])
@pytest.mark.parametrize("va,ea,vb,eb", [(57344.0, 95, 448.0, -100), (57344.0, 95, 448.0, -149), (2.0 ** -16, -100, 2.0 ** -9, 120),
                                         (2.0 ** -16, -100, 448.0, 127), (1.0, 0, 448.0, 110), (1.0, 60, 2.0 ** -9, -149)])
def test_scales_at_the_ends_of_their_range(m, n, k, b_rows, va, ea, vb, eb):
    """The largest and smallest operands with the largest and smallest scales of A that no step can take out of fp32's range, and
    any of B.  Operands and scales of one value each: every sum is k products, k v_a v_b of at most 24 bits, and exact."""
    a = torch.full((m, k), va).to(torch.float8_e5m2)
    b = torch.full((n, k), vb).to(torch.float8_e4m3fn)
    sa, sb = torch.full((m, F.up(k)), 2.0 ** ea), torch.full((F.up(n, b_rows), F.up(k)), 2.0 ** eb)
    want = np.float64(k) * va * vb * 2.0 ** (ea + eb)
    for c_dt in (F32, BF16):
        c = F.run_gemm(a, sa, b, sb, b_rows, c_dt, a_dt=E5M2)
        assert (c == (want if c_dt == F32 else torch.tensor(want).to(torch.bfloat16).double().item())).all(), (c.min(), c.max(), want)
