"""GPU: quantisation in blocks of 128 and the block-scaled 8-bit product, against their definitions."""
import numpy as np
import pytest
import torch

import paper_2511_03586_amd as perf
from tests import fp8_helpers as F
from tests import gpu_helpers as G
from tests import parity as P

pytestmark = pytest.mark.gpu

F32, BF16, E4M3, E5M2 = perf.PERF_F32, perf.PERF_BF16, perf.PERF_E4M3, perf.PERF_E5M2


def _x(rows, cols, seed, dt=F32):
    g = np.random.default_rng(seed)
    x = torch.from_numpy((g.standard_normal((rows, cols)) * np.exp(2 * g.standard_normal((rows, 1)))).astype(np.float32))
    return x.to(F.TORCH[dt])


def _same(got, ref):
    # bit for bit: the definition names each rounding
    assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8))


def _check_quantize(x, dt, q_dt, block_rows, row, transposed, **kw):
    q, s, qt, st = F.run_quantize(x, dt, q_dt, block_rows, row, transposed, **kw)
    if row:
        rq, rs = F.quantize_ref(x, block_rows, q_dt)
        assert torch.equal(s, rs)
        _same(q, rq)
    if transposed:
        rq, rs = F.quantize_ref(x.T.contiguous(), block_rows, q_dt)
        assert torch.equal(st, rs)
        _same(qt, rq)


SHAPES = [(1, 1), (1, 128), (3, 7), (2, 129), (127, 130), (128, 128), (129, 257), (300, 40), (5, 1000), (640, 384)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("block_rows,row,transposed", [(1, True, False), (1, False, True), (1, True, True), (128, True, False),
                                                       (128, False, True), (128, True, True)])
def test_quantize_is_the_definition(rows, cols, block_rows, row, transposed):
    for i, (dt, q_dt) in enumerate(((BF16, E4M3), (F32, E4M3), (BF16, E5M2), (F32, E5M2))):
        _check_quantize(_x(rows, cols, 10 * rows + cols + i, dt), dt, q_dt, block_rows, row, transposed)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_with_strides_and_odd_addresses(dt, block_rows):
    for pad, offset in ((1, 0), (16, 0), (3, 1), (5, 3)):
        _check_quantize(_x(150, 203, pad, dt), dt, E4M3, block_rows, True, True, ldx=203 + pad, pad=pad, offset=offset)
        _check_quantize(_x(150, 203, pad, dt), dt, E4M3, block_rows, True, False, ldx=203 + pad, pad=pad, offset=offset)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantize_extreme_blocks(block_rows):
    """Blocks of zeros, of the smallest numbers, next to the largest, of one value, and of values that tie."""
    x = torch.zeros(256, 512)
    x[128:, 128:256] = 2.0 ** -140
    x[:128, 128:256] = 3.0e38
    x[5, 200] = -3.4e38
    x[:128, 256:384] = -0.375
    x[128:, 256:384] = (torch.arange(128) * 0.25 + 448 - 64)[None]  # scale 1 where the block ends with 448
    x[128:, 383] = 448.0
    x[:, 384:] = torch.linspace(-1, 1, 128)[None] * 1e-37
    _check_quantize(x, F32, E4M3, block_rows, True, True)
    _check_quantize(x, F32, E5M2, block_rows, True, True)


@pytest.mark.parametrize("q_dt", [E4M3, E5M2])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_quantize_does_not_lose_what_is_not_finite(q_dt, bad):
    """A NaN or an infinity reads back as NaN at its place; other blocks are as without it."""
    x = _x(256, 256, 3)
    x[17, 130] = bad
    for block_rows in (1, 128):
        q, s, qt, st = F.run_quantize(x, F32, q_dt, block_rows)
        back = q.double() * F.spread(s.double(), block_rows, 256, 256)
        back_t = qt.double() * F.spread(st.double(), block_rows, 256, 256)
        assert torch.isnan(back[17, 130]) and torch.isnan(back_t[130, 17])
        rq, rs = F.quantize_ref(x, block_rows, q_dt)
        other = torch.ones(256, 256, dtype=torch.bool)
        other[(0 if block_rows == 128 else 17):(128 if block_rows == 128 else 18), 128:] = False
        assert torch.equal(q.float()[other], rq.float()[other])


def test_quantize_large_offsets():
    """Rows so far apart that offsets pass 32 bits."""
    rows, cols, ld = 40, 200, 1 << 26
    x = _x(rows, cols, 8, BF16)
    base = torch.empty((rows - 1) * ld + cols, dtype=torch.bfloat16, device="cuda")
    xd = torch.as_strided(base, (rows, cols), (ld, 1))
    xd.copy_(x.cuda())
    q, s = F.Held(rows, cols, E4M3), F.Held(rows, 2, F32)
    qt, st = F.Held(cols, rows, E4M3), F.Held(cols, 1, F32)
    perf.perf_quantize_fp8(base.data_ptr(), q.at(), s.at(), None, None, rows, cols, ld, cols, 2, 0, 0, 1, BF16, E4M3,
                           stream=G.stream())
    perf.perf_quantize_fp8(base.data_ptr(), None, None, qt.at(), st.at(), rows, cols, ld, 0, 0, rows, 1, 1, BF16, E4M3,
                           stream=G.stream())
    torch.cuda.synchronize()
    rq, rs = F.quantize_ref(x, 1, E4M3)
    _same(q.get(), rq)
    assert torch.equal(s.get(), rs)
    rq, rs = F.quantize_ref(x.T.contiguous(), 1, E4M3)
    _same(qt.get(), rq)
    assert torch.equal(st.get(), rs)


def test_quantize_of_more_blocks_than_a_launch_holds():
    """Rows of one block each, more than 2^29 of them (a dimension of 2^32 threads is cut short without an error): every element
    and scale is that of its value, of which there are seven."""
    rows, piece = (1 << 29) + 1000, 7 << 23
    few = torch.tensor([[0.0], [1.5], [-3.0], [0.3125], [1e-3], [-700.0], [5e30]]).to(torch.bfloat16)
    rq, rs = F.quantize_ref(few, 1, E4M3)
    few, rq, rs = few[:, 0].cuda(), rq.view(torch.uint8)[:, 0].cuda(), rs[:, 0].cuda()
    x = few.repeat(F.up(rows, 7))[:rows]
    q = torch.full((rows,), F.GUARD, dtype=torch.uint8, device="cuda")
    s = torch.full((rows,), float("nan"), device="cuda")
    perf.perf_quantize_fp8(x.data_ptr(), q.data_ptr(), s.data_ptr(), None, None, rows, 1, 1, 1, 1, 0, 0, 1, BF16, E4M3, stream=G.stream())
    for i in range(0, rows, piece):
        n = min(piece, rows - i)
        assert torch.equal(q[i:i + n], rq.repeat(F.up(n, 7))[:n]) and torch.equal(s[i:i + n], rs.repeat(F.up(n, 7))[:n]), i


# ---- product ----------------------------------------------------------------------------------------
def _check_gemm(m, n, k, b_rows, c_dt, a_dt=E4M3, alpha=1.0, seed=0, **kw):
    g = np.random.default_rng(1000 * m + 10 * n + k + seed)
    a, sa = F.random_operand(g, m, k, 1, a_dt)
    b, sb = F.random_operand(g, n, k, b_rows)
    ref, absdot = F.gemm_ref(a, sa, b, sb, b_rows, alpha)
    c = F.run_gemm(a, sa, b, sb, b_rows, c_dt, alpha, a_dt=a_dt, **kw)
    # fp32 C: a product of 8-bit values is exact in fp32; it is scaled twice and by alpha, and added to others: K + 3 roundings.
    # bf16 C: of eight products, seven may lose what lies below 2^-13 of the largest: less than 2^-10 = 2^13 * 2^-23 in all.
    P.assert_contraction_close(c, ref, absdot, k + 3 + (2 ** 13 if c_dt == BF16 else 0), out_bf16=c_dt == BF16)


GEMM_SHAPES = [(1, 1, 1), (1, 16, 128), (1, 4096, 512), (3, 70, 129), (16, 16, 127), (17, 33, 255), (5, 513, 15), (64, 64, 2048),
               (33, 200, 1000), (128, 256, 640), (130, 129, 384), (255, 257, 100), (300, 300, 300), (64, 1024, 96), (513, 384, 1040),
               (256, 512, 128), (257, 1025, 145), (1000, 777, 1299), (1024, 1024, 256)]


@pytest.mark.parametrize("m,n,k", GEMM_SHAPES)
@pytest.mark.parametrize("b_rows", [1, 128])
def test_gemm_against_the_definition(m, n, k, b_rows):
    _check_gemm(m, n, k, b_rows, F32)
    _check_gemm(m, n, k, b_rows, BF16, E5M2, alpha=-0.37)


@pytest.mark.parametrize("m,n,k", [(1930, 1800, 400), (2049, 1921, 129), (1900, 1920, 128), (3700, 3601, 300), (3585, 3841, 77)])
@pytest.mark.parametrize("b_rows", [1, 128])
def test_gemm_of_many_tiles(m, n, k, b_rows):
    _check_gemm(m, n, k, b_rows, BF16)
    _check_gemm(m, n, k, b_rows, F32, E5M2)


@pytest.mark.parametrize("m,n,k", [(7, 130, 200), (200, 140, 300), (600, 520, 333), (1930, 1800, 333)])
def test_gemm_with_strides(m, n, k):
    for c_dt in (F32, BF16):
        _check_gemm(m, n, k, 1, c_dt, lda=368, ldb=400, ldsa=5, ldsb=7, ldc=n + 3)
        _check_gemm(m, n, k, 128, c_dt, lda=432, ldb=384, ldsa=4, ldsb=9, ldc=n + 1)


@pytest.mark.parametrize("m,n,k,b_rows", [(1, 40, 384, 128), (50, 70, 257, 1), (300, 260, 640, 128), (520, 1040, 515, 1), (1800, 1937, 270, 128)])
def test_gemm_exact_integers(m, n, k, b_rows):
    """Small whole numbers and scales that are powers of two: every sum is exact, in any order, so the result is too."""
    g = np.random.default_rng(m + n + k)
    a = torch.from_numpy(g.integers(-4, 5, (m, k)).astype(np.float32)).to(torch.float8_e4m3fn)
    b = torch.from_numpy(g.integers(-4, 5, (n, k)).astype(np.float32)).to(torch.float8_e4m3fn)
    sa = torch.from_numpy(2.0 ** g.integers(-2, 3, (m, F.up(k)))).float()
    sb = torch.from_numpy(2.0 ** g.integers(-2, 3, (F.up(n, b_rows), F.up(k)))).float()
    ref, _ = F.gemm_ref(a, sa, b, sb, b_rows)
    assert np.array_equal(F.run_gemm(a, sa, b, sb, b_rows, F32), ref)


@pytest.mark.parametrize("m,n,k", [(3, 40, 130), (150, 130, 261), (520, 1040, 515), (1930, 1801, 261)])
def test_gemm_does_not_use_what_lies_behind_a_row(m, n, k):
    """Rows' padding full of NaN (0x7f in e4m3) and scales behind the last block of a row: no effect."""
    g = np.random.default_rng(m)
    a, sa = F.random_operand(g, m, k, 1)
    b, sb = F.random_operand(g, n, k, 1)
    ref, absdot = F.gemm_ref(a, sa, b, sb, 1)
    ld, kb = F.up(k, 16) * 16 + 16, F.up(k)
    ad = torch.full((m, ld), 0x7F, dtype=torch.uint8, device="cuda")
    bd = torch.full((n, ld), 0x7F, dtype=torch.uint8, device="cuda")
    ad[:, :k], bd[:, :k] = a.view(torch.uint8).cuda(), b.view(torch.uint8).cuda()
    sad, sbd = torch.full((m, kb + 3), float("nan"), device="cuda"), torch.full((n, kb + 3), float("nan"), device="cuda")
    sad[:, :kb], sbd[:, :kb] = sa.cuda(), sb.cuda()
    c = torch.empty((m, n), device="cuda")
    perf.perf_gemm_fp8(ad.data_ptr(), sad.data_ptr(), bd.data_ptr(), sbd.data_ptr(), c.data_ptr(), m, n, k, ld, kb + 3, ld, kb + 3, n,
                       1, c_dt=F32, stream=G.stream())
    torch.cuda.synchronize()
    P.assert_contraction_close(c.cpu().numpy(), ref, absdot, k + 3)
    cb = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    perf.perf_gemm_fp8(ad.data_ptr(), sad.data_ptr(), bd.data_ptr(), sbd.data_ptr(), cb.data_ptr(), m, n, k, ld, kb + 3, ld, kb + 3, n,
                       1, c_dt=BF16, stream=G.stream())
    torch.cuda.synchronize()
    P.assert_contraction_close(cb.cpu().double().numpy(), ref, absdot, k + 3 + 2 ** 13, out_bf16=True)


@pytest.mark.parametrize("m,n,k,batch", [(1, 200, 256, 3), (40, 72, 130, 5), (256, 256, 384, 9), (300, 520, 200, 2), (515, 700, 300, 11)])
def test_gemm_batch(m, n, k, batch):
    g = np.random.default_rng(batch)
    ops = [(F.random_operand(g, m, k, 1), F.random_operand(g, n, k, 128)) for _ in range(batch)]
    ld, kb = F.up(k, 16) * 16, F.up(k)
    stride_a, stride_sa, stride_b, stride_sb, stride_c = (m + 1) * ld, m * kb + 2, n * ld, F.up(n) * kb + 1, m * n + 5
    ad = torch.full((batch * stride_a,), 0x7F, dtype=torch.uint8, device="cuda")
    bd = torch.full((batch * stride_b,), 0x7F, dtype=torch.uint8, device="cuda")
    sad, sbd = torch.zeros(batch * stride_sa, device="cuda"), torch.zeros(batch * stride_sb, device="cuda")
    for i, ((a, sa), (b, sb)) in enumerate(ops):
        ad[i * stride_a:i * stride_a + m * ld].view(m, ld)[:, :k] = a.view(torch.uint8).cuda()
        bd[i * stride_b:(i + 1) * stride_b].view(n, ld)[:, :k] = b.view(torch.uint8).cuda()
        sad[i * stride_sa:i * stride_sa + m * kb] = sa.reshape(-1).cuda()
        sbd[i * stride_sb:i * stride_sb + F.up(n) * kb] = sb.reshape(-1).cuda()
    c = torch.full((batch * stride_c,), 7.0, device="cuda")
    perf.perf_gemm_fp8(ad.data_ptr(), sad.data_ptr(), bd.data_ptr(), sbd.data_ptr(), c.data_ptr(), m, n, k, ld, kb, ld, kb, n, 128,
                       batch, stride_a, stride_sa, stride_b, stride_sb, stride_c, c_dt=F32, stream=G.stream())
    torch.cuda.synchronize()
    c = c.cpu().view(batch, stride_c)
    assert bool((c[:, m * n:] == 7.0).all())
    for i, ((a, sa), (b, sb)) in enumerate(ops):
        ref, absdot = F.gemm_ref(a, sa, b, sb, 128)
        P.assert_contraction_close(c[i, :m * n].view(m, n).numpy(), ref, absdot, k + 3)


def test_gemm_shared_operand_in_a_batch():
    """A stride of zero: one matrix B for all."""
    m, n, k, batch = 20, 48, 256, 4
    g = np.random.default_rng(5)
    b, sb = F.random_operand(g, n, k, 1)
    ops = [F.random_operand(g, m, k, 1) for _ in range(batch)]
    ad = torch.stack([a.view(torch.uint8) for a, _ in ops]).cuda()
    sad = torch.stack([s for _, s in ops]).cuda()
    bd, sbd = b.view(torch.uint8).cuda(), sb.cuda()
    c = torch.empty(batch, m, n, device="cuda")
    perf.perf_gemm_fp8(ad.data_ptr(), sad.data_ptr(), bd.data_ptr(), sbd.data_ptr(), c.data_ptr(), m, n, k, k, 2, k, 2, n, 1, batch,
                       m * k, m * 2, 0, 0, m * n, c_dt=F32, stream=G.stream())
    torch.cuda.synchronize()
    for i, (a, sa) in enumerate(ops):
        ref, absdot = F.gemm_ref(a, sa, b, sb, 1)
        P.assert_contraction_close(c[i].cpu().numpy(), ref, absdot, k + 3)


@pytest.mark.parametrize("m,n,k", [(1, 64, 256), (200, 300, 256), (1900, 1920, 256)])
def test_gemm_scales_whose_product_leaves_fp32(m, n, k):
    """Scales of 2^-80 and of 2^90: their products alone are no normal numbers, the results are."""
    g = np.random.default_rng(1)
    for ea, eb, amp in ((-70, -70, 2.0 ** 8), (70, 70, 2.0 ** -9)):
        a = torch.from_numpy((g.standard_normal((m, k)) * amp / 8).astype(np.float32)).clamp(-448, 448).to(torch.float8_e5m2)
        b = torch.from_numpy((g.standard_normal((n, k)) * amp / 8).astype(np.float32)).clamp(-448, 448).to(torch.float8_e4m3fn)
        sa = torch.full((m, 2), 2.0 ** ea)
        sb = torch.full((n, 2), 2.0 ** eb)
        c = F.run_gemm(a, sa, b, sb, 1, F32, alpha=2.0 ** 20 if ea < 0 else 2.0 ** -20, a_dt=E5M2)
        ref, absdot = F.gemm_ref(a, sa, b, sb, 1, alpha=2.0 ** 20 if ea < 0 else 2.0 ** -20)
        # before alpha, a result of less than 2^-126 keeps the bits above 2^-149 only, at each of its additions
        bound = (k + 3) * 2.0 ** -23 * absdot + k * 2.0 ** -149 * (2.0 ** 20 if ea < 0 else 1.0)
        overflow = np.abs(ref) > 3.4e38
        assert np.all((np.abs(c - ref) <= bound) | overflow)


def test_gemm_is_the_same_every_time():
    g = np.random.default_rng(2)
    for m, n, k in ((1, 512, 4096), (300, 300, 2048), (512, 1024, 512)):
        a, sa = F.random_operand(g, m, k, 1)
        b, sb = F.random_operand(g, n, k, 1)
        first = F.run_gemm(a, sa, b, sb, 1, F32)
        for _ in range(3):
            assert np.array_equal(first, F.run_gemm(a, sa, b, sb, 1, F32))


@pytest.mark.parametrize("m,n,k", [(3, 200, 300), (200, 300, 256), (1930, 1921, 256), (3700, 3601, 300)])
@pytest.mark.parametrize("ea,eb", [(-100, 110), (95, -120), (-126, 100), (60, -149)])
@pytest.mark.parametrize("b_rows", [1, 128])
def test_gemm_scales_at_the_ends_of_fp32(m, n, k, ea, eb, b_rows):
    """One scale huge and one tiny (a subnormal one too): the results are ordinary numbers."""
    g = np.random.default_rng(1)
    a, _ = F.random_operand(g, m, k, 1)
    b, _ = F.random_operand(g, n, k, 1)
    sa = torch.full((m, F.up(k)), 2.0 ** ea)
    sb = torch.full((F.up(n, b_rows), F.up(k)), 2.0 ** eb)
    ref, absdot = F.gemm_ref(a, sa, b, sb, b_rows)
    for c_dt in (F32, BF16):
        c = F.run_gemm(a, sa, b, sb, b_rows, c_dt)
        # scales of powers of two change no rounding as long as nothing leaves the normal numbers (2^-89 * 2^-9 at least does not)
        P.assert_contraction_close(c, ref, absdot, k + 3 + (2 ** 13 if c_dt == BF16 else 0), out_bf16=c_dt == BF16)


@pytest.mark.parametrize("m,n,k", [(1999, 2999, 300), (2049, 2049, 129), (2050, 2113, 1000), (1153, 3650, 255)])
def test_gemm_of_narrow_tiles(m, n, k):
    """Numbers of tiles for which the product with a scale for each row of B takes narrower ones."""
    _check_gemm(m, n, k, 1, F32, E5M2)
    _check_gemm(m, n, k, 1, F32, alpha=0.5, ldc=n + 5)


@pytest.mark.parametrize("m,n,k", [(700, 3500, 128), (1025, 2000, 130), (1500, 1700, 513), (130, 16300, 700), (1100, 2100, 2900), (2048, 2048, 640)])
@pytest.mark.parametrize("b_rows", [1, 128])
def test_gemm_of_one_round_of_tiles(m, n, k, b_rows):
    """From 100 to 256 tiles, K from one block to more than the stages hold."""
    _check_gemm(m, n, k, b_rows, BF16, ldsa=F.up(k) + 3, ldsb=F.up(k) + 1)
    _check_gemm(m, n, k, b_rows, F32, E5M2)


@pytest.mark.parametrize("m,n,k", [(700, 1500, 300), (2700, 400, 713), (1024, 1536, 2100), (65, 17000, 256), (70, 16300, 1200)])
def test_gemm_of_more_than_one_round_of_small_tiles(m, n, k):
    _check_gemm(m, n, k, 128, BF16)
    _check_gemm(m, n, k, 1, F32, E5M2)
