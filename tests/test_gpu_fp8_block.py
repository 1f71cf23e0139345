"""GPU: the operators of a block in 8 bits as they are used together (a training step, a decoded token), in graphs, on streams
side by side, with values that are not finite, at offsets beyond 32 bits, and in place."""
import numpy as np
import pytest
import torch

import paper_2511_03586_amd as perf
from tests import fp8_helpers as F
from tests import gpu_helpers as G
from tests import parity as P
from tests import test_gpu_residual_norm as N

pytestmark = pytest.mark.gpu

F32, BF16, E4M3, E5M2 = perf.PERF_F32, perf.PERF_BF16, perf.PERF_E4M3, perf.PERF_E5M2
EPS = float(np.float32(1e-5))


def _dev(shape, dt):
    return torch.empty(shape, dtype=F.TORCH[dt], device="cuda")


class Quantized:
    """One matrix in both orientations; rows a multiple of 16 bytes apart."""

    def __init__(self, rows, cols, q_dt, block_rows):
        self.rows, self.cols, self.q_dt, self.block_rows = rows, cols, q_dt, block_rows
        self.ldq, self.ldqt = F.up(cols, 16) * 16, F.up(rows, 16) * 16
        self.q, self.qt = _dev((rows, self.ldq), q_dt), _dev((cols, self.ldqt), q_dt)
        self.s, self.st = _dev((F.up(rows, block_rows), F.up(cols)), F32), _dev((F.up(cols, block_rows), F.up(rows)), F32)

    def take(self, x, x_dt):
        perf.perf_quantize_fp8(x.data_ptr(), self.q.data_ptr(), self.s.data_ptr(), self.qt.data_ptr(), self.st.data_ptr(), self.rows,
                               self.cols, x.stride(0), self.ldq, F.up(self.cols), self.ldqt, F.up(self.rows), self.block_rows, x_dt,
                               self.q_dt, stream=G.stream())

    def operand(self, transposed):
        q, s, ld, cols = (self.qt, self.st, self.ldqt, self.rows) if transposed else (self.q, self.s, self.ldq, self.cols)
        return q, s, ld, F.up(cols)

    def values(self, transposed):
        q, s, _, _ = self.operand(transposed)
        cols = self.rows if transposed else self.cols
        return q[:, :cols].cpu(), s.cpu()


def _gemm(a, a_t, b, b_t, c, c_dt, k):
    qa, sa, lda, ldsa = a.operand(a_t)
    qb, sb, ldb, ldsb = b.operand(b_t)
    perf.perf_gemm_fp8(qa.data_ptr(), sa.data_ptr(), qb.data_ptr(), sb.data_ptr(), c.data_ptr(), c.shape[0], c.shape[1], k, lda, ldsa,
                       ldb, ldsb, c.shape[1], b.block_rows, a_dt=a.q_dt, c_dt=c_dt, stream=G.stream())


def _check_gemm(a, a_t, b, b_t, c, c_dt, k):
    ref, absdot = F.gemm_ref(*a.values(a_t), *b.values(b_t), b.block_rows)
    P.assert_contraction_close(c.cpu().double().numpy(), ref, absdot, k + 3 + (2 ** 13 if c_dt == BF16 else 0), out_bf16=c_dt == BF16)


class Step:
    """A block between its norms, forward and backward: y = norms(u, x), z = Y W^T in 8 bits, from dz the gradients of W, u, x, the
    gate and the gains.  Nothing is allocated by run()."""

    def __init__(self, tokens, hidden, out, gate_rows, seed):
        g = torch.Generator().manual_seed(seed)
        n = lambda *shape: torch.randn(shape, generator=g)  # noqa: E731
        t, d = tokens, hidden
        self.tokens, self.hidden, self.out, self.gate_rows = t, d, out, gate_rows
        self.inputs = {"u": n(t, d).bfloat16(), "x": n(t, d).bfloat16(), "dz": (n(t, out) * 0.01).bfloat16(), "dh": n(t, d).bfloat16()}
        self.params = {"gate": n(F.up(t, gate_rows), d), "post": 1 + 0.1 * n(d), "pre": 1 + 0.1 * n(d), "w": n(out, d) * 0.05}
        for k, v in {**self.inputs, **self.params}.items():
            setattr(self, k, v.cuda())
        self.h, self.y, self.dy, self.dx, self.du = (_dev((t, d), BF16) for _ in range(5))
        self.r_post, self.r_pre = _dev((t,), F32), _dev((t,), F32)
        self.qy, self.qdz, self.qw = Quantized(t, d, E4M3, 1), Quantized(t, out, E5M2, 1), Quantized(out, d, E4M3, 128)
        self.z, self.dw = _dev((t, out), BF16), _dev((out, d), F32)
        self.dgate, self.dpost, self.dpre = torch.empty_like(self.gate), _dev((d,), F32), _dev((d,), F32)
        self.ws = torch.empty(perf.perf_residual_norm_backward_workspace_bytes(t, d), dtype=torch.uint8, device="cuda")

    def run(self):
        t, d, p = self.tokens, self.hidden, lambda v: v.data_ptr()
        perf.perf_residual_norm(p(self.u), p(self.x), p(self.gate), p(self.post), p(self.pre), p(self.h), p(self.y), None, p(self.r_post),
                                p(self.r_pre), t, d, d, d, d, self.gate_rows, d, d, 0, 0.75, EPS, BF16, F32, F32, BF16, stream=G.stream())
        self.qy.take(self.y, BF16)
        self.qw.take(self.w, F32)
        _gemm(self.qy, False, self.qw, False, self.z, BF16, d)
        self.qdz.take(self.dz, BF16)
        _gemm(self.qdz, False, self.qw, True, self.dy, BF16, self.out)
        _gemm(self.qdz, True, self.qy, True, self.dw, F32, t)
        perf.perf_residual_norm_backward(p(self.dy), p(self.dh), p(self.h), p(self.u), p(self.gate), p(self.post), p(self.pre),
                                         p(self.r_post), p(self.r_pre), p(self.dx), p(self.du), p(self.dgate), p(self.dpost), p(self.dpre),
                                         p(self.ws), t, d, d, d, d, d, d, self.gate_rows, d, d, d, 0.75, BF16, F32, F32,
                                         stream=G.stream())

    NAMES = ("h", "y", "z", "dy", "dw", "dx", "du", "dgate", "dpost", "dpre", "r_post", "r_pre")

    def results(self):
        return {k: getattr(self, k).cpu().clone() for k in self.NAMES}


@pytest.mark.parametrize("tokens,hidden,out,gate_rows", [(300, 256, 384, 300), (257, 520, 200, 64), (1, 128, 128, 1), (1030, 1024, 640, 1)])
def test_training_step(tokens, hidden, out, gate_rows):
    """Each operator against its definition on what the one before it left."""
    s = Step(tokens, hidden, out, gate_rows, 3)
    s.run()
    torch.cuda.synchronize()
    r = s.results()
    h, y, r1, r2, mag = F.norm_ref(s.inputs["u"], s.inputs["x"], s.params["gate"], gate_rows, s.params["post"], s.params["pre"], 0.75, EPS)
    c, half = N._depth(hidden) * 2.0 ** -24, 2.0 ** -8
    assert torch.all((r["h"].double() - h).abs() <= c * mag + half * h.abs())
    rel = c + c * torch.sqrt((mag ** 2).mean(1)) * r2
    err = c * mag * r2[:, None] * s.params["pre"].double() + rel[:, None] * y.abs()
    assert torch.all((r["y"].double() - y).abs() <= err * (1 + half) + half * y.abs())
    for m, x, block in ((s.qy, r["y"], 1), (s.qdz, s.inputs["dz"], 1), (s.qw, s.params["w"], 128)):
        for transposed in (False, True):
            q, sc = m.values(transposed)
            rq, rs = F.quantize_ref(x.T.contiguous() if transposed else x, block, m.q_dt)
            assert torch.equal(sc, rs) and torch.equal(q.view(torch.uint8), rq.view(torch.uint8))
    _check_gemm(s.qy, False, s.qw, False, s.z, BF16, hidden)
    _check_gemm(s.qdz, False, s.qw, True, s.dy, BF16, out)
    _check_gemm(s.qdz, True, s.qy, True, s.dw, F32, tokens)
    args = (r["dy"], s.inputs["dh"], r["h"], s.inputs["u"], s.params["gate"], gate_rows, s.params["post"], s.params["pre"], r["r_post"],
            r["r_pre"], 0.75)
    ref, mag = F.grad_ref(*args), F.grad_ref(*args, magnitudes=True)
    for name in ("dx", "du", "dgate", "dpost", "dpre"):
        c = (2 * N._depth(hidden) + (0 if name in ("dx", "du") else tokens + 8)) * 2.0 ** -24
        step = half if name in ("dx", "du") else 2.0 ** -24
        assert torch.all((r[name].double() - ref[name]).abs() <= c * mag[name] * (1 + step) + step * ref[name].abs()), name


@pytest.mark.parametrize("tokens", [1, 6, 33])
@pytest.mark.parametrize("hidden,out", [(512, 1000), (1001, 256)])
def test_decoded_tokens(tokens, hidden, out):
    """The norms hand y on in 8 bits to the product that reads it."""
    g = np.random.default_rng(tokens + out)
    u, x, gate, post, pre = N._make(tokens, hidden, BF16, tokens, F32, F32, True, 1)
    b, sb = F.random_operand(g, out, hidden, 128)
    ld, kb = F.up(hidden, 16) * 16, F.up(hidden)
    ud, xd, gd, pd, qd = (v.cuda() for v in (u, x, gate, post, pre))
    y, ys = torch.full((tokens, ld), 0x7F, dtype=torch.uint8, device="cuda"), _dev((tokens, kb), F32)
    h, z = _dev((tokens, hidden), BF16), _dev((tokens, out), BF16)
    bd = torch.full((out, ld), 0x7F, dtype=torch.uint8, device="cuda")
    bd[:, :hidden] = b.view(torch.uint8).cuda()
    sbd = sb.cuda()
    perf.perf_residual_norm(ud.data_ptr(), xd.data_ptr(), gd.data_ptr(), pd.data_ptr(), qd.data_ptr(), h.data_ptr(), y.data_ptr(),
                            ys.data_ptr(), None, None, tokens, hidden, hidden, hidden, hidden, tokens, hidden, ld, kb, 1.0, EPS, BF16, F32,
                            F32, E4M3, stream=G.stream())
    perf.perf_gemm_fp8(y.data_ptr(), ys.data_ptr(), bd.data_ptr(), sbd.data_ptr(), z.data_ptr(), tokens, out, hidden, ld, kb, ld, kb, out,
                       128, c_dt=BF16, stream=G.stream())
    torch.cuda.synchronize()
    assert bool((y[:, hidden:] == 0x7F).all())
    ref, absdot = F.gemm_ref(y[:, :hidden].contiguous().view(torch.float8_e4m3fn).cpu(), ys.cpu(), b, sb, 128)
    P.assert_contraction_close(z.cpu().double().numpy(), ref, absdot, hidden + 3 + 2 ** 13, out_bf16=True)


def _same(a, b):
    return all(torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)) for k in a)


def test_graph_replays_are_the_eager_results():
    """A step captured once and replayed on new inputs, with eager steps and other work between the replays."""
    s, other = Step(300, 520, 256, 64, 5), Step(300, 520, 256, 64, 6)
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for round_ in range(4):
        g = torch.Generator().manual_seed(100 + round_)
        for name, v in s.inputs.items():
            new = torch.randn(v.shape, generator=g).to(v.dtype)
            getattr(s, name).copy_(new)
            getattr(other, name).copy_(new)
        for name in s.params:
            getattr(other, name).copy_(getattr(s, name))
        for name in Step.NAMES:
            getattr(s, name).zero_()
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        assert _same(s.results(), other.results()), round_
        torch.randn(1 << 20, device="cuda").sort()


def test_steps_side_by_side_on_two_streams():
    a, b = Step(700, 520, 384, 700, 1), Step(513, 1024, 300, 1, 2)
    a.run(), b.run()
    torch.cuda.synchronize()
    ra, rb = a.results(), b.results()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for s in (a, b):
            for name in Step.NAMES:
                getattr(s, name).zero_()
        torch.cuda.synchronize()
        for s, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                s.run()
        torch.cuda.synchronize()
        assert _same(ra, a.results()) and _same(rb, b.results())


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("cols", [200, 1001, 9000, 20000])
def test_norm_keeps_what_is_not_finite_to_its_row(cols, bad):
    u, x, gate, post, pre = N._make(9, cols, F32, 9, F32, F32, True, 4)
    clean = N._forward(u, x, gate, 9, post, pre, 1.0, F32)
    u[3, cols // 2] = bad
    h, y, _, r1, r2 = N._forward(u, x, gate, 9, post, pre, 1.0, F32)
    rest = [i for i in range(9) if i != 3]
    assert torch.equal(h[rest], clean[0][rest]) and torch.equal(y[rest], clean[1][rest]) and torch.equal(r2[rest], clean[4][rest])
    assert not bool(torch.isfinite(h[3, cols // 2])) and not bool(torch.isfinite(y[3, cols // 2]))
    dy, dh = torch.randn(9, cols), torch.randn(9, cols)
    good = N._backward(dy, dh, clean[0], x, gate, 9, post, pre, clean[3], clean[4], 1.0, F32)
    dy[5, 7] = bad
    got = N._backward(dy, dh, clean[0], x, gate, 9, post, pre, clean[3], clean[4], 1.0, F32)
    rest = [i for i in range(9) if i != 5]
    for name in ("dx", "du"):
        assert torch.equal(got[name][rest], good[name][rest]) and not bool(torch.isfinite(got[name][5, 7]))
    assert not bool(torch.isfinite(got["dpre"][7])) and torch.equal(got["dpre"][8:], good["dpre"][8:])


@pytest.mark.parametrize("m,n,k", [(5, 200, 300), (300, 260, 300), (1930, 1800, 200), (3700, 3601, 200)])
def test_gemm_keeps_what_is_not_finite_to_its_row_and_column(m, n, k):
    g = np.random.default_rng(m)
    a, sa = F.random_operand(g, m, k, 1)
    b, sb = F.random_operand(g, n, k, 1)
    for c_dt in (F32, BF16):
        clean = F.run_gemm(a, sa, b, sb, 1, c_dt)
        a2, sb2 = a.clone(), sb.clone()
        a2.view(torch.uint8)[m // 2, k - 1] = 0x7F  # a NaN
        sb2[n // 3, 0] = float("inf")
        c = F.run_gemm(a2, sa, b, sb2, 1, c_dt)
        assert np.isnan(c[m // 2]).all() and not np.isfinite(c[:, n // 3]).any()
        rows, cols = np.arange(m) != m // 2, np.arange(n) != n // 3
        assert np.array_equal(c[rows][:, cols], clean[rows][:, cols])


def test_gemm_large_offsets():
    """Rows of A and B so far apart, and matrices of a batch, that offsets pass 32 bits."""
    m, n, k, ld = 40, 530, 200, (1 << 23) - 16
    g = np.random.default_rng(8)
    a, sa = F.random_operand(g, m, k, 1)
    b, sb = F.random_operand(g, n, k, 128)
    ref, absdot = F.gemm_ref(a, sa, b, sb, 128)
    base = torch.empty((n - 1) * ld + 1024, dtype=torch.uint8, device="cuda")
    at = 512  # A's rows lie beside B's
    torch.as_strided(base, (n, k), (ld, 1)).copy_(b.view(torch.uint8).cuda())
    torch.as_strided(base[at:], (m, k), (ld, 1)).copy_(a.view(torch.uint8).cuda())
    sad, sbd = sa.cuda(), sb.cuda()
    for c_dt in (F32, BF16):
        c = _dev((m, n), c_dt)
        perf.perf_gemm_fp8(base.data_ptr() + at, sad.data_ptr(), base.data_ptr(), sbd.data_ptr(), c.data_ptr(), m, n, k, ld, 2, ld, 2, n,
                           128, c_dt=c_dt, stream=G.stream())
        torch.cuda.synchronize()
        P.assert_contraction_close(c.cpu().double().numpy(), ref, absdot, k + 3 + (2 ** 13 if c_dt == BF16 else 0), out_bf16=c_dt == BF16)
    # the same rows as matrices of one row each of a batch, each result a row
    c = _dev((n, n), F32)
    rows = torch.arange(n) % m
    sad = sa[rows].contiguous().cuda()
    torch.as_strided(base[at:], (n, k), (ld, 1)).copy_(a[rows].view(torch.uint8).cuda())
    perf.perf_gemm_fp8(base.data_ptr() + at, sad.data_ptr(), base.data_ptr(), sbd.data_ptr(), c.data_ptr(), 1, n, k, 208, 2, ld, 2, n, 128,
                       n, ld, 2, 0, 0, n, c_dt=F32, stream=G.stream())
    torch.cuda.synchronize()
    P.assert_contraction_close(c.cpu().double().numpy(), ref[rows], absdot[rows], k + 3)


@pytest.mark.parametrize("cols", [200, 5, 9001])
def test_norms_large_offsets(cols):
    """All operands in one stretch of memory, rows so far apart that offsets pass 32 bits."""
    rows, ld, apart = 40, 1 << 26, 10240
    u, x, gate, post, pre = N._make(rows, cols, BF16, 1, BF16, F32, True)
    base = torch.empty((rows - 1) * ld + 10 * apart, dtype=torch.bfloat16, device="cuda")
    part = lambda i: torch.as_strided(base[i * apart:], (rows, cols), (ld, 1))  # noqa: E731
    names = ("u", "x", "gate", "h", "y", "dy", "dx", "du", "dgate")
    m = {name: part(i) for i, name in enumerate(names)}
    at = {name: v.data_ptr() for name, v in m.items()}
    dy = torch.randn(rows, cols, generator=torch.Generator().manual_seed(1)).bfloat16()
    for name, v in (("u", u), ("x", x), ("gate", gate), ("dy", dy)):
        m[name].copy_(v.cuda())
    postd, pred, r1, r2, dpost, dpre = post.cuda(), pre.cuda(), _dev((rows,), F32), _dev((rows,), F32), _dev((cols,), F32), _dev((cols,), F32)
    ws = torch.empty(perf.perf_residual_norm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    p = lambda v: v.data_ptr()  # noqa: E731
    perf.perf_residual_norm(at["u"], at["x"], at["gate"], p(postd), p(pred), at["h"], at["y"], None, p(r1), p(r2), rows, cols, ld, ld, ld,
                            1, ld, ld, 0, 1.0, EPS, BF16, BF16, F32, BF16, stream=G.stream())
    perf.perf_residual_norm_backward(at["dy"], None, at["h"], at["u"], at["gate"], p(postd), p(pred), p(r1), p(r2), at["dx"], at["du"],
                                     at["dgate"], p(dpost), p(dpre), p(ws), rows, cols, ld, 0, ld, ld, ld, 1, ld, ld, ld, 1.0, BF16, BF16,
                                     F32, stream=G.stream())
    torch.cuda.synchronize()
    h, y, s, q1, q2 = N._forward(u, x, gate, 1, post, pre, 1.0, BF16, BF16)
    assert torch.equal(m["h"].cpu(), h) and torch.equal(m["y"].cpu(), y) and torch.equal(r1.cpu(), q1) and torch.equal(r2.cpu(), q2)
    got = N._backward(dy, None, h, u, gate, 1, post, pre, q1, q2, 1.0, BF16, BF16)
    for name in ("dx", "du", "dgate"):
        assert torch.equal(m[name].cpu(), got[name]), name
    assert torch.equal(dpost.cpu(), got["dpost"]) and torch.equal(dpre.cpu(), got["dpre"])


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("cols", [6, 300, 1023, 8192, 9001, 20000])
def test_results_in_the_place_of_operands(cols, dt):
    """h and y over u and x, in every pairing."""
    rows = 30
    u, x, gate, post, pre = N._make(rows, cols, dt, 7, F32, F32, True, 2)
    h, y, _, r1, r2 = N._forward(u, x, gate, 7, post, pre, 1.25, dt)
    gd, pd, qd = gate.cuda(), post.cuda(), pre.cuda()
    for hx in ("u", "x", None):
        for yx in ("u", "x", None):
            if hx == yx:
                continue
            m = {"u": u.cuda(), "x": x.cuda(), None: _dev((rows, cols), dt)}
            perf.perf_residual_norm(m["u"].data_ptr(), m["x"].data_ptr(), gd.data_ptr(), pd.data_ptr(), qd.data_ptr(), m[hx].data_ptr(),
                                    m[yx].data_ptr(), None, None, None, rows, cols, cols, cols, cols, 7, cols, cols, 0, 1.25, 1e-5, dt, F32,
                                    F32, dt, stream=G.stream())
            torch.cuda.synchronize()
            assert torch.equal(m[hx].cpu(), h) and torch.equal(m[yx].cpu(), y), (hx, yx)


@pytest.mark.parametrize("cols", [8193, 16377, 16385, 20000])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_norms_of_wide_rows(cols, dt):
    N._check_forward(20, cols, dt, 3, dt)
    N._check_forward(20, cols, dt, 20, y_dt=E4M3)
    N._check_backward(20, cols, dt, 3, dt)
    N._check_backward(300, cols, dt, 300)
    N._check_backward(300, cols, dt, 1, dt)


@pytest.mark.parametrize("m,n,k", [(1, 25700, 1100), (30, 25700, 1100), (33, 25700, 200), (100, 16384, 300), (20, 16384, 1500),
                                   (1200, 1300, 2700), (1200, 1300, 900), (2305, 4096, 130)])
def test_gemm_choices_of_a_kernel(m, n, k):
    """Few rows, few tiles and many, on both sides of the lengths of K at which the choice turns."""
    g = np.random.default_rng(m + n)
    a, sa = F.random_operand(g, m, k, 1)
    b, sb = F.random_operand(g, n, k, 128)
    ref, absdot = F.gemm_ref(a, sa, b, sb, 128)
    for c_dt in (F32, BF16):
        c = F.run_gemm(a, sa, b, sb, 128, c_dt)
        P.assert_contraction_close(c, ref, absdot, k + 3 + (2 ** 13 if c_dt == BF16 else 0), out_bf16=c_dt == BF16)


@pytest.mark.parametrize("rows,cols,gate_rows", [(1, 700, 1), (6, 5760, 6), (12, 13128, 12), (16, 76, 16), (16, 76, 0), (145, 336, 13), (300, 512, 2),
                                                 (2000, 2048, 7), (5000, 500, 16), (700, 300, 11), (1920, 136, 137), (400, 1000, 90)])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_gradient_of_few_rows_and_of_small_groups(rows, cols, gate_rows, dt):
    """One run of rows, whose sums are the results; groups taken by a team alone and by all; gates of two runs and of many."""
    N._check_backward(rows, cols, dt, gate_rows)
    N._check_backward(rows, cols, dt, gate_rows, F32, skip=("dpost",))
    N._check_backward(rows, cols, dt, gate_rows, BF16, post=False, skip=("dgate", "dpre"))


def test_gemm_of_more_matrices_than_a_launch_holds():
    """Batches beyond 65535, in both kernels' launches."""
    g = np.random.default_rng(4)
    for m, n, k, batch in ((1, 4, 20, 65539), (2, 3, 1100, 65537)):
        a, sa = F.random_operand(g, m, k, 1)
        b, sb = F.random_operand(g, n, k, 1)
        ref, absdot = F.gemm_ref(a, sa, b, sb, 1)
        ld, kb = F.up(k, 16) * 16, F.up(k)
        ad, bd = torch.zeros((m, ld), dtype=torch.uint8, device="cuda"), torch.zeros((n, ld), dtype=torch.uint8, device="cuda")
        ad[:, :k], bd[:, :k] = a.view(torch.uint8).cuda(), b.view(torch.uint8).cuda()
        sad, sbd = sa.cuda(), sb.cuda()
        scaled = torch.arange(1, batch + 1, device="cuda", dtype=torch.float32)[:, None, None] * sad  # each matrix its own scales
        c = torch.zeros((batch, m, n), device="cuda")
        perf.perf_gemm_fp8(ad.data_ptr(), scaled.data_ptr(), bd.data_ptr(), sbd.data_ptr(), c.data_ptr(), m, n, k, ld, kb, ld, kb, n, 1,
                           batch, 0, m * kb, 0, 0, m * n, c_dt=F32, stream=G.stream())
        torch.cuda.synchronize()
        for i in (0, 1, 65534, 65535, 65536, batch - 1):
            got = c[i].cpu().double().numpy()
            assert np.all(np.abs(got - (i + 1) * ref) <= (k + 4) * 2.0 ** -23 * (i + 1) * absdot), (m, i)
