"""GPU: the paged 8-bit cache's operators as they are used: a block's serving chain, prompts then single tokens; in graphs that are
replayed on other lengths and pages; on streams side by side; with caches and strides beyond 32 bits."""
import pytest
import torch

import paper_2511_03586_amd as perf
from tests import cache_helpers as C
from tests import gpu_helpers as G
from tests.fp8_helpers import TORCH, up

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = perf.PERF_F32, perf.PERF_BF16, perf.PERF_E4M3
HQ, HKV, DIM, PAGE, HIDDEN = 8, 2, 64, 16, 512


class Serving:
    """A block's attention for a batch of sequences in one pool of pages: quantise, project to q, k, v in 8 bits, rotate and append,
    attend, quantise, project back, norm. Buffers are for up to `most` rows; nothing is allocated by step()."""

    def __init__(self, sequences, most, columns, seed):
        g = torch.Generator().manual_seed(seed)
        self.sequences, self.most, self.columns, self.pages = sequences, most, columns, sequences * columns + 1
        cu8 = lambda *shape: torch.empty(shape, dtype=torch.uint8, device="cuda")  # noqa: E731
        f = lambda *shape: torch.empty(shape, dtype=torch.float32, device="cuda")  # noqa: E731
        b = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.width = (HQ + 2 * HKV) * DIM
        self.weights = []
        for rows, cols in ((self.width, HIDDEN), (HIDDEN, HQ * DIM)):
            w = (torch.randn((rows, cols), generator=g) * cols ** -0.5).cuda()
            q, s = cu8(rows, cols), f(up(rows), up(cols))
            perf.perf_quantize_fp8(w.data_ptr(), q.data_ptr(), s.data_ptr(), None, None, rows, cols, cols, cols, up(cols), 0, 0, 128, F32, E4M3,
                                   stream=G.stream())
            self.weights.append((q, s))
        self.x, self.x8, self.xs, self.qkv = b(most, HIDDEN), cu8(most, HIDDEN), f(most, up(HIDDEN)), b(most, self.width)
        self.q, self.o, self.o8, self.os, self.u = b(most, HQ, DIM), b(most, HQ, DIM), cu8(most, HQ * DIM), f(most, up(HQ * DIM)), b(most, HIDDEN)
        self.h, self.gamma = b(most, HIDDEN), torch.ones(HIDDEN, device="cuda")
        self.turn = C.rotation_table(columns * PAGE, DIM).cuda()
        self.cache = C.Cache(self.pages, HKV, PAGE, DIM)
        self.cache.to_gpu()
        table = torch.full((sequences, columns), -1, dtype=torch.int32)
        table[:] = torch.randperm(self.pages, generator=g)[:sequences * columns].reshape(sequences, columns)
        self.table = table.cuda()
        self.lengths, self.cu = torch.zeros(sequences, dtype=torch.int32, device="cuda"), torch.zeros(sequences + 1, dtype=torch.int32, device="cuda")
        self.held = [0] * sequences
        self.ws = cu8(perf.perf_cache_attention_fp8_workspace_bytes(most, sequences, most, HQ, HKV, DIM, PAGE, columns))
        self.g = g

    def inputs(self, new):
        """Puts new tokens' activations, rows and lengths in place."""
        self.new = list(new)
        self.x.zero_()
        self.x[:sum(new)] = torch.randn((sum(new), HIDDEN), generator=self.g).bfloat16().cuda()
        self.lengths.copy_(torch.tensor(self.held, dtype=torch.int32))
        self.cu.copy_(torch.tensor([0] + self.new).cumsum(0).int())

    def step(self, tokens, most_new, st=None):
        p, st = (lambda t: t.data_ptr()), G.stream() if st is None else st
        (wq, ws), (vq, vs) = self.weights
        c, w = self.cache.gpu, self.width
        perf.perf_quantize_fp8(p(self.x), p(self.x8), p(self.xs), None, None, tokens, HIDDEN, HIDDEN, HIDDEN, up(HIDDEN), 0, 0, 1, BF16, E4M3,
                               stream=st)
        perf.perf_gemm_fp8(p(self.x8), p(self.xs), p(wq), p(ws), p(self.qkv), tokens, w, HIDDEN, HIDDEN, up(HIDDEN), HIDDEN, up(HIDDEN), w, 128,
                           stream=st)
        perf.perf_cache_append_fp8(p(self.qkv), p(self.qkv) + 2 * HQ * DIM, p(self.qkv) + 2 * (HQ + HKV) * DIM, p(self.turn), p(self.q), p(c["k"]),
                                   p(c["v"]), p(c["ks"]), p(c["vs"]), p(self.table), p(self.lengths), p(self.cu), tokens, self.sequences, HQ, HKV,
                                   DIM, w, w, w, HQ * DIM, self.pages, PAGE, self.columns, self.columns, DIM, self.columns * PAGE, 0, BF16,
                                   stream=st)
        perf.perf_cache_attention_fp8(p(self.q), p(c["k"]), p(c["v"]), p(c["ks"]), p(c["vs"]), p(self.table), p(self.lengths), p(self.cu),
                                      p(self.o), None, p(self.ws), tokens, self.sequences, most_new, HQ, HKV, DIM, HQ * DIM, HQ * DIM, self.pages,
                                      PAGE, self.columns, self.columns, 0, DIM ** -0.5, BF16, stream=st)
        perf.perf_quantize_fp8(p(self.o), p(self.o8), p(self.os), None, None, tokens, HQ * DIM, HQ * DIM, HQ * DIM, up(HQ * DIM), 0, 0, 1, BF16,
                               E4M3, stream=st)
        perf.perf_gemm_fp8(p(self.o8), p(self.os), p(vq), p(vs), p(self.u), tokens, HIDDEN, HQ * DIM, HQ * DIM, up(HQ * DIM), HQ * DIM,
                           up(HQ * DIM), HIDDEN, 128, stream=st)
        perf.perf_residual_norm(p(self.u), p(self.x), None, None, p(self.gamma), p(self.h), p(self.x), None, None, None, tokens, HIDDEN, HIDDEN,
                                HIDDEN, HIDDEN, tokens, HIDDEN, HIDDEN, 0, 1.0, 1e-5, BF16, F32, F32, BF16, stream=st)

    def batch(self):
        b = C.Batch(self.held, self.new, PAGE)
        b.table, b.columns, b.pages = self.table.cpu(), self.columns, self.pages
        return b

    def check(self):
        """The step's cache and attention against their definitions on what was there; the reference moves on."""
        torch.cuda.synchronize()
        batch, n = self.batch(), sum(self.new)
        qkv = self.qkv[:n].cpu().view(n, HQ + 2 * HKV, DIM)
        q = C.append_ref(self.cache, batch, qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], self.turn.cpu(), DIM, False, self.q[:n].cpu())
        assert torch.equal(C.bits(self.q[:n].cpu()), C.bits(q))
        assert all(torch.equal(self.cache.gpu[k].cpu(), self.cache.host[k]) for k in self.cache.host)
        ref = C.attention_ref(self.cache, batch, q, 0, DIM ** -0.5)
        C.assert_attention_close(self.o[:n].cpu(), None, ref, BF16, DIM, self.columns * PAGE)
        assert bool(torch.isfinite(self.h[:n]).all())
        self.held = [a + b for a, b in zip(self.held, self.new)]


def test_prompts_then_single_tokens():
    s = Serving(5, 200, 12, 1)
    for new in ([33, 1, 90, 16, 0], [1, 1, 1, 1, 40], [1, 1, 1, 1, 1], [1, 0, 3, 1, 1], [5, 64, 1, 1, 1]):
        s.inputs(new)
        s.step(sum(new), max(new))
        s.check()


def test_captured_step_replayed_on_other_lengths_and_pages():
    """One graph for all steps of up to 24 rows; each replay against the definitions, eager work between."""
    s = Serving(6, 24, 12, 2)
    s.inputs([4] * 6)
    s.step(24, 24)  # (each kernel has run before the capture)
    s.check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.step(24, 24, side.cuda_stream)
    torch.cuda.synchronize()
    for new in ([1] * 6, [2, 1, 0, 7, 1, 1], [1] * 6, [0, 0, 19, 1, 0, 0], [1, 1, 1, 1, 1, 1]):
        s.inputs(new)
        graph.replay()
        s.check()
        torch.randn(1000, device="cuda").sum().item()


def test_two_streams_side_by_side():
    states = [Serving(5, 120, 12, seed) for seed in (3, 4)]
    streams = [torch.cuda.Stream() for _ in states]
    for new in ([33, 1, 70, 16, 0], [1] * 5, [1, 0, 3, 1, 1]):
        for s in states:
            s.inputs(new)
        torch.cuda.synchronize()
        for s, st in zip(states, streams):
            s.step(sum(new), max(new), st.cuda_stream)
        for s in states:
            s.check()


@pytest.mark.parametrize("new", [[1, 1, 1], [40, 1, 20]])
def test_pages_beyond_32_bits(new):
    """The last pages of pools of 4.5 GiB."""
    page, kv, dim, pool = 256, 8, 256, 9216
    batch = C.Batch([300, 0, 511], new, page, 5)
    cache = C.Cache(batch.pages, kv, page, dim)
    C.fill(cache, batch, 6, upto_new=False)
    first = pool - batch.pages
    small = batch.table.clone()
    batch.table = torch.where(small >= 0, small + first, small)
    batch.to_gpu()
    cache.gpu = {k: torch.empty((pool, *v.shape[1:]), dtype=torch.uint8, device="cuda") for k, v in cache.host.items()}
    for k, v in cache.host.items():
        cache.gpu[k][first:] = v.cuda()
    small_pages, cache.pages, batch.pages = cache.pages, pool, pool
    g = torch.Generator().manual_seed(7)
    k = torch.randn((batch.tokens, kv, dim), generator=g).bfloat16()
    v = torch.randn((batch.tokens, kv, dim), generator=g).bfloat16()
    q = C.random_queries(batch, 2 * kv, dim, BF16, 8)
    C.run_append(cache, batch, None, k, v, None, 0, False, BF16)
    call = C.Attention(cache, batch, q, 0, dim ** -0.5, BF16)
    call.run()
    o, lse = call.results()
    batch.table, batch.pages, cache.pages = small, small_pages, small_pages
    C.append_ref(cache, batch, None, k, v, None, 0, False, None)
    for name in cache.host:
        assert torch.equal(cache.gpu[name][first:].cpu(), cache.host[name])
    C.assert_attention_close(o, lse, C.attention_ref(cache, batch, q, 0, dim ** -0.5), BF16, dim, 600)


@pytest.mark.parametrize("new", [[1, 2], [1, 40]])
def test_scale_of_zero_where_no_key_is_seen(new):
    """Without keys lse is -infinity, whatever the scale; with keys the mean of their values."""
    batch = C.Batch([20, 30], new, 16, 1, absent=((0, 0), (0, 1), (1, 1)))
    cache = C.Cache(batch.pages, 1, 16, 64)
    C.fill(cache, batch, 2)
    cache.to_gpu()
    batch.to_gpu()
    q = C.random_queries(batch, 2, 64, BF16, 3)
    for window in (0, 4):
        call = C.Attention(cache, batch, q, window, 0.0, BF16)
        call.run()
        C.assert_attention_close(*call.results(), C.attention_ref(cache, batch, q, window, 0.0), BF16, 64, 80)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_rows_that_do_not_ascend_stay_inside(dt):
    """Which rows are computed where cu descends is not specified; nothing is read or written outside, and the next call is right."""
    held, new = [2000, 90, 700, 0, 300], [60, 1, 40, 9, 130]
    batch = C.Batch(held, new, 16, 1)
    cache = C.Cache(batch.pages, 2, 16, 64)
    C.fill(cache, batch, 2)
    cache.to_gpu()
    batch.to_gpu()
    q = C.random_queries(batch, 8, 64, dt, 3)
    cu, n, x = batch.dev[2], batch.tokens, q[:, :2].contiguous().cuda()
    call = C.Attention(cache, batch, q, 0, 0.125, dt)
    for bad in ([0, n, 10, n, 20, n], [n, n - 1, 100, 50, 7, 0], [0, 200, 100, n, n - 60, n], [30, 20, 150, 140, n, 1], [-5, 2 ** 30, -2 ** 31, 2 ** 31 - 1, 5, n]):
        cu.copy_(torch.tensor(bad, dtype=torch.int32))
        call.run()
        call.results()
    cu.copy_(batch.cu)
    call.run()
    C.assert_attention_close(*call.results(), C.attention_ref(cache, batch, q, 0, 0.125), dt, 64, 2100)
    for bad in ([0, n, 10, n, 20, n], [n, n - 1, 100, 50, 7, 0], [-5, 2 ** 30, -2 ** 31, 2 ** 31 - 1, 5, n]):
        cu.copy_(torch.tensor(bad, dtype=torch.int32))
        pages = [cache.gpu[name].data_ptr() for name in ("k", "v", "ks", "vs")]
        perf.perf_cache_append_fp8(None, x.data_ptr(), x.data_ptr(), None, None, *pages, *batch.addresses(), n, 5, 2, 2, 64, 128, 128, 128, 128,
                                   cache.pages, 16, batch.columns, batch.table.shape[1], 0, 0, 0, dt, stream=G.stream())
        torch.cuda.synchronize()


@pytest.mark.parametrize("held", [20, 0])
def test_rows_beyond_32_bits(held):
    """Rows of tokens 2^31 elements apart."""
    ld, dim, kv = 2 ** 31 + 64, 64, 1
    batch = C.Batch([held], [2], 16, 1)
    cache = C.Cache(batch.pages, kv, 16, dim)
    C.fill(cache, batch, 2, upto_new=False)
    cache.to_gpu()
    batch.to_gpu()
    rows = torch.randn((2, dim), generator=torch.Generator().manual_seed(1)).bfloat16()
    far = torch.empty(ld + dim, dtype=torch.bfloat16, device="cuda")
    far[:dim], far[ld:] = rows[0].cuda(), rows[1].cuda()
    out = torch.empty(ld + dim, dtype=torch.bfloat16, device="cuda")
    c = cache.gpu
    perf.perf_cache_append_fp8(far.data_ptr(), far.data_ptr(), far.data_ptr(), None, out.data_ptr(), c["k"].data_ptr(), c["v"].data_ptr(),
                               c["ks"].data_ptr(), c["vs"].data_ptr(), *batch.addresses(), 2, 1, 1, kv, dim, ld, ld, ld, ld, cache.pages, 16,
                               batch.columns, batch.table.shape[1], 0, 0, 0, BF16, stream=G.stream())
    torch.cuda.synchronize()
    x = rows.view(2, 1, dim)
    C.append_ref(cache, batch, None, x, x, None, 0, False, None)
    assert all(torch.equal(cache.gpu[n].cpu(), cache.host[n]) for n in cache.host)
    assert torch.equal(out[:dim].cpu(), rows[0]) and torch.equal(out[ld:].cpu(), rows[1])
    for most in (2, 40):  # few rows and many
        ws = torch.empty(perf.perf_cache_attention_fp8_workspace_bytes(2, 1, most, 1, kv, dim, 16, batch.columns), dtype=torch.uint8, device="cuda")
        out.zero_()
        perf.perf_cache_attention_fp8(far.data_ptr(), c["k"].data_ptr(), c["v"].data_ptr(), c["ks"].data_ptr(), c["vs"].data_ptr(),
                                      *batch.addresses(), out.data_ptr(), None, ws.data_ptr(), 2, 1, most, 1, kv, dim, ld, ld, cache.pages, 16,
                                      batch.columns, batch.table.shape[1], 0, 0.125, BF16, stream=G.stream())
        torch.cuda.synchronize()
        o = torch.stack((out[:dim].cpu(), out[ld:].cpu())).view(2, 1, dim)
        C.assert_attention_close(o, None, C.attention_ref(cache, batch, x, 0, 0.125), BF16, dim, held + 2)


@pytest.mark.parametrize("held", [20, 0])
@pytest.mark.parametrize("heads", [8, 16])
def test_rows_of_several_heads_beyond_32_bits(held, heads):
    """Two tokens 2^31 elements apart, whose heads share one of the cache: 16 rows to it are few, 32 many."""
    ld, dim = 2 ** 31 + 64, 64
    batch = C.Batch([held], [2], 16, 1)
    cache = C.Cache(batch.pages, 1, 16, dim)
    C.fill(cache, batch, 2)
    cache.to_gpu()
    batch.to_gpu()
    q = C.random_queries(batch, heads, dim, BF16, 3)
    width = heads * dim
    far, out = (torch.empty(ld + width, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    far[:width], far[ld:] = q[0].flatten().cuda(), q[1].flatten().cuda()
    out[width:2 * width] = 7.0  # behind the first row
    lse = torch.empty((2, heads), device="cuda")
    c = cache.gpu
    ws = torch.empty(perf.perf_cache_attention_fp8_workspace_bytes(2, 1, 2, heads, 1, dim, 16, batch.columns), dtype=torch.uint8, device="cuda")
    perf.perf_cache_attention_fp8(far.data_ptr(), c["k"].data_ptr(), c["v"].data_ptr(), c["ks"].data_ptr(), c["vs"].data_ptr(), *batch.addresses(),
                                  out.data_ptr(), lse.data_ptr(), ws.data_ptr(), 2, 1, 2, heads, 1, dim, ld, ld, cache.pages, 16, batch.columns,
                                  batch.table.shape[1], 0, 0.125, BF16, stream=G.stream())
    torch.cuda.synchronize()
    o = torch.stack((out[:width].cpu(), out[ld:].cpu())).view(2, heads, dim)
    C.assert_attention_close(o, lse.cpu(), C.attention_ref(cache, batch, q, 0, 0.125), BF16, dim, held + 2)
    assert bool((out[width:2 * width] == 7.0).all())


@pytest.mark.parametrize("dt", [BF16, F32])
def test_more_sequences_than_lds_holds(dt):
    """700 sequences, of which some bring nothing, one token, or a run."""
    held = [(37 * i) % 90 for i in range(700)]
    for new in ([(1, 0, 2, 1, 1)[i % 5] for i in range(700)], [(1, 0, 25, 1, 3)[i % 5] for i in range(700)]):
        batch = C.Batch(held, new, 16, 1)
        cache = C.Cache(batch.pages, 1, 16, 64)
        C.fill(cache, batch, 2, upto_new=False)
        cache.to_gpu()
        batch.to_gpu()
        g = torch.Generator().manual_seed(3)
        k, v = (torch.randn((batch.tokens, 1, 64), generator=g).to(TORCH[dt]) for _ in range(2))
        q = C.random_queries(batch, 2, 64, dt, 4)
        turn = C.rotation_table(200, 64)
        turned = C.run_append(cache, batch, q, k, v, turn, 64, False, dt)
        ref = C.append_ref(cache, batch, q, k, v, turn, 64, False, q)
        assert torch.equal(C.bits(turned), C.bits(ref))
        assert all(torch.equal(cache.gpu[n].cpu(), cache.host[n]) for n in cache.host)
        call = C.Attention(cache, batch, turned, 0, 0.125, dt)
        call.run()
        o, lse = call.results()
        C.assert_attention_close(o, lse, C.attention_ref(cache, batch, turned, 0, 0.125), dt, 64, 120)


@pytest.mark.parametrize("dt,dim,kv", [(BF16, 128, 16), (BF16, 64, 32), (F32, 64, 16), (F32, 128, 4), (BF16, 256, 4)])
def test_long_lists_of_work(dt, dim, kv):
    """Row tiles and contexts enough for every workgroup to have several."""
    batch = C.Batch([2000, 2300, 1900, 700], [200, 129, 256, 1], 64, 1)
    cache = C.Cache(batch.pages, kv, 64, dim)
    C.fill(cache, batch, 2)
    cache.to_gpu()
    batch.to_gpu()
    q = C.random_queries(batch, kv, dim, dt, 3)
    call = C.Attention(cache, batch, q, 0, dim ** -0.5, dt)
    call.run()
    C.assert_attention_close(*call.results(), C.attention_ref(cache, batch, q, 0, dim ** -0.5), dt, dim, 2500)


def test_very_many_sequences():
    """70000 of them, of which four bring a token."""
    count = 70000
    new = [1 if i in (0, 5, 66000, count - 1) else 0 for i in range(count)]
    batch = C.Batch([3] * count, new, 16, 1, spare=0, pad_columns=0)
    batch.table = torch.full((count, 1), -1, dtype=torch.int32)
    for n, i in enumerate(i for i in range(count) if new[i]):
        batch.table[i, 0] = n
    batch.pages = 4
    cache = C.Cache(4, 1, 16, 64)
    g = torch.Generator().manual_seed(2)
    for p in range(4):
        for name in ("k", "v"):
            cache.append(name, p, 0, torch.randn((3, 1, 64), generator=g))
    cache.to_gpu()
    batch.to_gpu()
    k = torch.randn((4, 1, 64), generator=g).bfloat16()
    q = torch.randn((4, 20, 64), generator=g).bfloat16()
    C.run_append(cache, batch, None, k, k, None, 0, False, BF16)
    rows = [i for i in range(count) if new[i]]
    small = C.Batch([3] * 4, [1] * 4, 16, 1)
    small.table, small.pages, small.columns = batch.table[rows], 4, 1
    C.append_ref(cache, small, None, k, k, None, 0, False, None)
    assert all(torch.equal(cache.gpu[n].cpu(), cache.host[n]) for n in cache.host)
    for heads in (2, 20):
        call = C.Attention(cache, batch, q[:, :heads].contiguous(), 0, 0.125, BF16)
        call.run()
        o, lse = call.results()
        C.assert_attention_close(o, lse, C.attention_ref(cache, small, q[:, :heads], 0, 0.125), BF16, 64, 4)
