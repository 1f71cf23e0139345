"""GPU: appending to a paged 8-bit cache (bit for bit) and the attention that reads it (against float64), at the sizes, masks and
orders where they can go wrong."""
import math

import pytest
import torch

import paper_2511_03586_amd as perf
from tests import cache_helpers as C
from tests.fp8_helpers import TORCH

pytestmark = pytest.mark.gpu

F32, BF16 = perf.PERF_F32, perf.PERF_BF16


# ---- appending ------------------------------------------------------------------------------------
def _tokens(batch, heads, head_dim, dt, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((batch.tokens, heads, head_dim), generator=g) * torch.exp(torch.randn((batch.tokens, heads, 1), generator=g))
    return x.to(TORCH[dt])


def _check_append(held, new, page, kv, group, dim, dt, rotary, interleaved=False, positions=None, absent=(), padding=0, pad=0, offset=0,
                  in_place=False, queries=True, change=None):
    batch = C.Batch(held, new, page, 1, absent, padding=padding)
    cache = C.Cache(batch.pages, kv, page, dim)
    C.fill(cache, batch, 2, upto_new=False)
    cache.to_gpu()
    batch.to_gpu()
    q = _tokens(batch, kv * group, dim, dt, 3) if queries else None
    k, v = _tokens(batch, kv, dim, dt, 4), _tokens(batch, kv, dim, dt, 5)
    if change:
        change(k, v)
    turn = C.rotation_table(positions or max(a + n for a, n in zip(held, new)), rotary) if rotary else None
    out = C.run_append(cache, batch, q, k, v, turn, rotary, interleaved, dt, pad, offset, in_place)
    blank = q if in_place else C.guard_rows(q.shape, dt) if queries else None
    ref = C.append_ref(cache, batch, q, k, v, turn, rotary, interleaved, blank)
    if queries:
        assert torch.equal(C.bits(out), C.bits(ref))
    for name in ("ks", "vs"):
        assert torch.equal(cache.gpu[name].cpu(), cache.host[name]), name
    for name in ("k", "v"):
        number = ~cache.marked[name]  # (a block that took no number reads as NaN whatever its bytes are)
        assert torch.equal(cache.gpu[name].cpu()[number], cache.host[name][number]), name
    return cache


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (128, 128), (128, 256), (256, 32), (256, 256), (64, 256)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_runs_of_tokens(dt, dim, page, interleaved):
    """Runs that begin and end inside pages, at their borders, cover some whole, and single tokens."""
    _check_append([0, 5, page - 1, page, 3 * page + 7, 2 * page - 3, 0], [1, 3 * page, 1, 1, 2 * page - 7, 4, 2 * page], page, 2, 3, dim, dt,
                  dim, interleaved)


@pytest.mark.parametrize("rotary,interleaved", [(0, False), (16, False), (96, False), (48, False), (16, True), (112, True)])
def test_append_part_of_the_head_is_rotated(rotary, interleaved):
    _check_append([0, 9, 40], [20, 40, 1], 16, 3, 1, 128, BF16, rotary, interleaved)


@pytest.mark.parametrize("kv,group", [(1, 1), (1, 16), (5, 1), (3, 7), (8, 4)])
def test_append_heads(kv, group):
    _check_append([3, 0, 17], [1, 50, 16], 32, kv, group, 64, BF16, 64)


def test_append_strides_and_alignments():
    _check_append([3, 0, 17], [1, 50, 16], 32, 2, 2, 64, BF16, 64, pad=5, offset=3)
    _check_append([3, 0, 17], [1, 50, 16], 32, 2, 2, 64, F32, 64, pad=3, offset=1)


@pytest.mark.parametrize("interleaved", [False, True])
def test_append_queries_in_place_and_without(interleaved):
    _check_append([3, 0, 17], [1, 50, 16], 32, 2, 2, 128, BF16, 128, interleaved, in_place=True)
    _check_append([3, 0, 17], [1, 50, 16], 32, 2, 2, 128, BF16, 128, interleaved, queries=False)


def test_append_many_sequences():
    """More sequences than the wave looks at in one step, some of which bring nothing; rows behind the last."""
    held = [(7 * i) % 90 for i in range(300)]
    new = [(0, 1, 1, 5, 0, 40)[i % 6] for i in range(300)]
    _check_append(held, new, 16, 1, 2, 64, BF16, 64, padding=37)
    _check_append([4] * 65, [0] * 64 + [3], 16, 1, 1, 64, BF16, 0)
    _check_append([4] * 65, [3] + [0] * 64, 16, 1, 1, 64, BF16, 0)


def test_append_a_run_among_single_tokens():
    """One sequence brings more tokens of a page than a wave holds in registers."""
    for dt in (BF16, F32):
        _check_append([5] * 40 + [3] + [9] * 30, [1] * 40 + [60] + [1] * 30, 256, 2, 1, 256, dt, 256)


def test_append_positions_and_pages_that_are_not_there():
    """Positions behind the rotation's end, columns behind the table's, entries that are no page."""
    _check_append([0, 30, 70, 100], [90, 60, 1, 2], 16, 2, 1, 64, BF16, 64, positions=75)
    _check_append([0, 30, 70], [90, 60, 1], 16, 2, 1, 64, BF16, 64, absent=((0, 1), (0, 5), (1, 2), (2, 4)))


def test_append_beyond_the_table():
    batch = C.Batch([30], [5], 16, 1)
    cache = C.Cache(batch.pages, 1, 16, 64)
    C.fill(cache, batch, 2, upto_new=False)
    cache.to_gpu()
    batch.columns = 2  # positions 32 to 34 have no column
    batch.to_gpu()
    k = _tokens(batch, 1, 64, BF16, 3)
    C.run_append(cache, batch, None, k, k, None, 0, False, BF16)
    C.append_ref(cache, batch, None, k, k, None, 0, False, None)
    assert all(torch.equal(cache.gpu[n].cpu(), cache.host[n]) for n in cache.host)


def test_append_bad_lengths_and_rows():
    """A sequence of negative length brings nothing; the others are served."""
    batch = C.Batch([5, 6, 7], [4, 4, 4], 16, 1)
    cache = C.Cache(batch.pages, 1, 16, 64)
    C.fill(cache, batch, 2, upto_new=False)
    cache.to_gpu()
    batch.lengths[1] = -3
    batch.to_gpu()
    k = _tokens(batch, 1, 64, BF16, 3)
    q = _tokens(batch, 2, 64, BF16, 4)
    out = C.run_append(cache, batch, q, k, k, None, 0, False, BF16)
    batch.new = [4, 0, 4]
    ref = C.append_ref(cache, batch, q, k, k, None, 0, False, C.guard_rows(q.shape, BF16))
    assert torch.equal(C.bits(out), C.bits(ref))
    assert all(torch.equal(cache.gpu[n].cpu(), cache.host[n]) for n in cache.host)


def test_append_values_at_the_ends():
    """Blocks of zeros, of the smallest and of the largest numbers, and maxima at a scale's border."""
    def change(k, v):
        k[0], v[0] = 0.0, 448.0
        k[1], v[1] = 448.0 * 2.0 ** 20, 450.0
        k[2], v[2] = 2.0 ** -130, 3.3e38
        k[3], v[3] = -449.0, 2.0 ** -126
    for dt in (BF16, F32):
        _check_append([0, 0, 0, 0], [1, 1, 1, 1], 16, 1, 1, 64, dt, 0, change=change)
        _check_append([3, 3, 3, 3], [1, 1, 1, 1], 16, 1, 1, 64, dt, 0, change=change)


def test_append_infinities_and_nan_mark_their_block():
    def change(k, v):
        k[0, 0, 5], v[1, 1, 63], k[2, 1, 0] = math.inf, math.nan, -math.inf
    cache = _check_append([0, 4, 9], [1, 6, 30], 16, 2, 1, 64, BF16, 0, change=change)
    assert int(cache.marked["k"].sum()) == 2 and int(cache.marked["v"].sum()) == 1


def test_append_token_by_token_is_append_at_once():
    """Power-of-two scales: the bytes do not depend on how many calls brought them, but for values that a larger scale made
    subnormal (rounded twice: off by at most one step of 2^-9)."""
    page, kv, dim, n = 32, 2, 64, 70
    g = torch.Generator().manual_seed(1)
    x = torch.randn((n, kv, dim), generator=g) * torch.exp(torch.randn((n, kv, 1), generator=g))
    k = x.bfloat16()
    turn = C.rotation_table(n, dim)
    caches = []
    for steps in ([n], [1] * n, [13, 1, 40, 16]):
        done, cache = 0, None
        for m in steps:
            batch = C.Batch([done], [m], page, 7, pad_columns=-(-n // page) - -(-(done + m) // page))
            batch.pages, batch.table = 6, torch.tensor([[4, 0, 3, -1]], dtype=torch.int32)
            batch.to_gpu()
            if cache is None:
                cache = C.Cache(6, kv, page, dim)
                cache.to_gpu()
            C.run_append(cache, batch, None, k[done:done + m], k[done:done + m], turn, dim, False, BF16)
            done += m
        caches.append({name: t.cpu() for name, t in cache.gpu.items()})
    for other in caches[1:]:
        for name in ("k", "v"):
            assert torch.equal(other[name + "s"], caches[0][name + "s"])
            a, b = caches[0][name].view(C.E4M3).float(), other[name].view(C.E4M3).float()
            same = torch.equal(torch.isnan(a), torch.isnan(b))
            assert same and bool(((a - b).abs().nan_to_num() <= torch.where(a.abs() <= 2.0 ** -6, 2.0 ** -9, 0.0)).all())


# ---- attention ------------------------------------------------------------------------------------
def _attention(held, new, page, kv, group, dim, dt, window=0, absent=(), padding=0, scale=None, seed=1, **more):
    batch = C.Batch(held, new, page, seed, absent, padding=padding)
    cache = C.Cache(batch.pages, kv, page, dim)
    C.fill(cache, batch, seed + 1)
    cache.to_gpu()
    batch.to_gpu()
    q = C.random_queries(batch, kv * group, dim, dt, seed + 2)
    scale = dim ** -0.5 if scale is None else scale
    return cache, batch, q, C.Attention(cache, batch, q, window, scale, dt, **more)


def _check_attention(*args, **kw):
    cache, batch, q, call = _attention(*args, **kw)
    call.run()
    o, lse = call.results()
    ref = C.attention_ref(cache, batch, q, call.window, call.scale)
    keys = max(a + n for a, n in zip(batch.held, batch.new))
    C.assert_attention_close(o, lse, ref, call.dt, cache.head_dim, keys)
    C.assert_left_alone(o, ref)
    return o, lse, ref


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_attention_single_tokens(dt, dim, page):
    """One new token on lengths around pages, tiles and their multiples."""
    _check_attention([0, 1, 14, 15, 16, 30, 31, 32, 33, 62, 63, 64, 127, 128, 129, 255, 256, 300, 700], [1] * 19, page, 2, 4, dim, dt)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("kv,group", [(1, 1), (5, 1), (2, 3), (1, 7), (2, 8), (1, 16), (1, 17), (1, 33), (2, 40), (1, 128)])
def test_attention_heads(dt, kv, group):
    _check_attention([0, 70, 200], [1, 1, 1], 16, kv, group, 64, dt)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("new", [2, 3, 5, 8, 16, 17, 33])
@pytest.mark.parametrize("group", [1, 4, 6])
def test_attention_a_few_tokens(dt, new, group):
    _check_attention([0, 61, 130, 250], [new, new, 1, new], 32, 2, group, 64, dt)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("dim,page", [(64, 16), (64, 64), (128, 64), (128, 256), (256, 32)])
def test_attention_long_runs(dt, dim, page):
    """Prompts from nothing and on held tokens, beside single tokens and sequences that bring none."""
    _check_attention([0, 37, 0, 129, 64], [200, 129, 0, 1, 128], page, 2, 2, dim, dt, padding=9)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("window", [1, 2, 16, 33, 100, 1000])
def test_attention_windows(dt, window):
    _check_attention([0, 130, 200, 511], [1, 1, 70, 200], 16, 1, 4, 64, dt, window=window)
    _check_attention([0, 130, 200, 511, 300], [1, 1, 2, 4, 3], 32, 2, 4, 128, dt, window=window)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_attention_pages_that_are_not_there(dt):
    """Their keys are not seen; a query that sees none gets zeros."""
    absent = ((0, 0), (1, 0), (1, 1), (1, 2), (2, 3), (2, 4), (3, 0))
    _check_attention([3, 40, 100, 0], [1, 1, 1, 12], 16, 2, 2, 64, dt, absent=absent)
    _check_attention([3, 0, 100, 0], [8, 48, 60, 40], 16, 2, 4, 64, dt, absent=absent)
    _check_attention([500, 600], [1, 50], 16, 1, 4, 128, dt, window=40, absent=tuple((s, c) for s in (0, 1) for c in range(28)))


def test_attention_columns_that_are_not_there():
    for new in (1, 40):
        batch = C.Batch([30], [new], 16, 1)
        cache = C.Cache(batch.pages, 1, 16, 64)
        C.fill(cache, batch, 2)
        cache.to_gpu()
        batch.columns = 2
        batch.to_gpu()
        q = C.random_queries(batch, 4, 64, BF16, 3)
        call = C.Attention(cache, batch, q, 0, 0.125, BF16)
        call.run()
        o, lse = call.results()
        C.assert_attention_close(o, lse, C.attention_ref(cache, batch, q, 0, 0.125), BF16, 64, 80)


def test_attention_bad_lengths_and_more_tokens_than_said():
    cache, batch, q, call = _attention([5, 60, 70], [4, 4, 40], 16, 1, 2, 64, BF16, max_tokens=4)
    batch.lengths[1] = -1
    batch.to_gpu()
    call.run()
    o, lse = call.results()
    ref = C.attention_ref(cache, batch, q, 0, call.scale)
    ref[0][4:8], ref[1][4:8] = math.nan, math.nan
    ref[0][12:], ref[1][12:] = math.nan, math.nan
    C.assert_attention_close(o, lse, ref, BF16, 64, 200)
    C.assert_left_alone(o, ref)


@pytest.mark.parametrize("scale", [0.0, -0.3, 40.0])
def test_attention_scales(scale):
    """All keys alike, the least first, and scores far apart."""
    for dt in (BF16, F32):
        _check_attention([0, 200, 90], [1, 1, 70], 16, 2, 2, 64, dt, scale=scale)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_attention_many_sequences(dt):
    held = [(37 * i) % 190 for i in range(200)]
    _check_attention(held, [(1, 0, 2, 1, 1)[i % 5] for i in range(200)], 16, 1, 2, 64, dt, padding=11)
    _check_attention(held, [(1, 0, 20, 1, 3)[i % 5] for i in range(200)], 16, 1, 4, 64, dt, padding=11)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_attention_long_contexts(dt):
    _check_attention([20000, 3, 9000], [1, 1, 1], 64, 1, 4, 128, dt)
    _check_attention([9000, 20], [150, 60], 64, 1, 4, 64, dt)


def test_attention_strides_alignments_and_no_lse():
    for dt, pad, offset in ((BF16, 3, 1), (F32, 5, 1), (BF16, 8, 8)):
        for new in ([1, 1], [3, 40]):
            _check_attention([20, 100], new, 16, 2, 2, 64, dt, pad=pad, offset=offset)
            cache, batch, q, call = _attention([20, 100], new, 16, 2, 2, 64, dt, pad=pad, offset=offset, want_lse=False)
            call.run()
            C.assert_attention_close(call.results()[0], None, C.attention_ref(cache, batch, q, 0, 0.125), dt, 64, 200)


def test_attention_shared_pages():
    """Two sequences with the same first pages."""
    for new in ([1, 1], [40, 30]):
        batch = C.Batch([64, 64], new, 16, 3)
        batch.table[1, :4] = batch.table[0, :4]
        cache = C.Cache(batch.pages, 2, 16, 64)
        C.fill(cache, batch, 4)
        cache.to_gpu()
        batch.to_gpu()
        q = C.random_queries(batch, 4, 64, BF16, 5)
        call = C.Attention(cache, batch, q, 0, 0.125, BF16)
        call.run()
        o, lse = call.results()
        C.assert_attention_close(o, lse, C.attention_ref(cache, batch, q, 0, 0.125), BF16, 64, 110)


@pytest.mark.parametrize("new", [[1, 1, 1], [1, 9, 130]])
def test_attention_marked_block_is_nan_where_it_is_seen(new):
    """A sequence whose block took no number; the others' results are what they are without it."""
    cache, batch, q, call = _attention([70, 100, 200], new, 16, 2, 2, 64, BF16)
    call.run()
    before = call.results()[0].clone()
    cache.gpu["ks"][batch.page(1, 20), 1] = C.NO_NUMBER
    call.run()
    after = call.results()[0]
    rows = slice(int(batch.cu[1]), int(batch.cu[2]))
    others = torch.ones(batch.tokens, dtype=torch.bool)
    others[rows] = False
    assert torch.equal(C.bits(before)[others], C.bits(after)[others])
    assert torch.equal(C.bits(before)[rows, :2], C.bits(after)[rows, :2]) and bool(torch.isnan(after[rows, 2:]).all())


def test_attention_twice_is_the_same():
    for args in (([3000, 5, 800], [1, 1, 1]), ([900, 0, 33], [64, 200, 1])):
        _, _, _, call = _attention(*args, 32, 2, 4, 128, BF16)
        call.run()
        o, lse = (x.clone() for x in call.results())
        call.ws.fill_(0xFF)
        call.run()
        again = call.results()
        assert torch.equal(C.bits(o), C.bits(again[0])) and torch.equal(C.bits(lse), C.bits(again[1]))
