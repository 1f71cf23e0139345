"""GPU: attention over a paged 8-bit cache with a window does not depend on what lies before the window: slots that no token has
written, pages that have slid out and hold another sequence's tokens or values that are no numbers."""
import pytest
import torch

import paper_2511_03586_amd as perf
from tests import cache_helpers as C

pytestmark = pytest.mark.gpu

F32, BF16 = perf.PERF_F32, perf.PERF_BF16
LARGEST = 0x7E  # 448; with the scale 2^127 more than any of these types holds


def _spoil(cache, batch, window, scale, byte):
    """In the cache on the GPU: pages wholly before the first key that a query sees take `scale` and `byte`, and of the page that
    it lies in the slots before it become NaN."""
    spoiled = 0
    for s in range(batch.sequences):
        low = batch.held[s] - window + 1
        for c in range(-(-max(low, 0) // batch.page_size) if batch.new[s] else 0):
            page, slots = batch.page(s, c * batch.page_size), min(low - c * batch.page_size, batch.page_size)
            whole = slots == batch.page_size
            for name in ("k", "v"):
                cache.gpu[name][page, :, :slots] = byte if whole else C.STALE
                if whole:
                    cache.gpu[name + "s"][page] = scale
            spoiled += slots
    return spoiled


def _check(lows, new, window, page, kv, group, dim, dt, scale, byte):
    """Sequences whose first query sees the keys from `lows` on."""
    batch = C.Batch([max(low + window - 1, 0) for low in lows], new, page, 1)
    cache = C.Cache(batch.pages, kv, page, dim)
    C.fill(cache, batch, 2)
    cache.to_gpu()
    batch.to_gpu()
    q = C.random_queries(batch, kv * group, dim, dt, 3)
    call = C.Attention(cache, batch, q, window, dim ** -0.5, dt)
    call.run()
    o, lse = (x.clone() for x in call.results())
    ref = C.attention_ref(cache, batch, q, window, dim ** -0.5)  # (of the cache on the CPU, which holds numbers everywhere)
    assert all(bool(torch.isfinite(x).all()) for x in ref)
    C.assert_attention_close(o, lse, ref, dt, dim, max(batch.held) + max(new))
    assert _spoil(cache, batch, window, scale, byte)
    call.run()
    after = call.results()
    assert torch.equal(C.bits(o), C.bits(after[0])) and torch.equal(C.bits(lse), C.bits(after[1]))


LOWS = [0, 1, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64, 65, 90, 130]


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("dim,page", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 256), (256, 16), (256, 128)])
@pytest.mark.parametrize("scale,byte", [(C.NO_NUMBER, C.STALE), (254, LARGEST)])
@pytest.mark.parametrize("window", [1, 20, 200])
def test_few_rows(dt, dim, page, scale, byte, window):
    _check(LOWS, [1, 2, 3, 1] * 4, window, page, 2, 4, dim, dt, scale, byte)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("dim,page", [(64, 16), (64, 64), (128, 16), (128, 32), (128, 256), (256, 16), (256, 128)])
@pytest.mark.parametrize("scale,byte", [(C.NO_NUMBER, C.STALE), (254, LARGEST)])
@pytest.mark.parametrize("window", [1, 20, 200])
def test_many_rows(dt, dim, page, scale, byte, window):
    """Row tiles that see all of their window's first block, a part of it, and later ones of the same sequence."""
    _check(LOWS, [20, 33, 70, 17] * 4, window, page, 1, 4, dim, dt, scale, byte)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("new", [[1, 1], [40, 1]])
def test_long_windows(dt, new):
    """Windows whose keys several workgroups divide."""
    _check([4001, 777], new, 5000, 16, 2, 4, 128, dt, C.NO_NUMBER, C.STALE)
