"""Glue and plain references for the tests of the paged 8-bit cache: caches with stale and guarded places, calls through the
binding, and the operators' definitions (appending step by step in float32, attention in float64; torch on the CPU)."""
import math

import numpy as np
import torch

import paper_2511_03586_amd as perf
from tests import gpu_helpers as G
from tests.fp8_helpers import TORCH, Held, at, up

E4M3 = torch.float8_e4m3fn
STALE, NO_NUMBER = 0x7F, 255  # what slots and scales hold that no token has written: NaN


def scale_bytes(amax):
    """The least b >= 1 with amax <= 448 * 2^(b - 127); 255 for what is no finite number."""
    m, e = torch.frexp(amax.double() / 448)  # exact: the quotient of a number by 448 is a power of two only if 448 divides out
    b = (e - (m == 0.5).int() + 127).clamp(min=1)
    b = torch.where(amax == 0, torch.ones_like(b), b)
    return torch.where(torch.isfinite(amax), b, torch.full_like(b, NO_NUMBER))


def power(e):
    return torch.ldexp(torch.ones(e.shape), e)


def rotation_table(positions, rotary, seed=0):
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(rotary // 2, dtype=torch.float64) / (rotary / 2))
    return torch.cat(((angle + seed).cos(), (angle + seed).sin()), 1).float()


def rotate(x, row, rotary, interleaved):
    """x [heads][head_dim] float32, every product and sum rounded."""
    if not rotary:
        return x
    half = rotary // 2
    c, s = row[:half], row[half:]
    y = x.clone()
    i1, i2 = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, half), slice(half, rotary))
    y[:, i1] = x[:, i1] * c - x[:, i2] * s
    y[:, i2] = x[:, i2] * c + x[:, i1] * s
    return y


class Cache:
    """Pages on the CPU (`host`, reference) and on the GPU; every slot and scale starts stale."""

    def __init__(self, pages, kv_heads, page_size, head_dim):
        self.pages, self.kv_heads, self.page_size, self.head_dim = pages, kv_heads, page_size, head_dim
        shape = (pages, kv_heads, page_size, head_dim)
        self.host = {"k": torch.full(shape, STALE, dtype=torch.uint8), "v": torch.full(shape, STALE, dtype=torch.uint8),
                     "ks": torch.full((pages, kv_heads), NO_NUMBER, dtype=torch.uint8),
                     "vs": torch.full((pages, kv_heads), NO_NUMBER, dtype=torch.uint8)}
        self.marked = {name: torch.zeros((pages, kv_heads), dtype=torch.bool) for name in ("k", "v")}  # blocks that took no number

    def to_gpu(self):
        self.gpu = {k: v.cuda() for k, v in self.host.items()}

    def values(self, name, page, head, slots):
        """float64 values of slots, as the bytes stand for them."""
        b = int(self.host[name + "s"][page, head])
        q = self.host[name][page, head, :slots].view(E4M3).double()
        return q * 2.0 ** (b - 127) if b != NO_NUMBER else q * math.nan

    def append(self, name, page, slot0, x):
        """x [tokens][kv_heads][head_dim] float32 into slots from slot0 on."""
        for h in range(self.kv_heads):
            need = scale_bytes(x[:, h].abs().amax())
            need = torch.tensor(NO_NUMBER) if not bool(torch.isfinite(x[:, h]).all()) else need
            before = int(self.host[name + "s"][page, h]) if slot0 else 0
            b = max(before, int(need))
            held = self.host[name][page, h]
            if b > before and slot0 and b != NO_NUMBER:
                held[:slot0] = (held[:slot0].view(E4M3).float() * power(torch.tensor(before - b))).to(E4M3).view(torch.uint8)
            self.host[name + "s"][page, h] = b
            self.marked[name][page, h] = b == NO_NUMBER
            if b != NO_NUMBER:
                held[slot0:slot0 + x.shape[0]] = (x[:, h] * power(torch.tensor(127 - b))).to(E4M3).view(torch.uint8)


class Batch:
    """Sequences of `held` and `new` tokens with pages in shuffled order; `absent` (sequence, column) entries have none."""

    def __init__(self, held, new, page_size, seed=0, absent=(), spare=2, padding=0, pad_columns=1):
        g = torch.Generator().manual_seed(seed)
        self.held, self.new, self.page_size = list(held), list(new), page_size
        self.sequences, self.tokens = len(held), sum(new) + padding
        need = [up(a + n, page_size) for a, n in zip(held, new)]
        self.columns = max(need) + pad_columns
        self.pages = sum(need) + spare
        order = torch.randperm(self.pages, generator=g).int()
        self.table = torch.full((self.sequences, self.columns + 3), -1, dtype=torch.int32)
        first = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[first:first + n]
            first += n
        for i, (s, c) in enumerate(absent):
            self.table[s, c] = (-1, self.pages, -7, 2 ** 31 - 1)[i % 4]
        self.lengths = torch.tensor(self.held, dtype=torch.int32)
        self.cu = torch.tensor([0] + self.new).cumsum(0).int()

    def to_gpu(self):
        self.dev = [x.cuda() for x in (self.table, self.lengths, self.cu)]

    def addresses(self):
        return [x.data_ptr() for x in self.dev]

    def page(self, s, position):
        """The page of a position, or None."""
        c = position // self.page_size
        p = int(self.table[s, c]) if c < self.columns else -1
        return p if 0 <= p < self.pages else None

    def rows(self):
        return [(s, int(self.cu[s]) + i, self.held[s] + i) for s in range(self.sequences) for i in range(self.new[s])]


def fill(cache, batch, seed, upto_new=True):
    """Random tokens for every position of the batch's sequences that has a page."""
    g = torch.Generator().manual_seed(seed)
    for s in range(batch.sequences):
        for c in range(up(batch.held[s] + (batch.new[s] if upto_new else 0), batch.page_size)):
            end = batch.held[s] + (batch.new[s] if upto_new else 0) - c * batch.page_size
            page, n = batch.page(s, c * batch.page_size), min(end, batch.page_size)
            if page is None:
                continue
            for name in ("k", "v"):
                x = torch.randn((n, cache.kv_heads, cache.head_dim), generator=g) * torch.exp(0.5 * torch.randn((1, cache.kv_heads, 1), generator=g))
                cache.append(name, page, 0, x)


# ---- appending --------------------------------------------------------------------------------------
def append_ref(cache, batch, q, k, v, rotation, rotary, interleaved, q_out):
    """Moves cache.host on and returns the rotated queries (rows without one: as q_out has them)."""
    positions = rotation.shape[0] if rotary else 1 << 30
    out = q_out.clone() if q is not None else None
    units = {}
    for s, row, p in batch.rows():
        if p >= positions:
            continue
        turn = rotation[p] if rotary else None
        if q is not None:
            out[row] = rotate(q[row].float(), turn, rotary, interleaved).to(q.dtype)
        page = batch.page(s, p)
        if page is not None:
            units.setdefault((page, s), []).append((p % batch.page_size, rotate(k[row].float(), turn, rotary, interleaved), v[row].float()))
    for (page, _), tokens in units.items():
        cache.append("k", page, tokens[0][0], torch.stack([t[1] for t in tokens]))
        cache.append("v", page, tokens[0][0], torch.stack([t[2] for t in tokens]))
    return out


def run_append(cache, batch, q, k, v, rotation, rotary, interleaved, dt, pad=0, offset=0, in_place=False, stream=None):
    """q, k, v [tokens][heads][head_dim] CPU; rows `pad` elements wider than the heads. The cache on the GPU moves on; the rotated
    queries come back."""
    d, kv = cache.head_dim, cache.kv_heads
    hold = lambda x: None if x is None else Held(x.shape[0], x.shape[1] * d, dt, x.shape[1] * d + pad, offset, x.flatten(1))  # noqa: E731
    qd, kd, vd = hold(q), hold(k), hold(v)
    out = None if q is None else qd if in_place else Held(qd.rows, qd.cols, dt, qd.cols + 2 * pad, offset)
    turn = rotation.cuda() if rotary else None
    c = cache.gpu
    perf.perf_cache_append_fp8(at(qd), at(kd), at(vd), turn.data_ptr() if rotary else None, at(out), c["k"].data_ptr(), c["v"].data_ptr(),
                               c["ks"].data_ptr(), c["vs"].data_ptr(), *batch.addresses(), batch.tokens, batch.sequences,
                               q.shape[1] if q is not None else kv, kv, d, qd.ld if qd else 0, kd.ld, vd.ld, out.ld if out else 0,
                               cache.pages, batch.page_size, batch.columns, batch.table.shape[1], rotary,
                               rotation.shape[0] if rotary else 0, int(interleaved), dt, stream=G.stream() if stream is None else stream)
    torch.cuda.synchronize()
    return None if out is None else out.get().view(q.shape)


def guard_rows(shape, dt):
    """What a Held that was never written holds."""
    return Held(shape[0], shape[1] * shape[2], dt).get().view(shape)


# ---- attention --------------------------------------------------------------------------------------
def attention_ref(cache, batch, q, window, scale):
    """o, lse in float64 (NaN rows: not computed), and two bounds' ingredients for each row and head: the magnitudes of the
    weighted values (as o) and of the score's terms (as lse, the largest of a key)."""
    d, kv = cache.head_dim, cache.kv_heads
    hq = q.shape[1]
    group = hq // kv
    o = torch.full(q.shape, math.nan, dtype=torch.float64)
    lse, terms = (torch.full(q.shape[:2], math.nan, dtype=torch.float64) for _ in range(2))
    mag = torch.zeros(q.shape, dtype=torch.float64)
    for s in range(batch.sequences):
        a, n, first = batch.held[s], batch.new[s], int(batch.cu[s])
        if n == 0:
            continue
        keys, ks, vs = [], [], []
        for c in range(up(a + n, batch.page_size)):
            page, m = batch.page(s, c * batch.page_size), min(batch.page_size, a + n - c * batch.page_size)
            if page is not None:
                keys += range(c * batch.page_size, c * batch.page_size + m)
                ks.append(torch.stack([cache.values("k", page, h, m) for h in range(kv)]))
                vs.append(torch.stack([cache.values("v", page, h, m) for h in range(kv)]))
        position = a + torch.arange(n)[:, None]
        keys = torch.tensor(keys, dtype=torch.int64)
        seen = keys[None] <= position
        if window:
            seen &= keys[None] > position - window
        for h in range(hq):
            rows = slice(first, first + n)
            o[rows, h], lse[rows, h], terms[rows, h] = 0.0, -math.inf, 0.0
            if not ks:
                continue
            k, v = torch.cat(ks, 1)[h // group], torch.cat(vs, 1)[h // group]
            x = q[rows, h].double()
            scores = torch.where(seen, scale * (x @ k.T), -math.inf)
            some = seen.any(1)
            lse[rows, h] = torch.logsumexp(scores, 1)
            w = torch.where(some[:, None], torch.exp(scores - torch.where(some, lse[rows, h], 0.0)[:, None]), 0.0)
            o[rows, h], mag[rows, h] = w @ v, w @ v.abs()
            terms[rows, h] = torch.where(seen, abs(scale) * (x.abs() @ k.abs().T), 0.0).amax(1)
    return o, lse, mag, terms


class Attention:
    """One call's buffers; run() may be repeated."""

    def __init__(self, cache, batch, q, window, scale, dt, pad=0, offset=0, max_tokens=None, want_lse=True):
        self.cache, self.batch, self.dt, self.window, self.scale = cache, batch, dt, window, scale
        self.shape, self.hq = q.shape, q.shape[1]
        width = q.shape[1] * cache.head_dim
        self.q = Held(q.shape[0], width, dt, width + pad, offset, q.flatten(1))
        self.o = Held(q.shape[0], width, dt, width + 2 * pad, offset)
        self.lse = Held(q.shape[0], self.hq, perf.PERF_F32) if want_lse else None
        self.max_tokens = max_tokens or max(1, max(batch.new))
        size = perf.perf_cache_attention_fp8_workspace_bytes(batch.tokens, batch.sequences, self.max_tokens, self.hq, cache.kv_heads,
                                                             cache.head_dim, batch.page_size, batch.columns)
        assert size >= 0
        self.ws = torch.full((size + 64,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN; the last bytes are a guard

    def run(self, stream=None):
        c, b = self.cache, self.batch
        perf.perf_cache_attention_fp8(self.q.at(), c.gpu["k"].data_ptr(), c.gpu["v"].data_ptr(), c.gpu["ks"].data_ptr(), c.gpu["vs"].data_ptr(),
                                      *b.addresses(), self.o.at(), at(self.lse), self.ws.data_ptr(), b.tokens, b.sequences,
                                      self.max_tokens, self.hq, c.kv_heads, c.head_dim, self.q.ld, self.o.ld, c.pages, b.page_size,
                                      b.columns, b.table.shape[1], self.window, self.scale, self.dt,
                                      stream=G.stream() if stream is None else stream)

    def results(self):
        torch.cuda.synchronize()
        assert bool((self.ws[-64:] == 0xFF).all()), "written behind the workspace"
        return self.o.get().view(self.shape), self.lse.get() if self.lse else None


def assert_attention_close(o, lse, ref, dt, head_dim, keys):
    """o = sum w v / sum w.  A score is a sum of head_dim products, each exact or within 2^-24, in fp32: off by at most
    e = (head_dim + 4) 2^-24 of its terms' magnitudes, and by 2 roundings of the score itself on its way to the exponential, whose
    argument, at most 2 |terms| + 1, may be rounded once more and whose result is within 2^-22.  That moves a weight by a factor
    within 2 e + ...; numerator and denominator both.  Sums over the keys: their number times 2^-24.  bf16: the weights in the
    numerator are rounded (2^-8), and the result is (2^-8 of it; fp32: 2^-24)."""
    ro, rlse, mag, terms = ref
    some = ~torch.isnan(ro)
    half = 2.0 ** -8 if dt == perf.PERF_BF16 else 2.0 ** -24
    score = ((head_dim + 4) + 8) * 2.0 ** -24 * terms
    rel = 2 * score + 2.0 ** -21 + 2 * (keys + 8) * 2.0 ** -24 + (2.0 ** -8 if dt == perf.PERF_BF16 else 2.0 ** -23)
    bound = rel[:, :, None] * mag * (1 + half) + half * ro.abs()
    diff = (o.double() - ro).abs()
    assert bool((diff <= bound)[some].all()), float((diff / bound.clamp(min=1e-300))[some].max())
    if lse is not None:
        rows = ~torch.isnan(rlse)
        empty = rows & (rlse == -math.inf)
        assert bool((lse[empty] == -math.inf).all()) and bool((o[empty] == 0).all())
        full = rows & ~empty
        off = (lse.double() - rlse).abs()
        assert bool((off <= score + 2.0 ** -21 + (keys + 8) * 2.0 ** -24 + 2.0 ** -22 * rlse.abs())[full].all()), float(off[full].max())


def bits(x):
    return x.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()])


def assert_left_alone(o, ref):
    """Rows that no sequence has hold what they held."""
    alone = torch.isnan(ref[0])
    assert bool((bits(o)[alone] == bits(guard_rows(o.shape, perf.PERF_BF16 if o.dtype == torch.bfloat16 else perf.PERF_F32))[alone]).all())


def random_queries(batch, heads, head_dim, dt, seed, std=2.0):
    g = torch.Generator().manual_seed(seed)
    return (std * torch.randn((batch.tokens, heads, head_dim), generator=g)).to(TORCH[dt])


def as_f64(x):
    return np.asarray(x.double())
