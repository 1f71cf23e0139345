"""Performance cases of a block's attention in serving: appending keys and values to a paged cache in 8 bits, with the position
rotation on the way, and the attention that reads that cache, for single tokens, a few and long runs of them.

A case is a dict of plain values; ``op`` names the operator. ``listed()`` holds the fixed cases, ``draw(rng)`` one more from
the same ranges. ``prepare`` makes the device buffers that a program holds before it calls, ``run`` is one call: of the
library where ``own`` is true, of the operator's plain form in elementary torch operations where it is not. ``exact`` is the
operator's definition in float64.

Sequence s holds ``lengths[s]`` tokens and brings those from ``cu[s]`` to ``cu[s + 1]``, at the positions that follow. A token
of position p lies in slot p % page of page ``table[s][p / page]``; keys and values are e4m3, [pages][kv_heads][page][head_dim], and
a byte b for each page and head, [pages][kv_heads], is their scale 2^(b - 127).
"""
import math
import random

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_CODE = {"f32": 0, "bf16": 1}  # PERF_F32, PERF_BF16
_E4M3 = torch.float8_e4m3fn


def _append(name, dtype, sequences, held, new, heads, head_dim, page, rotary, interleaved=False):
    return {"name": name, "op": "append", "dtype": dtype, "sequences": sequences, "held_least": held[0], "held_most": held[1],
            "new_least": new[0], "new_most": new[1], "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "page": page,
            "rotary": rotary, "interleaved": interleaved}


def _attention(name, dtype, sequences, held, new, heads, head_dim, page, window=0):
    return {"name": name, "op": "attention", "dtype": dtype, "sequences": sequences, "held_least": held[0], "held_most": held[1],
            "new_least": new[0], "new_most": new[1], "q_heads": heads[0], "kv_heads": heads[1], "head_dim": head_dim, "page": page,
            "window": window}


def listed():
    return [
        # two conversations, one token each: bound by the launch
        _append("append_bf16_2x1", "bf16", 2, (100, 700), (1, 1), (8, 2), 64, 16, 64),
        # a decoding step of a large batch: every token opens its page again
        _append("append_bf16_192x1", "bf16", 192, (40, 2000), (1, 1), (32, 8), 128, 64, 128),
        # prompts of a few thousand tokens
        _append("append_bf16_4x2048", "bf16", 4, (0, 900), (1500, 2700), (32, 8), 128, 64, 128),
        # float32 activations, wide heads of which a part is rotated, neighbours paired, pages that begin half full
        _append("append_f32_3x500", "f32", 3, (5, 77), (300, 517), (6, 2), 256, 32, 96, True),
        # one conversation's next token: bound by the launch
        _attention("attention_bf16_1x1_on_700", "bf16", 1, (700, 700), (1, 1), (16, 16), 64, 16),
        # a decoding step of a small batch, grouped heads
        _attention("attention_bf16_16x1_on_4096", "bf16", 16, (2048, 6000), (1, 1), (32, 8), 128, 64),
        # a decoding step of a large batch whose lengths differ by a factor of 500
        _attention("attention_bf16_64x1_on_32768", "bf16", 64, (64, 32768), (1, 1), (32, 8), 128, 32),
        # one long document
        _attention("attention_bf16_1x1_on_131071", "bf16", 1, (131071, 131071), (1, 1), (32, 8), 128, 128),
        # drafted tokens under check, in float32, every head with keys of its own, a window
        _attention("attention_f32_6x5_on_4000", "f32", 6, (300, 4000), (5, 5), (10, 10), 256, 16, 1000),
        # prompts of a few thousand tokens
        _attention("attention_bf16_4x2048", "bf16", 4, (0, 0), (1800, 2300), (32, 8), 128, 64),
        # prompts beside conversations in one batch: from one new token to a chunk of a prompt
        _attention("attention_bf16_20x512_on_12000", "bf16", 20, (200, 12000), (1, 512), (32, 8), 128, 64),
        # the attention shapes of the scores and softmax: 32 sequences of 512 tokens, 16 heads of 64
        _attention("attention_bf16_32x512", "bf16", 32, (0, 0), (512, 512), (16, 16), 64, 64),
    ]


# ---- lengths --------------------------------------------------------------------------------------
def _lengths(count, least, most, order):
    """`count` whole numbers from least to most, each a factor beyond the one before, in a shuffled order."""
    ratio = (most + 1) / (least + 1)
    v = [round((least + 1) * ratio ** (i / max(1, count - 1))) - 1 for i in range(count)]
    random.Random(order).shuffle(v)
    return v


def _held(case):
    return _lengths(case["sequences"], case["held_least"], case["held_most"], 1)


def _new(case):
    return _lengths(case["sequences"], case["new_least"], case["new_most"], 2)


def _pages(case):
    """Pages of each sequence behind the call."""
    return [-(-(a + b) // case["page"]) for a, b in zip(_held(case), _new(case))]


# ---- drawn cases ----------------------------------------------------------------------------------
def _size(rng, lo, hi):
    """A whole number in [lo, hi], uniform in its logarithm: three in ten regular, the others any."""
    v = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return max(lo, v // 16 * 16) if v >= 32 and rng.random() < 0.3 else v


def draw(rng):
    while True:
        kv = rng.choice([1, 2, 4, 8, 8, rng.randint(1, 12)])
        group = rng.choice([1, 2, 4, 4, 8, rng.randint(1, 16)])
        dtype, dim = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.choice([64, 128, 128, 256])
        page = rng.choice([16, 16, 32, 64, 64, 128, 256])
        sequences = _size(rng, 1, 128)
        if rng.random() < 0.4:
            held = sorted((_size(rng, 1, 4000), _size(rng, 1, 4000)))
            new = rng.choice([(1, 1), (1, _size(rng, 1, 64)), sorted((_size(rng, 1, 4096), _size(rng, 1, 4096)))])
            rotary = rng.choice([dim, dim, dim // 2, 16 * rng.randint(1, dim // 16), 0])
            case = _append("", dtype, sequences, held, new, (kv * group, kv), dim, page, rotary, rng.random() < 0.3)
        else:
            held = sorted((_size(rng, 1, 40000), _size(rng, 1, 40000)))
            new = rng.choice([(1, 1), (1, 1), (1, 1), (1, _size(rng, 1, 8)), (1, _size(rng, 1, 1024)),
                              sorted((_size(rng, 1, 4096), _size(rng, 1, 4096)))])
            if new[0] > 64 and rng.random() < 0.5:
                held = (0, 0)
            window = rng.choice([0, 0, 0, _size(rng, 16, 8192)])
            case = _attention("", dtype, sequences, held, new, (kv * group, kv), dim, page, window)
        del case["name"]
        w = work(case)
        cache = 2 * sum(_pages(case)) * page * kv * dim
        scores = max(a * (a + b) for a, b in zip(_new(case), _held(case))) * kv * group
        if case["op"] == "append" and w["bytes"] <= 1.8e8 and cache <= 3e8:
            return case
        if case["op"] == "attention" and w["bytes"] <= 6.5e8 and cache <= 8e8 and scores <= 5e8 and \
                w["flops"] <= (1.2e11 if dtype == "bf16" else 4e10):
            return case


# ---- what a program holds -------------------------------------------------------------------------
def _scale_bytes(amax):
    """The least b >= 1 for which amax <= 448 * 2^(b - 127), from the bits of amax (float32): 448 is 1.75 * 2^8."""
    bits = amax.view(torch.int32)
    return ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(min=1)


def _power(e):
    """2^e in float32, e from -126 to 127."""
    return ((e + 127) << 23).view(torch.float32)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    held, new, pages = _held(case), _new(case), _pages(case)
    kv, dim, page, dt = case["kv_heads"], case["head_dim"], case["page"], _TORCH[case["dtype"]]
    tokens, count = sum(new), sum(pages) + 3
    d = {"held": held, "new": new, "tokens": tokens, "pages": count, "width": max(pages) + 1}
    order = torch.randperm(count, generator=gen, device="cuda").int()
    d["table"] = torch.full((case["sequences"], d["width"]), -1, dtype=torch.int32, device="cuda")
    first = 0
    for s, n in enumerate(pages):
        d["table"][s, :n] = order[first:first + n]
        first += n
    d["lengths"] = torch.tensor(held, dtype=torch.int32, device="cuda")
    d["cu"] = torch.tensor([0] + new, device="cuda").cumsum(0).int()
    for name in ("k", "v"):
        # pages as earlier calls have left them: each head and page of a magnitude of its own
        held8 = torch.empty((count, kv, page, dim), dtype=_E4M3, device="cuda")
        scales = torch.empty((count, kv), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 25) // (kv * page * dim))
        for p in range(0, count, step):
            x = normal(min(step, count - p), kv, page, dim)
            x *= torch.exp(0.3 * normal(x.shape[0], kv, 1, 1))
            b = _scale_bytes(x.abs().amax((2, 3)))
            held8[p:p + step] = (x * _power(127 - b)[:, :, None, None]).to(_E4M3)
            scales[p:p + step] = b.to(torch.uint8)
        d[name + "_pages"], d[name + "_scales"] = held8, scales
    if case["op"] == "append":
        # the rows of one projection: queries, keys and values side by side
        d["qkv"] = (normal(tokens, case["q_heads"] + 2 * kv, dim) * torch.exp(0.3 * normal(tokens, 1, 1))).to(dt)
        half = case["rotary"] // 2
        positions = max(a + b for a, b in zip(held, new))
        if half:
            angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * \
                10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
            d["rotation"] = torch.cat((angle.cos(), angle.sin()), 1).float()
    else:
        d["q"] = (2.0 * normal(tokens, case["q_heads"], dim)).to(dt)
    return d


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    if case["op"] == "append":
        s["q_out"] = torch.empty((s["tokens"], case["q_heads"], case["head_dim"]), dtype=_TORCH[case["dtype"]], device="cuda")
        # of every sequence the pages that its new tokens reach, with the slots from which on they are new
        rows, columns, slots = [], [], []
        for i, (a, n) in enumerate(zip(s["held"], s["new"])):
            for c in range(a // case["page"], (a + n - 1) // case["page"] + 1):
                rows.append(i), columns.append(c), slots.append(max(0, a - c * case["page"]))
        s["reached"] = torch.tensor([rows, columns, slots], device="cuda")
    else:
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((s["tokens"], case["q_heads"]), device="cuda")
        if own:
            import paper_2511_03586_amd as perf
            s["ws"] = torch.empty(perf.perf_cache_attention_fp8_workspace_bytes(
                s["tokens"], case["sequences"], max(s["new"]), case["q_heads"], case["kv_heads"], case["head_dim"], case["page"],
                s["width"]), dtype=torch.uint8, device="cuda")
    return s


def _appended(s):
    return {"q": s["q_out"], **{name: s[name] for name in ("k_pages", "v_pages", "k_scales", "v_scales")}}


# ---- the operators in plain form ------------------------------------------------------------------
def _rotate(x, c, s, half, interleaved):
    """x: [tokens][heads][head_dim] in float32; c, s: [tokens][half]."""
    c, s = c[:, None], s[:, None]
    x1, x2 = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    y1, y2 = x1 * c - x2 * s, x2 * c + x1 * s
    turned = torch.stack((y1, y2), -1).flatten(-2) if interleaved else torch.cat((y1, y2), -1)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _plain_append(s):
    case = s["case"]
    hq, kv, half, page = case["q_heads"], case["kv_heads"], case["rotary"] // 2, case["page"]
    token = torch.arange(s["tokens"], device="cuda")
    sequence = torch.searchsorted(s["cu"], token, right=True) - 1
    position = s["lengths"][sequence] + token - s["cu"][sequence]
    at = s["table"][sequence, position // page].long()
    slot = position % page
    q, k, v = s["qkv"].float().split((hq, kv, kv), 1)
    if half:
        c, sn = s["rotation"][position].split(half, 1)
        q, k = (_rotate(x, c, sn, half, case["interleaved"]) for x in (q, k))
    s["q_out"].copy_(q)
    row, column, first_new = s["reached"]
    reached = s["table"][row, column].long()
    before = torch.arange(page, device="cuda")[None] < first_new[:, None]  # slots whose tokens stay
    for name, x in (("k", k), ("v", v)):
        pages, scales = s[name + "_pages"], s[name + "_scales"]
        amax = torch.zeros(scales.shape, device="cuda")
        amax.scatter_reduce_(0, at[:, None].expand(-1, kv), x.abs().amax(2), "amax")
        old = torch.where(first_new[:, None] > 0, scales[reached].int(), 0)
        b = torch.maximum(old, _scale_bytes(amax[reached]))
        stored = pages.view(torch.uint8)
        kept = stored[reached]
        again = (kept.view(_E4M3).float() * _power((old - b).clamp(min=-126))[:, :, None, None]).to(_E4M3)
        stored[reached] = torch.where(before[:, None, :, None], again.view(torch.uint8), kept)
        scales[reached] = b.to(torch.uint8)
        stored[at, :, slot] = (x * _power(127 - scales[at].int())[:, :, None]).to(_E4M3).view(torch.uint8)
    return _appended(s)


def _plain_attention(s):
    case = s["case"]
    kv, dim, page = case["kv_heads"], case["head_dim"], case["page"]
    group, first = case["q_heads"] // kv, 0
    for i, (a, n) in enumerate(zip(s["held"], s["new"])):
        low = max(0, a - case["window"] + 1) // page if case["window"] else 0
        at = s["table"][i, low:-(-(a + n) // page)].long()
        k, v = ((s[x + "_pages"].view(torch.uint8)[at].view(_E4M3).float()
                 * _power(s[x + "_scales"][at].int() - 127)[:, :, None, None]).transpose(0, 1).reshape(kv, -1, dim)
                for x in ("k", "v"))
        q = s["q"][first:first + n].float().view(n, kv, group, dim).transpose(0, 1).reshape(kv, n * group, dim)
        scores = torch.bmm(q, k.transpose(1, 2).contiguous()) * dim ** -0.5
        position = a + torch.arange(n, device="cuda").repeat_interleave(group)[:, None]
        key = low * page + torch.arange(k.shape[1], device="cuda")[None]
        hidden = key > position
        if case["window"]:
            hidden |= key <= position - case["window"]
        scores.masked_fill_(hidden, -math.inf)
        top = scores.amax(2, keepdim=True)
        p = (scores - top).exp_()
        total = p.sum(2, keepdim=True)
        o = torch.bmm(p, v) / total
        s["o"][first:first + n] = o.view(kv, n, group, dim).transpose(0, 1).reshape(n, -1, dim)
        s["lse"][first:first + n] = (top + total.log()).view(kv, n, group).transpose(0, 1).reshape(n, -1)
        first += n
    return {"o": s["o"], "lse": s["lse"]}


# ---- one pass -------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if not own:
        return _plain_append(s) if case["op"] == "append" else _plain_attention(s)
    import paper_2511_03586_amd as perf
    st = torch.cuda.current_stream().cuda_stream
    hq, kv, dim = case["q_heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "append":
        ld, size = (hq + 2 * kv) * dim, _BYTES[case["dtype"]] * dim
        q = s["qkv"].data_ptr()
        perf.perf_cache_append_fp8(q, q + hq * size, q + (hq + kv) * size, s["rotation"].data_ptr() if case["rotary"] else None,
                                   s["q_out"].data_ptr(), s["k_pages"].data_ptr(), s["v_pages"].data_ptr(), s["k_scales"].data_ptr(),
                                   s["v_scales"].data_ptr(), s["table"].data_ptr(), s["lengths"].data_ptr(), s["cu"].data_ptr(),
                                   s["tokens"], case["sequences"], hq, kv, dim, ld, ld, ld, hq * dim, s["pages"], case["page"],
                                   s["width"], s["width"], case["rotary"], s["rotation"].shape[0] if case["rotary"] else 0,
                                   int(case["interleaved"]), _CODE[case["dtype"]], stream=st)
        return _appended(s)
    perf.perf_cache_attention_fp8(s["q"].data_ptr(), s["k_pages"].data_ptr(), s["v_pages"].data_ptr(), s["k_scales"].data_ptr(),
                                  s["v_scales"].data_ptr(), s["table"].data_ptr(), s["lengths"].data_ptr(), s["cu"].data_ptr(),
                                  s["o"].data_ptr(), s["lse"].data_ptr(), s["ws"].data_ptr(), s["tokens"], case["sequences"],
                                  max(s["new"]), hq, kv, dim, hq * dim, hq * dim, s["pages"], case["page"], s["width"], s["width"],
                                  case["window"], dim ** -0.5, _CODE[case["dtype"]], stream=st)
    return {"o": s["o"], "lse": s["lse"]}


# ---- what a pass cannot do without ----------------------------------------------------------------
def _visible(held, new, window):
    """Keys that the queries of a sequence see, counted for each query, and the different ones among them."""
    if not window:
        return new * held + new * (new + 1) // 2, held + new
    short = max(0, min(new, window - held))  # queries that see all keys before them
    return short * held + short * (short + 1) // 2 + (new - short) * window, min(held + new, window + new - 1)


def work(case):
    hq, kv, dim, size = case["q_heads"], case["kv_heads"], case["head_dim"], _BYTES[case["dtype"]]
    held, new = _held(case), _new(case)
    tokens = sum(new)
    if case["op"] == "append":
        rotary = case["rotary"]
        rows = len({p for a, n in zip(held, new) for p in range(a, a + n)}) if rotary else 0
        reached = sum((a + n - 1) // case["page"] - a // case["page"] + 1 for a, n in zip(held, new))
        return {"bytes": 2 * size * tokens * hq * dim + 2 * (size + 1) * tokens * kv * dim + 4 * rotary * rows + 2 * kv * reached,
                "flops": 3 * tokens * (hq + kv) * rotary + 4 * tokens * kv * dim}
    seen = [_visible(a, n, case["window"]) for a, n in zip(held, new)]
    keys = sum(v for _, v in seen)
    return {"bytes": 2 * keys * kv * dim + 2 * kv * -(-keys // case["page"]) + 2 * size * tokens * hq * dim + 4 * tokens * hq,
            "flops": 4 * dim * hq * sum(v for v, _ in seen)}


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _round8(v):
    """float64 values to the nearest e4m3 value, ties to even: a multiple of 2^(exponent - 3)."""
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 3)
    return torch.round(v / step) * step


def _exact_append(case, d):
    hq, kv, dim, page, rotary = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], case["rotary"]
    x = d["qkv"].double()
    where = torch.cat([a + torch.arange(n, device="cuda") for a, n in zip(d["held"], d["new"])])
    if rotary:
        # each pair as a complex number, turned by its angle's
        half = rotary // 2
        turn = torch.complex(d["rotation"][:, :half].double(), d["rotation"][:, half:].double())[where][:, None]
        part = x[:, :hq + kv, :rotary]
        pair = part.unflatten(2, (half, 2)) if case["interleaved"] else part.unflatten(2, (2, half)).transpose(2, 3)
        pair = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        x = x.clone()
        x[:, :hq + kv, :rotary] = (pair if case["interleaved"] else pair.transpose(2, 3)).flatten(2)
    out = {"q": x[:, :hq]}
    for name, rows in (("k", x[:, hq:hq + kv]), ("v", x[:, hq + kv:])):
        pages, scales = d[name + "_pages"].double(), d[name + "_scales"].clone()
        one = torch.ones(kv, dtype=torch.float64, device="cuda")
        first = 0
        for i, (a, n) in enumerate(zip(d["held"], d["new"])):
            p = a
            while p < a + n:  # page by page
                end = min(a + n, (p // page + 1) * page)
                at, slot = int(d["table"][i, p // page]), p % page
                take = rows[first + p - a:first + end - a].transpose(0, 1)
                least = (take.abs().amax((1, 2)) / 448.0).clamp(min=2.0 ** -126)
                b = torch.ceil(torch.log2(least)).int() + 127
                if slot:
                    b = torch.maximum(b, scales[at].int())
                    pages[at, :, :slot] = _round8(pages[at, :, :slot] * torch.ldexp(one, scales[at].int() - b)[:, None, None])
                scales[at] = b.to(torch.uint8)
                pages[at, :, slot:slot + end - p] = _round8(take / torch.ldexp(one, b - 127)[:, None, None])
                p = end
            first += n
        out[name + "_pages"], out[name + "_scales"] = pages, scales
    return {k: out[k] for k in ("q", "k_pages", "v_pages", "k_scales", "v_scales")}


def _exact_attention(case, d):
    hq, kv, dim, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    out = {"o": torch.empty((d["tokens"], hq, dim), dtype=torch.float64, device="cuda"),
           "lse": torch.empty((d["tokens"], hq), dtype=torch.float64, device="cuda")}
    first = 0
    for i, (a, n) in enumerate(zip(d["held"], d["new"])):
        key = torch.arange(a + n, device="cuda")
        at, slot = d["table"][i].long()[key // page], key % page
        for h in range(kv):
            k, v = (torch.ldexp(d[x + "_pages"].view(torch.uint8)[at, h, slot].view(_E4M3).double(),
                                d[x + "_scales"][at, h].int()[:, None] - 127) for x in ("k", "v"))
            for j in range(h * (hq // kv), (h + 1) * (hq // kv)):
                for t in range(0, n, 1024):
                    rows = slice(first + t, first + min(n, t + 1024))
                    position = a + torch.arange(t, min(n, t + 1024), device="cuda")[:, None]
                    seen = key[None] <= position
                    if case["window"]:
                        seen &= key[None] + case["window"] > position
                    scores = torch.where(seen, (d["q"][rows, j].double() @ k.T) / math.sqrt(dim), -math.inf)
                    out["lse"][rows, j] = torch.logsumexp(scores, 1)
                    out["o"][rows, j] = torch.exp(scores - out["lse"][rows, j, None]) @ v
        first += n
    return out


def exact(case, seed):
    d = _inputs(case, seed)
    return _exact_append(case, d) if case["op"] == "append" else _exact_attention(case, d)
