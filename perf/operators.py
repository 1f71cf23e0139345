"""Performance cases of the 8-bit linear layer and the norms around it: quantisation in blocks of 128, the product of
block-scaled 8-bit matrices, and the norms before and after a block joined with its gate and residual scale, forward and
backward.

A case is a dict of plain values; ``op`` names the operator. ``listed()`` holds the fixed cases, ``draw(rng)`` one more from
the same ranges. ``prepare`` makes the device buffers that a program holds before it calls, ``run`` is one call: of the
library where ``own`` is true, of the operator's plain form in elementary torch operations where it is not. ``exact`` is the
operator's definition in float64.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_BYTES = {"f32": 4, "bf16": 2}
_CODE = {"f32": 0, "bf16": 1, "e4m3": 2, "e5m2": 3}  # PERF_F32, PERF_BF16, PERF_E4M3, PERF_E5M2
_LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
_EPS = 1e-5
BLOCK = 128


def listed():
    return [
        # serving: the activations of six tokens in front of the wide projection; bound by the launch
        {"name": "quantize_rows_bf16_6x14336", "op": "quantize", "rows": 6, "cols": 14336, "dtype": "bf16", "out": "e4m3",
         "block_rows": 1, "row_out": True, "transposed_out": False},
        # training: a batch of activations, as rows for the forward product and transposed for the weight gradient
        {"name": "quantize_both_bf16_8192x4096", "op": "quantize", "rows": 8192, "cols": 4096, "dtype": "bf16", "out": "e4m3",
         "block_rows": 1, "row_out": True, "transposed_out": True},
        # master weights of odd extents in tiles, for the forward product and for the input gradient
        {"name": "quantize_tiles_f32_2999x5003", "op": "quantize", "rows": 2999, "cols": 5003, "dtype": "f32", "out": "e4m3",
         "block_rows": 128, "row_out": True, "transposed_out": True},
        # one decoded token: bound by the weights' bytes
        {"name": "gemm_1x4096x4096", "op": "gemm", "batch": 1, "M": 1, "N": 4096, "K": 4096, "a": "e4m3", "out": "bf16", "b_rows": 128},
        # a batch of decoded tokens through the wide projection
        {"name": "gemm_64x14336x4096", "op": "gemm", "batch": 1, "M": 64, "N": 14336, "K": 4096, "a": "e4m3", "out": "bf16", "b_rows": 128},
        # the table's matmul: too few output tiles for the chip
        {"name": "gemm_768x1024x1024", "op": "gemm", "batch": 1, "M": 768, "N": 1024, "K": 1024, "a": "e4m3", "out": "f32", "b_rows": 128},
        # the large projection of a training batch
        {"name": "gemm_4096x4096x4096", "op": "gemm", "batch": 1, "M": 4096, "N": 4096, "K": 4096, "a": "e4m3", "out": "bf16", "b_rows": 128},
        # a weight gradient of ragged extents: both operands in row blocks, gradients in the wider exponent range
        {"name": "gemm_grad_1999x2999x5003", "op": "gemm", "batch": 1, "M": 1999, "N": 2999, "K": 5003, "a": "e5m2", "out": "f32", "b_rows": 1},
        # one decoded token through the norms of a block, handed on in 8 bits
        {"name": "norm_bf16_to_e4m3_1x4096", "op": "norm", "rows": 1, "cols": 4096, "dtype": "bf16", "out": "e4m3",
         "gate_rows": 1, "gate_dtype": "f32", "post": True},
        # training batch, one gate for all rows
        {"name": "norm_bf16_8192x4096", "op": "norm", "rows": 8192, "cols": 4096, "dtype": "bf16", "out": "same",
         "gate_rows": 8192, "gate_dtype": "f32", "post": True},
        # its gradient
        {"name": "norm_grad_bf16_8192x4096", "op": "norm_grad", "rows": 8192, "cols": 4096, "dtype": "bf16", "gate_rows": 8192,
         "gate_dtype": "f32", "post": True},
        # gradient in single precision, features of odd length, a gate of each sample's own
        {"name": "norm_grad_f32_6007x1023", "op": "norm_grad", "rows": 6007, "cols": 1023, "dtype": "f32", "gate_rows": 256,
         "gate_dtype": "f32", "post": True},
    ]


# ---- drawn cases ----------------------------------------------------------------------------------
def _size(rng, lo, hi):
    """An extent in [lo, hi], uniform in its logarithm: four in ten regular, three even, three any."""
    v = min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    kind = rng.random()
    step = (128 if v >= 512 else 16) if kind < 0.4 else 8 if kind < 0.7 else 1
    return min(hi, max(lo, v // step * step if v >= step else v))


def draw(rng):
    op = rng.choice(["quantize", "quantize", "gemm", "gemm", "gemm", "gemm", "norm", "norm", "norm_grad", "norm_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "gemm":
        # decoding, a linear layer's three products, and experts' products in a batch
        while True:
            batch = rng.choice([1, 1, 1, _size(rng, 2, 16)])
            m = rng.choice([_size(rng, 1, 64), _size(rng, 16, 4096), _size(rng, 16, 4096)])
            n, k = _size(rng, 64, 16384), _size(rng, 64, 8192)
            if 1e5 <= batch * m * n * k <= 6e10 and batch * (m * n + m * k + n * k) <= 1e8:
                return {"op": op, "batch": batch, "M": m, "N": n, "K": k, "a": rng.choice(["e4m3", "e4m3", "e5m2"]),
                        "out": rng.choice(["bf16", "f32"]), "b_rows": rng.choice([1, 128, 128])}
    cols = _size(rng, 64, 16384)
    rows = _size(rng, 1, min(16384, 33_000_000 // cols // (2 if dtype == "f32" else 1)))
    if op == "quantize":
        kind = rng.choice(["rows", "transposed", "both"])
        return {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "out": rng.choice(["e4m3", "e4m3", "e5m2"]),
                "block_rows": rng.choice([1, 1, 128]), "row_out": kind != "transposed", "transposed_out": kind != "rows"}
    # no gate, one of every element's own, one of each sample's, one for all rows
    gate_rows = rng.choice([0, 1, max(1, rows // rng.randint(2, 32)), rows])
    case = {"op": op, "rows": rows, "cols": cols, "dtype": dtype, "gate_rows": gate_rows,
            "gate_dtype": dtype if gate_rows == 1 else rng.choice(["f32", dtype]), "post": rng.random() < 0.75}
    if op == "norm":
        case["out"] = rng.choice(["same", "same", "e4m3"])
    return case


# ---- what a program holds -------------------------------------------------------------------------
def _up(v, to):
    return -(-v // to) * to


def _gate_shape(case):
    return (-(-case["rows"] // case["gate_rows"]), case["cols"])


def _blocks(x, block_rows):
    """The largest magnitudes of x's blocks, [rows / block_rows][cols / 128]; the last ones of either axis may be short."""
    rows, cols = x.shape[-2:]
    r, c = _up(rows, block_rows), _up(cols, BLOCK)
    p = torch.nn.functional.pad(x.abs(), (0, c - cols, 0, r - rows))
    return p.view(*x.shape[:-2], r // block_rows, block_rows, c // BLOCK, BLOCK).amax((-3, -1))


def _spread(s, block_rows, rows, cols):
    """A block's scale at each of its elements."""
    if block_rows > 1:
        s = s.repeat_interleave(block_rows, -2)[..., :rows, :]
    return s.repeat_interleave(BLOCK, -1)[..., :cols]


def _plain_quantize(x, block_rows, fmt):
    """8-bit values and scales of x (float32): s = amax / largest, at least the least normal number; q = x * (1 / s) rounded."""
    amax = _blocks(x, block_rows)
    s = (amax / torch.full_like(amax, _LARGEST[fmt])).clamp_(min=2.0 ** -126)
    return (x * _spread(1.0 / s, block_rows, *x.shape[-2:])).to(_TORCH[fmt]), s


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(shape, mean=0.0, std=1.0, dtype="f32"):
        return torch.randn(shape, generator=gen, device="cuda").mul_(std).add_(mean).to(_TORCH[dtype])

    def uniform(shape, lo, hi, dtype="f32"):
        return torch.rand(shape, generator=gen, device="cuda").mul_(hi - lo).add_(lo).to(_TORCH[dtype])

    op = case["op"]
    if op == "quantize":
        # rows of different magnitude, as tokens have
        x = normal((case["rows"], case["cols"])) * torch.exp(normal((case["rows"], 1)))
        return {"x": x.to(_TORCH[case["dtype"]])}
    if op == "gemm":
        b, m, n, k = case["batch"], case["M"], case["N"], case["K"]
        d = {}
        for name, rows, fmt, block in (("a", m, case["a"], 1), ("b", n, "e4m3", case["b_rows"])):
            q, s = _plain_quantize(normal((b, rows, k)) * torch.exp(normal((b, rows, 1), 0.0, 0.5)), block, fmt)
            held = torch.zeros((b, rows, _up(k, 16)), dtype=torch.uint8, device="cuda")
            held[:, :, :k] = q.view(torch.uint8)
            d[name], d["s" + name] = held.view(_TORCH[fmt])[:, :, :k], s
        return d
    rows, cols, dt = case["rows"], case["cols"], case["dtype"]
    d = {"u": normal((rows, cols), 0.1, 0.7, dt), "gamma_pre": uniform((cols,), 0.5, 1.5)}
    d["gamma_post"] = uniform((cols,), 0.5, 1.5) if case["post"] else None
    d["gate"] = normal(_gate_shape(case), 0.3, 0.3, case["gate_dtype"]) if case["gate_rows"] else None
    x = normal((rows, cols), 0.0, 2.0, dt)
    if op == "norm":
        d["x"] = x
    else:  # what the forward pass has left behind, and the gradients that come in
        d["h"], _, d["r_post"], d["r_pre"] = _plain_norm(case, {**d, "x": x}, _SCALE)
        d["h"] = d["h"].to(_TORCH[dt])
        d["dy"], d["dh"] = normal((rows, cols), 0.0, 1.0, dt), normal((rows, cols), 0.0, 0.5, dt)
    return d


_SCALE = 0.75  # the residual's, exact in every type


def prepare(case, seed):
    s = {"case": case, **_inputs(case, seed)}
    op = case["op"]

    def empty(shape, dt="f32"):
        return torch.empty(shape, dtype=_TORCH[dt], device="cuda")

    if op == "quantize":
        rows, cols, br, fmt = case["rows"], case["cols"], case["block_rows"], case["out"]
        if case["row_out"]:
            s["q"], s["scales"] = empty((rows, _up(cols, 16)), fmt), empty((-(-rows // br), -(-cols // BLOCK)))
        if case["transposed_out"]:
            s["qt"], s["scales_t"] = empty((cols, _up(rows, 16)), fmt), empty((-(-cols // br), -(-rows // BLOCK)))
    elif op == "gemm":
        s["c"] = empty((case["batch"], case["M"], case["N"]), case["out"])
    else:
        rows, cols, dt = case["rows"], case["cols"], case["dtype"]
        if op == "norm":
            s["h"], s["r_post"], s["r_pre"] = empty((rows, cols), dt), empty((rows,)), empty((rows,))
            if case["out"] == "same":
                s["y"] = empty((rows, cols), dt)
            else:
                s["y"], s["scales"] = empty((rows, _up(cols, 16)), case["out"]), empty((rows, -(-cols // BLOCK)))
        else:
            s["dx"], s["du"], s["dgamma_pre"] = empty((rows, cols), dt), empty((rows, cols), dt), empty((cols,))
            s["dgamma_post"] = empty((cols,)) if case["post"] else None
            s["dgate"] = empty(_gate_shape(case), case["gate_dtype"]) if case["gate_rows"] else None
            # scratch for sums over rows: at most 1024 partial sums of the three vectors of parameters
            s["ws"] = torch.empty(12 * 1024 * cols, dtype=torch.uint8, device="cuda")
    return s


# ---- the operators in plain form ------------------------------------------------------------------
def _group_rows(g, case):
    """The gate of each row."""
    return g.repeat_interleave(case["gate_rows"], 0)[:case["rows"]]


def _plain_norm(case, s, scale):
    """h, y in float32 and the reciprocal RMS of both norms."""
    u, x = s["u"].float(), s["x"].float()
    r_post = torch.rsqrt((u * u).mean(1) + _EPS)
    n = u * r_post[:, None] * s["gamma_post"].float() if case["post"] else u
    if case["gate_rows"]:
        n = n * _group_rows(s["gate"].float(), case)
    h = scale * x + n
    r_pre = torch.rsqrt((h * h).mean(1) + _EPS)
    return h, h * r_pre[:, None] * s["gamma_pre"].float(), r_post if case["post"] else None, r_pre


def _plain_norm_grad(case, s, scale, real):
    """Gradients with respect to x, u, the gate and both gains, in the type `real`."""
    dy, h, u = s["dy"].to(real), s["h"].to(real), s["u"].to(real)
    r_pre = s["r_pre"].to(real)[:, None]
    hn, t = h * r_pre, dy * s["gamma_pre"].to(real)
    whole = s["dh"].to(real) + r_pre * (t - hn * (t * hn).mean(1, keepdim=True))
    out = {"dx": scale * whole, "dgamma_pre": (dy * hn).sum(0)}
    dn = whole * _group_rows(s["gate"].to(real), case) if case["gate_rows"] else whole
    n = u
    if case["post"]:
        r_post = s["r_post"].to(real)[:, None]
        un, v = u * r_post, dn * s["gamma_post"].to(real)
        out["dgamma_post"] = (dn * un).sum(0)
        out["du"] = r_post * (v - un * (v * un).mean(1, keepdim=True))
        n = un * s["gamma_post"].to(real)
    else:
        out["du"] = dn
    if case["gate_rows"]:
        groups, per = _gate_shape(case)[0], case["gate_rows"]
        out["dgate"] = torch.nn.functional.pad(n * whole, (0, 0, 0, groups * per - case["rows"])).view(groups, per, -1).sum(1)
    return out


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "quantize":
        x, br, out = s["x"].float(), case["block_rows"], {}
        if case["row_out"]:
            out["q"], out["scales"] = _plain_quantize(x, br, case["out"])
        if case["transposed_out"]:
            out["qt"], out["scales_t"] = _plain_quantize(x.t().contiguous(), br, case["out"])
        return out
    if op == "gemm":
        m, n, k = case["M"], case["N"], case["K"]
        a = s["a"].float() * _spread(s["sa"], 1, m, k)
        b = s["b"].float() * _spread(s["sb"], case["b_rows"], n, k)
        return {"c": torch.matmul(a, b.transpose(1, 2)).to(_TORCH[case["out"]])}
    dt = _TORCH[case["dtype"]]
    if op == "norm":
        h, y, r_post, r_pre = _plain_norm(case, s, _SCALE)
        out = {"h": h.to(dt), "r_post": r_post, "r_pre": r_pre}
        if case["out"] == "same":
            out["y"] = y.to(dt)
        else:
            out["y"], out["scales"] = _plain_quantize(y, 1, case["out"])
        return out
    out = _plain_norm_grad(case, s, _SCALE, torch.float32)
    out["dx"], out["du"] = out["dx"].to(dt), out["du"].to(dt)
    if case["gate_rows"]:
        out["dgate"] = out["dgate"].to(_TORCH[case["gate_dtype"]])
    return out


# ---- one pass -------------------------------------------------------------------------------------
def _at(t):
    return None if t is None else t.data_ptr()


def run(s):
    if not own:
        return _plain(s)
    import paper_2511_03586_amd as perf
    case = s["case"]
    op, st = case["op"], torch.cuda.current_stream().cuda_stream
    if op == "quantize":
        rows, cols = case["rows"], case["cols"]
        q, qt = s.get("q"), s.get("qt")
        perf.perf_quantize_fp8(s["x"].data_ptr(), _at(q), _at(s.get("scales")), _at(qt), _at(s.get("scales_t")), rows, cols, cols,
                               _up(cols, 16), -(-cols // BLOCK), _up(rows, 16), -(-rows // BLOCK), case["block_rows"],
                               _CODE[case["dtype"]], _CODE[case["out"]], stream=st)
        out = {}
        if q is not None:
            out["q"], out["scales"] = q[:, :cols], s["scales"]
        if qt is not None:
            out["qt"], out["scales_t"] = qt[:, :rows], s["scales_t"]
        return out
    if op == "gemm":
        m, n, k = case["M"], case["N"], case["K"]
        ld, kb = _up(k, 16), -(-k // BLOCK)
        perf.perf_gemm_fp8(s["a"].data_ptr(), s["sa"].data_ptr(), s["b"].data_ptr(), s["sb"].data_ptr(), s["c"].data_ptr(), m, n, k,
                           ld, kb, ld, kb, n, case["b_rows"], case["batch"], m * ld, m * kb, n * ld, -(-n // case["b_rows"]) * kb,
                           m * n, 1.0, _CODE[case["a"]], perf.PERF_E4M3, _CODE[case["out"]], stream=st)
        return {"c": s["c"]}
    rows, cols, dt, gate_rows = case["rows"], case["cols"], _CODE[case["dtype"]], case["gate_rows"] or case["rows"]
    gate_dt = _CODE[case["gate_dtype"]]
    if op == "norm":
        same = case["out"] == "same"
        perf.perf_residual_norm(s["u"].data_ptr(), s["x"].data_ptr(), _at(s["gate"]), _at(s["gamma_post"]), s["gamma_pre"].data_ptr(),
                                s["h"].data_ptr(), s["y"].data_ptr(), None if same else s["scales"].data_ptr(),
                                s["r_post"].data_ptr() if case["post"] else None, s["r_pre"].data_ptr(), rows, cols, cols, cols, cols,
                                gate_rows, cols, cols if same else _up(cols, 16), -(-cols // BLOCK), _SCALE, _EPS, dt, gate_dt,
                                perf.PERF_F32, dt if same else _CODE[case["out"]], stream=st)
        out = {"h": s["h"], "y": s["y"] if same else s["y"][:, :cols], "r_post": s["r_post"] if case["post"] else None,
               "r_pre": s["r_pre"]}
        if not same:
            out["scales"] = s["scales"]
        return out
    perf.perf_residual_norm_backward(s["dy"].data_ptr(), s["dh"].data_ptr(), s["h"].data_ptr(), s["u"].data_ptr(), _at(s["gate"]),
                                     _at(s["gamma_post"]), s["gamma_pre"].data_ptr(), _at(s["r_post"]), s["r_pre"].data_ptr(),
                                     s["dx"].data_ptr(), s["du"].data_ptr(), _at(s["dgate"]), _at(s["dgamma_post"]),
                                     s["dgamma_pre"].data_ptr(), s["ws"].data_ptr(), rows, cols, cols, cols, cols, cols, cols, gate_rows,
                                     cols, cols, cols, _SCALE, dt, gate_dt, perf.PERF_F32, stream=st)
    out = {"dx": s["dx"], "du": s["du"], "dgamma_pre": s["dgamma_pre"]}
    if case["post"]:
        out["dgamma_post"] = s["dgamma_post"]
    if case["gate_rows"]:
        out["dgate"] = s["dgate"]
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "gemm":
        b, m, n, k = case["batch"], case["M"], case["N"], case["K"]
        kb = -(-k // BLOCK)
        return {"bytes": b * (m * k + n * k + 4 * kb * (m + -(-n // case["b_rows"])) + _BYTES[case["out"]] * m * n),
                "flops": 2 * b * m * n * k}
    rows, cols, sz = case["rows"], case["cols"], _BYTES[case["dtype"]]
    e = rows * cols
    if op == "quantize":
        sides = int(case["row_out"]) + int(case["transposed_out"])
        return {"bytes": sz * e + sides * (e + 4 * e // (BLOCK * case["block_rows"])), "flops": (1 + 2 * sides) * e}
    gate = _BYTES[case["gate_dtype"]] * math.prod(_gate_shape(case)) if case["gate_rows"] else 0
    gains = 4 * cols * (2 if case["post"] else 1)
    if op == "norm":
        y = sz * e if case["out"] == "same" else e + e // 32
        return {"bytes": 3 * sz * e + y + gate + gains + 8 * rows, "flops": 10 * e}
    return {"bytes": 6 * sz * e + 2 * gate + 2 * gains + 8 * rows, "flops": 24 * e}


# ---- the definitions in 64 bits -------------------------------------------------------------------
def _round8(v, fmt):
    """float64 values to the nearest 8-bit value, ties to even: a multiple of 2^(exponent - mantissa bits)."""
    bits, least = (3, -6) if fmt == "e4m3" else (2, -14)
    _, e = torch.frexp(v)
    step = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=least) - bits)
    return (torch.round(v / step) * step).clamp(-_LARGEST[fmt], _LARGEST[fmt])


def _exact_quantize(x, block_rows, fmt):
    s = (_blocks(x, block_rows) / _LARGEST[fmt]).clamp(min=2.0 ** -126)
    return _round8(x / _spread(s, block_rows, *x.shape[-2:]), fmt), s


def exact(case, seed):
    op = case["op"]
    d = {k: None if v is None else v.double() for k, v in _inputs(case, seed).items()}
    if op == "quantize":
        out = {}
        if case["row_out"]:
            out["q"], out["scales"] = _exact_quantize(d["x"], case["block_rows"], case["out"])
        if case["transposed_out"]:
            out["qt"], out["scales_t"] = _exact_quantize(d["x"].t().contiguous(), case["block_rows"], case["out"])
        return out
    if op == "gemm":
        c = torch.zeros((case["batch"], case["M"], case["N"]), dtype=torch.float64, device="cuda")
        for k in range(0, case["K"], BLOCK):  # block by block, as the operator is defined
            p = torch.matmul(d["a"][:, :, k:k + BLOCK], d["b"][:, :, k:k + BLOCK].transpose(1, 2).contiguous())
            sb = d["sb"][:, :, k // BLOCK].repeat_interleave(case["b_rows"], 1)[:, None, :case["N"]]
            c += p * d["sa"][:, :, k // BLOCK, None] * sb
        return {"c": c}
    if op == "norm":
        mean_square = lambda v: torch.linalg.vector_norm(v, dim=1, keepdim=True) ** 2 / case["cols"]  # noqa: E731
        out = {"r_post": None}
        n = d["u"]
        if case["post"]:
            r = (mean_square(n) + _EPS) ** -0.5
            n, out["r_post"] = d["u"] * r * d["gamma_post"], r[:, 0]
        if case["gate_rows"]:
            n = d["gate"][torch.arange(case["rows"], device="cuda") // case["gate_rows"]] * n
        out["h"] = d["x"] * _SCALE + n
        r = (mean_square(out["h"]) + _EPS) ** -0.5
        y, out["r_pre"] = out["h"] * r * d["gamma_pre"], r[:, 0]
        if case["out"] == "same":
            out["y"] = y
        else:
            out["y"], out["scales"] = _exact_quantize(y, 1, case["out"])
        return out
    # gradients of <dy, y(h)> + <dh, h> in terms of the held h, u and reciprocal RMS: r' = -r^3 x / cols
    rows, cols = case["rows"], case["cols"]
    r2 = d["r_pre"].view(rows, 1)
    t = d["dy"] * d["gamma_pre"]
    into_h = d["dh"] + t * r2 - d["h"] * r2 ** 3 * ((t * d["h"]).sum(1, keepdim=True) / cols)
    of_row = torch.arange(rows, device="cuda") // case["gate_rows"] if case["gate_rows"] else None
    into_n = into_h if of_row is None else into_h * d["gate"][of_row]
    out = {"dx": into_h * _SCALE, "dgamma_pre": (d["dy"] * d["h"] * r2).sum(0)}
    n = d["u"]
    if case["post"]:
        r1 = d["r_post"].view(rows, 1)
        w = into_n * d["gamma_post"]
        out["du"] = w * r1 - d["u"] * r1 ** 3 * ((w * d["u"]).sum(1, keepdim=True) / cols)
        out["dgamma_post"] = (into_n * d["u"] * r1).sum(0)
        n = d["u"] * r1 * d["gamma_post"]
    else:
        out["du"] = into_n
    if of_row is not None:
        out["dgate"] = torch.zeros(_gate_shape(case), dtype=torch.float64, device="cuda").index_add_(0, of_row, n * into_h)
    return out
