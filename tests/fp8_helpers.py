"""Glue and plain references for the tests of the 8-bit operators and of the norms around a block: buffers with guarded
padding, calls through the binding, and the operators' definitions in float64 (torch on the CPU)."""
import numpy as np
import torch

import paper_2511_03586_amd as perf
from tests import gpu_helpers as G

BLOCK = 128
F8 = {perf.PERF_E4M3: torch.float8_e4m3fn, perf.PERF_E5M2: torch.float8_e5m2}
LARGEST = {perf.PERF_E4M3: 448.0, perf.PERF_E5M2: 57344.0}
TORCH = {perf.PERF_F32: torch.float32, perf.PERF_BF16: torch.bfloat16, **F8}
SIZE = {perf.PERF_F32: 4, perf.PERF_BF16: 2, perf.PERF_E4M3: 1, perf.PERF_E5M2: 1}
INT = {1: torch.uint8, 2: torch.int16, 4: torch.int32}
GUARD = 0x5A  # what lies around a buffer's elements before a call, and has to lie there after it


def up(v, to=BLOCK):
    return -(-v // to)


class Held:
    """A rows x cols matrix of a dtype on the GPU, rows `ld` apart, `offset` elements into its memory, the rest GUARD bytes.
    The memory ends with the last row's last element."""

    def __init__(self, rows, cols, dt, ld=None, offset=0, data=None):
        self.rows, self.cols, self.dt, self.ld, self.size = rows, cols, dt, ld or cols, SIZE[dt]
        self.offset = offset
        count = offset + (rows - 1) * self.ld + cols
        self.bytes = torch.full((count * self.size,), GUARD, dtype=torch.uint8, device="cuda")
        if data is not None:
            self.put(data)

    def at(self):
        return self.bytes.data_ptr() + self.offset * self.size

    def _index(self):
        r = torch.arange(self.rows, device="cuda")[:, None] * self.ld + torch.arange(self.cols, device="cuda")[None]
        return (self.offset + r).reshape(-1)

    def put(self, data):
        flat = self.bytes.view(INT[self.size])
        d = data.to(TORCH[self.dt]).contiguous().cuda().reshape(-1).view(flat.dtype)
        flat[self._index()] = d

    def get(self):
        """The elements, on the CPU; the bytes around them are still GUARD."""
        kind = INT[self.size]
        flat = self.bytes.view(kind)
        index = self._index()
        around = torch.ones(flat.numel(), dtype=torch.bool, device="cuda")
        around[index] = False
        guard = torch.full((self.size,), GUARD, dtype=torch.uint8).view(kind).item()
        assert bool((flat[around] == guard).all()), "written outside the matrix"
        return flat[index].view(TORCH[self.dt]).reshape(self.rows, self.cols).cpu()


def vector(v, dt=perf.PERF_F32):
    return None if v is None else Held(1, v.numel(), dt, data=v.reshape(1, -1))


def at(h):
    return None if h is None else h.at()


# ---- quantisation -----------------------------------------------------------------------------------
def blocks_amax(x, block_rows):
    rows, cols = x.shape
    r, c = up(rows, block_rows) * block_rows, up(cols) * BLOCK
    p = torch.nn.functional.pad(x.abs(), (0, c - cols, 0, r - rows))
    return p.view(r // block_rows, block_rows, c // BLOCK, BLOCK).amax((1, 3))


def spread(s, block_rows, rows, cols):
    return s.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def quantize_ref(x, block_rows, q_dt):
    """The definition in float32, step by step: s = max(amax / F, 2^-126), q = x * (1 / s) rounded."""
    x = x.float()
    s = torch.maximum(blocks_amax(x, block_rows) / torch.tensor(LARGEST[q_dt]), torch.tensor(2.0 ** -126))
    return (x * spread(torch.tensor(1.0) / s, block_rows, *x.shape)).to(F8[q_dt]), s


def run_quantize(x, dt, q_dt, block_rows, row=True, transposed=True, ldx=None, pad=0, offset=0):
    rows, cols = x.shape
    xd = Held(rows, cols, dt, ldx, offset, x)
    q = Held(rows, cols, q_dt, cols + pad, offset) if row else None
    s = Held(up(rows, block_rows), up(cols), perf.PERF_F32, up(cols) + (1 if pad else 0)) if row else None
    qt = Held(cols, rows, q_dt, rows + pad, offset) if transposed else None
    st = Held(up(cols, block_rows), up(rows), perf.PERF_F32, up(rows) + (2 if pad else 0)) if transposed else None
    perf.perf_quantize_fp8(xd.at(), at(q), at(s), at(qt), at(st), rows, cols, xd.ld, q.ld if q else 0, s.ld if s else 0,
                           qt.ld if qt else 0, st.ld if st else 0, block_rows, dt, q_dt, stream=G.stream())
    torch.cuda.synchronize()
    return [None if h is None else h.get() for h in (q, s, qt, st)]


# ---- product ----------------------------------------------------------------------------------------
def gemm_ref(a, sa, b, sb, b_rows, alpha=1.0):
    """C and the sum of the magnitudes behind it, float64."""
    m, k = a.shape
    n = b.shape[0]
    a = a.double() * spread(sa.double(), 1, m, k)
    b = b.double() * spread(sb.double(), b_rows, n, k)
    return (alpha * (a @ b.T)).numpy(), (abs(alpha) * (a.abs() @ b.abs().T)).numpy()


def run_gemm(a, sa, b, sb, b_rows, c_dt, alpha=1.0, lda=None, ldb=None, ldsa=None, ldsb=None, ldc=None, a_dt=perf.PERF_E4M3):
    m, k = a.shape
    n = b.shape[0]
    to16 = up(k, 16) * 16
    ad, bd = Held(m, k, a_dt, lda or to16, 0, a), Held(n, k, perf.PERF_E4M3, ldb or to16, 0, b)
    sad, sbd = Held(m, up(k), perf.PERF_F32, ldsa, 0, sa), Held(up(n, b_rows), up(k), perf.PERF_F32, ldsb, 0, sb)
    c = Held(m, n, c_dt, ldc)
    perf.perf_gemm_fp8(ad.at(), sad.at(), bd.at(), sbd.at(), c.at(), m, n, k, ad.ld, sad.ld, bd.ld, sbd.ld, c.ld, b_rows,
                       alpha=alpha, a_dt=a_dt, c_dt=c_dt, stream=G.stream())
    torch.cuda.synchronize()
    return c.get().double().numpy()


def random_operand(g, rows, k, block_rows, q_dt=perf.PERF_E4M3):
    x = torch.from_numpy((g.standard_normal((rows, k)) * np.exp(g.standard_normal((rows, 1)))).astype(np.float32))
    return quantize_ref(x, block_rows, q_dt)


# ---- norms ------------------------------------------------------------------------------------------
def group_rows(gate, gate_rows, rows):
    return gate.repeat_interleave(gate_rows, 0)[:rows]


def norm_ref(u, x, gate, gate_rows, post, pre, scale, eps):
    """h, y, r_post, r_pre in float64, and how the magnitudes behind h add up."""
    u, x = u.double(), x.double()
    r1 = 1.0 / torch.sqrt((u * u).mean(1, keepdim=True) + eps)
    n = u * r1 * post.double() if post is not None else u
    if gate is not None:
        n = n * group_rows(gate.double(), gate_rows, u.shape[0])
    h = scale * x + n
    r2 = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    y = h * r2 * pre.double() if pre is not None else None
    return h, y, r1[:, 0], r2[:, 0], (scale * x).abs() + n.abs()


def grad_ref(dy, dh, h, u, gate, gate_rows, post, pre, r1, r2, scale, magnitudes=False):
    """Gradients in float64 by the formulas; with `magnitudes` the same sums with every term's magnitude: a bound for what
    their terms can amount to."""
    rows = u.shape[0]
    f = (lambda v: v.double().abs()) if magnitudes else (lambda v: v.double())
    sign = 1.0 if magnitudes else -1.0
    H = f(dh) if dh is not None else torch.zeros(u.shape, dtype=torch.float64)
    out = {}
    if dy is not None:
        r2 = r2.double()[:, None]
        t, hn = f(dy) * f(pre), f(h) * r2
        H = H + r2 * (t + sign * hn * (t * hn).mean(1, keepdim=True))
        out["dpre"] = (f(dy) * hn).sum(0)
    out["dx"] = abs(scale) * H if magnitudes else scale * H
    D = H * group_rows(f(gate), gate_rows, rows) if gate is not None else H
    n = f(u)
    if post is not None:
        r1 = r1.double()[:, None]
        un, v = n * r1, D * f(post)
        out["dpost"] = (D * un).sum(0)
        out["du"] = r1 * (v + sign * un * (v * un).mean(1, keepdim=True))
        n = un * f(post)
    else:
        out["du"] = D
    if gate is not None:
        groups = up(rows, gate_rows)
        padded = torch.nn.functional.pad(n * H, (0, 0, 0, groups * gate_rows - rows))
        out["dgate"] = padded.view(groups, gate_rows, -1).sum(1)
    return out
