"""GPU: the norms before and after a block with its gate and residual scale, and their gradient, against the definitions in
float64 and against differences."""
import numpy as np
import pytest
import torch

import paper_2511_03586_amd as perf
from tests import fp8_helpers as F
from tests import gpu_helpers as G

pytestmark = pytest.mark.gpu

F32, BF16, E4M3 = perf.PERF_F32, perf.PERF_BF16, perf.PERF_E4M3
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def _depth(cols):
    """Roundings on the way of a term into a row's sum: those of a lane (8 for each 8192 columns), 6 exchanges in a wave, 16
    waves, and a few for what surrounds the sum."""
    return 8 * F.up(cols, 8192) + 6 + 16 + 10


def _make(rows, cols, dt, gate_rows, gate_dt, param_dt, post, seed=0):
    g = np.random.default_rng(31 * rows + cols + seed)
    n = lambda *shape: torch.from_numpy(g.standard_normal(shape).astype(np.float32))  # noqa: E731
    u, x = (n(rows, cols) * 0.7 + 0.1).to(F.TORCH[dt]), (n(rows, cols) * 2).to(F.TORCH[dt])
    gate = (n(F.up(rows, gate_rows), cols) * 0.5 + 0.3).to(F.TORCH[gate_dt]) if gate_rows else None
    gain = lambda: (torch.from_numpy(g.uniform(0.5, 1.5, cols).astype(np.float32))).to(F.TORCH[param_dt])  # noqa: E731
    return u, x, gate, gain() if post else None, gain()


def _forward(u, x, gate, gate_rows, post, pre, scale, dt, gate_dt=F32, param_dt=F32, y_dt=None, pad=0, want_h=True, want_y=True,
             in_place=False, offset=0, eps=1e-5):
    rows, cols = u.shape
    y_dt = dt if y_dt is None else y_dt
    ud, xd = F.Held(rows, cols, dt, cols + pad, offset, u), F.Held(rows, cols, dt, cols + 2 * pad, offset, x)
    gd = F.Held(gate.shape[0], cols, gate_dt, cols + pad, offset, gate) if gate is not None else None
    h = xd if in_place else F.Held(rows, cols, dt, cols + pad, offset) if want_h else None
    y = F.Held(rows, cols, y_dt, cols + 3 * pad, offset) if want_y else None
    s = F.Held(rows, F.up(cols), F32, F.up(cols) + (1 if pad else 0)) if y_dt == E4M3 else None
    r1, r2 = (F.Held(1, rows, F32) for _ in range(2))
    postd, pred = F.vector(post, param_dt), F.vector(pre, param_dt)
    perf.perf_residual_norm(ud.at(), xd.at(), F.at(gd), F.at(postd), F.at(pred), F.at(h),
                            F.at(y), F.at(s), r1.at() if post is not None else None, r2.at() if want_y else None, rows, cols, ud.ld,
                            xd.ld, gd.ld if gd else cols, gate_rows or 1, h.ld if h else cols, y.ld if y else cols,
                            s.ld if s else 0, scale, eps, dt, gate_dt, param_dt, y_dt, stream=G.stream())
    torch.cuda.synchronize()
    get = lambda v: None if v is None else v.get()  # noqa: E731
    return get(h), get(y), get(s), r1.get()[0] if post is not None else None, r2.get()[0] if want_y else None


def _check_forward(rows, cols, dt, gate_rows=0, gate_dt=F32, param_dt=F32, post=True, y_dt=None, scale=0.75, seed=0, **kw):
    u, x, gate, gpost, gpre = _make(rows, cols, dt, gate_rows, gate_dt, param_dt, post, seed)
    eps = float(np.float32(1e-5))
    h, y, s, r1, r2 = _forward(u, x, gate, gate_rows, gpost, gpre, scale, dt, gate_dt, param_dt, y_dt, **kw)
    rh, ry, rr1, rr2, mag = F.norm_ref(u, x, gate, gate_rows, gpost, gpre, float(np.float32(scale)), eps)
    c = _depth(cols) * 2.0 ** -24
    if h is not None:
        assert torch.all((h.double() - rh).abs() <= c * mag + HALF_STEP[dt] * rh.abs())
    if r1 is not None:
        assert torch.all((r1.double() - rr1).abs() <= c * rr1)
    if y is None:
        return
    # r2 moves by the errors of h: at most those of the magnitudes' root mean square over that of h
    rel = c + c * torch.sqrt((mag ** 2).mean(1)) * rr2
    assert torch.all((r2.double() - rr2).abs() <= rel * rr2)
    err = c * mag * rr2[:, None] * gpre.double() + rel[:, None] * ry.abs()
    if y_dt != E4M3:
        assert torch.all((y.double() - ry).abs() <= err * (1 + HALF_STEP[dt]) + HALF_STEP[dt] * ry.abs())
        return
    amax = F.blocks_amax(ry, 1)
    rs = torch.clamp(amax / 448.0, min=2.0 ** -126)
    worst = F.blocks_amax(err, 1) / 448.0
    assert torch.all((s.double() - rs).abs() <= worst + 2.0 ** -23 * rs)
    # what is read back: half a step of e4m3 (2^-4 of the value, 2^-10 of the scale below the least normal number)
    sc = F.spread(s.double(), 1, rows, cols)
    assert torch.all((y.double() * sc - ry).abs() <= err + 2.0 ** -4 * (ry.abs() + err) * (1 + 2.0 ** -20) + 2.0 ** -10 * sc)
    assert torch.all(F.blocks_amax(y.double(), 1) == 448.0)  # every block uses the whole range


COLS = [1, 7, 8, 64, 130, 512, 520, 1023, 1024, 2048, 2049, 4096, 4100, 8192, 8200, 10001, 16384]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dt", [BF16, F32])
def test_forward_against_the_definition(cols, dt):
    rows = 11 if cols > 2048 else 37
    _check_forward(rows, cols, dt, rows)
    _check_forward(rows, cols, dt, 5, dt, post=False)
    _check_forward(rows, cols, dt, 1, dt, y_dt=E4M3)
    _check_forward(rows, cols, dt, 0, y_dt=E4M3, param_dt=BF16, scale=1.0)


@pytest.mark.parametrize("rows", [1, 2, 9, 100, 5000])
@pytest.mark.parametrize("cols", [96, 200])
def test_forward_numbers_of_rows(rows, cols):
    _check_forward(rows, cols, BF16, max(1, rows // 3), BF16)
    _check_forward(rows, cols, BF16, rows, y_dt=E4M3)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("cols", [200, 1001, 9001])
def test_forward_with_strides_and_odd_addresses(dt, cols):
    for pad, offset in ((1, 0), (8, 0), (3, 1)):
        _check_forward(13, cols, dt, 4, BF16, pad=pad, offset=offset)
        _check_forward(13, cols, dt, 13, y_dt=E4M3, pad=pad, offset=offset)


@pytest.mark.parametrize("cols", [300, 4096, 9000])
def test_forward_without_some_results(cols):
    _check_forward(20, cols, BF16, 20, want_y=False)
    _check_forward(20, cols, F32, 0, want_y=False, post=False)
    _check_forward(20, cols, BF16, 3, want_h=False, y_dt=E4M3)
    _check_forward(20, cols, F32, 0, want_h=False, post=False)


@pytest.mark.parametrize("cols", [60, 1024, 4096, 9000])
def test_forward_in_place(cols):
    _check_forward(70, cols, BF16, 70, in_place=True)
    _check_forward(70, cols, F32, 1, in_place=True, y_dt=E4M3)


@pytest.mark.parametrize("cols", [256, 4096, 9000])
def test_rows_of_zeros(cols):
    """Nothing in u, in x or in both: r = 1/sqrt(eps), results of zero, scales of 2^-126."""
    u, x = torch.randn(6, cols), torch.randn(6, cols)
    u[0], u[1], x[1], x[2] = 0, 0, 0, 0
    one = torch.ones(cols)
    h, y, s, r1, r2 = _forward(u, x, None, 0, one, one, 1.0, F32, y_dt=E4M3)
    assert torch.equal(h[0], x[0]) and bool((h[1] == 0).all()) and bool((y[1].float() == 0).all())
    assert bool((s[1] == 2.0 ** -126).all())
    root = 1.0 / np.sqrt(float(np.float32(1e-5)))
    assert abs(float(r1[0]) - root) <= 4 * 2.0 ** -24 * root and abs(float(r2[1]) - root) <= 4 * 2.0 ** -24 * root


# ---- gradient ---------------------------------------------------------------------------------------
def _backward(dy, dh, h, u, gate, gate_rows, post, pre, r1, r2, scale, dt, gate_dt=F32, param_dt=F32, pad=0, in_place=False,
              offset=0, skip=()):
    rows, cols = u.shape
    held = lambda v, k=1: None if v is None else F.Held(rows, cols, dt, cols + k * pad, offset, v)  # noqa: E731
    dyd, dhd, hd, ud = held(dy), held(dh, 2), held(h, 3), held(u)
    gd = F.Held(gate.shape[0], cols, gate_dt, cols + pad, offset, gate) if gate is not None else None
    dgd = F.Held(gate.shape[0], cols, gate_dt, cols + 2 * pad, offset) if gate is not None and "dgate" not in skip else None
    dx = dhd if in_place else F.Held(rows, cols, dt, cols + pad, offset)
    du = dyd if in_place else F.Held(rows, cols, dt, cols + 2 * pad, offset)
    dpost = F.Held(1, cols, F32) if post is not None and "dpost" not in skip else None
    dpre = F.Held(1, cols, F32) if dy is not None and "dpre" not in skip else None
    need = perf.perf_residual_norm_backward_workspace_bytes(rows, cols)
    ws = torch.full((need + 256,), F.GUARD, dtype=torch.uint8, device="cuda")
    postd, pred, r1d, r2d = F.vector(post, param_dt), F.vector(pre, param_dt), F.vector(r1), F.vector(r2)
    perf.perf_residual_norm_backward(
        F.at(dyd), F.at(dhd), F.at(hd) if dy is not None else None, ud.at(), F.at(gd), F.at(postd),
        F.at(pred) if dy is not None else None, F.at(r1d) if post is not None else None, F.at(r2d) if dy is not None else None,
        dx.at(), du.at(), F.at(dgd), F.at(dpost), F.at(dpre), ws.data_ptr(), rows, cols,
        dyd.ld if dyd else 0, dhd.ld if dhd else 0, hd.ld, ud.ld, gd.ld if gd else 0, gate_rows or 0, dx.ld, du.ld,
        dgd.ld if dgd else 0, scale, dt, gate_dt, param_dt, stream=G.stream())
    torch.cuda.synchronize()
    assert bool((ws[need:] == F.GUARD).all())
    out = {"dx": dx.get(), "du": du.get()}
    for name, v in (("dgate", dgd), ("dpost", dpost), ("dpre", dpre)):
        if v is not None:
            out[name] = v.get() if name == "dgate" else v.get()[0]
    return out


def _check_backward(rows, cols, dt, gate_rows=0, gate_dt=F32, param_dt=F32, post=True, with_dy=True, with_dh=True, scale=0.75, seed=0,
                    **kw):
    u, x, gate, gpost, gpre = _make(rows, cols, dt, gate_rows, gate_dt, param_dt, post, seed)
    g = np.random.default_rng(rows + cols)
    dy = torch.from_numpy(g.standard_normal((rows, cols)).astype(np.float32)).to(F.TORCH[dt]) if with_dy else None
    dh = torch.from_numpy(g.standard_normal((rows, cols)).astype(np.float32) * 0.5).to(F.TORCH[dt]) if with_dh else None
    h, _, r1, r2, _ = F.norm_ref(u, x, gate, gate_rows, gpost, gpre, scale, 1e-5)
    h, r1, r2 = h.to(F.TORCH[dt]), r1.float(), r2.float()
    got = _backward(dy, dh, h, u, gate, gate_rows, gpost, gpre, r1, r2, scale, dt, gate_dt, param_dt, **kw)
    args = (dy, dh, h, u, gate, gate_rows, gpost, gpre, r1, r2, scale)
    ref, mag = F.grad_ref(*args), F.grad_ref(*args, magnitudes=True)
    for name in got:
        # an element of dx or du: two sums over the row behind it, one inside the other; of the others: up to `rows` more
        # roundings, one for each row
        c = (2 * _depth(cols) + (0 if name in ("dx", "du") else rows + 8)) * 2.0 ** -24
        out_dt = dt if name in ("dx", "du") else gate_dt if name == "dgate" else F32
        bound = c * mag[name] * (1 + HALF_STEP[out_dt]) + HALF_STEP[out_dt] * ref[name].abs()
        worst = float(((got[name].double() - ref[name]).abs() - bound).max())
        assert worst <= 0, f"{name}: over its bound by {worst:.3e}"
    return got


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dt", [BF16, F32])
def test_backward_against_the_definition(cols, dt):
    rows = 23 if cols > 2048 else 61
    _check_backward(rows, cols, dt, rows)
    _check_backward(rows, cols, dt, 1, dt, param_dt=BF16)
    _check_backward(rows, cols, dt, 19, dt)
    _check_backward(rows, cols, dt, 5)
    _check_backward(rows, cols, dt, 0, post=False)


@pytest.mark.parametrize("rows,cols,gate_rows", [(1, 64, 1), (7, 520, 7), (1500, 100, 1500), (1500, 100, 400), (1500, 100, 17),
                                                 (1500, 100, 16), (1500, 100, 3), (1300, 1500, 700), (1300, 1500, 33), (700, 3000, 1),
                                                 (700, 3000, 100), (700, 3000, 16), (600, 5000, 250), (530, 8200, 200), (530, 8200, 2)])
def test_backward_groups_of_gates(rows, cols, gate_rows):
    """Groups inside a workgroup's run, across several runs, one for all, one for each row."""
    _check_backward(rows, cols, F32, gate_rows)
    _check_backward(rows, cols, BF16, gate_rows, BF16, post=False)


@pytest.mark.parametrize("cols", [300, 4096, 9000])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_backward_of_one_result_only(cols, dt):
    for post in (True, False):
        _check_backward(40, cols, dt, 40, with_dh=False, post=post)
        _check_backward(40, cols, dt, 0, with_dh=False, post=post)
        _check_backward(40, cols, dt, 3, with_dy=False, post=post)
        _check_backward(40, cols, dt, 0, with_dy=False, post=post)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("cols", [200, 1001, 9001])
def test_backward_with_strides_and_odd_addresses(dt, cols):
    for pad, offset in ((1, 0), (8, 0), (3, 1)):
        _check_backward(33, cols, dt, 20, BF16, pad=pad, offset=offset)


@pytest.mark.parametrize("cols", [60, 1024, 4096, 9000])
def test_backward_in_place_and_without_parameters(cols):
    for gate_rows in (1, 70):
        whole = _check_backward(70, cols, BF16, gate_rows)
        same = _check_backward(70, cols, BF16, gate_rows, in_place=True, skip=("dgate", "dpost", "dpre"))
        assert torch.equal(whole["dx"], same["dx"]) and torch.equal(whole["du"], same["du"])
        for skip in ("dgate", "dpost", "dpre"):
            some = _check_backward(70, cols, BF16, gate_rows, skip=(skip,))
            for name, v in some.items():
                assert torch.equal(v, whole[name]), name


def test_backward_against_differences():
    """Along random directions, the change of <dy, y> + <dh, h> in float64 is what the gradients say."""
    rows, cols, scale = 12, 40, 0.75
    for gate_rows, post in ((12, True), (5, True), (1, False), (0, True)):
        u, x, gate, gpost, gpre = _make(rows, cols, F32, gate_rows, F32, F32, post, seed=9)
        g = torch.Generator().manual_seed(4)
        dy, dh = (torch.randn(rows, cols, generator=g) for _ in range(2))
        names = {"du": u, "dx": x, "dpre": gpre, **({"dgate": gate} if gate_rows else {}), **({"dpost": gpost} if post else {})}

        def value(moved):
            v = {k: t.double() for k, t in names.items()}
            v.update(moved)
            h, y, _, _, _ = F.norm_ref(v["du"], v["dx"], v.get("dgate"), gate_rows, v.get("dpost"), v["dpre"], scale, 1e-5)
            return float((dy.double() * y).sum() + (dh.double() * h).sum())

        h, _, r1, r2, _ = F.norm_ref(u, x, gate, gate_rows, gpost, gpre, scale, 1e-5)
        got = _backward(dy, dh, h.float(), u, gate, gate_rows, gpost, gpre, r1.float(), r2.float(), scale, F32)
        for name, t in names.items():
            d = torch.randn(t.shape, generator=g).double()
            step = 1e-5
            change = (value({name: t.double() + step * d}) - value({name: t.double() - step * d})) / (2 * step)
            said = float((got[name].double() * d).sum())
            # differences of second order are off by about step^2; the gradient by 2^-20 of its terms
            assert abs(change - said) <= 1e-5 * float((got[name].double().abs() * d.abs()).sum()) + 1e-7, name


def test_backward_is_the_same_every_time():
    for cols in (100, 3000, 9000):
        a = _check_backward(300, cols, F32, 64)
        b = _check_backward(300, cols, F32, 64)
        assert all(torch.equal(a[k], b[k]) for k in a)


def test_backward_of_more_columns_than_a_launch_holds():
    """2^28 columns (a dimension of 2^32 threads is cut short without an error) in two runs of one row, which share a gate: small
    whole numbers in a pattern of 60 columns whose mean(t hn) is zero, so that every sum is exact."""
    rows, period, cols = 2, 60, 268436400
    c, r = torch.arange(period)[None], torch.arange(rows)[:, None]
    dy, h = 1 + (c // 2 + r) % 3, (1 - 2 * (c % 2)).expand(rows, period)  # t hn of columns 2 j and 2 j + 1 cancel
    dh, u, gate = c % 4 + r, c % 5 - 2 + r, 1 + c % 3
    H = dh + dy
    want = {"dpre": (dy * h).sum(0), "dpost": (2 * gate * H * u).sum(0), "dgate": (2 * u * H).sum(0)}  # (gamma_post and r2 are 1, r1 is 2)
    wide = lambda v: v.to(torch.bfloat16).cuda().repeat(1, cols // period)  # noqa: E731
    m = {"dy": wide(dy), "dh": wide(dh), "h": wide(h), "u": wide(u), "gate": wide(gate)}
    ones, r1, r2 = torch.ones(cols, device="cuda"), torch.full((rows,), 2.0, device="cuda"), torch.ones(rows, device="cuda")
    got = {k: torch.full((cols,), float("nan"), dtype=torch.bfloat16 if k == "dgate" else torch.float32, device="cuda") for k in want}
    dx, du = torch.empty_like(m["u"]), torch.empty_like(m["u"])
    ws = torch.empty(perf.perf_residual_norm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    p = {k: v.data_ptr() for k, v in m.items()}
    perf.perf_residual_norm_backward(p["dy"], p["dh"], p["h"], p["u"], p["gate"], ones.data_ptr(), ones.data_ptr(), r1.data_ptr(),
                                     r2.data_ptr(), dx.data_ptr(), du.data_ptr(), got["dgate"].data_ptr(), got["dpost"].data_ptr(),
                                     got["dpre"].data_ptr(), ws.data_ptr(), rows, cols, cols, cols, cols, cols, cols, rows, cols, cols, cols,
                                     1.0, BF16, BF16, F32, stream=G.stream())
    for name, v in want.items():
        assert bool((got[name].view(-1, period) == v.cuda().to(got[name].dtype)).all()), name
    assert bool((dx.view(rows, -1, period) == H.cuda().to(torch.bfloat16)[:, None]).all())
