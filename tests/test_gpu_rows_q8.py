"""Rows in 8 bits on the GPU against plain 64-bit forms: quantisation, the norm with the residual's addition, the gated
activation, and the two gradients.

Tolerances.  A scale is off by the relative error of the row's factor (q8_ref.ROW_EPS); q is within half a step of the
exact quotient, plus 127 steps times that error (a value next to a rounding boundary may fall on either side); `values`
and `h` are single roundings and must be equal bit for bit.  Gradients: every term is off by at most ROW_EPS of its
magnitude, then one rounding to the element type; sums over rows by one fp32 rounding per addition of the sum of magnitudes."""
import itertools

import pytest
import torch

from paper_2309_06973_b200 import binding as B
from paper_2309_06973_b200 import runtime as R
import q8_ref as P

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# one token and many; one column, odd widths, a vector more or less than a warp, a block, the registers of a row
SHAPES = [(1, 1), (1, 7), (3, 8), (5, 33), (2, 255), (300, 256), (300, 257), (301, 513), (200, 1024), (149, 1025), (1, 4096),
          (7, 4099), (160, 4104), (1, 8193), (2, 14336), (150, 9001), (1, 32768), (2, 32769), (151, 33000), (1, 70001)]
LAYOUTS = ["tight", "aligned", "shifted"]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def layout(rows, cols, dtype, kind, source=None):
    if kind == "tight":
        return P.Guarded(rows, cols, dtype, source=source)
    if kind == "aligned":
        return P.Guarded(rows, cols, dtype, ld=(cols + 15) // 16 * 16 + 16, source=source)
    return P.Guarded(rows, cols, dtype, ld=cols + 3, lead=1, source=source)


def out_rows(rows, cols, kind="tight", values=True):
    q = P.Guarded(rows, cols, torch.int8, ld=(cols + 15) // 16 * 16 + (16 if kind == "aligned" else 0))
    v = layout(rows, cols, BF16, kind) if values else None
    s = P.Guarded(1, rows, F32)
    out = R.RowsQ8.of(q.view, s.view[0], cols, None if v is None else v.view)
    return out, [q, s] + ([v] if v else [])


def intact(*guards):
    torch.cuda.synchronize()
    return all(g.intact() for g in guards)


@pytest.mark.parametrize("kind", LAYOUTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_rows(rows, cols, dtype, kind):
    x = layout(rows, cols, dtype, kind, torch.randn(rows, cols, generator=gen(rows + cols), device="cuda"))
    out, guards = out_rows(rows, cols, kind)
    R.quantize_rows(x.view, out)
    P.check_rows(out, x.view.double())
    assert intact(x, *guards)


@pytest.mark.parametrize("kind", LAYOUTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_rmsnorm(rows, cols, dtype, kind):
    g = gen(7 * rows + cols)
    rnd = lambda: torch.randn(rows, cols, generator=g, device="cuda")
    x, res = layout(rows, cols, dtype, kind, rnd()), layout(rows, cols, dtype, kind, 3 * rnd())
    w = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda")
    h = layout(rows, cols, dtype, kind)
    for weight, residual, hh in itertools.product((w, None), (res, None), (h, None)):
        out, guards = out_rows(rows, cols, kind, values=hh is not None)
        R.rmsnorm_q8(x.view, weight, 1e-5, out, residual=None if residual is None else residual.view, h=None if hh is None else hh.view)
        sum32 = x.view.float() + (0 if residual is None else residual.view.float())
        P.check_rows(out, P.norm_of(sum32.double(), None if weight is None else weight.double(), 1e-5))
        if hh is not None:
            assert torch.equal(hh.view, sum32.to(dtype))
        assert intact(x, res, h, *guards)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 64), (300, 200), (200, 4096), (9, 4099), (2, 40000)])
def test_rmsnorm_in_place(rows, cols, dtype):
    """The residual stream updated in place: h_out is the residual, or x, itself."""
    g = gen(rows * cols)
    x0, r0 = (torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(2))
    h = torch.empty_like(x0)
    apart = R.rmsnorm_q8(x0, None, 1e-5, R.RowsQ8(rows, cols), residual=r0, h=h)
    for onto in (0, 1):
        x, r = x0.clone(), r0.clone()
        same = R.rmsnorm_q8(x, None, 1e-5, R.RowsQ8(rows, cols), residual=r, h=(x, r)[onto])
        assert torch.equal((x, r)[onto], h) and torch.equal((r, x)[onto], (r0, x0)[onto])
        assert torch.equal(same.q[:, :cols], apart.q[:, :cols]) and torch.equal(same.scale, apart.scale)


@pytest.mark.parametrize("kind", LAYOUTS + ["halves"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_silu_gate(rows, cols, dtype, kind):
    g = gen(11 * rows + cols)
    both = 3 * torch.randn(rows, 2 * cols, generator=g, device="cuda")
    if kind == "halves":
        buf = layout(rows, 2 * cols, dtype, "tight", both)
        gate, up, bufs = buf.view[:, :cols], buf.view[:, cols:], [buf]
    else:
        bufs = [layout(rows, cols, dtype, kind, both[:, :cols]), layout(rows, cols, dtype, kind, both[:, cols:])]
        gate, up = bufs[0].view, bufs[1].view
    out, guards = out_rows(rows, cols, "tight" if kind == "halves" else kind)
    R.silu_gate_q8(gate, up, out)
    P.check_rows(out, P.silu_gate(gate.double(), up.double()))
    assert intact(*bufs, *guards)


@pytest.mark.parametrize("cols", [5, 64, 257, 4096, 4099, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_with_special_values(cols, dtype):
    """Zero rows, one Inf, one NaN, the type's lowest value, tiny rows, values at the rounding boundary."""
    x = torch.randn(9, cols, generator=gen(cols), device="cuda")
    x[0] = 0
    x[1, cols // 2] = float("inf")
    x[2, cols - 1] = float("nan")
    x[3, 0] = -float("inf")
    x = x.to(dtype)
    x[4, cols // 3] = torch.finfo(dtype).min
    x[5] = (torch.randn(cols, generator=gen(1), device="cuda") * 1e-36).to(dtype)
    x[6, : cols // 2] = -0.0
    x[7] = -x[7].abs()
    x[8] = ((torch.arange(cols, device="cuda") % 255) - 127.0).to(dtype)
    out = R.RowsQ8(9, cols, values=True)
    R.quantize_rows(x, out)
    lost = torch.tensor([1, 2, 3], device="cuda")
    fine = torch.tensor([0, 4, 5, 6, 7, 8], device="cuda")
    assert torch.isnan(out.scale[lost]).all() and not out.q[lost, :cols].any() and torch.isnan(out.values[lost]).all()
    some = R.RowsQ8.of(out.q[fine], out.scale[fine], cols, out.values[fine])
    P.check_rows(some, x[fine].double())
    assert out.scale[0] == 0 and not out.q[0, :cols].any() and not out.values[0].any()
    # the norm of the same rows: a zero row stays zero, one past fp32's squares is lost like an Inf
    R.rmsnorm_q8(x, None, 1e-6, out)
    lost = torch.tensor([1, 2, 3, 4], device="cuda")
    assert torch.isnan(out.scale[lost]).all() and not out.q[lost, :cols].any()
    assert out.scale[0] == 0 and not out.q[0, :cols].any()
    fine = torch.tensor([6, 7, 8], device="cuda")
    P.check_rows(R.RowsQ8.of(out.q[fine], out.scale[fine], cols), P.norm_of(x[fine].double(), None, 1e-6))


def test_subnormal_rows():
    """Rows whose largest value is subnormal: the step itself is subnormal (or 0), q still follows the quotients."""
    x = torch.zeros(3, 40, device="cuda")
    x[0] = torch.linspace(-1, 1, 40, device="cuda") * 1e-39
    x[1, 7] = 1e-45
    x[2] = torch.linspace(-1, 1, 40, device="cuda") * 2.0 ** -120
    out = R.quantize_rows(x, R.RowsQ8(3, 40))
    want, scale = P.rows_of(x.double())
    assert torch.all((out.q[:, :40].double() - want).abs() <= 0.5 + 127 * 2 * P.ROW_EPS)
    assert torch.all((out.scale.double() - scale).abs() <= 2.0 ** -149)


@pytest.mark.parametrize("cols", [3, 2048, 33001])
def test_no_rows_and_no_columns(cols):
    for n in (0,):
        out = R.RowsQ8(n, cols)
        R.quantize_rows(torch.empty(n, cols, device="cuda"), out)
        R.rmsnorm_q8(torch.empty(n, cols, device="cuda"), None, 1e-5, out)
        dw = torch.full((cols,), 3.0, device="cuda")
        e = torch.empty(n, cols, device="cuda")
        R.rmsnorm_q8_backward(e, e, None, 1e-5, e, dw, workspace=R.rmsnorm_q8_backward_workspace(n, cols))
        assert not dw.any()
        R.silu_gate_q8_backward(e, e, e, e, e)
    out = R.RowsQ8(5, 0)
    out.scale.fill_(7)
    R.silu_gate_q8(torch.empty(5, 0, device="cuda"), torch.empty(5, 0, device="cuda"), out)
    assert not out.scale.any()


# ---- gradients ---------------------------------------------------------------------------------------------
def norm_gradient(dy, h, w, eps, dh):
    n = h.shape[1]
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    g = dy if w is None else dy * w
    unit = h * r
    along = (g * unit).sum(1, keepdim=True) / n
    dx = r * (g - unit * along) + (0 if dh is None else dh)
    size = r * (g.abs() + unit.abs() * (g * unit).abs().sum(1, keepdim=True) / n) + (0 if dh is None else dh.abs())
    return dx, size, (dy * unit).sum(0), (dy * unit).abs().sum(0)


@pytest.mark.parametrize("kind", LAYOUTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES + [(700, 96), (1500, 1000)])
def test_rmsnorm_backward(rows, cols, dtype, kind):
    g = gen(3 * rows + cols)
    rnd = lambda: torch.randn(rows, cols, generator=g, device="cuda")
    dy, h, dh = (layout(rows, cols, dtype, kind, s * rnd()) for s in (1.0, 2.0, 0.5))
    w = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda")
    space = R.rmsnorm_q8_backward_workspace(rows, cols)
    for weight, past, want_dw in ((w, dh, True), (None, None, True), (w, None, False)):
        dx, dw = layout(rows, cols, dtype, kind), P.Guarded(1, cols, F32)
        space.fill_(0x7F)                                              # whatever the workspace held before
        R.rmsnorm_q8_backward(dy.view, h.view, weight, 1e-5, dx.view, dw.view[0] if want_dw else None,
                              dh=None if past is None else past.view, workspace=space if want_dw else None)
        ex, size, ew, wsize = norm_gradient(dy.view.double(), h.view.double(), None if weight is None else weight.double(), 1e-5,
                                            None if past is None else past.view.double())
        u = P.U32 if dtype is F32 else P.UBF
        assert torch.all((dx.view.double() - ex).abs() <= u * ex.abs() + (1 + u) * P.ROW_EPS * size)
        if want_dw:
            assert torch.all((dw.view[0].double() - ew).abs() <= (P.ROW_EPS + rows * P.U32) * wsize)
        assert intact(dy, h, dh, dx, dw)


@pytest.mark.parametrize("starts", ["shared", "any"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(2500, 5), (2400, 249), (2400, 250), (2400, 256), (900, 505), (901, 512), (310, 4089), (310, 4090), (310, 4097), (300, 5369),
                                       (300, 5371), (170, 8185), (160, 8186), (150, 16377), (150, 16384)])
def test_rmsnorm_backward_rows_off_16_bytes(rows, cols, dtype, starts):
    """Rows that start anywhere, the same way in all matrices or not, around the widths that fill a team's registers; what stands
    beside them is NaN, and reaches no result.  Rows with an infinity stay by themselves."""
    g = gen(rows + cols)
    places = [(3, 3)] * 4 if starts == "shared" else [(3, 3), (0, 1), (5, 7), (1, 1)]   # columns before and between rows
    def matrix(i, source=None):
        before, between = places[i]
        flat = torch.full((before + rows * (cols + between),), float("nan"), device="cuda", dtype=dtype)
        view = flat[before:].as_strided((rows, cols), (cols + between, 1))
        if source is not None:
            view.copy_(source)
        return flat, view
    rnd = lambda: torch.randn(rows, cols, generator=g, device="cuda")
    (_, dy), (_, h), (_, dh) = matrix(0, rnd()), matrix(1, 2 * rnd()), matrix(2, rnd())
    flat, dx = matrix(3)
    w = 1 + 0.3 * torch.randn(cols + 1, generator=g, device="cuda")[1:]
    dw = torch.empty(cols, device="cuda")
    space = R.rmsnorm_q8_backward_workspace(rows, cols)
    R.rmsnorm_q8_backward(dy, h, w, 1e-5, dx, dw, dh=dh, workspace=space)
    ex, size, ew, wsize = norm_gradient(dy.double(), h.double(), w.double(), 1e-5, dh.double())
    u = P.U32 if dtype is F32 else P.UBF
    assert torch.all((dx.double() - ex).abs() <= u * ex.abs() + (1 + u) * P.ROW_EPS * size)
    assert torch.all((dw.double() - ew).abs() <= (P.ROW_EPS + rows * P.U32) * wsize)
    assert int(flat.isnan().sum()) == flat.numel() - rows * cols                         # written: the rows and nothing else
    first = dx.clone()
    row = rows // 2
    dy[row, cols - 1] = float("inf")
    R.rmsnorm_q8_backward(dy, h, w, 1e-5, dx, dh=dh)
    assert not dx[row].isfinite().any()
    dx[row] = first[row]
    assert torch.equal(dx, first)


@pytest.mark.parametrize("starts", ["even", "shared", "any"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(300, 64), (300, 1000), (200, 4096), (40, 4099), (9, 8200), (5, 16384), (3, 40000)])
def test_rmsnorm_backward_of_lost_rows(rows, cols, dtype, starts):
    """A row whose squares pass fp32 is lost as in the norm itself: its gradient is NaN, and with it the sum over rows, instead of one
    that looks like a number.  The other rows keep their bits."""
    if starts == "even":
        cols = (cols + 7) // 8 * 8
    g = gen(rows + cols)
    def matrix(i, scale):
        before, between = {"even": (0, (-cols) % 8), "shared": (3, 3), "any": [(3, 3), (0, 1), (5, 7), (1, 1)][i]}[starts]
        flat = torch.zeros(before + rows * (cols + between) + 8, device="cuda", dtype=dtype)
        view = flat[before:].as_strided((rows, cols), (cols + between, 1))
        view.copy_(scale * torch.randn(rows, cols, generator=g, device="cuda"))
        return view
    dy, h, dh, dx = matrix(0, 1.0), matrix(1, 2.0), matrix(2, 0.5), matrix(3, 1.0)
    w = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda")
    dw, space = torch.empty(cols, device="cuda"), R.rmsnorm_q8_backward_workspace(rows, cols)
    R.rmsnorm_q8_backward(dy, h, w, 1e-5, dx, dw, dh=dh, workspace=space)
    first = dx.clone()
    assert first.isfinite().all() and dw.isfinite().all()
    lost = [0, rows // 2]
    h[lost[0]] = 1e25
    h[lost[1], cols // 3] = float("inf")
    R.rmsnorm_q8_backward(dy, h, w, 1e-5, dx, dw, dh=dh, workspace=space)
    assert dx[lost].isnan().all() and dw.isnan().all()
    dx[lost] = first[lost]
    assert torch.equal(dx, first)
    forward = R.rmsnorm_q8(h, w, 1e-5, R.RowsQ8(rows, cols))
    assert forward.scale[lost].isnan().all() and int(forward.scale.isnan().sum()) == len(set(lost))


@pytest.mark.parametrize("rows,cols", [(3, 33), (40, 520), (2, 4099)])
def test_rmsnorm_backward_against_differences(rows, cols):
    """<dx, d> + <dweight, e> against the difference quotient of the norm itself (64 bits), and the sum of both for x and
    the residual, which share dx."""
    g = gen(cols)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    h, dy, w = rnd(rows, cols), rnd(rows, cols), 1 + 0.3 * rnd(cols)
    dx, dw = torch.empty_like(h), torch.empty_like(w)
    R.rmsnorm_q8_backward(dy, h, w, 1e-5, dx, dw, workspace=R.rmsnorm_q8_backward_workspace(rows, cols))
    d, e = rnd(rows, cols).double(), rnd(cols).double()
    loss = lambda s: float((dy.double() * P.norm_of(h.double() + s * d, w.double() + s * e, 1e-5)).sum())
    step = 1e-5
    slope = (loss(step) - loss(-step)) / (2 * step)
    got = float((dx.double() * d).sum() + (dw.double() * e).sum())
    terms = float((dx.double() * d).abs().sum() + (dw.double() * e).abs().sum())
    assert abs(got - slope) <= (P.ROW_EPS + rows * P.U32) * terms + 1e-7 * terms


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(5, 100), (400, 4096), (3, 4099), (2, 20000)])
def test_rmsnorm_backward_in_place_and_repeatable(rows, cols, dtype):
    g = gen(cols + 1)
    src = [torch.randn(rows, cols, generator=g, device="cuda").to(dtype) for _ in range(3)]
    w = torch.randn(cols, generator=g, device="cuda")
    space = R.rmsnorm_q8_backward_workspace(rows, cols)
    dx, dw = torch.empty_like(src[0]), torch.empty_like(w)
    R.rmsnorm_q8_backward(src[0], src[1], w, 1e-5, dx, dw, dh=src[2], workspace=space)
    for onto in range(3):
        dy, h, dh = (s.clone() for s in src)
        dw2 = torch.empty_like(w)
        R.rmsnorm_q8_backward(dy, h, w, 1e-5, (dy, h, dh)[onto], dw2, dh=dh, workspace=space)
        assert torch.equal((dy, h, dh)[onto], dx) and torch.equal(dw2, dw)


@pytest.mark.parametrize("kind", LAYOUTS + ["halves"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_silu_gate_backward(rows, cols, dtype, kind):
    g = gen(5 * rows + cols)
    rnd = lambda c=cols: torch.randn(rows, c, generator=g, device="cuda")
    dy = layout(rows, cols, dtype, "tight" if kind == "halves" else kind, rnd())
    if kind == "halves":
        src, dst = layout(rows, 2 * cols, dtype, "tight", 3 * rnd(2 * cols)), layout(rows, 2 * cols, dtype, "tight")
        gate, up, dgate, dup, bufs = src.view[:, :cols], src.view[:, cols:], dst.view[:, :cols], dst.view[:, cols:], [src, dst]
    else:
        bufs = [layout(rows, cols, dtype, kind, 3 * rnd()), layout(rows, cols, dtype, kind, rnd())] + [layout(rows, cols, dtype, kind) for _ in range(2)]
        gate, up, dgate, dup = (b.view for b in bufs)
    R.silu_gate_q8_backward(dy.view, gate, up, dgate, dup)
    d, a, b = dy.view.double(), gate.double(), up.double()
    s = 1 / (1 + torch.exp(-a))
    eg, eu = d * b * s * (1 + a * (1 - s)), d * a * s
    size = (d * b * s).abs() * (1 + (a * (1 - s)).abs())
    u = P.U32 if dtype is F32 else P.UBF
    # exp in single precision is good to a few units in the last place of its argument's size: |gate| < 32 here
    assert float(a.abs().max()) < 32
    assert torch.all((dgate.double() - eg).abs() <= u * eg.abs() + (1 + u) * P.ROW_EPS * size)
    assert torch.all((dup.double() - eu).abs() <= u * eu.abs() + (1 + u) * P.ROW_EPS * eu.abs())
    assert intact(dy, *bufs)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(3, 1), (3, 2), (9, 7), (17, 9), (5, 241), (9, 247), (9, 248), (9, 249), (9, 255), (9, 257), (3, 496), (2, 1985), (5, 5003), (2, 11003)])
def test_silu_gate_backward_rows_off_16_bytes(rows, cols, dtype):
    """Every place within 16 bytes at which a row of each matrix may begin, what stands beside the rows NaN; and in place."""
    g = gen(7 * rows + cols)
    u = P.U32 if dtype is F32 else P.UBF
    for turn in range(16):
        def matrix(i, source=None):
            before, between = [(0, 0, 0, turn % 8, turn // 2), (1, 3, turn, 2, 5), (turn, 1, 8, 3 * turn, 7), (5, 5, 5, 5, turn), (turn, 0, 1, 2, 3)][turn % 5][i], (turn + (i * turn) % 3) % 9
            flat = torch.full((before + rows * (cols + between) + 8,), float("nan"), device="cuda", dtype=dtype)
            view = flat[before:].as_strided((rows, cols), (cols + between, 1))
            if source is not None:
                view.copy_(source)
            return flat, view
        rnd = lambda s: s * torch.randn(rows, cols, generator=g, device="cuda")
        (_, dy), (fg, gate), (fu, up) = matrix(0, rnd(1)), matrix(1, rnd(3)), matrix(2, rnd(1))
        (fdg, dgate), (fdu, dup) = matrix(3), matrix(4)
        R.silu_gate_q8_backward(dy, gate, up, dgate, dup)
        d, a, b = dy.double(), gate.double(), up.double()
        s = 1 / (1 + torch.exp(-a))
        eg, eu = d * b * s * (1 + a * (1 - s)), d * a * s
        size = (d * b * s).abs() * (1 + (a * (1 - s)).abs())
        assert torch.all((dgate.double() - eg).abs() <= u * eg.abs() + (1 + u) * P.ROW_EPS * size)
        assert torch.all((dup.double() - eu).abs() <= u * eu.abs() + (1 + u) * P.ROW_EPS * eu.abs())
        for flat in (fdg, fdu):
            assert int(flat.isnan().sum()) == flat.numel() - rows * cols                  # written: the rows and nothing else
        R.silu_gate_q8_backward(dy, gate, up, gate, up)
        assert torch.equal(gate, dgate) and torch.equal(up, dup)
        for flat in (fg, fu):
            assert int(flat.isnan().sum()) == flat.numel() - rows * cols


def test_silu_gate_backward_against_differences_and_in_place():
    rows, cols = 6, 77
    g = gen(2)
    gate, up, dy, d, e = (torch.randn(rows, cols, generator=g, device="cuda") for _ in range(5))
    dg, du = torch.empty_like(gate), torch.empty_like(up)
    R.silu_gate_q8_backward(dy, gate, up, dg, du)
    loss = lambda s: float((dy.double() * P.silu_gate(gate.double() + s * d.double(), up.double() + s * e.double())).sum())
    slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
    terms = float((dg.double() * d.double()).abs().sum() + (du.double() * e.double()).abs().sum())
    assert abs(float((dg.double() * d).sum() + (du.double() * e).sum()) - slope) <= P.ROW_EPS * terms + 1e-7 * terms
    a, b = gate.clone(), up.clone()
    R.silu_gate_q8_backward(dy, a, b, a, b)                            # the gradients take their inputs' place
    assert torch.equal(a, dg) and torch.equal(b, du)


def test_gates_of_every_size():
    """The sigmoid's argument is rounded to fp32 before its power of two, and so is that factor's constant: each leaves an error of |gate| units
    of 2^-24 at most; the power, the reciprocal and the sum between them take twelve more.  Above 17 the sum is 1."""
    rows, cols = 400, 1001
    g = gen(6)
    gate = (torch.rand(rows, cols, generator=g, device="cuda") * 2 - 1) * 87.3
    dy, up = (torch.randn(rows, cols, generator=g, device="cuda") for _ in range(2))
    dg, du = torch.empty_like(gate), torch.empty_like(gate)
    R.silu_gate_q8_backward(dy, gate, up, dg, du)
    d, a, b = dy.double(), gate.double(), up.double()
    s = 1 / (1 + torch.exp(-a))
    least = 2.0 ** -126 * (1 + a.abs()) * (1 + d.abs())                # (what is below fp32's normal numbers)
    eu = d * a * s
    assert torch.all((du.double() - eu).abs() <= (2 * a.abs() + 14) * P.U32 * eu.abs() + least)
    size = (d * b * s).abs() * (1 + (a * (1 - s)).abs())
    assert torch.all((dg.double() - d * b * s * (1 + a * (1 - s))).abs() <= (3 * a.abs() + 16) * P.U32 * size + least * (1 + b.abs()))
    out = R.silu_gate_q8(gate, up, R.RowsQ8(rows, cols))
    P.check_rows(out, P.silu_gate(a, b), eps=(2 * 87.3 + 16) * P.U32)


def test_large_gates_saturate():
    gate = torch.tensor([[-200.0, -90.0, -88.0, -50.0, 50.0, 88.0, 90.0, 200.0, 0.0, -0.0]], device="cuda")
    ones = torch.ones_like(gate)
    dg, du = torch.empty_like(gate), torch.empty_like(gate)
    R.silu_gate_q8_backward(ones, gate, ones, dg, du)
    s = 1 / (1 + torch.exp(-gate.double()))
    assert torch.allclose(du.double(), gate.double() * s, rtol=1e-4, atol=1e-30)
    assert torch.allclose(dg.double(), s * (1 + gate.double() * (1 - s)), rtol=1e-4, atol=1e-30)


# ---- streams, graphs, long rows' offsets, refusals -----------------------------------------------------------
def test_on_a_side_stream_and_in_a_graph():
    rows, cols = 257, 1031
    x = torch.randn(rows, cols, generator=gen(9), device="cuda").to(BF16)
    want = R.rmsnorm_q8(x, None, 1e-5, R.RowsQ8(rows, cols))
    torch.cuda.synchronize()
    side, out = torch.cuda.Stream(), R.RowsQ8(rows, cols)
    with torch.cuda.stream(side):
        R.rmsnorm_q8(x, None, 1e-5, out)
        side.synchronize()
        assert torch.equal(out.q[:, :cols], want.q[:, :cols])
        out.q.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            R.rmsnorm_q8(x, None, 1e-5, out)
        x.mul_(2.0)                                                    # a replay works on what is there now
        graph.replay()
        side.synchronize()
    again = R.rmsnorm_q8(x, None, 1e-5, R.RowsQ8(rows, cols))
    assert torch.equal(out.q[:, :cols], again.q[:, :cols]) and torch.equal(out.scale, again.scale)


def test_offsets_past_32_bits():
    """Rows so far apart that the last one starts past 2^32 elements."""
    ld, rows, cols = (1 << 30) + 16, 5, 40
    buf = torch.empty(4 * ld + 64, dtype=BF16, device="cuda")
    x = buf.as_strided((rows, cols), (ld, 1), 0)
    x.copy_(torch.randn(rows, cols, generator=gen(4), device="cuda"))
    out = R.quantize_rows(x, R.RowsQ8(rows, cols, values=True))
    P.check_rows(out, x.double())
    dg = torch.empty(rows, cols, dtype=BF16, device="cuda")
    R.silu_gate_q8_backward(dg.fill_(1), x, x, x, dg)                  # written there, too
    torch.cuda.synchronize()
    assert torch.isfinite(x.float()).all()


def test_runtime_refuses_wrong_tensors():
    out = R.RowsQ8(4, 32)
    x = torch.zeros(4, 32, device="cuda")
    for bad in (x[:, :31], x.t(), x.half(), x.cpu(), torch.zeros(32, 4, device="cuda").t(), x.double()):
        with pytest.raises(ValueError):
            R.quantize_rows(bad, out)
    with pytest.raises(ValueError):
        R.rmsnorm_q8(x, torch.ones(31, device="cuda"), 1e-5, out)
    with pytest.raises(ValueError):
        R.rmsnorm_q8(x, None, 1e-5, out, residual=x.to(BF16))
    with pytest.raises(B.DnnsError):
        R.quantize_rows(x[:1].expand(4, 32), out)                      # rows on top of one another: ld below the columns
    with pytest.raises(B.DnnsError):
        R.rmsnorm_q8(x, None, 0.0, out)
