"""What the calls on rows in 8 bits promise beside their results."""
import ctypes as C

import pytest
import torch

from paper_2309_06973_b200 import binding as B
from paper_2309_06973_b200 import runtime as R

pytestmark = pytest.mark.gpu


def rows8(rows, cols, values=False):
    out = R.RowsQ8(rows, cols, values=values)
    return R.quantize_rows(torch.randn(rows, cols, device="cuda"), out)


def test_tensors_of_rows_are_fixed():
    """Another tensor put in a tensor's place would go unseen: it is refused."""
    rows = rows8(4, 64)
    for name in ("q", "scale", "values"):
        with pytest.raises(AttributeError):
            setattr(rows, name, torch.zeros(4, 64, device="cuda"))


def test_rows_whose_tensors_are_given_other_storage():
    """Addresses are those of the call, not of the time when the rows were made."""
    x, w, y = torch.randn(4, 600, device="cuda"), rows8(8, 600), torch.empty(4, 8, device="cuda")
    rows = R.RowsQ8(4, 600, values=True)
    old = [t.detach() for t in (rows.q, rows.scale, rows.values)]
    R.quantize_rows(x, rows)
    want = [t.clone() for t in old]
    for t, o in zip((rows.q, rows.scale, rows.values), old):
        t.data = torch.empty_like(o)
        o.fill_(5)
    R.quantize_rows(x, rows)
    for t, o, v in zip((rows.q, rows.scale, rows.values), old, want):
        assert t.data_ptr() != o.data_ptr() and torch.equal(t[..., :600], v[..., :600]) and bool((o == 5).all())
    R.LinearQ8(w)(rows, y)
    part = rows.q[:, :600].double() @ w.q[:, :600].double().t()
    assert torch.allclose(y.double(), part * rows.scale.double()[:, None] * w.scale.double(), rtol=1e-6)


def test_rows_whose_tensors_lost_their_storage_are_refused():
    """(512 columns at their own distance, which a layer uses where they are: nothing here touches what is gone.)"""
    x, good, y = torch.randn(4, 512, device="cuda"), rows8(4, 512), torch.empty(4, 8, device="cuda")
    for lose in (lambda t: t.untyped_storage().resize_(0), lambda t: t.resize_(0), lambda t: t.untyped_storage().resize_(t.untyped_storage().nbytes() - 2 * t.element_size()),
                 lambda t: t.unsqueeze_(0)):
        for which in ("scale", "values", "q"):
            rows = R.RowsQ8.of(torch.zeros(4, 512, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda"), 512,
                               torch.zeros(4, 512, dtype=torch.bfloat16, device="cuda"))
            lose(getattr(rows, which))
            for call in (lambda: R.quantize_rows(x, rows), lambda: R.rmsnorm_q8(x, None, 1e-5, rows), lambda: R.silu_gate_q8(x, x, rows),
                         lambda: R.LinearQ8(rows8(8, 512))(rows, y), lambda: R.LinearQ8(rows)(good, torch.empty(4, 4, device="cuda"))):
                with pytest.raises(ValueError, match="rows: a tensor of the rows"):
                    call()


def needs_grad(*shape, dtype=torch.float32):
    return torch.randn(*shape, device="cuda").to(dtype).requires_grad_()


TENSORS = {"quantize_rows": ["x"], "rmsnorm_q8": ["x", "weight", "residual", "h"],
           "rmsnorm_q8_backward": ["dy", "h", "weight", "dx", "dweight", "dh"], "silu_gate_q8": ["gate", "up"],
           "silu_gate_q8_backward": ["dy", "gate", "up", "dgate", "dup"], "LinearQ8": ["bias", "y"]}


def call_of(name, which):
    """The call, with that tensor of its own requiring a gradient."""
    vectors = {"weight": (64,), "dweight": (64,), "bias": (8,), "y": (4, 8)}
    t = [torch.randn(*vectors.get(n, (4, 64)), device="cuda").requires_grad_(n == which) for n in TENSORS[name]]
    out, space = R.RowsQ8(4, 64, values=True), R.rmsnorm_q8_backward_workspace(4, 64)
    return {"quantize_rows": lambda: R.quantize_rows(t[0], out),
            "rmsnorm_q8": lambda: R.rmsnorm_q8(t[0], t[1], 1e-5, out, residual=t[2], h=t[3]),
            "rmsnorm_q8_backward": lambda: R.rmsnorm_q8_backward(t[0], t[1], t[2], 1e-5, t[3], t[4], dh=t[5], workspace=space),
            "silu_gate_q8": lambda: R.silu_gate_q8(t[0], t[1], out),
            "silu_gate_q8_backward": lambda: R.silu_gate_q8_backward(*t),
            "LinearQ8": lambda: R.LinearQ8(rows8(8, 64), t[0])(rows8(4, 64), t[1])}[name]


@pytest.mark.parametrize("name,which", [(name, which) for name in TENSORS for which in TENSORS[name]])
def test_a_result_is_not_cut_off_from_a_graph_unsaid(name, which):
    """The calls record nothing for autograd: a tensor that requires a gradient is refused where it would be recorded, and taken
    under no_grad and inference_mode."""
    with pytest.raises(ValueError, match=f"{which}: requires a gradient.*no_grad"):
        call_of(name, which)()
    with torch.no_grad():
        call_of(name, which)()
    with torch.inference_mode():
        call_of(name, which)()
    call_of(name, None)()


def test_scales_and_values_that_require_a_gradient():
    q = torch.zeros(4, 64, dtype=torch.int8, device="cuda")
    for scale, values in ((needs_grad(4), None), (torch.ones(4, device="cuda"), needs_grad(4, 64, dtype=torch.bfloat16))):
        rows = R.RowsQ8.of(q, scale, 64, values)
        with pytest.raises(ValueError, match="no_grad"):
            R.quantize_rows(torch.randn(4, 64, device="cuda"), rows)
        with torch.no_grad():
            R.quantize_rows(torch.randn(4, 64, device="cuda"), rows)
    with pytest.raises(ValueError, match="no_grad"):
        R.LinearQ8(rows8(8, 64))(R.RowsQ8.of(q, needs_grad(4), 64), torch.empty(4, 8, device="cuda"))


def test_writes_are_counted():
    """Every output's version goes up, as after any write of torch, so that autograd notices a saved tensor that was overwritten."""
    new = lambda *s, dtype=torch.float32: torch.randn(*s, device="cuda").to(dtype)
    out, dx, dw, y, h = R.RowsQ8(4, 64, values=True), new(4, 64), new(64), new(4, 8), new(4, 64)
    space, layer, dg, du = R.rmsnorm_q8_backward_workspace(4, 64), R.LinearQ8(rows8(8, 64)), new(4, 64), new(4, 64)
    rows = [out.q, out.scale, out.values]
    calls = [(lambda: R.quantize_rows(new(4, 64), out), rows),
             (lambda: R.rmsnorm_q8(new(4, 64), None, 1e-5, out, h=h), rows + [h]),
             (lambda: R.silu_gate_q8(new(4, 64), new(4, 64), out), rows),
             (lambda: R.rmsnorm_q8_backward(new(4, 64), new(4, 64), None, 1e-5, dx, dw, workspace=space), [dx, dw]),
             (lambda: R.silu_gate_q8_backward(new(4, 64), new(4, 64), new(4, 64), dg, du), [dg, du]),
             (lambda: layer(rows8(4, 64), y), [y])]
    for call, written in calls:
        before = [t._version for t in written]
        call()
        assert all(t._version > b for t, b in zip(written, before))
    # the residual stream, saved by an ordinary operator and then updated in place
    w, res = needs_grad(4, 64), new(4, 64)
    loss = (w * res).sum()
    R.rmsnorm_q8(new(4, 64), None, 1e-5, out, residual=res, h=res)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_rows_at_addresses():
    """Memory that a program keeps itself, without tensors: the same results."""
    x, w, y = torch.randn(4, 600, device="cuda"), rows8(8, 600), torch.empty(2, 4, 8, device="cuda")
    rows, raw = R.quantize_rows(x, R.RowsQ8(4, 600, values=True)), R.RowsQ8(4, 600, values=True)
    plain = R._native.rows(raw.q.data_ptr(), raw.q.stride(0), raw.scale.data_ptr(), raw.values.data_ptr(), 600, 4, 600, 0)
    assert R._native.quantize_rows(x, plain) == 0
    for name in ("q", "scale", "values"):
        assert torch.equal(getattr(rows, name)[..., :600], getattr(raw, name)[..., :600])
    layer = R.LinearQ8(w)
    for r, out in ((rows._c, y[0]), (plain, y[1])):
        assert R._native.linear(r, w._c, None, out, layer.status.data_ptr()) == 0
    assert torch.equal(y[0], y[1])


def test_status_of_a_layer_that_ran_on_another_stream():
    """device_status() waits for whatever stream the layer ran on."""
    layer, side = R.LinearQ8(rows8(8, 64)), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
        layer.status.fill_(B.DNNS_ERR_TIMEOUT)                         # what a kernel of the layer would do there
    assert layer.device_status() == B.DNNS_ERR_TIMEOUT
    assert layer.device_status() == B.DNNS_OK


def test_an_error_is_reported_by_its_own_call_only():
    """A launch that CUDA refuses (on the legacy stream while a stream that waits for it is captured) fails its call; the next one,
    which runs, does not report it again."""
    cuda = C.CDLL("libcuda.so.1")
    torch.cuda.synchronize()
    x, out, w, h = torch.randn(4, 64, device="cuda"), rows8(4, 64), rows8(8, 64), torch.randn(4, 64, device="cuda")
    y, dw, status = torch.empty(4, 8, device="cuda"), torch.empty(64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    space = R.rmsnorm_q8_backward_workspace(4, 64)
    L, p = B.lib(), lambda t: t.data_ptr()
    calls = [lambda: L.dnns_quantize_rows(p(x), 64, 0, 4, 64, p(out.q), 64, p(out.scale), None, 0, None),
             lambda: L.dnns_rmsnorm_backward(p(x), 64, p(h), 64, None, 1e-5, None, 0, 0, 4, 64, p(x), 64, p(dw), p(space), space.numel(), None),
             lambda: L.dnns_silu_gate_backward(p(x), 64, p(h), 64, p(h), 64, 0, 4, 64, p(x), 64, p(h), 64, None),
             lambda: L.dnns_linear_quantized(p(out.q), 64, p(out.scale), p(w.q), 64, p(w.scale), None, 4, 64, 8, 0, p(y), 8, p(status), None)]
    torch.cuda.synchronize()
    for call in calls:
        stream, graph = C.c_void_p(), C.c_void_p()
        assert cuda.cuStreamCreate(C.byref(stream), 0) == 0            # a stream that waits for the legacy one
        assert cuda.cuStreamBeginCapture_v2(stream, 2) == 0            # (relaxed: other calls of this thread stay allowed)
        refused = call()
        cuda.cuStreamEndCapture(stream, C.byref(graph))
        if graph.value:
            cuda.cuGraphDestroy(graph)
        assert cuda.cuStreamDestroy_v2(stream) == 0
        assert refused == B.DNNS_ERR_CUDA
        assert call() == B.DNNS_OK
    torch.cuda.synchronize()


def test_the_binding_makes_the_same_calls():
    """binding.py's functions on device addresses against the calls from torch tensors, bit for bit, and their errors."""
    rows, cols, out_cols = 5, 600, 72
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x, res, dh = (torch.randn(rows, cols, generator=g, device="cuda").bfloat16() for _ in range(3))
    w, bias = torch.randn(cols, generator=g, device="cuda"), torch.randn(out_cols, generator=g, device="cuda")
    layer = R.LinearQ8(R.quantize_rows(torch.randn(out_cols, cols, generator=g, device="cuda"), R.RowsQ8(out_cols, cols)), bias)
    space, p = R.rmsnorm_q8_backward_workspace(rows, cols), lambda t: t.data_ptr()
    assert space.numel() == B.dnns_rmsnorm_backward_workspace_bytes(rows, cols) and B.dnns_quantized_row_bytes(cols) == 608
    a, b = R.RowsQ8(rows, cols, values=True), R.RowsQ8(rows, cols, values=True)
    ld, stream = a.q.stride(0), torch.cuda.current_stream().cuda_stream
    new = lambda: [torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16) for _ in range(2)]

    def same(*pairs):
        for r in (a, b):
            pairs += ((r.q[:, :cols].clone(), r.scale.clone(), r.values.clone()),)
        for u, v in list(pairs[:-2]) + list(zip(*pairs[-2:])):
            assert torch.equal(u, v)

    R.quantize_rows(x, a)
    B.dnns_quantize_rows(p(x), cols, B.DNNS_BF16, rows, cols, p(b.q), ld, p(b.scale), p(b.values), cols, stream)
    same()
    R.silu_gate_q8(x, res, a)
    B.dnns_silu_gate_quantize(p(x), cols, p(res), cols, B.DNNS_BF16, rows, cols, p(b.q), ld, p(b.scale), p(b.values), cols, stream)
    same()
    h1, h2 = new()
    R.rmsnorm_q8(x, w, 1e-5, a, residual=res, h=h1)
    B.dnns_rmsnorm_quantize(p(x), cols, p(res), cols, p(w), 1e-5, B.DNNS_BF16, rows, cols, p(h2), cols, p(b.q), ld, p(b.scale), p(b.values), cols, stream)
    same((h1, h2))
    (d1, d2), (w1, w2) = new(), (torch.empty_like(w), torch.empty_like(w))
    R.rmsnorm_q8_backward(x, h1, w, 1e-5, d1, w1, dh=dh, workspace=space)
    B.dnns_rmsnorm_backward(p(x), cols, p(h1), cols, p(w), 1e-5, p(dh), cols, B.DNNS_BF16, rows, cols, p(d2), cols, p(w2), p(space), space.numel(), stream)
    same((d1, d2), (w1, w2))
    (g1, g2), (u1, u2) = new(), new()
    R.silu_gate_q8_backward(dh, x, res, g1, u1)
    B.dnns_silu_gate_backward(p(dh), cols, p(x), cols, p(res), cols, B.DNNS_BF16, rows, cols, p(g2), cols, p(u2), cols, stream)
    same((g1, g2), (u1, u2))
    y1, y2 = torch.empty(rows, out_cols, device="cuda"), torch.empty(rows, out_cols, device="cuda")
    layer(a, y1)
    B.dnns_linear_quantized(p(a.q), ld, p(a.scale), p(layer.weight.q), ld, p(layer.weight.scale), p(bias), rows, cols, out_cols, B.DNNS_F32, p(y2), out_cols,
                            p(layer.status), stream)
    same((y1, y2))
    for bad in (lambda: B.dnns_quantize_rows(p(x), cols - 1, B.DNNS_BF16, rows, cols, p(b.q), ld, p(b.scale)),
                lambda: B.dnns_rmsnorm_quantize(p(x), cols, 0, 0, 0, 0.0, B.DNNS_BF16, rows, cols, 0, 0, p(b.q), ld, p(b.scale)),
                lambda: B.dnns_rmsnorm_backward(p(x), cols, p(h1), cols, 0, 1e-5, 0, 0, B.DNNS_BF16, rows, cols, p(d2), cols, p(w2), p(space), 16),
                lambda: B.dnns_silu_gate_quantize(p(x), cols, 0, cols, B.DNNS_BF16, rows, cols, p(b.q), ld, p(b.scale)),
                lambda: B.dnns_silu_gate_backward(p(dh), cols, p(x), cols, p(res), cols, 7, rows, cols, p(g2), cols, p(u2), cols),
                lambda: B.dnns_linear_quantized(p(a.q), ld, p(a.scale), p(layer.weight.q), ld, p(layer.weight.scale), 0, rows, cols, out_cols, B.DNNS_F32, p(y2),
                                                out_cols, 0)):
        with pytest.raises(B.DnnsError):
            bad()


@pytest.mark.parametrize("rows,n", [(1, 1), (1, 3000), (3, 257), (70000, 5)])
def test_products_of_no_columns(rows, n):
    """The bias alone, but a NaN scale is still seen, in its row and in its channel; rows of y apart."""
    for dtype in (torch.float32, torch.bfloat16):
        xs, ws, bias = torch.ones(rows, device="cuda"), torch.ones(n, device="cuda"), torch.randn(n, device="cuda")
        x, w = (R.RowsQ8.of(torch.zeros(len(s), 16, dtype=torch.int8, device="cuda"), s, 0) for s in (xs, ws))
        flat = torch.full((rows * (n + 3),), 7.0, device="cuda", dtype=dtype)
        y = flat.as_strided((rows, n), (n + 3, 1))
        R.LinearQ8(w, bias)(x, y)
        assert torch.equal(y, bias.to(dtype).expand(rows, n))
        xs[rows - 1] = ws[n // 2] = float("nan")
        R.LinearQ8(w, bias)(x, y)
        assert y[rows - 1].isnan().all() and y[:, n // 2].isnan().all() and int(y.isnan().sum()) == rows + n - 1
        assert bool((flat.as_strided((rows, 3), (n + 3, 1), n) == 7).all())
