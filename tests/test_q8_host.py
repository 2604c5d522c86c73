"""CPU checks of the calls on rows in 8 bits: every refusal comes from the host, before anything is launched."""
import pytest

from paper_2309_06973_b200 import binding as B

A = 0x10000000           # made-up aligned device addresses: nothing here gets as far as a launch
OK, INVALID, UNSUPPORTED, WORKSPACE = B.DNNS_OK, B.DNNS_ERR_INVALID_ARG, B.DNNS_ERR_UNSUPPORTED, B.DNNS_ERR_WORKSPACE


def call(name, defaults, **change):
    args = dict(defaults)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(B.lib(), name)(*args.values(), None)


QUANT = dict(x=A, ldx=64, dtype=0, rows=4, cols=64, q=A, ldq=64, scale=A, values=None, ldv=0)
NORM = dict(x=A, ldx=64, res=None, ldr=0, weight=None, eps=1e-5, dtype=1, rows=4, cols=64, h=None, ldh=0, q=A, ldq=64, scale=A,
            values=None, ldv=0)
GATE = dict(gate=A, ldg=64, up=A, ldu=64, dtype=1, rows=4, cols=64, q=A, ldq=64, scale=A, values=None, ldv=0)
NORM_BACK = dict(dy=A, lddy=64, h=A, ldh=64, weight=None, eps=1e-5, dh=None, lddh=0, dtype=0, rows=4, cols=64, dx=A, lddx=64,
                 dweight=None, ws=None, ws_bytes=0)
GATE_BACK = dict(dy=A, lddy=64, gate=A, ldg=64, up=A, ldu=64, dtype=1, rows=4, cols=64, dgate=A, lddg=64, dup=A, lddu=64)
LINEAR = dict(xq=A, ldx=64, xs=A, wq=A, ldw=64, ws=A, bias=None, rows=4, k=64, n=8, dtype=1, y=A, ldy=8, status=A)


@pytest.mark.parametrize("change,want", [
    (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(ldx=63), INVALID), (dict(ldq=48), INVALID),
    (dict(ldq=72), INVALID), (dict(q=A + 8), INVALID), (dict(x=A + 2), INVALID), (dict(scale=A + 2), INVALID), (dict(rows=-1), INVALID),
    (dict(cols=-1), INVALID), (dict(values=A, ldv=63), INVALID), (dict(values=A + 1, ldv=64), INVALID), (dict(dtype=2), UNSUPPORTED),
    (dict(rows=1 << 31), UNSUPPORTED), (dict(cols=1 << 31), UNSUPPORTED), (dict(ldx=1 << 60), UNSUPPORTED), (dict(rows=0), OK),
    (dict(rows=0, x=None, q=None, scale=None), OK)])
def test_quantize_rows_refuses(change, want):
    assert call("dnns_quantize_rows", QUANT, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(eps=1e-39), INVALID), (dict(x=None), INVALID), (dict(res=A, ldr=1), INVALID), (dict(res=A + 1, ldr=64), INVALID),
    (dict(h=A, ldh=63), INVALID), (dict(h=A + 1, ldh=64), INVALID), (dict(weight=A + 2), INVALID), (dict(dtype=-1), UNSUPPORTED),
    (dict(res=A, ldr=1 << 60), UNSUPPORTED), (dict(rows=0), OK)])
def test_rmsnorm_refuses(change, want):
    assert call("dnns_rmsnorm_quantize", NORM, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(up=None), INVALID), (dict(gate=None), INVALID), (dict(ldu=63), INVALID), (dict(up=A + 1), INVALID), (dict(dtype=5), UNSUPPORTED),
    (dict(rows=0, up=None), OK)])
def test_silu_gate_refuses(change, want):
    assert call("dnns_silu_gate_quantize", GATE, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(dy=None), INVALID), (dict(h=None), INVALID), (dict(dx=None), INVALID), (dict(lddy=63), INVALID), (dict(ldh=63), INVALID),
    (dict(lddx=63), INVALID), (dict(dh=A, lddh=63), INVALID), (dict(eps=0.0), INVALID), (dict(dweight=A), INVALID),
    (dict(dweight=A, ws=A + 8, ws_bytes=1 << 20), INVALID), (dict(dweight=A + 1, ws=A, ws_bytes=1 << 20), INVALID),
    (dict(dweight=A, ws=A, ws_bytes=16), WORKSPACE), (dict(dtype=2), UNSUPPORTED), (dict(rows=-1), INVALID),
    (dict(lddx=1 << 60), UNSUPPORTED), (dict(cols=0), OK), (dict(rows=0), OK)])
def test_rmsnorm_backward_refuses(change, want):
    assert call("dnns_rmsnorm_backward", NORM_BACK, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(dy=None), INVALID), (dict(gate=None), INVALID), (dict(up=None), INVALID), (dict(dgate=None), INVALID), (dict(dup=None), INVALID),
    (dict(ldg=63), INVALID), (dict(lddu=63), INVALID), (dict(dup=A + 1), INVALID), (dict(dtype=9), UNSUPPORTED), (dict(cols=1 << 31), UNSUPPORTED),
    (dict(rows=0), OK), (dict(cols=0), OK)])
def test_silu_gate_backward_refuses(change, want):
    assert call("dnns_silu_gate_backward", GATE_BACK, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(xq=None), INVALID), (dict(wq=None), INVALID), (dict(xs=None), INVALID), (dict(ws=None), INVALID), (dict(y=None), INVALID),
    (dict(status=None), INVALID), (dict(status=A + 2), INVALID), (dict(xq=A + 8), INVALID), (dict(wq=A + 4), INVALID), (dict(ldx=72), INVALID),
    (dict(ldw=48), INVALID), (dict(ldy=7), INVALID), (dict(y=A + 1), INVALID), (dict(bias=A + 2), INVALID), (dict(rows=-1), INVALID),
    (dict(k=-1), INVALID), (dict(n=-1), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(k=131072, ldx=131072, ldw=131072), UNSUPPORTED),
    (dict(rows=1 << 31), UNSUPPORTED), (dict(n=1 << 31, ldy=1 << 31), UNSUPPORTED), (dict(ldy=1 << 60), UNSUPPORTED), (dict(ldx=1 << 60), UNSUPPORTED),
    (dict(rows=0), OK), (dict(n=0), OK)])
def test_linear_refuses(change, want):
    assert call("dnns_linear_quantized", LINEAR, **change) == want


def test_sizes():
    assert [B.dnns_quantized_row_bytes(c) for c in (0, 1, 16, 17, 4099)] == [0, 16, 16, 32, 4112]
    assert B.dnns_rmsnorm_backward_workspace_bytes(0, 64) == 0 == B.dnns_rmsnorm_backward_workspace_bytes(4, 0)
    assert B.dnns_rmsnorm_backward_workspace_bytes(-1, 64) == 0
    a, b = B.dnns_rmsnorm_backward_workspace_bytes(4, 64), B.dnns_rmsnorm_backward_workspace_bytes(1 << 20, 64)
    assert 64 * 4 <= a < b <= 1 << 20                          # at least one slice of partial sums
    assert B.DNNS_LINEAR_MAX_IN * 128 * 128 < 2 ** 31          # what an int32 sum holds


def test_native_calls_refuse_what_is_not_on_the_device():
    """The calls from torch tensors check them before they enter the library."""
    import torch

    from paper_2309_06973_b200 import runtime as R
    rows = R._native.rows(A, 16, A, 0, 0, 2, 3, 0)
    x = torch.zeros(2, 3)
    for call in (lambda: R._native.quantize_rows(x, rows), lambda: R._native.rmsnorm(x, None, 1e-5, rows, None, None),
                 lambda: R._native.silu_gate(x, x, rows), lambda: R._native.rmsnorm_backward(x, x, None, 1e-5, x, None, None, None),
                 lambda: R._native.silu_gate_backward(x, x, x, x, x), lambda: R._native.linear(rows, R._native.rows(A, 16, A, 0, 0, 3, 3, 0), None, x, A),
                 lambda: R._native.quantize_rows(x.t(), rows), lambda: R._native.quantize_rows(x.half(), rows),
                 lambda: R._native.quantize_rows("x", rows), lambda: R._native.quantize_rows(x, x), lambda: R.RowsQ8.of(x.to(torch.int8), x[:, 0], 3)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: R._native.quantize_rows(x), lambda: R._native.rows(1, 2), lambda: R._native.bind(1)):
        with pytest.raises(TypeError):
            call()
