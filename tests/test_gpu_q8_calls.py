"""What the calls on rows in 8 bits promise beside their results."""
import pytest
import torch

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
