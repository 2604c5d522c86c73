"""Plain 64-bit forms of the operators on rows in 8 bits, and guarded device buffers (used by the GPU tests)."""
import torch

U32, UBF = 2.0 ** -24, 2.0 ** -8          # unit roundoff of fp32 (24 significant bits) and bf16 (8): half a last place at 1
# Largest relative error of a row's factor: a sum of non-negative squares over a chain of at most 32 terms a thread, ten
# shuffle steps and a few single operations (half of it after the square root), and one product, one division.
ROW_EPS = 64 * U32
GUARD, PATTERN = 64, 0x5A


def rows_of(y):
    """(q before rounding, scale) of the rows of y in 64 bits."""
    top = y.abs().amax(1)
    scale = top / 127
    return torch.where(top[:, None] > 0, y / torch.where(top > 0, scale, 1.0)[:, None], torch.zeros_like(y)), scale


def norm_of(h, w, eps):
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h * r if w is None else h * r * w


def silu_gate(g, u):
    return g / (1 + torch.exp(-g)) * u


def check_rows(out, y, eps=ROW_EPS):
    """out (RowsQ8) against the rows of y (64 bits, finite)."""
    want, scale = rows_of(y)
    got_s, q = out.scale.double(), out.q[:, : out.cols].double()
    assert torch.all((got_s - scale).abs() <= eps * scale), "scale"
    assert torch.all((q - want).abs() <= 0.5 + 127 * 2 * eps), "q"
    assert int(out.q[:, : out.cols].abs().max() if q.numel() else 0) <= 127
    if out.values is not None:
        again = (out.q[:, : out.cols].float() * out.scale[:, None]).to(torch.bfloat16)
        assert torch.equal(out.values, again), "values"


class Guarded:
    """A rows x cols matrix inside a larger buffer: `lead` elements in front, rows `ld` apart, all else a pattern."""

    def __init__(self, rows, cols, dtype, ld=None, lead=0, source=None):
        size = torch.empty(0, dtype=dtype).element_size()
        self.ld = cols if ld is None else ld
        n = lead + max(rows, 1) * self.ld + GUARD
        self.raw = torch.full(((n + GUARD) * size,), PATTERN, dtype=torch.uint8, device="cuda")
        flat = self.raw.view(dtype)
        self.at = GUARD + lead
        self.view = flat.as_strided((rows, cols), (self.ld, 1), self.at)
        if source is not None:
            self.view.copy_(source)
        self.mask = torch.ones(flat.numel(), dtype=torch.bool, device="cuda")
        self.mask.as_strided((rows, cols), (self.ld, 1), self.at).fill_(False)
        self.size = size

    def intact(self):
        b = self.raw.view(-1, self.size)[self.mask]
        return bool((b == PATTERN).all())
