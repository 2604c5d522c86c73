"""The operators on rows in 8 bits together, as examples/gated_block_q8.py uses them: a feed-forward block through the pruning
path, its rebuilt matrices quantised where they lie, run and differentiated."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import oracle as O
from paper_2309_06973_b200 import binding as B
from paper_2309_06973_b200 import workloads as W
import q8_ref as P

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def block_of(dtype, width=192, hidden=700, seed=3, tokens=40):
    import gated_block_q8 as E
    wl = W.gated_block(width, hidden, seed)
    ses, mats = E.prune(wl, dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    norm_weight = 1 + 0.1 * torch.randn(width, generator=g, device="cuda")
    x = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    res = (2 * torch.randn(tokens, width, generator=g, device="cuda")).bfloat16()
    return E, wl, ses, mats, norm_weight, x, res, g


def product_close(y, want):
    """A product of rows in 8 bits, stored in bf16: the exact sum rounded to fp32 and scaled twice, then to bf16."""
    tol = 4 * P.U32 * want.abs()
    assert torch.all((y.double() - want).abs() <= tol + P.UBF * (want.abs() + tol))


@pytest.mark.parametrize("dtype", [B.DNNS_F32, B.DNNS_BF16])
def test_rebuilt_block_matches_the_oracle_and_runs_in_8_bits(dtype):
    E, wl, ses, mats, norm_weight, x, res, _ = block_of(dtype)
    om = O.OracleModel(wl, dtype)
    rec = O.threshold(om, wl.scope, wl.ks)
    masked, _ = O.apply_mask(om, wl.scope, rec[0])
    _, out_nz, in_nz = O.zero_structures(masked)
    _, ki, kc, _ = O.propagate_keep(masked, out_nz, in_nz)
    want, *_ = O.compact(masked, ki, kc)
    assert 0 < mats[0].shape[0] < 700                                  # some hidden units went, some stayed
    for got, w in zip(mats, want):
        bits = got.contiguous().view(torch.int32 if dtype == B.DNNS_F32 else torch.int16).cpu().numpy()
        assert np.array_equal(bits.ravel(), np.ascontiguousarray(w).view(bits.dtype).ravel())
    block = E.GatedBlockQ8(*mats, norm_weight, x.shape[0])
    def product(t, w):                    # the sum of whole numbers exact, scaled in 64 bits
        return (t.q[:, : t.cols].double() @ w.q[:, : w.cols].double().t()) * t.scale.double()[:, None] * w.scale.double()[None, :]

    for tokens in (1, 5, x.shape[0]):
        r = res[:tokens].clone()
        y = block(x[:tokens].contiguous(), r)
        h = x[:tokens].float() + res[:tokens].float()
        assert torch.equal(r, h.bfloat16())
        # every step against 64 bits on what the step before it left, with that step's own tolerance
        n, a = block._rows(block.n, tokens), block._rows(block.a, tokens)
        P.check_rows(n, P.norm_of(h.double(), norm_weight.double(), E.EPS))
        gu = block.gu[:tokens]
        product_close(gu, product(n, block.gate_up.weight))
        P.check_rows(a, P.silu_gate(gu[:, : block.hidden].double(), gu[:, block.hidden:].double()))
        product_close(y, product(a, block.down.weight))
    assert block.device_status() == B.DNNS_OK
    ses.close()


def test_gradients_against_autograd():
    """The fine-tuning step against torch's gradients of the same block in 64 bits, roundings taken as constants added."""
    E, _, ses, mats, norm_weight, x, res, g = block_of(B.DNNS_F32)
    block = E.GatedBlockQ8(*mats, norm_weight, x.shape[0])
    h = res.clone()
    block(x, h)
    dy = torch.randn(*x.shape, generator=g, device="cuda").bfloat16()
    dh = torch.randn(*x.shape, generator=g, device="cuda").bfloat16()
    dx, dw, dgu, ddown = block.gradients(dy, h, dh)
    hid = block.hidden
    hd, wd = h.double().requires_grad_(), norm_weight.double().requires_grad_()
    gu_w = block.gate_up.weight.values.double().requires_grad_()
    down_w = block.down.weight.values.double().requires_grad_()
    n = hd / torch.sqrt((hd * hd).mean(1, keepdim=True) + E.EPS) * wd
    n = n + (block.n.values.double() - n).detach()                      # the rounding, passed straight through
    gu = n @ gu_w.t()
    gu = gu + (block.gu.double() - gu).detach()
    a = gu[:, :hid] * torch.sigmoid(gu[:, :hid]) * gu[:, hid:]
    a = a + (block.a.values.double() - a).detach()
    loss = ((a @ down_w.t()) * dy.double()).sum() + (hd * dh.double()).sum()
    loss.backward()
    # intermediate gradients are stored in bf16: three roundings of 2^-8 on the way to dx and dw, two to the weights'
    for got, want, roundings in ((dx, hd.grad, 4), (dw, wd.grad, 3), (dgu, gu_w.grad, 3), (ddown, down_w.grad, 1)):
        assert (got.double() - want).norm() <= roundings * 2.0 ** -8 * want.norm()
    ses.close()
