"""A language model's feed-forward block, pruned and run in 8 bits.

    python examples/gated_block_q8.py [width] [hidden]

The block h = x + residual, y = down(silu(gate(n)) * up(n)) with n = norm(h) goes through the pruning path (threshold, zero
structures, keep sets, rebuild); the rebuilt matrices, which kept an arbitrary number of hidden units, are quantised per output
channel where they lie, and the block runs in 8 bits: norm, one product for gate and up, gated activation, product.
`gradients` is the step that fine-tunes it with the rounding in the loop.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2309_06973_b200 import binding as B                      # noqa: E402
from paper_2309_06973_b200 import runtime as R                      # noqa: E402
from paper_2309_06973_b200 import workloads as W                    # noqa: E402

EPS = 1e-6


def prune(wl, dtype=B.DNNS_F32):
    """The rebuilt matrices of the workload's first variant, as device tensors in the session's arena (kept by the caller)."""
    ses = R.Session(R.DeviceModel(wl, dtype), wl.scope, len(wl.ks), want_mask_bits=False, want_nz_map=False, portfolio_slots=1)
    ses.magnitude_threshold(wl.ks)
    ses.zero_structures_portfolio(0, 1)
    ses.propagate_keep_portfolio(1)
    ses.compact_portfolio(0, 0)
    assert ses.device_status() == B.DNNS_OK
    offsets, shapes = ses.dst_offsets.tolist(), ses.dst_shapes.tolist()
    kind = torch.float32 if dtype == B.DNNS_F32 else torch.bfloat16
    size = 4 if dtype == B.DNNS_F32 else 2
    out = []
    for i in range(len(wl.tensors)):
        o, n = shapes[2 * i], shapes[2 * i + 1]
        out.append(ses.compact_arena[offsets[i]: offsets[i] + o * n * size].view(kind).reshape(o, n))
    return ses, out


class GatedBlockQ8:
    """The block with its matrices in 8 bits; buffers for up to max_tokens tokens."""

    def __init__(self, gate, up, down, norm_weight, max_tokens):
        self.hidden, self.width = gate.shape
        both = R.RowsQ8(2 * self.hidden, self.width, values=True)
        for half, w in ((slice(0, self.hidden), gate), (slice(self.hidden, None), up)):
            R.quantize_rows(w, R.RowsQ8.of(both.q[half], both.scale[half], self.width, both.values[half]))
        self.gate_up = R.LinearQ8(both)
        self.down = R.LinearQ8(R.quantize_rows(down, R.RowsQ8(self.width, self.hidden, values=True)))
        self.norm_weight, self.max_tokens = norm_weight, max_tokens
        self.n, self.a = R.RowsQ8(max_tokens, self.width, values=True), R.RowsQ8(max_tokens, self.hidden, values=True)
        new = lambda cols: torch.empty(max_tokens, cols, dtype=torch.bfloat16, device="cuda:0")
        self.gu, self.y = new(2 * self.hidden), new(self.width)

    def _rows(self, r, tokens):
        return r if tokens == r.rows else R.RowsQ8.of(r.q[:tokens], r.scale[:tokens], r.cols, r.values[:tokens])

    def __call__(self, x, residual):
        """y for x (tokens, width) in bf16; the residual stream is updated in place."""
        tokens = x.shape[0]
        n, a, gu, y = self._rows(self.n, tokens), self._rows(self.a, tokens), self.gu[:tokens], self.y[:tokens]
        R.rmsnorm_q8(x, self.norm_weight, EPS, n, residual=residual, h=residual)
        self.gate_up(n, gu)
        R.silu_gate_q8(gu[:, : self.hidden], gu[:, self.hidden:], a)
        return self.down(a, y)

    def gradients(self, dy, h, dh):
        """For the latest call: (gradient that reaches x and the residual, of the norm's weight, of [gate; up], of down),
        roundings passed straight through.  dy: gradient of y, dh: gradient that reaches the residual stream past the block.
        The products are ordinary ones of what the 8-bit rows stand for."""
        tokens = dy.shape[0]
        gu, n, a = self.gu[:tokens], self.n.values[:tokens], self.a.values[:tokens]
        da, dgu = dy @ self.down.weight.values, torch.empty_like(gu)
        R.silu_gate_q8_backward(da, gu[:, : self.hidden], gu[:, self.hidden:], dgu[:, : self.hidden], dgu[:, self.hidden:])
        dn = dgu @ self.gate_up.weight.values
        dx, dw = torch.empty_like(h), torch.empty_like(self.norm_weight)
        R.rmsnorm_q8_backward(dn, h, self.norm_weight, EPS, dx, dw, dh=dh,
                              workspace=R.rmsnorm_q8_backward_workspace(tokens, self.width))
        return dx, dw, dgu.t() @ n, dy.t() @ a

    def device_status(self):
        return self.gate_up.device_status() or self.down.device_status()


def exact(gate, up, down, norm_weight, x, residual):
    """The same block in 64 bits, nothing rounded but its inputs."""
    h = x.double() + residual.double()
    n = h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * norm_weight.double()
    g, u = n @ gate.double().t(), n @ up.double().t()
    return (g / (1 + torch.exp(-g)) * u) @ down.double().t()


def main():
    width, hidden = (int(v) for v in (sys.argv[1:3] or ("2048", "8192")))
    wl = W.gated_block(width, hidden, seed=1)
    ses, (gate, up, down) = prune(wl)
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    norm_weight = 1 + 0.1 * rnd(width)
    block = GatedBlockQ8(gate, up, down, norm_weight, 2048)
    print(f"{wl.name}: {hidden} -> {gate.shape[0]} hidden units, {wl.n_prunable} -> {gate.numel() + up.numel() + down.numel()} weights")
    for tokens in (1, 16, 2048):
        x, residual = rnd(tokens, width).bfloat16(), (2 * rnd(tokens, width)).bfloat16()
        want = exact(gate, up, down, norm_weight, x, residual)
        y = block(x, residual.clone())
        off = float((y.double() - want).norm() / want.norm())
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                block(x, residual)
            graph.replay()
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record(stream)
            for _ in range(100):
                graph.replay()
            end.record(stream)
            stream.synchronize()
        print(f"{tokens:5d} tokens: {start.elapsed_time(end) * 10:8.1f} us, off the 64-bit block by {off:.4f} (2-norm)")
    assert block.device_status() == B.DNNS_OK
    ses.close()


if __name__ == "__main__":
    main()
