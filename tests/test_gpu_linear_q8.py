"""The product of rows in 8 bits on the GPU against the exact sum.

Tolerance: the int32 sum is exact, its conversion to fp32, the product with the channel's scale and the fused step with
the token's scale and the bias round once each: 3 half units of the scaled sum, 1 of the result, and one rounding to the
output's type.  With scales that are powers of two, no bias and sums below 2^24 nothing rounds: fp32 results are equal."""
import pytest
import torch

from paper_2309_06973_b200 import binding as B
from paper_2309_06973_b200 import runtime as R
import q8_ref as P

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows8(rows, cols, seed, extra=0, scale=None, extreme=False):
    """Rows in 8 bits whose padding holds other bytes than 0: they must not count."""
    g = gen(seed)
    ld = (cols + 15) // 16 * 16 + extra
    q = torch.randint(-127, 128, (rows, ld), generator=g, device="cuda", dtype=torch.int8)
    if extreme:
        q = torch.where(torch.rand(rows, ld, generator=g, device="cuda") < 0.5, 127, -127).to(torch.int8)
        q[0] = 127
    s = torch.rand(rows, generator=g, device="cuda") * 0.02 + 1e-3 if scale is None else torch.full((rows,), scale, device="cuda")
    return R.RowsQ8.of(q, s, cols)


def product(x, w, bias):
    acc = x.q[:, : x.cols].double() @ w.q[:, : w.cols].double().t()   # every partial sum below 2^53: exact
    y = acc * x.scale.double()[:, None] * w.scale.double()[None, :]
    return y, y if bias is None else y + bias.double()


def check(rows, k, n, dtype, bias=False, extra=0, ldy=None, lead=0, seed=0, extreme=False):
    x, w = rows8(rows, k, seed + 1, extra, extreme=extreme), rows8(n, k, seed + 2, extra, extreme=extreme)
    b = torch.randn(n, generator=gen(seed + 3), device="cuda") if bias else None
    layer, y = R.LinearQ8(w, b), P.Guarded(rows, n, dtype, ld=ldy, lead=lead)
    layer(x, y.view)
    part, want = product(x, w, b)
    u = P.U32 if dtype is F32 else P.UBF
    tol = 3 * P.U32 * part.abs() + P.U32 * want.abs()
    assert torch.all((y.view.double() - want).abs() <= tol + u * (want.abs() + tol))
    assert layer.device_status() == B.DNNS_OK and y.intact()


# one token, small batches, around every tile edge, odd everything
ROWS = [1, 2, 3, 5, 8, 9, 16, 17, 31, 33, 64, 65, 100, 127, 128, 129, 200, 256, 257, 333, 513]


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("k,n", [(1, 1), (16, 8), (100, 37), (129, 300), (513, 127), (1000, 513), (4096, 257)])
def test_rows_and_odd_widths(rows, k, n):
    check(rows, k, n, F32, seed=rows)
    check(rows, k, n, BF16, bias=True, seed=rows + 50)


@pytest.mark.parametrize("k", [1, 15, 16, 17, 31, 32, 33, 63, 64, 127, 128, 129, 255, 256, 257, 511, 640, 1023, 1025])
@pytest.mark.parametrize("rows", [1, 6, 40, 150, 300])
def test_every_end_of_a_row(k, rows):
    check(rows, k, 260, F32, bias=True, extra=16, seed=k)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 127, 128, 129, 255, 256, 257, 1000, 4097])
@pytest.mark.parametrize("rows", [1, 7, 70, 260])
def test_every_number_of_channels(n, rows):
    check(rows, 200, n, BF16, seed=n)
    check(rows, 300, n, F32, bias=True, ldy=n + 5, lead=1, seed=n)     # rows of y apart and off 16 bytes


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,k,n", [(1, 4096, 4096), (4, 11003, 2741), (24, 4096, 14336), (333, 5003, 2741), (1024, 4096, 1024),
                                      (2048, 1024, 4096), (4096, 512, 6000), (700, 14336, 4096), (1100, 131071, 300), (3, 131071, 200)])
def test_layers(rows, k, n, dtype):
    check(rows, k, n, dtype, bias=True, seed=rows)


@pytest.mark.parametrize("rows", [1, 20, 128, 600])
def test_largest_sums(rows):
    """Every product +-127 * 127 over the longest row: the sum passes 2^30."""
    check(rows, 131071, 130, F32, seed=rows, extreme=True)


@pytest.mark.parametrize("rows", [1, 4, 9, 33, 130, 513])
def test_exact_results(rows):
    x, w = rows8(rows, 1000, 1, scale=0.5), rows8(300, 1000, 2, scale=0.25)
    y = torch.empty(rows, 300, device="cuda")
    R.LinearQ8(w)(x, y)
    assert torch.equal(y.double(), product(x, w, None)[0])


@pytest.mark.parametrize("rows", [1, 6, 40, 300])
def test_nan_scales_stay_in_their_row_and_zero_rows_give_the_bias(rows):
    x, w = rows8(rows, 260, 1), rows8(290, 260, 2)
    bias = torch.randn(290, generator=gen(1), device="cuda")
    x.scale[rows - 1] = float("nan")
    x.q[rows - 1].zero_()
    w.scale[7] = float("nan")
    y = torch.empty(rows, 290, device="cuda")
    R.LinearQ8(w, bias)(x, y)
    assert torch.isnan(y[rows - 1]).all() and torch.isnan(y[:, 7]).all()
    assert rows == 1 or int(torch.isnan(y).sum()) == 290 + (rows - 1)
    x.scale[rows - 1] = 0.0
    w.scale[7] = 1.0
    R.LinearQ8(w, bias)(x, y)
    assert torch.equal(y[rows - 1], bias)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_rows_channels_or_columns(dtype):
    b = torch.randn(7, generator=gen(1), device="cuda")
    for rows in (1, 5, 300):
        y = torch.full((rows, 7), 5.0, dtype=dtype, device="cuda")
        R.LinearQ8(rows8(7, 0, 1), b)(rows8(rows, 0, 2), y)
        assert torch.equal(y, b.to(dtype).expand(rows, 7))
        R.LinearQ8(rows8(7, 0, 1))(rows8(rows, 0, 2), y)
        assert not y.any()
    R.LinearQ8(rows8(7, 64, 1), b)(rows8(0, 64, 2), torch.empty(0, 7, dtype=dtype, device="cuda"))
    R.LinearQ8(rows8(0, 64, 1))(rows8(5, 64, 2), torch.empty(5, 0, dtype=dtype, device="cuda"))


@pytest.mark.parametrize("rows", [1, 24, 300, 2000])
def test_repeated_calls_streams_and_graphs(rows):
    """The same call again and again, on another stream and replayed from a graph gives the same bits."""
    x, w = rows8(rows, 3000, 5), rows8(1500, 3000, 6)
    layer, y = R.LinearQ8(w), torch.empty(rows, 1500, dtype=BF16, device="cuda")
    layer(x, y)
    first = y.clone()
    for _ in range(20):
        y.zero_()
        layer(x, y)
        assert torch.equal(y, first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y.zero_()
        layer(x, y)
        side.synchronize()
        assert torch.equal(y, first)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer(x, y)
        for _ in range(3):
            y.zero_()
            graph.replay()
        side.synchronize()
    assert torch.equal(y, first) and layer.device_status() == B.DNNS_OK


@pytest.mark.parametrize("tokens", [1, 8, 40, 300])
def test_chains_of_calls_see_each_others_results(tokens):
    """Norm -> product -> gated activation -> product over the same buffers, call after call without waiting, from a stream
    and from a graph: each link begins before the one in front of it has ended, and must still read what that one wrote."""
    width, hidden, rounds = 1040, 700, 40
    g = gen(tokens)
    gate_up, down = R.LinearQ8(rows8(2 * hidden, width, 1)), R.LinearQ8(rows8(width, hidden, 2))
    n, a = R.RowsQ8(tokens, width), R.RowsQ8(tokens, hidden)
    gu, h = torch.empty(tokens, 2 * hidden, dtype=BF16, device="cuda"), torch.empty(tokens, width, dtype=BF16, device="cuda")
    xs = torch.randn(rounds, tokens, width, generator=g, device="cuda").to(BF16)

    def step(x, y, wait=lambda: None):
        for call in (lambda: R.rmsnorm_q8(x, None, 1e-6, n, residual=x, h=h), lambda: gate_up(n, gu),
                     lambda: R.silu_gate_q8(gu[:, :hidden], gu[:, hidden:], a), lambda: down(a, y)):
            call()
            wait()

    want, got = torch.empty_like(xs), torch.zeros_like(xs)
    for x, y in zip(xs, want):
        step(x, y, torch.cuda.synchronize)
    for _ in range(3):
        for x, y in zip(xs, got):
            step(x, y)
        assert torch.equal(got, want)
        got.zero_()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for x, y in zip(xs, got):
                step(x, y)
        for _ in range(3):
            got.zero_()
            graph.replay()
        side.synchronize()
    assert torch.equal(got, want) and gate_up.device_status() == B.DNNS_OK == down.device_status()


def test_fork_and_join_in_a_capture():
    """Two branches of a captured graph with the calls in both, then one that needs both."""
    x, w = rows8(64, 1000, 1), rows8(500, 1000, 2)
    ys = [torch.empty(64, 500, dtype=BF16, device="cuda") for _ in range(2)]
    layers, out = [R.LinearQ8(w) for _ in range(2)], R.RowsQ8(64, 500, values=True)
    main, side = torch.cuda.Stream(), torch.cuda.Stream()

    def both():
        layers[0](x, ys[0])
        side.wait_stream(main)
        layers[0](x, ys[0])
        with torch.cuda.stream(side):
            layers[1](x, ys[1])
        main.wait_stream(side)
        R.silu_gate_q8(ys[0], ys[1], out)

    with torch.cuda.stream(main):
        both()
        main.synchronize()
        want = out.q.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=main):
            both()
        for _ in range(20):
            ys[0].zero_(), ys[1].zero_(), out.q.zero_()
            graph.replay()
            main.synchronize()
            assert torch.equal(out.q[:, :500], want[:, :500])


def test_offsets_past_32_bits():
    """Output rows so far apart that the last ones start past 2^32 elements."""
    ld, rows, n = (1 << 30) + 3, 5, 40
    buf = torch.empty(4 * ld + 64, dtype=BF16, device="cuda")
    y = buf.as_strided((rows, n), (ld, 1), 0)
    x, w = rows8(rows, 70, 1), rows8(n, 70, 2)
    R.LinearQ8(w)(x, y)
    near = torch.empty(rows, n, dtype=BF16, device="cuda")
    R.LinearQ8(w)(x, near)
    assert torch.equal(y, near)


def test_runtime_refuses_wrong_tensors():
    x, w = rows8(4, 64, 1), rows8(8, 64, 2)
    layer = R.LinearQ8(w)
    good = torch.empty(4, 8, device="cuda")
    for bad in (good[:3], good.t(), good.half(), good.cpu(), torch.empty(4, 9, device="cuda")):
        with pytest.raises(ValueError):
            layer(x, bad)
    with pytest.raises(ValueError):
        layer(rows8(4, 65, 1), good)
    with pytest.raises(ValueError):
        R.LinearQ8(w, torch.zeros(7, device="cuda"))
    with pytest.raises(B.DnnsError):                                    # rows that do not start on 16 bytes
        layer(R.RowsQ8.of(torch.zeros(4, 72, dtype=torch.int8, device="cuda"), x.scale, 64), good)
    with pytest.raises(B.DnnsError):
        R.LinearQ8(rows8(3, 131072, 1))(rows8(2, 131072, 2), torch.empty(2, 3, device="cuda"))
