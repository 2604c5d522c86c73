"""Weights that change after a layer was made of them: the layer computes with what its rows hold now, wherever rows start.

Every comparison is with a layer made anew of a copy of the rows: the sums are exact, so the bits are equal."""
import pytest
import torch

from paper_2309_06973_b200 import binding as B
from paper_2309_06973_b200 import runtime as R

pytestmark = pytest.mark.gpu

N, K = 300, 5003
TOKENS = [1, 20, 300]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def matrix(seed, rows=N, cols=K):
    return torch.randn(rows, cols, generator=gen(seed), device="cuda") * (1 + seed)


def weights(distance, seed=1):
    """Rows in 8 bits at a distance of 5008 (laid out anew by the layer) or 5120 (used where they are)."""
    q, scale = torch.zeros(N, distance, dtype=torch.int8, device="cuda"), torch.empty(N, device="cuda")
    rows = R.RowsQ8.of(q, scale, K, torch.empty(N, K, dtype=torch.bfloat16, device="cuda"))
    return q, scale, R.quantize_rows(matrix(seed), rows)


def tokens_of(count):
    return R.quantize_rows(matrix(0, count), R.RowsQ8(count, K))


def anew(x, rows):
    return R.LinearQ8(R.RowsQ8.of(rows.q.clone(), rows.scale.clone(), K))(x, torch.empty(x.rows, N, device="cuda"))


def write(how, q, scale, rows, seed):
    """New weights into the rows, in the ways a program has."""
    if how == "call":
        R.quantize_rows(matrix(seed), rows)
    elif how == "other rows":                                          # a second and third view of the same tensors
        for part in (slice(0, 100), slice(100, None)):
            R.quantize_rows(matrix(seed)[part], R.RowsQ8.of(q[part], scale[part], K))
    elif how == "scales":
        scale.mul_(1.5)
    else:
        new = R.quantize_rows(matrix(seed), R.RowsQ8(N, K))
        q[:, :K], scale[:] = new.q[:, :K], new.scale


@pytest.mark.parametrize("how", ["call", "other rows", "scales", "torch"])
@pytest.mark.parametrize("distance", [5008, 5120])
@pytest.mark.parametrize("count", TOKENS)
def test_layer_follows_its_rows(count, distance, how):
    q, scale, rows = weights(distance)
    x, y = tokens_of(count), torch.empty(count, N, device="cuda")
    layer = R.LinearQ8(rows)
    assert torch.equal(layer(x, y), anew(x, rows))
    for seed in (2, 3):
        before = y.clone()
        write(how, q, scale, rows, seed)
        assert torch.equal(layer(x, y), anew(x, rows)) and not torch.equal(y, before)
        assert torch.equal(layer.weight.q[:, :K], q[:, :K]) and torch.equal(layer.weight.scale, scale)
    assert layer.device_status() == B.DNNS_OK


@pytest.mark.parametrize("distance", [5008, 5120])
@pytest.mark.parametrize("count", TOKENS)
def test_captured_calls_follow_the_rows(count, distance):
    """A graph of the product sees weights quantised after its capture; one that quantises them does both in each replay."""
    _, _, rows = weights(distance)
    x, y, w = tokens_of(count), torch.empty(count, N, device="cuda"), matrix(1)
    layer, other = R.LinearQ8(rows), R.LinearQ8(rows)
    layer(x, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        product, both = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(product, stream=side):
            layer(x, y)
        R.quantize_rows(matrix(2), rows)
        product.replay()
        want = anew(x, rows)
        side.synchronize()
        assert torch.equal(y, want)
        with torch.cuda.graph(both, stream=side):
            R.quantize_rows(w, rows)
            layer(x, y)
        for seed in (3, 4):
            w.copy_(matrix(seed))
            both.replay()
            want = anew(x, rows)
            side.synchronize()
            assert torch.equal(y, want)
            assert torch.equal(other(x, torch.empty_like(y)), want)    # another layer of the same rows


@pytest.mark.parametrize("distance", [5008, 5120])
def test_rows_of_an_inference_program(distance):
    """Tensors made under inference_mode count no versions: the module's own writes are followed all the same."""
    with torch.inference_mode():
        _, _, rows = weights(distance)
        x, y = tokens_of(20), torch.empty(20, N, device="cuda")
        layer = R.LinearQ8(rows)
        layer(x, y)
        R.quantize_rows(matrix(2), rows)
        assert torch.equal(layer(x, y), anew(x, rows))
    R.quantize_rows(matrix(3), rows)
    assert torch.equal(layer(x, y), anew(x, rows)) and layer.device_status() == B.DNNS_OK


@pytest.mark.parametrize("distance", [5008, 5120])
def test_layer_outlives_the_rows_it_was_made_of(distance):
    q, scale, rows = weights(distance)
    x, y = tokens_of(20), torch.empty(20, N, device="cuda")
    want, layer = anew(x, rows), R.LinearQ8(rows)
    del q, scale, rows
    rubbish = [torch.full((N, 5120), 77, dtype=torch.int8, device="cuda") for _ in range(4)]
    assert torch.equal(layer(x, y), want) and len(rubbish) == 4
