"""FeedForwardBlock behind a RAF layer: norm, products, update and 8-bit inference as a program runs them together.

The reference is the block's formula in 64 bits on the same layer output.  fp32: every stage's relative error is below 1e-5 (products
of up to 128 terms: 300 u of sum |a||b|, u = 2^-24, which is at most 10 times a result's typical size), and five stages
follow one another: 1e-4 of the result's norm.  bf16: ten roundings of 2^-8 at most between input and output, 2^-8 * sqrt(10) = 1.2e-2
of the norm where they are independent; 8-bit rows add 2^-4 of every factor of the first product, which averages out over its terms and
passes the residual by: 5e-2.
"""
import math

import pytest
import torch

import paper_2408_09697_amd as heta

pytestmark = pytest.mark.gpu


def act(x):
    return x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))


def formula(x, agg, W1, W2, gamma, b1, b2, eps=1e-6):
    h = x + agg
    n = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * gamma
    return h + act(n @ W1 + b1) @ W2 + b2


def parameters(d, hidden, dtype):
    g = torch.Generator(device="cuda").manual_seed(4)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return (r(d, hidden) * d ** -0.5).to(dtype), (r(hidden, d) * hidden ** -0.5).to(dtype), 1 + 0.1 * r(d), 0.1 * r(hidden), 0.1 * r(d)


def rel(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


@pytest.fixture(scope="module")
def layer():
    """A graph of two node types and the layer's output for one of them, 32 columns."""
    g = torch.Generator().manual_seed(1)
    n_dst, n_src, edges = 700, 500, 4000
    dst = torch.sort(torch.randint(n_dst, (edges,), generator=g)).values
    rowptr = torch.searchsorted(dst, torch.arange(n_dst + 1)).numpy()
    col = torch.randint(n_src, (edges,), generator=g, dtype=torch.int32).numpy()
    graph = heta.heta_graph_create([(n_src, 48, 0), (n_dst, 32, 0)], [(0, 1, rowptr, col)])
    tables = [torch.randn(n_src, 48, generator=g).cuda(), torch.randn(n_dst, 32, generator=g).cuda()]
    raf = heta.RafLayer(graph, heta.HETA_MEAN, tables, [torch.randn(48, 32, generator=g).cuda() * 0.15], 32)
    yield graph, raf, tables
    graph.destroy()


@pytest.mark.parametrize("dtype,most", [(torch.float32, 1e-4), (torch.bfloat16, 1.2e-2)])
def test_block_behind_a_layer(layer, dtype, most):
    graph, raf, tables = layer
    agg = raf.forward()[1].to(dtype)
    x = tables[1].to(dtype)
    W1, W2, gamma, b1, b2 = parameters(32, 128, dtype)
    block = heta.FeedForwardBlock(graph, W1, W2, gamma, b1, b2)
    out = block.forward(x, agg)
    leaves = [t.double().requires_grad_(True) for t in (x, W1, W2, gamma, b1, b2)]
    ref = formula(leaves[0], agg.double(), *leaves[1:])
    assert rel(out, ref.detach()) <= most
    assert rel(block.infer(x, agg), ref.detach()) <= most
    go = torch.randn(out.shape, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda").to(dtype)
    ref.backward(go.double())
    gx = block.backward(go)
    assert rel(gx, leaves[0].grad) <= most
    for name, leaf in zip(("W1", "W2", "gamma", "b1", "b2"), leaves[1:]):
        assert rel(block.grads[name], leaf.grad) <= most, name
    if dtype is torch.float32:  # the gradient that the layer's own backward pass takes
        raf.backward({1: gx})


def test_updates_lower_a_loss(layer):
    graph, raf, tables = layer
    agg, x = raf.forward()[1].clone(), tables[1]
    block = heta.FeedForwardBlock(graph, *parameters(32, 128, torch.float32))
    want = torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda")
    losses = []
    for _ in range(30):
        off = block.forward(x, agg) - want
        losses.append(float(off.square().mean()))
        block.backward(off * (2.0 / off.numel()))
        block.update(lr=0.02, weight_decay=0.01)
    assert losses[-1] < 0.8 * losses[0]


def test_eight_bit_inference(layer):
    graph, raf, tables = layer
    agg, x = raf.forward()[1].bfloat16(), tables[1].bfloat16()
    W1, W2, gamma, b1, b2 = parameters(32, 128, torch.bfloat16)
    block = heta.FeedForwardBlock(graph, W1, W2, gamma, b1, b2)
    ref = formula(x.double(), agg.double(), W1.double(), W2.double(), gamma.double(), b1.double(), b2.double())
    for coarse in (False, True):
        assert rel(block.infer(x, agg, block.pack(), coarse_sums=coarse), ref) <= 5e-2
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = block.infer(x, agg, block.pack())
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other, block.infer(x, agg, block.pack()))


def test_shapes_are_checked(layer):
    graph = layer[0]
    with pytest.raises(ValueError):
        heta.FeedForwardBlock(graph, torch.empty(32, 64, device="cuda"), torch.empty(32, 64, device="cuda"))
    with pytest.raises(RuntimeError):
        heta.FeedForwardBlock(graph, torch.empty(32, 64, device="cuda"), torch.empty(64, 32, device="cuda")).backward(torch.empty(4, 32, device="cuda"))
