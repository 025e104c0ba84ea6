"""Edges of the norm, linear and momentum calls and of FeedForwardBlock: empty and extreme inputs, and kernels that only some sizes reach.

Where operands are small integers every product and sum is exact in fp32, so results are compared for equality of bits: a lost row, tile or
partial sum cannot hide in a tolerance.
"""
import math

import pytest
import torch

import paper_2408_09697_amd as heta

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def handle():
    g = heta.heta_graph_create([(1, 1, 0)], [])
    yield g
    g.destroy()


def randn(seed, *shape, scale=1.0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale


@pytest.mark.parametrize("agg", [False, True])
def test_a_block_of_no_rows(handle, agg):
    block = heta.FeedForwardBlock(handle, randn(1, 32, 64).to(BF16), randn(2, 64, 32).to(BF16), torch.ones(32, device="cuda"), torch.ones(64, device="cuda"))
    x = torch.empty(0, 32, device="cuda", dtype=BF16)
    for packed in (None, block.pack()):
        assert block.infer(x, x.clone() if agg else None, packed).shape == (0, 32)
    assert block.forward(x, x.clone() if agg else None).shape == (0, 32)
    assert block.backward(x).shape == (0, 32)
    assert all((v == 0).all() for v in block.grads.values() if v is not None)
