"""Weights of more columns than one launch has wavefronts for (2^26 of 64 lanes: a grid holds 2^32 threads)."""
import pytest
import torch

import paper_2408_09697_amd as heta

pytestmark = pytest.mark.gpu
PACK = {torch.int8: (heta.binding.heta_linear_pack_i8, 127.0), torch.float8_e4m3fn: (heta.binding.heta_linear_pack_e4m3, 448.0)}


@pytest.mark.parametrize("dtype", list(PACK))
def test_weights_of_many_columns(dtype):
    """One row: every column's code is its type's largest value, with the column's sign, and its scale times that the weight, to fp32's rounding."""
    pack, top = PACK[dtype]
    n = 2 ** 26 + 1000
    W = torch.randn(1, n, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").clamp_min_(-4)
    W[W.abs() < 0.01] = 1.0
    packed, scale = torch.zeros(n, 1, device="cuda", dtype=torch.uint8).view(dtype), torch.zeros(n, device="cuda")
    pack(W, packed, scale)
    for i in range(0, n, 1 << 24):
        at = slice(i, min(n, i + (1 << 24)))
        codes, w = packed[at, 0].float(), W[0, at]
        assert torch.equal(codes, torch.copysign(torch.full_like(w, top), w))
        assert ((codes.double() * scale[at].double() - w.double()).abs() <= 2.0 ** -22 * w.double().abs()).all()
