"""heta_muon_multi against the definition in 64 bits.

Tolerances.  m is one fused multiply-add: 2^-24 of its value.  The polynomial p(s) = 3.4445 s - 4.7750 s^3 + 2.0315 s^5 has |p(s) / s| and |p'(s)|
of at most 3.4445 where singular values stay (below 1.21), so what one step rounds off, relative to |X|_F, reaches the end of the
following j steps multiplied by at most 3.4445^j: 683 altogether after five steps.  A step rounds X, its Gram matrix and the
polynomial and forms three products; eight roundings of u = 2^-24 each would give 683 * 8 u = 3.3e-4 of |X|_F, and ones of 2^-17 (two
bf16 terms) 683 * 8 * 2^-17 = 4.2e-2.  The kernels keep two terms; the bound for fp32 weights is the tighter one all the same: the
roundings of a matrix's elements are independent, and what they add up to stays well below their worst case.  W is off by lr scale times that and its own rounding.
"""
import math

import pytest
import torch

import paper_2408_09697_amd as heta

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
A, B, C = 3.4445, -4.7750, 2.0315
LOSS = {F32: 683 * 8 * 2.0 ** -24, BF16: 683 * 8 * 2.0 ** -17}
STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def handle():
    g = heta.heta_graph_create([(1, 1, 0)], [])
    yield g
    g.destroy()


def matrix(r, c, dtype, seed, pad=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((r, c + pad), float("nan"), device="cuda").to(dtype)
    buf[:, :c] = (torch.randn(r, c, generator=g, device="cuda") * scale).to(dtype)
    return buf[:, :c]


def reference(W, m, g, lr, mu, nesterov, wd, eps, steps):
    # the ABI takes these as fp32 numbers; 1 - lr wd is formed from them and rounded
    lr, mu, wd, eps = (float(torch.tensor(v, dtype=F32)) for v in (lr, mu, wd, eps))
    g, m = g.double(), mu * m.double() + g.double()
    u = g + mu * m if nesterov else m
    x = u / (u.norm() + eps)
    for _ in range(steps):
        p = x @ x.t()
        x = A * x + (B * p + C * (p @ p)) @ x
    return (1 - lr * wd) * W.double() - lr * math.sqrt(max(1.0, W.shape[1] / W.shape[0])) * x, m, x


def check(W, m, ref, lr, dtype):
    want, mref, x = ref
    assert ((m.double() - mref).abs() <= 2.0 ** -23 * mref.abs() + 2.0 ** -140).all(), "momentum"
    scale = lr * math.sqrt(max(1.0, W.shape[1] / W.shape[0]))
    off = (W.double() - want - 0.0).abs() - STEP[dtype] * 2 * want.abs()
    assert torch.isfinite(W.double()).all()
    assert float(off.clamp_min(0).norm()) <= scale * LOSS[dtype] * float(x.norm()), f"{float(off.clamp_min(0).norm())} {scale * LOSS[dtype] * float(x.norm())}"


SHAPES = [(1, 1), (1, 40), (33, 1), (7, 5), (16, 64), (64, 16), (128, 256), (256, 128), (100, 300), (129, 130), (789, 64), (320, 513)]


@pytest.mark.parametrize("r,c", SHAPES)
@pytest.mark.parametrize("dtype,grad_dtype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("pad", [0, 3])
def test_one_matrix(handle, r, c, dtype, grad_dtype, pad):
    W, m, g = matrix(r, c, dtype, 1, pad, 0.05), matrix(r, c, F32, 2, pad, 0.01), matrix(r, c, grad_dtype, 3, pad, 0.02)
    nesterov, wd = (r + c) % 2 == 0, 0.1 if c > r else 0.0
    ref = reference(W, m, g, 0.03, 0.9, nesterov, wd, 1e-7, 5)
    heta.heta_muon_multi(handle, [(W, m, g)], lr=0.03, momentum=0.9, nesterov=nesterov, weight_decay=wd)
    check(W, m, ref, 0.03, dtype)


def test_many_matrices_are_those_of_calls_of_their_own(handle):
    shapes = SHAPES[3:] + [(64, 64)] * 6
    make = lambda: [(matrix(r, c, (F32, BF16)[i % 2], i, 0, 0.05), matrix(r, c, F32, 50 + i, 0, 0.01), matrix(r, c, F32, 90 + i)) for i, (r, c) in enumerate(shapes)]  # noqa: E731
    together, alone = make(), make()
    refs = [reference(W, m, g, 0.02, 0.95, True, 0.0, 1e-7, 5) for W, m, g in together]
    heta.heta_muon_multi(handle, together)
    for (W, m, g), ref in zip(together, refs):
        check(W, m, ref, 0.02, W.dtype)
    for it, (W, m, g) in zip(alone, together):
        heta.heta_muon_multi(handle, [it])
        assert torch.equal(it[1], m)
        check(it[0], it[1], (W.double(), m.double(), torch.ones(min(W.shape), device="cuda", dtype=torch.float64)), 0.04, W.dtype)
    heta.heta_muon_multi(handle, [])


@pytest.mark.parametrize("steps", [0, 1, 2, 7])
def test_steps(handle, steps):
    W, m, g = matrix(48, 96, F32, 1), torch.zeros(48, 96, device="cuda"), matrix(48, 96, F32, 3)
    ref = reference(W, m, g, 0.5, 0.0, False, 0.0, 1e-7, steps)
    heta.heta_muon_multi(handle, [(W, m, g)], lr=0.5, momentum=0.0, nesterov=False, steps=steps)
    want, _, x = ref
    assert float((W.double() - want).norm()) <= 0.5 * math.sqrt(2) * 3.4445 ** (steps + 1) * 8 * 2.0 ** -24 * float(x.norm()) + 2.0 ** -23 * float(want.norm())


def test_orthogonal_in_effect(handle):
    """Singular values of the update, over lr and scale, lie where five steps of the quintic leave those from 0.03 up: 0.68 to 1.21."""
    u, _ = torch.linalg.qr(matrix(200, 120, F32, 1).double())
    v, _ = torch.linalg.qr(matrix(120, 120, F32, 2).double())
    s = torch.logspace(math.log10(0.3), 0, 120, device="cuda", dtype=torch.float64)  # 0.3 / |s| = 0.04 after scaling
    g = ((u * s) @ v.t()).float()
    W, m = torch.zeros(200, 120, device="cuda"), torch.zeros(200, 120, device="cuda")
    heta.heta_muon_multi(handle, [(W, m, g)], lr=1.0, momentum=0.0)
    sv = torch.linalg.svdvals(W.double())
    assert float(sv.min()) > 0.6 and float(sv.max()) < 1.25


def test_zero_gradient_and_nan(handle):
    W0 = matrix(64, 96, F32, 1)
    items = [(W0.clone(), torch.zeros(64, 96, device="cuda"), torch.zeros(64, 96, device="cuda")), (W0.clone(), torch.zeros(64, 96, device="cuda"), matrix(64, 96, F32, 2)),
             (W0.clone(), torch.zeros(64, 96, device="cuda"), matrix(64, 96, F32, 2))]
    items[1][2][5, 6] = float("nan")
    heta.heta_muon_multi(handle, items, weight_decay=0.5)
    assert torch.equal(items[0][0], W0 * torch.tensor(1 - 0.02 * 0.5, dtype=F32, device="cuda"))
    assert items[1][0].isnan().any() and torch.isfinite(items[2][0]).all()


def test_same_bits_again_on_another_stream_and_in_a_graph(handle):
    def make():
        return [(matrix(128, 256, F32, 1), matrix(128, 256, F32, 2), matrix(128, 256, F32, 3)), (matrix(300, 70, BF16, 4), matrix(300, 70, F32, 5), matrix(300, 70, BF16, 6))]

    want, other, kept, start = make(), make(), make(), make()
    heta.heta_muon_multi(handle, want)
    torch.cuda.synchronize()
    heta.heta_muon_multi(handle, other, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        heta.heta_muon_multi(handle, kept)
    for _ in range(3):
        for k, s in zip(kept, start):
            k[0].copy_(s[0]), k[1].copy_(s[1])
        graph.replay()
        torch.cuda.synchronize()
        for a, b, k in zip(want, other, kept):
            assert torch.equal(a[0], b[0]) and torch.equal(a[0], k[0]) and torch.equal(a[1], b[1]) and torch.equal(a[1], k[1])
        heta.heta_muon_multi(handle, make())
