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


@pytest.fixture
def workspace_limit():
    """Sets what a handle's workspace may grow to, as if the device were full beyond it."""
    yield heta.binding.heta_workspace_limit
    heta.binding.heta_workspace_limit(0)


def test_momentum_that_cannot_have_its_workspace_updates_nothing(workspace_limit):
    """More matrices than share launches, the last of them large: the call fails before the first ones are touched, and can be repeated."""
    g = heta.heta_graph_create([(1, 1, 0)], [])
    make = lambda: [(randn(i, 24, 40), randn(50 + i, 24, 40), randn(90 + i, 24, 40)) for i in range(12)] + [(randn(40, 300, 500), randn(41, 300, 500), randn(42, 300, 500))]  # noqa: E731
    items, start, want = make(), make(), make()
    heta.heta_muon_multi(g, want)
    g.destroy()
    g = heta.heta_graph_create([(1, 1, 0)], [])
    workspace_limit(1 << 20)
    with pytest.raises(heta.HetaError) as e:
        heta.heta_muon_multi(g, items)
    assert e.value.args and "workspace" in str(e.value)
    for a, b in zip(items, start):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    workspace_limit(0)
    heta.heta_muon_multi(g, items)
    for a, b in zip(items, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    g.destroy()


def integers(seed, r, c, dtype, most=2, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((r, c + pad), float("nan"), device="cuda").to(dtype)
    buf[:, :c] = torch.randint(-most, most + 1, (r, c), generator=g, device="cuda").to(dtype)
    return buf[:, :c]


def test_linear_backward_in_little_memory(workspace_limit):
    """Copies of unaligned operands are left out where there is no room for them (the same result), and where there is none for the partial sums
    the call fails with its outputs untouched."""
    n, d_in, d_out = 100_000, 301, 517  # copies of 165 MB, partial sums of 26 MB
    x, W, go = integers(1, n, d_in, BF16), integers(2, d_in, d_out, BF16), integers(3, n, d_out, BF16)
    outs = lambda: (torch.full((n, d_in), 7.0, device="cuda", dtype=BF16), torch.full((d_in, d_out), 7.0, device="cuda"), torch.full((d_out,), 7.0, device="cuda"))  # noqa: E731
    want = (go.float() @ W.float().t()).to(BF16), x.float().t() @ go.float(), go.float().sum(0)
    for limit in (0, 64 << 20, 1 << 20):
        g, (gi, gw, gb) = heta.heta_graph_create([(1, 1, 0)], []), outs()
        workspace_limit(limit)
        if limit == 1 << 20:
            with pytest.raises(heta.HetaError):
                heta.heta_linear_bwd(g, x, W, go, grad_in=gi, grad_W=gw, grad_bias=gb)
            assert all((t == 7.0).all() for t in (gi, gw, gb))
            workspace_limit(0)
        heta.heta_linear_bwd(g, x, W, go, grad_in=gi, grad_W=gw, grad_bias=gb)
        for got, ref in zip((gi, gw, gb), want):
            assert torch.equal(got, ref), limit
        g.destroy()


def test_weight_gradient_of_many_elements(handle):
    """16,384 x 8,200: more columns than a launch of one workgroup per eight of them would hold."""
    x, go = integers(1, 70, 16384, BF16), integers(2, 70, 8200, BF16)
    gw = torch.full((16384, 8200), 7.0, device="cuda")
    heta.heta_linear_bwd(handle, x, None, go, grad_W=gw)
    assert torch.equal(gw, x.float().t() @ go.float())


@pytest.mark.parametrize("d", [24, 200, 789, 2048, 2500])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_8_bit_rows_with_nan_and_infinities(d, dtype):
    """A NaN among a row's outputs makes its scale and values NaN, as in packed weights; an infinity times the reciprocal root of an infinite sum is one."""
    x = randn(1, 20, d).to(dtype)
    clean = x.clone()
    x[2, d - 1], x[5, 0], x[9, d // 2], x[12] = float("nan"), float("inf"), -float("inf"), float("nan")
    out, ref, scale, scale0 = torch.empty(20, d, device="cuda", dtype=E4M3), torch.empty(20, d, device="cuda", dtype=E4M3), torch.empty(20, device="cuda"), torch.empty(20, device="cuda")
    heta.heta_rms_norm(x, out, scale=scale)
    heta.heta_rms_norm(clean, ref, scale=scale0)
    bad = [2, 5, 9, 12]
    keep = [i for i in range(20) if i not in bad]
    assert scale[bad].isnan().all() and out.float()[bad].isnan().all()
    assert torch.equal(scale[keep], scale0[keep]) and torch.equal(out.float()[keep], ref.float()[keep])
    W = x.t().contiguous()
    packed, ws = torch.empty(20, d, device="cuda", dtype=E4M3), torch.empty(20, device="cuda")
    heta.heta_linear_pack_e4m3(W, packed, ws)
    assert ws[[2, 12]].isnan().all() and packed.float()[[2, 12]].isnan().all() and torch.isfinite(ws[keep]).all()


@pytest.mark.parametrize("d", [16, 200, 2500])
def test_8_bit_rows_near_the_smallest_numbers(d):
    """Rows x whose largest value is m, with eps = 1: their reciprocal roots are 1, and out = x.  A value is off by half a step of e4m3 (2^-4 of it, or 2^-10 of the scale),
    the factor and the scale by three roundings and by half a subnormal step of the scale; from 2^-119 down rows are zeros with scale 0."""
    tops = [1e-30, 6e-36, 5e-36, 2e-36, 1.6e-36, 1.4e-36, 1e-37, 1e-38, 1e-42]
    x = torch.rand(len(tops), d, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda", dtype=torch.float64) * 2 - 1
    x[:, d // 3] = 1.0
    x = (x * torch.tensor(tops, device="cuda", dtype=torch.float64)[:, None]).float()
    q, scale = torch.empty(len(tops), d, device="cuda", dtype=E4M3), torch.empty(len(tops), device="cuda")
    w8, ws = torch.empty_like(q), torch.empty_like(scale)
    heta.heta_rms_norm(x, q, eps=1.0, scale=scale)
    heta.heta_linear_pack_e4m3(x.t().contiguous(), w8, ws)
    assert torch.equal(ws, scale) and torch.equal(w8.float(), q.float())
    kept = [i for i, t in enumerate(tops) if t >= 2.0 ** -119]
    gone = [i for i, t in enumerate(tops) if t < 2.0 ** -119]
    assert (scale[gone] == 0).all() and (q[gone].float() == 0).all()
    s, y = scale[kept].double()[:, None], x[kept].double()
    off = (q[kept].float().double() * s - y).abs()
    assert (off <= (2.0 ** -4 + 4 * U) * y.abs() + 2.0 ** -10 * (1 + 4 * U) * s + 448 * 2.0 ** -150).all()


@pytest.mark.parametrize("d", [24, 256, 789, 2500])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_zeros_without_eps(handle, d, dtype):
    """No reciprocal root of 0: such rows give zeros, and gradients that pass the norm by alone; their neighbours are those of other calls."""
    x, go, gs = randn(1, 9, d).to(dtype), randn(2, 9, d).to(dtype), randn(3, 9, d).to(dtype)
    clean = x.clone()
    x[2], x[6] = 0.0, 0.0
    keep = [i for i in range(9) if i not in (2, 6)]
    for out_dtype in (dtype, E4M3):
        out, ref = torch.empty(9, d, device="cuda", dtype=out_dtype), torch.empty(9, d, device="cuda", dtype=out_dtype)
        scale = torch.empty(9, device="cuda") if out_dtype is E4M3 else None
        rstd, rstd0 = torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
        heta.heta_rms_norm(x, out, eps=0.0, scale=scale, rstd=rstd)
        heta.heta_rms_norm(clean, ref, eps=0.0, scale=None if scale is None else torch.empty(9, device="cuda"), rstd=rstd0)
        assert (out[[2, 6]].float() == 0).all() and (rstd[[2, 6]] == 0).all() and (scale is None or (scale[[2, 6]] == 0).all())
        assert torch.equal(out[keep].float(), ref[keep].float()) and torch.equal(rstd[keep], rstd0[keep])
    gx, gg, gg0 = torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    heta.heta_rms_norm_bwd(handle, x, rstd, go, gx, grad_sum=gs, grad_gamma=gg)
    assert torch.equal(gx[[2, 6]], gs[[2, 6]]) and torch.isfinite(gx.float()).all()
    heta.heta_rms_norm_bwd(handle, x[keep], rstd[keep].contiguous(), go[keep], torch.empty_like(x[keep]), grad_gamma=gg0)
    assert float((gg - gg0).abs().max()) <= 160 * U * float((go.double() * x.double() * rstd.double()[:, None]).abs().sum(0).max())


def same_with_infinities(got, ref, bound, what):
    got = got.double()
    assert torch.equal(got.isnan(), ref.isnan()), what
    inf = ref.isinf()
    assert torch.equal(got[inf], ref[inf]), what
    fine = torch.isfinite(ref)
    assert ((got - ref).abs()[fine] <= bound[fine]).all(), what


@pytest.mark.parametrize("n,d_in,d_out", [(40, 24, 56), (300, 203, 136), (40000, 64, 264), (257, 2050, 40)])
def test_fp32_products_of_infinities_and_of_the_largest_numbers(handle, n, d_in, d_out):
    """The definition's results: infinity times 0 is NaN, times anything else infinity of their signs.  Other sums are those of the values: at most (2 k + 16) u of sum |a||b| off,
    also where a value is beyond bf16's largest."""
    x, W = integers(1, n, d_in, F32, 3), integers(2, d_in, d_out, F32, 3) / 16
    go = integers(3, n, d_out, F32, 3)
    x[3, 5], x[7, 1], x[7, 2], x[11, d_in - 1], x[12, 4] = float("inf"), float("inf"), -float("inf"), -float("inf"), float("nan")
    x[15, 3], x[16, 4], x[16, 7], x[17, 0] = 3.4028234e38, -3.4e38, 3.3961775e38, 3.39e38
    W[2, 9], W[8, 11] = -float("inf"), float("inf")
    go[n - 1, 2], go[n - 2, 3], go[5, 4] = float("inf"), -float("inf"), -3.402e38
    a, b, c = x.cpu().double(), W.cpu().double(), go.cpu().double()
    out = torch.empty(n, d_out, device="cuda")
    heta.heta_linear(handle, x, W, out)
    fin = lambda t: torch.where(torch.isfinite(t), t, torch.zeros_like(t)).abs()  # noqa: E731
    same_with_infinities(out.cpu(), a @ b, (2 * d_in + 16) * U * (fin(a) @ fin(b)), "out")
    gi, gw = torch.empty_like(x), torch.empty_like(W)
    heta.heta_linear_bwd(handle, x, W, go, grad_in=gi, grad_W=gw)
    same_with_infinities(gi.cpu(), c @ b.t(), (2 * d_out + 16) * U * (fin(c) @ fin(b).t()), "grad_in")
    x = integers(4, n, d_in, F32, 1) / 64
    x[3, 5], x[7, 1], x[12, 4], x[15, 3] = float("inf"), -float("inf"), float("nan"), 3.4028234e38
    a, c = x.cpu().double(), torch.where(c.abs() > 1e30, torch.ones_like(c), c) / 4
    heta.heta_linear_bwd(handle, x, None, c.float().cuda(), grad_W=gw)
    same_with_infinities(gw.cpu(), a.t() @ c, (2 * n + 600) * U * (fin(a).t() @ fin(c)), "grad_W")


@pytest.mark.parametrize("r,c", [(16, 16), (16, 48), (60, 16), (130, 16)])
@pytest.mark.parametrize("grad_dtype", [F32, BF16])
def test_momentum_of_fp32_weights_keeps_fp32(handle, r, c, grad_dtype):
    """Update of zero weights: -X scale.  Without steps X is u over its norm: a sum of r c squares whose terms add up in chains of at most 48, root, quotient and product, 48 u of
    every element in all.  One step on a matrix whose singular values are all 1 / 4 rounds X, its Gram matrix and the polynomial and forms three products over 16
    terms or the long side's, each off by a few u of the result in root mean square and multiplied by at most p(s) / s = 3.2 behind: 24 u of the norm.  (16 bits would be off by
    2^-17 = 128 u of the largest elements and 2^-18 = 64 u in root mean square at every rounding.)"""
    g = randn(1, r, c).to(grad_dtype)
    W, m = torch.zeros(r, c, device="cuda"), torch.zeros(r, c, device="cuda")
    scale = math.sqrt(max(1.0, c / r))
    heta.heta_muon_multi(handle, [(W, m, g)], lr=1.0, momentum=0.0, nesterov=False, steps=0)
    want = -scale * g.double() / (g.double().norm() + 1e-7)
    assert ((W.double() - want).abs() <= 48 * U * want.abs()).all()
    k = min(r, c)
    q = torch.linalg.qr(randn(2, max(r, c), k).double())[0]
    g = (q if r > c else q.t()).contiguous().float()
    W, m = torch.zeros(r, c, device="cuda"), torch.zeros(r, c, device="cuda")
    heta.heta_muon_multi(handle, [(W, m, g)], lr=1.0, momentum=0.0, nesterov=False, steps=1)
    x = g.double() / (g.double().norm() + 1e-7)
    x = x.t() if r > c else x
    a = x @ x.t()
    x = 3.4445 * x + (-4.7750 * a + 2.0315 * a @ a) @ x
    want = -scale * (x.t() if r > c else x)
    assert float((W.double() - want).norm()) <= 24 * U * float(want.norm())


def test_momentum_of_mixed_types_is_that_of_calls_of_their_own(handle):
    """Bits do not depend on what else is in the list, in whatever order."""
    shapes = [(64, 200, F32), (200, 64, BF16), (40, 40, BF16), (300, 128, F32), (16, 16, F32), (128, 128, BF16)] * 3
    make = lambda: [(randn(i, r, c, scale=0.1).to(t), randn(50 + i, r, c, scale=0.01), randn(90 + i, r, c)) for i, (r, c, t) in enumerate(shapes)]  # noqa: E731
    together, apart = make(), make()
    heta.heta_muon_multi(handle, together)
    for t in (F32, BF16):
        mine = [it for it in apart if it[0].dtype is t]
        for i in range(0, len(mine), 12):
            heta.heta_muon_multi(handle, mine[i:i + 12])
    for a, b in zip(together, apart):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_momentum_in_16_bits_on_request(handle):
    """The same for bf16 weights; fp32 ones then differ by what the header says, 2.5e-5 of the update's norm, here with four times as much room."""
    make = lambda t: [(randn(1, 100, 300, scale=0.1).to(t), randn(2, 100, 300, scale=0.01), randn(3, 100, 300))]  # noqa: E731
    for t in (F32, BF16):
        a, b, c = make(t), make(t), make(t)
        heta.heta_muon_multi(handle, a, lr=1.0)
        heta.heta_muon_multi(handle, b, lr=1.0, coarse=True)
        off, size = float((a[0][0].double() - b[0][0].double()).norm()), float((a[0][0].double() - c[0][0].double()).norm())
        assert off == 0.0 if t is BF16 else 0.0 < off <= 1e-4 * size
        assert torch.equal(a[0][1], b[0][1])


def test_8_bit_inference_adds_exactly_unless_asked(handle):
    block = heta.FeedForwardBlock(handle, randn(1, 256, 1024, scale=1 / 16).to(BF16), randn(2, 1024, 256, scale=1 / 32).to(BF16))
    x, packed = randn(3, 2000, 256).to(BF16), block.pack()
    exact, coarse = block.infer(x, packed=packed, coarse_sums=False), block.infer(x, packed=packed, coarse_sums=True)
    assert not torch.equal(exact, coarse)
    assert torch.equal(block.infer(x, packed=packed), exact)


@pytest.mark.parametrize("n,d_in,d_out", [(300, 1024, 4096), (2304, 256, 1000), (3000, 1024, 4096), (2400, 1792, 1024), (5000, 2048, 4096), (64, 300, 1100)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_few_row_blocks_and_splits(handle, n, d_in, d_out, dtype):
    """Counts of row blocks and of splits that eight does not divide: every tile is formed, by exact sums."""
    x, W, go = integers(1, n, d_in, dtype), integers(2, d_in, d_out, dtype), integers(3, n, d_out, dtype)
    out, gi, gw, gb = torch.empty(n, d_out, device="cuda"), torch.empty(n, d_in, device="cuda", dtype=dtype), torch.empty(d_in, d_out, device="cuda"), torch.empty(d_out, device="cuda")
    heta.heta_linear(handle, x, W, out)
    assert torch.equal(out, x.float() @ W.float())
    heta.heta_linear_bwd(handle, x, W, go, grad_in=gi, grad_W=gw, grad_bias=gb)
    assert torch.equal(gi, (go.float() @ W.float().t()).to(dtype)) and torch.equal(gw, x.float().t() @ go.float()) and torch.equal(gb, go.float().sum(0))


def test_copies_without_room_are_not_tried_again(workspace_limit):
    """A second call leaves the workspace alone, so that it can be captured into a graph like any warmed-up call."""
    n, d_in, d_out = 100_000, 301, 517
    x, go = integers(1, n, d_in, BF16), integers(3, n, d_out, BF16)
    want = x.float().t() @ go.float()
    g, gw = heta.heta_graph_create([(1, 1, 0)], []), torch.empty(d_in, d_out, device="cuda")
    workspace_limit(64 << 20)
    heta.heta_linear_bwd(g, x, None, go, grad_W=gw)
    workspace_limit(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        heta.heta_linear_bwd(g, x, None, go, grad_W=gw)
    for _ in range(3):
        gw.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gw, want)
    del graph
    g.destroy()
