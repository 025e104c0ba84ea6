"""heta_linear, heta_linear_bwd and heta_linear_pack_e4m3 against the definition in 64 bits.

Tolerances, u = 2^-24 (one fp32 rounding).  Products of bf16, 8-bit or fp32 (as three bf16 terms, each product to 2^-24) operands
are added in fp32; an accumulator that truncates loses 2 u per addition: pre is off by at most (2 k + 16) u of sum |a||b| (+ |bias|).
Activations have slopes of at most 1.13, and x sigmoid(z) evaluates exp to |z| 2 u relative and rounds four times more, which
(|z| + 8) 4 u |y| covers; a result is rounded once to its type (2^-8 of its value for bf16, u for fp32).  Slopes act' are
bounded by 1.13 and off by 64 u.  Weight gradients add n products and then the partial sums: (2 n + 600) u of sum |a||b|, where a
rounded grad_pre (bf16) adds 2^-8 of every |b|.
"""
import math

import pytest
import torch

import paper_2408_09697_amd as heta

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
STEP = {F32: U, BF16: 2.0 ** -8}
NONE, RELU, GELU, SILU = range(4)


@pytest.fixture(scope="module")
def handle():
    g = heta.heta_graph_create([(1, 1, 0)], [])
    yield g
    g.destroy()


def rows(n, d, dtype, seed, pad=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((n, d + pad), float("nan"), device="cuda").to(dtype)
    buf[:, :d] = (torch.randn(n, d, generator=g, device="cuda") * scale).to(dtype)
    return buf[:, :d]


def act(x, kind):
    if kind == NONE:
        return x
    if kind == RELU:
        return x.clamp_min(0)
    z = x if kind == SILU else 2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)
    return x * torch.sigmoid(z)


def slope(x, kind):
    x = x.detach().clone().requires_grad_(True)
    with torch.enable_grad():
        return torch.autograd.grad(act(x, kind).sum(), x)[0] if kind != RELU else (x > 0).to(x.dtype)


def within(got, ref, bound, what):
    off = (got.double() - ref).abs()
    assert torch.isfinite(got.double()).all(), what
    assert (off <= bound).all(), f"{what}: {float((off - bound).max()):.3e} over its bound, worst {float(off.max()):.3e}"


# rows, d_in, d_out: one of each, tails of every tile dimension, more than one tile, long contractions, wide outputs
SHAPES = [(1, 1, 1), (1, 64, 64), (3, 7, 5), (64, 256, 1024), (65, 72, 24), (100, 300, 200), (257, 128, 264), (515, 789, 65), (33, 2050, 40), (1000, 16, 512),
          (700, 64, 2000), (40000, 256, 264)]


def check_forward(handle, n, d_in, d_out, dtype, out_dtype, kind, pad, res, want_pre):
    x, W = rows(n, d_in, dtype, 1, pad), rows(d_in, d_out, dtype, 2, pad, d_in ** -0.5)
    bias = rows(1, d_out, F32, 3)[0] if kind != RELU else None
    residual = rows(n, d_out, out_dtype, 4, pad) if res else None
    out, pre = rows(n, d_out, out_dtype, 5, pad), rows(n, d_out, out_dtype, 6, pad) if want_pre else None
    heta.heta_linear(handle, x, W, out, bias=bias, act=kind, residual=residual, pre=pre)
    p = x.double() @ W.double()
    size = x.double().abs() @ W.double().abs()
    if bias is not None:
        p, size = p + bias.double(), size + bias.double().abs()
    check_outputs(p, size, d_in, kind, residual, out, pre)


def check_outputs(p, size, k, kind, residual, out, pre):
    step, perr = STEP[out.dtype], (2 * k + 16) * U * size
    if pre is not None:
        within(pre, p, perr + step * (p.abs() + perr), "pre")
    y = act(p, kind)
    z = (p if kind != GELU else 1.6 * (p + 0.0448 * p.abs() ** 3)).abs()
    err = 1.13 * perr + (0 if kind in (NONE, RELU) else (z + 8) * 4 * U * y.abs())
    if residual is not None:
        y = y + residual.double()
        err = err + U * y.abs()
    within(out, y, err + step * (y.abs() + err), "out")


@pytest.mark.parametrize("n,d_in,d_out", SHAPES)
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("kind", [NONE, RELU, GELU, SILU])
def test_forward(handle, n, d_in, d_out, dtype, out_dtype, pad, kind):
    check_forward(handle, n, d_in, d_out, dtype, out_dtype, kind, pad, kind in (NONE, GELU), kind in (RELU, GELU))


@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("kind", [NONE, RELU, GELU, SILU])
@pytest.mark.parametrize("n,d_in,d_out,pad", [(40000, 252, 260, 4), (20011, 256, 514, 6), (24000, 1100, 516, 12)])
def test_large_products_with_tails_in_aligned_rows(handle, n, d_in, d_out, pad, dtype, out_dtype, kind):
    check_forward(handle, n, d_in, d_out, dtype, out_dtype, kind, pad, True, True)


@pytest.mark.parametrize("n,d_in,d_out", SHAPES)
@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("pad", [0, 16, 3])
def test_forward_of_8_bit_operands(handle, n, d_in, d_out, out_dtype, pad):
    x, W = rows(n, d_in, F32, 1), rows(d_in, d_out, F32, 2, 0, d_in ** -0.5)
    q, qs = torch.empty(n, d_in + pad, device="cuda", dtype=E4M3)[:, :d_in], torch.empty(n, device="cuda")
    heta.heta_rms_norm(x, q, scale=qs)
    w8, ws = torch.empty(d_out, d_in + pad, device="cuda", dtype=E4M3)[:, :d_in], torch.empty(d_out, device="cuda")
    heta.heta_linear_pack_e4m3(W, w8, ws)
    top = W.double().abs().amax(0)
    within(ws, top / 448, 4 * U * top / 448, "weights' scales")
    wd = w8.float().double() * ws.double()[:, None]
    within(wd, W.double().t(), (2.0 ** -4 + 8 * U) * W.double().t().abs() + 2.0 ** -10 * 1.001 * ws.double()[:, None], "8-bit weights")
    kind = (NONE, RELU, GELU, SILU)[(n + d_in) % 4]
    bias, residual = rows(1, d_out, F32, 3)[0], rows(n, d_out, out_dtype, 4, pad)
    out, pre = rows(n, d_out, out_dtype, 5, pad), rows(n, d_out, out_dtype, 6, pad)
    heta.heta_linear(handle, q, w8, out, bias=bias, act=kind, residual=residual, pre=pre, in_scale=qs, w_scale=ws)
    xd = q.float().double() * qs.double()[:, None]
    p, size = xd @ wd.t() + bias.double(), xd.abs() @ wd.t().abs() + bias.double().abs()
    check_outputs(p, size, d_in, kind, residual, out, pre)


@pytest.mark.parametrize("n,d_in,d_out", SHAPES)
@pytest.mark.parametrize("pad", [0, 3])
def test_coarse_sums_of_8_bit_operands(handle, n, d_in, d_out, pad):
    """An instruction of the 8-bit pipe keeps some 14 bits below its largest product: at most 2^-12 of sum |a||b| in all."""
    x, W = rows(n, d_in, F32, 1), rows(d_in, d_out, F32, 2, 0, d_in ** -0.5)
    q, qs = torch.empty(n, d_in + pad, device="cuda", dtype=E4M3)[:, :d_in], torch.empty(n, device="cuda")
    heta.heta_rms_norm(x, q, scale=qs)
    w8, ws = torch.empty(d_out, d_in + pad, device="cuda", dtype=E4M3)[:, :d_in], torch.empty(d_out, device="cuda")
    heta.heta_linear_pack_e4m3(W, w8, ws)
    out = torch.empty(n, d_out, device="cuda")
    heta.heta_linear(handle, q, w8, out, in_scale=qs, w_scale=ws, coarse_sums=True)
    a, b = q.float().double() * qs.double()[:, None], (w8.float().double() * ws.double()[:, None]).t()
    size = a.abs() @ b.abs()
    within(out, a @ b, (2.0 ** -12 + (2 * d_in + 16) * U) * size, "out")
    with pytest.raises(heta.HetaError):
        heta.heta_linear(handle, x, W, out, coarse_sums=True)


def test_residual_may_be_the_output(handle):
    x, W, h = rows(300, 128, BF16, 1), rows(128, 64, BF16, 2), rows(300, 64, BF16, 3)
    want, same = torch.empty_like(h), h.clone()
    heta.heta_linear(handle, x, W, want, act=SILU, residual=h)
    heta.heta_linear(handle, x, W, same, act=SILU, residual=same)
    assert torch.equal(want, same)


def test_infinite_pre_activations(handle):
    x = torch.tensor([[float("inf")], [-float("inf")], [float("nan")], [1e30], [-1e30], [0.0]], device="cuda")
    W = torch.ones(1, 1, device="cuda")
    for kind in (RELU, GELU, SILU):
        for bias in (None,):
            out = torch.empty(6, 1, device="cuda")
            pre = x.clone()
            # the terms of an infinite fp32 operand are not finite, so pre is given to the backward pass only
            heta.heta_linear(handle, x[3:], W, out[3:], act=kind, bias=bias)
            assert torch.equal(out[3:, 0].cpu(), torch.tensor([1e30, 0.0, 0.0]))
        gp, go = torch.empty_like(x), torch.ones_like(x)
        heta.heta_linear_bwd(handle, None, None, go, act=kind, pre=pre, grad_pre=gp)
        got = gp[:, 0].cpu()
        assert got[0] == 1 and abs(float(got[1])) < 1e-20 and got[2].isnan() and got[3] == 1 and abs(float(got[4])) < 1e-20
        assert float(got[5]) == (0.0 if kind == RELU else 0.5)


def test_rows_with_infinities_and_nan_keep_to_themselves(handle):
    for dtype in (F32, BF16):
        x, W = rows(300, 200, dtype, 1), rows(200, 136, dtype, 2)
        clean, dirty = torch.empty(300, 136, device="cuda", dtype=dtype), torch.empty(300, 136, device="cuda", dtype=dtype)
        heta.heta_linear(handle, x, W, clean, act=GELU)
        y = x.clone()
        y[17, 3], y[255, 199] = float("nan"), float("nan")
        heta.heta_linear(handle, y, W, dirty, act=GELU)
        keep = [i for i in range(300) if i not in (17, 255)]
        assert torch.equal(clean[keep], dirty[keep]) and dirty[17].isnan().all() and dirty[255].isnan().all()


@pytest.mark.parametrize("n,d_in,d_out", SHAPES)
@pytest.mark.parametrize("dtype,dw_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("kind", [NONE, RELU, GELU, SILU])
def test_backward(handle, n, d_in, d_out, dtype, dw_dtype, pad, kind):
    x, W = rows(n, d_in, dtype, 1, pad), rows(d_in, d_out, dtype, 2, pad, d_out ** -0.5)
    go, pre = rows(n, d_out, dtype, 3, pad), rows(n, d_out, dtype, 4, pad)
    in_act = (SILU, NONE, RELU, GELU)[kind]
    in_pre = rows(n, d_in, dtype, 5, pad) if in_act != NONE else None
    gp = rows(n, d_out, dtype, 6, pad) if kind != NONE else None
    gi, gw, gb = rows(n, d_in, dtype, 7, pad), rows(d_in, d_out, dw_dtype, 8, pad), torch.empty(d_out, device="cuda")
    heta.heta_linear_bwd(handle, x, W, go, act=kind, pre=pre if kind != NONE else None, grad_pre=gp, grad_in=gi, in_act=in_act, in_pre=in_pre,
                         grad_W=gw, grad_bias=gb)
    step = STEP[dtype]
    gpd = go.double() * slope(pre.double(), kind)
    gp_err = (0 if kind == NONE else 64 * 1.13 * U) * go.double().abs()
    if gp is not None:
        within(gp, gpd, gp_err + step * (gpd.abs() + gp_err), "grad_pre")
        gp_err = gp_err + step * (gpd.abs() + gp_err)
    within(gb, gpd.sum(0), (64 * 1.13 * U * (kind != NONE) + (n / 16 + 160) * U) * go.double().abs().sum(0), "grad_bias")
    Wd, xd = W.double(), x.double()
    ref, size = gpd @ Wd.t(), gpd.abs() @ Wd.abs().t()
    err = gp_err @ Wd.abs().t() if gp is not None else 0
    err = err + (2 * d_out + 16) * U * size
    if in_act != NONE:
        sl = slope(in_pre.double(), in_act)
        err = 1.13 * err + 64 * U * 1.13 * ref.abs()
        ref = ref * sl
    within(gi, ref, err + step * (ref.abs() + err), "grad_in")
    ref, size = xd.t() @ gpd, xd.abs().t() @ gpd.abs()
    err = (xd.abs().t() @ gp_err if gp is not None else 0) + (2 * n + 600) * U * size
    within(gw, ref, err + STEP[dw_dtype] * (ref.abs() + err), "grad_W")


def test_backward_agrees_with_differences(handle):
    """f = <act(x W + b), c> in 64 bits, central differences at t = 1e-5."""
    n, k, m = 20, 33, 17
    for kind in (GELU, SILU):
        x, W, b, c = rows(n, k, F32, 1), rows(k, m, F32, 2), rows(1, m, F32, 3)[0], rows(n, m, F32, 4)
        pre, out = torch.empty(n, m, device="cuda"), torch.empty(n, m, device="cuda")
        heta.heta_linear(handle, x, W, out, bias=b, act=kind, pre=pre)
        gi, gw, gb = torch.empty_like(x), torch.empty_like(W), torch.empty_like(b)
        heta.heta_linear_bwd(handle, x, W, c, act=kind, pre=pre, grad_pre=torch.empty_like(pre), grad_in=gi, grad_W=gw, grad_bias=gb)

        def f(xx, ww, bb):
            return (act(xx @ ww + bb, kind) * c.double()).sum()

        at, t = [x.double(), W.double(), b.double()], 1e-5
        for i, g in enumerate((gi, gw, gb)):
            v = torch.randn(at[i].shape, generator=torch.Generator(device="cuda").manual_seed(9 + i), device="cuda", dtype=torch.float64)
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + t * v, at[i] - t * v
            diff = float((f(*up) - f(*down)) / (2 * t))
            assert abs(float((g.double() * v).sum()) - diff) <= 2e-5 * float((g.double() * v).abs().sum())


@pytest.mark.parametrize("n,d_in,d_out,pad", [(20011, 301, 517, 0), (40011, 301, 517, 3), (70000, 264, 512, 3), (40000, 512, 789, 0), (90000, 256, 189, 0)])
@pytest.mark.parametrize("kind", [NONE, GELU])
def test_large_products_of_unaligned_rows(handle, n, d_in, d_out, pad, kind):
    check_forward(handle, n, d_in, d_out, BF16, BF16, kind, pad, True, True)
    test_backward(handle, n, d_in, d_out, BF16, BF16, pad, kind)


def test_a_workspace_that_grows_between_the_gradients():
    g = heta.heta_graph_create([(1, 1, 0)], [])
    test_backward(g, 40011, 301, 517, BF16, F32, 3, SILU)
    g.destroy()


def test_gradients_in_the_place_of_their_operands(handle):
    go, pre, x, W, ip = rows(500, 72, BF16, 1), rows(500, 72, BF16, 2), rows(500, 40, BF16, 3), rows(40, 72, BF16, 4), rows(500, 40, BF16, 5)
    gp, gi = torch.empty_like(go), torch.empty_like(x)
    heta.heta_linear_bwd(handle, x, W, go, act=SILU, pre=pre, grad_pre=gp, grad_in=gi, in_act=GELU, in_pre=ip)
    for on in ("grad_out", "pre"):
        a, b, c = go.clone(), pre.clone(), ip.clone()
        heta.heta_linear_bwd(handle, x, W, a, act=SILU, pre=b, grad_pre=a if on == "grad_out" else b, grad_in=c, in_act=GELU, in_pre=c)
        assert torch.equal(a if on == "grad_out" else b, gp) and torch.equal(c, gi)


def test_no_rows(handle):
    x, W, go = torch.empty(0, 24, device="cuda"), rows(24, 40, F32, 1), torch.empty(0, 40, device="cuda")
    heta.heta_linear(handle, x, W, torch.empty(0, 40, device="cuda"))
    gw, gb = torch.full((24, 40), 3.0, device="cuda"), torch.full((40,), 3.0, device="cuda")
    heta.heta_linear_bwd(handle, x, W, go, grad_in=torch.empty(0, 24, device="cuda"), grad_W=gw, grad_bias=gb)
    assert (gw == 0).all() and (gb == 0).all()


def test_same_bits_again_on_another_stream_and_in_a_graph(handle):
    x, W, go, pre = rows(3000, 256, BF16, 1), rows(256, 512, BF16, 2, 0, 0.06), rows(3000, 512, BF16, 3), rows(3000, 512, BF16, 4)
    bufs = lambda: (torch.full_like(go, 9), torch.full_like(x, 9), torch.full((256, 512), 9.0, device="cuda"), torch.full((512,), 9.0, device="cuda"))  # noqa: E731

    def call(b, stream=None):
        heta.heta_linear_bwd(handle, x, W, go, act=GELU, pre=pre, grad_pre=b[0], grad_in=b[1], grad_W=b[2], grad_bias=b[3], stream=stream)

    want = bufs()
    call(want)
    torch.cuda.synchronize()
    other = bufs()
    torch.cuda.synchronize()
    call(other, torch.cuda.Stream())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    kept = bufs()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(kept)
    for _ in range(3):
        for b in kept:
            b.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, kept))
        call(bufs())


def test_offsets_past_32_bits(handle):
    """in [200, 64] whose rows lie 12,000,000 elements apart; out [70, 64] 40,000,000 apart (the tile's offsets need 64 bits)."""
    buf = torch.empty(200 * 12_000_000, device="cuda", dtype=BF16)
    src, W = rows(200, 64, BF16, 1), rows(64, 64, BF16, 2)
    x = buf.as_strided((200, 64), (12_000_000, 1))
    x.copy_(src)
    out, want = torch.empty(200, 64, device="cuda", dtype=BF16), torch.empty(200, 64, device="cuda", dtype=BF16)
    heta.heta_linear(handle, src, W, want)
    heta.heta_linear(handle, x, W, out)
    ref = src.double() @ W.double()
    err = (2 * 64 + 16) * U * (src.double().abs() @ W.double().abs())
    within(out, ref, err + 2.0 ** -8 * (ref.abs() + err), "far rows in")
    far = buf.as_strided((70, 64), (30_000_000, 1))
    heta.heta_linear(handle, src[:70], W, far)
    assert torch.equal(far, want[:70])
