"""The kernels of the norm, linear and momentum calls that only large calls reach: whole 256 x 256 tiles and what is left of them, walks over several tiles
and rows per workgroup, splits and copies, streaming accesses, the momentum's large and small tiles.

Operands are small integers wherever the operator allows it: every product and sum is then exact in fp32 (below 2^24), a bf16 result is that sum rounded
once, and results are compared for equality, so that a lost row or tile shows whatever the size.  The norm's rows are compared, bit by bit, with those of calls on
parts of the rows, which run without streaming accesses and in one pass of their workgroups.
"""
import pytest
import torch

import paper_2408_09697_amd as heta
from tests import test_gpu_muon as small_muon

pytestmark = pytest.mark.gpu
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
NONE, RELU = heta.HETA_ACT_NONE, heta.HETA_ACT_RELU


@pytest.fixture(scope="module")
def handle():
    g = heta.heta_graph_create([(1, 1, 0)], [])
    yield g
    g.destroy()


def integers(seed, r, c, dtype, most=2, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((r, c + pad), float("nan"), device="cuda").to(dtype)
    buf[:, :c] = torch.randint(-most, most + 1, (r, c), generator=g, device="cuda").to(dtype)
    return buf[:, :c]


def randn(seed, *shape, scale=1.0):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale


# aligned rows with whole and with ragged tiles, rows in 16-byte steps only by their padding, and unaligned ones
@pytest.mark.parametrize("n,d_in,d_out,pad", [(70_000, 256, 512, 0), (70_011, 252, 264, 4), (40_000, 1100, 520, 0), (50_000, 301, 517, 0), (33_000, 64, 1000, 8)])
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("res", [False, True])
def test_forward(handle, n, d_in, d_out, pad, dtype, out_dtype, res):
    x, W, bias = integers(1, n, d_in, dtype, 2, pad), integers(2, d_in, d_out, dtype, 2, pad), integers(3, 1, d_out, F32, 5)[0]
    residual = integers(4, n, d_out, out_dtype, 9, pad) if res else None
    out, pre = (integers(5, n, d_out, out_dtype, 1, pad) for _ in range(2))
    heta.heta_linear(handle, x, W, out, bias=bias, act=RELU, residual=residual, pre=pre)
    want = x.float() @ W.float() + bias
    assert torch.equal(pre, want.to(out_dtype))
    want = want.clamp_min(0) + (residual.float() if res else 0)
    assert torch.equal(out, want.to(out_dtype))


@pytest.mark.parametrize("n,d_in,d_out,pad", [(40_000, 256, 264, 0), (40_011, 250, 264, 6), (40_000, 1000, 520, 8), (33_000, 384, 1001, 0), (30_000, 203, 520, 0)])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
@pytest.mark.parametrize("res", [False, True])
@pytest.mark.parametrize("coarse", [False, True])
def test_forward_of_8_bit_operands(handle, n, d_in, d_out, pad, out_dtype, res, coarse):
    """Coarse sums may miss 2^-12 of sum |a||b|, at most 1,000 * 9 * 2^-12 = 2.2 of results in steps of 1; the others miss nothing."""
    x, W = integers(1, n, d_in, F32, 3).to(E4M3), integers(2, d_out, d_in, F32, 3).to(E4M3)
    a, b = (torch.empty(t.shape[0], d_in + pad, device="cuda", dtype=E4M3)[:, :d_in] for t in (x, W))
    a.copy_(x), b.copy_(W)
    xs, ws, bias = 2.0 ** integers(3, 1, n, F32, 1)[0], 2.0 ** integers(4, 1, d_out, F32, 1)[0], integers(5, 1, d_out, F32, 5)[0]
    residual = integers(6, n, d_out, out_dtype, 9) if res else None
    out = torch.empty(n, d_out, device="cuda", dtype=out_dtype)
    heta.heta_linear(handle, a, b, out, bias=bias, act=RELU, residual=residual, in_scale=xs, w_scale=ws, coarse_sums=coarse)
    size = (x.float().abs() @ W.float().abs().t()) * (xs[:, None] * ws)
    want = ((x.float() @ W.float().t()) * (xs[:, None] * ws) + bias).clamp_min(0) + (residual.float() if res else 0)
    if not coarse:
        assert torch.equal(out, want.to(out_dtype))
    else:
        err = 2.0 ** -12 * size
        assert ((out.float() - want).abs() <= err + (2.0 ** -8 if out_dtype is BF16 else 2.0 ** -24) * (want.abs() + err)).all()


@pytest.mark.parametrize("n,d_in,d_out,pad", [(300_000, 256, 512, 0), (300_000, 100, 520, 4), (90_000, 1024, 264, 0), (150_000, 301, 203, 0), (20_011, 1030, 517, 3)])
@pytest.mark.parametrize("dtype,dw_dtype", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("form", ["own activation", "activation of the input", "none"])
def test_backward(handle, n, d_in, d_out, pad, dtype, dw_dtype, form):
    x, W, go = integers(1, n, d_in, dtype, 2, pad), integers(2, d_in, d_out, dtype, 2, pad), integers(3, n, d_out, dtype, 2, pad)
    act, in_act = (RELU if form == "own activation" else NONE), (RELU if form == "activation of the input" else NONE)
    pre, gp = (integers(4, n, d_out, dtype, 2, pad), integers(5, n, d_out, dtype, 1, pad)) if act else (None, None)
    in_pre = integers(6, n, d_in, dtype, 2, pad) if in_act else None
    gi, gw, gb = integers(7, n, d_in, dtype, 1, pad), integers(8, d_in, d_out, dw_dtype, 1, pad), torch.empty(d_out, device="cuda")
    heta.heta_linear_bwd(handle, x, W, go, act=act, pre=pre, grad_pre=gp, grad_in=gi, in_act=in_act, in_pre=in_pre, grad_W=gw, grad_bias=gb)
    g = go.float() * (pre > 0) if act else go.float()
    if act:
        assert torch.equal(gp, g.to(dtype))
    assert torch.equal(gb, g.sum(0))
    assert torch.equal(gw, (x.float().t() @ g).to(dw_dtype))
    want = g @ W.float().t()
    assert torch.equal(gi, (want * (in_pre > 0) if in_act else want).to(dtype))


SIZES = [(700_000, 256), (300_000, 300), (400_003, 203), (150_000, 1000), (40_000, 2500)]


@pytest.mark.parametrize("n,d", SIZES)
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (F32, E4M3), (BF16, BF16), (BF16, E4M3)])
def test_norm(n, d, dtype, out_dtype):
    x, res, gamma = randn(1, n, d).to(dtype), randn(2, n, d).to(dtype), 1 + 0.1 * randn(3, d)
    new = lambda m: (torch.empty(m, d, device="cuda", dtype=dtype), torch.empty(m, d, device="cuda", dtype=out_dtype), torch.empty(m, device="cuda"),  # noqa: E731
                     torch.empty(m, device="cuda") if out_dtype is E4M3 else None)
    total, out, rstd, scale = new(n)
    heta.heta_rms_norm(x, out, residual=res, sum=total, gamma=gamma, scale=scale, rstd=rstd)
    for at in (0, 8191, n // 2, n - 5000):
        part = slice(at, at + 5000)
        t, o, r, s = new(5000)
        heta.heta_rms_norm(x[part], o, residual=res[part], sum=t, gamma=gamma, scale=s, rstd=r)
        assert torch.equal(total[part], t) and torch.equal(rstd[part], r) and torch.equal(out[part].view(torch.uint8), o.view(torch.uint8))
        assert s is None or torch.equal(scale[part], s)
    # every row: the sum is exact, and its mean square within 64 roundings of what torch adds up
    assert torch.equal(total, (x.float() + res.float()).to(dtype))
    step = 1 << 16
    for i in range(0, n, step):
        want = 1 / torch.sqrt(total[i:i + step].double().square().mean(1) + 1e-6)
        assert ((rstd[i:i + step].double() - want).abs() <= 64 * 2.0 ** -24 * want).all()


@pytest.mark.parametrize("n,d", SIZES)
@pytest.mark.parametrize("dtype,go_dtype", [(F32, F32), (F32, BF16), (BF16, BF16)])
def test_norm_backward(handle, n, d, dtype, go_dtype):
    x, go, gs = integers(1, n, d, dtype), integers(2, n, d, go_dtype), integers(3, n, d, dtype)
    rstd, gamma = 2.0 ** integers(4, 1, n, F32, 1)[0], 1 + 0.1 * randn(5, d)
    gx, gg = torch.empty_like(x), torch.empty(d, device="cuda")
    heta.heta_rms_norm_bwd(handle, x, rstd, go, gx, gamma=gamma, grad_sum=gs, grad_gamma=gg)
    want = torch.zeros(d, device="cuda", dtype=torch.float64)
    for i in range(0, n, 1 << 16):
        part = slice(i, min(n, i + (1 << 16)))
        want += (go[part].double() * x[part].double() * rstd[part].double()[:, None]).sum(0)
    assert torch.equal(gg.double(), want)  # steps of 1 / 2, below 2^23
    for at in (0, 8191, n // 2, n - 5000):
        part = slice(at, at + 5000)
        p = torch.empty_like(x[part])
        heta.heta_rms_norm_bwd(handle, x[part], rstd[part].contiguous(), go[part], p, gamma=gamma, grad_sum=gs[part])
        assert torch.equal(gx[part], p)


@pytest.mark.parametrize("shapes", [[(1000, 2050), (2050, 1000)], [(777, 1300)] * 4, [(515, 515)] * 5, [(64, 5000), (5000, 72), (900, 900), (33, 33)]])
@pytest.mark.parametrize("dtype,coarse", [(F32, False), (F32, True), (BF16, False)])
def test_momentum(handle, shapes, dtype, coarse):
    """Against the definition in 64 bits with the bounds of the small matrices; a lost tile or row is percents of the update's norm."""
    items = [(randn(3 * i, r, c, scale=0.05).to(dtype), randn(3 * i + 1, r, c, scale=0.01), randn(3 * i + 2, r, c, scale=0.02)) for i, (r, c) in enumerate(shapes)]
    refs = [small_muon.reference(W, m, g, 0.02, 0.95, True, 0.01, 1e-7, 5) for W, m, g in items]
    heta.heta_muon_multi(handle, items, weight_decay=0.01, coarse=coarse)
    for (W, m, g), (want, mref, x) in zip(items, refs):
        assert ((m.double() - mref).abs() <= 2.0 ** -23 * mref.abs() + 2.0 ** -140).all()
        scale = 0.02 * max(1.0, W.shape[1] / W.shape[0]) ** 0.5
        loss, step = small_muon.LOSS[BF16 if coarse else dtype], small_muon.STEP[dtype]
        off = (W.double() - want).abs() - step * 2 * want.abs()
        assert float(off.clamp_min(0).norm()) <= scale * loss * float(x.norm())
