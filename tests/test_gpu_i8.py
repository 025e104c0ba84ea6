"""heta_linear on 8-bit whole numbers, and the calls that make them, against the definition in 64 bits.

Tolerances, u = 2^-24.  The sum of the products is exact; it is rounded to fp32 (u; where a long contraction is split, once a part and once an addition: 40 u of
the sum of magnitudes), multiplied by the product of the scales (2 u) and added to the bias (u of the result).  Activations as in the other products: slopes of
at most 1.13, and (|z| + 8) 4 u |y| for their evaluation.  Results are rounded once to their type.  Rows: x * (1 / max * 127) is three roundings, so a
value within 4 u of 127 of a half may go to either neighbour."""
import math

import pytest
import torch

import paper_2408_09697_amd as heta

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, I8 = torch.float32, torch.bfloat16, torch.int8
STEP = {F32: U, BF16: 2.0 ** -8}


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


def whole(n, d, seed, pad=0, lo=-128):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((n, d + pad), 99, device="cuda", dtype=I8)
    buf[:, :d] = torch.randint(lo, 128, (n, d), generator=g, device="cuda").to(I8)
    return buf[:, :d]


def act(x, kind):
    if kind == 0:
        return x
    if kind == 1:
        return x.clamp_min(0)
    z = x if kind == 3 else 2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)
    return x * torch.sigmoid(z)


def within(got, ref, bound, what):
    off = (got.double() - ref).abs()
    assert torch.isfinite(got.double()).all(), what
    assert (off <= bound).all(), f"{what}: {float((off - bound).max()):.3e} over its bound, worst {float(off.max()):.3e}"


SHAPES = [(1, 1, 1), (1, 64, 64), (3, 7, 5), (64, 256, 1024), (65, 72, 24), (100, 300, 200), (257, 128, 264), (515, 789, 65), (33, 2050, 40), (1000, 16, 512), (700, 64, 2000),
          (40000, 256, 264), (5000, 384, 1030), (3, 131071, 2)]


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("n,k,m", SHAPES)
def test_products(handle, n, k, m, out_dtype):
    for kind, pad, residual in ((0, 0, False), (1, 16, True), (2, 3, False), (3, 0, True)):
        q, W = whole(n, k, 1, pad), whole(m, k, 2, pad)
        si, sw = rows(1, n, F32, 3)[0].abs() / 100, rows(1, m, F32, 4)[0].abs() / 100
        bias = rows(1, m, F32, 5)[0] if kind else None
        res = rows(n, m, out_dtype, 6, pad) if residual else None
        out, pre = rows(n, m, out_dtype, 7, pad), rows(n, m, out_dtype, 8, pad) if kind == 2 else None
        heta.heta_linear(handle, q, W, out, bias=bias, act=kind, residual=res, pre=pre, in_scale=si, w_scale=sw)
        s = si.double()[:, None] * sw.double()
        p = (q.double() @ W.double().t()) * s  # whole numbers below 2^53: exact
        size = (q.double().abs() @ W.double().abs().t()) * s
        perr = 40 * U * size + 4 * U * p.abs()
        if bias is not None:
            p = p + bias.double()
            perr = perr + 2 * U * (p.abs() + bias.double().abs())
        if pre is not None:
            within(pre, p, perr + STEP[out_dtype] * (p.abs() + perr), "pre")
        y = act(p, kind)
        z = p.abs() if kind == 3 else 1.6 * (p.abs() + 0.045 * p.abs() ** 3)
        err = 1.13 * perr + ((z + 8) * 4 * U * y.abs() if kind >= 2 else 0)
        if res is not None:
            y = y + res.double()
            err = err + U * (y.abs() + err)
        within(out, y, err + STEP[out_dtype] * (y.abs() + err), "out")


def test_largest_sums_are_exact(handle):
    """2^17 - 1 products of -128 by -128 are 2^31 - 2^14."""
    k = (1 << 17) - 1
    q, W = torch.full((2, k), -128, dtype=I8, device="cuda"), torch.full((3, k), -128, dtype=I8, device="cuda")
    W[1] = 127
    W[2, 1:] = 0
    out = torch.empty(2, 3, device="cuda")
    heta.heta_linear(handle, q, W, out, in_scale=torch.ones(2, device="cuda"), w_scale=torch.ones(3, device="cuda"))
    want = q.double() @ W.double().t()
    assert ((out.double() - want).abs() <= 40 * U * want.abs()).all()
    # few products with many rows: no split, every value below 2^24 is exact
    q, W = whole(3000, 500, 1), whole(700, 500, 2)
    out = torch.empty(3000, 700, device="cuda")
    heta.heta_linear(handle, q, W, out, in_scale=torch.ones(3000, device="cuda"), w_scale=torch.ones(700, device="cuda"))
    assert torch.equal(out.double(), q.double() @ W.double().t())


def check_rows(x, q, scale):
    top = x.double().abs().amax(1)
    within(scale, top / 127, 2 * U * top / 127, "scale")
    y = x.double() * (127 / top)[:, None].nan_to_num(0, 0, 0)
    assert ((q.double() - y).abs() <= 0.5 + 127 * 4 * U).all() and (q.int().abs() <= 127).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d", [(1, 1), (5, 7), (300, 64), (257, 65), (100, 128), (100, 200), (64, 256), (50, 257), (33, 512), (40, 789), (20, 1024), (20, 1025), (9, 2048), (9, 2049), (3, 5000)])
def test_rows(n, d, dtype):
    for pad in (0, 3):
        x, q, scale = rows(n, d, dtype, 1, pad), whole(n, d, 2, pad), torch.empty(n, device="cuda")
        if n > 3:
            x[2] = 0
        heta.heta_linear_rows_i8(x, q, scale)
        check_rows(x, q, scale)
        if pad:
            assert (q.as_strided((n, pad), (d + pad, 1), q.storage_offset() + d) == 99).all()


def test_rows_that_hold_no_numbers(handle):
    x = rows(6, 100, F32, 1)
    x[1, 7], x[2, 99], x[3, 0] = float("nan"), float("inf"), -float("inf")
    x[4] *= 2.0 ** -140
    q, scale = whole(6, 100, 2), torch.empty(6, device="cuda")
    heta.heta_linear_rows_i8(x, q, scale)
    assert torch.isnan(scale[1]) and (scale[2:4] == float("inf")).all() and scale[4] == 0 and (q[4] == 0).all()
    check_rows(x[[0, 5]], q[[0, 5]], scale[[0, 5]])
    W, out = whole(8, 100, 3), torch.empty(6, 8, device="cuda")
    heta.heta_linear(handle, q, W, out, in_scale=scale, w_scale=torch.ones(8, device="cuda"))
    assert torch.isnan(out[1:4]).all() and (out[4] == 0).all() and torch.isfinite(out[[0, 5]]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("k,m", [(1, 1), (7, 5), (256, 1024), (300, 200), (789, 65)])
def test_weights(k, m, dtype):
    W, packed, scale = rows(k, m, dtype, 1, 3), whole(m, k, 2, 5), torch.empty(m, device="cuda")
    heta.heta_linear_pack_i8(W, packed, scale)
    check_rows(W.t(), packed, scale)


def test_no_rows_and_an_empty_call(handle):
    q, out = torch.empty(0, 32, dtype=I8, device="cuda"), torch.empty(0, 8, device="cuda")
    heta.heta_linear(handle, q, whole(8, 32, 1), out, in_scale=torch.empty(0, device="cuda"), w_scale=torch.ones(8, device="cuda"))
    heta.heta_linear_rows_i8(torch.empty(0, 32, device="cuda"), q, torch.empty(0, device="cuda"))


def test_captured_together(handle):
    x, W = rows(300, 200, BF16, 1), rows(200, 500, BF16, 2)
    packed, ws = torch.empty(500, 200, dtype=I8, device="cuda"), torch.empty(500, device="cuda")
    heta.heta_linear_pack_i8(W, packed, ws)
    q, s, out = torch.empty(300, 200, dtype=I8, device="cuda"), torch.empty(300, device="cuda"), torch.empty(300, 500, dtype=BF16, device="cuda")

    def run():
        heta.heta_linear_rows_i8(x, q, s)
        heta.heta_linear(handle, q, packed, out, act=2, in_scale=s, w_scale=ws)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for k in range(3):
        x.copy_(rows(300, 200, BF16, 10 + k))
        run()
        want = out.clone()
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


# contractions that are split over workgroups, large products by tiles of every width, rows that are copied first (one operand or both)
@pytest.mark.parametrize("pad_in,pad_w", [(0, 0), (0, 3), (5, 0), (1, 1)])
@pytest.mark.parametrize("n,k,m", [(3, 131071, 2), (64, 5008, 40), (1, 20000, 16), (700, 1024, 320), (40000, 304, 100), (3000, 500, 700), (5000, 3200, 384), (20000, 789, 349)])
def test_sums_are_exact_however_they_are_formed(handle, n, k, m, pad_in, pad_w):
    """With scales of 1 the result is the exact sum, rounded to fp32 once."""
    q, W = whole(n, k, 1, pad_in, 60), whole(m, k, 2, pad_w, 60)  # values of one sign: sums beyond 2^24
    out = torch.empty(n, m, device="cuda")
    heta.heta_linear(handle, q, W, out, in_scale=torch.ones(n, device="cuda"), w_scale=torch.ones(m, device="cuda"))
    assert torch.equal(out, (q.double() @ W.double().t()).float())
