"""heta_adamw_multi against the definition in 64 bits.

Tolerances, u = 2^-24.  m: two products, a sum, three roundings: 3 u (b1 |m| + (1 - b1) |g|); v: four: 4 u v (all its terms are positive).  W: the factor and
its product 2 u |W|; the step's numerator 3 u and m's error, its denominator 5 u relative (half of v's error, the root, a product, a sum) and half a unit each
of the two constants, the quotient: |step| 16 u + lr c1 e_m / denominator; the difference, u of the result; then a rounding to W's type (2^-8 for bf16).
8-bit states are read as code times scale (u), r^2 is a product (u): m is off by e_m = 3 u (b1 |m| + (1 - b1) |g|) + u b1 |m|, which is more than a multiple of u of
the new m where the two terms cancel, v by (4 + 3) u v and r = sqrt(v) by e_r = 5 u r.  A scale is off by the largest e of its block / 448 and 3 u of itself.
The codes are checked against the rounding that the kernel states: a value's is that of the 64-bit value, or its neighbour where the value in units of a step, y, plus the
random part of one, comes as near to the border between two as these errors bring it: 2^-12 steps (fp32's roundings of y < 16 are 2^-20 and, where 2^-6 is added, 2^-15), e in
steps, and y times the relative error of the scale.
"""
import math

import pytest
import torch

import paper_2408_09697_amd as heta

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
LR, B1, B2, EPS = 2.0 ** -10, 0.875, 0.9990234375, 2.0 ** -27  # exact in fp32
M32 = 0xffffffff


def rows(n, d, dtype, seed, pad=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((n, d + pad), float("nan"), device="cuda").to(dtype)
    buf[:, :d] = (torch.randn(n, d, generator=g, device="cuda") * scale).to(dtype)
    return buf[:, :d]


def mix(x):
    x ^= x >> 16
    x = x * 0x85ebca6b & M32
    x ^= x >> 13
    x = x * 0xc2b2ae35 & M32
    return x ^ x >> 16


def random_bits(ids, d, seed, step):
    k0 = mix((seed + 0x9e3779b9 * step) & M32)
    k1 = mix((k0 + 0x7f4a7c15) & M32)
    x = ids[:, None] * d + torch.arange(d, device=ids.device)
    x = ((x & M32) + (x >> 32) * 0x9e3779b9 + k0) & M32
    x = (x ^ x >> 16) * 0x85ebca6b & M32
    x = ((x ^ x >> 13) + k1) & M32
    x = x * 0xc2b2ae35 & M32
    return x ^ x >> 16


def spread(scale, d):
    return scale.double().repeat_interleave(128, 1)[:, :d]


def values(state, d):
    return state[0].double() * spread(state[1], d), state[2].double() * spread(state[3], d)


def step64(W, m, v, g, wd, step):
    m2, v2 = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    lr_c1, den = LR / (1 - B1 ** step), torch.sqrt(v2 / (1 - B2 ** step)) + EPS
    d = lr_c1 * m2 / den
    e_m = 3 * U * (B1 * m.abs() + (1 - B1) * g.abs())
    e_w = 3 * U * W.abs() + 16 * U * d.abs() + lr_c1 * e_m / den
    return W * (1 - LR * wd) - d, m2, v2, e_w, e_m, 4 * U * v2


def within(got, ref, bound, what):
    off = (got.double() - ref).abs()
    assert (off <= bound).all(), f"{what}: {float((off - bound).max()):.3e} over its bound, worst {float(off.max()):.3e}"


def check_codes(codes, scale, want, err, bits, positive, what):
    """codes and scales of the 64-bit values `want`, which fp32 has to within err."""
    n, d = want.shape
    size = torch.zeros(n, -(-d // 128) * 128, device="cuda", dtype=torch.float64)
    size[:, :d] = want.abs()
    top = size.view(n, -1, 128).amax(2)
    block_err = torch.zeros_like(size)
    block_err[:, :d] = err
    block_err = block_err.view(n, -1, 128).amax(2)
    within(scale, top / 448, (block_err + 3 * U * top) / 448, what + " scale")
    y = want.abs() / spread(top / 448, d).clamp_min(1e-300)
    unit = torch.exp2((torch.frexp(y)[1] - 4).clamp_min(-9).double())
    at = y / unit + bits.double() / 65536
    lower = torch.floor(at)
    got = codes.double().abs() / unit
    expect = torch.where((lower == 0) & (y > 0), 1.0, lower) if positive else lower
    steps = spread(top / 448, d).clamp_min(1e-300) * unit
    near = (at - torch.round(at)).abs() <= 2.0 ** -12 + err / steps + y / unit * spread(block_err / top.clamp_min(1e-300), d)
    # at the top of a binade the next number is one of the upper one's steps away, the same value
    ok = (got == expect) | (near & ((got - expect).abs() <= 1))
    assert ok.all(), (what, int((~ok).sum()))
    assert float(near.double().mean()) < 0.01 or n * d < 5000 or float((bits == 0).double().mean()) > 0.5
    sign = torch.signbit(codes.float()) == torch.signbit(want.float())
    assert (sign | (want == 0)).all(), what


def state8(n, d, seed, pad=0):
    m, r = rows(n, d, F32, seed, scale=1e-3), rows(n, d, F32, seed + 1, scale=1e-3).abs() + 1e-4
    out = []
    for x in (m, r):
        size = torch.zeros(n, -(-d // 128) * 128, device="cuda")
        size[:, :d] = x.abs()
        top = size.view(n, -1, 128).amax(2)
        buf = torch.zeros(n, d + pad, device="cuda", dtype=torch.uint8).view(E4M3)
        buf.view(torch.uint8)[:, :d] = (x / (top / 448).repeat_interleave(128, 1)[:, :d]).clamp(-448, 448).to(E4M3).view(torch.uint8)
        out += [buf[:, :d], top / 448]
    return tuple(out)


SHAPES = [(1, 1), (1, 5), (3, 8), (1, 1000), (7, 33), (64, 128), (100, 129), (33, 300), (5, 4097), (2000, 189), (257, 64)]


@pytest.mark.parametrize("dtype,gdtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,d", SHAPES)
def test_fp32_states(n, d, dtype, gdtype):
    for pad, wd, step in ((0, 0.0, 1), (3, 0.0625, 7)):
        W, g = rows(n, d, dtype, 1, pad), rows(n, d, gdtype, 2, pad, 1e-2)
        m, v = rows(n, d, F32, 3, pad, 1e-2), rows(n, d, F32, 4, pad, 1e-2).square()
        if pad:  # rows apart, as columns of wider buffers
            v = torch.full((n, d + pad), float("nan"), device="cuda")[:, :d].copy_(v)
        want = step64(W.double(), m.double(), v.double(), g.double(), wd, step)
        heta.heta_adamw_multi([(W, (m, v), g, wd)], lr=LR, beta1=B1, beta2=B2, eps=EPS, step=step)
        within(W, want[0], want[3] + (2.0 ** -8 if dtype == BF16 else U) * (want[0].abs() + want[3]), "W")
        within(m, want[1], want[4], "m")
        within(v, want[2], want[5], "v")


@pytest.mark.parametrize("dtype,gdtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,d", SHAPES)
def test_8bit_states(n, d, dtype, gdtype):
    for pad, wd, step in ((0, 0.0, 1), (3, 0.0625, 7)):
        W, g = rows(n, d, dtype, 1, pad), rows(n, d, gdtype, 2, pad, 1e-3)
        state = state8(n, d, 3, pad)
        m, r = values(state, d)
        want = step64(W.double(), m, r * r, g.double(), wd, step)
        heta.heta_adamw_multi([(W, state, g, wd, None, 12345)], lr=LR, beta1=B1, beta2=B2, eps=EPS, step=step)
        within(W, want[0], want[3] + 8 * U * want[0].abs() + (2.0 ** -8 if dtype == BF16 else U) * (want[0].abs() + want[3]), "W")
        bits = random_bits(torch.arange(n, device="cuda"), d, 12345, step)
        check_codes(state[0], state[1], want[1], want[4] + U * B1 * m.abs(), bits & 0xffff, False, "m")
        check_codes(state[2], state[3], torch.sqrt(want[2]), 5 * U * torch.sqrt(want[2]), bits >> 16, True, "r")


@pytest.mark.parametrize("bits", [8, 32])
def test_listed_rows(bits):
    n, d = 500, 200
    W = rows(n, d, F32, 1)
    state = state8(n, d, 3) if bits == 8 else (rows(n, d, F32, 3, scale=1e-2), rows(n, d, F32, 4, scale=1e-2).square())
    ids = torch.randperm(n, device="cuda")[:77].clone()
    ids[5], ids[6] = -1, n + 3  # skipped
    g = rows(77, d, F32, 2, scale=1e-3)
    before = [W.clone()] + [x.clone() for x in state]
    whole_W, whole_state, grad = W.clone(), tuple(x.clone() for x in state), torch.zeros(n, d, device="cuda")
    ok = (ids >= 0) & (ids < n)
    grad[ids[ok]] = g[ok]
    heta.heta_adamw_multi([(whole_W, whole_state, grad, 0.5, None, 9)], lr=LR, step=3)
    heta.heta_adamw_multi([(W, state, g, 0.5, ids, 9)], lr=LR, step=3)
    listed = torch.zeros(n, dtype=torch.bool, device="cuda")
    listed[ids[ok]] = True
    view = lambda x: x.view(torch.uint8) if x.dtype == E4M3 else x  # noqa: E731
    for got, whole, old in zip([W, *state], [whole_W, *whole_state], before):
        assert torch.equal(view(got)[listed], view(whole)[listed])
        assert torch.equal(view(got)[~listed], view(old)[~listed])


def test_many_tensors_at_once_are_the_single_updates():
    shapes = [(1, 7 + 3 * i) for i in range(70)] + [(40, 129), (3, 1000), (256, 16)]
    make = lambda: [(rows(n, d, (F32, BF16)[i % 2], i), (rows(n, d, F32, 100 + i), rows(n, d, F32, 200 + i).square()) if i % 3 else state8(n, d, 300 + i),  # noqa: E731
                     rows(n, d, (F32, BF16)[i // 2 % 2], 400 + i), 0.1 * (i % 4), None, i) for i, (n, d) in enumerate(shapes)]
    a, b = make(), make()
    plan = heta.heta_adamw_plan(a)
    for step in (1, 2):
        heta.heta_adamw_multi(plan, lr=LR, step=step)
        for it in b:
            heta.heta_adamw_multi([it], lr=LR, step=step)
    for x, y in zip(a, b):
        assert torch.equal(x[0], y[0])
        for s, t in zip(x[1], y[1]):
            assert torch.equal(s.view(torch.uint8), t.view(torch.uint8))
    heta.heta_adamw_multi([])


def test_vectors_and_first_steps():
    W = rows(1, 300, F32, 1)[0].clone()
    g = rows(1, 300, F32, 2)[0].clone()
    for bits in (8, 32):
        w, state = W.clone(), heta.heta_adamw_state(W, bits)
        heta.heta_adamw_multi([(w, state, g, 0.0, None, 1)], lr=LR, eps=0.0, step=1)
        within(w, W.double() - LR * torch.sign(g).double(), 40 * U * (W.abs() + LR), "first step")  # m c1 / sqrt(v c2) = g / |g|
    zero = heta.heta_adamw_state(W, 8)
    w = W.clone()
    heta.heta_adamw_multi([(w, zero, torch.zeros_like(g), 0.0, None, 1)], lr=LR, step=1)
    assert torch.equal(w, W) and all((x.float() == 0).all() for x in zero)


def test_rounding_is_right_in_the_mean_and_moves_slow_states():
    """Gradients of a constant magnitude below a block's largest: r^2 has to reach its square, where rounding to the nearest leaves it at its start.  After t steps v = g^2 (1 -
    b2^t) for all elements; a code's rounding has a relative deviation of at most 2^-4 sqrt(1/4) a step, fed back with weight b2: the mean of n = 64,512
    elements is within 6 standard deviations of 2^-5 sqrt(t) / sqrt(n) plus the deviation's own bias in r^2 (its variance, below 2^-10 a step, t = 300: 0.3 as a bound)."""
    n, d, t = 512, 128, 300
    W = torch.zeros(n, d, device="cuda")
    g = torch.full((n, d), 0.37, device="cuda")
    g[:, 0] = 1.0  # the block's largest
    state = heta.heta_adamw_state(W, 8)
    for step in range(1, t + 1):
        heta.heta_adamw_multi([(W, state, g, 0.0, None, 77)], lr=0.0, beta2=B2, step=step)
    m, r = values(state, d)
    want = 0.37 * math.sqrt(1 - B2 ** t)
    assert abs(float(r[:, 1:].mean()) / want - 1) < 0.3
    assert abs(float(m[:, 1:].mean()) / 0.37 - 1) < 0.01
    assert float(r[:, 1:].std()) > 0


def test_nan_and_infinity_stay_in_their_block():
    n, d = 4, 300
    for bad in (float("nan"), float("inf")):
        W, g, state = rows(n, d, F32, 1), rows(n, d, F32, 2, scale=1e-3), state8(n, d, 3)
        g[1, 140] = bad
        clean = (W.clone(), tuple(x.clone() for x in state))
        other = g.clone()
        other[1, 140] = 0
        heta.heta_adamw_multi([(clean[0], clean[1], other, 0.0, None, 5)], lr=LR, step=2)
        heta.heta_adamw_multi([(W, state, g, 0.0, None, 5)], lr=LR, step=2)
        hit = torch.zeros(n, d, dtype=torch.bool, device="cuda")
        hit[1, 128:256] = True
        m, r = values(state, d)
        mc, rc = values(clean[1], d)
        assert torch.isnan(m[hit]).all() and torch.isnan(r[hit]).all()
        assert torch.equal(m[~hit], mc[~hit]) and torch.equal(r[~hit], rc[~hit])
        only = torch.zeros_like(hit)
        only[1, 140] = True
        assert torch.equal(W[~only], clean[0][~only])
        assert torch.isnan(W[only]).all()


def test_states_below_the_range():
    W, g, state = torch.ones(1, 128, device="cuda"), torch.full((1, 128), 1e-38, device="cuda"), heta.heta_adamw_state(torch.ones(1, 128, device="cuda"), 8)
    heta.heta_adamw_multi([(W, state, g, 0.0, None, 5)], lr=LR, step=1)
    assert torch.isfinite(W).all() and all((x.float() == 0).all() for x in state)


def test_captured_on_another_stream():
    W, g, state = rows(100, 200, BF16, 1), rows(100, 200, BF16, 2, scale=1e-3), state8(100, 200, 3)
    W2, state2 = W.clone(), tuple(x.clone() for x in state)
    plan = heta.heta_adamw_plan([(W, state, g, 0.1, None, 3)])
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        heta.heta_adamw_multi(plan, lr=LR, step=5)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        heta.heta_adamw_multi([(W2, state2, g, 0.1, None, 3)], lr=LR, step=5)
        torch.cuda.synchronize()
        assert torch.equal(W, W2)
        for a, b in zip(state, state2):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
