"""heta_adamw_multi where its other tests do not come: listed rows beyond the last-level cache, places beyond 2^32, roots over whole binades.  Tolerances as in test_gpu_adamw.py; where
two paths form the same value, its bits."""
import numpy as np
import pytest
import torch

import paper_2408_09697_amd as heta
from tests.test_gpu_adamw import B1, B2, BF16, E4M3, EPS, F32, LR, U, check_codes, random_bits, rows, state8, step64, values, within

pytestmark = pytest.mark.gpu


def bits_of(x):
    return x.view(torch.uint8) if x.dtype == E4M3 else x


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype,gdtype", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_many_listed_rows_are_the_rows_of_a_whole_update(dtype, gdtype, bits):
    """150,000 of 170,000 rows of 189 columns, 289 MB and more: the last lane of a row steps back by three."""
    n, k, d = 170_000, 150_000, 189
    W = rows(n, d, dtype, 1)
    state = state8(n, d, 3) if bits == 8 else (rows(n, d, F32, 3, scale=1e-2), rows(n, d, F32, 4, scale=1e-2).square())
    ids = torch.randperm(n, generator=torch.Generator(device="cuda").manual_seed(7), device="cuda")[:k].clone()
    g = rows(k, d, gdtype, 2, scale=1e-3)
    before = [x.clone() for x in (W, *state)]
    whole_W, whole_state, grad = W.clone(), tuple(x.clone() for x in state), torch.zeros(n, d, device="cuda", dtype=gdtype)
    grad[ids] = g
    heta.heta_adamw_multi([(whole_W, whole_state, grad, 0.5, None, 9)], lr=LR, step=3)
    heta.heta_adamw_multi([(W, state, g, 0.5, ids, 9)], lr=LR, step=3)
    listed = torch.zeros(n, dtype=torch.bool, device="cuda")
    listed[ids] = True
    for got, whole, old in zip((W, *state), (whole_W, *whole_state), before):
        assert torch.equal(bits_of(got)[listed], bits_of(whole)[listed])
        assert torch.equal(bits_of(got)[~listed], bits_of(old)[~listed])
    assert not torch.equal(W, before[0])


def test_places_beyond_32_bits():
    """Rows of a table of more than 2^32 elements; 2^32 lies three columns before the end of a lane's eight."""
    d = 4101
    cross = 2 ** 32 // d
    assert (2 ** 32 - cross * d) % 8 == 3
    n = cross + 5
    ids = torch.tensor([0, 1, 1000, cross - 1, cross, cross + 1, n - 1], device="cuda")
    k = len(ids)
    part = state8(k, d, 3)
    blocks = part[1].shape[1]
    W = torch.zeros(n, d, device="cuda", dtype=BF16)
    state = tuple(torch.zeros(n, c, device="cuda", dtype=t).view(s) for c, t, s in ((d, torch.uint8, E4M3), (blocks, F32, F32)) * 2)
    w, g = rows(k, d, BF16, 1), rows(k, d, F32, 2, scale=1e-3)
    W[ids] = w
    for whole, x in zip(state, part):
        bits_of(whole)[ids] = bits_of(x)
    m, r = values(part, d)
    want = step64(w.double(), m, r * r, g.double(), 0.0625, 7)
    heta.heta_adamw_multi([(W, state, g, 0.0625, ids, 12345)], lr=LR, beta1=B1, beta2=B2, eps=EPS, step=7)
    within(W[ids], want[0], want[3] + 8 * U * want[0].abs() + 2.0 ** -8 * (want[0].abs() + want[3]), "W")
    new = [bits_of(x)[ids].view(x.dtype) for x in state]
    bits = random_bits(ids, d, 12345, 7)
    check_codes(new[0], new[1], want[1], want[4] + U * B1 * m.abs(), bits & 0xffff, False, "m")
    check_codes(new[2], new[3], torch.sqrt(want[2]), 5 * U * torch.sqrt(want[2]), bits >> 16, True, "r")
    assert (W[2:1000] == 0).all() and (W[cross + 2:n - 1] == 0).all()
    del W, state
    torch.cuda.empty_cache()


def test_roots_are_correctly_rounded():
    """A column alone in its block: its scale is the root times 1 / 448, each rounded once.  v = 0.5 (code scale)^2 + 0.5 g^2, formed in fp32 step by step here; its root in 64 bits rounds
    to the correctly rounded fp32 root (53 >= 2 * 24 + 2 bits).  From 2^-90 to 2^100, all parts of two binades."""
    n = 1 << 22
    rng = np.random.RandomState(1)
    r = (rng.uniform(1, 2, n) * 2.0 ** np.repeat(rng.randint(-45, 50, n // 64), 64)).astype(np.float32)
    r[: n // 2] = rng.uniform(1, 4, n // 2).astype(np.float32)
    g = (r * rng.uniform(0, 2, n)).astype(np.float32)
    scale = (r / np.float32(448)).astype(np.float32)
    old = np.float32(448) * scale
    v = np.float32(0.5) * (old * old) + (np.float32(0.5) * g) * g
    root = np.sqrt(v.astype(np.float64)).astype(np.float32)
    want = root * np.float32(1 / 448)
    as_column = lambda x: torch.from_numpy(x).cuda()[:, None]  # noqa: E731
    codes = torch.full((n, 1), 448.0, device="cuda").to(E4M3)
    state = (torch.zeros(n, 1, device="cuda", dtype=torch.uint8).view(E4M3), torch.zeros(n, 1, device="cuda"), codes, as_column(scale))
    heta.heta_adamw_multi([(torch.zeros(n, 1, device="cuda"), state, as_column(g), 0.0, None, 1)], lr=0.0, beta1=0.0, beta2=0.5, eps=1e-8, step=1)
    assert (v >= 2.0 ** -95).all() and np.isfinite(v).all()
    got = state[3][:, 0].cpu().numpy()
    assert (got.view(np.int32) == want.view(np.int32)).all(), int((got.view(np.int32) != want.view(np.int32)).sum())
