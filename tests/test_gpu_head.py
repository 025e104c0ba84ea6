"""ClassifierHead behind a layer and a feed-forward block, the trainer's update with 8-bit states, and 8-bit whole numbers through norm and products, as a program
runs them together.

The reference is the formula in 64 bits.  fp32: a product's result is off by 300 u of sum |a||b| (u = 2^-24), at most 10 times a result's typical size, and up to eight such stages
follow one another: 1e-4 of a result's norm.  bf16: up to 16 roundings of 2^-8 between input and gradient, 2^-8 * 4 = 1.6e-2 of the norm where they are independent.
Rows and weights of 8-bit whole numbers: a row's values are off by half a step, 1 / 254 of its largest (3 to 4 times its root mean square of d = 32 to 128 values), so
by 0.5 / 127 * 4 / sqrt(3) = 9e-3 of the norm on both sides of a product: 1.3e-2, and bf16's roundings: 2.5e-2."""
import math

import numpy as np
import pytest
import torch

import paper_2408_09697_amd as heta

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def act(x):
    return x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3))


def rel(got, ref):
    return float((got.double() - ref).norm() / ref.norm())


def randn(*s, seed=1, scale=1.0):
    return torch.randn(*s, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale


@pytest.fixture(scope="module")
def layer():
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


def labels_of(n, classes):
    y = torch.randint(0, classes, (n,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    y[::7] = -1
    return y


def mean_loss(z, y):
    has = y >= 0
    return (torch.logsumexp(z, 1) - z.gather(1, y.clamp_min(0)[:, None])[:, 0])[has].mean()


@pytest.mark.parametrize("dtype,most,classes", [(F32, 1e-4, 349), (BF16, 1.6e-2, 349), (BF16, 1.6e-2, 5000)])
def test_layer_block_and_head(layer, dtype, most, classes):
    graph, raf, tables = layer
    agg, x = raf.forward()[1].to(dtype), tables[1].to(dtype)
    W1, W2, W = randn(32, 128, seed=4, scale=32 ** -0.5).to(dtype), randn(128, 32, seed=5, scale=128 ** -0.5).to(dtype), randn(32, classes, seed=6, scale=0.3).to(dtype)
    gamma, b1, b2, bias = 1 + 0.1 * randn(32, seed=7), 0.1 * randn(128, seed=8), 0.1 * randn(32, seed=9), 0.1 * randn(classes, seed=10)
    y = labels_of(len(x), classes)
    block, head = heta.FeedForwardBlock(graph, W1, W2, gamma, b1, b2), heta.ClassifierHead(graph, W, bias, weight_decay=0.01)
    loss = head.loss(block.forward(x, agg), y)
    gx = block.backward(head.backward())
    leaves = [t.double().requires_grad_(True) for t in (x, W1, W2, gamma, b1, b2, W, bias)]
    h = leaves[0] + agg.double()
    n = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * leaves[3]
    ref = mean_loss((h + act(n @ leaves[1] + leaves[4]) @ leaves[2] + leaves[5]) @ leaves[6] + leaves[7], y)
    ref.backward()
    assert abs(float(loss) - float(ref)) <= most * float(ref)
    got = [gx] + [block.grads[k] for k in ("W1", "W2", "gamma", "b1", "b2")] + [head.grads["W"], head.grads["bias"]]
    for name, g, leaf in zip(("x", "W1", "W2", "gamma", "b1", "b2", "W", "bias"), got, leaves):
        assert rel(g, leaf.grad) <= most, name
    if dtype is F32:
        raf.backward({1: gx})
    # one update of all that has no matrix's optimizer, in one call: what the tensors' own calls do
    items = head.adamw_items() + block.vector_items()
    assert len(items) == 5
    kept = [(t[0].clone(), tuple(s.clone() for s in t[1]), *t[2:]) for t in items]
    heta.heta_adamw_multi(items, lr=0.01, step=1)
    for it in kept:
        heta.heta_adamw_multi([it], lr=0.01, step=1)
    for a, b in zip(items, kept):
        assert torch.equal(a[0], b[0]) and all(torch.equal(s, t) for s, t in zip(a[1], b[1]))
    block.update(lr=0.02)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores(layer, dtype):
    graph = layer[0]
    W, bias, h = randn(100, 349, seed=6, scale=0.3).to(dtype), 0.1 * randn(349, seed=10), randn(300, 100, seed=11).to(dtype)
    head = heta.ClassifierHead(graph, W, bias)
    ref = h.double() @ W.double() + bias.double()
    assert rel(head.scores(h), ref) <= (1e-5 if dtype is F32 else 4e-3)
    assert rel(head.scores(h, head.pack()), ref) <= 2.5e-2


def test_head_update_is_a_step_of_the_tensors(layer):
    for bits in (32, 8):
        W, bias, h, y = randn(64, 500, seed=6, scale=0.3), 0.1 * randn(500, seed=10), randn(300, 64, seed=11), labels_of(300, 500)
        head = heta.ClassifierHead(layer[0], W.clone(), bias.clone(), state_bits=bits, weight_decay=0.1, seed=5)
        w, b, sw, sb = W.clone(), bias.clone(), heta.heta_adamw_state(W, bits), heta.heta_adamw_state(bias)
        for step in (1, 2, 3):
            head.loss(h, y)
            head.backward()
            heta.heta_adamw_multi([(w, sw, head.grads["W"], 0.1, None, 5), (b, sb, head.grads["bias"])], lr=0.01, step=step)
            head.update(lr=0.01)
            assert torch.equal(head.W, w) and torch.equal(head.bias, b)
        assert not torch.equal(w, W)
    with pytest.raises(RuntimeError):
        heta.ClassifierHead(layer[0], W).backward()


def test_loss_gradients_and_update_captured(layer):
    """A step of a head captured into a graph and replayed, beside eager steps of another head on the same handle between the replays."""
    graph = layer[0]
    make = lambda: heta.ClassifierHead(graph, randn(64, 900, seed=6, scale=0.3).bfloat16(), None, state_bits=8, seed=5)  # noqa: E731
    h, y = randn(600, 64, seed=11).bfloat16(), labels_of(600, 900)
    a, b = make(), make()

    def one(head):
        head.loss(h, y)
        g = head.backward()
        head.step = 0
        head.update(lr=0.01)
        return g, head.saved["loss"]

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        warm = make()
        one(warm)  # the workspace grows outside of the capture
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured, stream=s):
        outs = one(a)
    for _ in range(3):
        captured.replay()
        torch.cuda.synchronize()
        want = one(b)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]) and torch.equal(a.W, b.W)
        for x, z in zip(a.states[0], b.states[0]):
            assert torch.equal(x.view(torch.uint8), z.view(torch.uint8))


def _trainer(state_bits, weight_decay, seed=777):
    from gen import workloads
    from tests.harness import dev_table
    wl = "tests/head"
    base = workloads.academic_graph(scale=0.01, workload=wl)
    tables = workloads._tables(base, wl, "f32", False)
    W = [workloads._weights(base, (lambda i, l=l: base.ntypes[base.relations[i].src_type].feat_dim if l == 0 else 64), 64, f"{wl}/L{l}", "f32", False) for l in range(2)]
    hg = heta.heta_graph_create([(t.num_nodes, t.feat_dim, int(t.learnable)) for t in base.ntypes], [(r.src_type, r.dst_type, r.rowptr, r.col) for r in base.relations])
    return base, hg, heta.MiniBatchTrainer(hg, [dev_table(x, "f32", 4) for x in tables], [[dev_table(w, "f32", 4) for w in ws] for ws in W], [6, 4], 64, heta.HETA_MEAN, 0, lr=1e-2,
                                           seed=seed, state_bits=state_bits, weight_decay=weight_decay)


@pytest.mark.parametrize("bits,wd", [(32, 0.0625), (8, 0.0), (8, 0.0625)])
def test_trainer_with_a_head(bits, wd):
    """Two iterations of the mini-batch trainer behind a head's loss.  What it did to every tensor is what heta_adamw_multi does to that tensor alone with the gradients
    that the iteration left; rows that the mini-batch did not touch stay."""
    base, hg, tr = _trainer(bits, wd)
    head = heta.ClassifierHead(hg, randn(64, 349, seed=6, scale=0.3), 0.1 * randn(349, seed=10), state_bits=bits)
    seeds_of = np.random.RandomState(0)
    view = lambda x: x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x  # noqa: E731
    for step in (1, 2):
        seeds = torch.from_numpy(np.sort(seeds_of.choice(base.ntypes[0].num_nodes, 128, replace=False)).astype(np.int64)).cuda()
        y = labels_of(128, 349)
        old = {("W", l, r): (tr.W[l][r].clone(), tuple(s.clone() for s in tr.sW[l][r])) for l in range(2) for r in range(len(tr.W[l]))}
        old.update({("T", t): (tr.tables[t].clone(), tuple(s.clone() for s in tr.sT[t])) for t in tr.learnable})
        H = tr.step(seeds, head.loss_grad(y), keep_blocks=True)
        head.update(lr=0.01)
        n_w = [len(ws) for ws in tr.W]
        for l, lay in enumerate(tr.last_layers):
            for r in lay.rels:
                w, s = old["W", l, r]
                heta.heta_adamw_multi([(w, s, lay.dW[r], wd, None, tr.seed + sum(n_w[:l]) + r)], lr=tr.lr, step=step)
                assert torch.equal(w, tr.W[l][r]) and all(torch.equal(view(a), view(b)) for a, b in zip(s, tr.sW[l][r]))
        first = tr.last_layers[0]
        assert tr.learnable
        for t in tr.learnable:
            w, s = old["T", t]
            if t in first.dH0 and tr.last_blocks[0].src_ids[t].numel() > 0:
                heta.heta_adamw_multi([(w, s, first.dH0[t], 0.0, tr.last_blocks[0].src_ids[t], tr.seed + sum(n_w) + t)], lr=tr.lr, step=step)
            assert torch.equal(w, tr.tables[t]) and all(torch.equal(view(a), view(b)) for a, b in zip(s, tr.sT[t]))
        z = H.double() @ head.W.double()  # the head has been updated: only its inputs are looked at here
        assert torch.isfinite(z).all()
        for b in tr.last_blocks:
            b.graph.destroy()
    hg.destroy()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,d", [(1, 1), (5, 7), (300, 64), (64, 256), (50, 257), (40, 789), (20, 1024), (9, 2048), (9, 2049)])
def test_norm_writes_whole_numbers(dtype, n, d):
    """Outputs s rstd gamma are off by (d / 2 + 16) u of their size (the sum of squares, its root, three products), rows are rounded as heta_linear_rows_i8's: a value within
    127 (d / 2 + 24) u of a half may go to either neighbour."""
    x, res = randn(n, d, seed=1).to(dtype), randn(n, d, seed=2).to(dtype)
    gamma = 1 + 0.1 * randn(d, seed=3)
    q, scale, s = torch.empty(n, d, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x)
    heta.heta_rms_norm(x, q, residual=res, sum=s, gamma=gamma, scale=scale)
    out = s.double() / torch.sqrt((s.double() ** 2).mean(1, keepdim=True) + 1e-6) * gamma.double()
    top = out.abs().amax(1)
    err = (d / 2 + 24) * U
    assert ((scale.double() - top / 127).abs() <= 2 * err * top / 127).all()
    assert ((q.double() - out * (127 / top)[:, None]).abs() <= 0.5 + 127 * 2 * err).all() and (q.int().abs() <= 127).all()


def test_block_infers_on_whole_numbers(layer):
    graph, raf, tables = layer
    agg, x = raf.forward()[1].bfloat16(), tables[1].bfloat16()
    W1, W2 = randn(32, 128, seed=4, scale=32 ** -0.5).bfloat16(), randn(128, 32, seed=5, scale=128 ** -0.5).bfloat16()
    gamma, b1, b2 = 1 + 0.1 * randn(32, seed=7), 0.1 * randn(128, seed=8), 0.1 * randn(32, seed=9)
    block = heta.FeedForwardBlock(graph, W1, W2, gamma, b1, b2)
    h = x.double() + agg.double()
    n = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * gamma.double()
    ref = h + act(n @ W1.double() + b1.double()) @ W2.double() + b2.double()
    packed = block.pack(torch.int8)
    assert packed[0].dtype is torch.int8 and rel(block.infer(x, agg, packed), ref) <= 2.5e-2
    assert torch.equal(block.infer(x, agg, packed), block.infer(x, agg, packed, coarse_sums=True))
