"""The operators at the end of a model over node embeddings, as cases that can be measured: its loss, the update of what it
learned, and its answers in 8-bit integers.

  xent  : heta_linear_xent      z = in W + bias, lse = log sum_j exp z_j, loss = lse - z[label] (0 without a label), mean of the losses
          heta_linear_xent_bwd  D = (exp(z - lse) - onehot(label)) / labelled rows, grad_in = D W^T, grad_W = in^T D, grad_bias = sum D;
                                the logits z are in memory at no time
  adamw : heta_adamw_multi      m = b1 m + (1 - b1) g, v = b2 v + (1 - b2) g^2, W = (1 - lr wd) W - lr c1 m / (sqrt(c2 v) + eps) for
                                all tensors of a model; states in fp32, or m and r = sqrt(v) as e4m3 with a scale for each 128 columns of
                                a row, rounded up or down at random (a hash of the element's place, the step and a seed)
  i8    : heta_linear_rows_i8   q = round(127 x / max|x|) for each row, scale = max|x| / 127
          heta_linear           out = act(scale_i w_scale_j (q . Wq^T) + bias) + residual, the sums in 32-bit integers

Widths are those of the library's own workloads (7 to 1,024 columns, blocks four times as wide inside); classes range from a handful
over the 349 venues of the academic graph to the nodes of a type themselves, 1.1 M (which node is the other end of a link); rows from
one request of a few nodes to the 700,000 papers or 1.1 M authors of that graph.
"""
import math

import torch

own = False

NONE, RELU, GELU, SILU = "none", "relu", "gelu", "silu"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
BLOCK = 128
# the hyper-parameters as fp32 holds them
LR, BETA1, BETA2, EPS, DECAY = 0.0010000000474974513, 0.8999999761581421, 0.9990000128746033, 9.99999993922529e-09, 0.009999999776482582
STEP, SEED = 1000, 20240809
MOST_ADAM, MOST_OUT, MOST_LOGITS = 281_600_000, 819_200_000, 1_073_741_824


def listed():
    return [
        # the loss of one request's 64 nodes over the academic graph's venues: latency
        {"name": "xent_serve_bf16", "op": "xent", "train": False, "n": 64, "d": 256, "classes": 349, "dtype": "bf16"},
        # which of 1.1 M authors stands at the other end of a link, for four nodes: the weights are read once
        {"name": "xent_few_rows_bf16", "op": "xent", "train": False, "n": 4, "d": 1024, "classes": 1_100_000, "dtype": "bf16"},
        # training on all papers at once, 349 venues (rows of W start at any address)
        {"name": "xent_papers_bf16", "op": "xent", "train": True, "n": 700_000, "d": 256, "classes": 349, "dtype": "bf16"},
        # training with the nodes of a type as the classes: a mini-batch of 8,192
        {"name": "xent_entities_bf16", "op": "xent", "train": True, "n": 8192, "d": 512, "classes": 131_072, "dtype": "bf16"},
        # training in fp32, ragged in every size
        {"name": "xent_ragged_f32", "op": "xent", "train": True, "n": 5003, "d": 300, "classes": 2983, "dtype": "f32"},
        # the vectors of a deep model (gains and biases of its blocks): latency
        {"name": "adamw_vectors_f32", "op": "adamw", "tensors": 64, "rows": 1, "d": 1024, "dtype": "f32", "grad": "f32", "bits": 32, "listed_rows": 0},
        # the matrices of a deep model, bf16 with fp32 states
        {"name": "adamw_weights_bf16", "op": "adamw", "tensors": 24, "rows": 1024, "d": 4096, "dtype": "bf16", "grad": "bf16", "bits": 32, "listed_rows": 0},
        # a learnable table of 1.1 M authors, states in 8 bits, all rows
        {"name": "adamw_table_8bit", "op": "adamw", "tensors": 1, "rows": 1_100_000, "d": 256, "dtype": "bf16", "grad": "bf16", "bits": 8, "listed_rows": 0},
        # the rows of an fp32 table that a mini-batch touched, width no multiple of anything
        {"name": "adamw_rows_8bit", "op": "adamw", "tensors": 1, "rows": 1_000_000, "d": 189, "dtype": "f32", "grad": "f32", "bits": 8, "listed_rows": 200_000},
        # one request through the block's first product: latency
        {"name": "i8_serve", "op": "i8", "rows": 64, "d_in": 256, "d_out": 1024, "dtype": "bf16", "act": GELU, "residual": False},
        # inference through a block of hidden width 1,024
        {"name": "i8_wide", "op": "i8", "rows": 200_000, "d_in": 1024, "d_out": 4096, "dtype": "bf16", "act": SILU, "residual": False},
        # scores of a ragged width over the venues, the residual added
        {"name": "i8_ragged", "op": "i8", "rows": 100_000, "d_in": 789, "d_out": 349, "dtype": "bf16", "act": NONE, "residual": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


WIDTHS = [7, 16, 32, 64, 100, 128, 189, 256, 300, 512, 768, 789, 1024]


def draw(rng):
    op = rng.choice(["xent", "xent", "xent", "adamw", "adamw", "i8", "i8"])
    width = lambda most: rng.choice([w for w in WIDTHS if w <= most]) if rng.random() < 0.5 else _log(rng, 8, most)  # noqa: E731
    if op == "xent":
        dtype = rng.choice(["f32", "bf16", "bf16"])
        d = width(1024)
        classes = rng.choice([2, 8, 153, 349, 2983]) if rng.random() < 0.4 else _log(rng, 3, min(1_100_000, 2 ** 30 // d))
        most = min(700_000, MOST_LOGITS // classes, (2 ** 39 if dtype == "bf16" else 2 ** 36) // (d * classes))
        return {"op": op, "train": rng.random() < 0.7, "n": _log(rng, 1, most), "d": d, "classes": classes, "dtype": dtype}
    if op == "adamw":
        d, tensors = width(4096), rng.choice([1, 1, 2, 3, 7, 24, 100])
        rows = _log(rng, 1, min(1_100_000, MOST_ADAM // 2 // (d * tensors)))
        part = rng.random() < 0.4
        return {"op": op, "tensors": tensors, "rows": rows, "d": d, "dtype": rng.choice(["f32", "bf16"]), "grad": rng.choice(["f32", "bf16"]),
                "bits": rng.choice([32, 8, 8]), "listed_rows": _log(rng, 1, rows) if part else 0}
    d_in, d_out = width(4096), width(4096)
    most = min(200_000, MOST_OUT // max(d_in, d_out), int(8e11 / (d_in * d_out)))
    return {"op": op, "rows": _log(rng, 1, most), "d_in": d_in, "d_out": d_out, "dtype": rng.choice(["f32", "bf16", "bf16"]),
            "act": rng.choice([NONE, RELU, GELU, SILU]), "residual": rng.random() < 0.4}


# ---- inputs ---------------------------------------------------------------------------------------------

def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(scale)


def _state_8bit(x):
    """Rows as an earlier step left them: e4m3 and a scale for each 128 columns."""
    n, d = x.shape
    amax = torch.nn.functional.pad(x.abs(), (0, -d % BLOCK)).view(n, -1, BLOCK).amax(2)
    codes = (x * (448.0 / amax).repeat_interleave(BLOCK, 1)[:, :d]).clamp_(-448, 448).to(E4M3)
    return codes, amax / 448.0


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": case}
    t = DTYPES[case["dtype"]]
    if case["op"] == "xent":
        n, d, c = case["n"], case["d"], case["classes"]
        s["in"] = _randn(g, n, d, dtype=t)
        s["W"] = _randn(g, d, c, dtype=t, scale=2.0 * d ** -0.5)
        s["bias"] = _randn(g, c, scale=0.5)
        # classes of falling frequency; a tenth of the rows has no label
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        s["labels"] = (u * u * c).long().clamp_(max=c - 1)
        s["labels"][torch.rand(n, generator=g, device="cuda") < 0.1] = -1
        s["loss"], s["lse"], s["mean"] = (torch.empty(k, device="cuda") for k in (n, n, 2))
        if case["train"]:
            s["grad_in"], s["grad_W"], s["grad_bias"] = torch.empty_like(s["in"]), torch.empty_like(s["W"]), torch.empty(c, device="cuda")
    elif case["op"] == "adamw":
        n, d, k = case["rows"], case["d"], case["listed_rows"] or case["rows"]
        items = []
        for i in range(case["tensors"]):
            ids = torch.randperm(n, generator=g, device="cuda")[:k].clone() if case["listed_rows"] else None
            W = _randn(g, n, d, dtype=t, scale=0.05)
            grad = _randn(g, k, d, dtype=DTYPES[case["grad"]], scale=1e-3)
            # gradients of a column have a size of their own
            r = _randn(g, 1, d).exp_().mul(_randn(g, n, d).mul_(0.1).exp_()).mul_(1e-3)
            m = _randn(g, n, d).mul_(r).mul_(0.3)
            state = (m, r.square_()) if case["bits"] == 32 else (*_state_8bit(m), *_state_8bit(r))
            items.append((W, state, grad, DECAY if n > 1 else 0.0, ids, SEED + i))
        # the tensors of a model lie side by side, as do their states
        s["all"] = [torch.stack([x.view(torch.uint8) for x in same]).view(E4M3) if same[0].dtype == E4M3 else torch.stack(same)
                    for same in zip(*([W, *state] for W, state, *_ in items))]
        s["items"] = [(s["all"][0][i], tuple(x[i] for x in s["all"][1:]), *items[i][2:]) for i in range(len(items))]
    else:
        n, k, m = case["rows"], case["d_in"], case["d_out"]
        s["x"] = _randn(g, n, k, dtype=t)
        w = _randn(g, m, k, scale=k ** -0.5)
        s["w_scale"] = w.abs().amax(1) / 127
        s["Wq"] = torch.round(w / s["w_scale"][:, None]).to(torch.int8)
        s["bias"] = _randn(g, m, scale=0.1)
        s["residual"] = _randn(g, n, m, dtype=t) if case["residual"] else None
        s["q"], s["scale"], s["out"] = torch.empty(n, k, device="cuda", dtype=torch.int8), torch.empty(n, device="cuda"), torch.empty(n, m, device="cuda", dtype=t)
    if own:
        from paper_2408_09697_amd import binding as hb
        s["g"] = hb.heta_graph_create([(1, 1, 0)], [])  # the handle whose workspace the calls use
        s["hb"] = hb
        if case["op"] == "adamw":
            s["plan"] = hb.heta_adamw_plan(s["items"])  # the tensors of a model stay where they are from step to step
    return s


# ---- the plain form: elementary operations in 32 bits, rounded once at the end -----------------------------------

def _plain_xent(s, case):
    x, W, y = s["in"].float(), s["W"].float(), s["labels"]
    z = x @ W
    z += s["bias"]
    top = z.amax(1, keepdim=True)
    lse = (z - top).exp_().sum(1).log() + top[:, 0]
    has = y >= 0
    count = has.sum().float()
    at = y.clamp_min(0)[:, None]
    loss = torch.where(has, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    r = {"loss": loss, "lse": lse, "mean": torch.stack([loss.double().sum().float() / count.clamp_min(1), count])}
    if case["train"]:
        D = z.sub_(lse[:, None]).exp_()
        D.scatter_add_(1, at, torch.full_like(D[:, :1], -1.0))
        D *= (has / count.clamp_min(1))[:, None]
        r["grad_in"], r["grad_W"], r["grad_bias"] = (D @ W.t()).to(s["in"].dtype), (x.t() @ D).to(s["W"].dtype), D.sum(0)
    return r


M32 = 0xffffffff


def _mix(x):
    x ^= x >> 16
    x = x * 0x85ebca6b & M32
    x ^= x >> 13
    x = x * 0xc2b2ae35 & M32
    return x ^ x >> 16


def _random(rows, d, seed, step):
    """32 random bits for each element of these rows of a matrix d wide."""
    k0 = _mix((seed + 0x9e3779b9 * step) & M32)
    k1 = _mix((k0 + 0x7f4a7c15) & M32)
    x = rows[:, None] * d + torch.arange(d, device=rows.device)
    x = ((x & M32) + (x >> 32) * 0x9e3779b9 + k0) & M32
    x ^= x >> 16
    x = x * 0x85ebca6b & M32
    x ^= x >> 13
    x = (x + k1) & M32
    x = x * 0xc2b2ae35 & M32
    return x ^ x >> 16


def _by_block(per_block, d):
    return per_block.repeat_interleave(BLOCK, 1)[:, :d]


def _round_8bit(x, bits, least):
    """x as e4m3 with a scale for each 128 columns; `bits` (16 random ones) say whether a value goes up or down."""
    n, d = x.shape
    size = x.abs()
    amax = torch.nn.functional.pad(size, (0, -d % BLOCK)).view(n, -1, BLOCK).amax(2)
    f = torch.where(amax >= 2.0 ** -119, 448.0 / amax, torch.zeros_like(amax))
    y = (size * _by_block(f, d)).clamp_max(448.0)
    low = y < 2.0 ** -6
    y = torch.where(low, y + 2.0 ** -6, y)
    code = ((y.view(torch.int32) + (bits << 4).int()) >> 20) - torch.where(low, 968, 960).int()
    if least:
        code = torch.where((size > 0) & (_by_block(f, d) > 0), code.clamp_min(1), code)
    code |= (x.view(torch.int32) >> 24) & 128
    return code.to(torch.uint8).view(E4M3), torch.where(f > 0, amax / 448.0, torch.zeros_like(amax))


def _plain_adamw(s, case):
    c1, root_c2 = 1 / (1 - BETA1 ** STEP), math.sqrt(1 / (1 - BETA2 ** STEP))
    for W, state, grad, decay, ids, seed in s["items"]:
        at = slice(None) if ids is None else ids
        n, d = W.shape
        g, w = grad.float(), W[at].float()
        if case["bits"] == 32:
            m, v = state[0][at], state[1][at]
        else:
            m = state[0][at].float() * _by_block(state[1][at], d)
            r = state[2][at].float() * _by_block(state[3][at], d)
            v = r * r
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g * g
        r = v.sqrt()
        w = w * (1 - LR * decay) - (LR * c1) * m / (r * root_c2 + EPS)
        W[at] = w.to(W.dtype)
        if case["bits"] == 32:
            state[0][at], state[1][at] = m, v
        else:
            bits = _random(torch.arange(n, device=W.device) if ids is None else ids, d, seed, STEP)
            new = _round_8bit(m, bits & 0xffff, False) + _round_8bit(r, bits >> 16, True)
            for old, x in zip(state, new):
                old.view(torch.uint8 if old.dtype == E4M3 else old.dtype)[at] = x.view(torch.uint8) if x.dtype == E4M3 else x
    return s["all"]


def _act(x, kind):
    if kind == RELU:
        return x.clamp_min(0)
    if kind == GELU:
        return x / (1 + torch.exp(-2 * 0.7978845608028654 * (x + 0.044715 * x * x * x)))
    return x / (1 + torch.exp(-x)) if kind == SILU else x


def _plain_i8(s, case):
    x = s["x"].float()
    amax = x.abs().amax(1, keepdim=True)
    q = torch.round(x * torch.where(amax > 0, 127.0 / amax, torch.zeros_like(amax)))
    out = _act((q @ s["Wq"].float().t()) * ((amax / 127.0) * s["w_scale"]) + s["bias"], case["act"])
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return {"out": out.to(s["out"].dtype)}


# ---- the calls that a user makes ------------------------------------------------------------------------------

def _own(s, case):
    hb = s["hb"]
    if case["op"] == "xent":
        hb.heta_linear_xent(s["g"], s["in"], s["W"], s["labels"], s["loss"], s["lse"], bias=s["bias"], mean=s["mean"])
        r = {"loss": s["loss"], "lse": s["lse"], "mean": s["mean"]}
        if case["train"]:
            hb.heta_linear_xent_bwd(s["g"], s["in"], s["W"], s["labels"], s["lse"], bias=s["bias"], mean=s["mean"], grad_in=s["grad_in"],
                                    grad_W=s["grad_W"], grad_bias=s["grad_bias"])
            r.update(grad_in=s["grad_in"], grad_W=s["grad_W"], grad_bias=s["grad_bias"])
        return r
    if case["op"] == "adamw":
        hb.heta_adamw_multi(s["plan"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, step=STEP)
        return s["all"]
    act = {NONE: hb.HETA_ACT_NONE, RELU: hb.HETA_ACT_RELU, GELU: hb.HETA_ACT_GELU, SILU: hb.HETA_ACT_SILU}[case["act"]]
    hb.heta_linear_rows_i8(s["x"], s["q"], s["scale"])
    hb.heta_linear(s["g"], s["q"], s["Wq"], s["out"], bias=s["bias"], act=act, residual=s["residual"], in_scale=s["scale"], w_scale=s["w_scale"])
    return {"out": s["out"]}


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    return {"xent": _plain_xent, "adamw": _plain_adamw, "i8": _plain_i8}[case["op"]](state, case)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2}
    e = size[case["dtype"]]
    if case["op"] == "xent":
        n, d, c = case["n"], case["d"], case["classes"]
        moved, rows = (n * d + d * c) * e, n * 16 + c * 4
        # the logits and, of their gradient, two products
        return {"bytes": 2 * moved + rows + 4 * c, "flops": 6.0 * n * d * c} if case["train"] else {"bytes": moved + rows, "flops": 2.0 * n * d * c}
    if case["op"] == "adamw":
        n, d = case["tensors"] * (case["listed_rows"] or case["rows"]), case["d"]
        states = 16 * d if case["bits"] == 32 else 4 * d + 16 * -(-d // BLOCK)
        return {"bytes": n * (d * (2 * e + size[case["grad"]]) + states + (8 if case["listed_rows"] else 0)), "flops": 15.0 * n * d}
    n, k, m = case["rows"], case["d_in"], case["d_out"]
    return {"bytes": n * k * e + k * m + n * m * e * (2 if case["residual"] else 1) + 8 * m, "flops": 2.0 * n * k * m}


# ---- the operators' definitions in 64 bits ------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(s, case)
    n = case["n"] if case["op"] == "xent" else case["rows"]
    step = max(1, (1 << 27) // (case["classes"] if case["op"] == "xent" else case["d_in"] + case["d_out"]))
    parts = [slice(i, min(n, i + step)) for i in range(0, n, step)]
    if case["op"] == "i8":
        return {"out": torch.cat([_exact_i8(s, case, at) for at in parts])}
    W, b = s["W"].double(), s["bias"].double()
    known = int((s["labels"] >= 0).sum())
    whole = {"loss": [], "lse": [], "grad_in": [], "grad_W": 0, "grad_bias": 0}
    for at in parts:
        x, y = s["in"][at].double(), s["labels"][at]
        z = torch.addmm(b, x, W)
        lse = torch.logsumexp(z, 1)
        rows = torch.nonzero(y >= 0)[:, 0]
        loss = torch.zeros_like(lse)
        loss[rows] = lse[rows] - z[rows, y[rows]]
        whole["loss"].append(loss)
        whole["lse"].append(lse)
        if case["train"]:
            p = torch.softmax(z, 1)
            del z
            p[rows, y[rows]] -= 1
            p[y < 0] = 0
            p /= max(known, 1)
            whole["grad_in"].append(torch.mm(p, W.mT))
            whole["grad_W"] = whole["grad_W"] + torch.mm(x.mT, p)
            whole["grad_bias"] = whole["grad_bias"] + p.sum(0)
    r = {"loss": torch.cat(whole["loss"]), "lse": torch.cat(whole["lse"])}
    r["mean"] = torch.stack([r["loss"].sum() / max(known, 1), torch.tensor(float(known), device="cuda", dtype=torch.float64)])
    if case["train"]:
        r.update(grad_in=torch.cat(whole["grad_in"]), grad_W=whole["grad_W"], grad_bias=whole["grad_bias"])
    return r


def _exact_states(x, chance, positive):
    """Values, relative to the scales, of the nearest or the next e4m3 number above x / scale below (by `chance` in [0, 1))."""
    rows, d = x.shape
    blocks = torch.zeros(rows, -(-d // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    blocks[:, :d] = x.abs()
    scale = blocks.view(rows, -1, BLOCK).max(2).values / 448
    y = blocks.view(rows, -1, BLOCK) / scale.clamp_min(1e-300)[:, :, None]
    y = y.view(rows, -1)[:, :d]
    unit = torch.exp2((torch.frexp(y)[1] - 4).clamp_min(-9).double())
    v = torch.floor(y / unit + chance) * unit
    if positive:
        v = torch.where((y > 0) & (v == 0), unit, v)
    return torch.copysign(v, x), scale


def _exact_adamw(s, case):
    done = []
    for W, state, grad, decay, ids, seed in s["items"]:
        rows = torch.arange(W.shape[0], device="cuda") if ids is None else ids
        d = W.shape[1]
        w, parts = W.double(), [x.double() for x in state]
        piece = max(1, (1 << 26) // d)
        for first in range(0, len(rows), piece):
            i, g = rows[first:first + piece], grad[first:first + piece].double()
            if case["bits"] == 32:
                m, v = parts[0][i], parts[1][i]
            else:
                spread = lambda q, sc: q[i] * sc[i].repeat_interleave(BLOCK, dim=1).narrow(1, 0, d)  # noqa: E731
                m, v = spread(parts[0], parts[1]), spread(parts[2], parts[3]) ** 2
            m = torch.lerp(g, m, BETA1)
            v = torch.lerp(g ** 2, v, BETA2)
            ahead = (m / (1 - BETA1 ** STEP)) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS)
            w[i] = w[i] - LR * (decay * w[i] + ahead)
            if case["bits"] == 32:
                parts[0][i], parts[1][i] = m, v
            else:
                h = _random(i, d, seed, STEP)
                parts[0][i], parts[1][i] = _exact_states(m, h.remainder(65536).double() / 65536, False)
                parts[2][i], parts[3][i] = _exact_states(torch.sqrt(v), h.div(65536, rounding_mode="floor").double() / 65536, True)
        done.append([w, *parts])
    return [torch.stack(same) for same in zip(*done)]


def _exact_i8(s, case, at):
    x = s["x"][at].double()
    top = torch.linalg.vector_norm(x, float("inf"), dim=1)
    q = torch.round(s["x"][at].float() * (127.0 / top.float())[:, None].nan_to_num(0, 0, 0)).double()  # which integer is the rounding's choice
    pre = torch.mm(q, s["Wq"].double().mT) * torch.outer(top / 127, s["w_scale"].double()) + s["bias"].double()
    if case["act"] == RELU:
        pre = torch.relu(pre)
    elif case["act"] != NONE:
        pre = pre * torch.sigmoid(pre if case["act"] == SILU else math.sqrt(8 / math.pi) * (pre + 0.044715 * pre ** 3))
    return pre if s["residual"] is None else pre + s["residual"][at].double()
