"""The operators of a residual feed-forward block over node embeddings, as cases that can be measured.

A deep model of this library follows the relation aggregation of a node type with a residual block of the kind that
language models are made of: the aggregate is added to the residual stream and normalised (root mean square), passes a
product with bias and activation and a second one whose epilogue adds the residual, and the weight matrices, those of
the relations and those of the block, are updated with orthogonalised momentum.  For inference the normalised rows may
be written as 8-bit values with a scale a row, which an 8-bit product reads.

  norm   : heta_rms_norm      s = x + r (rounded to the type it is stored in), out = s / sqrt(mean(s^2) + eps) * gamma
           heta_rms_norm_bwd  gradients of s and gamma; the gradient that reaches s past the norm is added
  linear : heta_linear        pre = in W + bias, out = act(pre) + residual; 8-bit: in and W times a scale a row / a column
           heta_linear_bwd    grad_pre = grad_out act'(pre), grad_in = grad_pre W^T, grad_W = in^T grad_pre, grad_bias
  muon   : heta_muon_multi    m = mu m + g, u = g + mu m, O = five steps X <- a X + (b X X^T + c (X X^T)^2) X from
           u / (|u| + eps), W <- (1 - lr wd) W - lr sqrt(max(1, d_out / d_in)) O, for all matrices of a model

Rows and widths are those of the library's own workloads (7 to 1,024 columns, one request of 64 nodes up to the
1.1 M nodes of the largest type of the academic graph; blocks four times as wide inside) and what lies between them.
"""
import math

import torch

own = False

EPS = 1e-6
NONE, RELU, GELU, SILU = "none", "relu", "gelu", "silu"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LR, MU, DECAY, MUON_EPS, STEPS = 0.02, 0.95, 0.01, 1e-7, 5
COEFFS = (3.4445, -4.7750, 2.0315)
MAX_ELEMS, MAX_FLOPS = 281_600_000, 2.0e12


def listed():
    return [
        # one serving request's 64 nodes: latency
        {"name": "norm_serve_bf16", "op": "norm", "back": False, "rows": 64, "d": 256, "dtype": "bf16", "out": "bf16", "residual": True},
        # inference over the largest node type of the academic graph, the rows written in 8 bits for the product behind
        {"name": "norm_authors_e4m3", "op": "norm", "back": False, "rows": 1_100_000, "d": 256, "dtype": "bf16", "out": "e4m3", "residual": True},
        # backward over a node type whose width is no multiple of anything (789 columns, rows unaligned)
        {"name": "norm_bwd_wide_f32", "op": "norm", "back": True, "rows": 100_000, "d": 789, "dtype": "f32", "out": "f32", "residual": True},
        # backward of a training step over all papers of the academic graph
        {"name": "norm_bwd_papers_bf16", "op": "norm", "back": True, "rows": 700_000, "d": 256, "dtype": "bf16", "out": "bf16", "residual": True},
        # one serving request through the block's first product: latency again
        {"name": "linear_serve_bf16", "op": "linear", "back": False, "rows": 64, "d_in": 256, "d_out": 1024, "dtype": "bf16", "act": GELU, "residual": False},
        # inference with 8-bit rows and weights, hidden width 1,024 and a block four times as wide
        {"name": "linear_wide_e4m3", "op": "linear", "back": False, "rows": 200_000, "d_in": 1024, "d_out": 4096, "dtype": "e4m3", "act": SILU, "residual": False},
        # the block's second product over all papers, the residual added in its epilogue
        {"name": "linear_papers_bf16", "op": "linear", "back": False, "rows": 700_000, "d_in": 1024, "d_out": 256, "dtype": "bf16", "act": NONE, "residual": True},
        # backward of the block's first product over all papers: both gradients and the bias's
        {"name": "linear_bwd_papers_bf16", "op": "linear", "back": True, "rows": 700_000, "d_in": 256, "d_out": 1024, "dtype": "bf16", "act": GELU, "residual": False},
        # backward in fp32 of a ragged product (a type of 300 columns) on a sampled block
        {"name": "linear_bwd_ragged_f32", "op": "linear", "back": True, "rows": 50_000, "d_in": 300, "d_out": 200, "dtype": "f32", "act": RELU, "residual": True},
        # the update of one layer's relation matrices, 7 of 128 x 256
        {"name": "muon_academic_f32", "op": "muon", "n": 7, "d_in": 128, "d_out": 256, "dtype": "f32"},
        # the update of a two-layer model of hidden width 1,024: bf16 weights
        {"name": "muon_mag_bf16", "op": "muon", "n": 10, "d_in": 768, "d_out": 1024, "dtype": "bf16"},
        # the update of a block's two products, 1,024 -> 4,096 (and back: the transposed shape)
        {"name": "muon_block_f32", "op": "muon", "n": 2, "d_in": 4096, "d_out": 1024, "dtype": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


WIDTHS = [7, 16, 24, 32, 64, 100, 128, 200, 256, 300, 512, 768, 789, 1000, 1024]


def draw(rng):
    op = rng.choice(["norm", "norm", "linear", "linear", "linear", "muon"])
    if op == "norm":
        d = rng.choice(WIDTHS) if rng.random() < 0.6 else _log(rng, 8, 4096)
        rows = _log(rng, 16, min(1_100_000, MAX_ELEMS // d))
        back = rng.random() < 0.4
        dtype = rng.choice(["f32", "bf16"])
        out = dtype if back else rng.choice([dtype, "bf16", "e4m3"])
        return {"op": op, "back": back, "rows": rows, "d": d, "dtype": dtype, "out": out, "residual": rng.random() < 0.7}
    if op == "linear":
        back = rng.random() < 0.4
        dtype = rng.choice(["f32", "bf16", "bf16"] if back else ["f32", "bf16", "bf16", "e4m3"])
        d_in, d_out = (rng.choice(WIDTHS) if rng.random() < 0.6 else _log(rng, 16, 4096) for _ in range(2))
        most = min(700_000, 800_000_000 // max(d_in, d_out), int((MAX_FLOPS if dtype == "e4m3" else MAX_FLOPS / 4) / (2 * d_in * d_out * (2 if back else 1))))
        return {"op": op, "back": back, "rows": _log(rng, 16, most), "d_in": d_in, "d_out": d_out, "dtype": dtype,
                "act": rng.choice([NONE, RELU, GELU, SILU]), "residual": rng.random() < 0.5}
    d_in, d_out = (rng.choice([64, 128, 256, 512, 768, 1024, 2048]) if rng.random() < 0.6 else _log(rng, 16, 2048) for _ in range(2))
    k = min(d_in, d_out)
    most = max(1, min(12, int(6e11 / (STEPS * (6.0 * k * d_in * d_out + 2.0 * k ** 3)))))
    return {"op": op, "n": rng.randint(1, most), "d_in": d_in, "d_out": d_out, "dtype": rng.choice(["f32", "bf16"])}


# ---- inputs ---------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=dtype if dtype is torch.bfloat16 else torch.float32) * scale).to(dtype)


def _rows(g, n, d, dtype):
    """Rows as a residual stream holds them: columns of different magnitude, a few large ones."""
    col = torch.exp(0.5 * torch.randn(d, generator=g, device="cuda")).to(dtype)
    return _randn(g, n, d, dtype=dtype).mul_(col)


def _quantise(x):
    """8-bit rows with a scale a row (what an earlier call of the model wrote, or the weights as they are stored)."""
    amax = x.abs().amax(1, keepdim=True)
    return (x * (448.0 / amax)).to(torch.float8_e4m3fn), (amax / 448.0).squeeze(1).contiguous()


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    f32 = torch.float32
    if case["op"] == "norm":
        n, d, t = case["rows"], case["d"], DTYPES[case["dtype"]]
        s["gamma"] = 1.0 + _randn(g, d, scale=0.1)
        if not case["back"]:
            s["x"] = _rows(g, n, d, t)
            s["residual"] = _rows(g, n, d, t) if case["residual"] else None
            s["sum"] = torch.empty_like(s["x"]) if case["residual"] else None
            s["out"] = torch.empty(n, d, device="cuda", dtype=torch.float8_e4m3fn if case["out"] == "e4m3" else DTYPES[case["out"]])
            s["scale"] = torch.empty(n, device="cuda") if case["out"] == "e4m3" else None
            s["rstd"] = torch.empty(n, device="cuda")
        else:
            s["x"] = _rows(g, n, d, t)
            s["rstd"] = torch.cat([(c.float().square().mean(1) + EPS).rsqrt() for c in s["x"].split(1 << 18)])
            s["grad_out"] = _randn(g, n, d, dtype=t)
            s["grad_sum"] = _randn(g, n, d, dtype=t) if case["residual"] else None
            s["grad_x"] = torch.empty_like(s["x"])
            s["grad_gamma"] = torch.empty(d, device="cuda")
    elif case["op"] == "linear":
        n, k, m = case["rows"], case["d_in"], case["d_out"]
        if case["dtype"] == "e4m3":
            s["in"], s["in_scale"] = _quantise(_randn(g, n, k))
            s["W"], s["w_scale"] = _quantise(_randn(g, m, k, scale=k ** -0.5))  # [d_out, d_in]
            t = torch.bfloat16
        else:
            t = DTYPES[case["dtype"]]
            s["in"], s["W"] = _randn(g, n, k, dtype=t), _randn(g, k, m, dtype=t, scale=k ** -0.5)
        s["bias"] = _randn(g, m, scale=0.1)
        if not case["back"]:
            s["residual"] = _randn(g, n, m, dtype=t) if case["residual"] else None
            s["out"] = torch.empty(n, m, device="cuda", dtype=t)
        else:
            s["pre"], s["grad_out"] = _randn(g, n, m, dtype=t), _randn(g, n, m, dtype=t)
            s["grad_pre"] = torch.empty_like(s["pre"]) if case["act"] != NONE else None
            s["grad_in"], s["grad_W"], s["grad_bias"] = torch.empty_like(s["in"]), torch.empty_like(s["W"]), torch.empty(m, device="cuda")
    else:
        t = DTYPES[case["dtype"]]
        s["items"] = []
        for i in range(case["n"]):
            # every other matrix leads back: its shape is the transposed one
            a, b = (case["d_in"], case["d_out"]) if i % 2 == 0 else (case["d_out"], case["d_in"])
            low = _randn(g, a, 4) @ _randn(g, 4, b)  # gradients are a few strong directions and noise
            grad = 1e-3 * (_randn(g, a, b) + 2.0 * low)
            s["items"].append((_randn(g, a, b, dtype=t, scale=a ** -0.5), 1e-2 * _randn(g, a, b), grad.to(t)))
    if own:
        from paper_2408_09697_amd import binding as hb
        s["g"] = hb.heta_graph_create([(1, 1, 0)], [])  # the handle whose workspace the calls use
        s["hb"] = hb
        s["act"] = {NONE: hb.HETA_ACT_NONE, RELU: hb.HETA_ACT_RELU, GELU: hb.HETA_ACT_GELU, SILU: hb.HETA_ACT_SILU}[case.get("act", NONE)]
    return s


# ---- the plain form: elementary operations in 32 bits, rounded once at the end -----------------------------------

def _act(x, kind):
    if kind == RELU:
        return x.clamp_min(0)
    if kind == GELU:
        return x / (1 + torch.exp(-2 * 0.7978845608028654 * (x + 0.044715 * x * x * x)))
    if kind == SILU:
        return x / (1 + torch.exp(-x))
    return x


def _act_grad(x, kind):
    if kind == RELU:
        return (x > 0).to(x.dtype)
    if kind == GELU:
        c = 2 * 0.7978845608028654
        sg = 1 / (1 + torch.exp(-c * (x + 0.044715 * x * x * x)))
        return sg + x * sg * (1 - sg) * c * (1 + 3 * 0.044715 * x * x)
    if kind == SILU:
        sg = 1 / (1 + torch.exp(-x))
        return sg + x * sg * (1 - sg)
    return torch.ones_like(x)


def _plain_norm(s, case):
    t = s["x"].dtype
    r = {}
    x = s["x"].float()
    if s["residual"] is not None:
        r["sum"] = (x + s["residual"].float()).to(t)
        x = r["sum"].float()
    rstd = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    y = x * rstd * s["gamma"]
    r["rstd"] = rstd.squeeze(1)
    if case["out"] == "e4m3":
        amax = y.abs().amax(1, keepdim=True)
        inv = torch.where(amax > 0, 448.0 / amax, torch.zeros_like(amax))
        r["scale"] = (amax / 448.0).squeeze(1)
        r["out"] = (y * inv).to(torch.float8_e4m3fn)
    else:
        r["out"] = y.to(s["out"].dtype)
    return r


def _plain_norm_bwd(s, case):
    x, go, rstd = s["x"].float(), s["grad_out"].float(), s["rstd"][:, None]
    xh = x * rstd
    w = go * s["gamma"]
    gx = rstd * (w - xh * (w * xh).mean(1, keepdim=True))
    if s["grad_sum"] is not None:
        gx = gx + s["grad_sum"].float()
    return {"grad_x": gx.to(s["x"].dtype), "grad_gamma": (go * xh).sum(0)}


def _plain_linear(s, case):
    if case["dtype"] == "e4m3":
        pre = (s["in"].float() @ s["W"].float().t()) * s["in_scale"][:, None] * s["w_scale"]
    else:
        pre = s["in"].float() @ s["W"].float()
    out = _act(pre + s["bias"], case["act"])
    if s["residual"] is not None:
        out = out + s["residual"].float()
    return {"out": out.to(s["out"].dtype)}


def _plain_linear_bwd(s, case):
    t = s["in"].dtype
    gp = s["grad_out"].float() * _act_grad(s["pre"].float(), case["act"])
    r = {"grad_in": (gp @ s["W"].float().t()).to(t), "grad_W": (s["in"].float().t() @ gp).to(t), "grad_bias": gp.sum(0)}
    if case["act"] != NONE:
        r["grad_pre"] = gp.to(t)
    return r


def _plain_muon(s, case):
    r = []
    for W, m, g in s["items"]:
        g32 = g.float()
        m.mul_(MU).add_(g32)
        u = g32 + MU * m
        x = u / (u.square().sum().sqrt() + MUON_EPS)
        tall = x.shape[0] > x.shape[1]
        x = x.t() if tall else x
        for _ in range(STEPS):
            a = x @ x.t()
            x = COEFFS[0] * x + (COEFFS[1] * a + COEFFS[2] * (a @ a)) @ x
        x = x.t() if tall else x
        W.copy_((1 - LR * DECAY) * W.float() - LR * math.sqrt(max(1.0, W.shape[1] / W.shape[0])) * x)
        r.append((W, m))
    return r


# ---- the calls that a user makes ------------------------------------------------------------------------------

def _own(s, case):
    hb = s["hb"]
    if case["op"] == "norm" and not case["back"]:
        hb.heta_rms_norm(s["x"], s["out"], residual=s["residual"], sum=s["sum"], gamma=s["gamma"], eps=EPS, scale=s["scale"], rstd=s["rstd"])
        r = {"rstd": s["rstd"], "out": s["out"]}
        if s["sum"] is not None:
            r["sum"] = s["sum"]
        if case["out"] == "e4m3":
            r["scale"] = s["scale"]
        return r
    if case["op"] == "norm":
        hb.heta_rms_norm_bwd(s["g"], s["x"], s["rstd"], s["grad_out"], s["grad_x"], gamma=s["gamma"], grad_sum=s["grad_sum"],
                             grad_gamma=s["grad_gamma"])
        return {"grad_x": s["grad_x"], "grad_gamma": s["grad_gamma"]}
    if case["op"] == "linear" and not case["back"]:
        # 8-bit inference lets the 8-bit matrix instruction add: its sums are a hundred times closer than the bf16 output
        hb.heta_linear(s["g"], s["in"], s["W"], s["out"], bias=s["bias"], act=s["act"], residual=s["residual"],
                       in_scale=s.get("in_scale"), w_scale=s.get("w_scale"), coarse_sums=case["dtype"] == "e4m3")
        return {"out": s["out"]}
    if case["op"] == "linear":
        hb.heta_linear_bwd(s["g"], s["in"], s["W"], s["grad_out"], act=s["act"], pre=s["pre"], grad_pre=s["grad_pre"],
                           grad_in=s["grad_in"], grad_W=s["grad_W"], grad_bias=s["grad_bias"])
        r = {"grad_in": s["grad_in"], "grad_W": s["grad_W"], "grad_bias": s["grad_bias"]}
        if case["act"] != NONE:
            r["grad_pre"] = s["grad_pre"]
        return r
    hb.heta_muon_multi(s["g"], s["items"], lr=LR, momentum=MU, weight_decay=DECAY, eps=MUON_EPS, steps=STEPS)
    return [(W, m) for W, m, _ in s["items"]]


def run(state):
    case = state["case"]
    if own:
        return _own(state, case)
    if case["op"] == "muon":
        return _plain_muon(state, case)
    if case["op"] == "norm":
        return _plain_norm_bwd(state, case) if case["back"] else _plain_norm(state, case)
    return _plain_linear_bwd(state, case) if case["back"] else _plain_linear(state, case)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    size = {"f32": 4, "bf16": 2, "e4m3": 1}
    if case["op"] == "norm":
        n, d, e = case["rows"], case["d"], size[case["dtype"]]
        if case["back"]:
            return {"bytes": n * d * e * (4 if case["residual"] else 3) + 4 * n + 8 * d, "flops": 9 * n * d}
        out = n * d * size[case["out"]] + (4 * n if case["out"] == "e4m3" else 0)
        return {"bytes": n * d * e * (3 if case["residual"] else 1) + out + 4 * n + 4 * d, "flops": 6 * n * d}
    if case["op"] == "linear":
        n, k, m, e = case["rows"], case["d_in"], case["d_out"], size[case["dtype"]]
        if case["back"]:
            moved = 2 * n * k + 2 * k * m + n * m * (1 + (2 if case["act"] != NONE else 0))
            return {"bytes": moved * e + 4 * m, "flops": 4.0 * n * k * m}
        o = 2 if case["dtype"] == "e4m3" else e
        scales = 4 * (n + m) if case["dtype"] == "e4m3" else 0
        return {"bytes": (n * k + k * m) * e + n * m * o * (2 if case["residual"] else 1) + 4 * m + scales, "flops": 2.0 * n * k * m}
    a, b, e = case["d_in"], case["d_out"], size[case["dtype"]]
    k, l = min(a, b), max(a, b)
    # a step: X X^T and its square are symmetric (half of their products), the last product is whole
    return {"bytes": case["n"] * a * b * (3 * e + 8), "flops": case["n"] * STEPS * (k * k * l + k ** 3 + 2.0 * k * k * l)}


# ---- the operators' definitions in 64 bits ------------------------------------------------------------------------

def _sigmoid_arg(x, kind):
    """z and dz/dx of act(x) = x sigmoid(z)."""
    if kind == SILU:
        return x, torch.ones_like(x)
    c = math.sqrt(8.0 / math.pi)
    return c * (x + 0.044715 * x ** 3), c * (1.0 + 0.134145 * x ** 2)


def _exact_act(x, kind):
    if kind == NONE:
        return x
    if kind == RELU:
        return torch.where(x > 0, x, torch.zeros_like(x))
    return x * torch.sigmoid(_sigmoid_arg(x, kind)[0])


def _exact_slope(x, kind):
    if kind == NONE:
        return torch.ones_like(x)
    if kind == RELU:
        return torch.where(x > 0, 1.0, 0.0).to(x.dtype)
    z, dz = _sigmoid_arg(x, kind)
    sg = torch.sigmoid(z)
    return sg * (1.0 + x * (1.0 - sg) * dz)


def _exact_e4m3(v):
    """v to the nearest of 3 significand bits behind the leading one, exponents from -6 up, ties to even."""
    step = torch.exp2(torch.frexp(v)[1].clamp_min(-5).double() - 4.0)
    return torch.round(v / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "muon":
        return _exact_muon(s)
    n = case["rows"]
    width = case["d"] if case["op"] == "norm" else case["d_in"] + case["d_out"]
    step = max(1, (1 << 27) // width)
    kind = _exact_norm_bwd if case["op"] == "norm" and case["back"] else _exact_norm if case["op"] == "norm" else _exact_linear_bwd if case["back"] else _exact_linear
    parts = [kind(s, case, slice(i, min(n, i + step))) for i in range(0, n, step)]
    whole = {}
    for key in parts[0]:
        values = [p[key] for p in parts]
        whole[key] = sum(values[1:], values[0]) if key in ("grad_gamma", "grad_W", "grad_bias") else torch.cat(values)
    return whole


def _exact_norm(s, case, at):
    v = s["x"][at].double()
    r = {}
    if s["residual"] is not None:
        r["sum"] = (v + s["residual"][at].double()).to(s["x"].dtype).double()  # what is stored is what is normalised
        v = r["sum"]
    r["rstd"] = torch.rsqrt(torch.linalg.vecdot(v, v) / case["d"] + EPS)
    y = torch.einsum("ij,i,j->ij", v, r["rstd"], s["gamma"].double())
    if case["out"] == "e4m3":
        top = y.abs().max(dim=1).values
        r["scale"] = top / 448.0
        y = _exact_e4m3(y / r["scale"].clamp_min(1e-300)[:, None])
    r["out"] = y
    return r


def _exact_norm_bwd(s, case, at):
    v, go, rs = s["x"][at].double(), s["grad_out"][at].double(), s["rstd"][at].double()[:, None]
    w = go * s["gamma"].double()
    along = torch.linalg.vecdot(w, v)[:, None]
    gx = rs * w - rs ** 3 * v * along / case["d"]
    if s["grad_sum"] is not None:
        gx = gx + s["grad_sum"][at].double()
    return {"grad_x": gx, "grad_gamma": (go * v * rs).sum(0)}


def _exact_linear(s, case, at):
    a, w = s["in"][at].double(), s["W"].double()
    if case["dtype"] == "e4m3":
        a, w = a * s["in_scale"][at].double()[:, None], (w * s["w_scale"].double()[:, None]).t()
    out = _exact_act(torch.addmm(s["bias"].double(), a, w), case["act"])
    return {"out": out if s["residual"] is None else out + s["residual"][at].double()}


def _exact_linear_bwd(s, case, at):
    gp = _exact_slope(s["pre"][at].double(), case["act"]) * s["grad_out"][at].double()
    r = {"grad_in": torch.mm(gp, s["W"].double().t()), "grad_W": torch.mm(s["in"][at].double().t(), gp), "grad_bias": gp.sum(0)}
    if case["act"] != NONE:
        r["grad_pre"] = gp
    return r


def _exact_muon(s):
    r = []
    for W, m, g in s["items"]:
        g64 = g.double()
        m64 = MU * m.double() + g64
        u = g64 + MU * m64
        x = u / (torch.linalg.matrix_norm(u) + MUON_EPS)
        # the polynomial acts on the singular values; on the smaller side's Gram matrix it is the same
        for _ in range(STEPS):
            if x.shape[0] <= x.shape[1]:
                p = x @ x.mT
                x = COEFFS[0] * x + COEFFS[1] * (p @ x) + COEFFS[2] * (p @ (p @ x))
            else:
                p = x.mT @ x
                x = COEFFS[0] * x + COEFFS[1] * (x @ p) + COEFFS[2] * ((x @ p) @ p)
        rows, cols = W.shape
        r.append((W.double() * (1 - LR * DECAY) - x * (LR * max(1.0, cols / rows) ** 0.5), m64))
    return r
