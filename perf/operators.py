"""Cases for the training operators of language-model learners: the loss over a
large vocabulary, the norms around a block, and activations kept in 8 bits.

`own` false runs the operators in plain torch operations; true calls the
framework.  Every case has k learners (replicas) that live on one GPU, as
everywhere in the framework; n is the number of rows (tokens) of one learner.

  xent_step   loss, log-sum-exp, dh and dW of softmax cross-entropy of h W^T
  xent_eval   loss and log-sum-exp alone (validation, scoring)
  norm_step   x' = x + s gate (post norm(o)), y = pre norm(x'), then backward
  norm_fwd    the same forward alone (serving)
  ckpt_keep   activations to 8 bits and back
  ckpt_step   activations to 8 bits in the forward pass, the weight gradient
              of the layer that read them from those 8 bits in the backward
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
IGNORE = -100
EPS = 1e-5
GROUP = 32  # columns that share a scale in an 8-bit checkpoint


def listed():
    return [
        # the smallest training call: the repository's eight learners of 16 rows, 64 features, 1000 classes
        {"name": "xent-step-k8", "op": "xent_step", "type": "fp32", "k": 8, "n": 16, "d": 64, "v": 1000,
         "ignored": 0.0, "scale": 1.0},
        # a word-level vocabulary in the framework's own type
        {"name": "xent-step-fp32", "op": "xent_step", "type": "fp32", "k": 4, "n": 512, "d": 768, "v": 10007,
         "ignored": 0.1, "scale": 1.0},
        # two learners under loss scaling, ragged sizes, padded batches: two rows in five do not count
        {"name": "xent-step-ragged", "op": "xent_step", "type": "fp16", "k": 2, "n": 1023, "d": 1000, "v": 32001,
         "ignored": 0.4, "scale": 4096.0},
        # a training step of one large learner: 8192 tokens, 128,000 words
        {"name": "xent-step-large", "op": "xent_step", "type": "bf16", "k": 1, "n": 8192, "d": 4096, "v": 128000,
         "ignored": 0.1, "scale": 1.0},
        # scoring a single token
        {"name": "xent-eval-token", "op": "xent_eval", "type": "bf16", "k": 1, "n": 1, "d": 4096, "v": 128000,
         "ignored": 0.0, "scale": 1.0},
        # eight small learners' block
        {"name": "norm-step-k8", "op": "norm_step", "type": "fp32", "k": 8, "n": 16, "d": 64, "gate_rows": 16,
         "post": True},
        # a gate for every row, no multiple of any vector width, no norm after the block
        {"name": "norm-step-ragged", "op": "norm_step", "type": "fp16", "k": 2, "n": 1000, "d": 1001, "gate_rows": 1,
         "post": False},
        # a block of a large learner: eight sequences of 2048 tokens, one gate vector each
        {"name": "norm-step-large", "op": "norm_step", "type": "bf16", "k": 1, "n": 16384, "d": 4096,
         "gate_rows": 2048, "post": True},
        # one token of it while serving
        {"name": "norm-token", "op": "norm_fwd", "type": "bf16", "k": 1, "n": 1, "d": 4096, "gate_rows": 1,
         "post": True},
        # a large block's activations kept and given back
        {"name": "ckpt-keep-large", "op": "ckpt_keep", "type": "bf16", "k": 1, "n": 16384, "d": 4096},
        # LeNet's widest FC layer, eight learners of 16 images
        {"name": "ckpt-step-k8", "op": "ckpt_step", "type": "fp32", "k": 8, "n": 16, "d": 400, "out": 120},
        # the up projection of a large block
        {"name": "ckpt-step-large", "op": "ckpt_step", "type": "bf16", "k": 1, "n": 8192, "d": 2048, "out": 8192},
    ]


def _span(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng, lo, hi):
    """A row width: mostly a multiple of 64, at times of 8, at times odd."""
    d, r = _span(rng, lo, hi), rng.random()
    step = 64 if r < 0.6 else 8 if r < 0.8 else 1
    return max(step, d // step * step)


def draw(rng):
    op = rng.choice(["xent_step", "xent_step", "xent_eval", "norm_step", "norm_fwd", "ckpt_keep", "ckpt_step"])
    c = {"op": op, "type": rng.choice(["fp32", "bf16", "fp16"]), "k": rng.choice([1, 1, 2, 3, 4, 8])}
    if op in ("xent_step", "xent_eval"):
        while True:
            n, d, v = _span(rng, 1, 8192), _width(rng, 16, 4096), _span(rng, 10, 128000)
            if c["k"] * d * v <= 4096 * 128000 and c["k"] * n * d * v <= 2**40 and c["k"] * n * v <= 2**31:
                break
        c |= {"n": n, "d": d, "v": v, "ignored": rng.choice([0.0, 0.1, 0.4, 0.9]),
              "scale": 4096.0 if c["type"] == "fp16" else 1.0}
    elif op in ("norm_step", "norm_fwd"):
        while True:
            n, d = _span(rng, 1, 16384), _width(rng, 16, 8192)
            if c["k"] * n * d <= 2**26:
                break
        c |= {"n": n, "d": d, "gate_rows": rng.choice([1, n, max(1, n // 3), 7]), "post": rng.random() < 0.6}
    elif op == "ckpt_keep":
        while True:
            n, d = _span(rng, 1, 16384), _width(rng, 16, 8192)
            if c["k"] * n * d <= 2**26:
                break
        c |= {"n": n, "d": d}
    else:
        while True:
            n, d, out = _span(rng, 1, 8192), _width(rng, 16, 4096), _width(rng, 16, 8192)
            if c["k"] * n * d * out <= 2**37 and c["k"] * n * max(d, out) <= 2**27 and c["k"] * d * out <= 2**27:
                break
        c |= {"n": n, "d": d, "out": out}
    return c


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    t, k, n, d = TYPES[case["type"]], case["k"], case["n"], case["d"]

    def normal(*shape, std=1.0):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)

    s = {"case": case}
    if case["op"] in ("xent_step", "xent_eval"):
        v = case["v"]
        w = normal(k, v, d, std=1.0 / math.sqrt(d)).to(t)
        y = torch.randint(0, v, (k, n), generator=g, device="cuda", dtype=torch.int32)
        # a normed row that points to its label's weights by more or less: some words are sure, some are not
        learner = torch.arange(k, device="cuda")[:, None]
        h = normal(k, n, d) + w[learner, y.long()].float() * (8.0 * uniform(k, n, 1))
        # the last rows of every learner's batch are padding, and so are some between: at least one row counts
        pad = uniform(k, n) < case["ignored"] / 2
        pad |= torch.arange(n, device="cuda") >= n - int(n * case["ignored"] / 2)
        pad[:, 0] = False
        s |= {"h": h.to(t), "w": w, "labels": y.masked_fill_(pad, IGNORE)}
    elif case["op"] in ("norm_step", "norm_fwd"):
        groups = -(-n // case["gate_rows"])
        s |= {"x": normal(k, n, d, std=3.0).to(t), "o": normal(k, n, d).to(t),
              "gate": normal(k, groups, d, std=0.5).to(t),
              "post": 1.0 + normal(k, d, std=0.1) if case["post"] else None, "pre": 1.0 + normal(k, d, std=0.1)}
        if case["op"] == "norm_step":
            s |= {"dy": normal(k, n, d, std=0.1).to(t), "dres": normal(k, n, d, std=0.1).to(t)}
    else:
        # activations with a few loud columns, as trained blocks have them
        s["x"] = (normal(k, n, d) * (1.0 + 20.0 * (uniform(d) < 0.01))).to(t)
        if case["op"] == "ckpt_step":
            s["dy"] = normal(k, n, case["out"], std=0.1).to(t)
    return s


RES_SCALE = 0.5  # the residual scale of the norm cases


# --- the plain forms ---------------------------------------------------------

def _xent_plain(s, backward):
    h, w, y = s["h"], s["w"], s["labels"]
    keep = (y != IGNORE)[:, :, None]
    count = keep.sum(1).clamp(min=1).float()
    hf, wf = h.float() * keep, w.float()
    logits = torch.matmul(hf, wf.transpose(1, 2).contiguous())
    at = y.long().clamp(min=0)[:, :, None]
    top = logits.amax(2, keepdim=True)
    lse = top + (logits - top).exp().sum(2, keepdim=True).log()
    loss = ((lse - logits.gather(2, at)) * keep).sum(1) / count
    out = {"loss": loss[:, 0], "lse": (lse * keep)[:, :, 0]}
    if backward:
        p = (logits - lse).exp()
        p.scatter_add_(2, at, torch.full_like(lse, -1.0))
        p *= keep * (s["case"]["scale"] / count)[:, :, None]
        out["dh"] = torch.matmul(p, wf).to(h.dtype)
        out["dw"] = torch.matmul(p.transpose(1, 2).contiguous(), hf).to(w.dtype)
    return out


def _gates(s):
    """The gate of every row."""
    return s["gate"].float().repeat_interleave(s["case"]["gate_rows"], 1)[:, :s["x"].shape[1]]


def _norm_plain(s, backward):
    x, o, gate = s["x"].float(), s["o"].float(), _gates(s)
    pre = s["pre"][:, None, :]
    post = s["post"][:, None, :] if s["post"] is not None else 1.0
    ro = (o.square().mean(2, keepdim=True) + EPS).rsqrt() if s["post"] is not None else 1.0
    oh = o * ro
    xo = x + RES_SCALE * gate * (post * oh)
    y = pre * (xo * (xo.square().mean(2, keepdim=True) + EPS).rsqrt())
    out = {"x": xo.to(s["x"].dtype), "y": y.to(s["x"].dtype)}
    if not backward:
        return out
    xo, dy = out["x"].float(), s["dy"].float()  # the stored stream is what the backward reads
    r = (xo.square().mean(2, keepdim=True) + EPS).rsqrt()
    xh = xo * r
    a = pre * dy
    dx = s["dres"].float() + r * (a - xh * (a * xh).mean(2, keepdim=True))
    dgate = RES_SCALE * dx * post * oh
    b = RES_SCALE * gate * dx
    out["dpre"] = (dy * xh).sum(1)
    if s["post"] is not None:
        out["dpost"] = (b * oh).sum(1)
        b = post * b
        b = ro * (b - oh * (b * oh).mean(2, keepdim=True))
    k, n, d = x.shape
    rows = s["case"]["gate_rows"]
    groups = s["gate"].shape[1]
    dgate = torch.nn.functional.pad(dgate, (0, 0, 0, groups * rows - n))
    out["dgate"] = dgate.reshape(k, groups, rows, d).sum(2).to(s["gate"].dtype)
    out["dx"], out["dblock"] = dx.to(s["x"].dtype), b.to(s["o"].dtype)
    return out


def _pack_plain(x):
    """The values that x stands for in 8 bits (fp32): whole multiples, -127 to 127, of a power of two for each 32
    columns, the least that reaches the largest of them."""
    k, n, d = x.shape
    xg = torch.nn.functional.pad(x.float(), (0, -d % GROUP)).reshape(k, n, -1, GROUP)
    m, e = torch.frexp(xg.abs().amax(3, keepdim=True))
    e = e - 7 + (m > 127.0 / 128.0).int()
    e = e.clamp(min=-24 if x.dtype == torch.float16 else -126)
    q = torch.ldexp(xg, -e).round()
    return torch.ldexp(q, e).reshape(k, n, -1)[:, :, :d]


# --- one pass ----------------------------------------------------------------

def run(s):
    c = s["case"]
    op = c["op"]
    if own:
        return _run_own(s, c, op)
    if op in ("xent_step", "xent_eval"):
        return _xent_plain(s, op == "xent_step")
    if op in ("norm_step", "norm_fwd"):
        return _norm_plain(s, op == "norm_step")
    xh = _pack_plain(s["x"])
    if op == "ckpt_keep":
        return {"x": xh.to(s["x"].dtype)}
    return {"dw": torch.matmul(s["dy"].float().transpose(1, 2).contiguous(), xh).to(s["x"].dtype)}


def _run_own(s, c, op):
    import paper_1901_02244_amd as cb

    if op in ("xent_step", "xent_eval"):
        loss, lse = cb.cb_vocab_xent_fwd(s["h"], s["w"], s["labels"], ignore=IGNORE)
        out = {"loss": loss, "lse": lse}
        if op == "xent_step":
            out["dh"], out["dw"] = cb.cb_vocab_xent_bwd(s["h"], s["w"], s["labels"], lse, grad_scale=c["scale"],
                                                        ignore=IGNORE)
        return out
    if op in ("norm_step", "norm_fwd"):
        how = {"block": s["o"], "gate": s["gate"], "gate_rows": c["gate_rows"], "res_scale": RES_SCALE,
               "post": s["post"], "pre": s["pre"], "eps": EPS}
        xo, y = cb.cb_gated_norm_fwd(s["x"], **how)
        out = {"x": xo, "y": y}
        if op == "norm_step":
            g = cb.cb_gated_norm_bwd(xo, s["dy"], dres=s["dres"], **how)
            out |= {key: g[key] for key in ("dx", "dblock", "dgate", "dpre")}
            if s["post"] is not None:
                out["dpost"] = g["dpost"]
        return out
    kept = cb.cb_ckpt_pack(s["x"])
    if op == "ckpt_keep":
        return {"x": cb.cb_ckpt_unpack(kept)}
    return {"dw": cb.cb_ckpt_wgrad(kept, s["dy"])}


# --- what a pass cannot do without -------------------------------------------

def work(case):
    b = 4 if case["type"] == "fp32" else 2
    k, n, d, op = case["k"], case["n"], case["d"], case["op"]
    if op in ("xent_step", "xent_eval"):
        v, step = case["v"], op == "xent_step"
        rows = k * (n - int(n * case["ignored"] / 2))  # rows that are not padding, give or take those between
        rows = max(k, rows * (1 - case["ignored"] / 2))
        each = rows * d * b + k * v * d * b
        # each logit once for the sums and once more for the gradient, which is not kept between the two
        return {"bytes": each * (2 if step else 1) + k * n * 8, "flops": rows * d * v * (8 if step else 2)}
    if op in ("norm_step", "norm_fwd"):
        gate = -(-n // case["gate_rows"])
        step = op == "norm_step"
        # forward: x, o, x', y; backward: dy, dres, dx, dblock beside what the forward has read and written
        return {"bytes": k * d * b * ((8 if step else 4) * n + (2 if step else 1) * gate),
                "flops": k * n * d * (40 if step else 10)}
    if op == "ckpt_keep":
        return {"bytes": k * n * d * 2 * b, "flops": k * n * d * 4}
    return {"bytes": k * (n * (d + case["out"]) + d * case["out"]) * b, "flops": 2 * k * n * d * case["out"]}


# --- the definitions in 64 bits ----------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op, k = case["op"], case["k"]
    wide = {key: v.double() for key, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if op in ("xent_step", "xent_eval"):
        parts = [_xent_exact(wide["h"][j], wide["w"][j], s["labels"][j], case["scale"], op == "xent_step")
                 for j in range(k)]
        return {key: torch.stack([p[key] for p in parts]) for key in parts[0]}
    if op in ("norm_step", "norm_fwd"):
        parts = [_norm_exact({key: v[j] for key, v in wide.items()}, TYPES[case["type"]], case["gate_rows"])
                 for j in range(k)]
        return {key: torch.stack([p[key] for p in parts]) for key in parts[0]}
    parts = [_kept_exact(wide["x"][j], TYPES[case["type"]]) for j in range(k)]
    if op == "ckpt_keep":
        return {"x": torch.stack(parts)}
    return {"dw": torch.stack([torch.mm(wide["dy"][j].t().contiguous(), parts[j]) for j in range(k)])}


def _xent_exact(h, w, y, scale, backward):
    counted = torch.nonzero(y != IGNORE)[:, 0]
    hc, yc = h[counted], y[counted].long()
    logp = torch.mm(hc, w.t().contiguous())
    lse_c = torch.logsumexp(logp, 1)
    logp -= lse_c[:, None]
    rows = torch.arange(len(yc), device=h.device)
    lse = torch.zeros(len(y), dtype=torch.float64, device=h.device)
    lse[counted] = lse_c
    out = {"loss": -logp[rows, yc].sum() / max(1, len(yc)), "lse": lse}
    if backward:
        g = logp.exp_()
        g[rows, yc] -= 1.0
        g *= scale / max(1, len(yc))
        dh = torch.zeros_like(h)
        dh[counted] = torch.mm(g, w)
        out["dh"], out["dw"] = dh, torch.mm(g.t().contiguous(), hc)
    return out


def _unit(v):
    """v over its root mean square, and that root's inverse."""
    r = 1.0 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * r, r


def _unit_back(d, unit, r):
    """The gradient at v for the gradient d at _unit(v)."""
    return (d - unit * (d * unit).mean(-1, keepdim=True)) * r


def _norm_exact(s, t, gate_rows):
    n = len(s["x"])
    of = torch.arange(n, device="cuda") // gate_rows
    gate = s["gate"][of] * RES_SCALE
    if "post" in s:
        unit, r = _unit(s["o"])
        inner = unit * s["post"]
    else:
        inner = s["o"]
    x = s["x"] + gate * inner
    out = {"x": x, "y": _unit(x)[0] * s["pre"]}
    if "dy" not in s:
        return out
    xu, xr = _unit(x.to(t).double())
    dx = s["dres"] + _unit_back(s["dy"] * s["pre"], xu, xr)
    out |= {"dx": dx, "dpre": (s["dy"] * xu).sum(0)}
    out["dgate"] = torch.zeros_like(s["gate"]).index_add_(0, of, dx * inner * RES_SCALE)
    dinner = dx * gate
    if "post" in s:
        out["dpost"] = (dinner * unit).sum(0)
        dinner = _unit_back(dinner * s["post"], unit, r)
    out["dblock"] = dinner
    return out


def _kept_exact(x, t):
    n, d = x.shape
    groups = torch.zeros(n, -(-d // GROUP) * GROUP, dtype=torch.float64, device=x.device)
    groups[:, :d] = x
    groups = groups.view(n, -1, GROUP)
    most = groups.abs().max(2, keepdim=True).values
    step = torch.full_like(most, 2.0 ** (-24 if t == torch.float16 else -126))
    # 2^ceil(log2(most / 127)), put right where the logarithm is off by a rounding
    found = torch.exp2(torch.ceil(torch.log2((most / 127.0).clamp(min=1e-300))))
    found = torch.where(found * 127.0 < most, found * 2, found)
    found = torch.where(found * 63.5 >= most, found / 2, found)
    step = torch.maximum(step, found)
    return ((groups / step).round() * step).view(n, -1)[:, :d]
