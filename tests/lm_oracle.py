"""The language-model operators in 64 bits on the CPU, with a bound on what
fp32 arithmetic and one rounding to the result's type may differ by.

Every function returns {name: (value, bound)}, elementwise.  U is half a step
of fp32 (2^-24 relative), u(t) half a step of the result's type.  A sum of m
products in fp32 is off by at most (m + 1) U times the sum of their
magnitudes, whatever the order; 32 more U cover the handful of elementary
operations before and after it."""
import torch

U = 2.0 ** -24
TINY = {torch.float64: 0.0, torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def u(t):
    return torch.finfo(t).eps / 2


def rounded(v, bound, t):
    """Adds the rounding of v to t (half a step, or half the least subnormal; past the largest
    value and half a step it rounds to infinity)."""
    bound = bound * (1 + u(t)) + u(t) * v.abs() + TINY[t] / 2
    past = v.abs() >= torch.finfo(t).max * (1 + u(t))
    return torch.where(past, torch.inf * v.sign(), v), bound


def xent(h, w, labels, ignore, scale):
    """h [n, d], w [v, d], labels [n] of one learner."""
    t = h.dtype
    n, d = h.shape
    v = w.shape[0]
    keep = labels != ignore
    count = max(1, int(keep.sum()))
    H = torch.where(keep[:, None], h.double(), 0.0)
    W = w.double()
    logits = H @ W.T
    el = (d + 32) * U * (H.abs() @ W.abs().T).amax(1)  # a row's logits
    lse = torch.logsumexp(logits, 1)
    spread = torch.softmax(logits, 1) * (lse[:, None] - logits).clamp(max=1e4)
    elz = 2 * el + (v + 64) * U + 4 * U * spread.sum(1) + 4 * U * lse.abs()
    y = labels.long()
    inside = keep & (y >= 0) & (y < v)
    at = torch.where(inside, y, 0)
    rows = lse - logits.gather(1, at[:, None])[:, 0]
    rows = torch.where(inside, rows, torch.nan)
    loss = torch.where(keep, rows, 0.0).sum() / count
    eloss = (torch.where(keep, elz + el + 4 * U * (lse.abs() + rows.nan_to_num().abs()), 0.0).sum()
             / count + 2 * U * loss.nan_to_num().abs())
    zero = torch.zeros((), dtype=torch.float64)
    out = {"loss": (loss, eloss), "lse": (torch.where(keep, lse, zero), torch.where(keep, elz, zero))}
    p = torch.where(keep[:, None], (logits - lse[:, None]).exp(), 0.0)
    g = p.clone()
    g[inside, y[inside]] -= 1.0
    # exp's argument x is rounded to fp32 (|x| U, and again in the product with log2 e), then the
    # function's own few units; g is rounded to fp32 and to its type (fp16: stored 2^14 larger)
    far = (logits - lse[:, None]).abs().clamp(max=1e4)
    # and below fp32's least normal number, 2^-126, the hardware's exp2 is 0: for x < -87.4 the
    # function is off by up to 2^-126, whatever its relative error
    eg = p * ((el + elz)[:, None] + (4 * far + 16) * U) + 2 * U * g.abs() + 2.0 ** -126
    if t != torch.float32:
        eg = eg + u(t) * (eg + g.abs()) + TINY[t] / (2 ** 15 if t == torch.float16 else 2)
    eg = torch.where(keep[:, None], eg, 0.0)
    f = abs(scale) / count
    dh, dw = scale / count * (g @ W), scale / count * (g.T @ H)
    edh = f * ((eg + (v + 32) * U * g.abs()) @ W.abs())
    edw = f * ((eg + (n + 32) * U * g.abs()).T @ H.abs())
    out["dh"], out["dw"] = rounded(dh, edh, t), rounded(dw, edw, t)
    return out


def rms(x, eps):
    return 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + eps)


def norm_fwd(x, block, gate, gate_rows, s, post, pre, eps):
    """x, block [n, d], gate [groups, d], post, pre [d] of one learner, or None."""
    t = x.dtype
    n, d = x.shape
    X = x.double()
    er = (d + 64) * U  # relative error of r(.) and the few products around it
    size = X.abs()
    if block is not None:
        o = block.double()
        g = gate.double()[torch.arange(n) // gate_rows] if gate is not None else torch.ones(1, 1).double()
        P = post.double() if post is not None else 1.0
        add = s * g * (P * (o * (rms(o, eps) if post is not None else 1.0)))
        X = X + add
        size = size + add.abs()
    ex = er * size
    out = {"x": rounded(X, ex, t)}
    if pre is not None:
        r = rms(X, eps)
        y = pre.double() * (X * r)
        # x' enters its own norm: the root mean square moves at most by the mean of |ex|
        ey = pre.double().abs() * r * (ex + X.abs() * r * r * (X.abs() * ex).mean(1, keepdim=True))
        out["y"] = rounded(y, 2 * ey + er * y.abs(), t)
    return out


def norm_bwd(xo, dy, dres, block, gate, gate_rows, s, post, pre, eps):
    t = xo.dtype
    n, d = xo.shape
    er = (d + 64) * U
    dx = dres.double() if dres is not None else torch.zeros(n, d, dtype=torch.float64)
    size = dx.abs()
    out = {}
    if pre is not None:
        X, DY = xo.double(), dy.double()
        r = rms(X, eps)
        unit, a = X * r, pre.double() * DY
        dx = dx + r * (a - unit * (a * unit).mean(1, keepdim=True))
        size = size + r * (a.abs() + unit.abs() * (a * unit).abs().mean(1, keepdim=True))
        out["dpre"] = ((DY * unit).sum(0), (n + d + 64) * U * (DY * unit).abs().sum(0))
    edx = er * size
    out["dx"] = rounded(dx, edx, t)
    if block is None:
        return out
    o = block.double()
    ro = rms(o, eps) if post is not None else 1.0
    w = o * ro
    of = torch.arange(n) // gate_rows if gate is not None else torch.zeros(n, dtype=torch.long)
    g = gate.double()[of] if gate is not None else torch.ones(n, d, dtype=torch.float64)
    P = post.double() if post is not None else torch.ones(d, dtype=torch.float64)
    if gate is not None:
        term, mag = s * dx * P * w, (s * P * w).abs() * (edx + er * dx.abs())
        dg = torch.zeros(gate.shape, dtype=torch.float64).index_add_(0, of, term)
        eg = torch.zeros(gate.shape, dtype=torch.float64).index_add_(
            0, of, mag + (n + 32) * U * term.abs())
        out["dgate"] = rounded(dg, eg, t)
    b0 = s * g * dx
    eb0 = (s * g).abs() * (edx + er * dx.abs())
    if post is not None:
        out["dpost"] = ((b0 * w).sum(0), (eb0 * w.abs() + (n + d + 64) * U * (b0 * w).abs()).sum(0))
        b, eb = b0 * P, eb0 * P.abs()
        m = (b * w).mean(1, keepdim=True)
        em = (eb * w.abs() + er * (b * w).abs()).mean(1, keepdim=True)
        do = ro * (b - w * m)
        edo = ro * (eb + w.abs() * em + 2 * er * (b.abs() + w.abs() * (b * w).abs().mean(1, keepdim=True)))
    else:
        do, edo = b0, eb0
    out["dblock"] = rounded(do, edo, t)
    return out


def kept(x):
    """What x [rows, d] stands for in 8 bits, from the definition, group by group."""
    t = x.dtype
    low = -24 if t == torch.float16 else -126
    top = 10 if t == torch.float16 else 122
    out = torch.empty(x.shape, dtype=torch.float64)
    for r in range(x.shape[0]):
        for c in range(0, x.shape[1], 32):
            part = x[r, c:c + 32].double()
            if not torch.isfinite(part).all():
                out[r, c:c + 32] = torch.nan
                continue
            most, e = float(part.abs().max()), low
            while most > 127 * 2.0 ** e:
                e += 1
            lim = 63 if e == top else 127
            out[r, c:c + 32] = (part / 2.0 ** e).round().clamp(-lim, lim) * 2.0 ** e
    return out


def wgrad(x, dy):
    """dw [out, d] for the kept values x [n, d] and dy [n, out]."""
    X, DY = x.double(), dy.double()
    return {"dw": rounded(DY.T @ X, (len(X) + 2) * U * (DY.abs().T @ X.abs()), dy.dtype)}
