"""The language-model operators through the package (GPU) against their
definitions in 64 bits, at the sizes and masks where they can go wrong."""
import pytest

import lm_oracle as ref
import paper_1901_02244_amd as cb

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
IGNORE = -100


def rand(gen, *shape, std=1.0, t=F32):
    return (torch.randn(*shape, generator=gen) * std).to(t)


def close(name, got, want):
    v, bound = want
    got = got.detach().double().cpu()
    assert got.shape == v.shape, name
    assert torch.equal(torch.isnan(got), torch.isnan(v)), f"{name}: NaN in other places"
    off = (got - v).abs().nan_to_num()
    worst = (off - bound.nan_to_num()).max().item()
    assert worst <= 0, (f"{name}: off by {off.max().item():.3e}, past its bound by {worst:.3e} "
                        f"(ratio {(off / bound.clamp(min=1e-300)).max().item():.2f})")


# --- loss over a vocabulary ---------------------------------------------------

def xent_inputs(k, n, d, v, t, pad=0.0, seed=0):
    gen = torch.Generator().manual_seed(seed + 7919 * n + 31 * d + v)
    h = rand(gen, k, n, d, t=t)
    w = rand(gen, k, v, d, std=d ** -0.5, t=t)
    y = torch.randint(0, v, (k, n), generator=gen, dtype=torch.int32)
    y[torch.rand(k, n, generator=gen) < pad] = IGNORE
    return h, w, y


def xent_check(h, w, y, scale=1.0, ignore=IGNORE, hg=None, wg=None, **how):
    hg = h.cuda() if hg is None else hg
    wg = w.cuda() if wg is None else wg
    yg = y.cuda()
    loss, lse = cb.cb_vocab_xent_fwd(hg, wg, yg, ignore=ignore)
    dh, dw = cb.cb_vocab_xent_bwd(hg, wg, yg, lse, grad_scale=scale, ignore=ignore, **how)
    torch.cuda.synchronize()
    for j in range(h.shape[0]):
        want = ref.xent(h[j], w[j], y[j], ignore, scale)
        for name, got in (("loss", loss), ("lse", lse), ("dh", dh), ("dw", dw)):
            close(f"{name}[{j}]", got[j], want[name])
    return loss, lse, dh, dw


# (k, n, d, v): single rows and words, widths that are no whole 16 bytes or no whole step, rows
# and words around every tile size (32, 128, 256), learners side by side
XENT = [
    (1, 1, 1, 1), (1, 1, 8, 2), (2, 3, 7, 5), (1, 1, 64, 1000), (8, 16, 64, 1000), (1, 31, 33, 127),
    (1, 32, 72, 129), (1, 33, 64, 257), (2, 64, 104, 255), (1, 127, 128, 130), (1, 129, 40, 513),
    (3, 65, 84, 10), (1, 257, 96, 300), (1, 300, 136, 1025),
]


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", XENT, ids=str)
def test_xent(size, t):
    scale = 256.0 if t == F16 else 1.0
    xent_check(*xent_inputs(*size, t), scale=scale)


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_xent_big_tiles(t):
    """Enough tiles of 256 by 256 for the largest shape, with ragged edges."""
    xent_check(*xent_inputs(1, 520, 72, 33000, t, pad=0.2), scale=256.0 if t == F16 else 1.0)


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_xent_ignored_rows_have_no_effect(t):
    """Rows that do not count hold NaN and infinities; one learner has none that counts."""
    h, w, y = xent_inputs(3, 70, 48, 300, t, pad=0.5)
    y[1] = IGNORE
    y[2, :69] = IGNORE
    h[y == IGNORE] = torch.nan
    h[0][y[0] == IGNORE] = torch.inf
    loss, lse, dh, dw = xent_check(h, w, y)
    assert loss[1] == 0 and (dw[1] == 0).all() and (dh[1] == 0).all() and (lse[1] == 0).all()
    assert (dh[y.cuda() == IGNORE] == 0).all()


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_xent_few_ignored_rows_read_in_place(t):
    """Up to 32 rows the forward reads h where it lies, ignored rows and all."""
    h, w, y = xent_inputs(2, 21, 64, 300, t)
    y[0, ::2] = IGNORE
    y[1] = IGNORE
    h[y == IGNORE] = torch.nan
    loss, lse, dh, dw = xent_check(h, w, y)
    assert loss[1] == 0 and (dw[1] == 0).all()


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_xent_shared_sums(t):
    """Few tiles and long sums, which workgroups share: logits over many columns, dW over many rows,
    dh over many words; rows for every kernel that adds them up."""
    scale = 256.0 if t == F16 else 1.0
    for size in ((1, 20, 1600, 40), (2, 70, 2056, 1100), (1, 1700, 48, 33), (1, 200, 1030, 700)):
        xent_check(*xent_inputs(*size, t, pad=0.3), scale=scale)


@pytest.mark.parametrize("t", [F16, BF16], ids=str)
def test_xent_past_four_gib(t):
    """600,000 words of 4096: W and dW of 4.9 GB each.  All words but the last 300 are zero, so their
    logits are 0 and their rows of dW one and the same."""
    v, d, n, m = 600000, 4096, 3, 300
    gen = torch.Generator().manual_seed(9)
    tail, h = rand(gen, m, d, std=0.05, t=t), rand(gen, 1, n, d, t=t)
    w = torch.zeros(1, v, d, dtype=t, device="cuda")
    w[0, v - m:] = tail.cuda()
    y = torch.tensor([[v - 1, v - m, 5]], dtype=torch.int32)
    loss, lse = cb.cb_vocab_xent_fwd(h.cuda(), w, y.cuda())
    dh, dw = cb.cb_vocab_xent_bwd(h.cuda(), w, y.cuda(), lse, grad_scale=4096.0)
    H, L = h[0].double(), h[0].double() @ tail.double().T
    want = torch.log((v - m) + L.exp().sum(1))
    # sums of 600,000 terms in fp32, tile by tile: 20 roundings deep at the most
    assert ((lse[0].cpu().double() - want).abs() < 1e-5).all()
    hit = torch.stack([L[0, m - 1], L[1, 0], torch.tensor(0.0).double()])
    assert abs(loss[0].item() - (want - hit).mean().item()) < 1e-5
    p = (L - want[:, None]).exp()
    g = p.clone()
    g[0, m - 1] -= 1
    g[1, 0] -= 1
    f, u = 4096.0 / n, ref.u(t)
    got, exp = dw[0, v - m:].cpu().double(), f * g.T @ H
    assert ((got - exp).abs() <= 3 * u * f * (g.abs().T @ H.abs()) + 1e-6).all()
    same = f * torch.exp(-want)[:, None].T @ H  # a zero word's row
    rest = dw[0, 6:v - m]
    assert (rest == rest[0]).all()
    assert ((rest[0].cpu().double() - same[0]).abs() <= 3 * u * f * (torch.exp(-want) @ H.abs()) + 1e-6).all()
    got, exp = dh[0].cpu().double(), f * g @ tail.double()
    assert ((got - exp).abs() <= 3 * u * f * (g.abs() @ tail.double().abs()) + 1e-5).all()


@pytest.mark.parametrize("t", [F16, BF16], ids=str)
def test_xent_few_counted_rows_of_many_words(t):
    """250 of 300,000 rows count, of 5,000,000 words: all the pieces that a launch could take together would make
    g's rows 9.6 MB apart, and 250 of those pass 2 GiB.  All words but the last 300 are zero.  (The lse is the
    test's own: a forward of as many rows and words is more than a launch holds.)"""
    n, d, v, m, c = 300000, 2304, 5000000, 300, 250
    gen = torch.Generator().manual_seed(10)
    tail = rand(gen, m, d, std=0.05, t=t)
    w = torch.zeros(1, v, d, dtype=t, device="cuda")
    w[0, v - m:] = tail.cuda()
    h = torch.zeros(1, n, d, dtype=t, device="cuda")
    y = torch.full((1, n), IGNORE, dtype=torch.int32, device="cuda")
    at = torch.arange(c) * 1199 + 7
    rows, hit = rand(gen, c, d, t=t), torch.randint(0, m, (c,), generator=gen)
    h[0, at.cuda()] = rows.cuda()
    y[0, at.cuda()] = (v - m + hit).int().cuda()
    H, W = rows.double(), tail.double()
    logits = H @ W.T
    want = torch.log((v - m) + logits.exp().sum(1))
    lse = torch.zeros(1, n, device="cuda")
    lse[0, at.cuda()] = want.float().cuda()
    dh, dw = cb.cb_vocab_xent_bwd(h, w, y, lse, grad_scale=float(c))
    g = (logits - want[:, None]).exp()
    g[torch.arange(c), hit] -= 1
    u = ref.u(t)
    # g is rounded to its type and the result once more: two of the three u.  The rest is for fp32's errors in
    # probabilities below 0.01, and 1e-7 for fp16's subnormals
    got, exp = dh[0, at.cuda()].cpu().double(), g @ W
    assert ((got - exp).abs() <= (3 * u + 1e-5) * (g.abs() @ W.abs()) + 1e-7).all()
    got, exp = dw[0, v - m:].cpu().double(), g.T @ H
    assert ((got - exp).abs() <= (3 * u + 1e-5) * (g.abs().T @ H.abs()) + 1e-7).all()
    dh[0, at.cuda()] = 0
    assert (dh == 0).all()


@pytest.mark.parametrize("t", [F32, BF16], ids=str)
def test_xent_of_more_tiles_than_a_launch_holds(t):
    """Two million rows (fp32; four in 16 bits) of 131,075 words: 2^24 tiles of 256 threads and some more (2^23 of
    512), past what one grid holds.  All words but 16 are zero; those lie at both ends."""
    n, d, v = (2 ** 21 if t == F32 else 2 ** 22) + 300, 8, 2 ** 17 + 3
    gen = torch.Generator("cuda").manual_seed(21)
    some = torch.cat([torch.arange(8), v - 8 + torch.arange(8)]).cuda()
    w = torch.zeros(1, v, d, dtype=t, device="cuda")
    w[0, some] = torch.randn(16, d, generator=gen, device="cuda").to(t)
    h = torch.randn(1, n, d, generator=gen, device="cuda").to(t)
    y = some[torch.randint(0, 16, (1, n), generator=gen, device="cuda")].int()
    loss, lse = cb.cb_vocab_xent_fwd(h, w, y)
    logits = h[0].double() @ w[0, some].double().t().contiguous()
    want = torch.log((v - 16) + logits.exp().sum(1))
    # sums of 131,075 terms in fp32, tile by tile, 20 roundings deep at the most, of logits that are off by el
    el = (d + 32) * ref.U * (h[0].double().abs() @ w[0, some].double().abs().t().contiguous()).amax(1)
    assert ((lse[0].double() - want).abs() < 1e-5 + 2 * el).all()
    hit = torch.where(y[0] < 8, y[0], y[0] - (v - 16)).long()
    rows = want - logits.gather(1, hit[:, None])[:, 0]
    assert abs(loss[0].item() - rows.mean().item()) < 1e-5 + 4 * el.mean().item()


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_xent_label_out_of_range(t):
    """As in cb_step: the learner's loss is NaN, the gradient has no one-hot term."""
    h, w, y = xent_inputs(2, 5, 24, 50, t)
    y[0, 2], y[0, 3] = 50, -1
    loss = xent_check(h, w, y)[0]
    assert torch.isnan(loss[0]) and torch.isfinite(loss[1])


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("n", [16384, 16385, 40001])
def test_xent_many_rows(n, t):
    """Rows whose labels are counted, and losses added, in chunks; one learner counts none of its first chunks."""
    h, w, y = xent_inputs(2, n, 24, 50, t, pad=0.4)
    y[1, :3000] = IGNORE
    xent_check(h, w, y)


def test_xent_other_ignored_label():
    h, w, y = xent_inputs(1, 9, 16, 20, F32)
    y[0, 4] = 0
    xent_check(h, w, y, ignore=0)


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_xent_far_logits(t):
    """Logits in the thousands: exp of none of them may overflow; certain rows have no loss."""
    h, w, y = xent_inputs(1, 40, 32, 200, t)
    h *= 200
    y[0] = (h[0].double() @ w[0].double().T).argmax(1).int()
    y[0, ::3] = 7
    xent_check(h, w, y)


def test_xent_pieces():
    """A vocabulary of several pieces (4096 words at least) at many rows."""
    n = 16640  # 16640 rows * 4 bytes * 4096 words is past the piece's 256 MB
    gen = torch.Generator().manual_seed(5)
    h, w = rand(gen, 1, n, 8), rand(gen, 1, 9001, 8, std=0.5)
    y = torch.randint(0, 9001, (1, n), generator=gen, dtype=torch.int32)
    xent_check(h, w, y)


@pytest.mark.parametrize("t", [F32, BF16], ids=str)
@pytest.mark.parametrize("d", [200, 1000])
def test_xent_pieces_of_few_counted_rows(d, t):
    """Learners that need one, two and all of the launches of a pass in pieces, and one that counts nothing."""
    k, n, v = 5, 1100, 30000
    gen = torch.Generator("cuda").manual_seed(d)
    h = torch.randn(k, n, d, generator=gen, device="cuda").to(t)
    w = (torch.randn(k, v, d, generator=gen, device="cuda") * d ** -0.5).to(t)
    y = torch.randint(0, v, (k, n), generator=gen, device="cuda", dtype=torch.int32)
    for j, part in enumerate((0.9, 0.55, 0.0, 1.0, 0.7)):
        y[j][torch.rand(n, generator=gen, device="cuda") < part] = IGNORE
    h[0][y[0] == IGNORE] = torch.nan
    loss, lse = cb.cb_vocab_xent_fwd(h, w, y)
    dh, dw = cb.cb_vocab_xent_bwd(h, w, y, lse, grad_scale=3.0)
    h[0][y[0] == IGNORE] = 0
    for j in range(k):
        want = ref.xent(h[j], w[j], y[j], IGNORE, 3.0)
        for name, got in (("loss", loss), ("lse", lse), ("dh", dh), ("dw", dw)):
            x, bound = want[name]
            close(f"{name}[{j}]", got[j], (torch.as_tensor(x).cpu(), torch.as_tensor(bound).cpu()))


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", [(1, 3, 64, 140001), (2, 5, 40, 70001), (1, 1, 16, 131073), (3, 32, 24, 90000)], ids=str)
def test_xent_few_rows_many_words(size, t):
    """More tiles of few rows than run together."""
    xent_check(*xent_inputs(*size, t))


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_xent_strides(t):
    """h a slice of wider rows, W and dW slices of flat parameter vectors, at places with and
    without 16-byte alignment; what lies between stays as it was."""
    k, n, d, v = 2, 21, 40, 77
    h, w, y = xent_inputs(k, n, d, v, t)
    for lead in (8, 3):
        wide = torch.full((k, n, d + 13), torch.nan, dtype=t, device="cuda")
        wide[:, :, 5:5 + d] = h.cuda()
        flat = torch.full((k, v * d + lead + 8), torch.nan, dtype=t, device="cuda")
        grads = torch.full_like(flat, 5.0)
        wg = flat[:, lead:lead + v * d].view(k, v, d)
        wg.copy_(w)
        xent_check(h, w, y, hg=wide[:, :, 5:5 + d], wg=wg,
                   dw=grads[:, lead:lead + v * d].view(k, v, d))
        assert (grads[:, :lead] == 5).all() and (grads[:, lead + v * d:] == 5).all()


def test_xent_gradient_by_differences():
    """dh and dw against central differences of the loss (in 64 bits)."""
    h, w, y = xent_inputs(1, 6, 10, 17, F32, pad=0.2, seed=3)
    _, lse = cb.cb_vocab_xent_fwd(h.cuda(), w.cuda(), y.cuda())
    dh, dw = cb.cb_vocab_xent_bwd(h.cuda(), w.cuda(), y.cuda(), lse)

    def loss(H, W):
        keep = y[0] != IGNORE
        return torch.nn.functional.cross_entropy((H @ W.T)[keep], y[0][keep].long())

    H, W, s = h[0].double(), w[0].double(), 1e-4
    for X, got in ((H, dh[0]), (W, dw[0])):
        for at in range(0, X.numel(), 7):
            flat = X.view(-1)
            keep = flat[at].item()
            flat[at] = keep + s
            up = loss(H, W)
            flat[at] = keep - s
            down = loss(H, W)
            flat[at] = keep
            # the central difference is off by s^2/6 times a third derivative of order one
            assert abs((up - down) / (2 * s) - got.cpu().view(-1)[at]) < 1e-6


def test_xent_repeats_bit_for_bit():
    h, w, y = (x.cuda() for x in xent_inputs(2, 300, 72, 5000, BF16, pad=0.3))
    _, lse = cb.cb_vocab_xent_fwd(h, w, y)
    first = cb.cb_vocab_xent_bwd(h, w, y, lse)
    for _ in range(3):
        assert torch.equal(cb.cb_vocab_xent_fwd(h, w, y)[1], lse)
        for a, b in zip(first, cb.cb_vocab_xent_bwd(h, w, y, lse)):
            assert torch.equal(a, b)


# --- norms around a block -------------------------------------------------------

def norm_inputs(k, n, d, gate_rows, t, post=True, pre=True, block=True, seed=0):
    gen = torch.Generator().manual_seed(seed + 101 * n + d + gate_rows)
    i = {"x": rand(gen, k, n, d, std=2.0, t=t), "block": rand(gen, k, n, d, t=t) if block else None,
         "gate": rand(gen, k, -(-n // gate_rows), d, std=0.5, t=t) if block and gate_rows else None,
         "post": 1 + rand(gen, k, d, std=0.2) if post and block else None,
         "pre": 1 + rand(gen, k, d, std=0.2) if pre else None}
    return i, rand(gen, k, n, d, std=0.3, t=t), rand(gen, k, n, d, std=0.3, t=t)


def on(i, j=None):
    f = (lambda x: x.cuda()) if j is None else (lambda x: x[j])
    return {key: None if x is None else f(x) for key, x in i.items()}


def norm_check(i, dy, dres, gate_rows, s=0.7, eps=1e-5):
    how = dict(gate_rows=max(gate_rows, 1), res_scale=s, eps=eps)
    g = on(i)
    x = g.pop("x")
    xo, y = cb.cb_gated_norm_fwd(x, **g, **how)
    dyg = dy.cuda() if i["pre"] is not None else None
    back = cb.cb_gated_norm_bwd(xo, dyg, dres=None if dres is None else dres.cuda(), **g, **how)
    torch.cuda.synchronize()
    s32, e32 = float(torch.tensor(s)), float(torch.tensor(eps))
    for j in range(dy.shape[0]):
        a = on(i, j)
        want = ref.norm_fwd(a["x"], a["block"], a["gate"], max(gate_rows, 1), s32, a["post"], a["pre"], e32)
        close(f"x[{j}]", xo[j], want["x"])
        if i["pre"] is not None:
            close(f"y[{j}]", y[j], want["y"])
        else:
            assert y is None
        want = ref.norm_bwd(xo[j].cpu(), dy[j], None if dres is None else dres[j], a["block"], a["gate"],
                            max(gate_rows, 1), s32, a["post"], a["pre"], e32)
        assert set(want) == set(back)
        for name in want:
            close(f"{name}[{j}]", back[name][j], want[name])
    return xo, y, back


# (k, n, d, gate_rows): one value, one row, widths on both sides of every worker size, odd widths,
# gate rows for one row, a few, many and all, more rows than the workers
NORM = [
    (1, 1, 1, 1), (1, 1, 64, 1), (8, 16, 64, 16), (2, 5, 65, 2), (1, 9, 127, 3), (1, 7, 256, 100),
    (3, 11, 264, 4), (1, 6, 512, 0), (2, 4, 520, 2), (1, 5, 1001, 1), (1, 3, 1032, 3), (1, 5, 2048, 2),
    (1, 3, 2056, 1), (2, 3, 4096, 2), (1, 3, 4104, 0), (1, 2, 8200, 1), (1, 3, 16384, 2),
    (1, 1500, 24, 7), (1, 2500, 72, 1), (2, 1300, 40, 600), (1, 3000, 16, 5000),
]


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", NORM, ids=str)
def test_norm(size, t):
    i, dy, dres = norm_inputs(*size, t)
    norm_check(i, dy, dres, size[3])


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("parts", [(p, q, b, r) for p in (0, 1) for q in (0, 1) for b in (0, 1) for r in (0, 1)
                                   if q or b], ids=str)
def test_norm_parts(parts, t):
    """Every choice of norm after, norm before, block and gradient of the stream."""
    post, pre, block, res = parts
    i, dy, dres = norm_inputs(2, 13, 72, 4, t, post, pre, block)
    if not pre and not res:
        return  # no gradient comes in at all: refused
    norm_check(i, dy, dres if res else None, 4 if block else 0)


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("post", [0, 1])
def test_norm_without_a_gradient(post, t):
    """Without the norm before the next block and without a gradient of the stream there is nothing to go back: the
    forward runs, the backward is refused."""
    i, dy, dres = norm_inputs(2, 13, 72, 4, t, post, False, True)
    g = on(i)
    x = g.pop("x")
    xo, y = cb.cb_gated_norm_fwd(x, **g, gate_rows=4, res_scale=0.5)
    assert y is None
    for j in range(2):
        a = on(i, j)
        close(f"x[{j}]", xo[j], ref.norm_fwd(a["x"], a["block"], a["gate"], 4, 0.5, a["post"], None, 1e-5)["x"])
    with pytest.raises(cb.CBError) as e:
        cb.cb_gated_norm_bwd(xo, **g, gate_rows=4, res_scale=0.5)
    assert e.value.code == cb.CB_EINVAL


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_norm_rows_of_zeros_and_nan(t):
    """A row of zeros has a finite norm; a row with a NaN spoils no other row."""
    i, dy, dres = norm_inputs(1, 6, 96, 1, t)
    i["x"][0, 1] = 0
    i["block"][0, 1] = 0
    i["block"][0, 2] = 0
    clean, _, _ = norm_check(i, dy, dres, 1)
    i["block"][0, 4, 3] = torch.nan
    g = on(i)
    x = g.pop("x")
    xo, y = cb.cb_gated_norm_fwd(x, **g, gate_rows=1, res_scale=0.7)
    rest = [0, 1, 2, 3, 5]
    assert torch.equal(xo[0, rest], clean[0, rest])
    assert torch.isnan(y[0, 4]).all() and torch.isfinite(y[0, rest]).all()


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_norm_unaligned_and_strided(t):
    """Activations one element off 16 bytes; gammas and their gradients in flat vectors."""
    k, n, d = 2, 7, 64
    i, dy, dres = norm_inputs(k, n, d, 1, t)
    g = on(i)

    def off(x):
        flat = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")
        return flat[1:].view(x.shape).copy_(x)

    want = norm_check(i, dy, dres, 1)
    flat = torch.full((k, 2 * d + 3), torch.nan, device="cuda")
    grads = torch.full_like(flat, 5.0)
    flat[:, 1:1 + d], flat[:, d + 2:2 * d + 2] = g["post"], g["pre"]
    how = dict(block=off(g["block"]), gate=off(g["gate"]), gate_rows=1, res_scale=0.7,
               post=flat[:, 1:1 + d], pre=flat[:, d + 2:2 * d + 2])
    xo, y = cb.cb_gated_norm_fwd(off(g["x"]), **how)
    back = cb.cb_gated_norm_bwd(off(xo), off(dy.cuda()), dres=off(dres.cuda()), **how,
                                dpost=grads[:, 1:1 + d], dpre=grads[:, d + 2:2 * d + 2])
    assert torch.equal(xo, want[0]) and torch.equal(y, want[1])
    for name in back:
        assert torch.equal(back[name], want[2][name]), name
    assert (grads[:, 0] == 5).all() and (grads[:, d + 1] == 5).all() and (grads[:, -1] == 5).all()


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", [(1, 1, 5), (2, 9, 64), (1, 5, 100), (3, 4, 777), (1, 3, 4096)], ids=str)
def test_norm_keeps_its_output(size, t):
    """keep=True gives what cb_ckpt_pack gives of y, bit for bit."""
    i, _, _ = norm_inputs(*size, 1, t)
    g = on(i)
    x = g.pop("x")
    _, y, kept = cb.cb_gated_norm_fwd(x, **g, gate_rows=1, keep=True)
    k, n, d = size
    used = k * n * -(-d // 32) * 33
    assert torch.equal(kept.data[:used], cb.cb_ckpt_pack(y).data[:used])


@pytest.mark.parametrize("parts", [(0, 1, 0), (0, 1, 1), (1, 0, 1), (1, 1, 1)], ids=str)
@pytest.mark.parametrize("size", [(4100, 1030), (2050, 4096), (1030, 9000)], ids=str)
@pytest.mark.parametrize("t", TYPES, ids=str)
def test_norm_rows_do_not_depend_on_the_call(t, size, parts):
    """A row of a long call, where several waves walk many rows together, is what it is in a call of few rows."""
    n, d = size
    gen = torch.Generator("cuda").manual_seed(31)
    post, pre, block = parts
    x, o, dy, dres = (torch.randn(1, n, d, generator=gen, device="cuda").to(t) for _ in range(4))
    gammas = {name: torch.rand(1, d, generator=gen, device="cuda") + 0.5 for name, there in (("post", post), ("pre", pre)) if there}

    def both(rows):
        how = dict(gammas, res_scale=0.5, **({"block": o[:, rows]} if block else {}))
        xo, y = cb.cb_gated_norm_fwd(x[:, rows].contiguous(), **how)
        back = cb.cb_gated_norm_bwd(xo, dy[:, rows].contiguous() if pre else None, dres=dres[:, rows].contiguous(), **how)
        return [v for v in (xo if block else None, y if pre else None, back["dx"], back.get("dblock")) if v is not None]

    whole = both(slice(0, n))
    for at in range(0, n, 205):
        for a, b in zip(whole, both(slice(at, at + 205))):
            assert torch.equal(a[:, at:at + 205], b), at


def test_norm_stream_is_the_rounded_sum():
    """x' is the sum in fp32, rounded once more to fp16: the same however the instructions were chosen."""
    gen = torch.Generator("cuda").manual_seed(32)
    x, o, g = (torch.randn(1, 500, 1001, generator=gen, device="cuda").half() for _ in range(3))
    xo, _ = cb.cb_gated_norm_fwd(x * 3, block=o, gate=g, gate_rows=1, res_scale=0.5, pre=torch.ones(1, 1001, device="cuda"))
    # the product of two fp16 numbers is exact in fp32, so that its sum with x has one rounding
    assert torch.equal(xo, ((x * 3).float() + 0.5 * (g.float() * o.float())).half())


def test_norm_gradients_by_differences():
    """Every gradient against central differences (in 64 bits) of <y, dy> + <x', dres>."""
    i, dy, dres = norm_inputs(1, 5, 12, 2, F32, seed=8)
    s, eps = 0.5, 2.0 ** -10
    _, _, back = norm_check(i, dy, dres, 2, s=s, eps=eps)
    X, O, G, P, Q = (i[name].double().clone() for name in ("x", "block", "gate", "post", "pre"))

    def value():
        xo = X[0] + s * G[0][torch.arange(5) // 2] * (P[0] * O[0] * ref.rms(O[0], eps))
        return (Q[0] * xo * ref.rms(xo, eps) * dy[0].double()).sum() + (xo * dres[0].double()).sum()

    step = 1e-5
    for wrt, name in ((X, "dx"), (O, "dblock"), (G, "dgate"), (P, "dpost"), (Q, "dpre")):
        flat, got = wrt.view(-1), back[name].double().cpu().view(-1)
        for at in range(flat.numel()):
            keep = flat[at].item()
            flat[at] = keep + step
            up = value()
            flat[at] = keep - step
            down = value()
            flat[at] = keep
            # fp32's rounding of sums of order ten, and a third derivative of order ten times step^2
            assert abs((up - down) / (2 * step) - got[at]) < 2e-5, (name, at)


def test_ckpt_wgrad_by_differences():
    """dw against differences of <unpacked W^T, dy>, which is linear in W."""
    gen = torch.Generator().manual_seed(6)
    x, dy = rand(gen, 1, 9, 40), rand(gen, 1, 9, 6)
    kept = cb.cb_ckpt_pack(x.cuda())
    dw, X = cb.cb_ckpt_wgrad(kept, dy.cuda())[0].cpu(), cb.cb_ckpt_unpack(kept)[0].cpu().double()
    w = rand(gen, 6, 40).double()

    def value(w):
        return ((X @ w.T) * dy[0].double()).sum()

    for o, c in ((0, 0), (2, 17), (5, 39), (3, 31), (4, 32)):
        e = torch.zeros_like(w)
        e[o, c] = 0.5
        assert abs(value(w + e) - value(w - e) - dw[o, c]) < 1e-5


def test_norm_and_ckpt_past_four_gib():
    """Rows past 2^32 bytes: every row is worth what it is worth in a small call."""
    n, d, m = 300000, 8192, 40
    gen = torch.Generator("cuda").manual_seed(3)
    x = torch.randint(-100, 100, (1, n, d), generator=gen, device="cuda", dtype=torch.int8).to(BF16)
    pre = torch.rand(1, d, generator=gen, device="cuda") + 0.5
    tail = x[:, n - m:].clone()
    _, y = cb.cb_gated_norm_fwd(x, pre=pre)
    assert torch.equal(y[:, n - m:], cb.cb_gated_norm_fwd(tail, pre=pre)[1])
    xo, y = cb.cb_gated_norm_fwd(x, block=x, pre=pre, post=pre, res_scale=0.5)
    to, ty = cb.cb_gated_norm_fwd(tail, block=tail, pre=pre, post=pre, res_scale=0.5)
    assert torch.equal(y[:, n - m:], ty) and torch.equal(xo[:, n - m:], to)
    how = dict(pre=pre, post=pre, res_scale=0.5)
    big = cb.cb_gated_norm_bwd(xo, y, block=x, **how)
    small = cb.cb_gated_norm_bwd(to, ty, block=tail, **how)
    assert torch.equal(big["dx"][:, n - m:], small["dx"])
    assert torch.equal(big["dblock"][:, n - m:], small["dblock"])
    del big, xo, y
    kept = cb.cb_ckpt_pack(x)
    back = cb.cb_ckpt_unpack(kept)
    assert torch.equal(back[:, n - m:], cb.cb_ckpt_unpack(cb.cb_ckpt_pack(tail)))
    del back
    dy = torch.zeros(1, n, 24, dtype=BF16, device="cuda")
    dy[:, n - m:] = 1  # only the last rows count
    dw = cb.cb_ckpt_wgrad(kept, dy)
    want = cb.cb_ckpt_unpack(cb.cb_ckpt_pack(tail)).float().sum(1)  # whole numbers: exact
    assert torch.equal(dw[0], want.expand(24, d).to(BF16))


def test_norm_in_place():
    """dx may be written over dres (through the C entry point)."""
    import ctypes

    i, dy, dres = norm_inputs(1, 50, 200, 1, BF16)
    want = norm_check(i, dy, dres, 1)
    g = on(i)
    x = g.pop("x")
    d = cb.cb_gated_norm(2, 1, 50, 200, 1, 0.7, 1e-5, g["block"].data_ptr(), g["gate"].data_ptr(),
                         g["post"].data_ptr(), g["pre"].data_ptr(), 0, 0)
    L = cb.lib()
    ws = torch.empty(L.cb_gated_norm_workspace_bytes(ctypes.byref(d)), dtype=torch.uint8, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    y = torch.empty_like(x)
    assert L.cb_gated_norm_fwd(ctypes.byref(d), x.data_ptr(), x.data_ptr(), y.data_ptr(), None, s) == 0
    assert torch.equal(x, want[0]) and torch.equal(y, want[1])
    stream, out = dres.cuda(), want[2]
    new = {name: torch.empty_like(out[name]) for name in ("dblock", "dgate", "dpost", "dpre")}
    dyg = dy.cuda()
    assert L.cb_gated_norm_bwd(ctypes.byref(d), x.data_ptr(), dyg.data_ptr(), stream.data_ptr(),
                               stream.data_ptr(), new["dblock"].data_ptr(), new["dgate"].data_ptr(),
                               new["dpost"].data_ptr(), 0, new["dpre"].data_ptr(), 0, ws.data_ptr(),
                               ws.numel(), s) == 0
    assert torch.equal(stream, out["dx"])
    for name in new:
        assert torch.equal(new[name], out[name]), name


# --- 8-bit checkpoints ------------------------------------------------------------

@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", [(1, 1, 1), (1, 3, 31), (2, 2, 32), (1, 5, 33), (3, 7, 100), (1, 2, 1000),
                                  (1, 40, 256)], ids=str)
def test_ckpt_keeps(size, t):
    gen = torch.Generator().manual_seed(size[2])
    x = rand(gen, *size, t=t) * torch.exp2(torch.randint(-9, 9, (*size[:2], 1), generator=gen)).to(t)
    x[..., ::7] *= 20
    got = cb.cb_ckpt_unpack(cb.cb_ckpt_pack(x.cuda())).cpu()
    assert got.dtype == t
    assert torch.equal(got.double().view(-1, size[2]), ref.kept(x.view(-1, size[2])))


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_ckpt_extremes(t):
    """Zeros, subnormals, ties, both sides of every step of the scale, the type's largest values,
    infinities and NaN."""
    f = torch.finfo(t)
    sub = f.smallest_normal * f.eps  # the least subnormal
    rows = [[0.0] * 32, [-0.0] * 32, [sub] * 32, [-sub, 3 * sub] * 16, [f.smallest_normal] * 32,
            [f.max] * 32, [-f.max, f.max / 2] * 16, [f.max, sub] * 16, [torch.inf] + [1.0] * 31,
            [torch.nan] * 32, [1.0] * 31 + [-torch.inf], [2.0] + [torch.nan] + [0.0] * 30]
    for e in (-20, -10, 0, 3):
        for m in (126.5, 127.0, 127.5, 128.0, 254.0, 255.0):
            rows.append([m * 2.0 ** e] + [(i + 0.5) * 2.0 ** e for i in range(-15, 16)])
    x = torch.tensor(rows).to(t)[None]
    got = cb.cb_ckpt_unpack(cb.cb_ckpt_pack(x.cuda())).cpu()[0].double()
    want = ref.kept(x[0])
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(), want.nan_to_num())
    assert not torch.isinf(got).any()


# (k, n, d, out): single rows, widths that are no whole 16 bytes, tile edges, LeNet's layers, rows
# enough to be split
WGRAD = [(1, 1, 1, 1), (1, 1, 32, 8), (8, 16, 400, 120), (2, 16, 84, 10), (1, 63, 33, 65), (1, 64, 128, 128),
         (2, 65, 129, 127), (1, 700, 96, 40), (1, 2100, 130, 258), (3, 257, 72, 7)]


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", WGRAD, ids=str)
def test_ckpt_wgrad(size, t):
    k, n, d, out = size
    gen = torch.Generator().manual_seed(n + d + out)
    x, dy = rand(gen, k, n, d, t=t), rand(gen, k, n, out, std=0.3, t=t)
    kept = cb.cb_ckpt_pack(x.cuda())
    flat = torch.full((k, out * d + 9), 5.0, dtype=t, device="cuda")
    dw = flat[:, 3:3 + out * d].view(k, out, d)
    assert cb.cb_ckpt_wgrad(kept, dy.cuda(), dw=dw) is dw
    own = cb.cb_ckpt_wgrad(kept, dy.cuda())
    assert torch.equal(own, dw)
    assert (flat[:, :3] == 5).all() and (flat[:, 3 + out * d:] == 5).all()
    for j in range(k):
        close(f"dw[{j}]", own[j], ref.wgrad(ref.kept(x[j]), dy[j])["dw"])


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_ckpt_wgrad_big_tiles(t):
    gen = torch.Generator().manual_seed(2)
    k, n, d, out = 1, 130, 4104, 4100
    x, dy = rand(gen, k, n, d, t=t), rand(gen, k, n, out, t=t)
    kept = cb.cb_ckpt_pack(x.cuda())
    dw = cb.cb_ckpt_wgrad(kept, dy.cuda())
    close("dw", dw[0], ref.wgrad(cb.cb_ckpt_unpack(kept)[0].cpu(), dy[0])["dw"])


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", [(3, 4110, 1500, 1890), (2, 4110, 2790, 3080)], ids=str)
def test_ckpt_wgrad_few_tiles_behind_many(size, t):
    """A last round of tiles whose rows are shared, of learners that start inside a round."""
    k, n, d, out = size
    gen = torch.Generator("cuda").manual_seed(5)
    x, dy = (torch.randn(k, n, w, generator=gen, device="cuda").to(t) for w in (d, out))
    kept = cb.cb_ckpt_pack(x)
    dw = cb.cb_ckpt_wgrad(kept, dy)
    values = cb.cb_ckpt_unpack(kept)
    for j in range(k):
        want, bound = ref.wgrad(values[j], dy[j])["dw"]
        close(f"dw[{j}]", dw[j], (want.cpu(), bound.cpu()))


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_ckpt_wgrad_of_nan(t):
    """A group of NaNs spoils its own 32 columns of dw and no others."""
    gen = torch.Generator().manual_seed(4)
    x, dy = rand(gen, 1, 20, 100, t=t), rand(gen, 1, 20, 30, t=t)
    clean = cb.cb_ckpt_wgrad(cb.cb_ckpt_pack(x.cuda()), dy.cuda())
    x[0, 5, 40] = torch.nan
    dw = cb.cb_ckpt_wgrad(cb.cb_ckpt_pack(x.cuda()), dy.cuda())
    assert torch.isnan(dw[0, :, 32:64]).all()
    assert torch.equal(dw[0, :, :32], clean[0, :, :32]) and torch.equal(dw[0, :, 64:], clean[0, :, 64:])


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("size", [(2, 40, 96, 40), (1, 130, 4104, 4100)], ids=str)
def test_ckpt_wgrad_of_the_largest_values(size, t):
    """Groups up to the type's largest value, zeros and small values among them, at both tile sizes: dw is the
    product of what unpacking gives."""
    k, n, d, out = size
    gen = torch.Generator().manual_seed(12)
    x, dy = rand(gen, *size[:3], t=t), rand(gen, k, n, out, std=2.0 ** -10, t=t)
    most = torch.finfo(t).max
    x[:, 0::5, 0::32], x[:, 1::5, 3::32], x[:, 2::5, 7::32], x[:, 3::5, 9::32] = most, -most, 0.6 * most, -0.3 * most
    x[:, :, 11::32] = 0
    dy[:, :, 5] = 0
    kept = cb.cb_ckpt_pack(x.cuda())
    values = cb.cb_ckpt_unpack(kept).cpu()
    assert torch.isfinite(values).all()
    dw = cb.cb_ckpt_wgrad(kept, dy.cuda())
    for j in range(k):
        close(f"dw[{j}]", dw[j], ref.wgrad(values[j], dy[j])["dw"])


@pytest.mark.parametrize("t", [F16, BF16], ids=str)
@pytest.mark.parametrize("size", [(2, 40, 96, 40), (1, 130, 4104, 4100)], ids=str)
def test_ckpt_wgrad_of_the_smallest_values(size, t):
    """Groups at the least power of two and dy of subnormal numbers count at both tile sizes."""
    k, n, d, out = size
    gen = torch.Generator().manual_seed(13)
    low, other = (2.0 ** -20, 1.0) if t == F16 else (2.0 ** -122, 2.0 ** 100)
    for sx, sy in ((low, other), (other, low / 64)):
        x, dy = rand(gen, k, n, d, std=sx, t=t), rand(gen, k, n, out, std=sy, t=t)
        kept = cb.cb_ckpt_pack(x.cuda())
        values = cb.cb_ckpt_unpack(kept).cpu()
        dw = cb.cb_ckpt_wgrad(kept, dy.cuda())
        for j in range(k):
            close(f"dw[{j}]", dw[j], ref.wgrad(values[j], dy[j])["dw"])


# --- together, streams, graphs ------------------------------------------------------

def learner_step(x, o, wo, gate, post, pre, w, y):
    """The last block's seam and the head of k learners: forward, loss, and back to the block's input
    projection, whose input was kept in 8 bits."""
    kept_o = cb.cb_ckpt_pack(o)                       # what the projection read
    block = torch.matmul(o.float(), wo.float().transpose(1, 2).contiguous()).to(x.dtype)
    how = dict(block=block, gate=gate, gate_rows=8, res_scale=0.5, post=post, pre=pre)
    xo, h, kept_h = cb.cb_gated_norm_fwd(x, **how, keep=True)
    loss, lse = cb.cb_vocab_xent_fwd(h, w, y)
    dh, dw = cb.cb_vocab_xent_bwd(h, w, y, lse, grad_scale=64.0)
    g = cb.cb_gated_norm_bwd(xo, dh, **how)
    dwo = cb.cb_ckpt_wgrad(kept_o, g["dblock"])
    return {"loss": loss, "dw": dw, "dwo": dwo, "kept": cb.cb_ckpt_unpack(kept_h), **g}, (xo, h, block)


def step_inputs(t, seed=0):
    gen = torch.Generator().manual_seed(seed)
    k, n, d, f, v = 2, 48, 64, 96, 500
    y = torch.randint(0, v, (k, n), generator=gen, dtype=torch.int32)
    y[:, -5:] = IGNORE
    return [a.cuda() for a in (rand(gen, k, n, d, t=t), rand(gen, k, n, f, t=t),
                               rand(gen, k, d, f, std=0.1, t=t), rand(gen, k, 6, d, t=t),
                               1 + rand(gen, k, d, std=0.1), 1 + rand(gen, k, d, std=0.1),
                               rand(gen, k, v, d, std=0.2, t=t), y)]


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_operators_together(t):
    """Each operator's result, on what the one before it gave, is within its own bound."""
    a = step_inputs(t)
    x, o, wo, gate, post, pre, w, y = (v.cpu() for v in a)
    got, (xo, h, block) = learner_step(*a)
    xo, h, block = xo.cpu(), h.cpu(), block.cpu()
    for j in range(2):
        head = ref.xent(h[j], w[j], y[j], IGNORE, 64.0)
        close("loss", got["loss"][j], head["loss"])
        close("dw", got["dw"][j], head["dw"])
        f = ref.norm_fwd(x[j], block[j], gate[j], 8, 0.5, post[j], pre[j], float(torch.tensor(1e-5)))
        close("x", xo[j], f["x"])
        close("h", h[j], f["y"])
        assert torch.equal(got["kept"][j].cpu().double(), ref.kept(h[j]))
        close("dwo", got["dwo"][j], ref.wgrad(ref.kept(o[j]), got["dblock"][j].cpu())["dw"])


@pytest.mark.parametrize("t", TYPES, ids=str)
def test_operators_together_gradients(t):
    """The gradients of a step, each within its own bound of what the operator before it gave: dh of the loss, then
    all five of the norm's, and the same values in the step as in calls one by one."""
    a = step_inputs(t)
    got, (xo, h, block) = learner_step(*a)
    x, o, wo, gate, post, pre, w, y = a
    _, lse = cb.cb_vocab_xent_fwd(h, w, y)
    dh, dw = cb.cb_vocab_xent_bwd(h, w, y, lse, grad_scale=64.0)
    g = cb.cb_gated_norm_bwd(xo, dh, block=block, gate=gate, gate_rows=8, res_scale=0.5, post=post, pre=pre)
    assert set(g) == {"dx", "dblock", "dgate", "dpost", "dpre"} and torch.equal(dw, got["dw"])
    for name in g:
        assert torch.equal(g[name], got[name]), name
    xo, h, block, dh, gate, post, pre, w, y = (v.cpu() for v in (xo, h, block, dh, gate, post, pre, w, y))
    for j in range(2):
        close("dh", dh[j], ref.xent(h[j], w[j], y[j], IGNORE, 64.0)["dh"])
        want = ref.norm_bwd(xo[j], dh[j], None, block[j], gate[j], 8, 0.5, post[j], pre[j], float(torch.tensor(1e-5)))
        assert set(want) == set(g)
        for name in want:
            close(f"{name}[{j}]", got[name][j], want[name])


def test_operators_on_another_stream():
    a = step_inputs(BF16)
    want = learner_step(*a)[0]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = learner_step(*a)[0]
    loss, lse = cb.cb_vocab_xent_fwd(a[0], a[6], a[7])
    s.wait_stream(torch.cuda.current_stream())
    other, lse2 = cb.cb_vocab_xent_fwd(a[0], a[6], a[7], stream=s)
    torch.cuda.synchronize()
    for name in want:
        assert torch.equal(want[name], got[name]), name
    assert torch.equal(loss, other) and torch.equal(lse, lse2)


def test_operators_in_a_graph():
    """Captured once and replayed on new inputs, with eager work between the replays."""
    a = step_inputs(BF16)
    learner_step(*a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        learner_step(*a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = learner_step(*a)[0]
    for seed in (1, 2, 3, 4):
        new = step_inputs(BF16, seed)
        want = learner_step(*new)[0]
        for to, v in zip(a, new):
            to.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for name in want:
            assert torch.equal(want[name], got[name]), (seed, name)


def test_operators_on_two_streams_at_once():
    """Calls that overlap in time, each with workspaces of its own, give what they give alone."""
    inputs = [step_inputs(BF16, seed) for seed in (5, 6)]
    want = [learner_step(*a)[0] for a in inputs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(learner_step(*inputs[i])[0])
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            for name in want[i]:
                assert torch.equal(want[i][name], g[name]), (i, name)


def test_xent_of_many_rows_in_a_graph():
    """The labels of a replay are counted anew, chunk by chunk."""
    n, d, v = 20000, 32, 300
    gen = torch.Generator("cuda").manual_seed(9)
    h = torch.randn(1, n, d, generator=gen, device="cuda").to(BF16)
    w = torch.randn(1, v, d, generator=gen, device="cuda").to(BF16)

    def labels(part):
        y = torch.randint(0, v, (1, n), generator=gen, device="cuda", dtype=torch.int32)
        return torch.where(torch.rand(1, n, generator=gen, device="cuda") < part, IGNORE, y).to(torch.int32)

    def step(y):
        loss, lse = cb.cb_vocab_xent_fwd(h, w, y)
        return (loss, lse, *cb.cb_vocab_xent_bwd(h, w, y, lse))

    y = labels(0.5)
    step(y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(y)
    for part in (0.9, 0.0, 0.3, 1.0):
        new = labels(part)
        want = step(new)
        y.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), part


def test_workspace_of_the_caller():
    """One workspace for calls in turn, filled with NaN bits before; a short one is refused."""
    import ctypes

    h, w, y = (v.cuda() for v in xent_inputs(1, 40, 64, 900, BF16, pad=0.2))
    want = cb.cb_vocab_xent_fwd(h, w, y)
    grads = cb.cb_vocab_xent_bwd(h, w, y, want[1])
    x = cb._xent("test", h, w, y, IGNORE)
    need = cb.lib().cb_vocab_xent_workspace_bytes(ctypes.byref(x), 1)
    assert need >= cb.lib().cb_vocab_xent_workspace_bytes(ctypes.byref(x), 0) > 0
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        got = cb.cb_vocab_xent_fwd(h, w, y, workspace=ws)
        assert all(torch.equal(p, q) for p, q in zip(want, got))
        ws.fill_(255)
        got = cb.cb_vocab_xent_bwd(h, w, y, want[1], workspace=ws)
        assert all(torch.equal(p, q) for p, q in zip(grads, got))
    with pytest.raises(cb.CBError) as e:
        cb.cb_vocab_xent_bwd(h, w, y, want[1], workspace=ws[:need - 256])
    assert e.value.code == cb.CB_ENOMEM


def test_package_refuses_on_the_gpu():
    """Shapes, types and strides that do not fit are refused before anything runs."""
    h, w, y = (v.cuda() for v in xent_inputs(2, 8, 16, 30, F32))
    lse = torch.zeros(2, 8, device="cuda")
    x, pre = torch.zeros(2, 8, 16, device="cuda"), torch.zeros(2, 16, device="cuda")
    kept = cb.cb_ckpt_pack(x)
    bad = [
        lambda: cb.cb_vocab_xent_fwd(h, w[:, :, :8], y),
        lambda: cb.cb_vocab_xent_fwd(h, w[:1], y),
        lambda: cb.cb_vocab_xent_fwd(h, w.half(), y),
        lambda: cb.cb_vocab_xent_fwd(h, w, y.long()),
        lambda: cb.cb_vocab_xent_fwd(h, w, y[:, :4]),
        lambda: cb.cb_vocab_xent_fwd(h, w, y.cpu()),
        lambda: cb.cb_vocab_xent_fwd(h.transpose(1, 2), w, y),
        lambda: cb.cb_vocab_xent_fwd(h.expand(2, 8, 16)[:, ::2], w, y[:, :4]),  # learners not n rows apart
        lambda: cb.cb_vocab_xent_fwd(h, w[:, ::2], y),
        lambda: cb.cb_vocab_xent_fwd(h[:, :0], w, y[:, :0]),
        lambda: cb.cb_vocab_xent_fwd(h, w, y, workspace=torch.zeros(1 << 20, device="cuda")),
        lambda: cb.cb_vocab_xent_bwd(h, w, y, lse[:, :4]),
        lambda: cb.cb_vocab_xent_bwd(h, w, y, lse, dw=torch.zeros(2, 30, 17, device="cuda")[:, :, :16]),
        lambda: cb.cb_vocab_xent_bwd(h, w, y, lse, grad_scale=float("inf")),
        lambda: cb.cb_gated_norm_fwd(x),
        lambda: cb.cb_gated_norm_fwd(x[:, ::2], pre=pre),
        lambda: cb.cb_gated_norm_fwd(x, pre=pre.half()),
        lambda: cb.cb_gated_norm_fwd(x, pre=pre[:, :8]),
        lambda: cb.cb_gated_norm_fwd(x, gate=x, pre=pre),
        lambda: cb.cb_gated_norm_fwd(x, block=x, gate=x, gate_rows=2),
        lambda: cb.cb_gated_norm_fwd(x, block=x, gate=x, gate_rows=0),
        lambda: cb.cb_gated_norm_fwd(x, block=x, keep=True),
        lambda: cb.cb_gated_norm_fwd(x, pre=pre, eps=0.0),
        lambda: cb.cb_gated_norm_fwd(torch.zeros(1, 1, 16392, device="cuda"), pre=torch.zeros(1, 16392, device="cuda")),
        lambda: cb.cb_gated_norm_bwd(x, pre=pre),
        lambda: cb.cb_gated_norm_bwd(x, dy=x, block=x),
        lambda: cb.cb_gated_norm_bwd(x, block=x),
        lambda: cb.cb_gated_norm_bwd(x, dy=x, pre=pre, dpost=pre),
        lambda: cb.cb_ckpt_pack(x[:, :, ::2]),
        lambda: cb.cb_ckpt_unpack(cb.Kept(kept.data[:-64], kept.shape, kept.dtype)),
        lambda: cb.cb_ckpt_unpack(cb.Kept(kept.data, (2, 8, 64), kept.dtype)),
        lambda: cb.cb_ckpt_wgrad(kept, x.half()),
        lambda: cb.cb_ckpt_wgrad(kept, x[:, :4]),
        lambda: cb.cb_ckpt_wgrad(kept, x, dw=torch.zeros(2, 16, 15, device="cuda")),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(cb.CBError) as e:
            f()
        assert e.value.code == cb.CB_EINVAL, i


def test_memory_of_a_given_stream():
    """A call on another stream takes none of the blocks that were just freed on the current one."""
    h, w, y = (v.cuda() for v in xent_inputs(2, 40, 64, 900, BF16, pad=0.2))
    want = cb.cb_vocab_xent_fwd(h, w, y)
    grads = cb.cb_vocab_xent_bwd(h, w, y, want[1])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()  # the inputs are there for every stream
    sizes = [v.numel() * v.element_size() for v in (*want, *grads)]
    freed = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    spans = [(v.data_ptr(), v.data_ptr() + v.numel()) for v in freed]
    del freed
    loss, lse = cb.cb_vocab_xent_fwd(h, w, y, stream=s)
    dh, dw = cb.cb_vocab_xent_bwd(h, w, y, lse, stream=s)
    for v in (loss, lse, dh, dw):
        at, end = v.data_ptr(), v.data_ptr() + v.numel() * v.element_size()
        assert all(end <= a or b <= at for a, b in spans)
    assert torch.cuda.current_stream().cuda_stream == torch.cuda.default_stream().cuda_stream
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip((*want, *grads), (loss, lse, dh, dw)))


def test_given_stream_in_a_graph():
    """Two calls beside each other in a graph, one on a stream that the caller forks and joins."""
    k, n, d, v = 2, 40, 64, 900

    def inputs(seed):
        return [x.cuda() for x in (*xent_inputs(k, n, d, v, BF16, pad=0.2, seed=seed),
                                   *xent_inputs(k, n, d, v, BF16, pad=0.4, seed=seed + 50))]

    def step(a, side=None):
        now = torch.cuda.current_stream()
        if side is not None:
            side.wait_stream(now)
        other = cb.cb_vocab_xent_fwd(*a[3:], stream=side)
        grads = cb.cb_vocab_xent_bwd(*a[3:], other[1], stream=side)
        mine = cb.cb_vocab_xent_fwd(*a[:3])
        mine_grads = cb.cb_vocab_xent_bwd(*a[:3], mine[1])
        if side is not None:
            now.wait_stream(side)
        return (*other, *grads, *mine, *mine_grads)

    a, side = inputs(1), torch.cuda.Stream()
    step(a, side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(a, side)
    for seed in (2, 3, 4, 5):
        new = inputs(seed)
        want = step(new)
        for to, x in zip(a, new):
            to.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, got)), seed
        eager = step(new, side)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, eager)), seed
