"""Where the sequence operators meet their documented bounds (GPU): operands whose
low bits all count, teachers at the ends of fp32, sequences cut in many segments
at every width, words that most of a batch holds."""
import pytest

import lm_seq_oracle as ref
import paper_1901_02244_amd as cb
from test_lm_seq_operators import (BF16, F16, F32, I32, TYPES, attn_check, attn_inputs, close, distill_check,
                                   distill_inputs, rand)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U = 2.0 ** -24


# --- attention ------------------------------------------------------------------

def cancelling(t, rows):
    """Rows of a (at column 0; 1 at column 1), b (at column 0; the last row 32 at column 1) and c: behind `rows` equal
    rows of a b c, every factor with low bits of ones and of one sign, comes one that takes nearly all of it back, so
    that the result's own rounding hides nothing.  A learner a triple."""
    # the last bits of fp16's eleven behind bf16's eight, and the last of bf16's
    values = [1 + x / 1024 for x in (7, 15, 23, 31, 39, 47, 55, 127, 255, 511, 1023)] if t == F16 else \
        [1 + x / 128 for x in (1, 3, 63, 127)]
    triples = [(x, y, z) for x in values for y in values[::3] for z in values]
    abc = torch.tensor(triples, dtype=torch.float64)
    k, n, d = len(triples), rows + 1, 8
    a, b, c = (torch.zeros(k, n, 1, d, dtype=torch.float64) for _ in range(3))
    a[:, :, 0, 0], a[:, :, 0, 1] = abc[:, :1], 1.0
    b[:, :rows, 0, 0] = abc[:, 1:2]
    b[:, rows, 0, 1] = 32.0
    c[:, :rows, 0] = abc[:, 2][:, None, None]
    total = rows * abc.prod(1)
    c[:, rows, 0] = -(total / 32).to(BF16).double()[:, None]
    out = [x.to(t) for x in (a, b, c)]
    assert all(torch.equal(x.double(), y) for x, y in zip(out, (a, b, c)))
    return out, total + 32 * c[:, rows, 0, 0], total


@pytest.mark.parametrize("t", [F16, BF16], ids=str)
@pytest.mark.parametrize("rows", [31, 32, 64, 97])
@pytest.mark.parametrize("states", [True, False])
def test_attn_every_part_of_an_operand_counts(states, rows, t):
    """In 16-bit types scores and states enter a product as two bf16 numbers, the first cut off and the second rounded:
    less than 2^-7 of the number is left for the second, whose rounding leaves out 2^-16 at the most.  Where no state
    is returned the state's own sum does the same with c: 2^-15 in all.  Nothing else but fp32 sums: of n + 8 terms
    here, each product's rounding among them, in two products; and the result's rounding."""
    (a, b, c), want, size = cancelling(t, rows)
    k, n = a.shape[:2]
    decay = torch.zeros(k, 1).cuda()
    ag, bg, cg = (x.cuda() for x in (a, b, c))
    zero = torch.zeros(k, 1, 1, 8, 8, device="cuda")
    if states:
        o, _ = cb.cb_decay_attn_fwd(ag, bg, cg, decay, keep_state=True)
        with_state = dict(state=zero, dstate=zero)
    else:
        o, with_state = cb.cb_decay_attn_fwd(ag, bg, cg, decay), {}
    got = {"o": o}
    got["dq"] = cb.cb_decay_attn_bwd(ag, cg, bg, decay, ag, **with_state)["dq"]
    back = [x.flip(1).contiguous() for x in (ag, bg, cg)]
    got["dval"] = cb.cb_decay_attn_bwd(back[1], back[0], back[2], decay, back[2], **with_state)["dval"].flip(1)
    got["dkey"] = cb.cb_decay_attn_bwd(back[2], back[2], back[0], decay, back[1], **with_state)["dkey"].flip(1)
    bound = size * (2.0 ** (-16 if states else -15) + 4 * (n + 8) * U) + torch.finfo(t).eps / 2 * want.abs()
    for name, x in got.items():
        close(name, x[:, rows, 0], (want[:, None].expand(k, 8), bound[:, None].expand(k, 8)))


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("width", [(128, 128), (96, 128), (256, 256), (130, 200)], ids=str)
def test_attn_uneven_sequences_in_many_segments(width, t):
    """Uneven sequences of three to nine segments, whose states are carried from one to the next, for heads past 64
    and past 128 columns."""
    k, n, heads = 2, 1300, 2
    q, key, val, decay, dout, gen = attn_inputs(k, n, heads, 1, *width, t, fused=True)
    decay = decay * 0.02  # a segment's state reaches over the next ones
    starts = torch.tensor([[0, 3, 40, 1200, 1290], [10, 10, 500, 501, 1300]], dtype=I32)
    state, dstate = rand(gen, k, 4, heads, *width), rand(gen, k, 4, heads, *width)
    attn_check(q, key, val, decay, dout, scale=1.0 / 16, starts=starts, state=state, dstate=dstate)
    attn_check(q, key, val, decay, dout, scale=1.0 / 16, starts=starts)


# --- distillation ---------------------------------------------------------------

@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("temp", [0.5, 1.0, 4.0])
def test_distill_teachers_at_the_ends_of_fp32(temp, t):
    """Logits masked with fp32's lowest value, or at its largest: shares depend on differences only, so rows of them
    alone are rows of equal logits, and beside others the lowest have none."""
    h, w, words, teacher = distill_inputs(2, 40, 32, 60, 6, t)
    words = words.abs()
    low, high = torch.finfo(F32).min, torch.finfo(F32).max
    ends, plain = teacher.clone(), teacher.clone()
    ends[:, 0::4], plain[:, 0::4] = low, 0.0
    ends[:, 1::4], plain[:, 1::4] = high, 0.0
    ends[:, 2::4, 1:4], plain[:, 2::4, 1:4] = low, -1e5
    ends[:, 3::4, 2], plain[:, 3::4, 2] = high, 1e5
    what = (h.cuda(), w.cuda(), words.cuda())
    results = []
    for x in (ends, plain):
        loss, lse, picked = cb.cb_vocab_distill_fwd(*what, x.cuda(), temperature=temp)
        results.append((loss, lse, picked, *cb.cb_vocab_distill_bwd(*what, x.cuda(), lse, picked, temperature=temp)))
    for a, b in zip(*results):
        assert a.isfinite().all() and torch.equal(a, b)
    for j in range(2):
        want = ref.distill(h[j], w[j], words[j], plain[j], temp, 1.0)
        for name, got in zip(("loss", "lse", "picked", "dh", "dw"), results[0]):
            close(name, got[j], want[name])


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_distill_teachers_without_a_softmax(bad, t):
    """A logit that counts and is NaN or infinite: the learner's loss, its row's dh and its words' dW are NaN, also
    where all of a row's logits are; nothing else is."""
    h, w, words, teacher = distill_inputs(3, 40, 32, 4000, 6, t)
    teacher[0, 3, 2], words[0, 3, 2] = bad, 17
    teacher[2, 5], words[2, 5, 0] = bad, 3
    words[2, 5, 1:] = -1
    loss, *_ = distill_check(h, w, words, teacher)
    assert loss[0].isnan() and not loss[1].isnan() and loss[2].isnan()


def test_distill_repeats_bit_for_bit():
    h, w, words, teacher = (x.cuda() for x in distill_inputs(2, 300, 96, 3000, 9, BF16))
    first = None
    for _ in range(3):
        loss, lse, picked = cb.cb_vocab_distill_fwd(h, w, words, teacher, temperature=2.0)
        got = [loss, lse, picked, *cb.cb_vocab_distill_bwd(h, w, words, teacher, lse, picked, temperature=2.0)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))


# --- embedding ------------------------------------------------------------------

def pass_us(f):
    """Median time of f in a graph."""
    f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f()
    times = []
    for _ in range(9):
        a, b = torch.cuda.Event(True), torch.cuda.Event(True)
        a.record()
        for _ in range(4):
            graph.replay()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 250)
    return sorted(times)[4]


def test_embed_zeros_take_no_longer_for_frequent_words():
    """The zeros of few words are a handful of stores, however often the words occur: a call that writes them takes
    less than twice one that adds to a gradient and writes none."""
    gen = torch.Generator().manual_seed(1)
    n, d, v = 1 << 20, 8, 64
    tok, dy = torch.randint(0, v - 1, (1, n), generator=gen, dtype=I32).cuda(), rand(gen, 1, n, d).cuda()
    dw = torch.zeros(1, v, d, device="cuda")
    zeros = pass_us(lambda: cb.cb_embed_bwd(dy, tok, dw=dw))
    assert (dw[0, v - 1] == 0).all()
    adds = pass_us(lambda: cb.cb_embed_bwd(dy, tok, dw=dw, accumulate=True))
    assert zeros < 2 * adds, (zeros, adds)


@pytest.mark.parametrize("t", TYPES, ids=str)
@pytest.mark.parametrize("v", [3, 64, 65, 200])
def test_embed_frequent_words_beside_words_that_no_token_names(v, t):
    """A stretch of words whose tokens are more than one step of the search, with gaps before, between and behind; a
    learner whose every token is the last word, one whose every token is the first."""
    gen = torch.Generator().manual_seed(v)
    n, d = 3000, 8
    tok = (torch.randint(0, (v + 2) // 3, (4, n), generator=gen) * 3).clamp(max=v - 1).to(I32)
    tok[1], tok[2] = v - 1, 0
    tok[3, 1500:] = -100
    dy = rand(gen, 4, n, d, t=t)
    dw = cb.cb_embed_bwd(dy.cuda(), tok.cuda(), v)
    for j in range(4):
        close(f"dw[{j}]", dw[j], ref.embed_bwd(dy[j], tok[j], v, 1.0, -100))
