"""What the language-model operators refuse, on the host: every check is made
before any device is touched, so these run without a GPU, on addresses that
are never followed."""
import ctypes

import pytest

import paper_1901_02244_amd as cb

torch = pytest.importorskip("torch")

A = 1 << 40  # an aligned address
BIG = 1 << 44


def _err():
    return cb.lib().cb_last_error(None).decode()


def xent(**kw):
    f = dict(type=2, k=2, n=16, d=64, v=1000, ignore=-100, h=A, ldh=64, w=A, pstride=64000, labels=A)
    f.update(kw)
    return cb.cb_vocab_xent(*(f[name] for name, _ in cb.cb_vocab_xent._fields_))


XENT_WRONG = [dict(type=3), dict(type=-1), dict(k=0), dict(n=0), dict(d=0), dict(v=0), dict(k=70000),
              dict(n=1 << 30, k=2), dict(d=(1 << 20) + 1), dict(h=None), dict(w=None), dict(labels=None),
              dict(h=A + 1), dict(w=A + 1), dict(labels=A + 2), dict(ldh=63), dict(pstride=63999),
              dict(k=-1), dict(n=-5), dict(v=1 << 30, n=1 << 20)]


@pytest.mark.parametrize("kw", XENT_WRONG, ids=str)
def test_xent_refuses(kw):
    L, x = cb.lib(), xent(**kw)
    assert L.cb_vocab_xent_workspace_bytes(ctypes.byref(x), 0) == 0
    assert L.cb_vocab_xent_workspace_bytes(ctypes.byref(x), 1) == 0
    assert L.cb_vocab_xent_fwd(ctypes.byref(x), A, A, A, BIG, None) == cb.CB_EINVAL
    assert _err().startswith("cb_vocab_xent_fwd: ")
    assert L.cb_vocab_xent_bwd(ctypes.byref(x), A, 1.0, A, A, 64000, A, BIG, None) == cb.CB_EINVAL
    assert _err().startswith("cb_vocab_xent_bwd: ")


def test_xent_refuses_outputs():
    L, x = cb.lib(), xent()
    r = ctypes.byref(x)
    need = [L.cb_vocab_xent_workspace_bytes(r, b) for b in (0, 1)]
    assert min(need) > 0
    E, M = cb.CB_EINVAL, cb.CB_ENOMEM
    fwd, bwd = L.cb_vocab_xent_fwd, L.cb_vocab_xent_bwd
    assert fwd(None, A, A, A, BIG, None) == E and L.cb_vocab_xent_workspace_bytes(None, 0) == 0
    assert fwd(r, None, A, A, BIG, None) == E and fwd(r, A, None, A, BIG, None) == E
    assert fwd(r, A, A, None, BIG, None) == E and fwd(r, A, A, A + 128, BIG, None) == E
    assert fwd(r, A, A, A, need[0] - 1, None) == M and "workspace" in _err()
    assert bwd(r, A, 1.0, A, A, 64000, A, need[1] - 1, None) == M
    assert bwd(r, None, 1.0, A, A, 64000, A, BIG, None) == E
    assert bwd(r, A, float("nan"), A, A, 64000, A, BIG, None) == E
    assert bwd(r, A, 1.0, None, A, 64000, A, BIG, None) == E
    assert bwd(r, A, 1.0, A, None, 64000, A, BIG, None) == E
    assert bwd(r, A, 1.0, A, A + 1, 64000, A, BIG, None) == E
    assert bwd(r, A, 1.0, A, A, 63999, A, BIG, None) == E
    assert bwd(r, A, 1.0, A, A, 64000, A + 8, BIG, None) == E


def test_xent_workspace_holds_no_logits():
    """128,000 words: the backward's workspace stays at its piece, whatever the vocabulary; a copy of
    W only where its rows do not start on 16 bytes."""
    L = cb.lib()
    one = lambda **kw: L.cb_vocab_xent_workspace_bytes(ctypes.byref(xent(k=1, n=8192, d=4096, ldh=4096, **kw)), 1)
    piece = 1 << 28
    assert one(v=128000) < piece + 3 * 8192 * 4096 * 4
    assert one(v=128000) == one(v=64000)
    assert one(v=128000, w=A + 2) > one(v=128000) + 128000 * 4096 * 2 - 1


def norm(**kw):
    f = dict(type=2, k=2, n=16, d=64, gate_rows=4, res_scale=1.0, eps=1e-5, block=A, gate=A, post=A, pre=A,
             post_stride=64, pre_stride=64)
    f.update(kw)
    return cb.cb_gated_norm(*(f[name] for name, _ in cb.cb_gated_norm._fields_))


NORM_WRONG = [dict(type=3), dict(k=0), dict(n=0), dict(d=0), dict(d=16385), dict(n=1 << 30),
              dict(res_scale=float("inf")), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")),
              dict(block=None), dict(block=None, gate=None), dict(block=None, post=None),
              dict(block=None, gate=None, post=None, pre=None), dict(gate_rows=0), dict(gate_rows=-1),
              dict(block=A + 1), dict(gate=A + 1), dict(post=A + 2), dict(pre=A + 2), dict(post_stride=63),
              dict(pre_stride=63)]


@pytest.mark.parametrize("kw", NORM_WRONG, ids=str)
def test_norm_refuses(kw):
    L, g = cb.lib(), norm(**kw)
    assert L.cb_gated_norm_workspace_bytes(ctypes.byref(g)) == 0
    assert L.cb_gated_norm_fwd(ctypes.byref(g), A, A, A, None, None) == cb.CB_EINVAL
    assert L.cb_gated_norm_bwd(ctypes.byref(g), A, A, A, A, A, A, A, 64, A, 64, A, BIG, None) == cb.CB_EINVAL
    assert _err().startswith("cb_gated_norm_bwd: ")


def test_norm_refuses_tensors():
    L, E = cb.lib(), cb.CB_EINVAL
    g = norm()
    r = ctypes.byref(g)
    need = L.cb_gated_norm_workspace_bytes(r)
    assert need > 0
    fwd = L.cb_gated_norm_fwd
    assert fwd(r, None, A, A, None, None) == E and fwd(r, A, None, A, None, None) == E
    assert fwd(r, A, A, None, None, None) == E and fwd(r, A, A, A, A + 8, None) == E
    no_pre = norm(pre=None)
    assert fwd(ctypes.byref(no_pre), A, A, None, A, None) == E  # 8 bits of nothing
    args = [A, A, A, A, A, A, A, 64, A, 64, A, need, None]

    def bwd(d, at, v):
        a = list(args)
        a[at] = v
        return L.cb_gated_norm_bwd(ctypes.byref(d), *a)

    for at in (0, 1, 3, 4, 5, 6, 8, 10):  # every buffer but dres is needed here
        assert bwd(g, at, None) == E, at
    for at in (0, 1, 2, 3, 4, 5, 6, 8, 10):
        assert bwd(g, at, A + 1) == E, at
    assert bwd(g, 7, 63) == E and bwd(g, 9, 63) == E
    assert bwd(g, 11, need - 1) == cb.CB_ENOMEM
    assert bwd(no_pre, 2, A) == E  # dy without pre
    a = list(args)
    a[1] = a[2] = None
    assert L.cb_gated_norm_bwd(ctypes.byref(no_pre), *a) == E  # no gradient comes in


def test_ckpt_refuses():
    L, E = cb.lib(), cb.CB_EINVAL
    assert L.cb_ckpt_bytes(0, 32) == 0 and L.cb_ckpt_bytes(4, 0) == 0 and L.cb_ckpt_bytes(1, 1 << 21) == 0
    assert L.cb_ckpt_bytes((1 << 30) + 1, 1) == 0
    assert L.cb_ckpt_bytes(3, 33) >= 3 * 66
    for f in (L.cb_ckpt_pack, L.cb_ckpt_unpack):
        assert f(3, 4, 32, A, A, None) == E and f(0, 0, 32, A, A, None) == E and f(0, 4, 0, A, A, None) == E
        assert f(0, 4, 32, None, A, None) == E and f(0, 4, 32, A, None, None) == E
    assert L.cb_ckpt_pack(2, 4, 32, A + 1, A, None) == E and L.cb_ckpt_pack(2, 4, 32, A, A + 8, None) == E
    assert L.cb_ckpt_unpack(2, 4, 32, A + 8, A, None) == E and L.cb_ckpt_unpack(2, 4, 32, A, A + 1, None) == E
    size, w = L.cb_ckpt_wgrad_workspace_bytes, L.cb_ckpt_wgrad
    need = size(2, 2, 16, 64, 32, A)
    assert need > 0
    for bad in ((3, 2, 16, 64, 32), (2, 0, 16, 64, 32), (2, 2, 0, 64, 32), (2, 2, 16, 0, 32), (2, 2, 16, 64, 0),
                (2, 2, 16, (1 << 20) + 1, 32), (2, 2, 16, 64, (1 << 20) + 1), (2, 2, 1 << 30, 64, 32)):
        assert size(*bad, A) == 0
        assert w(*bad, A, A, A, 1 << 30, A, BIG, None) == E
    # a copy of dy only where its rows do not start on 16 bytes
    assert size(2, 1, 64, 64, 4096, A + 2) - size(2, 1, 64, 64, 4096, A) >= 64 * 4096 * 2 - 256
    ok = (2, 2, 16, 64, 32)
    assert w(*ok, None, A, A, 2048, A, BIG, None) == E and w(*ok, A, None, A, 2048, A, BIG, None) == E
    assert w(*ok, A, A, None, 2048, A, BIG, None) == E and w(*ok, A, A, A, 2047, A, BIG, None) == E
    assert w(*ok, A, A, A, 2048, A + 64, BIG, None) == E
    assert w(*ok, A, A, A, 2048, A, need - 1, None) == cb.CB_ENOMEM


def test_package_refuses_cpu_and_misshapen_tensors():
    """The package checks shapes, types and places before it calls the library."""
    z = torch.zeros
    i = z(1, 4, dtype=torch.int32)
    bad = [
        lambda: cb.cb_vocab_xent_fwd(z(1, 4, 8), z(1, 9, 8), i),  # not on a GPU
        lambda: cb.cb_vocab_xent_fwd(z(1, 4, 8, dtype=torch.float64), z(1, 9, 8), i),
        lambda: cb.cb_vocab_xent_fwd(z(4, 8), z(9, 8), i),
        lambda: cb.cb_vocab_xent_bwd(z(1, 4, 8), z(1, 9, 8), i, z(1, 4)),
        lambda: cb.cb_gated_norm_fwd(z(1, 4, 8), pre=z(1, 8)),
        lambda: cb.cb_gated_norm_fwd(z(4, 8), pre=z(1, 8)),
        lambda: cb.cb_gated_norm_fwd(z(1, 0, 8), pre=z(1, 8)),
        lambda: cb.cb_gated_norm_bwd(z(1, 4, 8), dy=z(1, 4, 8), pre=z(1, 8)),
        lambda: cb.cb_ckpt_pack(z(1, 4, 8)),
        lambda: cb.cb_ckpt_pack(z(1, 4, 8, dtype=torch.int32)),
        lambda: cb.cb_ckpt_wgrad(cb.Kept(z(64, dtype=torch.uint8), (1, 4, 8), torch.float32), z(1, 4, 3)),
        lambda: cb.cb_ckpt_unpack(cb.Kept(z(64, dtype=torch.uint8), (1, 4, 8), torch.float32)),
    ]
    for f in bad:
        with pytest.raises(cb.CBError) as e:
            f()
        assert e.value.code == cb.CB_EINVAL


def test_package_refuses_what_32_bits_do_not_hold():
    """The library's sizes and labels are 32-bit: larger ones are refused, not taken modulo 2^32."""
    big = 2 ** 32 + 4

    def m(*shape, t=torch.float32):
        return torch.empty(*shape, dtype=t, device="meta")

    i, z = torch.int32, m(1, 4, 8)
    kept = cb.Kept(torch.zeros(1 << 10, dtype=torch.uint8), (1, 4, 8), torch.float32)
    bad = [
        lambda: cb.cb_vocab_xent_fwd(z, m(1, 9, 8), m(1, 4, t=i), ignore=2 ** 32 - 100),
        lambda: cb.cb_vocab_xent_fwd(z, m(1, 9, 8), m(1, 4, t=i), ignore=-2 ** 31 - 1),
        lambda: cb.cb_vocab_xent_bwd(z, m(1, 9, 8), m(1, 4, t=i), m(1, 4), ignore=2 ** 31),
        lambda: cb.cb_vocab_xent_fwd(m(1, big, 1), m(1, 9, 1), m(1, big, t=i)),
        lambda: cb.cb_vocab_xent_fwd(m(1, 4, 1), m(1, big, 1), m(1, 4, t=i)),
        lambda: cb.cb_vocab_xent_fwd(m(1, 4, big), m(1, 9, big), m(1, 4, t=i)),
        lambda: cb.cb_vocab_xent_fwd(m(big, 1, 1), m(big, 1, 1), m(big, 1, t=i)),
        lambda: cb.cb_gated_norm_fwd(m(1, big, 8), pre=m(1, 8)),
        lambda: cb.cb_gated_norm_fwd(m(1, 4, big), pre=m(1, big)),
        lambda: cb.cb_gated_norm_bwd(m(1, big, 8), dy=m(1, big, 8), pre=m(1, 8)),
        lambda: cb.cb_ckpt_pack(m(1, 4, big)),
        lambda: cb.cb_ckpt_unpack(cb.Kept(kept.data, (1, 4, big), torch.float32)),
        lambda: cb.cb_ckpt_wgrad(cb.Kept(kept.data, (1, big, 8), torch.float32), m(1, big, 3)),
        lambda: cb.cb_ckpt_wgrad(kept, m(1, 4, big)),
    ]
    for n, f in enumerate(bad):
        with pytest.raises(cb.CBError, match="32 bits") as e:
            f()
        assert e.value.code == cb.CB_EINVAL, n


def test_last_error_of_another_thread():
    """Without a context there is one last failure, whichever thread made the call: one thread may create and another
    report."""
    import threading

    L = cb.lib()
    m = cb.model("lenet5", 1, 28, 28, 10)
    out = ctypes.c_void_p()

    def create():
        P = cb.cb_num_params(m)
        w0 = (ctypes.c_float * P)()
        assert L.cb_create(ctypes.byref(m), 2, 4, 0.5, 0.01, 0.9, w0, P, A, 256, None,
                           ctypes.byref(out)) == cb.CB_ENOMEM

    assert L.cb_vocab_xent_fwd(None, A, A, A, BIG, None) == cb.CB_EINVAL and "cb_vocab_xent_fwd" in _err()
    t = threading.Thread(target=create)
    t.start()
    t.join()
    assert "workspace" in _err() and "cb_vocab_xent_fwd" not in _err()


def test_last_error_of_many_threads():
    """Threads that fail and read at the same time: every message is a whole one."""
    import threading

    L, seen = cb.lib(), [set() for _ in range(8)]

    def work(i):
        bad = [xent(n=0), xent(ldh=63), xent(h=None), xent(pstride=3)][i % 4]
        for _ in range(2000):
            L.cb_vocab_xent_fwd(ctypes.byref(bad), A, A, A, BIG, None)
            L.cb_vocab_xent_bwd(ctypes.byref(bad), A, 1.0, A, A, 64000, A, BIG, None)
            seen[i].add(_err())

    threads = [threading.Thread(target=work, args=(i,)) for i in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    why = ["k or n out of range", "ldh is less than d", "h, w or labels NULL or misaligned", "pstride is less than v * d"]
    assert set().union(*seen) <= {f"cb_vocab_xent_{f}: {w}" for f in ("fwd", "bwd") for w in why}


# (description, forward fits, backward fits): a launch has fewer than 2^32 threads along its grid's first axis
XENT_GRIDS = [
    # 2^24 tiles of 128 x 128, 256 threads each, and 2^23 of 256 x 256, 512 each: the loss takes several launches
    (dict(type=0, k=1, n=1 << 19, v=1 << 19), True, True),
    (dict(type=2, k=1, n=1 << 20, v=1 << 19), True, True),
    (dict(k=1, n=1 << 29, v=10), False, False),  # 32 rows a workgroup of 256
    (dict(k=1, n=(1 << 29) - 32, v=10), True, True),
    (dict(type=0, k=1, n=1 << 26, v=5000), True, False),  # 32 tiles of the piece's 4096 words, 2^19 of its rows
    (dict(type=0, k=1, n=(1 << 26) - 2048, v=4096), True, True),
    (dict(k=65535, n=1, d=1 << 20, ldh=1 << 20, v=1, pstride=1 << 20), True, False),  # 2^13 columns' tiles of dW
    # 2^12 tiles of dh and 2^13 of dW a learner, in one launch: 2^24 / 12,288 is 1365
    (dict(k=1366, n=1, d=1 << 20, ldh=1 << 20, v=1, pstride=1 << 20), True, False),
    (dict(k=1365, n=1, d=1 << 20, ldh=1 << 20, v=1, pstride=1 << 20), True, True),
]


@pytest.mark.parametrize("kw, forward, backward", XENT_GRIDS, ids=str)
def test_xent_refuses_what_a_launch_does_not_hold(kw, forward, backward):
    """Before anything has run, and not by a launch that fails behind others."""
    L, x = cb.lib(), xent(**kw)
    r = ctypes.byref(x)
    assert (L.cb_vocab_xent_workspace_bytes(r, 0) > 0) == forward
    assert (L.cb_vocab_xent_workspace_bytes(r, 1) > 0) == backward
    if not forward:
        assert L.cb_vocab_xent_fwd(r, A, A, A, BIG, None) == cb.CB_EINVAL and "launch" in _err()
    if not backward:
        assert L.cb_vocab_xent_bwd(r, A, 1.0, A, A, x.pstride, A, BIG, None) == cb.CB_EINVAL and "launch" in _err()


def test_ckpt_wgrad_refuses_what_a_launch_does_not_hold():
    L = cb.lib()
    for size, fits in (((0, 2048, 1, 1 << 20, 1), False), ((0, 2047, 1, 1 << 20, 1), True),
                       ((2, 65535, 1, 1 << 20, 1 << 20), False), ((2, 4096, 1, 1 << 20, 1), False),
                       ((2, 2040, 1, 1 << 20, 1), True)):
        assert (L.cb_ckpt_wgrad_workspace_bytes(*size, A) > 0) == fits, size
        if not fits:
            stride = size[3] * size[4]
            assert L.cb_ckpt_wgrad(*size, A, A, A, stride, A, BIG, None) == cb.CB_EINVAL and "launch" in _err()


def test_xent_workspace_of_a_piece():
    """The backward's workspace is its piece of 128 MB, the gathered rows, fp32 sums of dh and a few numbers a row."""
    L = cb.lib()

    def one(**kw):
        return L.cb_vocab_xent_workspace_bytes(ctypes.byref(xent(k=1, n=8192, d=4096, ldh=4096, **kw)), 1)

    assert (1 << 27) < one(v=128000) <= (1 << 27) + 8192 * 4096 * (2 + 4) + 8192 * 12 + 16 * 256
    assert one(v=128000) == one(v=64000)


SHARED = [(512, 4096, 2048), (128, 1 << 20, 100), (1, 1 << 16, 1), (20, 1600, 40), (300, 20000, 5000), (64, 8192, 30000),
          (40000, 16384, 100), (33, 1 << 20, 256), (129, 1 << 18, 129)]


@pytest.mark.parametrize("type", [0, 1, 2])
@pytest.mark.parametrize("k", [1, 3])
@pytest.mark.parametrize("size", SHARED, ids=str)
def test_xent_workspace_of_shared_logits(size, k, type):
    """Where few tiles share long sums the workspace also holds the shares' logits: 64 MB at the most."""
    n, d, v = size
    x = xent(type=type, k=k, n=n, d=d, ldh=d, v=v, pstride=d * v)
    got = cb.lib().cb_vocab_xent_workspace_bytes(ctypes.byref(x), 0)
    bytes_of = 4 if type == 0 else 2
    cap, dp = -(-n // 64) * 64, -(-d * bytes_of // 128) * 128
    rows = k * cap * dp + k * n * 8 + k * cap * 12 + 12 * 256  # the gathered rows, and a few numbers each
    copy = 0 if d * bytes_of % 16 == 0 else k * v * dp + 256
    parts = k * cap * 8 * -(-v // 16)  # a pair for a tile's words, 16 at the least
    assert 0 < got <= rows + copy + parts + (64 << 20)
