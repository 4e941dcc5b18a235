"""Workspaces of the sequence operators against what the header says of them; no
GPU."""
import ctypes
import itertools

import pytest

import paper_1901_02244_amd as cb
from test_lm_seq_boundary import attn, described, distill


def attn_bytes(backward, **kw):
    need = cb.lib().cb_decay_attn_workspace_bytes(ctypes.byref(attn(**kw)), backward)
    assert need > 0, kw
    return need


@pytest.mark.parametrize("backward", [0, 1])
@pytest.mark.parametrize("starts", [None, 1 << 40])
def test_attn_workspace_is_states_and_sequences(starts, backward):
    """34 MB of segments' states at the most, with starts 68 MB and 20 bytes a sequence, and the fp32 shares of shared
    heads: from one sequence to the most that a call takes, long and short."""
    worst, bound = 0, 68_000_000 if starts else 34_000_000
    for t, k, heads, share, d, seqs, rows in itertools.product(
            (0, 2), (1, 3), (1, 2, 16), (1, 2), (16, 64, 65, 128, 129, 256), (1, 7, 1024, 1 << 20),
            (1, 130, 4096, 1 << 20)):
        n = seqs * rows
        if heads % share or k * n > 1 << 30 or k * seqs * heads > 1 << 20:
            continue
        need = attn_bytes(backward, type=t, k=k, n=n, seqs=seqs, heads=heads, kv_heads=heads // share, dk=d, dv=d,
                          ldq=heads * d, ldk=heads * d, ldv=heads * d, decay_stride=heads, starts=starts)
        shares = 2 * (k * n * heads * d * 4 + 256) if backward and share > 1 else 0
        states = need - shares - (20 * k * seqs if starts else 0)
        assert states <= bound, (t, k, heads, share, d, seqs, rows, states)
        worst = max(worst, states)
    assert worst > 0.9 * bound  # the bound is not far from what the rule takes


def test_attn_workspace_of_the_most_sequences():
    need = attn_bytes(0, k=1, n=1 << 20, seqs=1 << 20, heads=1, kv_heads=1, dk=128, dv=128, ldq=128, ldk=128, ldv=128,
                      decay_stride=1, starts=1 << 40)
    assert 70_000_000 < need <= 68_000_000 + (20 << 20)


@pytest.mark.parametrize("k, n, m", [(1, 8192, 64), (3, 1000, 1), (8, 16, 1024)])
def test_distill_workspace_is_the_losss_and_the_lists(k, n, m):
    """8 bytes a row beside the loss of labels, backward 4 and 8 for every entry, each array up to 256 bytes."""
    L, d, v = cb.lib(), 64, 1000
    size = dict(type=2, k=k, n=n, d=d, v=v, h=1 << 40, ldh=d, w=1 << 40, pstride=v * d)
    x = described(cb.cb_vocab_xent, dict(size, ignore=0, labels=1 << 40), {})
    for back, arrays in ((0, [4, 4]), (1, [4, 4 * m, 4 * m])):
        a = L.cb_vocab_xent_workspace_bytes(ctypes.byref(x), back)
        b = L.cb_vocab_distill_workspace_bytes(ctypes.byref(distill(**size, m=m)), back)
        assert b - a == sum((k * n * each + 255) // 256 * 256 for each in arrays)
