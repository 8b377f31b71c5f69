"""Sequences past a call's max_len and max_rows, row starts and lengths out of order."""
import copy

import pytest
import torch

import paper_2512_21835_amd as P
from tests import ops_oracle as O
from tests.test_gpu_ops import _append_case, _check_append, _run_append, _run_window, _window_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["fp32", "bf16"])
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,held,hq,hkv", [([1, 1, 1], [60, 300, 20], 8, 2), ([37, 1, 70, 30], [30, 60, 200, 0], 8, 2),
                                              ([37, 1, 70, 30], [30, 60, 200, 0], 72, 9)])
def test_window_of_sequences_past_max_len(rows, held, hq, hkv, cache, act):
    """Tokens from max_len on are not seen, by rows of positions past it neither; a window of 0 or beyond max_len still
    reaches back to the first token."""
    b, q, out = c = _window_case(rows, held, hq, hkv, 64, act, cache)
    b.max_len = 48
    seen = copy.copy(b)
    seen.table = b.table.clone()
    seen.table[:, 3:] = -7                     # the oracle: blocks that lead nowhere
    for window, sinks in ((0, 0), (60, 0), (100, 3), (20, 5), (1 << 30, 0), ((1 << 31) - 1, 2)):
        got = _run_window(c, window, sinks)
        want, off32, off16 = O.window(seen, q, out, b.pool, hq, window, sinks)
        off = off32 + off16 if act == "bf16" else off32
        O.assert_within(got, want, O.rounded(want, off, q.dtype), (window, sinks))


@pytest.mark.parametrize("hq,hkv", [(8, 2), (72, 9)])
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
def test_window_of_more_rows_than_max_rows(hq, hkv, cache):
    """The rows beyond keep what out holds; the others are as with all of them."""
    b, q, out = c = _window_case([37, 1, 70, 30], [30, 60, 200, 0], hq, hkv, 64, "fp32", cache)
    b.max_rows = 32
    got = _run_window(c, 40, 2)
    want, off32, _ = O.window(b, q, out, b.pool, hq, 40, 2)
    for i, n in enumerate(b.rows):
        at = int(b.start[i])
        want[at + 32:at + n], off32[at + 32:at + n] = out[at + 32:at + n], 0
        assert torch.equal(got[at + 32:at + n].cpu(), out[at + 32:at + n])
    O.assert_within(got, want, O.rounded(want, off32, torch.float32))


def test_append_past_max_len():
    c = _append_case([20, 6, 40], [10, 60, 20], 4, 2, 64)
    c[0].max_len = 48
    _check_append(c, *_run_append(c))


@pytest.mark.parametrize("length", [-1, -5, -(1 << 31), -(1 << 31) + 3])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (72, 9)])
def test_lengths_below_zero_hold_nothing(length, hq, hkv):
    b, q, out = c = _window_case([30, 40, 60], [20, 0, 33], hq, hkv, 64, "fp32", "bf16")
    b.lengths[1] = 0                           # (the oracle: as many tokens)
    b.length[1] = length
    got = _run_window(c, 0, 16)
    want, off32, _ = O.window(b, q, out, b.pool, hq, 0, 16)
    assert not bool(got[30:70].any())
    O.assert_within(got, want, O.rounded(want, off32, torch.float32))
    c = _append_case([30, 40, 60], [20, 0, 33], 8, 2, 64)
    c[0].lengths[1] = 0
    c[0].length[1] = length
    _check_append(c, *_run_append(c))


def test_rows_before_the_first_row_start_are_nobodys():
    """row_start from 3: the rows before it, as those behind the last, change nothing."""
    b, qkv, q, cos, sin, gains, _, _, eps = _append_case([5, 4], [12, 30], 8, 2, 64, pad=3)
    b.start = b.start + 3
    got, pool = q.cuda(), b.pool.cuda()
    P.stage_norm_rope_append(qkv.cuda(), got, pool, b.stage_batch(P), cos.cuda(), sin.cuda(), gains[0].cuda(), gains[1].cuda(), eps)
    want_q, want_kv, off_q, off_kv = O.append(b, qkv[3:], q[3:], b.pool, cos, sin, 8, *gains, eps)
    assert torch.equal(got[:3].cpu(), q[:3])
    O.assert_within(got[3:], want_q, O.rounded(want_q, off_q, torch.float32), "q")
    O.assert_within(pool, want_kv, O.rounded(want_kv, off_kv, torch.bfloat16) * (off_kv > 0) + (off_kv == 0) * want_kv.abs() * O.U16, "pool")
    kept = (off_kv == 0) & (want_kv == b.pool.double())
    assert torch.equal(pool.cpu()[kept], b.pool[kept])
    out = q.cuda()
    P.stage_window_attention(got, out, pool, b.stage_batch(P), window=20)
    assert torch.equal(out[:3].cpu(), q[:3])


@pytest.mark.parametrize("sections", [(0, 32, 0), (0, 0, 32), (32, 0, 0), (0, 5, 27), (7, 0, 25), (12, 20, 0)])
def test_positions_of_axes_without_pairs_do_not_matter(sections):
    c = list(_append_case([6, 5], [3, 30], 8, 4, 64, axes=3))
    c[7] = list(sections)
    want = _run_append(c)
    _check_append(c, *want)
    for axis, n in enumerate(sections):
        if n == 0:
            c[6][axis] = torch.tensor([-1, 1 << 30] * 6)[:11]
    got = _run_append(c)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
