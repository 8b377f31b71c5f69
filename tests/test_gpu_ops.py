"""The operators of include/stage_ops.h against plain float64 implementations (tests/ops_oracle.py)."""
import ctypes
import math

import pytest
import torch

import paper_2512_21835_amd as P
from tests import ops_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _tables(n, d, theta=10000.0):
    angle = torch.arange(n, dtype=torch.float64)[:, None] * theta ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)
    return angle.cos().float(), angle.sin().float()


def _append_case(rows, held, hq, hkv, d, act="fp32", cache="bf16", norm=True, axes=1, pad=0, seed=1, q_act=None, eps=1e-5):
    b = O.Batch(rows, held, hkv, d, cache, seed, pad)
    n = b.total + pad
    qkv = torch.randn(n, hq + 2 * hkv, d, generator=b.gen).to(O.TYPES[act])
    q = torch.randn(n, hq, d, generator=b.gen).to(O.TYPES[q_act or act])
    cos, sin = _tables(b.max_len + 5, d)
    gains = [(1 + 0.2 * torch.randn(d, generator=b.gen)).bfloat16() for _ in range(2)] if norm else [None, None]
    positions = sections = None
    if axes == 3:
        positions = torch.randint(0, b.max_len + 5, (3, n), generator=b.gen, dtype=torch.int32)
        sections = [d // 8, d // 4 - 3, d // 2 - d // 8 - d // 4 + 3]
    return b, qkv, q, cos, sin, gains, positions, sections, eps


def _gpu(t):
    return None if t is None else t.to(DEV)


def _run_append(c, **kw):
    b, qkv, q, cos, sin, gains, positions, sections, eps = c
    q, pool = q.to(DEV), b.pool.to(DEV)
    P.stage_norm_rope_append(qkv.to(DEV), q, pool, b.stage_batch(P), cos.to(DEV), sin.to(DEV), _gpu(gains[0]),
                             _gpu(gains[1]), eps, _gpu(positions), sections, **kw)
    return q, pool


def _check_append(c, got_q, got_pool):
    b, qkv, q, cos, sin, gains, positions, sections, eps = c
    want_q, want_kv, off_q, off_kv = O.append(b, qkv, q, b.pool, cos, sin, q.shape[1], *gains, eps, positions, sections)
    for got, want, off, old, what in ((got_q, want_q, off_q, q, "q"), (got_pool, want_kv, off_kv, b.pool, "pool")):
        kept = off == 0
        O.assert_within(got, want, O.rounded(want, off, old.dtype), what)
        same = got.cpu()[kept & (want == old.double())]
        assert torch.equal(same, old[kept & (want == old.double())])   # what no row names keeps its bits


@pytest.mark.parametrize("rows,held,hq,hkv,d,act,cache,norm,axes,pad", [
    ([1], [0], 4, 2, 64, "fp32", "bf16", True, 1, 0),
    ([1], [1000], 32, 8, 128, "fp32", "fp32", True, 1, 0),
    ([3, 0, 17, 1], [0, 5, 15, 31], 8, 8, 128, "bf16", "bf16", True, 1, 2),
    ([5, 2], [13, 0], 16, 2, 64, "bf16", "fp32", True, 3, 0),
    ([7, 1, 9], [3, 64, 0], 28, 14, 128, "fp32", "bf16", True, 3, 5),
    ([33], [47], 5, 5, 64, "fp32", "fp32", False, 1, 1),
    ([2] * 70, list(range(70)), 4, 1, 64, "bf16", "bf16", True, 1, 3),     # more sequences than a wavefront has lanes
    ([0] * 100 + [3] + [0] * 40, [2] * 141, 2, 1, 128, "fp32", "bf16", True, 1, 0),
])
def test_append(rows, held, hq, hkv, d, act, cache, norm, axes, pad):
    c = _append_case(rows, held, hq, hkv, d, act, cache, norm, axes, pad)
    _check_append(c, *_run_append(c))


def test_append_one_gain_of_two_and_other_type_of_q():
    c = list(_append_case([4], [9], 8, 2, 128, "fp32", "bf16", q_act="bf16"))
    c[5] = [None, c[5][1]]
    _check_append(c, *_run_append(c))


def test_append_positions_of_one_axis():
    c = list(_append_case([4, 3], [9, 0], 8, 2, 64))
    c[6] = torch.randint(0, 12, (1, 7), dtype=torch.int32, generator=c[0].gen)
    b, qkv, q, cos, sin, gains, positions, _, eps = c
    got, pool = q.to(DEV), b.pool.to(DEV)
    P.stage_norm_rope_append(qkv.to(DEV), got, pool, b.stage_batch(P), cos.to(DEV), sin.to(DEV), _gpu(gains[0]),
                             _gpu(gains[1]), eps, positions[0].to(DEV))
    _check_append(c, got, pool)


def test_append_leaves_out_rows_that_lead_nowhere():
    c = list(_append_case([20, 6, 4], [10, 20, 5], 4, 2, 64, axes=3))
    b = c[0]
    b.table[0, 1] = b.n_blocks            # blocks past the pool and below it
    b.table[1, 1] = -1
    c[6][1, 25] = c[3].shape[0]           # angles past the tables and below them
    c[6][2, 27] = -1
    b.lengths[2] = 2                      # more rows than tokens: negative positions
    b.length[2] = 2
    _check_append(c, *_run_append(c))


def test_append_zero_heads_and_values_that_are_not_finite():
    c = _append_case([3], [2], 4, 2, 64, "fp32", "fp32", eps=1e-5)
    c[1][0] = 0.0                          # a zero head: eps keeps it
    got_q, got_pool = _run_append(c)
    assert torch.equal(got_q[0].cpu(), torch.zeros(4, 64))
    _check_append(c, got_q, got_pool)
    c[1][1, 0, 5] = math.inf               # reaches its own head only
    got_q, _ = _run_append(c)
    assert bool(torch.isfinite(got_q[1, 1:]).all()) and bool(torch.isfinite(got_q[[0, 2]]).all())
    assert not bool(torch.isfinite(got_q[1, 0]).all())


def test_append_in_place_and_strided():
    b, qkv, q, cos, sin, gains, _, _, eps = c = _append_case([6, 5], [3, 30], 8, 4, 64, "fp32", "bf16")
    want = _run_append(c)
    wide = torch.zeros(b.total, 20, 64, device=DEV)       # rows farther apart than they are wide
    wide[:, 2:18] = qkv.to(DEV)
    pool = b.pool.to(DEV)
    x = wide[:, 2:18]
    P.stage_norm_rope_append(x, wide[:, 2:10], pool, b.stage_batch(P), cos.to(DEV), sin.to(DEV), gains[0].to(DEV),
                             gains[1].to(DEV), eps)
    assert torch.equal(wide[:, 2:10], want[0]) and torch.equal(pool, want[1])
    assert torch.equal(wide[:, 10:18].cpu(), qkv[:, 8:]) and not bool(wide[:, :2].any()) and not bool(wide[:, 18:].any())


# ------------------------------------------------------------------------------------------------ window attention

def _window_case(rows, held, hq, hkv, d, act, cache, pad=0, seed=2, scale=1.0):
    b = O.Batch(rows, held, hkv, d, cache, seed, pad)
    n = b.total + pad
    q = (scale * torch.randn(n, hq, d, generator=b.gen)).to(O.TYPES[act])
    out = torch.randn(n, hq, d, generator=b.gen).to(O.TYPES[act])
    return b, q, out


def _run_window(c, window, sinks, **kw):
    b, q, out = c
    out = out.to(DEV)
    P.stage_window_attention(q.to(DEV), out, b.pool.to(DEV), b.stage_batch(P), window=window, sinks=sinks, **kw)
    return out


def _check_window(c, got, window, sinks, scale=0.0):
    b, q, out = c
    want, off32, off16 = O.window(b, q, out, b.pool, q.shape[1], window, sinks, scale)
    off = off32 + off16 if q.dtype == torch.bfloat16 else off32
    O.assert_within(got[:b.total], want[:b.total], O.rounded(want, off, q.dtype)[:b.total])
    assert torch.equal(got[b.total:].cpu(), out[b.total:])


HEADS = [(4, 2, 64), (3, 3, 128), (8, 1, 64), (8, 2, 128), (8, 1, 128), (2, 2, 64), (4, 1, 64), (4, 2, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["fp32", "bf16"])
def test_window_single_tokens(hq, hkv, d, cache, act):
    """Lengths around pages, tiles and the window; windows within a page, over several tiles and beyond the sequence."""
    held = [0, 1, 14, 15, 16, 31, 62, 63, 64, 130, 500]
    c = _window_case([1] * len(held), held, hq, hkv, d, act, cache, pad=1)
    for window, sinks in ((0, 0), (1, 0), (16, 4), (33, 1), (100, 40), (128, 64), (1000, 3)):
        _check_window(c, _run_window(c, window, sinks), window, sinks)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["fp32", "bf16"])
def test_window_prompts(hq, hkv, d, cache, act):
    """Prompts and chunks of them next to single tokens and sequences without rows."""
    c = _window_case([37, 1, 0, 70, 2], [0, 90, 12, 45, 200], hq, hkv, d, act, cache, pad=3)
    for window, sinks in ((0, 0), (1, 0), (20, 3), (64, 70)):
        _check_window(c, _run_window(c, window, sinks), window, sinks)


# as many KV heads as make these the calls that take whole tiles of rows at a time
MANY_HEADS = [(50, 50, 64), (50, 50, 128), (64, 32, 128), (68, 17, 64), (72, 9, 64), (72, 9, 128)]


@pytest.mark.parametrize("hq,hkv,d", MANY_HEADS)
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["fp32", "bf16"])
def test_window_prompts_of_many_heads(hq, hkv, d, cache, act):
    c = _window_case([37, 1, 0, 70, 2], [0, 90, 12, 45, 200], hq, hkv, d, act, cache, pad=3)
    for window, sinks in ((0, 0), (1, 0), (20, 3), (64, 70)):
        _check_window(c, _run_window(c, window, sinks), window, sinks)


@pytest.mark.parametrize("last,hq,hkv", [(50, 4, 2), (5, 1, 1), (900, 8, 1)])    # (the last: whole tiles)
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
def test_window_more_sequences_than_a_wavefront_has_lanes(cache, last, hq, hkv):
    rows = [1, 0, 3] * 30 + [last] + [2] * 9
    c = _window_case(rows, [7 * i % 90 for i in range(len(rows))], hq, hkv, 64, "fp32", cache, pad=2)
    for window, sinks in ((0, 0), (30, 5)):
        _check_window(c, _run_window(c, window, sinks), window, sinks)


@pytest.mark.parametrize("hkv", [1, 8])
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
def test_window_long_prompt_and_long_cache(cache, hkv):
    c = _window_case([150], [1800], 8 * hkv, hkv, 128, "fp32", cache)
    for window, sinks in ((300, 4), (0, 0)):
        _check_window(c, _run_window(c, window, sinks), window, sinks)
    if hkv > 1:
        return
    c = _window_case([1, 1], [9000, 3000], 8, 2, 128, "fp32", cache)
    for window, sinks in ((4096, 4), (0, 0), (200, 1000)):
        _check_window(c, _run_window(c, window, sinks), window, sinks)


@pytest.mark.parametrize("rows,held,hkv", [([1, 1, 1], [3, 40, 200], 1), ([30, 5], [4, 100], 1), ([30, 5], [4, 100], 52)])
@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ["fp32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_window_hides_what_is_not_finite(rows, held, hkv, cache, act, d):
    """Places that a row does not see may hold anything: past the sequence, before the window, and later rows'."""
    c = _window_case(rows, held, 4 * hkv, hkv, d, act, cache)
    b = c[0]
    used = torch.zeros(b.n_blocks, 16, dtype=torch.bool)
    for i, n in enumerate(b.lengths):
        j = torch.arange(n)
        first = n - b.rows[i]
        see = (j < 2) | (j > first - 17)
        used[b.table[i, j // 16].long()[see], (j % 16)[see]] = True
    junk = torch.tensor([math.nan, math.inf, -math.inf, 3e38])
    fill = junk[torch.randint(0, 4, (b.n_blocks, 2, 1, 16, d), generator=b.gen)].to(b.pool.dtype)
    b.pool = torch.where(used[:, None, None, :, None], b.pool, fill)
    _check_window(c, _run_window(c, 17, 2), 17, 2)
    if max(rows) > 1:     # a later row's token, seen by the rows from it on
        n, p = rows[0], b.lengths[0] - 3
        want = _run_window(c, 17, 2)
        clean = b.pool.clone()
        b.pool[int(b.table[0, p // 16]), 1, 0, p % 16, 1::7] = math.inf
        b.pool[int(b.table[0, p // 16]), 1, 0, p % 16, 2] = math.nan
        got = _run_window(c, 17, 2)
        assert torch.equal(got[:n - 3], want[:n - 3]) and torch.equal(got[n:], want[n:])
        assert torch.equal(got[:, 4:], want[:, 4:])
        assert bool(torch.isnan(got[n - 3:n, :4, 2]).all()) and bool(torch.isinf(got[n - 3:n, :4, 1::7]).all())
        assert bool(torch.isfinite(got[n - 3:n, :4, 3::7]).all())
        b.pool = clean
        b.pool[int(b.table[0, p // 16]), 0, 0, p % 16] = math.nan     # and its key
        got = _run_window(c, 17, 2)
        assert torch.equal(got[:n - 3], want[:n - 3]) and torch.equal(got[n:], want[n:])
        assert torch.equal(got[:, 4:], want[:, 4:])
        assert bool(torch.isnan(got[n - 3:n, :4]).all())


@pytest.mark.parametrize("act,cache", [("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16")])
@pytest.mark.parametrize("rows,hkv", [([1, 1, 1, 1], 2), ([20, 3, 40, 9], 2), ([20, 3, 40, 9], 24)])
def test_window_blocks_that_lead_nowhere_and_rows_that_see_nothing(rows, hkv, act, cache):
    c = _window_case(rows, [50, 0, 33, 2], 4 * hkv, hkv, 64, act, cache)
    b = c[0]
    b.table[0, 2] = b.n_blocks
    b.table[2, 0] = -1
    b.table[2, 1] = 1 << 30
    b.lengths[3] = b.length[3] = 0          # rows at negative positions
    b.table[1, 0] = -5                      # nothing of the sequence is there
    got = _run_window(c, 24, 5)
    _check_window(c, got, 24, 5)
    assert not bool(got[rows[0]:rows[0] + rows[1]].any()) and not bool(got[b.total - rows[3]:].any())


@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("hkv", [2, 76])
def test_window_scores_of_any_size(hkv, cache):
    """Scores beyond exp's range, equal scores, and a scale of the caller's."""
    for scale, q_scale in ((0.0, 60.0), (4.0, 10.0), (1e-6, 1.0), (-0.5, 3.0)):
        c = _window_case([1, 1, 30], [100, 3, 20], 2 * hkv, hkv, 64, "fp32", cache, scale=q_scale)
        _check_window(c, _run_window(c, 40, 4, scale=scale), 40, 4, scale)
    c = _window_case([1, 9], [100, 3], 2 * hkv, hkv, 64, "fp32", cache, scale=0.0)
    _check_window(c, _run_window(c, 40, 4), 40, 4)


def test_window_strides_stream_and_given_workspace():
    b, q, out = c = _window_case([1, 1, 1], [700, 20, 3000], 8, 2, 128, "bf16", "bf16")
    want = _run_window(c, 2000, 4)
    wide_q, wide_o = (torch.zeros(3, 11, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    wide_q[:, 1:9] = q.to(DEV)
    pool, batch = b.pool.to(DEV), b.stage_batch(P)
    need = P.stage_window_workspace(wide_q[:, 1:9], wide_o[:, 3:11], pool, batch, 2000, 4)
    stream = torch.cuda.Stream()
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device=DEV)     # NaN in every float: nothing relies on it
    stream.wait_stream(torch.cuda.current_stream())
    P.stage_window_attention(wide_q[:, 1:9], wide_o[:, 3:11], pool, batch, window=2000, sinks=4, workspace=ws, stream=stream)
    stream.synchronize()
    assert torch.equal(wide_o[:, 3:11], want) and not bool(wide_o[:, :3].any())
    if need:
        with pytest.raises(P.StageError):
            P.stage_window_attention(wide_q[:, 1:9], wide_o[:, 3:11], pool, batch, window=2000, sinks=4, workspace=ws[:need - 16])


@pytest.mark.parametrize("act,cache", [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("rows,hkv", [([30, 5], 52), ([30, 5], 2)])     # (whole tiles, and 16 columns at a time)
def test_window_prompts_strided_on_a_stream_and_captured(rows, hkv, act, cache):
    b, q, out = c = _window_case(rows, [70, 3], 4 * hkv, hkv, 64, act, cache)
    want = _run_window(c, 40, 2)
    wide_q, wide_o = (torch.zeros(35, 4 * hkv + 3, 64, dtype=q.dtype, device=DEV) for _ in range(2))
    wide_q[:, 1:-2] = q.to(DEV)
    pool, batch = b.pool.to(DEV), b.stage_batch(P)
    need = P.stage_window_workspace(wide_q[:, 1:-2], wide_o[:, 2:-1], pool, batch, 40, 2)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device=DEV)

    def call(stream):
        P.stage_window_attention(wide_q[:, 1:-2], wide_o[:, 2:-1], pool, batch, window=40, sinks=2, workspace=ws, stream=stream)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    call(stream)
    stream.synchronize()
    assert torch.equal(wide_o[:, 2:-1], want) and not bool(wide_o[:, :2].any()) and not bool(wide_o[:, -1].any())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(stream)
    for _ in range(3):
        wide_o.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(wide_o[:, 2:-1], want)


# ------------------------------------------------------------------------------------------------ adapters

def _adapter_case(rows, k, n, adapters, rank, act, ids, ranks=None, scales=True, seed=3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, k, generator=g).to(O.TYPES[act])
    base = torch.randn(rows, n, generator=g).to(O.TYPES[act])
    a = (torch.randn(adapters, rank, k, generator=g) * k ** -0.5).bfloat16()
    b = torch.randn(adapters, n, rank, generator=g).bfloat16()
    ids = torch.tensor(ids, dtype=torch.int32)
    ranks = None if ranks is None else torch.tensor(ranks, dtype=torch.int32)
    return x, base, a, b, ids, ranks, torch.rand(adapters, generator=g) - 0.3 if scales else None


def _run_adapter(c, **kw):
    x, base, a, b, ids, ranks, scales = (_gpu(t) for t in c)
    out = torch.empty_like(base)
    return P.stage_adapter_add(x, base, out, a, b, ids, ranks, scales, **kw)


def _check_adapter(c, got):
    want, off = O.adapter(*c)
    O.assert_within(got, want, O.rounded(want, off, c[0].dtype))


@pytest.mark.parametrize("act", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,k,n,adapters,rank,ids,ranks", [
    (1, 8, 8, 1, 4, [0], None),
    (1, 256, 688, 2, 16, [1], None),
    (5, 1000, 264, 3, 12, [2, 0, -1, 2, 1], [12, 3, 0]),
    (16, 512, 512, 16, 16, list(range(16)), None),
    (40, 264, 1000, 7, 64, [i * 5 % 9 - 1 for i in range(40)], [64, 1, 17, 63, 32, 200, -3]),
    (130, 128, 72, 3, 32, [i // 50 for i in range(130)], [32, 16, 8]),
    (70, 4096, 256, 2, 8, [i // 33 for i in range(70)], None),
    (300, 520, 136, 2, 256, [1] * 200 + [0] * 100, [256, 129]),
    (33, 64, 4096, 5, 20, [3] * 33, None),
])
def test_adapter(rows, k, n, adapters, rank, ids, ranks, act):
    c = _adapter_case(rows, k, n, adapters, rank, act, ids, ranks)
    _check_adapter(c, _run_adapter(c))


def test_adapter_rows_without_one_are_base_to_the_bit():
    for act in ("fp32", "bf16"):
        c = _adapter_case(9, 64, 64, 2, 8, act, [-1, 2, 1 << 30, -1 << 31, 0, -1, 1, 2, -9], [0, 8], scales=False)
        c[2][0], c[3][0] = math.nan, math.inf            # of rank 0: never looked at
        got = _run_adapter(c).cpu()
        for r, i in enumerate(c[4].tolist()):
            assert i == 1 or torch.equal(got[r], c[1][r])
        _check_adapter((c[0], c[1], c[2][1:], c[3][1:], torch.where(c[4] == 1, 0, -1), None, None), got)


def test_adapter_rows_do_not_meet_each_others_values():
    """Infinities and NaN of one row's input and of one adapter's weights stay with them."""
    for rows in (12, 100):
        c = _adapter_case(rows, 128, 128, 4, 16, "fp32", [i % 4 for i in range(rows)])
        want = _run_adapter(c)
        c[0][5, 7], c[0][5, 90], c[2][2, 3, 11], c[3][2, 9, 4] = math.inf, math.nan, math.nan, -math.inf
        got = _run_adapter(c)
        fine = [r for r in range(rows) if r != 5 and r % 4 != 2]
        assert torch.equal(got[fine], want[fine]) and bool(torch.isnan(got[5]).any())


def test_adapter_result_does_not_depend_on_the_other_rows():
    c = _adapter_case(40, 512, 320, 3, 24, "bf16", [i % 3 for i in range(40)])
    want = _run_adapter(c)
    back = [t.flip(0) if t is not None and t.shape[0] == 40 else t for t in c]
    assert torch.equal(_run_adapter(back).flip(0), want)
    assert torch.equal(_run_adapter(c), want)


def test_adapter_in_place_strided_and_on_a_stream():
    x, base, a, b, ids, ranks, scales = c = _adapter_case(21, 96, 160, 2, 12, "bf16", [i % 3 - 1 for i in range(21)])
    want = _run_adapter(c)
    wide_x, wide_y = torch.zeros(21, 112, dtype=torch.bfloat16, device=DEV), torch.zeros(21, 200, dtype=torch.bfloat16, device=DEV)
    wide_x[:, 8:104], wide_y[:, 16:176] = x.to(DEV), base.to(DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    y = wide_y[:, 16:176]
    P.stage_adapter_add(wide_x[:, 8:104], y, y, a.to(DEV), b.to(DEV), ids.to(DEV), None, scales.to(DEV), stream=stream)
    stream.synchronize()
    assert torch.equal(y, want) and not bool(wide_y[:, :16].any()) and not bool(wide_y[:, 176:].any())


# ------------------------------------------------------------------------------------------------ together

def _steps(d=128, hq=8, hkv=2, hidden=256):
    """What a layer runs around its attention, one new token per sequence: adapters on the QKV product, norm, rotation
    and append, attention, adapters on the output product."""
    g = torch.Generator().manual_seed(9)
    rows = [1, 1, 1, 1]
    b = O.Batch(rows, [200, 15, 16, 90], hkv, d, "bf16", 5)
    n_qkv = (hq + 2 * hkv) * d
    new = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    w = {"x": new(4, hidden), "qkv": new(4, n_qkv), "a1": (new(3, 8, hidden) * hidden ** -0.5).bfloat16(),
         "b1": (0.3 * new(3, n_qkv, 8)).bfloat16(), "a2": (new(3, 8, hq * d) * (hq * d) ** -0.5).bfloat16(),
         "b2": (0.3 * new(3, hidden, 8)).bfloat16(), "ids": torch.tensor([2, -1, 0, 2], dtype=torch.int32),
         "gq": (1 + 0.1 * new(d)).bfloat16(), "gk": (1 + 0.1 * new(d)).bfloat16(), "res": new(4, hidden)}
    w["cos"], w["sin"] = _tables(b.max_len, d)
    return b, w


def _layer(b, w, pool, batch, t, window, sinks):
    P.stage_adapter_add(w["x"], w["qkv"], t["qkv"], w["a1"], w["b1"], w["ids"], workspace=t["ws"])
    P.stage_norm_rope_append(t["qkv"].view(4, 12, 128), t["q"], pool, batch, w["cos"], w["sin"], w["gq"], w["gk"])
    P.stage_window_attention(t["q"], t["o"], pool, batch, window=window, sinks=sinks, workspace=t["ws"])
    P.stage_adapter_add(t["o"].view(4, 1024), w["res"], t["y"], w["a2"], w["b2"], w["ids"], workspace=t["ws"])


def _layer_setup():
    b, w = _steps()
    dw = {k: v.to(DEV) for k, v in w.items()}
    t = {"qkv": torch.empty(4, 12 * 128, device=DEV), "q": torch.empty(4, 8, 128, device=DEV),
         "o": torch.empty(4, 8, 128, device=DEV), "y": torch.empty(4, 256, device=DEV),
         "ws": torch.empty(1 << 22, dtype=torch.uint8, device=DEV)}
    return b, w, dw, t, b.pool.to(DEV), b.stage_batch(P)


def test_a_layers_run_of_them():
    b, w, dw, t, pool, batch = _layer_setup()
    _layer(b, dw, pool, batch, t, 64, 4)
    qkv, off = O.adapter(w["x"], w["qkv"], w["a1"], w["b1"], w["ids"], None, None)
    O.assert_within(t["qkv"], qkv, O.rounded(qkv, off, torch.float32), "qkv")
    # each next step from what the one before gave, so that the bounds do not add up
    qkv = t["qkv"].cpu().view(4, 12, 128)
    q, kv, q_off, kv_off = O.append(b, qkv, torch.zeros(4, 8, 128), b.pool, w["cos"], w["sin"], 8, w["gq"], w["gk"], 1e-5)
    O.assert_within(t["q"], q, O.rounded(q, q_off, torch.float32), "q")
    O.assert_within(pool, kv, O.rounded(kv, kv_off, torch.bfloat16), "pool")
    o, off, _ = O.window(b, t["q"].cpu(), torch.zeros(4, 8, 128), pool.cpu(), 8, 64, 4)
    O.assert_within(t["o"], o, O.rounded(o, off, torch.float32), "o")
    y, off = O.adapter(t["o"].cpu().view(4, 1024), w["res"], w["a2"], w["b2"], w["ids"], None, None)
    O.assert_within(t["y"], y, O.rounded(y, off, torch.float32), "y")


def test_a_captured_run_of_them_replayed():
    """Two graphs that share a workspace, replayed one after the other with eager work between, on changing inputs."""
    b, _, w, t, pool, batch = _layer_setup()
    start = pool.clone()
    _layer(b, w, pool, batch, t, 64, 4)        # before the capture: modules loaded
    torch.cuda.synchronize()
    graphs, windows = [], ((64, 4), (0, 0))
    for window, sinks in windows:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _layer(b, w, pool, batch, t, window, sinks)
        graphs.append(g)
    for step in range(3):
        w["x"].normal_()
        w["qkv"].normal_()
        for g, (window, sinks) in zip(graphs, windows):
            pool.copy_(start)
            _layer(b, w, pool, batch, t, window, sinks)
            want = [v.clone() for v in (t["q"], t["o"], t["y"], pool)]
            for v in (t["q"], t["o"], t["y"]):
                v.fill_(math.nan)
            pool.copy_(start)
            g.replay()
            torch.cuda.synchronize()
            for got, v in zip((t["q"], t["o"], t["y"], pool), want):
                assert torch.equal(got, v), step


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes and 2^31 elements, its sequence in the last blocks."""
    hkv, d, n = 8, 128, 66000      # 32768 elements a block: 2.16e9
    pool = torch.zeros(n, 2, hkv, 16, d, dtype=torch.bfloat16, device=DEV)
    b = O.Batch([3, 1], [40, 21], hkv, d, "bf16", 4)
    b.table = torch.where(b.table >= 0, n - 1 - b.table, b.table)
    small = b.pool
    pool[n - b.n_blocks:] = small.flip(0).to(DEV)
    q = torch.randn(4, 16, d, generator=b.gen)
    out = torch.zeros(4, 16, d, device=DEV)
    qkv = torch.randn(4, 32, d, generator=b.gen).to(DEV)
    cos, sin = (t.to(DEV) for t in _tables(64, d))
    P.stage_norm_rope_append(qkv, torch.empty(4, 16, d, device=DEV), pool, b.stage_batch(P), cos, sin)
    P.stage_window_attention(q.to(DEV), out, pool, b.stage_batch(P), window=30, sinks=2)
    b.table = torch.where(b.table >= 0, n - 1 - b.table, b.table)
    b.pool = pool[n - b.n_blocks:].flip(0).cpu()
    assert not torch.equal(b.pool, small)
    _check_window((b, q, out.cpu()), out, 30, 2)


# ------------------------------------------------------------------------------------------------ refusals

def _refused(fn, args, change, *more):
    for name, value in change.items():
        at = args
        *path, last = name.split(".")
        for p in path:
            at = getattr(at, p)
        old = getattr(at, last)
        setattr(at, last, value)
        assert fn(ctypes.byref(args), *more) == P.STAGE_EINVAL, name
        setattr(at, last, old)


def test_refusals():
    """Each argument out of what the header takes: refused before anything is enqueued."""
    L = P.lib()
    b = O.Batch([2], [3], 2, 64, "bf16")
    batch, pool = b.stage_batch(P), b.pool.to(DEV)
    x = torch.zeros(2, 8, 64, device=DEV)
    cos = torch.zeros(8, 32, device=DEV)
    cache = P.StageCache(pool.data_ptr(), b.n_blocks, 2, 64, P.STAGE_BF16)
    sizes = {"batch.n_seqs": 0, "batch.max_rows": 0, "batch.max_len": 16 * b.width + 1, "batch.max_blocks": 0,
             "cache.head_dim": 96, "cache.type": 2, "cache.n_blocks": 0, "cache.n_kv_heads": 3, "n_q_heads": 6, "rows": -1,
             "device": 99}
    pointers = {"batch.row_start": None, "batch.length": None, "batch.block_table": None, "cache.pool": pool.data_ptr() + 8}
    a = P.StageAppendArgs(0, batch, cache, 2, 4, x.data_ptr(), x.data_ptr(), 512, 512, 0, 0, None, None, 1e-5, 8, cos.data_ptr(),
                          cos.data_ptr(), None, 1, (ctypes.c_int32 * 3)(32, 0, 0))
    _refused(L.stage_norm_rope_append, a, sizes | pointers | {
        "qkv": None, "qkv_ld": 508, "q_ld": 252, "q_type": 1, "qkv_type": 3, "eps": math.nan, "n_angles": 0, "cos": None,
        "sin": cos.data_ptr() + 4, "q_gain": cos.data_ptr() + 2, "q_out": x.data_ptr() + 4}, None)
    a.positions = batch.row_start
    _refused(L.stage_norm_rope_append, a, {"n_axes": 2, "section": (ctypes.c_int32 * 3)(31, 0, 0)}, None)
    a.n_axes = 3
    for s in ((40, -8, 0), (32, 1, 0), (0, 0, 0)):
        _refused(L.stage_norm_rope_append, a, {"section": (ctypes.c_int32 * 3)(*s)}, None)
    w = P.StageWindowArgs(0, batch, cache, 2, 4, 8, 1, 0.0, x.data_ptr(), x.data_ptr(), 512, 512, 0)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    bad = {"window": -1, "sinks": -1, "scale": math.inf, "type": 2}
    need = ctypes.c_int64()
    _refused(L.stage_window_attention, w, sizes | pointers | bad | {"q": None, "out": x.data_ptr() + 8, "q_ld": 255, "out_ld": 258},
             ws.data_ptr(), 1 << 20, None)
    _refused(L.stage_window_workspace, w, sizes | bad, ctypes.byref(need))
    h = torch.zeros(1, 8, 16, device=DEV, dtype=torch.bfloat16)
    d = P.StageAdapterArgs(0, 2, 16, 16, 1, 8, 0, x.data_ptr(), x.data_ptr(), x.data_ptr(), 512, 512, 512, h.data_ptr(),
                           h.data_ptr(), batch.row_start, None, None)
    bad = {"k": 12, "n": 0, "n_adapters": 0, "max_rank": 6, "type": -1, "rows": -1, "device": -1}
    _refused(L.stage_adapter_add, d, bad | {"a": None, "b": h.data_ptr() + 2, "ids": None, "x": None, "x_ld": 8, "base_ld": 500,
                                            "out_ld": 514, "max_rank": 260}, ws.data_ptr(), 1 << 20, None)
    _refused(L.stage_adapter_workspace, d, bad, ctypes.byref(need))
    assert L.stage_adapter_workspace(ctypes.byref(d), ctypes.byref(need)) == P.STAGE_OK
    if need.value:
        assert L.stage_adapter_add(ctypes.byref(d), ws.data_ptr(), need.value - 1, None) == P.STAGE_ENOMEM
        assert L.stage_adapter_add(ctypes.byref(d), None, need.value, None) == P.STAGE_EINVAL


def test_binding_refuses_what_does_not_fit():
    b = O.Batch([2], [3], 2, 64, "bf16")
    batch, pool = b.stage_batch(P), b.pool.to(DEV)
    q = torch.zeros(2, 4, 64, device=DEV)
    for bad_q, bad_out, bad_pool in ((q.half(), q.half(), pool), (q, q.bfloat16(), pool), (q[:, :, ::2], q[:, :, ::2], pool),
                                     (q.transpose(0, 1), q.transpose(0, 1), pool), (q, q, pool[:, :, :, :8]), (q, q[:1], pool)):
        with pytest.raises(ValueError):
            P.stage_window_attention(bad_q, bad_out, bad_pool, batch)
    with pytest.raises(ValueError):
        P.stage_norm_rope_append(q, q, pool, batch, q[0], q[0])
    with pytest.raises(ValueError):
        P.stage_batch(batch.tensors[0].long(), *batch.tensors[1:], 2, 5)
    empty = q[:0]
    assert P.stage_window_attention(empty, empty, pool, batch) is empty
