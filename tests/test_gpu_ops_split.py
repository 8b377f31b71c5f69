"""Window attention of a few prompt rows behind long lists of keys: 16 columns a workgroup, the keys cut over wavefronts and
workgroups, against float64 (tests/ops_oracle.py)."""
import math

import pytest
import torch

import paper_2512_21835_amd as P
from tests.test_gpu_ops import DEV, _check_window, _run_window, _window_case
from tests.test_gpu_ops_exact import _check_poisoned, _poisoned, _same

pytestmark = pytest.mark.gpu
ROWS, HELD = [20, 1, 0, 5], [3000, 90, 7, 1000]
TYPES = pytest.mark.parametrize("act,cache", [("fp32", "bf16"), ("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])


def _is_cut(c, window, sinks):
    """Whether the call cuts its keys over workgroups, which whole tiles of rows never are."""
    b, q, out = c
    return P.stage_window_workspace(q.to(DEV), out.to(DEV), b.pool.to(DEV), b.stage_batch(P), window, sinks) > 0


@TYPES
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (8, 2, 128), (2, 2, 128), (8, 1, 64), (4, 2, 128)])
def test_prompts_behind_long_lists(hq, hkv, d, act, cache):
    c = _window_case(ROWS, HELD, hq, hkv, d, act, cache, pad=2)
    for window, sinks in ((0, 0), (2000, 70), (1500, 0), (1493, 3)):
        assert _is_cut(c, window, sinks)
        _check_window(c, _run_window(c, window, sinks), window, sinks)


@TYPES
@pytest.mark.parametrize("d", [64, 128])
def test_what_rows_do_not_see(d, act, cache):
    """Unseen places hold anything; a later row's token that is not finite is not seen by the rows before it."""
    c = _window_case(ROWS, HELD, 4, 1, d, act, cache)
    b = c[0]
    used = torch.zeros(b.n_blocks, 16, dtype=torch.bool)
    for i, n in enumerate(b.lengths):
        j = torch.arange(n)
        see = (j < 2) | (j > n - b.rows[i] - 1500)
        used[b.table[i, j // 16].long()[see], (j % 16)[see]] = b.rows[i] > 0
    junk = torch.tensor([math.nan, math.inf, -math.inf, 3e38])
    fill = junk[torch.randint(0, 4, (b.n_blocks, 2, 1, 16, d), generator=b.gen)].to(b.pool.dtype)
    b.pool = torch.where(used[:, None, None, :, None], b.pool, fill)
    assert _is_cut(c, 1500, 2)
    _check_window(c, _run_window(c, 1500, 2), 1500, 2)
    want = _run_window(c, 1500, 2)
    for what in (1, 0):
        n, p = ROWS[0], b.lengths[0] - 3
        clean = b.pool.clone()
        b.pool[int(b.table[0, p // 16]), what, 0, p % 16] = math.nan
        got = _run_window(c, 1500, 2)
        assert torch.equal(got[:n - 3], want[:n - 3]) and torch.equal(got[n:], want[n:])
        assert bool(torch.isnan(got[n - 3:n]).all())
        b.pool = clean


@TYPES
@pytest.mark.parametrize("d", [64, 128])
def test_infinities_that_rows_see(d, act, cache):
    inf = float("inf")
    for window, sinks in ((0, 0), (1500, 2)):
        b, q, out, clean = _poisoned(ROWS, HELD, 8, 2, d, act, cache, 1, (9, 10), (inf, -inf))
        assert _is_cut((b, q, out), window, sinks)
        assert bool(_check_poisoned(b, q, out, clean, window, sinks).any())
        b, q, out, clean = _poisoned(ROWS, HELD, 8, 2, d, act, cache, 0, (9,), (-inf,))
        q[..., 9] = q[..., 9].abs() + 0.1
        assert not bool(_check_poisoned(b, q, out, clean, window, sinks).any())


@pytest.mark.parametrize("cache", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_values_near_the_largest_number(d, cache):
    b, q, out = c = _window_case(ROWS, HELD, 8, 2, d, "fp32", cache)
    b.pool[:, 1, :, :, 9] = 3.4e38 if cache == "fp32" else 3.3e38
    for window, sinks in ((0, 0), (1500, 2)):
        _check_window(c, _run_window(c, window, sinks), window, sinks)


@TYPES
def test_blocks_that_lead_nowhere_and_rows_that_see_nothing(act, cache):
    c = _window_case([20, 3, 40, 9], [3000, 0, 33, 2], 8, 2, 64, act, cache)
    b = c[0]
    b.table[0, 2], b.table[0, 100], b.table[0, 187] = b.n_blocks, -1, 1 << 30
    b.table[2, 0] = -1
    b.lengths[3] = b.length[3] = 0          # rows at negative positions
    b.table[1, 0] = -5                      # nothing of the sequence is there
    for window, sinks in ((0, 0), (1500, 5)):
        got = _run_window(c, window, sinks)
        _check_window(c, got, window, sinks)
        assert not bool(got[20:23].any()) and not bool(got[63:].any())


@pytest.mark.parametrize("cache", ["bf16", "fp32"])
def test_scores_of_any_size(cache):
    for scale, q_scale in ((0.0, 60.0), (4.0, 10.0), (1e-6, 1.0), (-0.5, 3.0)):
        c = _window_case(ROWS, HELD, 4, 2, 64, "fp32", cache, scale=q_scale)
        _check_window(c, _run_window(c, 1500, 4, scale=scale), 1500, 4, scale)


@TYPES
def test_in_place_strided_on_a_stream_and_captured(act, cache):
    b, q, out = c = _window_case(ROWS, HELD, 8, 2, 64, act, cache)
    want = _run_window(c, 1500, 2)
    n = b.total
    wide = torch.zeros(n, 11, 64, dtype=q.dtype, device=DEV)
    x, src = wide[:, 1:9], q.to(DEV)
    pool, batch = b.pool.to(DEV), b.stage_batch(P)
    need = P.stage_window_workspace(x, x, pool, batch, 1500, 2)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
    stream = torch.cuda.Stream()

    def call():
        x.copy_(src)
        P.stage_window_attention(x, x, pool, batch, window=1500, sinks=2, workspace=ws, stream=stream)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
    stream.synchronize()
    assert _same(x, want) and not bool(wide[:, 0].any()) and not bool(wide[:, 9:].any())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for _ in range(3):
        wide.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(x, want)


@TYPES
@pytest.mark.parametrize("rows,held", [(ROWS, HELD), ([1] * 9, [100, 3000, 5, 700, 64, 0, 15, 16, 2048]), ([200, 1, 33], [10, 40, 0])])
def test_the_same_call_gives_the_same_bits(rows, held, act, cache):
    c = _window_case(rows, held, 8, 2, 128, act, cache)
    for window, sinks in ((0, 0), (1500, 2)):
        want = _run_window(c, window, sinks)
        assert all(torch.equal(_run_window(c, window, sinks), want) for _ in range(3))
