"""What a stage's operator fields refuse, beside tests/test_gpu_stage_ops.py."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2512_21835_amd as P
from tests import harness
from tests.test_gpu_stage_ops import FEATURES, IDS, SHAPES, TARGETS, Model, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rank", [-4, -256])
def test_an_adapter_rank_below_zero_is_refused(rank):
    cfg = Model(SHAPES[64]).config()
    cfg.adapter_rank = rank
    with pytest.raises(P.StageError) as e:
        P.stage_destroy(P.stage_init(cfg))
    assert e.value.code == P.STAGE_EINVAL


def _nodes(graph):
    """Nodes of a captured graph."""
    hip = ctypes.CDLL("libamdhip64.so")
    n = ctypes.c_size_t()
    assert hip.hipGraphGetNodes(ctypes.c_void_p(graph.raw_cuda_graph()), None, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("B", [2, 20])       # few and many rows
@pytest.mark.parametrize("head_norm", [False, True])
def test_a_call_without_adapters_launches_none(B, head_norm):
    """A captured decode step has as many nodes as the stage without adapters while no sequence of the call has one that is set,
    and more when one has; the outputs are the same bits while none has."""
    m = Model(SHAPES[64], head_norm=head_norm, adapters=True)
    steps, outs = [], []
    x, step = torch.randn(B, 9, 256, device="cuda"), torch.randn(B, 1, 256, device="cuda")
    for loaded in (False, True):
        with harness.compute_stream() as cs:
            h = P.stage_init(m.config(compute_stream=cs.handle))
            try:
                if loaded:
                    m.load(h)
                    for l in range(m.s.n_layers):
                        P.stage_load_adapter(h, l, TARGETS[2], 0, None, None)      # adapter 0: of the other two projections
                        for t in TARGETS[:2]:
                            P.stage_load_adapter(h, l, t, 2, None, None)           # adapter 2: of this one alone
                else:
                    for l, w in enumerate(m.w):
                        P.stage_load_layer(h, l, w, P.STAGE_RES_RESIDENT)
                P.stage_prefill(h, [0], B, 9, x, torch.empty_like(x))
                P.stage_sync(h)
                for id in (-1, 0, 2) if loaded else (-1, 0):
                    P.stage_set_adapter(h, 0, 1, id)
                    out = torch.zeros_like(step)
                    graph = torch.cuda.CUDAGraph(keep_graph=True)
                    with torch.cuda.graph(graph, stream=cs.stream):
                        P.stage_decode_noalloc(h, [0], B, step, out)
                    steps.append(_nodes(graph))
                    if len(outs) == 0 or (loaded and id == -1):
                        graph.instantiate()
                        graph.replay()
                        P.stage_sync(h)
                        outs.append(out.clone())
                    del graph
            finally:
                P.stage_destroy(h)
    plain, unset, none, two, one = steps
    assert torch.equal(*outs)
    assert plain == none < one < two
    assert unset <= plain + 1                # (that a sequence has one is told to the device)


@pytest.mark.parametrize("kv_fp32", [False, True])
def test_micro_batches_of_one_call_or_one_by_one(kv_fp32):
    """A window's keys may be added up in another order: both groupings are held to the float64 forward, an fp32 cache's to the
    fp32 bounds, a bf16 cache's to a rounding step of K and V (2^-8 of each, and as much again by the scores)."""
    m = Model(SHAPES[64], kv_fp32=kv_fp32, **FEATURES["all"])
    x, step = torch.randn(4, 40, 256), torch.randn(4, 1, 256)
    m.of = {b: IDS[b] for b in range(4)}
    want = [np.stack([m.forward(b, z[b]) for b in range(4)]) for z in (x, step)]
    for groups in ([[0, 1]], [[0], [1]], [[1], [0]]):
        with harness.compute_stream() as cs:
            h = P.stage_init(m.config(compute_stream=cs.handle))
            try:
                m.load(h)
                for b in range(4):
                    P.stage_set_adapter(h, b // 2, b % 2, IDS[b])
                for call, z, ref in ((P.stage_prefill, x, want[0]), (P.stage_decode, step, want[1])):
                    got = torch.empty(z.shape)
                    for g in groups:
                        at = [2 * mb + b for mb in g for b in range(2)]
                        z_in = z[at].cuda()
                        z_out = torch.empty_like(z_in)
                        call(h, g, 2, z.shape[1], z_in, z_out) if call is P.stage_prefill else call(h, g, 2, z_in, z_out)
                        P.stage_sync(h)
                        got[at] = z_out.cpu()
                    if kv_fp32:
                        _check([got], [ref])
                    else:
                        assert harness.fp32_errors(got.numpy(), ref)[0] < 2 ** -7
            finally:
                P.stage_destroy(h)
