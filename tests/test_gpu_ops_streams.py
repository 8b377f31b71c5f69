"""The operators' binding on other streams: memory, captures."""
import pytest
import torch

import paper_2512_21835_amd as P
from tests.test_gpu_ops import _tables

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _place(t):
    return range(t.data_ptr(), t.data_ptr() + t.nbytes)


def _calls():
    """Each call on temporary tensors, none of which is alive when it returns: the memory that it used."""
    def batch():
        return P.stage_batch(torch.arange(0, 2049, 2, device=DEV, dtype=torch.int32), torch.full((1024,), 2, device=DEV, dtype=torch.int32),
                             torch.arange(1024, device=DEV, dtype=torch.int32).view(1024, 1), 2, 16)

    def append(stream):
        b, pool, qkv = batch(), torch.zeros(1024, 2, 2, 16, 64, device=DEV), torch.zeros(2048, 8, 64, device=DEV)
        cos, sin = (t.to(DEV) for t in _tables(16, 64))
        gain = torch.ones(64, device=DEV, dtype=torch.bfloat16)
        q, at = torch.zeros(2048, 4, 64, device=DEV), torch.zeros(2048, device=DEV, dtype=torch.int32)
        P.stage_norm_rope_append(qkv, q, pool, b, cos, sin, gain, gain, positions=at, stream=stream)
        return [_place(t) for t in (pool, qkv, cos, sin, gain, q, at, *b.tensors)]

    def window(stream):
        b, pool = batch(), torch.zeros(1024, 2, 2, 16, 64, device=DEV)
        q, out = torch.zeros(2048, 4, 64, device=DEV), torch.zeros(2048, 4, 64, device=DEV)
        ws = torch.zeros(1 << 21, dtype=torch.uint8, device=DEV)
        P.stage_window_attention(q, out, pool, b, workspace=ws, stream=stream)
        return [_place(t) for t in (pool, q, out, ws, *b.tensors)]

    def adapter(stream):
        x, base, out = (torch.zeros(2048, 256, device=DEV) for _ in range(3))
        a, b = torch.zeros(8, 16, 256, device=DEV, dtype=torch.bfloat16), torch.zeros(8, 256, 16, device=DEV, dtype=torch.bfloat16)
        ids, ranks, scales = torch.zeros(2048, device=DEV, dtype=torch.int32), torch.full((8,), 4, device=DEV, dtype=torch.int32), torch.ones(8, device=DEV)
        ws = torch.zeros(1 << 21, dtype=torch.uint8, device=DEV)
        P.stage_adapter_add(x, base, out, a, b, ids, ranks, scales, workspace=ws, stream=stream)
        return [_place(t) for t in (x, base, out, a, b, ids, ranks, scales, ws)]
    return [append, window, adapter]


def _taken_next(used):
    """How many of these places the allocator gives to who comes next."""
    sizes = (256, 1024, 4096, 8192, 65536, 1 << 21, 1 << 22, 1 << 23)
    later = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(20)]
    return sum(any(p.start < q.stop and q.start < p.stop for q in map(_place, later)) for p in used)


@pytest.mark.parametrize("which", range(3))
def test_memory_of_tensors_used_on_another_stream_is_kept(which):
    """Freed behind the call, their memory goes to nobody before it has run."""
    call = _calls()[which]
    used = call(None)
    assert _taken_next(used) >= len(used) // 2    # (on their own stream it goes to others at once: that is seen here)
    stream = torch.cuda.Stream()
    busy = torch.zeros(8192, 8192, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(20):                       # some 10 ms each
            busy @ busy
    stream.wait_stream(torch.cuda.current_stream())
    used = call(stream)
    taken = _taken_next(used)
    assert not stream.query(), "the stream is done already"
    assert taken == 0
    torch.cuda.synchronize()
