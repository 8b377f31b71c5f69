"""Stages with normalised heads, a window with sinks, and low-rank adapters, against a plain float64 forward."""
import dataclasses
import itertools

import numpy as np
import pytest
import torch

import paper_2512_21835_amd as P
import synth
from oracle import stage_oracle as SO
from tests import harness

pytestmark = pytest.mark.gpu
F64 = torch.float64
SHAPES = {
    64: synth.StageShape("ops64", 901, 2, 256, 8, 2, 64, 512),
    128: synth.StageShape("ops128", 902, 2, 384, 4, 4, 128, 416),
    40: synth.StageShape("ops off 32", 903, 1, 200, 8, 1, 64, 328),     # widths that no GEMM tile divides
}
WINDOW, SINKS, ADAPTERS, RANK = 24, 3, 3, 12
TARGETS = (P.STAGE_ADAPT_QKV, P.STAGE_ADAPT_O, P.STAGE_ADAPT_DOWN)


def _bits(gen, *shape, std=0.05, mean=0.0):
    return (mean + std * torch.randn(*shape, generator=gen)).bfloat16()


class Model:
    """Weights and adapters of a shape, and their plain forward: one cache per sequence, everything in float64."""

    def __init__(self, shape, head_norm=False, window=0, sinks=0, adapters=False, kv_fp32=True, seed=5):
        self.s, self.head_norm, self.window, self.sinks, self.kv_fp32 = shape, head_norm, window, sinks, kv_fp32
        g = torch.Generator().manual_seed(seed)
        H, F, d, qd, kd = shape.hidden, shape.ffn, shape.head_dim, shape.q_dim, shape.kv_dim
        sizes = dict(wq=(qd, H), wk=(kd, H), wv=(kd, H), wo=(H, qd), wg=(F, H), wu=(F, H), wd=(H, F))
        self.w = [dict({n: _bits(g, *z) for n, z in sizes.items()},
                       **{n: _bits(g, z, mean=1.0, std=0.2) for n, z in (("g1", H), ("g2", H), ("gq", d), ("gk", d))})
                  for _ in range(shape.n_layers)]
        self.ad = {}
        io = {TARGETS[0]: (H, qd + 2 * kd), TARGETS[1]: (qd, H), TARGETS[2]: (F, H)}
        if adapters:
            for l, t, i in itertools.product(range(shape.n_layers), TARGETS, range(ADAPTERS)):
                r = (RANK, 5, 8)[(i + t + l) % 3]
                if (i, t) != (1, TARGETS[1]):      # adapter 1 has none of the O projection
                    self.ad[l, t, i] = _bits(g, r, io[t][0]), _bits(g, io[t][1], r, std=0.2), (0.5, -1.0, 2.0)[i]
        self.kv, self.of = {}, {}

    def config(self, **kw):
        n = ADAPTERS if self.ad else 0
        kw = {**dict(max_microbatches=2, max_batch=24, max_context=128, n_resident_max=self.s.n_layers), **kw}
        return P.config_for(self.s, kv_fp32=self.kv_fp32, head_norm=self.head_norm, window=self.window, sinks=self.sinks,
                            max_adapters=n, adapter_rank=RANK if n else 0, **kw)

    def load(self, h, resident=P.STAGE_RES_RESIDENT):
        for l, w in enumerate(self.w):
            P.stage_load_layer(h, l, w, resident)
        for (l, t, i), (a, b, scale) in self.ad.items():
            P.stage_load_adapter(h, l, t, i, a, b.cuda() if i == 2 else b, scale)     # (from either memory)

    def adapt(self, l, t, seq, x, y):
        a, b, scale = self.ad.get((l, t, self.of.get(seq, -1)), (None, None, 0.0))
        return y if a is None else y + scale * (x @ a.to(F64).T) @ b.to(F64).T

    def forward(self, seq, x):
        s, d = self.s, self.s.head_dim
        x = torch.as_tensor(x, dtype=F64)
        hq, hkv = s.n_q_heads, s.n_kv_heads
        keep = SO.round_to_f32 if self.kv_fp32 else SO.round_to_bf16
        for l, bits in enumerate(self.w):
            w = {n: v.to(F64) for n, v in bits.items()}
            K, V = self.kv.get((seq, l), (torch.zeros(0, hkv, d, dtype=F64),) * 2)
            pos = torch.arange(len(K), len(K) + len(x))
            y = SO.rms_norm(x, w["g1"], s.rms_eps)
            qkv = self.adapt(l, TARGETS[0], seq, y, y @ torch.cat([w["wq"], w["wk"], w["wv"]]).T).view(len(x), -1, d)
            q, k, v = qkv.split([hq, hkv, hkv], 1)
            if self.head_norm:
                q, k = SO.rms_norm(q, w["gq"], s.rms_eps), SO.rms_norm(k, w["gk"], s.rms_eps)
            q, k = SO.rope(q, pos, s.rope_theta), SO.rope(k, pos, s.rope_theta)
            K, V = torch.cat([K, keep(k)]), torch.cat([V, keep(v)])
            self.kv[seq, l] = K, V
            j, p = torch.arange(len(K))[None], pos[:, None]
            see = (j <= p) & ((j > p - self.window) | (j < self.sinks) if self.window else True)
            Kh, Vh = (z.repeat_interleave(hq // hkv, 1).transpose(0, 1) for z in (K, V))
            sc = (q.transpose(0, 1) @ Kh.transpose(1, 2)) * d ** -0.5
            o = (torch.softmax(sc.masked_fill(~see, -torch.inf), 2) @ Vh).transpose(0, 1).reshape(len(x), -1)
            x = x + self.adapt(l, TARGETS[1], seq, o, o @ w["wo"].T)
            y = SO.rms_norm(x, w["g2"], s.rms_eps)
            f = SO.silu(y @ w["wg"].T) * (y @ w["wu"].T)
            x = x + self.adapt(l, TARGETS[2], seq, f, f @ w["wd"].T)
        return x.numpy()


FEATURES = {"norm": dict(head_norm=True), "window": dict(window=WINDOW, sinks=SINKS), "adapters": dict(adapters=True),
            "all": dict(head_norm=True, window=WINDOW, sinks=SINKS, adapters=True)}
IDS = [0, -1, 2, 1]


def _calls(B, T, steps):
    return [("prefill", T)] + [("decode", 1)] * steps + [("prefill", 3)]


def _run(m, B, T, steps=3, decode=P.stage_decode, x_seed=9, before=None, resident=P.STAGE_RES_RESIDENT, **cfg):
    """The stage's outputs [rows, H] per call, and the inputs."""
    g = torch.Generator().manual_seed(x_seed)
    xs, outs = [], []
    with harness.compute_stream() as cs:
        h = P.stage_init(m.config(compute_stream=cs.handle, **cfg))
        try:
            m.load(h, resident)
            for b in range(B):
                if m.ad:
                    P.stage_set_adapter(h, 1, b, IDS[b % 4])
            for kind, t in _calls(B, T, steps):
                x = torch.randn(B, t, m.s.hidden, generator=g)
                x_in, x_out = x.cuda(), torch.empty(B, t, m.s.hidden, device="cuda")
                if kind == "prefill":
                    P.stage_prefill(h, [1], B, t, x_in, x_out)
                else:
                    decode(h, [1], B, x_in, x_out)
                P.stage_sync(h)
                xs.append(x)
                outs.append(x_out.cpu())
        finally:
            P.stage_destroy(h)
    return xs, outs


def _want(m, B, xs):
    m.kv.clear()
    m.of = {b: IDS[b % 4] for b in range(B)} if m.ad else {}
    return [np.stack([m.forward(b, x[b]) for b in range(B)]) for x in xs]


def _check(outs, want):
    for got, ref in zip(outs, want):
        rows = got.shape[-1]
        e = harness.fp32_errors(got.numpy().reshape(-1, rows), ref.reshape(-1, rows))
        assert harness.fp32_close(got.numpy().reshape(-1, rows), ref.reshape(-1, rows)), e


# 4 sequences: decode by the projections of few rows; 20: by those of many
@pytest.mark.parametrize("B,T", [(4, 45), (20, 18), (1, 70)])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("what", FEATURES)
def test_stage(what, shape, B, T):
    m = Model(SHAPES[shape], **FEATURES[what])
    xs, outs = _run(m, B, T)
    want = _want(m, B, xs)
    _check(outs, want)
    plain = _want(Model(SHAPES[shape]), B, xs)     # and the features are seen at all
    assert what == "window" and T < WINDOW or harness.fp32_errors(plain[1], want[1])[0] > 20 * harness.FP32_REL


def test_stage_of_more_rows_than_k_is_cut_for():
    m = Model(dataclasses.replace(SHAPES[64], n_layers=1), **FEATURES["all"])
    xs, outs = _run(m, 24, 46, steps=1)
    _check(outs, _want(m, 24, xs))


def test_stage_with_a_bf16_cache():
    """K and V may be a rounding step off where fp32 and float64 fall on either side of a boundary: at most 2^-8 of
    each, so 2^-8 of what the values add up to, and as much again of scores of size 1 or so through the keys."""
    m = Model(SHAPES[128], kv_fp32=False, **FEATURES["all"])
    xs, outs = _run(m, 4, 45)
    for got, ref in zip(outs, _want(m, 4, xs)):
        assert harness.fp32_errors(got.numpy(), ref)[0] < 2 ** -7


@pytest.mark.parametrize("B", [2, 6, 20])
@pytest.mark.parametrize("kv_fp32", [False, True])
def test_other_ways_to_run_a_call_give_the_same_bits(B, kv_fp32):
    m = Model(SHAPES[64], kv_fp32=kv_fp32, **FEATURES["all"])
    _, want = _run(m, B, 20)

    def lane(h, mbs, n, x_in, x_out):
        torch.cuda.current_stream().synchronize()
        P.stage_decode_lane(h, 1, mbs, n, x_in, x_out)
    for kw in (dict(decode=P.stage_decode_noalloc), dict(decode=lane, n_lanes=2),
               dict(resident=P.STAGE_RES_OFFLOADED, n_resident_max=0), dict(resident=P.STAGE_RES_OFFLOADED, n_resident_max=0, zero_copy=True),
               dict(resident=P.STAGE_RES_MLP_OFFLOADED)):
        _, got = _run(m, B, 20, **kw)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), kw


def test_a_captured_decode_replayed():
    """Window and adapters in a captured call: each replay repeats the captured step, whatever ran in between."""
    m = Model(SHAPES[64], **FEATURES["all"])
    with harness.compute_stream() as cs:
        h = P.stage_init(m.config(compute_stream=cs.handle))
        try:
            m.load(h)
            for b in range(3):
                P.stage_set_adapter(h, 0, b, IDS[b])
            x = torch.randn(3, 30, 256, device="cuda")
            P.stage_prefill(h, [0], 3, 30, x, torch.empty_like(x))
            step, out = torch.randn(3, 1, 256, device="cuda"), torch.zeros(3, 1, 256, device="cuda")
            P.stage_sync(h)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=cs.stream):
                P.stage_decode_noalloc(h, [0], 3, step, out)
            other = torch.randn(2, 9, 256, device="cuda")
            seen = []
            for _ in range(4):
                graph.replay()
                seen.append(out.clone())
                P.stage_set_adapter(h, 1, 0, 1)
                P.stage_prefill(h, [1], 2, 9, other, torch.empty_like(other))
                P.stage_sync(h)
                out.zero_()
            m.of = {b: IDS[b] for b in range(3)}
            for b in range(3):
                m.forward(b, x[b].cpu())
            want = np.stack([m.forward(b, step[b].cpu()) for b in range(3)])
            _check([s.cpu() for s in seen], [want] * 4)
            assert all(torch.equal(s, seen[0]) for s in seen)
        finally:
            P.stage_destroy(h)


def test_a_window_beyond_every_sequence_is_none():
    big = (1 << 31) - 1
    plain, wide = Model(SHAPES[64], head_norm=True), Model(SHAPES[64], head_norm=True, window=big, sinks=big)
    xs, outs = _run(wide, 3, 40)
    _check(outs, _want(plain, 3, xs))


def test_more_rows_than_the_operators_take_are_refused():
    s = dataclasses.replace(SHAPES[64], n_layers=1)
    m = Model(s, head_norm=True)
    h = P.stage_init(m.config(max_microbatches=1, max_batch=64, max_context=16384, kv_pool_blocks=64))
    try:
        m.load(h)
        x = torch.zeros(1, 1, 256, device="cuda")       # (not read)
        with pytest.raises(P.StageError) as e:           # 2^20 rows
            P.stage_prefill(h, [0], 64, 16384, x, x.clone())
        assert e.value.code == P.STAGE_EINVAL
        assert P.stage_get_length(h, 0, 0) == 0
    finally:
        P.stage_destroy(h)


def test_adapters_come_and_go():
    m = Model(SHAPES[64], adapters=True)
    with harness.compute_stream() as cs:
        h = P.stage_init(m.config(compute_stream=cs.handle))
        try:
            m.load(h)
            x = torch.randn(1, 5, 256, device="cuda")

            def run(id):
                out = torch.empty_like(x)
                P.stage_reset_sequence(h, 0, 0)
                if id is not None:
                    P.stage_set_adapter(h, 0, 0, id)
                P.stage_prefill(h, [0], 1, 5, x, out)
                P.stage_sync(h)
                return out.cpu()
            none = run(-1)
            assert not torch.equal(run(0), none)
            assert torch.equal(run(None), none)            # a sequence that was reset has none
            for (l, t, i) in m.ad:
                if i == 0:
                    P.stage_load_adapter(h, l, t, 0, None, None)
            assert torch.equal(run(0), none)
            m.of = {0: 1}
            _check([run(1)], [m.forward(0, x[0].cpu())[None]])
        finally:
            P.stage_destroy(h)


def test_refusals():
    m = Model(SHAPES[64], **FEATURES["all"])
    base = m.config()
    for name, bad in (("head_norm", 2), ("head_norm", -1), ("window", -1), ("sinks", -1), ("max_adapters", -1),
                      ("max_adapters", 0), ("adapter_rank", 0), ("adapter_rank", 10), ("adapter_rank", 260), ("head_dim", 96),
                      ("n_q_heads", 6), ("max_adapters", 1 << 20)):
        cfg = m.config()
        setattr(cfg, name, bad)
        with pytest.raises(P.StageError) as e:
            P.stage_init(cfg)
        assert e.value.code == P.STAGE_EINVAL, name
    cfg = m.config()
    cfg.window = 0                                          # sinks without a window
    with pytest.raises(P.StageError):
        P.stage_init(cfg)
    h = P.stage_init(base)
    try:
        w = {n: v for n, v in m.w[0].items() if n not in ("gq", "gk")}
        with pytest.raises(P.StageError) as e:
            P.stage_load_layer(h, 0, w, P.STAGE_RES_RESIDENT)
        assert e.value.code == P.STAGE_EINVAL
        m.load(h)
        a, b = torch.zeros(4, 256).bfloat16(), torch.zeros(768, 4).bfloat16()
        P.stage_load_adapter(h, 0, 0, 0, a, b)
        for args in ((2, 0, 0, a, b), (-1, 0, 0, a, b), (0, 3, 0, a, b), (0, -1, 0, a, b), (0, 0, ADAPTERS, a, b), (0, 0, -1, a, b),
                     (0, 0, 0, a, b, float("nan")), (0, 0, 0, a, b, float("inf")),
                     (0, 0, 0, torch.zeros(RANK + 1, 256).bfloat16(), torch.zeros(768, RANK + 1).bfloat16())):
            with pytest.raises(P.StageError) as e:
                P.stage_load_adapter(h, *args)
            assert e.value.code == P.STAGE_EINVAL, args[:3]
        with pytest.raises(ValueError):
            P.stage_load_adapter(h, 0, 0, 0, a, torch.zeros(768, 5).bfloat16())
        for args in ((2, 0, 0), (0, 24, 0), (0, 0, ADAPTERS), (0, 0, -2)):
            with pytest.raises(P.StageError) as e:
                P.stage_set_adapter(h, *args)
            assert e.value.code == P.STAGE_EINVAL
        x = torch.randn(1, 2, 256, device="cuda")           # and the handle still works
        P.stage_prefill(h, [0], 1, 2, x, torch.empty_like(x))
        P.stage_sync(h)
    finally:
        P.stage_destroy(h)
