"""Plain float64 implementations of the operators of include/stage_ops.h, on the CPU, and bounds on what the
kernels' arithmetic may be off.

Bounds are worst cases: u = 2^-24 is half a step of fp32 relative to the value, 2^-8 of bf16.
"""
import math

import numpy as np
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


class Batch:
    """Sequences with these new rows and held tokens, on pages of a pool in random order."""

    def __init__(self, rows, held, hkv, d, cache, seed=0, pad=0, spare=3, device="cpu"):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.lengths = list(rows), [r + h for r, h in zip(rows, held)]
        pages = [(n + 15) // 16 for n in self.lengths]
        self.n_blocks = sum(pages) + spare
        self.width = max(max(pages), 1) + 1
        order = torch.randperm(self.n_blocks, generator=g).tolist()
        self.table = torch.full((len(rows), self.width), -7, dtype=torch.int32)   # unused entries lead nowhere
        for i, n in enumerate(pages):
            self.table[i, :n] = torch.tensor(order[:n], dtype=torch.int32)
            order = order[n:]
        self.start = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32)
        self.length = torch.tensor(self.lengths, dtype=torch.int32)
        self.max_rows, self.max_len = max(max(rows), 1), max(max(self.lengths), 1)
        self.total, self.pad = sum(rows), pad
        self.pool = torch.randn(self.n_blocks, 2, hkv, 16, d, generator=g).to(TYPES[cache])
        self.gen = g

    def tensors(self, device):
        return [t.to(device) for t in (self.start, self.length, self.table)]

    def stage_batch(self, P, device="cuda"):
        return P.stage_batch(*self.tensors(device), self.max_rows, self.max_len)

    def held_tokens(self, pool, i):
        """K and V of sequence i, [length, 2, hkv, d] in float64; rows of blocks out of the pool are NaN."""
        j = torch.arange(self.lengths[i])
        block = self.table[i, j // 16].long()
        ok = (block >= 0) & (block < pool.shape[0])
        kv = pool[torch.where(ok, block, 0), :, :, j % 16].double()
        kv[~ok] = math.nan
        return kv, ok


def append(b, qkv, q_out, pool, cos, sin, hq, q_gain, k_gain, eps, positions=None, sections=None):
    """(q_out, pool) in float64, and per element what fp32 arithmetic may be off."""
    hkv, d = pool.shape[2], pool.shape[4]
    q, kv = q_out.double().clone(), pool.double().clone()
    q_off, kv_off = torch.zeros_like(q), torch.zeros_like(kv)
    axis = np.repeat(np.arange(3), sections) if sections else np.zeros(d // 2, dtype=int)
    at = 0
    for i, n in enumerate(b.rows):
        for t in range(n):
            r, p = at + t, b.lengths[i] - n + t
            if p < 0 or p >= b.max_len:
                continue
            block = int(b.table[i, p // 16])
            turn = [p] * 3 if positions is None else [int(positions[a, r]) for a in range(positions.shape[0])]
            if not 0 <= block < pool.shape[0] or any(not 0 <= x < cos.shape[0] for x in turn):
                continue
            x = qkv[r].double()
            c = torch.stack([cos[turn[a], j] for j, a in enumerate(axis)]).double()
            s = torch.stack([sin[turn[a], j] for j, a in enumerate(axis)]).double()
            for h in range(hq + 2 * hkv):
                y, gain = x[h], q_gain if h < hq else k_gain
                off = torch.zeros(d, dtype=torch.float64)
                if h < hq + hkv:
                    if gain is not None:
                        y = y / math.sqrt(float((y * y).mean()) + eps) * gain.double()
                    a, e = y[:d // 2], y[d // 2:]
                    y = torch.cat([a * c - e * s, a * s + e * c])
                    # the norm: a chain of at most 16 + 4 sums of squares (its relative error halved by the root),
                    # mean, eps, root, quotient, two products: 20 / 2 + 8; the turn: two products, a difference
                    off = 21 * U32 * torch.cat([(a * c).abs() + (e * s).abs(), (a * s).abs() + (e * c).abs()])
                if h < hq:
                    q[r, h], q_off[r, h] = y, off
                else:
                    w = (h - hq) // hkv
                    kv[block, w, (h - hq) % hkv, p % 16], kv_off[block, w, (h - hq) % hkv, p % 16] = y, off
        at += n
    return q, kv, q_off, kv_off


def window(b, q, out, pool, hq, window, sinks, scale=0.0):
    """The output in float64 (rows of no sequence keep `out`), and per element what the kernel may be off before
    its last rounding: a first term for fp32 arithmetic, a second for probabilities rounded to bf16."""
    hkv, d = pool.shape[2], pool.shape[4]
    scale = scale or d ** -0.5
    o = out.double().clone()
    off32, off16 = torch.zeros_like(o), torch.zeros_like(o)
    at = 0
    for i, n in enumerate(b.rows):
        kv, ok = b.held_tokens(pool, i)
        j = torch.arange(b.lengths[i])
        for t in range(n):
            p = b.lengths[i] - n + t
            see = (j <= p) & ok
            if window:
                see &= (j > p - window) | (j < sinks)
            if not bool(see.any()):
                o[at + t] = 0
                continue
            k, v = (kv[see, x].transpose(0, 1) for x in (0, 1))     # [hkv, keys, d]
            x = q[at + t].double().view(hkv, hq // hkv, d)
            w = torch.softmax(x @ k.transpose(1, 2) * scale, 2)
            o[at + t] = (w @ v).view(hq, d)
            # a score's sum of d products and its scaling, then exp's argument and its result (a few steps; the
            # argument's rounding grows with it), all doubled as numerator and denominator may be off
            # by as much; sums of as many probabilities as keys
            size = (x.abs() @ k.abs().transpose(1, 2)).amax(2).view(hq, 1) * abs(scale)
            term = (w @ v.abs()).view(hq, d)
            off32[at + t] = term * U32 * (2 * (d + 8) * size + 2 * k.shape[1] + 32)
            off16[at + t] = term * U16
        at += n
    return o, off32, off16


def adapter(x, base, a, b, ids, ranks, scales):
    y = base.double().clone()
    off = U32 * y.abs()
    for r, i in enumerate(ids.tolist()):
        if not 0 <= i < a.shape[0]:
            continue
        n = a.shape[1] if ranks is None else min(max(int(ranks[i]), 0), a.shape[1])
        s = 1.0 if scales is None else float(scales[i])
        A, B, v = a[i, :n].double(), b[i, :, :n].double(), x[r].double()
        y[r] += s * (B @ (A @ v))
        # sums of k and of n products, the scaling, the last sum
        off[r] += (x.shape[1] + n + 8) * U32 * abs(s) * (B.abs() @ (A.abs() @ v.abs())) + U32 * y[r].abs()
    return y, off


def rounded(y, off, dtype):
    """What a result of this type may be off: its arithmetic and the rounding of what that gives."""
    return off + (y.abs() + off) * (U32 if dtype == torch.float32 else U16) + 1e-37


def assert_within(got, want, off, what=""):
    got = got.double().cpu()
    bad = ~((got - want).abs() <= off)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} off, first at "
                                 f"{tuple(int(v) for v in bad.nonzero()[0])}: {float(got[bad][0])} for {float(want[bad][0])}, "
                                 f"{float(off[bad][0]):.3g} allowed")
