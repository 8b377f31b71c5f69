"""Timed cases of the operators on the caller's tensors (``paper_2512_21835_amd``: the functions of include/stage_ops.h).

Three operators: the norm of each query and key head with the position rotation and the append to the paged cache;
attention with a sliding window and sinks over that cache; low-rank adapters beside a shared projection.  ``run`` computes
them in their plain form (torch, 32 bits, rounded once at the end) or, with ``own``, through the library.

Head shapes are those of the repository's workloads: tiny (4/2 heads of 64), 8B (32/8 of 128), 70B and 32B (64/8 of 128) and
13B (40/40 of 128).  Lengths, rows and adapter ids that the work depends on follow from the case alone; values, page
tables and which slots hold which tokens from the seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
PAGE = 16
EPS, THETA = 1e-5, 10000.0
GOLDEN = 0.6180339887498949
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}


def _append(name, hq, hkv, d, seqs, rows, held, act, cache, norm=True, axes=1, ragged=False, pad=0):
    return {"name": name, "op": "append", "hq": hq, "hkv": hkv, "d": d, "seqs": seqs, "rows": rows, "held": held,
            "act": act, "cache": cache, "norm": norm, "axes": axes, "ragged": ragged, "pad": pad}


def _window(name, hq, hkv, d, seqs, rows, held, window, sinks, act, cache, ragged=False, pad=0):
    return {"name": name, "op": "window", "hq": hq, "hkv": hkv, "d": d, "seqs": seqs, "rows": rows, "held": held,
            "window": window, "sinks": sinks, "act": act, "cache": cache, "ragged": ragged, "pad": pad}


def _adapter(name, rows, k, n, adapters, rank, act, runs, ragged=False):
    return {"name": name, "op": "adapter", "rows": rows, "k": k, "n": n, "adapters": adapters, "rank": rank, "act": act,
            "runs": runs, "ragged": ragged}


def listed():
    return [
        # One new token of one request on an 8B-shaped layer, fp32 activations as the stage keeps them: launch latency.
        _append("append_8b_1row", 32, 8, 128, 1, 1, 1000, "fp32", "bf16"),
        # Prompts of three axes (text between images) of very different lengths, a cache kept in fp32, a KV head per
        # query head, and rows of padding behind the last sequence.
        _append("append_13b_axes_ragged", 40, 40, 128, 5, 401, 77, "fp32", "fp32", axes=3, ragged=True, pad=13),
        # Four long prompts at once on a 70B-shaped layer, bf16 activations: the largest append, bound by its bytes.
        _append("append_70b_4x2048", 64, 8, 128, 4, 2048, 0, "bf16", "bf16"),
        # One token of the smallest stage, a short window: latency alone.
        _window("window_tiny_1row", 4, 2, 64, 1, 1, 300, 128, 4, "fp32", "bf16"),
        # A decode step of 64 requests of different lengths up to the longest context, wide window: the cache's bytes.
        _window("window_70b_64rows", 64, 8, 128, 64, 1, 16000, 4096, 4, "bf16", "bf16", ragged=True),
        # A decode step over an fp32 cache.
        _window("window_8b_16rows_fp32", 32, 8, 128, 16, 1, 2900, 1024, 4, "fp32", "fp32", ragged=True),
        # Four long prompts: matrix work.
        _window("window_70b_4x2048", 64, 8, 128, 4, 2048, 0, 1024, 4, "bf16", "bf16"),
        # A mixed call: chunks of prompts next to single tokens, fp32 activations, and rows of padding.
        _window("window_8b_mixed", 32, 8, 128, 12, 500, 1700, 512, 16, "fp32", "bf16", ragged=True, pad=7),
        # Prompts over an fp32 cache with a KV head per query head.
        _window("window_13b_2x600_fp32", 40, 40, 128, 2, 600, 300, 256, 4, "fp32", "fp32"),
        # A decode step of 16 requests, each with an adapter of its own, beside an 8B-shaped projection: latency.
        _adapter("adapter_8b_16rows", 16, 4096, 4096, 16, 16, "fp32", False),
        # 64 requests on a 70B-shaped up projection, some adapters shared, some rows without one: the adapters' bytes.
        _adapter("adapter_70b_64rows", 64, 8192, 28672, 48, 64, "bf16", False, ragged=True),
        # Prompts of a few requests, rows in runs of one adapter: the activations' bytes.
        _adapter("adapter_13b_4001rows", 4001, 5120, 5120, 3, 32, "bf16", True),
    ]


HEADS = [(4, 2, 64), (8, 8, 64), (16, 2, 64), (32, 8, 128), (64, 8, 128), (40, 40, 128), (8, 1, 128), (28, 14, 128)]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("append", "window", "window", "adapter"))
    act, cache = rng.choice(("fp32", "bf16")), rng.choice(("fp32", "bf16"))
    hq, hkv, d = rng.choice(HEADS)
    if op == "append":
        total = _log(rng, 1, 5000)
        seqs = min(total, _log(rng, 1, 64))
        c = _append("", hq, hkv, d, seqs, max(1, total // seqs), _log(rng, 1, 1500), act, cache, rng.random() < 0.7,
                    rng.choice((1, 3)), rng.random() < 0.5, rng.choice((0, 0, 5)))
    elif op == "window" and rng.random() < 0.5:   # single tokens
        held = _log(rng, 1, 12000)
        c = _window("", hq, hkv, d, _log(rng, 1, 40 if hkv < 40 else 12), 1, held, _log(rng, 16, 4000),
                    rng.choice((0, 1, 4, 17, 64)), act, cache, rng.random() < 0.7, rng.choice((0, 0, 3)))
    elif op == "window":                          # prompts
        total = _log(rng, 8, 2200)
        seqs = min(total, _log(rng, 1, 8))
        c = _window("", hq, hkv, d, seqs, total // seqs, _log(rng, 1, 3000) - 1, _log(rng, 16, 900),
                    rng.choice((0, 1, 4, 17, 64)), act, cache, rng.random() < 0.5, rng.choice((0, 0, 3)))
    else:
        rows, adapters = _log(rng, 1, 3500), _log(rng, 1, 48)
        k, n = rng.choice((256, 1000, 2048, 4096, 5120)), rng.choice((256, 1000, 2048, 4096, 5120))
        c = _adapter("", rows, k, n, adapters, rng.choice((4, 8, 16, 32, 64)), act, rng.random() < 0.5, rng.random() < 0.5)
    del c["name"]
    return c


def _spread(n, most, least, ragged):
    """n numbers from `least` to `most`, the first the largest; all `most` where nothing is ragged."""
    if not ragged:
        return [most] * n
    return [most if i == 0 else max(least, int(most * ((i * GOLDEN) % 1.0) ** 2)) for i in range(n)]


def _rows_of(c):
    """New rows of each sequence, and tokens that it holds with them."""
    rows = _spread(c["seqs"], c["rows"], 1, c["ragged"])
    held = _spread(c["seqs"], c["held"], min(1, c["held"]), c["ragged"])
    return rows, [r + h for r, h in zip(rows, held)]


def _ids_of(c):
    """The adapter of each row; -1: none (every ninth row, or run, of a ragged case)."""
    n, a = c["rows"], c["adapters"]
    if c["runs"]:
        group = [i * (2 * a + 1) // n for i in range(n)]     # runs of rows, every adapter more than once
    else:
        group = [int(((i + 1) * GOLDEN % 1.0) * a) if c["ragged"] else i for i in range(n)]
    return [-1 if c["ragged"] and g % 9 == 8 else g % a for g in group]


def _ranks_of(c):
    return [max(1, c["rank"] >> (i % 3)) if c["ragged"] else c["rank"] for i in range(c["adapters"])]


def _sections(c):
    half = c["d"] // 2
    return [half // 4, (half - half // 4) // 2, half - half // 4 - (half - half // 4) // 2] if c["axes"] == 3 else [half]


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(c, seed):
    gen = _generator(seed)
    normal = lambda shape, kind, scale=1.0: (torch.randn(shape, generator=gen, device=DEV) * scale).to(TYPES[kind])  # noqa: E731
    if c["op"] == "adapter":
        s = {"c": c, "x": normal((c["rows"], c["k"]), c["act"]), "base": normal((c["rows"], c["n"]), c["act"]),
             "a": normal((c["adapters"], c["rank"], c["k"]), "bf16", c["k"] ** -0.5),
             "b": normal((c["adapters"], c["n"], c["rank"]), "bf16", 0.1), "ids": _ints(_ids_of(c)), "ranks": _ints(_ranks_of(c)),
             "scales": 0.5 + torch.rand(c["adapters"], generator=gen, device=DEV)}
        s["out"] = torch.empty_like(s["base"])
        return s
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    rows, lengths = _rows_of(c)
    total, longest = sum(rows), max(lengths)
    pages = [(n + PAGE - 1) // PAGE for n in lengths]
    width, n_blocks = max(pages) + 1, sum(pages) + 3
    order = torch.randperm(n_blocks, generator=gen, device=DEV).to(torch.int32)
    table, at = torch.zeros((c["seqs"], width), dtype=torch.int32, device=DEV), 0
    for i, n in enumerate(pages):
        table[i, :n] = order[at:at + n]
        at += n
    s = {"c": c, "row_start": _ints(np.concatenate([[0], np.cumsum(rows)]).tolist()), "length": _ints(lengths), "table": table,
         "max_rows": max(rows), "max_len": longest, "pool": normal((n_blocks, 2, hkv, PAGE, d), c["cache"])}
    buffer_rows = total + c["pad"]
    if c["op"] == "window":
        s["q"] = normal((buffer_rows, hq, d), c["act"])
        s["out"] = torch.zeros_like(s["q"])
        return s
    half = d // 2
    angles = longest + 8
    turn = torch.arange(angles, device=DEV, dtype=torch.float64)[:, None] * THETA ** (
        -torch.arange(half, device=DEV, dtype=torch.float64) / half)
    s |= {"qkv": normal((buffer_rows, hq + 2 * hkv, d), c["act"]), "cos": turn.cos().float(), "sin": turn.sin().float(),
          "q_gain": (1 + normal((d,), "fp32", 0.1)).bfloat16() if c["norm"] else None,
          "k_gain": (1 + normal((d,), "fp32", 0.1)).bfloat16() if c["norm"] else None,
          "positions": torch.randint(0, angles, (3, buffer_rows), generator=gen, device=DEV, dtype=torch.int32)
          if c["axes"] == 3 else None}
    s["q"] = torch.zeros((buffer_rows, hq, d), dtype=TYPES[c["act"]], device=DEV)
    return s


def _of_rows(s, buffer_rows):
    """For each row of the buffers: whether it is one, its sequence, its place in it and its position."""
    row = torch.arange(buffer_rows, device=DEV, dtype=torch.int32)
    start = s["row_start"]
    real = row < start[-1]
    row = torch.minimum(row, start[-1] - 1)
    seq = torch.bucketize(row, start[1:], right=True)
    place = row - start[seq]
    return real, row, seq, place, s["length"][seq] - (start[seq + 1] - start[seq]) + place


def _append_plain(s):
    c, hq, hkv, half = s["c"], s["c"]["hq"], s["c"]["hkv"], s["c"]["d"] // 2
    real, row, seq, _, pos = _of_rows(s, s["qkv"].shape[0])
    x = s["qkv"][row].float()

    def head(x, gain):
        if gain is None:
            return x
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()

    turn = torch.cat([head(x[:, :hq], s["q_gain"]), head(x[:, hq:hq + hkv], s["k_gain"])], 1)
    if s["positions"] is None:
        cos, sin = s["cos"][pos], s["sin"][pos]
    else:
        axis = torch.repeat_interleave(torch.arange(3, device=DEV), _ints(_sections(c)), output_size=half)
        at, pair = s["positions"][axis][:, row].T.long(), torch.arange(half, device=DEV)
        cos, sin = s["cos"][at, pair], s["sin"][at, pair]
    cos, sin, x1, x2 = cos[:, None], sin[:, None], turn[..., :half], turn[..., half:]
    turn = torch.cat([x1 * cos - x2 * sin, x1 * sin + x2 * cos], -1)
    q, pool = s["q"], s["pool"]
    q.copy_(torch.where(real[:, None, None], turn[:, :hq].to(q.dtype), q))
    block, slot = s["table"][seq, pos // PAGE], pos % PAGE   # rows of padding write the last row's values again
    pool[block, 0, :, slot] = turn[:, hq:].to(pool.dtype)
    pool[block, 1, :, slot] = x[:, hq + hkv:].to(pool.dtype)
    return q, pool


def _window_plain(s):
    c, hq, hkv, d = s["c"], s["c"]["hq"], s["c"]["hkv"], s["c"]["d"]
    n, most, group = c["seqs"], s["max_rows"], s["c"]["hq"] // s["c"]["hkv"]
    start, length = s["row_start"], s["length"]
    count = start[1:] - start[:-1]
    first = length - count
    t = torch.arange(most, device=DEV, dtype=torch.int32)
    # the keys that some row of a sequence may see: its first tokens, then from the first row's window on
    low = torch.clamp(first - c["window"] + 1, min=0)
    reach = min(c["window"] + most - 1, s["max_len"])
    key = torch.cat([torch.arange(c["sinks"], device=DEV, dtype=torch.int32).expand(n, -1),
                     low[:, None] + torch.arange(reach, device=DEV, dtype=torch.int32)], 1)
    is_key = key < length[:, None]
    is_key[:, c["sinks"]:] &= key[:, c["sinks"]:] >= c["sinks"]
    held = torch.where(is_key, key, 0)
    pages = s["pool"][s["table"].gather(1, (held // PAGE).long()).long(), :, :, held % PAGE].float()  # [n, keys, 2, hkv, d]
    k, v = pages[:, :, 0].permute(0, 2, 3, 1).contiguous(), pages[:, :, 1].transpose(1, 2).contiguous()
    q = s["q"][torch.clamp(start[:-1, None] + t, max=s["q"].shape[0] - 1)].float()      # [n, most, hq, d]
    q = q.reshape(n, most, hkv, group, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, group * most, d)
    pos, key = (first[:, None] + t)[:, :, None], key[:, None]
    seen = is_key[:, None] & (key <= pos) & ((key > pos - c["window"]) | (key < c["sinks"]))
    score = torch.matmul(q, k).view(n, hkv, group, most, -1) * (1.0 / math.sqrt(d))
    score = torch.where(seen[:, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, hkv, group * most, -1), v).view(n, hkv, group, most, d) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(n, most, hq, d)
    real, _, seq, place, _ = _of_rows(s, s["q"].shape[0])
    s["out"].copy_(torch.where(real[:, None, None], o[seq, place].to(s["out"].dtype), s["out"]))
    return s["out"]


def _adapter_plain(s):
    c = s["c"]
    ids, every = s["ids"][:, None], torch.arange(c["adapters"], device=DEV)
    part = torch.matmul(s["x"].float(), s["a"].float().view(-1, c["k"]).T).view(c["rows"], c["adapters"], c["rank"])
    inside = torch.arange(c["rank"], device=DEV) < s["ranks"][:, None]
    part = torch.where((ids == every)[:, :, None] & inside, part * s["scales"][:, None], 0.0)
    b = s["b"].float().permute(0, 2, 1).reshape(-1, c["n"])
    s["out"].copy_((s["base"].float() + torch.matmul(part.view(c["rows"], -1), b)).to(s["out"].dtype))
    return s["out"]


def run(s):
    c = s["c"]
    if own:
        import paper_2512_21835_amd as P
        if c["op"] == "adapter":
            return P.stage_adapter_add(s["x"], s["base"], s["out"], s["a"], s["b"], s["ids"], ranks=s["ranks"], scales=s["scales"])
        batch = P.stage_batch(s["row_start"], s["length"], s["table"], s["max_rows"], s["max_len"])
        if c["op"] == "window":
            return P.stage_window_attention(s["q"], s["out"], s["pool"], batch, window=c["window"], sinks=c["sinks"])
        q = P.stage_norm_rope_append(s["qkv"], s["q"], s["pool"], batch, s["cos"], s["sin"], q_gain=s["q_gain"],
                                     k_gain=s["k_gain"], eps=EPS, positions=s["positions"],
                                     sections=_sections(c) if c["axes"] == 3 else None)
        return q, s["pool"]
    if c["op"] == "adapter":
        return _adapter_plain(s)
    return _window_plain(s) if c["op"] == "window" else _append_plain(s)


def _seen(c):
    """Sum over rows of the keys that they see, and over sequences of the keys that some row sees."""
    pairs, keys = 0, 0
    for rows, length in zip(*_rows_of(c)):
        first, w, sinks = length - rows, c["window"], c["sinks"]
        p = np.arange(first, length)
        low = np.maximum(p - w + 1, 0)
        pairs += int((p + 1 - low + np.minimum(low, sinks)).sum())
        low = max(first - w + 1, 0)
        keys += length - low + min(low, sinks)
    return pairs, keys


def work(c):
    if c["op"] == "adapter":
        ids, ranks, e = _ids_of(c), _ranks_of(c), BYTES[c["act"]]
        used = [i for i in ids if i >= 0]
        return {"bytes": c["rows"] * e * (c["k"] + 2 * c["n"]) + 4 * c["rows"] + sum(ranks[i] for i in set(used)) * 2 * (c["k"] + c["n"]),
                "flops": 2 * sum(ranks[i] for i in used) * (c["k"] + c["n"])}
    hq, hkv, d, e = c["hq"], c["hkv"], c["d"], BYTES[c["act"]]
    total = sum(_rows_of(c)[0])
    if c["op"] == "window":
        pairs, keys = _seen(c)
        return {"bytes": 2 * total * hq * d * e + 2 * keys * hkv * d * BYTES[c["cache"]], "flops": 4 * d * hq * pairs}
    angles = min(total, max(_rows_of(c)[1]) + 8) * d * 4     # a table row each of cos and sin, or the tables once
    return {"bytes": total * d * ((2 * hq + 2 * hkv) * e + 2 * hkv * BYTES[c["cache"]]) + angles,
            "flops": total * d * (hq + hkv) * (7 if c["norm"] else 3)}


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "adapter":
        out = s["base"].double()
        for i, rank in enumerate(_ranks_of(c)):
            rows = torch.tensor([r for r, a in enumerate(_ids_of(c)) if a == i], device=DEV, dtype=torch.long)
            if len(rows):
                low = s["x"][rows].double() @ s["a"][i, :rank].double().T.contiguous()
                out[rows] += float(s["scales"][i]) * (low @ s["b"][i, :, :rank].double().T.contiguous())
        return out
    hq, hkv, d, at = c["hq"], c["hkv"], c["d"], 0
    if c["op"] == "window":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
        for i, (rows, length) in enumerate(zip(*_rows_of(c))):
            j = torch.arange(length, device=DEV)
            kv = s["pool"][s["table"][i, j // PAGE].long(), :, :, j % PAGE].double()   # [length, 2, hkv, d]
            p = torch.arange(length - rows, length, device=DEV)[:, None]
            hidden = (j > p) | ((j <= p - c["window"]) & (j >= c["sinks"]))
            for h in range(hq):
                g = h // (hq // hkv)
                score = s["q"][at:at + rows, h].double() @ kv[:, 0, g].T.contiguous() * d ** -0.5
                out[at:at + rows, h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ kv[:, 1, g].contiguous()
            at += rows
        return out
    q, pool = s["q"].double(), s["pool"].double()
    axis = np.repeat(np.arange(c["axes"]), _sections(c))
    for i, (rows, length) in enumerate(zip(*_rows_of(c))):
        x, p = s["qkv"][at:at + rows].double(), torch.arange(length - rows, length, device=DEV)
        if c["axes"] == 3:
            turn = [s["positions"][a, at:at + rows].long() for a in axis]
        else:
            turn = [p] * (d // 2)
        cos = torch.stack([s["cos"][t, j] for j, t in enumerate(turn)], 1).double()[:, None]
        sin = torch.stack([s["sin"][t, j] for j, t in enumerate(turn)], 1).double()[:, None]
        for h0, h1, gain in ((0, hq, s["q_gain"]), (hq, hq + hkv, s["k_gain"])):
            y = x[:, h0:h1]
            if gain is not None:
                y = y / ((y * y).mean(-1, keepdim=True) + EPS).sqrt() * gain.double()
            a, b = y[..., :d // 2], y[..., d // 2:]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
            if h0 == 0:
                q[at:at + rows] = y
            else:
                pool[s["table"][i, p // PAGE].long(), 0, :, p % PAGE] = y
        pool[s["table"][i, p // PAGE].long(), 1, :, p % PAGE] = x[:, hq + hkv:]
        at += rows
    return q, pool
