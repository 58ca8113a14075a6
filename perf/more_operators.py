"""What the operators of a paged key/value cache in the storage type are measured on.

The rows of a fused QKV product go into a cache of bf16 or fp32 pages - query and key heads normalised and rotated on the
way, where the model does that -, and the new rows attend over it: one token per sample, or packed pieces of prompts, with
all earlier positions in sight or a sliding window of them and a few first ones that stay.

`run` calls the operators through `paper_2505_18164_amd.mdi` where `own` is true, and computes the same with elementary
torch operations where it is false.  The inputs are what a user's program holds: parts of a fused product, pages handed out
in no order, tables with room for more than is used, keys with a few loud channels; behind a window the pages that nobody
sees any more have been given back.
"""
import math

import torch

own = False

PLAIN_SCORES = 1 << 28            # scores the plain form of the attention holds at a time
POOL_PIECE = 1 << 26              # elements of the cache made at a time
EPS = 1e-6
ROPE_BASE = 10000.0

# (query heads, kv heads, channels of a head): the shapes of synth.py ...
HEADS = {"gpt2": (12, 12, 64), "nanollama": (16, 16, 64), "tinyllama": (32, 4, 64), "llama2_7b": (32, 32, 128), "llama3_8b": (32, 8, 128),
         # ... and heads whose groups are no power of two, a single kv head, heads of other sizes
         "groups of 3": (6, 2, 64), "groups of 5": (10, 2, 128), "one kv head": (20, 1, 128), "heads of 96": (12, 4, 96), "heads of 256": (8, 4, 256)}
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _text(numbers):
    return " ".join(str(x) for x in numbers)


def _rows(case):
    """New rows of every sample, and the positions each has behind it."""
    if "ctx" in case:
        ctx = [int(x) for x in case["ctx"].split()]
        return [1] * len(ctx), [c - 1 for c in ctx]
    return [int(x) for x in case["lens"].split()], [int(x) for x in case["behind"].split()]


def listed():
    return [
        # -- into the cache
        # A round of 16 samples in flight: each rotates and appends its newest position.  The smallest call, all latency.
        {"name": "append 16 of llama3-8b", "op": "append", "heads": "llama3_8b", "dtype": "bf16", "page": 64, "rot": 128, "norm": "none", "lens": _text([1] * 16), "behind": _text([2048 + 411 * i for i in range(16)])},
        # Short and odd prompts of an fp32 program that normalises its heads and rotates half of their channels; pages that divide nothing.
        {"name": "append 9 prompts of tinyllama, fp32", "op": "append", "heads": "tinyllama", "dtype": "fp32", "page": 24, "rot": 32, "norm": "layer", "lens": "333 1 517 64 1200 97 2 800 1500", "behind": "0 0 5 0 0 100 31 0 0"},
        # The first visits of eight samples of the benchmark's 7B partition, one layer of it, with norms of queries and keys.
        {"name": "append 8 prompts of llama2-7b, norms", "op": "append", "heads": "llama2_7b", "dtype": "bf16", "page": 64, "rot": 128, "norm": "rms", "lens": _text([1024] * 8), "behind": _text([0] * 8)},
        # -- one new token per sample
        # The smallest: a fresh sample with a cache of one position.
        {"name": "token 2 of tinyllama", "op": "token", "heads": "tinyllama", "dtype": "bf16", "page": 16, "window": 0, "sinks": 0, "ctx": "1"},
        # An ordinary round of the 7B partition: eight samples of different ages, every head with its own cache.
        {"name": "8 tokens of llama2-7b", "op": "token", "heads": "llama2_7b", "dtype": "bf16", "page": 64, "window": 0, "sinks": 0, "ctx": "1030 2047 4096 1 333 2900 1600 3777"},
        # One sample with a very long cache, in odd pages: only the split over its length fills the chip.
        {"name": "one token of llama3-8b behind 120001", "op": "token", "heads": "llama3_8b", "dtype": "bf16", "page": 40, "window": 0, "sinks": 0, "ctx": "120001"},
        # Sixteen generations that never end: the newest 4096 positions and the first four.
        {"name": "16 tokens of llama3-8b, window", "op": "token", "heads": "llama3_8b", "dtype": "bf16", "page": 64, "window": 4096, "sinks": 4, "ctx": _text([3000 + 5987 * i for i in range(16)])},
        # -- packed prompts
        # Many short prompts wait at a small node: lengths from one token on.
        {"name": "24 short prompts of gpt2", "op": "prompts", "heads": "gpt2", "dtype": "bf16", "page": 16, "window": 0, "sinks": 0, "lens": _text([1 + (37 * i) % 64 for i in range(24)]), "behind": _text([0] * 24)},
        # Pieces of four long prompts: few rows, many earlier positions.
        {"name": "4 pieces of 64 behind 8000, llama3-8b", "op": "prompts", "heads": "llama3_8b", "dtype": "bf16", "page": 64, "window": 0, "sinks": 0, "lens": "64 64 64 64", "behind": "8000 7936 7000 8100"},
        # Ragged prompts of the small fp32 model, with a window.
        {"name": "5 ragged prompts of nanollama, fp32, window", "op": "prompts", "heads": "nanollama", "dtype": "fp32", "page": 24, "window": 300, "sinks": 4, "lens": "333 100 1500 17 512", "behind": "0 0 0 1000 5"},
        # A long document and two shorter ones, every head with its own cache, a window of 1024 and four first tokens.
        {"name": "prompts of 6000, 2000 and 500, llama2-7b, window", "op": "prompts", "heads": "llama2_7b", "dtype": "bf16", "page": 64, "window": 1024, "sinks": 4, "lens": "6000 2000 500", "behind": "0 0 300"},
        # The largest: the same lengths with everything in sight.
        {"name": "prompts of 6000, 2000 and 500, llama3-8b", "op": "prompts", "heads": "llama3_8b", "dtype": "bf16", "page": 64, "window": 0, "sinks": 0, "lens": "6000 2000 500", "behind": "0 0 300"},
    ]


def _spread(rng, lo, hi):
    """A whole number of [lo, hi], its logarithm uniform."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "token", "prompts"])
    case = {"op": op, "heads": rng.choice(sorted(HEADS)), "dtype": rng.choice(["bf16", "bf16", "bf16", "fp32"]), "page": rng.choice([16, 64, 128, 256, _spread(rng, 5, 200)])}
    H, K, h = HEADS[case["heads"]]
    if op == "append":
        case["rot"] = rng.choice([h, h, h // 2, 0])
        case["norm"] = rng.choice(["none", "rms", "layer"])
    else:
        case["window"] = rng.choice([0, _spread(rng, 1, 6000)])
        case["sinks"] = rng.choice([0, 1, 4, _spread(rng, 1, 500)]) if case["window"] else 0
    if op == "token":
        n = _spread(rng, 1, 64)
        most = max(2, min(120000, (1 << 26) // (n * K * h)))             # no more cache than the largest listed case reads
        top = _spread(rng, 1, most)
        case["ctx"] = _text(max(1, min(top, int(top * rng.uniform(0.2, 1.0)))) for _ in range(n))
        return case
    n = _spread(rng, 1, 32)
    if op == "append":
        rows = _spread(rng, n, max(n, min(16384, (1 << 25) // (K * h))))
    else:
        rows = _spread(rng, n, 8192)
    cuts = sorted(rng.uniform(0, 1) for _ in range(n - 1))
    lens = [max(1, int(rows * (b - a))) for a, b in zip([0.0] + cuts, cuts + [1.0])]
    # earlier positions: none, or so many that the attention costs no more than that of the largest listed case (an eighth of
    # its products in fp32)
    left = 6000 * 6000 * 32 * 128 // (H * h) // (8 if case["dtype"] == "fp32" else 1)
    used = sum(t * t for t in lens)
    while op == "prompts" and used > left:
        lens = [max(1, t * 3 // 4) for t in lens]
        used = sum(t * t for t in lens)
    room = max(1, min(16000, (left - used) // (2 * sum(lens)) + 1, (1 << 26) // (n * K * h)))
    case["lens"] = _text(lens)
    case["behind"] = _text(0 if rng.random() < 0.5 else _spread(rng, 1, room) for _ in lens)
    return case


# ---------------------------------------------------------------------------------------------------------------------
# What a user's program has in hand

def _inputs(case, seed):
    """Everything that both forms and the 64-bit values are computed from."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    H, K, h = HEADS[case["heads"]]
    dtype, pt = TYPES[case["dtype"]], case["page"]
    lens, behind = _rows(case)
    total = [a + b for a, b in zip(lens, behind)]
    n, rows = len(lens), sum(lens)
    stride = max((t + pt - 1) // pt for t in total) + 2                   # tables have room to grow
    window, sinks = case.get("window", 0), case.get("sinks", 0)
    # the pages that some row sees (or that are written); the others' entries are stale
    live = []
    for t, p0 in zip(total, behind):
        lo = max(0, p0 + 1 - window) if window else 0
        live.append([at for at in range((t + pt - 1) // pt) if (at + 1) * pt > lo or at * pt < sinks])
    n_pages = sum(len(x) for x in live) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    tables = torch.full((n, stride), -1, dtype=torch.int32, device="cuda")
    done = 0
    for i, pages in enumerate(live):
        tables[i, torch.tensor(pages, device="cuda")] = order[done:done + len(pages)]
        done += len(pages)
    starts = [0]
    for t in lens:
        starts.append(starts[-1] + t)
    s = {"case": case, "H": H, "K": K, "h": h, "pt": pt, "n": n, "rows": rows, "lens": lens, "behind": behind, "window": window, "sinks": sinks, "max_ctx": max(total), "tables": tables,
         "start": torch.tensor(starts, dtype=torch.int32, device="cuda"), "pos": torch.tensor(behind, dtype=torch.int32, device="cuda"),
         "data": torch.empty((n_pages, K, 2, pt, h), dtype=dtype, device="cuda")}
    loud = 1 + 9 * (torch.rand((K, h), generator=g, device="cuda") < 0.03).float()        # a few channels of the keys
    if case["op"] == "append":
        s["data"].zero_()
        # rows of the fused product: query heads, key heads, value heads
        qkv = torch.randn((rows, H + 2 * K, h), generator=g, device="cuda")
        qkv[:, H:H + K] *= loud
        qkv = qkv.to(dtype)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
        for name in ("q_gain", "k_gain"):
            s[name] = 1 + 0.3 * torch.randn(h, generator=g, device="cuda")
        for name in ("q_bias", "k_bias"):
            s[name] = 0.2 * torch.randn(h, generator=g, device="cuda") if case["norm"] == "layer" else None
        half = case["rot"] // 2
        s["freq"] = torch.tensor([ROPE_BASE ** (-i / half) for i in range(half)], dtype=torch.float64, device="cuda")
        return s
    piece = max(1, POOL_PIECE // (K * 2 * pt * h))
    gain = torch.stack([loud, torch.ones_like(loud)], 1).unsqueeze(2)    # keys, values
    for lo in range(0, n_pages, piece):
        m = min(piece, n_pages - lo)
        s["data"][lo:lo + m] = torch.randn((m, K, 2, pt, h), generator=g, device="cuda") * gain
    s["q"] = torch.randn((rows, H, h), generator=g, device="cuda").to(dtype)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "append":
        s["q_out"] = torch.empty((s["rows"], s["H"], s["h"]), dtype=s["q"].dtype, device="cuda")
    else:
        s["out"] = torch.empty_like(s["q"])
    if own:
        from paper_2505_18164_amd import mdi
        cache = mdi.KvCache(s["data"], s["tables"])
        s["cache"] = cache
        s["plan"] = cache.rows(s["pos"], start=None if case["op"] == "token" else s["start"], n_rows=s["rows"], max_ctx=s["max_ctx"])
        if case["op"] == "append":
            norm = {} if case["norm"] == "none" else {"norm": case["norm"], "q_gain": s["q_gain"], "k_gain": s["k_gain"], "q_bias": s["q_bias"], "k_bias": s["k_bias"], "eps": EPS}
            s["prep"] = cache.prep(freq=s["freq"] if case["rot"] else None, **norm)
        else:
            s["workspace"] = cache.workspace(s["plan"], s["H"], window=s["window"], sinks=s["sinks"])
    return s


# ---------------------------------------------------------------------------------------------------------------------
# The plain forms

def _positions(s):
    """Sample and position of every row of the call."""
    row = torch.arange(s["rows"], device="cuda")
    which = torch.searchsorted(s["start"], row.to(torch.int32), right=True) - 1
    return which, s["pos"][which].long() + row - s["start"][which].long()


def _plain_heads(s, x, gain, bias, pos):
    """Norm and rotation of heads x [rows, heads, h] (fp32)."""
    norm, rot = s["case"]["norm"], s["case"]["rot"]
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    if norm != "none":
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain
        if bias is not None:
            x = x + bias
    if rot:
        angle = pos.double().unsqueeze(-1) * s["freq"]                   # [rows, rot / 2]
        cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        x = torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., rot:]], -1)
    return x


def _plain_append(s):
    which, pos = _positions(s)
    page, slot = s["tables"][which, pos // s["pt"]].long(), pos % s["pt"]
    s["q_out"].copy_(_plain_heads(s, s["q"].float(), s["q_gain"], s["q_bias"], pos))
    s["data"][page, :, 0, slot] = _plain_heads(s, s["k"].float(), s["k_gain"], s["k_bias"], pos).to(s["data"].dtype)
    s["data"][page, :, 1, slot] = s["v"]
    return [s["q_out"], s["data"]]


def _plain_attend(s):
    """Every row against the positions in its sight, sample by sample and some rows at a time."""
    H, K, h, window, sinks = s["H"], s["K"], s["h"], s["window"], s["sinks"]
    G, row = H // K, 0
    for i, (T, p0) in enumerate(zip(s["lens"], s["behind"])):
        step = max(1, min(T, PLAIN_SCORES // (H * min(p0 + T, window + sinks + 256 if window else p0 + T))))
        if window:
            step = min(step, 256)
        for lo in range(0, T, step):
            m = min(step, T - lo)
            first = max(0, p0 + lo + 1 - window) if window else 0
            at = torch.arange(first, p0 + lo + m, device="cuda")
            if window and first > 0 and sinks:
                at = torch.cat([torch.arange(min(sinks, first), device="cuda"), at])
            page, slot = s["tables"][i, at // s["pt"]].long(), at % s["pt"]
            kt = s["data"][page, :, 0, slot].float().permute(1, 2, 0).contiguous()        # [K, h, positions]
            v = s["data"][page, :, 1, slot].float().permute(1, 0, 2).contiguous()
            q = s["q"][row + lo:row + lo + m].float().reshape(m, K, G, h).permute(1, 2, 0, 3).reshape(K, G * m, h)
            w = torch.matmul(q, kt).mul_(1 / math.sqrt(h)).view(K, G, m, -1)
            own_pos = (p0 + lo + torch.arange(m, device="cuda")).unsqueeze(-1)
            hidden = at > own_pos
            if window:
                hidden = hidden | ((own_pos - at >= window) & (at >= sinks))
            w.masked_fill_(hidden, -math.inf)
            w = (w - w.amax(-1, keepdim=True)).exp_()
            w = w / w.sum(-1, keepdim=True)
            o = torch.matmul(w.view(K, G * m, -1), v).view(K, G, m, h).permute(2, 0, 1, 3).reshape(m, H, h)
            s["out"][row + lo:row + lo + m] = o
        row += T
    return s["out"]


def run(s):
    append = s["case"]["op"] == "append"
    if own:
        if append:
            s["cache"].append(s["plan"], s["k"], s["v"], s["q"], prep=s["prep"], q_out=s["q_out"])
            return [s["q_out"], s["data"]]
        return s["cache"].attn(s["plan"], s["q"], window=s["window"], sinks=s["sinks"], out=s["out"], workspace=s["workspace"])
    return _plain_append(s) if append else _plain_attend(s)


# ---------------------------------------------------------------------------------------------------------------------

def work(case):
    H, K, h = HEADS[case["heads"]]
    size = {"bf16": 2, "fp32": 4}[case["dtype"]]
    lens, behind = _rows(case)
    rows = sum(lens)
    if case["op"] == "append":
        # three operations a rotated channel, six a normalised one
        each = (H + K) * ((3 * case["rot"]) + (0 if case["norm"] == "none" else 6 * h))
        return {"bytes": 2 * rows * (H + 2 * K) * h * size, "flops": rows * each}
    window, sinks = case["window"], case["sinks"]
    cached = pairs = 0
    for T, p0 in zip(lens, behind):
        if not window:
            cached += p0 + T
            pairs += T * p0 + T * (T + 1) // 2
            continue
        first = max(0, p0 + 1 - window)
        cached += p0 + T - first + min(sinks, first)
        pairs += sum(min(p + 1, window) + min(sinks, max(0, p + 1 - window)) for p in range(p0, p0 + T))
    return {"bytes": cached * K * 2 * h * size + 2 * rows * H * h * size, "flops": 4 * pairs * H * h}


def exact(case, seed):
    s = _inputs(case, seed)
    H, K, h, pt = s["H"], s["K"], s["h"], s["pt"]
    if case["op"] == "append":
        q_out = torch.empty((s["rows"], H, h), dtype=torch.float64, device="cuda")
        pool = s["data"].double()
        half, at = case["rot"] // 2, 0
        for i, (T, p0) in enumerate(zip(s["lens"], s["behind"])):
            where = torch.arange(p0, p0 + T, device="cuda")
            turn = torch.polar(torch.ones((T, 1, half), dtype=torch.float64, device="cuda"), torch.outer(where.double(), s["freq"]).unsqueeze(1))
            page, slot = s["tables"][i, where // pt].long(), where % pt
            for name in ("q", "k"):
                x = s[name][at:at + T].double()
                if case["norm"] != "none":
                    centre = torch.sum(x, -1, keepdim=True) / h if case["norm"] == "layer" else 0.0
                    spread = torch.linalg.vector_norm(x - centre, dim=-1, keepdim=True) ** 2 / h
                    x = (x - centre) * torch.rsqrt(spread + EPS) * s[name + "_gain"].double()
                    if s[name + "_bias"] is not None:
                        x = x + s[name + "_bias"].double()
                if half:
                    z = torch.complex(x[..., :half], x[..., half:2 * half]) * turn
                    x = torch.cat([z.real, z.imag, x[..., 2 * half:]], -1)
                if name == "q":
                    q_out[at:at + T] = x
                else:
                    pool[page, :, 0, slot] = x
            pool[page, :, 1, slot] = s["v"][at:at + T].double()
            at += T
        return [q_out, pool]
    # in 64 bits, a head at a time
    G, window, sinks = H // K, s["window"], s["sinks"]
    out = torch.empty((s["rows"], H, h), dtype=torch.float64, device="cuda")
    at = 0
    for i, (T, p0) in enumerate(zip(s["lens"], s["behind"])):
        every = torch.arange(p0 + T, device="cuda")
        stays = (every < sinks) | (every > p0 - window) if window else every >= 0
        every = every[stays]                                             # what some row of the sample sees
        page, slot = s["tables"][i, torch.div(every, pt, rounding_mode="floor")].long(), every % pt
        for kv in range(K):
            k = s["data"][page, kv, 0, slot].double()
            v = s["data"][page, kv, 1, slot].double()
            for lo in range(0, T, 1024):
                m = min(1024, T - lo)
                mine = p0 + lo + torch.arange(m, device="cuda").unsqueeze(1)
                cols = every.unsqueeze(0)
                seen = cols <= mine
                if window:
                    seen = seen & ((cols > mine - window) | (cols < sinks))
                for head in range(kv * G, (kv + 1) * G):
                    q = s["q"][at + lo:at + lo + m, head].double()
                    x = torch.mm(q, k.t().contiguous()) / math.sqrt(h)
                    x = torch.where(seen, x, torch.full_like(x, -math.inf))
                    p = torch.softmax(x, -1)
                    out[at + lo:at + lo + m, head] = torch.mm(p, v)
        at += T
    return out
