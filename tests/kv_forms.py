"""Calls of attention over the cache in the storage type, one for every form of its kernels.  Which form serves a call is asked of the plan itself
(csrc/kv_plan.h), so a call is found for a form whatever the plan's constants are."""
import functools
import os
import subprocess
import tempfile

import numpy as np
import torch

BF16, F32 = torch.bfloat16, torch.float32

_PLAN = r"""
#include <cstdio>
#include "kv_plan.h"
int main() {
  int dtype, K, h, packed, n, n_rows, max_ctx, H, window, sinks, some;
  while (std::scanf("%d %d %d %d %d %d %d %d %d %d", &dtype, &K, &h, &packed, &n, &n_rows, &max_ctx, &H, &window, &sinks) == 10) {
    mdi::KvCache c{};
    c.K = K; c.h = h; c.dtype = dtype;
    const mdi::KvRows r{nullptr, packed ? &some : nullptr, nullptr, n, n_rows, max_ctx};
    const int all = 1 << 30;
    const mdi::KvSight w{window ? window : all, window ? sinks : 0};
    const mdi::KvPlan p = mdi::kv_plan(c, r, H, w);
    std::printf("%d %d %d %d %d %d %d %d\n", (int)p.kernel, p.chunk, p.splits, p.wgs, p.groups, p.rows, (int)mdi::kv_decode_once(c, r, w), mdi::kv_padded(h));
  }
}
"""
MANY = 384                                                        # samples; more of them are searched for (kInOrder)


@functools.lru_cache(None)
def _program():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    d = _program.dir.name
    src, exe = os.path.join(d, "plan.cpp"), os.path.join(d, "plan")
    open(src, "w").write(_PLAN)
    subprocess.run(["g++", "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
                    "-I", os.path.join(root, "paper_2505_18164_amd", "csrc"), "-I", os.path.join(root, "include"), src, "-o", exe], check=True)
    return exe


_program.dir = tempfile.TemporaryDirectory()


def plans(calls):
    """Of every (dtype, K, h, packed, n, n_rows, max_ctx, H, window, sinks): kernel, chunk, splits, wgs, groups, rows, once, padded."""
    lines = ["%d %d %d %d %d %d %d %d %d %d" % ((1 if c[0] == BF16 else 0,) + tuple(c[1:])) for c in calls]
    out = subprocess.run([_program()], input="\n".join(lines) + "\n", check=True, capture_output=True, text=True).stdout.splitlines()
    return [[int(x) for x in line.split()] for line in out]


def form(call, pt, plan):
    """What of the kernels serves it: their instances, and whether the work is divided."""
    dtype, K, h, packed, n = call[:5]
    kernel, _, splits, wgs, groups, rows, once, padded = plan
    add = lambda text, *on: text + "".join(" " + name for name, x in on if x)
    if kernel == 0:
        return add(f"decode {h}", ("whole", pt % 16 == 0), ("once", once), ("shares", wgs), ("of many", wgs and n > 64))
    if kernel == 2:
        how = f"{groups} sets" if packed else "tokens"
        return add(f"any {'bf16' if dtype == BF16 else 'f32'} {padded} {how}", ("many", packed and n > MANY), ("pieces", splits > 1))
    which = f"prompt {groups} groups" if h == 64 else "wide 4 by 2" if groups == 2 else "wide 4" if rows == 256 else "wide 2"
    return add(which, ("whole", pt % 64 == 0), ("many", n > MANY), ("pieces", splits > 1))


def _all_forms():
    mix = lambda names: [" ".join([""] + [x for i, x in enumerate(names) if m >> i & 1]) for m in range(1 << len(names))]
    f = [f"decode {h}{x}{y}" for h in (64, 128) for x in mix(["whole", "once"]) for y in ("", " shares", " shares of many")]
    for t, size in (("bf16", 2), ("f32", 4)):
        for p in (32, 64, 128, 256):
            f += [f"any {t} {p} tokens{x}" for x in mix(["pieces"])] + [f"any {t} {p} 1 sets{x}" for x in mix(["many", "pieces"])]
            if p * size <= 256:
                f += [f"any {t} {p} 2 sets{x}" for x in mix(["many"])]       # (so many workgroups are not divided)
    f += [f"{k}{x}" for k in ("prompt 1 groups", "prompt 2 groups", "wide 4", "wide 4 by 2", "wide 2") for x in mix(["whole", "many", "pieces"])]
    # (rows of so many samples that are few enough to be divided are other kernels': of 1.8 million calls with sizes drawn over all the limits
    # none had these)
    return [x for x in f if not (x.startswith(("prompt 1", "wide 4")) and x.endswith("many pieces"))]


FORMS = _all_forms()
# Calls with a window that are not tried: what they see would have to be tens of thousands of positions.
NO_WINDOW = [f"{k}{w} many pieces" for k in ("prompt 2 groups", "wide 2") for w in ("", " whole")]


def _candidates():
    """Calls, the cheap ones first: what kv_cases.Setup takes, and max_ctx and one_each."""
    rng = np.random.default_rng(0)
    many = [int(x) for x in rng.integers(0, 3, 400)]
    far = [int(x) for x in rng.integers(0, 90, 400)]
    few = [5 if i == 7 else 2 if i == 300 else 1 if i == 399 else 0 for i in range(400)]
    packed = [([20, 3, 40], [0, 40, 300]), ([30, 9], [2900, 1500]), ([3], [2500]), ([100, 64, 80, 90], [3000, 2500, 2900, 2000]), (many, far), (few, [2500 if t > 1 else 40 for t in few])]
    tokens = [[1, 17, 200, 64, 250], [1, 17, 300, 64, 1000, 2], [2600, 90], [int(x) for x in rng.integers(1, 600, 50)], [int(x) for x in rng.integers(1, 600, 300)]]
    sights = {False: [(0, 0)], True: [(50, 3), (700, 65), (1800, 100), (6000, 100)]}
    for H, K in ((4, 2), (4, 1), (32, 2), (32, 4), (8, 8)):
        for h in (24, 32, 40, 64, 96, 128, 256):
            for dtype in (BF16, F32):
                for pt in (64, 24, 16):
                    for window in sights:
                        for sight in sights[window]:
                            for lens, behind in packed:
                                real = max(a + b for a, b in zip(lens, behind))
                                for crowd in (0, 3000, 10000, 30000, 80000, 200000, 800000):
                                    yield window, dict(H=H, K=K, h=h, pt=pt, lens=lens, behind=behind, dtype=dtype, window=sight[0], sinks=sight[1], rows_behind=crowd // H), real, False
                            for ctx in tokens:
                                for top in (0, 150000):
                                    yield window, dict(H=H, K=K, h=h, pt=pt, lens=[1] * len(ctx), behind=[c - 1 for c in ctx], dtype=dtype, window=sight[0], sinks=sight[1],
                                                       spare=2 + top // pt), max(max(ctx), top), True
    long = [20000 if t > 1 else 40 for t in few]
    for pt in (64, 24):
        for H, h, crowd, top in ((64, 64, 24, 34054), (64, 64, 24, 60000), (64, 64, 56, 60000), (32, 128, 820, 20600), (32, 128, 820, 34000)):
            yield False, dict(H=H, K=1, h=h, pt=pt, lens=few, behind=long, dtype=BF16, window=0, sinks=0, rows_behind=crowd, spare=2 + (top - 20000) // pt), top, False


@functools.lru_cache(None)
def calls():
    """{(form, with a window): (what Setup takes, max_ctx, one token each)}, the first candidate of each."""
    every = list(_candidates())
    asked = [(s["dtype"], s["K"], s["h"], int(not one), len(s["lens"]), sum(s["lens"]) + s.get("rows_behind", 0), ctx, s["H"], s["window"], s["sinks"]) for _, s, ctx, one in every]
    found = {}
    for (window, s, ctx, one), call, plan in zip(every, asked, plans(asked)):
        if call[5] * call[7] < 1 << 24:
            found.setdefault((form(call, s["pt"], plan), window), (s, ctx, one))
    return found


def ones(K, h, border):
    """For Setup's `change`: keys of zeros, and a one per position in one of its sample's K * h channels - of more than a hundred for each
    channel those about multiples of `border`, and the first and last ones."""
    def change(_, x):
        n = x.shape[1]
        p = np.arange(n)
        if n > 100 * K * h:
            p = p[(p < 64) | (p >= n - 64) | ((p + 64) % border < 128)]
        x[0] = 0
        x[1] = 0
        x[1, p, p % (K * h) // h, p % h] = 1
    return change
