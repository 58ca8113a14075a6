"""The cache in the storage type through the C ABI: rows appended with norms and rotation, attention with a window or without, against
64 bits."""
import numpy as np
import pytest
import torch

from kv_cases import HALF, Setup, attention, bound, dev, heads, within
from kv_forms import plans
from paper_2505_18164_amd import mdi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
TYPES = dict(argvalues=[BF16, F32], ids=["bf16", "f32"])

APPEND = [  # H, K, h, page tokens, new rows, positions behind, channels that turn
    (1, 1, 8, 1, [1], [0], 8),
    (4, 2, 64, 16, [5, 0, 40], [3, 7, 0], 64),
    (10, 5, 128, 24, [33, 1, 2], [100, 0, 23], 128),
    (6, 3, 40, 7, [20, 9], [1, 0], 40),
    (32, 8, 128, 64, [3], [61], 64),
    (4, 1, 256, 5, [11] * 3, [0, 4, 9], 256),
    (8, 4, 64, 32, [1] * 70, list(range(70)), 32),
    (3, 3, 96, 16, [17, 2], [0, 30], 24),
    (2, 2, 72, 9, [10], [5], 16),
    (32, 32, 128, 16, [9, 4], [0, 77], 0),
]


def appended(H, K, h, pt, lens, behind, rot, dtype, norm, g=None, seed=0, in_place=False, queries=True, q_gain=True, k_gain=True, bias=True, freq=None, scale=1.0, spare_rows=3):
    """Append such rows and check everything that was and was not written."""
    rng = np.random.default_rng(seed)
    total = [a + b for a, b in zip(lens, behind)]
    used = [(t + pt - 1) // pt for t in total]
    n_pages, rows, n = sum(used) + 2, sum(lens), len(lens)
    order = rng.permutation(n_pages).astype(np.int32)
    tables = np.full((n, max(used) + 1), -5, dtype=np.int32)
    for i in range(n):
        tables[i, :used[i]] = order[sum(used[:i]):sum(used[:i + 1])]
    size = scale * np.exp(rng.uniform(-6, 6, (rows + spare_rows, H + 2 * K, 1)))
    fused = torch.from_numpy(rng.standard_normal((rows + spare_rows, H + 2 * K, h)) * size).to(dtype).to(DEV)
    before = fused.clone()
    data = torch.from_numpy(rng.standard_normal((n_pages, K, 2, pt, h)).astype(np.float32)).to(dtype)
    vec = lambda on, about: torch.from_numpy((about + 0.3 * rng.standard_normal(h)).astype(np.float32)).to(DEV) if on else None
    named = {"q_gain": vec(q_gain and norm, 1), "k_gain": vec(k_gain and norm, 1), "q_bias": vec(q_gain and norm and bias, 0), "k_bias": vec(k_gain and norm and bias, 0)}
    freq = (mdi.rope_freq(rot) if rot else None) if freq is None else freq
    cache = mdi.KvCache(data.to(DEV), dev(tables), torch.zeros(1, dtype=torch.int32, device=DEV))
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    plan = cache.rows(dev(np.asarray(behind, np.int32)), start=dev(start), n_rows=rows + spare_rows)
    prep = cache.prep(freq=freq, norm=norm or "rms", eps=1e-5, **named) if (norm or rot) else None
    q, k, v = fused[:, :H], fused[:, H:H + K], fused[:, H + K:]
    out = q if in_place else torch.full((rows + spare_rows, H, h), 7.0, dtype=dtype, device=DEV)
    if queries and in_place:
        out = q = q.contiguous()
        assert cache.append(plan, k, v, q, prep, q_out=q) is q
    elif queries:
        assert cache.append(plan, k, v, q, prep, q_out=out) is out
    else:
        assert cache.append(plan, k, v, prep=prep) is None
        assert torch.equal(out, torch.full_like(out, 7.0))
    assert torch.equal(fused, before)
    cache.check()

    pos = np.concatenate([np.arange(b, b + t) for b, t in zip(behind, lens)] + [[]]).astype(np.int64)
    x = before.cpu().double().numpy()
    f = freq.cpu().numpy() if freq is not None else None
    host = {name: None if t is None else t.cpu().double().numpy() for name, t in named.items()}
    want_q = heads(x[:rows, :H], pos, host["q_gain"], host["q_bias"], norm, 1e-5, f)
    want_k = heads(x[:rows, H:H + K], pos, host["k_gain"], host["k_bias"], norm, 1e-5, f)
    if queries:
        within(out[:rows], want_q[0], want_q[1] + HALF[dtype] * (np.abs(want_q[0]) + want_q[1]) + 1e-30, "q")
        assert torch.equal(out[rows:], before[rows:, :H] if in_place else torch.full_like(out[rows:], 7.0))
    got = cache.data.cpu()
    where = np.repeat(np.arange(n), lens)
    page, slot = tables[where, pos // pt], pos % pt
    k_got, v_got = got[page, :, 0, slot], got[page, :, 1, slot]
    within(k_got, want_k[0], want_k[1] + HALF[dtype] * (np.abs(want_k[0]) + want_k[1]) + 1e-30, "k")
    assert torch.equal(v_got, before[:rows, H + K:].cpu())
    data[page, :, 0, slot], data[page, :, 1, slot] = k_got, v_got
    assert torch.equal(got, data)                                  # the written rows, and nothing else


@pytest.mark.parametrize("dtype", **TYPES)
@pytest.mark.parametrize("norm", [None, "rms", "layer"])
@pytest.mark.parametrize("case", APPEND, ids=[f"{c[0]}of{c[1]}x{c[2]}-turn{c[6]}" for c in APPEND])
def test_rows_appended(case, norm, dtype):
    appended(*case, dtype, norm, seed=sum(case[:4]))


@pytest.mark.parametrize("dtype", **TYPES)
def test_rows_appended_in_place_without_queries_and_with_half_of_a_norm(dtype):
    case = (8, 2, 64, 16, [5, 33], [3, 0], 64)
    appended(*case, dtype, "rms", in_place=True)
    appended(*case, dtype, "layer", in_place=True)
    appended(*case, dtype, "rms", queries=False)
    appended(*case, dtype, None, queries=False)
    appended(*case, dtype, "rms", q_gain=False)
    appended(*case, dtype, "layer", k_gain=False, bias=False)
    appended(8, 2, 64, 16, [0, 0], [3, 0], 64, dtype, "rms")


@pytest.mark.parametrize("dtype", **TYPES)
def test_far_positions_turn_as_they_should(dtype):
    """Angles of 2^24 turns and more, and frequencies that are not of the usual kind."""
    H, K, h, pt = 4, 2, 64, 64
    at = np.array([0, 1, 4095, 120001, (1 << 24) - 1], np.int64)
    rng = np.random.default_rng(3)
    tables = np.full((5, 1 << 18), -1, np.int32)
    tables[np.arange(5), at // pt] = [4, 0, 3, 1, 2]
    freq = mdi.rope_freq(h)
    freq[3], freq[5], freq[7] = 3.1, -0.7, 0.0
    cache = mdi.KvCache(torch.zeros((5, K, 2, pt, h), dtype=dtype, device=DEV), dev(tables), torch.zeros(1, dtype=torch.int32, device=DEV))
    x = torch.from_numpy(rng.standard_normal((5, H + 2 * K, h))).to(dtype).to(DEV)
    q = cache.append(cache.rows(dev(at.astype(np.int32))), x[:, H:H + K], x[:, H + K:], x[:, :H], cache.prep(freq=freq))
    cache.check()
    want, off = heads(x.cpu().double().numpy(), at, freq=freq.cpu().numpy())
    off = off + 1e-9 * np.abs(want) + HALF[dtype] * (np.abs(want) + off)
    within(q, want[:, :H], off[:, :H])
    page = np.array([4, 0, 3, 1, 2])
    within(cache.data.cpu()[page, :, 0, at % pt], want[:, H:H + K], off[:, H:H + K])


def test_appends_of_samples_that_take_no_part_and_other_tables():
    rng = np.random.default_rng(5)
    K, h, pt = 2, 64, 16
    x = torch.from_numpy(rng.standard_normal((4, 8, h)).astype(np.float32)).to(DEV)
    cache = mdi.KvCache(torch.full((4, K, 2, pt, h), 9.0, device=DEV), dev(np.array([[3, 0], [2, 0], [1, 0]], np.int32)), torch.zeros(1, dtype=torch.int32, device=DEV))
    plan = cache.rows(dev(np.array([4, -1, 2, 0], np.int32)), table=dev(np.array([2, 0, 0, 1], np.int32)), max_ctx=5)
    q = torch.full((4, 4, h), 3.0, device=DEV)
    cache.append(plan, x[:, 4:6], x[:, 6:], x[:, :4], q_out=q)
    want = torch.full((4, K, 2, pt, h), 9.0)
    for row, (page, slot) in {0: (1, 4), 2: (3, 2), 3: (2, 0)}.items():
        want[page, :, 0, slot], want[page, :, 1, slot] = x[row, 4:6].cpu(), x[row, 6:].cpu()
    assert torch.equal(cache.data.cpu(), want)
    assert (q[1] == 3.0).all() and torch.equal(q[[0, 2, 3]], x[[0, 2, 3], :4])
    out = cache.attn(plan, q, out=torch.full_like(q, 5.0))
    assert (out[1] == 0).all()                                    # sample 1 takes no part
    cache.check()


ATTN = [  # H, K, h, page tokens, new rows, positions behind
    (1, 1, 64, 16, [1], [0]),
    (4, 2, 64, 16, [1, 17, 0, 64, 65], [0, 0, 4, 0, 0]),
    (32, 4, 64, 24, [33, 130], [100, 0]),
    (8, 8, 128, 64, [128, 1, 63], [0, 200, 1]),
    (6, 2, 128, 7, [70], [59]),
    (10, 2, 128, 48, [40, 3], [0, 777]),
    (20, 1, 64, 1, [37], [5]),
    (16, 2, 128, 128, [300], [300]),
    (24, 4, 128, 32, [5] * 9, [0, 31, 32, 33, 63, 64, 65, 500, 1023]),
    (3, 1, 8, 4, [9, 2], [0, 3]),
    (4, 2, 40, 16, [21], [20]),
    (5, 5, 96, 16, [10, 11], [6, 0]),
    (2, 1, 256, 16, [19], [2]),
    (34, 2, 32, 64, [130, 70], [0, 40]),
]
IDS = [f"{c[0]}of{c[1]}x{c[2]}-page{c[3]}" for c in ATTN]
SIGHTS = [(0, 0), (1, 0), (1, 3), (16, 1), (50, 0), (33, 20), (64, 64), (200, 5), (5, 300), (100000, 4)]


@pytest.mark.parametrize("dtype", **TYPES)
@pytest.mark.parametrize("sight", SIGHTS, ids=[f"{w}+{s}" for w, s in SIGHTS])
@pytest.mark.parametrize("case", ATTN, ids=IDS)
def test_packed_rows_against_64_bits(case, sight, dtype):
    s = Setup(*case, dtype, *sight, seed=3, rows_behind=3)
    cache = s.cache()
    wide = torch.zeros((s.rows, s.H + 2 * s.K, s.h), dtype=dtype, device=DEV)   # the query heads of a fused product
    wide[:, :s.H] = s.q.to(DEV)
    out = torch.full((s.rows, s.H, s.h), 5.0, dtype=dtype, device=DEV)
    assert cache.attn(s.plan(cache), wide[:, :s.H], window=sight[0], sinks=sight[1], out=out) is out
    s.check(out)
    assert (out[s.start[-1]:] == 5.0).all()                       # rows of nobody
    cache.check()


# Rows of nobody behind the last sample, times heads: so many that the call is taken for a large one, for each of the ways to divide that.
CROWDS = {64: [30000, 80000], 128: [30000, 80000, 200000]}


@pytest.mark.parametrize("sight", SIGHTS, ids=[f"{w}+{s}" for w, s in SIGHTS])
@pytest.mark.parametrize("case,crowd", [(c, n) for c in ATTN for n in CROWDS.get(c[2], [])], ids=[f"{i}-of-{n}" for c, i in zip(ATTN, IDS) for n in CROWDS.get(c[2], [])])
def test_rows_of_a_large_call_against_64_bits(case, sight, crowd):
    s = Setup(*case, BF16, *sight, seed=3, rows_behind=crowd // case[0])
    cache = s.cache()
    out = torch.full((s.rows, s.H, s.h), 5.0, dtype=BF16, device=DEV)
    s.check(s.attn(cache, s.plan(cache), out=out))
    assert (out[s.start[-1]:] == 5.0).all()
    cache.check()


@pytest.mark.parametrize("dtype", **TYPES)
@pytest.mark.parametrize("sight", SIGHTS, ids=[f"{w}+{s}" for w, s in SIGHTS])
@pytest.mark.parametrize("case", ATTN, ids=IDS)
def test_one_new_token_against_64_bits(case, sight, dtype):
    H, K, h, pt, lens, behind = case
    ctx = [a + b for a, b in zip(lens, behind)]
    s = Setup(H, K, h, pt, [1] * len(ctx), [max(c, 1) - 1 for c in ctx], dtype, *sight, seed=4)
    cache = s.cache()
    s.check(s.attn(cache, s.plan(cache, one_each=True)))
    cache.check()


@pytest.mark.parametrize("sight", SIGHTS, ids=[f"{w}+{s}" for w, s in SIGHTS])
@pytest.mark.parametrize("H,K,h,pt", [(8, 2, 64, 16), (6, 3, 64, 40), (4, 2, 128, 64), (10, 2, 128, 7)])
def test_one_new_token_of_what_may_be_a_large_cache(H, K, h, pt, sight):
    """Tables for so many positions that the cache is read as a large one, with and without a window that makes it a small one after all."""
    ctx = [1, 17, 300, 0, 64, 1000]
    s = Setup(H, K, h, pt, [1] * 6, [max(c, 1) - 1 for c in ctx], BF16, *sight, seed=4, spare=150000 // pt)
    cache = s.cache()
    s.check(s.attn(cache, s.plan(cache, one_each=True, max_ctx=150000)))
    cache.check()


@pytest.mark.parametrize("dtype", **TYPES)
@pytest.mark.parametrize("one_each", [False, True], ids=["packed", "tokens"])
@pytest.mark.parametrize("sight", [(0, 0), (1700, 100)], ids=["all", "window"])
@pytest.mark.parametrize("H,K,h,pt,ctx", [(8, 2, 64, 16, [5000, 1, 300]), (4, 4, 128, 40, [2100, 2111]), (16, 1, 128, 64, [3333]), (3, 1, 32, 16, [1500]), (2, 1, 256, 128, [2600, 90])])
def test_long_contexts_are_divided_and_joined(H, K, h, pt, ctx, sight, one_each, dtype):
    s = Setup(H, K, h, pt, [1] * len(ctx), [c - 1 for c in ctx], dtype, *sight, seed=6, stale=float("inf"), rows_behind=0 if one_each else 2)
    cache = s.cache()
    plan = s.plan(cache, one_each=one_each)
    space = cache.workspace(plan, H, *sight)
    if space is not None:
        space.fill_(0xFF)                                         # NaN everywhere: nothing is taken from a workspace that the call has not put there
    want = s.want()
    first = s.attn(cache, plan, workspace=space)
    s.check(first, want)
    for _ in range(3):
        assert torch.equal(s.attn(cache, plan, workspace=space)[:len(ctx)], first[:len(ctx)])
    # divided for longer samples than there are
    long = s.plan(cache, one_each=one_each, max_ctx=s.tables.shape[1] * pt)
    s.check(s.attn(cache, long), want)
    cache.check()


@pytest.mark.parametrize("dtype", **TYPES)
@pytest.mark.parametrize("one_each", [False, True], ids=["packed", "tokens"])
def test_pieces_of_prompts_behind_long_contexts(one_each, dtype):
    """Few rows and many positions: what they see is cut into pieces, with rows that see the beginning, the end or none of one."""
    for H, K, h, pt, lens, behind, sight in ((8, 2, 128, 64, [64, 40], [3000, 2500], (0, 0)), (8, 2, 64, 24, [100, 1], [2000, 2500], (1500, 600)),
                                             (4, 4, 128, 16, [130], [1900], (1000, 0)), (4, 2, 96, 16, [30], [2100], (0, 0))):
        if one_each:
            behind, lens = [b + i for b, t in zip(behind, lens) for i in range(min(t, 3))], [1] * sum(min(t, 3) for t in lens)
        s = Setup(H, K, h, pt, lens, behind, dtype, *sight, seed=9)
        cache = s.cache()
        s.check(s.attn(cache, s.plan(cache, one_each=one_each)), what=(H, K, h, pt))
        cache.check()


@pytest.mark.parametrize("H,K,h,pt,lens,behind,sight", [
    (32, 4, 128, 64, [100, 100], [4900, 4000], (0, 0)), (32, 4, 128, 64, [100, 64, 80, 90], [3000, 2500, 2900, 2000], (0, 0)), (32, 2, 128, 24, [100, 64, 80, 90], [3000, 2500, 2900, 2000], (1500, 5)),
    (32, 4, 64, 24, [130, 100, 90, 130], [3000, 2500, 2500, 2500], (1500, 600)), (32, 4, 64, 64, [130, 100, 1, 130], [3000, 2500, 2500, 0], (0, 0))])
def test_many_heads_behind_long_contexts(H, K, h, pt, lens, behind, sight):
    s = Setup(H, K, h, pt, lens, behind, BF16, *sight, seed=5, stale=float("inf"), rows_behind=2)
    cache = s.cache()
    plan = s.plan(cache)
    space = cache.workspace(plan, H, *sight)
    space.fill_(0xFF)
    first = s.attn(cache, plan, workspace=space)
    s.check(first)
    for _ in range(3):
        assert torch.equal(s.attn(cache, plan, workspace=space)[:s.start[-1]], first[:s.start[-1]])
    cache.check()


KINDS = [(64, BF16, 0), (128, BF16, 0), (48, BF16, 0), (64, F32, 0), (128, F32, 0), (48, F32, 0)] + [(h, BF16, c) for h in CROWDS for c in CROWDS[h]]
KIND_IDS = [f"{h}-{'bf16' if d is BF16 else 'f32'}" + (f"-of-{c}" if c else "") for h, d, c in KINDS]


@pytest.mark.parametrize("h,dtype,crowd", KINDS, ids=KIND_IDS)
def test_scores_that_decide_alone_and_far_apart(h, dtype, crowd):
    """Loud keys: one position's weight is all but 1; scores of hundreds either way, growing and falling along the cache."""
    ramps = [lambda p: 0.01 + p / 8.0, lambda p: 30 - p / 8.0, lambda p: np.where(p % 67 == 66, 40.0, 0.01), lambda p: np.where(p < 200, 60.0, 0.0), lambda p: 0.0 * p]
    for seed, gain in ((1, 40.0), (2, 300.0)):
        s = Setup(4, 2, h, 16, [50, 3], [90, 400], dtype, seed=seed, k_gain=gain, rows_behind=crowd // 4)
        cache = s.cache()
        s.check(s.attn(cache, s.plan(cache)))
    for i, ramp in enumerate(ramps):
        def change(_, x):
            x[0] *= ramp(np.arange(x.shape[1]))[:, None, None].astype(np.float32)
        s = Setup(4, 2, h, 16, [40, 70], [200, 0], dtype, *((0, 0) if i % 2 else (90, 9)), seed=8, change=change, rows_behind=crowd // 4)
        cache = s.cache()
        for scale in (None, 0.0, -0.3, 2.0):
            s.check(s.attn(cache, s.plan(cache), scale=scale), s.want(scale), (i, scale))
        token = Setup(4, 2, h, 16, [1, 1], [239, 100], dtype, seed=8, change=change)
        cache = token.cache()
        token.check(token.attn(cache, token.plan(cache, one_each=True)))


GAINS = {"growing": lambda p: 2.0 ** np.minimum(p / 8.0 - 30, 60), "falling": lambda p: 2.0 ** np.maximum(20 - p / 8.0, -90),
         "tiny": lambda p: 2.0 ** -94 + 0.0 * p, "huge": lambda p: np.where(p < 100, 1.0, 2.0 ** 100), "zeros": lambda p: 0.0 * p}


@pytest.mark.parametrize("h,dtype,crowd", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("gain", list(GAINS))
def test_values_of_all_sizes(gain, h, dtype, crowd):
    for lens, behind, pt in (([150, 1, 64], [0, 330, 500], 64), ([20, 9], [900, 1500], 24)):
        s = Setup(4, 2, h, pt, lens, behind, dtype, seed=3, v_gain=GAINS[gain], rows_behind=crowd // 4)
        cache = s.cache()
        s.check(s.attn(cache, s.plan(cache)), what=(lens, pt))
    s = Setup(4, 2, h, 16, [1, 1, 1], [0, 500, 79], dtype, seed=4, v_gain=GAINS[gain])
    cache = s.cache()
    s.check(s.attn(cache, s.plan(cache, one_each=True)))


@pytest.mark.parametrize("h,dtype,crowd", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("sight", [(0, 0), (25, 2)], ids=["all", "window"])
def test_what_is_not_finite_reaches_only_rows_that_see_it(sight, h, dtype, crowd):
    """A value that is infinite in one channel, one that is NaN in another, a key with a NaN: those that do not see them are what they are
    without them."""
    T, p0, window = 100, 30, sight[0]
    for what, p in (("inf", 60), ("-inf", 60), ("nan", 61), ("key", 62), ("two", 60)):
        def change(_, x):
            if what == "key":
                x[0, p, 1, 5] = np.nan
            else:
                x[1, p, 1, 3] = {"inf": np.inf, "-inf": -np.inf, "nan": np.nan, "two": np.inf}[what]
            if what == "two":
                x[1, 20, 1, 3] = -np.inf
        s = Setup(4, 2, h, 16, [T], [p0], dtype, *sight, seed=2, change=change, rows_behind=crowd // 4)
        clean = Setup(4, 2, h, 16, [T], [p0], dtype, *sight, seed=2)
        cache = s.cache()
        out = s.attn(cache, s.plan(cache))[:T]
        tokens = cache.rows(dev(np.arange(p0, p0 + T).astype(np.int32)), table=dev(np.zeros(T, np.int32)), max_ctx=p0 + T)
        each = cache.attn(tokens, s.q[:T].to(DEV), window=sight[0], sinks=sight[1])
        want, mag, big, n = clean.want()
        may = bound(want, mag, big, n, h, dtype)
        pos = p0 + np.arange(T)
        hit = np.zeros((T, 4, h), bool)
        sees_p = (pos >= p) & ((pos - p < window) if window else True)
        sees_20 = (pos >= 20) & ((pos - 20 < window) if window else True)
        if what == "key":
            hit[sees_p, 2:] = True
        else:
            hit[sees_p, 2:, 3] = True
            if what == "two":
                hit[sees_20, 2:, 3] = True
        for got in (out, each):
            got = got.float().cpu().double().numpy()
            within(np.where(hit, 0, got), np.where(hit, 0, want), np.where(hit, 1, may), what)
            if what == "inf":
                assert (got[sees_p, 2:, 3] == np.inf).all()
            elif what == "-inf":
                assert (got[sees_p, 2:, 3] == -np.inf).all()
            elif what != "two":
                assert np.isnan(got[hit]).all()
            else:
                assert np.isnan(got[sees_p & sees_20, 2:, 3]).all() and (got[sees_20 & ~sees_p, 2:, 3] == -np.inf).all()


@pytest.mark.parametrize("h,dtype,crowd", [(24, BF16, 0), (24, F32, 0)] + [k for k in KINDS if k[0] != 48], ids=["24-bf16", "24-f32"] + [i for k, i in zip(KINDS, KIND_IDS) if k[0] != 48])
def test_what_is_not_of_the_cache_is_reported(h, dtype, crowd):
    for what in ("page", "negative page", "table", "position"):
        for op in ("append", "attn", "tokens", "window"):
            s = Setup(4, 2, h, 16, [20, 3], [0, 40], dtype, seed=1, rows_behind=crowd // 4)
            if what == "page":
                s.tables[0, 1] = s.data.shape[0]
            if what == "negative page":
                s.tables[0, 1] = -1
            table = dev(np.array([0, 2 if what == "table" else 1], np.int32))
            max_ctx = 42 if what == "position" else s.max_ctx
            q, k = s.q.to(DEV), torch.randn((s.rows, 2, h), device=DEV).to(dtype)
            cache = s.cache()
            plan = s.plan(cache, table=table, max_ctx=max_ctx)
            tokens = cache.rows(dev(np.array([19, 42], np.int32)), table=table, max_ctx=max_ctx)

            def call(cache):
                if op == "tokens":
                    cache.attn(tokens, q[:2].contiguous())
                elif op == "append":
                    cache.append(plan, k, k.clone(), q, cache.prep(freq=mdi.rope_freq(h)))
                else:
                    cache.attn(plan, q, window=8 if op == "window" else 0, sinks=2 if op == "window" else 0)

            call(cache)
            with pytest.raises(mdi.MdiError) as e:
                cache.check()
            assert e.value.status == mdi.MDI_ERR_ARG, (what, op)
            call(s.cache(err=False))                              # nobody asks: nothing is written
            torch.cuda.synchronize()


@pytest.mark.parametrize("h,crowd", [(128, 0), (96, 0), (128, 30000), (128, 80000), (128, 200000), (64, 80000)])
def test_offsets_past_32_bits(h, crowd):
    """The last pages of a pool of 4.5 GiB."""
    K, pt, H = 8, 64, 16
    n_pages = (9 << 29) // (K * 2 * pt * h * 2)
    data = torch.empty((n_pages, K, 2, pt, h), dtype=BF16, device=DEV)
    tables = dev(np.array([[n_pages - 1, 0, n_pages - 2]], np.int32))
    cache = mdi.KvCache(data, tables, torch.zeros(1, dtype=torch.int32, device=DEV))
    T = 150
    x = torch.randn((T, H + 2 * K, h), device=DEV).to(BF16)
    plan = cache.rows(dev(np.array([0], np.int32)), start=dev(np.array([0, T], np.int32)), n_rows=T, max_ctx=T)
    large = cache.rows(dev(np.array([0], np.int32)), start=dev(np.array([0, T], np.int32)), n_rows=T + crowd // H, max_ctx=T)
    q = cache.append(plan, x[:, H:H + K], x[:, H + K:], x[:, :H])
    assert torch.equal(q, x[:, :H])
    host = x.cpu().double().numpy()
    many = torch.cat([q, torch.zeros((crowd // H, H, h), dtype=BF16, device=DEV)])
    for window, sinks in ((0, 0), (40, 3)):
        want = attention(host[:, :H], host[:, H:H + K], host[:, H + K:], 0, h ** -0.5, window, sinks)
        within(cache.attn(large, many, window=window, sinks=sinks)[:T], want[0], bound(*want, h, BF16))
        last = cache.rows(dev(np.array([T - 1], np.int32)), max_ctx=T)
        within(cache.attn(last, q[T - 1:], window=window, sinks=sinks), want[0][T - 1:], bound(*[w[T - 1:] for w in want], h, BF16))
    cache.check()


@pytest.mark.parametrize("dtype", **TYPES)
@pytest.mark.parametrize("H,K,h,pt,window,sinks,norm", [(8, 2, 64, 16, 0, 0, None), (4, 4, 128, 24, 70, 4, "rms"), (6, 2, 40, 16, 33, 0, "layer"), (8, 1, 128, 64, 100, 20, "rms")])
def test_prompts_and_tokens_one_after_the_other(H, K, h, pt, window, sinks, norm, dtype):
    """As a program uses them: prompts of two samples, another piece, then single tokens, pages given out as positions need them and taken
    back (and handed on) behind the window; every call is compared with all of the sample's rows in 64 bits."""
    rng = np.random.default_rng(11)
    n_pages, stride = 24 if window else 80, 64
    free = list(rng.permutation(n_pages))
    tables = np.full((2, stride), -1, np.int32)
    cache = mdi.KvCache(torch.full((n_pages, K, 2, pt, h), float("nan"), dtype=dtype, device=DEV), dev(tables), torch.zeros(1, dtype=torch.int32, device=DEV))
    g = torch.from_numpy((1 + 0.2 * rng.standard_normal(h)).astype(np.float32)).to(DEV)
    prep = cache.prep(freq=mdi.rope_freq(h, 500.0), norm=norm or "rms", q_gain=g if norm else None, k_gain=g if norm else None)
    freq, gain = mdi.rope_freq(h, 500.0).cpu().numpy(), g.cpu().double().numpy() if norm else None
    past = [[np.zeros((0, K, h)), np.zeros((0, K, h))] for _ in range(2)]
    steps = [[90, 17], [40, 0], [1, 1], [1, 1], [0, 30], [1, 1], [70, 1], [1, 1]]
    for lens in steps:
        behind = [p[0].shape[0] for p in past]
        for i in range(2):
            for at in range(stride):
                lo, hi = at * pt, (at + 1) * pt
                if lens[i] and window and tables[i, at] >= 0 and hi <= behind[i] + 1 - window and lo >= sinks:
                    free.insert(0, tables[i, at])                 # nobody sees it any more
                    cache.data[int(tables[i, at])] = float("nan")
                    tables[i, at] = -1
                if lens[i] and hi > behind[i] and lo < behind[i] + lens[i] and tables[i, at] < 0:
                    tables[i, at] = free.pop()
        cache.tables.copy_(torch.from_numpy(tables))
        rows = sum(lens)
        x = torch.from_numpy(rng.standard_normal((rows, H + 2 * K, h)).astype(np.float32)).to(dtype).to(DEV)
        start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        one_each = lens == [1, 1]
        plan = cache.rows(dev(np.asarray(behind, np.int32)), start=None if one_each else dev(start), n_rows=rows, max_ctx=max(a + b for a, b in zip(behind, lens)))
        q = cache.append(plan, x[:, H:H + K], x[:, H + K:], x[:, :H], prep)
        out = cache.attn(plan, q, window=window, sinks=sinks)
        host = x.cpu().double().numpy()
        for i in range(2):
            if not lens[i]:
                continue
            mine = slice(start[i], start[i + 1])
            pos = behind[i] + np.arange(lens[i])
            want_q, off_q = heads(host[mine, :H], pos, gain, None, norm, 1e-6, freq)
            want_k, off_k = heads(host[mine, H:H + K], pos, gain, None, norm, 1e-6, freq)
            within(q[mine], want_q, off_q + HALF[dtype] * (np.abs(want_q) + off_q))
            kept = cache.data.cpu().double().numpy()[tables[i, pos // pt], :, :, pos % pt]
            within(kept[:, :, 0], want_k, off_k + HALF[dtype] * (np.abs(want_k) + off_k))
            past[i][0] = np.concatenate([past[i][0], kept[:, :, 0]])
            past[i][1] = np.concatenate([past[i][1], host[mine, H + K:]])
            want = attention(q[mine].cpu().double().numpy(), past[i][0], past[i][1], behind[i], h ** -0.5, window, sinks)
            within(out[mine], want[0], bound(*want, h, dtype), lens)
    cache.check()


@pytest.mark.parametrize("h,dtype,rows", [(64, BF16, 8), (128, BF16, 8), (96, BF16, 8), (64, F32, 8), (64, BF16, 10000), (128, BF16, 4000), (128, BF16, 10000)])
def test_captured_calls_replayed_with_later_positions(h, dtype, rows):
    """Two graphs that share a workspace - rows appended and attended to, for single tokens and for packed rows -, replayed in turns with
    the program's own work between, each replay against the eager result."""
    H, K, pt, ctx = 8, 2, 16, 2000
    s = Setup(H, K, h, pt, [5, 3], [ctx, 700], dtype, seed=12, spare=8)
    for i, total in enumerate((ctx + 5, 703)):
        s.tables[i, (total + pt - 1) // pt:][:8] = np.arange(8) + 8 * i + s.data.shape[0]
    s.data = torch.cat([s.data, torch.zeros((16,) + s.data.shape[1:], dtype=dtype)])
    s.data = torch.nan_to_num(s.data)
    top = s.tables.shape[1] * pt
    cache = s.cache()
    freq = mdi.rope_freq(h)
    prep = cache.prep(freq=freq)
    pos = [torch.zeros(2, dtype=torch.int32, device=DEV) for _ in range(2)]
    tokens = cache.rows(pos[0], max_ctx=top)
    packed = cache.rows(pos[1], start=dev(np.array([0, 5, 8], np.int32)), n_rows=rows, max_ctx=top)
    x = [torch.randn((m, H + 2 * K, h), device=DEV).to(dtype) for m in (2, rows)]
    spaces = [cache.workspace(p, H, 900, 4) for p in (tokens, packed)]
    both = max((w for w in spaces if w is not None), key=lambda w: w.numel(), default=None)
    outs = [torch.zeros((m, H, h), dtype=dtype, device=DEV) for m in (2, rows)]
    qs = [torch.zeros((m, H, h), dtype=dtype, device=DEV) for m in (2, rows)]

    def run(i, workspace):
        plan = (tokens, packed)[i]
        cache.append(plan, x[i][:, H:H + K], x[i][:, H + K:], x[i][:, :H], prep, q_out=qs[i])
        cache.attn(plan, qs[i], window=900, sinks=4, out=outs[i], workspace=workspace)

    graphs = []
    for i in range(2):
        pos[i].copy_(torch.tensor([10, 20], dtype=torch.int32))
        run(i, both)                                              # (kernels are loaded before they are captured)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(i, both)
        graphs.append(g)
    for turn in range(4):
        for i in range(2):
            pos[i].copy_(torch.tensor([ctx + 5 * turn, 700 + 40 * turn], dtype=torch.int32))
            x[i].copy_(torch.randn(x[i].shape, device=DEV))
            if both is not None:
                both.fill_(0xFF)
            graphs[i].replay()
            torch.cuda.synchronize()
            got = outs[i].clone()
            outs[i].zero_()
            run(i, None)
            torch.cuda.synchronize()
            assert torch.equal(got[:8], outs[i][:8]), (turn, i)
    cache.check()


def test_two_calls_at_once_on_other_streams():
    made = []
    for seed in range(2):
        s = Setup(16, 4, 128, 64, [40, 200], [1800, 0], seed=seed)
        made.append((s, s.cache()))
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for i, (s, cache) in enumerate(made):
        with torch.cuda.stream(streams[i]):
            plan, q = s.plan(cache), s.q.to(DEV)
            space = cache.workspace(plan, s.H)
            for _ in range(20):
                outs[i] = cache.attn(plan, q, workspace=space)
    torch.cuda.synchronize()
    for (s, cache), out in zip(made, outs):
        s.check(out)
        cache.check()


@pytest.mark.parametrize("dtype,crowd", [(BF16, 0), (F32, 0), (BF16, 1500000)], ids=["bf16", "f32", "bf16-large"])
def test_many_samples(dtype, crowd):
    """More samples than a wavefront looks at at a time, with empty ones between, packed and one token each."""
    rng = np.random.default_rng(4)
    lens = [int(x) for x in rng.integers(0, 4, 700)]
    behind = [int(x) for x in rng.integers(0, 90, 700)]
    for h in (64, 128) if crowd else (64, 48):
        for sight in ((0, 0), (20, 3)):
            s = Setup(4, 2, h, 16, lens, behind, dtype, *sight, seed=1, rows_behind=crowd // 4)
            cache = s.cache()
            s.check(s.attn(cache, s.plan(cache)))
            t = Setup(4, 2, h, 16, [1] * 700, behind, dtype, *sight, seed=2)
            cache = t.cache()
            t.check(t.attn(cache, t.plan(cache, one_each=True)))


@pytest.mark.parametrize("h,dtype,crowd", KINDS, ids=KIND_IDS)
def test_samples_that_take_no_part_may_have_any_table(h, dtype, crowd):
    """An idle place of a server's batch: no position, and the table number of a sample that is gone.  Nothing depends on it, so nothing is
    reported; appended rows and queries of it are left as they are, its results are zeros."""
    s = Setup(4, 2, h, 16, [20, 3, 40], [0, 40, 700], dtype, seed=1, rows_behind=crowd // 4)
    pos, table = dev(np.array([0, -1, 700], np.int32)), dev(np.array([0, 10 ** 9, 2], np.int32))
    cache = s.cache()
    k = torch.randn((s.rows, 2, h), device=DEV).to(dtype)
    for behind in (0, 3000):                                      # divided into pieces, too
        plan = cache.rows(pos, start=dev(s.start), table=table, n_rows=s.rows, max_ctx=min(s.max_ctx + behind, s.tables.shape[1] * 16))
        out = s.attn(cache, plan)
        assert (out[20:23] == 0).all()
        want = s.want()
        may = bound(*want, h, dtype)
        rows = np.r_[0:20, 23:63]
        within(out[rows], want[0][rows], may[rows])
    tokens = cache.rows(dev(np.array([19, -1, 739], np.int32)), table=table)
    out = cache.attn(tokens, s.q[[19, 22, 62]].to(DEV))
    assert (out[1] == 0).all()
    within(out[[0, 2]], want[0][[19, 62]], may[[19, 62]])
    q = torch.full((3, 4, h), 5.0, device=DEV).to(dtype)
    cache.append(tokens, k[:3], k[:3].clone(), q.clone(), cache.prep(freq=mdi.rope_freq(h)), q_out=q)
    assert (q[1] == 5.0).all()
    cache.check()


@pytest.mark.parametrize("H,K,h,pt,lens,behind,rise,value", [
    (32, 4, 128, 64, [100, 100], [4900, 4000], 11.0, 1.5 * 2.0 ** 100), (32, 4, 128, 64, [100, 64, 80, 90], [3000, 2500, 2900, 2000], 11.0, 1.5 * 2.0 ** 100),
    (32, 2, 128, 24, [100, 64, 80, 90], [3000, 2500, 2900, 2000], 11.0, 1.5 * 2.0 ** 100), (16, 16, 128, 64, [64], [4000], 11.0, 1.5 * 2.0 ** 100), (8, 8, 128, 64, [1000], [3100], 11.0, 1.5 * 2.0 ** 100),
    (32, 4, 64, 24, [130, 100, 90, 130], [3000, 2500, 2500, 2500], 7.0, 1.5 * 2.0 ** 106), (32, 4, 64, 64, [130, 100, 1, 130], [3000, 2500, 2500, 0], 7.0, 1.5 * 2.0 ** 106),
    (32, 4, 64, 64, [1000], [3100], 7.0, 1.5 * 2.0 ** 106), (4, 2, 96, 16, [30], [4000], 5.0, 1.5 * 2.0 ** 106)])
def test_sums_that_are_finite_until_they_are_added(H, K, h, pt, lens, behind, rise, value):
    """Values near the largest that the call takes, behind first keys whose scores are lower: weights are counted from those, and groups' and
    pieces' sums, each within binary32's range, would exceed it when they are added."""
    for crowd in (0, 30000, 80000):
        rows, ctx = sum(lens) + crowd // H, max(a + b for a, b in zip(lens, behind))
        piece = plans([(BF16, K, h, 1, len(lens), rows, ctx, H, 0, 0)])[0][1]

        def change(_, x):
            x[0] = 0
            x[0, :, :, 0] = np.where(np.arange(x.shape[1]) // 64 % piece < 2, 0, rise)[:, None]   # (the first two blocks of every piece)
            x[1] = value
        s = Setup(H, K, h, pt, lens, behind, BF16, seed=5, change=change, rows_behind=crowd // H)
        s.q = torch.zeros_like(s.q)
        s.q[:, :, 0] = 1
        cache = s.cache()
        out = s.attn(cache, s.plan(cache), scale=1.0)
        assert (out[:s.start[-1]] == torch.tensor(value).to(BF16).item()).all()
        cache.check()
