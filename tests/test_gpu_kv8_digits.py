"""Attention over the 8-bit cache where values and scores are of very different sizes: rows keep the digits of what they see."""
import numpy as np
import pytest
import torch

from kv8_digits import Setup, check_digits, form_of, rekeyed

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


# a loud value just behind a row, in the row's own block of positions and in later ones; what is seen before it is of size one
BEHIND = {
    "2^12": lambda p: np.where(p >= 100, 2.0 ** 12, 1.0),
    "2^19": lambda p: np.where(p >= 100, 2.0 ** 19, 1.0),
    "2^24": lambda p: np.where(p >= 100, 2.0 ** 24, 1.0),
    "2^30": lambda p: np.where(p >= 100, 2.0 ** 30, 1.0),
    "2^40, one": lambda p: np.where(p == 100, 2.0 ** 40, 1.0),
    "2^100 behind 2^-80": lambda p: np.where(p >= 100, 2.0 ** 100, 2.0 ** -80),
    "a factor of four each block": lambda p: 4.0 ** (p // 64),
    "2^15 each block": lambda p: 2.0 ** np.minimum(15.0 * (p // 64), 90),
    "zeros, then 2^90, then one": lambda p: np.where(p < 70, 0.0, np.where(p == 130, 2.0 ** 90, 1.0)),
}


@pytest.mark.parametrize("h", [64, 128, 40])
@pytest.mark.parametrize("gain", list(BEHIND))
def test_a_row_does_not_depend_on_values_behind_it(gain, h):
    for H, lens, behind, pt in ((4, [150, 1, 64], [0, 330, 90], 64), (2, [260], [40], 24), (2, [20, 9], [90, 900], 16), (10, [110], [0], 48)):
        s = Setup(H, 2, h, pt, lens, behind, seed=3, v_gain=BEHIND[gain])
        cache = s.cache()
        check_digits(cache.attn(s.plan(cache), s.q.to(DEV)), s, form_of(h), what=(lens, pt))
        assert int(s.err.cpu()[0]) == 0
    s = Setup(4, 2, h, 16, [1, 1, 1], [99, 100, 330], seed=4, v_gain=BEHIND[gain])
    cache = s.cache()
    check_digits(cache.attn(s.plan(cache, one_each=True), s.q.to(DEV)), s, form_of(h, True), what="one each")


@pytest.mark.parametrize("h", [64, 128])
def test_a_row_does_not_depend_on_values_of_no_weight(h):
    """Every sixteenth value is 2^40 times as large, and its key's score 300 and more below the others'."""
    gain = lambda p: np.where(p % 16 == 5, 2.0 ** 40, 1.0)
    for lens, behind, pt in (([150, 70], [0, 200], 64), ([40], [1000], 24)):
        s = Setup(4, 2, h, pt, lens, behind, seed=5, v_gain=gain, k_gain=0.5)
        s.q = s.q.abs() + 1
        for i in range(len(lens)):
            at = [p for p in range(lens[i] + behind[i]) if p % 16 == 5]
            for p in at:
                s.scales[s.tables[i, p // pt], :, 0, p % pt] *= np.float32(256)
                s.kv[i][0, p] *= 256
            rekeyed(s, i, at, -1)
        cache = s.cache()
        check_digits(cache.attn(s.plan(cache), s.q.to(DEV)), s, "general", what=(lens, pt))   # both sizes in every block of positions: binary32


@pytest.mark.parametrize("h", [64, 128])
def test_pieces_of_sizes_far_apart_are_joined(h):
    """A few rows behind many positions: pieces whose values are of one size beside pieces whose sizes are far apart."""
    s = Setup(16, 2, h, 64, [9], [6000], seed=6, v_gain=lambda p: np.where((p > 2500) & (p % 3 == 0), 2.0 ** 35, 1.0))
    cache = s.cache()
    rows = s.plan(cache)
    assert cache.workspace(rows, 16) is not None                  # divided
    first = cache.attn(rows, s.q.to(DEV))
    check_digits(first, s, "packed")
    assert torch.equal(cache.attn(rows, s.q.to(DEV)), first)


def test_a_size_further_apart_in_a_captured_call():
    """The same graph, with values of one size and of sizes far apart, in turn."""
    near, far = (Setup(4, 2, 128, 64, [150, 20], [0, 200], seed=7, v_gain=lambda p, e=e: np.where(p >= 100, 2.0 ** e, 1.0)) for e in (3, 50))
    assert np.array_equal(near.tables, far.tables) and torch.equal(near.q, far.q)
    cache = near.cache()
    rows, q = near.plan(cache), near.q.to(DEV)
    out = torch.empty_like(q)
    scales = [torch.from_numpy(x.scales).to(DEV) for x in (near, far)]
    cache.attn(rows, q, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attn(rows, q, out=out)
    for i in (0, 1, 1, 0, 1, 0):
        cache.scales.copy_(scales[i])
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check_digits(out, (near, far)[i], "packed", what=i)


def low_first(H, h, lens, behind, pt, low, depth, seed=8):
    """Queries above zero; the keys of the first `low` positions are `depth` and more below the others in their scores, which are small."""
    s = Setup(H, 2, h, pt, lens, behind, seed=seed, k_gain=0.1)
    s.q = s.q.abs() + 1
    for i in range(len(lens)):
        for p in range(min(low, lens[i] + behind[i])):
            by = np.float32(20 * depth(p) * h ** -0.5)
            at = s.tables[i, p // pt], slice(None), 0, p % pt
            s.scales[at] *= by
            s.kv[i][0, p] = s.codes[at].astype(np.float64) * s.scales[at].astype(np.float64)[:, None]
        rekeyed(s, i, range(min(low, lens[i] + behind[i])), -1)
    return s


@pytest.mark.parametrize("h", [64, 128, 40])
@pytest.mark.parametrize("depth", [300.0, 1e3, 1e5, 1e6, 1e7])
def test_scores_behind_far_lower_ones(depth, h):
    """What decides a row stands behind keys whose scores are far below: it keeps the digits of its own scores."""
    for lens, behind, pt, low in (([200, 90], [0, 100], 64, 64), ([30], [250], 24, 200), ([9], [3000], 64, 1500)):
        s = low_first(4, h, lens, behind, pt, low, lambda p: depth)
        cache = s.cache()
        check_digits(cache.attn(s.plan(cache), s.q.to(DEV)), s, form_of(h), what=(lens, low))
    s = low_first(4, h, [1, 1], [250, 99], 16, 200, lambda p: depth)
    cache = s.cache()
    check_digits(cache.attn(s.plan(cache, one_each=True), s.q.to(DEV)), s, form_of(h, True), what="one each")


@pytest.mark.parametrize("h", [64, 128])
def test_scores_that_rise_from_block_to_block(h):
    """Steps of 40, of 600 and of 6000 a block of positions, up to small ones."""
    for step in (40, 600, 6000):
        s = low_first(4, h, [40, 3], [400, 420], 64, 384, lambda p: step * (6.5 - p // 64))
        cache = s.cache()
        check_digits(cache.attn(s.plan(cache), s.q.to(DEV)), s, "packed", what=step)


SHORT = [  # H, K, h, page tokens, new rows, positions behind: contexts of so few keys that roundings do not average out
    (4, 2, 64, 16, [1, 17, 0, 64, 65], [0, 0, 4, 0, 0]),
    (32, 4, 64, 24, [33, 130], [100, 0]),
    (8, 8, 128, 64, [128, 1, 63], [0, 200, 1]),
    (6, 2, 128, 7, [70], [59]),
    (20, 1, 64, 1, [37], [5]),
    (24, 4, 128, 32, [5] * 9, [0, 31, 32, 33, 63, 64, 65, 500, 1023]),
    (4, 2, 40, 16, [21], [20]),
    (2, 1, 256, 16, [19], [2]),
]


@pytest.mark.parametrize("loud", [1.0, 4.0], ids=["even", "few keys decide"])
@pytest.mark.parametrize("case", SHORT, ids=lambda c: f"{c[0]}of{c[1]}x{c[2]}-page{c[3]}")
def test_results_keep_the_digits_of_their_products(case, loud):
    """Packed rows keep eleven digits of weights and values, single tokens sixteen of a weight times a scale, others all."""
    H, K, h, pt, lens, behind = case
    s = Setup(*case, seed=21, k_gain=loud)
    cache = s.cache()
    check_digits(cache.attn(s.plan(cache), s.q.to(DEV)), s, form_of(h), what="packed")
    ctx = [a + b for a, b in zip(lens, behind) if a + b] + [2, 3, 5, 9]
    s = Setup(H, K, h, pt, [1] * len(ctx), [c - 1 for c in ctx], seed=22, k_gain=loud)
    cache = s.cache()
    check_digits(cache.attn(s.plan(cache, one_each=True), s.q.to(DEV)), s, form_of(h, True), what="one each")


@pytest.mark.parametrize("one_each", [False, True], ids=["packed", "tokens"])
@pytest.mark.parametrize("H,K,h,pt,ctx", [(8, 2, 64, 16, [5000, 1, 300]), (4, 4, 128, 40, [2100, 2111]), (16, 1, 128, 64, [3333]), (3, 1, 32, 16, [1500])])
def test_divided_results_keep_their_digits(H, K, h, pt, ctx, one_each):
    s = Setup(H, K, h, pt, [1] * len(ctx), [c - 1 for c in ctx], seed=23)
    cache = s.cache()
    check_digits(cache.attn(s.plan(cache, one_each=one_each), s.q.to(DEV)), s, form_of(h, one_each))


@pytest.mark.parametrize("h", [64, 128, 40])
@pytest.mark.parametrize("loud", [False, True], ids=["even values", "values far apart"])
def test_a_query_that_is_not_finite_is_its_own(loud, h):
    """A row and head with an infinity or NaN in its query is NaN (or whatever binary32 makes of it); the others know nothing of it."""
    gain = (lambda p: np.where(p % 7 == 2, 2.0 ** 30, 1.0)) if loud else None
    s = Setup(4, 2, h, 64, [70, 5], [0, 300], seed=31, v_gain=gain)
    marks = {3: float("nan"), 40: float("inf"), 69: float("-inf"), 72: float("nan")}
    q = s.q.clone()
    for row, x in marks.items():
        q[row, row % 4, 5] = x
    cache = s.cache()
    out = cache.attn(s.plan(cache), q.to(DEV)).cpu()
    for row in marks:
        assert not torch.isfinite(out[row, row % 4]).any()
        out[row, row % 4] = cache.attn(s.plan(cache), s.q.to(DEV)).cpu()[row, row % 4]
    check_digits(out, s, form_of(h), what="packed")
    s = Setup(4, 2, h, 16, [1, 1, 1], [50, 300, 0], seed=32, v_gain=gain)
    q = s.q.clone()
    q[1, 2, 0], q[2, 3, h - 1] = float("nan"), float("inf")
    cache = s.cache()
    rows = s.plan(cache, one_each=True)
    out, plain = cache.attn(rows, q.to(DEV)).cpu(), cache.attn(rows, s.q.to(DEV)).cpu()
    for row, head in ((1, 2), (2, 3)):
        assert not torch.isfinite(out[row, head]).any()
        out[row, head] = plain[row, head]
    check_digits(out, s, form_of(h, True), what="one each")


@pytest.mark.parametrize("h", [64, 128, 40])
@pytest.mark.parametrize("size", [2.0 ** -99, 2.0 ** -60, 2.0 ** 60, 2.0 ** 105])
def test_values_at_the_ends_of_the_range(size, h):
    """Values of every size from 2^-100 on, and as large as sums of them hold (mdi.h: their number times their size below 2^120)."""
    s = Setup(4, 2, h, 16, [90, 3], [0, 300], seed=33, v_gain=lambda p: size + 0.0 * p)
    cache = s.cache()
    check_digits(cache.attn(s.plan(cache), s.q.to(DEV)), s, form_of(h), what="packed")
    s = Setup(4, 2, h, 16, [1, 1, 1, 1], [50, 300, 0, 2000], seed=34, v_gain=lambda p: size + 0.0 * p)
    cache = s.cache()
    check_digits(cache.attn(s.plan(cache, one_each=True), s.q.to(DEV)), s, form_of(h, True), what="one each")
