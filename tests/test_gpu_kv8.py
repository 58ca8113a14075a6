"""The 8-bit cache through the C ABI: rows written and read back bit for bit, attention against 64 bits."""
import numpy as np
import pytest
import torch

from kv8_cases import Setup, attention, check, quantise
from paper_2505_18164_amd import mdi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def to_dev(a):
    return torch.from_numpy(np.array(a)).to(DEV)


def awkward_rows(rng, rows, K, h):
    """Rows of every size, with zeros, denormals, lone values, ties, infinities and NaN among them."""
    x = rng.standard_normal((rows, K, h)).astype(np.float32) * np.exp(rng.uniform(-40, 40, (rows, K, 1))).astype(np.float32)
    for i in range(rows):
        kind = i % 9
        if kind == 1:
            x[i] = 0
        elif kind == 2:
            x[i] = np.float32(2.0 ** -100) * rng.uniform(-0.999, 0.999, (K, h)).astype(np.float32)
        elif kind == 3:
            x[i, 0, rng.integers(h)] = np.inf if i % 2 else -np.inf
        elif kind == 4:
            x[i, -1, rng.integers(h)] = np.nan
        elif kind == 5:                                           # halves of a step: ties
            x[i] = rng.integers(-254, 255, (K, h)) / 2.0
            x[i, :, 0] = 127
        elif kind == 6:
            x[i] = 0
            x[i, :, h - 1] = -3e38
        elif kind == 7:
            x[i] = 2.0 ** -100
    return x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("K,h,pt,lens,behind", [(1, 8, 1, [1], [0]), (2, 64, 16, [5, 0, 40], [3, 7, 0]), (5, 128, 24, [33, 1, 2], [100, 0, 23]),
                                                (3, 40, 7, [20, 9], [1, 0]), (32, 128, 64, [3], [61]), (1, 256, 5, [11] * 3, [0, 4, 9]),
                                                (4, 64, 32, [1] * 70, list(range(70)))])
def test_written_and_read_back(K, h, pt, lens, behind, dtype):
    rng = np.random.default_rng(K * h + pt)
    total = [a + b for a, b in zip(lens, behind)]
    used = [(t + pt - 1) // pt for t in total]
    n_pages, rows, n = sum(used) + 2, sum(lens), len(lens)
    order = rng.permutation(n_pages).astype(np.int32)
    tables = np.full((n, max(used) + 1), -5, dtype=np.int32)
    for i in range(n):
        tables[i, :used[i]] = order[sum(used[:i]):sum(used[:i + 1])]
    x = torch.from_numpy(np.stack([awkward_rows(rng, rows + 3, K, h) for _ in range(2)])).to(dtype)     # three rows belong to nobody
    codes = rng.integers(-127, 128, (n_pages, K, 2, pt, h)).astype(np.int8)
    scales = rng.standard_normal((n_pages, K, 2, pt)).astype(np.float32)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    cache = mdi.Kv8Cache(to_dev(codes), to_dev(scales), to_dev(tables), err)
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    plan = cache.rows(to_dev(np.asarray(behind, np.int32)), start=to_dev(start), n_rows=rows + 3)
    # rows of a fused product, with four other heads in front
    fused = torch.zeros((rows + 3, 4 + 2 * K, h), dtype=dtype, device=DEV)
    fused[:, 4:4 + K], fused[:, 4 + K:] = x[0].to(DEV), x[1].to(DEV)
    cache.write(plan, fused[:, 4:4 + K], fused[:, 4 + K:])
    code, scale = quantise(x.double().numpy())
    for i in range(n):
        for r in range(lens[i]):
            p, row = behind[i] + r, start[i] + r
            codes[tables[i, p // pt], :, :, p % pt] = code[:, row].transpose(1, 0, 2)
            scales[tables[i, p // pt], :, :, p % pt] = scale[:, row].T
    assert np.array_equal(cache.codes.cpu().numpy(), codes)       # the written rows, and nothing else
    assert np.array_equal(cache.scales.cpu().numpy(), scales, equal_nan=True)
    for out_dtype in (torch.float32, torch.bfloat16):
        k, v = (torch.full((K, rows + 3, h), 7.0, dtype=out_dtype, device=DEV).transpose(0, 1) for _ in range(2))
        assert cache.read(plan, k, v) == (k, v)
        for got, side in ((k, 0), (v, 1)):
            want = torch.from_numpy(code[side].astype(np.float32) * scale[side][..., None]).to(out_dtype)
            want[rows:] = 7.0
            assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
            assert torch.equal(torch.nan_to_num(got.cpu(), nan=0.5), torch.nan_to_num(want, nan=0.5)), (out_dtype, side)
    # half a step, of the formula's two roundings a little more
    top = np.abs(x.double().numpy()).max(-1, keepdims=True)
    with np.errstate(all="ignore"):
        off = np.abs(code.astype(np.float64) * scale.astype(np.float64)[..., None] - x.double().numpy())
        fine = np.isfinite(top) & (top >= 2.0 ** -100)
        assert (off <= np.where(fine, top / 254 * (1 + 2.0 ** -15), np.inf))[np.broadcast_to(fine, off.shape)].all()
    cache.check()


def test_samples_that_take_no_part_and_other_tables():
    rng = np.random.default_rng(5)
    K, h, pt = 2, 64, 16
    x = torch.from_numpy(rng.standard_normal((2, 4, K, h)).astype(np.float32)).to(DEV)
    err = torch.zeros(1, dtype=torch.int32, device=DEV)
    cache = mdi.Kv8Cache(torch.full((4, K, 2, pt, h), 9, dtype=torch.int8, device=DEV), torch.full((4, K, 2, pt), 9.0, device=DEV),
                         to_dev(np.array([[3, 0], [2, 0], [1, 0]], np.int32)), err)
    plan = cache.rows(to_dev(np.array([4, -1, 2, 0], np.int32)), table=to_dev(np.array([2, 0, 0, 1], np.int32)), max_ctx=5)
    cache.write(plan, x[0], x[1])
    code, scale = quantise(x.cpu().double().numpy())
    codes = np.full((4, K, 2, pt, h), 9, np.int8)
    for row, (page, slot) in {0: (1, 4), 2: (3, 2), 3: (2, 0)}.items():
        codes[page, :, :, slot] = code[:, row].transpose(1, 0, 2)
    assert np.array_equal(cache.codes.cpu().numpy(), codes)
    q = torch.randn((4, 6, h), device=DEV).bfloat16()
    out = torch.full_like(q, 3.0)
    cache.attn(plan, q, out=out)
    assert (out[1] == 0).all()                                    # sample 1 takes no part
    assert torch.isfinite(out[3]).all() and (out[3] != 3).any()
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
]
IDS = [f"{c[0]}of{c[1]}x{c[2]}-page{c[3]}-{i}" for i, c in enumerate(ATTN)]


@pytest.mark.parametrize("case", ATTN, ids=IDS)
def test_packed_rows_against_64_bits(case):
    s = Setup(*case, seed=3, rows_behind=3)
    cache = s.cache()
    wide = torch.zeros((s.rows, s.H + 2 * s.K, s.h), dtype=torch.bfloat16, device=DEV)   # the query heads of a fused product
    wide[:, :s.H] = s.q.to(DEV)
    out = torch.full((s.rows, s.H, s.h), 5.0, dtype=torch.bfloat16, device=DEV)
    assert cache.attn(s.plan(cache), wide[:, :s.H], out=out) is out
    check(out, s.want(), s.h)
    assert (out[s.start[-1]:] == 5.0).all()                       # rows of nobody
    cache.check()


@pytest.mark.parametrize("case", ATTN, ids=IDS)
def test_one_new_token_against_64_bits(case):
    H, K, h, pt, lens, behind = case
    ctx = [a + b for a, b in zip(lens, behind)]
    s = Setup(H, K, h, pt, [1] * len(ctx), [c - 1 for c in ctx], seed=4)
    cache = s.cache()
    out = cache.attn(s.plan(cache, one_each=True), s.q.to(DEV))
    check(out, s.want(), s.h)
    cache.check()


@pytest.mark.parametrize("one_each", [False, True], ids=["packed", "tokens"])
@pytest.mark.parametrize("H,K,h,pt,ctx", [(8, 2, 64, 16, [5000, 1, 300]), (4, 4, 128, 40, [2100, 2111]), (16, 1, 128, 64, [3333]), (3, 1, 32, 16, [1500])])
def test_long_contexts_are_divided_and_joined(H, K, h, pt, ctx, one_each):
    s = Setup(H, K, h, pt, [1] * len(ctx), [c - 1 for c in ctx], seed=6, stale="inf")
    cache = s.cache()
    plan = s.plan(cache, one_each=one_each)
    space = cache.workspace(plan, H)
    assert space is not None
    space.fill_(0xFF)                                             # NaN everywhere: nothing is taken from a workspace that the call has not put there
    want = s.want()
    first = cache.attn(plan, s.q.to(DEV), workspace=space)
    check(first, want, h)
    for _ in range(3):
        assert torch.equal(cache.attn(plan, s.q.to(DEV), workspace=space), first)
    # divided for longer samples than there are
    long = s.plan(cache, one_each=one_each, max_ctx=s.tables.shape[1] * pt)
    check(cache.attn(long, s.q.to(DEV)), want, h)
    cache.check()


GAINS = {
    "growing": lambda p: 2.0 ** np.minimum(p / 8.0 - 30, 60),                   # every block of positions larger than the one before
    "falling": lambda p: 2.0 ** np.maximum(20 - p / 8.0, -90),
    "here and there": lambda p: np.where(p % 67 == 66, 2.0 ** 14, np.where(p % 5 == 3, 2.0 ** -9, 1.0)),
    "zeros first": lambda p: np.where(p < 70, 0.0, 1.0),
    "all zeros": lambda p: 0.0 * p,
    "tiny": lambda p: 2.0 ** -94 + 0.0 * p,
    "huge": lambda p: np.where(p < 100, 1.0, 2.0 ** 90),
}


@pytest.mark.parametrize("h", [64, 128])
@pytest.mark.parametrize("gain", list(GAINS))
def test_values_of_all_sizes(gain, h):
    """Values are multiplied as fp16 of a size that the kernel keeps up with."""
    for lens, behind, pt in (([150, 1, 64], [0, 330, 500], 64), ([260], [40], 24), ([20, 9], [900, 1500], 64)):
        s = Setup(4, 2, h, pt, lens, behind, seed=3, v_gain=GAINS[gain])
        cache = s.cache()
        check(cache.attn(s.plan(cache), s.q.to(DEV)), s.want(), h, (lens, pt))
        assert int(s.err.cpu()[0]) == 0
    s = Setup(4, 2, h, 16, [1, 1, 1], [0, 500, 79], seed=4, v_gain=GAINS[gain])
    cache = s.cache()
    check(cache.attn(s.plan(cache, one_each=True), s.q.to(DEV)), s.want(), h, "one each")


@pytest.mark.parametrize("h", [64, 128, 48])
def test_values_that_decide_alone_and_far_apart(h):
    """Loud keys: one position's weight is all but 1; scores of hundreds either way, and growing along the cache."""
    for seed, gain in ((1, 40.0), (2, 300.0)):
        s = Setup(4, 2, h, 16, [50, 3], [90, 400], seed=seed, k_gain=gain)
        s.q *= 2
        cache = s.cache()
        check(cache.attn(s.plan(cache), s.q.to(DEV)), s.want(), h)
    s = Setup(4, 2, h, 16, [40], [200], seed=8, k_gain=1.0)
    ramp = np.linspace(0.01, 30, 240)
    for side in (0,):
        for p in range(240):
            s.scales[s.tables[0, p // 16], :, side, p % 16] *= np.float32(ramp[p])
    s.kv[0][0] = np.stack([s.codes[s.tables[0, p // 16], :, 0, p % 16].astype(np.float64) * s.scales[s.tables[0, p // 16], :, 0, p % 16].astype(np.float64)[:, None] for p in range(240)])
    cache = s.cache()
    check(cache.attn(s.plan(cache), s.q.to(DEV)), s.want(), h)
    for scale in (0.0, -0.3, 2.0):
        check(cache.attn(s.plan(cache), s.q.to(DEV), scale=scale), s.want(scale), h)


def test_a_row_with_nan_reaches_only_those_that_see_it():
    s = Setup(4, 2, 64, 16, [40], [10], seed=2)
    page, slot = s.tables[0, 30 // 16], 30 % 16
    s.scales[page, 1, 1, slot] = np.nan                           # the value of position 30, kv head 1
    cache = s.cache()
    out = cache.attn(s.plan(cache), s.q.to(DEV)).float().cpu()
    assert torch.isfinite(out[:20]).all() and torch.isfinite(out[:, :2]).all()
    assert torch.isnan(out[20:, 2:]).all()
    one = s.plan(cache, max_ctx=64)
    token = cache.rows(to_dev(np.array([29, 30], np.int32)), table=to_dev(np.zeros(2, np.int32)), max_ctx=64)
    out = cache.attn(token, s.q[:2].contiguous().to(DEV)).float().cpu()
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[1, :2]).all() and torch.isnan(out[1, 2:]).all()


@pytest.mark.parametrize("h", [64, 128, 24])
def test_what_is_not_of_the_cache_is_reported(h):
    good = Setup(4, 2, h, 16, [20, 3], [0, 40], seed=1)
    q = good.q.to(DEV)
    k = torch.randn((good.rows, 2, h), device=DEV)
    for what in ("page", "negative page", "table", "position"):
        s = Setup(4, 2, h, 16, [20, 3], [0, 40], seed=1)
        if what == "page":
            s.tables[0, 1] = s.codes.shape[0]
        if what == "negative page":
            s.tables[0, 0] = -1
        table = to_dev(np.array([0, 2 if what == "table" else 1], np.int32))
        for op in ("write", "read", "attn", "tokens"):
            cache = s.cache()
            plan = s.plan(cache, table=table, max_ctx=42 if what == "position" else s.max_ctx)
            if op == "tokens":
                tokens = cache.rows(to_dev(np.array([19, 42], np.int32)), table=table, max_ctx=42 if what == "position" else s.max_ctx)
                cache.attn(tokens, q[:2].contiguous())
            elif op == "attn":
                cache.attn(plan, q)
            else:
                getattr(cache, op)(plan, k, k.clone())
            with pytest.raises(mdi.MdiError) as e:
                cache.check()
            assert e.value.status == mdi.MDI_ERR_ARG, (what, op)
            plan = s.plan(s.cache(err=False), table=table)        # nobody asks: nothing is written
            torch.cuda.synchronize()


def test_offsets_past_32_bits():
    """The last pages of a pool of 4.5 GiB."""
    K, h, pt, H = 8, 128, 64, 16
    n_pages = (9 << 29) // (K * 2 * pt * h)
    codes = torch.empty((n_pages, K, 2, pt, h), dtype=torch.int8, device=DEV)
    scales = torch.empty((n_pages, K, 2, pt), dtype=torch.float32, device=DEV)
    tables = to_dev(np.array([[n_pages - 1, 0, n_pages - 2]], np.int32))
    cache = mdi.Kv8Cache(codes, scales, tables, torch.zeros(1, dtype=torch.int32, device=DEV))
    x = torch.randn((2, 150, K, h), device=DEV).bfloat16()
    plan = cache.rows(to_dev(np.array([0], np.int32)), start=to_dev(np.array([0, 150], np.int32)), n_rows=150)
    cache.write(plan, x[0], x[1])
    q = torch.randn((150, H, h), device=DEV).bfloat16()
    s = Setup(H, K, h, pt, [150], [0])
    code, scale = quantise(x.cpu().double().numpy())
    s.kv, s.q = [code.astype(np.float64) * scale.astype(np.float64)[..., None]], q.cpu()
    k, v = (torch.empty((150, K, h), device=DEV) for _ in range(2))
    cache.read(plan, k, v)
    assert np.array_equal(k.cpu().numpy(), code[0].astype(np.float32) * scale[0][..., None])
    check(cache.attn(plan, q), s.want(), h)
    last = cache.rows(to_dev(np.array([149], np.int32)))
    got = cache.attn(last, q[149:])
    check(got, [w[149:] for w in s.want()], h)
    cache.check()


def test_captured_and_replayed_with_growing_samples():
    """Write and attend as one graph: every replay appends a token, the positions live on the device."""
    H, K, h, pt = 8, 2, 64, 16
    s = Setup(H, K, h, pt, [1, 1, 1], [255, 300, 9], seed=12, spare=4)
    cache = s.cache()
    pos = to_dev(s.pos)
    plan = cache.rows(pos, max_ctx=(s.tables.shape[1]) * pt)
    k, v = (torch.empty((3, K, h), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q, out = s.q.to(DEV), torch.empty((3, H, h), dtype=torch.bfloat16, device=DEV)
    space = cache.workspace(plan, H)
    fresh = torch.arange(s.codes.shape[0] - 3, s.codes.shape[0], dtype=torch.int32)
    for i, b in enumerate(s.pos):                                 # a page for the positions to come, where the next one starts
        cache.tables[i, (int(b) + 1 + pt - 1) // pt] = int(np.setdiff1d(np.arange(s.codes.shape[0]), np.concatenate([s.tables[j, :(s.pos[j] + pt) // pt] for j in range(3)]))[i])
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        cache.write(plan, k, v)
        cache.attn(plan, q, out=out, workspace=space)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        cache.write(plan, k, v)
        cache.attn(plan, q, out=out, workspace=space)
    for step in range(4):
        x = torch.from_numpy(np.random.default_rng(step).standard_normal((2, 3, K, h)).astype(np.float32)).bfloat16()
        k.copy_(x[0]); v.copy_(x[1])
        code, scale = quantise(x.double().numpy())
        new = code.astype(np.float64) * scale.astype(np.float64)[..., None]
        for i in range(3):
            p = int(s.pos[i]) + step
            s.kv[i] = np.concatenate([s.kv[i][:, :p], new[:, i][:, None]], axis=1)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        s.behind = [int(b) + step for b in s.pos]
        check(out, s.want(), h, step)
        eager = cache.attn(plan, q)
        assert torch.equal(eager, out)
        pos += 1
    cache.check()


def test_on_another_stream():
    s = Setup(4, 2, 64, 16, [30, 4], [0, 11], seed=9)
    cache = s.cache()
    plan, q = s.plan(cache), s.q.to(DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)
        out = cache.attn(plan, q * 1)
    stream.synchronize()
    check(out, s.want(), 64)


def test_nothing_to_do_and_refusals():
    s = Setup(4, 2, 64, 16, [30, 4], [0, 11], seed=9)
    cache = s.cache()
    none = cache.rows(torch.empty(0, dtype=torch.int32, device=DEV), start=torch.zeros(1, dtype=torch.int32, device=DEV), n_rows=0)
    empty = torch.empty((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    assert cache.attn(none, empty).shape == (0, 4, 64)
    cache.write(none, empty[:, :2], empty[:, :2])
    left = cache.rows(torch.empty(0, dtype=torch.int32, device=DEV), start=torch.zeros(1, dtype=torch.int32, device=DEV), n_rows=2)
    out = torch.full((2, 4, 64), 2.0, dtype=torch.bfloat16, device=DEV)
    assert (cache.attn(left, torch.randn_like(out), out=out) == 2).all()
    plan, q = s.plan(cache), s.q.to(DEV)
    space = torch.empty(16, dtype=torch.uint8, device=DEV)
    for bad in (lambda: cache.attn(plan, q.float()), lambda: cache.attn(plan, q[:-1]), lambda: cache.attn(plan, q[..., :32]),
                lambda: cache.attn(plan, q.transpose(0, 1).contiguous().transpose(0, 1)), lambda: cache.attn(plan, q.cpu()),
                lambda: cache.write(plan, q, q), lambda: cache.write(plan, q[:, :2], q[:, :2].float()), lambda: cache.read(plan, q[:, :2].half(), q[:, :2].half()),
                lambda: cache.rows(s.pos), lambda: cache.rows(to_dev(s.pos), start=to_dev(s.start)), lambda: cache.rows(to_dev(s.pos).long()),
                lambda: cache.rows(to_dev(s.pos), start=to_dev(s.start)[1:], n_rows=3), lambda: mdi.Kv8Cache(cache.codes, cache.scales[:1], cache.tables),
                lambda: mdi.Kv8Cache(cache.codes.float(), cache.scales, cache.tables), lambda: mdi.Kv8Cache(cache.codes, cache.scales, cache.tables.cpu())):
        with pytest.raises((ValueError, AttributeError)):
            bad()
    three = torch.randn((s.rows, 3, 64), device=DEV).bfloat16()
    with pytest.raises(mdi.MdiError) as e:
        cache.attn(plan, three)                                   # two kv heads do not divide three
    assert e.value.status == mdi.MDI_ERR_ARG
    with pytest.raises(mdi.MdiError):
        cache.attn(plan, q, scale=float("inf"))
    odd = torch.empty(s.rows * 4 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(s.rows, 4, 64)
    with pytest.raises(mdi.MdiError):
        cache.attn(plan, odd)
    with pytest.raises(mdi.MdiError):
        cache.write(plan, odd[:, :2], odd[:, 2:])
    s = Setup(4, 2, 64, 16, [1], [3000], seed=9)
    cache = s.cache()
    with pytest.raises(mdi.MdiError) as e:
        cache.attn(s.plan(cache), s.q.to(DEV), workspace=space)
    assert e.value.status == mdi.MDI_ERR_NOMEM


@pytest.mark.parametrize("H,K,h,pt,ctx", [(4, 1, 64, 16, [70000, 5]), (2, 1, 128, 1, [5000, 300]), (4, 2, 64, 3, [6200, 1])], ids=["many pieces", "pages of one", "pages of three"])
def test_more_pieces_and_pages_than_are_looked_at_at_a_time(H, K, h, pt, ctx):
    s = Setup(H, K, h, pt, [1] * len(ctx), [c - 1 for c in ctx], seed=6)
    cache = s.cache()
    q = s.q.to(DEV)
    check(cache.attn(s.plan(cache, one_each=True), q), s.want(), h, "one each")
    check(cache.attn(s.plan(cache), q), s.want(), h, "packed")
    assert int(s.err.cpu()[0]) == 0


@pytest.mark.parametrize("h", [64, 128, 16])
def test_more_samples_than_are_looked_at_at_a_time(h):
    """131 samples, three of 64 and one: some without rows, some that take no part, long ones last."""
    lens = [(7 * i) % 4 for i in range(128)] + [40, 0, 3]
    behind = [(13 * i) % 90 for i in range(128)] + [0, 9, 1900]
    s = Setup(4, 2, h, 16, lens, behind, seed=7)
    absent = [5, 63, 64, 127, 128]
    s.pos[absent] = -1
    cache = s.cache()
    want = s.want()
    rows = np.concatenate([np.arange(s.start[i], s.start[i + 1]) for i in absent])
    for w in want:
        w[rows] = 0
    check(cache.attn(s.plan(cache), s.q.to(DEV)), want, h, "packed")
    s = Setup(4, 2, h, 16, [1] * 131, [(13 * i) % 90 for i in range(129)] + [2500, 700], seed=8)
    s.pos[absent] = -1
    cache = s.cache()
    want = s.want()
    for w in want:
        w[absent] = 0
    check(cache.attn(s.plan(cache, one_each=True), s.q.to(DEV)), want, h, "one each")


def test_two_graphs_share_a_workspace_and_one_sample_is_asked_twice():
    a = Setup(8, 2, 64, 16, [1, 1], [4000, 900], seed=9)
    b = Setup(8, 2, 64, 16, [64], [6000], seed=10)
    ca, cb = a.cache(), b.cache()
    twice = torch.tensor([1, 1], dtype=torch.int32, device=DEV)
    pos = torch.tensor([900, 500], dtype=torch.int32, device=DEV)     # the second sees less of the same sample
    ra, rb = ca.rows(pos, table=twice, max_ctx=4001), b.plan(cb)
    qa, qb = a.q.to(DEV), b.q.to(DEV)
    wa, wb = ca.workspace(ra, 8), cb.workspace(rb, 8)
    assert wa is not None and wb is not None                          # both are divided
    work = torch.empty(max(wa.numel(), wb.numel()), dtype=torch.uint8, device=DEV)
    oa, ob = torch.empty_like(qa), torch.empty_like(qb)
    ca.attn(ra, qa, out=oa, workspace=work)
    cb.attn(rb, qb, out=ob, workspace=work)
    first = oa.clone(), ob.clone()
    q = a.q.double().numpy()
    for i, p in enumerate((900, 500)):
        k, v = a.kv[1]
        check(oa[i:i + 1], attention(q[i:i + 1], k, v, p, 64 ** -0.5), 64, ("twice", i))
    check(ob, b.want(), 64)
    graphs = []
    for c, r, q, o in ((ca, ra, qa, oa), (cb, rb, qb, ob)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.attn(r, q, out=o, workspace=work)
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0):
        for o in (oa, ob):
            o.zero_()
        graphs[i].replay()
        graphs[1 - i].replay()
        torch.cuda.synchronize()
        assert torch.equal(oa, first[0]) and torch.equal(ob, first[1])


@pytest.mark.parametrize("pt", [16, 24])
@pytest.mark.parametrize("h", [64, 128])
def test_tokens_of_a_call_that_may_read_more_than_the_caches_hold(h, pt):
    """By its bound of the positions, that is: the tables have room for 200000 of each sample."""
    s = Setup(4, 2, h, pt, [1, 1, 1], [700, 0, 3000], seed=11, spare=200000 // pt)
    cache = s.cache()
    rows = cache.rows(to_dev(s.pos))
    assert 3 * s.tables.shape[1] * pt * 2 * 2 * (h + 4) > 128e6
    check(cache.attn(rows, s.q.to(DEV)), s.want(), h)
    cache.check()


def test_two_calls_at_once():
    """Two streams, a workspace each, the same cache: every result is the one of the call alone."""
    a = Setup(8, 2, 128, 64, [200, 33], [1500, 0], seed=13)
    cache = a.cache()
    rows, tokens = a.plan(cache), cache.rows(to_dev(np.array([1600, 20], np.int32)))
    q = a.q.to(DEV)
    alone = cache.attn(rows, q), cache.attn(tokens, q[:2])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(cache.attn(rows, q) if i == 0 else cache.attn(tokens, q[:2]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, alone[i]) for i in range(2) for x in got[i])
