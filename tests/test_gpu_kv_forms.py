"""Every form of the kernels of the cache in the storage type against 64 bits: digits, and every position counted once."""
import numpy as np
import pytest
import torch

import kv_forms as F
from kv_cases import Setup, bound, dev, sees, within
from kv_digits import PARTS, check_digits, interval, limits
from paper_2505_18164_amd import mdi

pytestmark = pytest.mark.gpu
CALLS = [(f, w) for f in F.FORMS for w in (False, True) if not (w and f in F.NO_WINDOW)]


def tried(form, window, **more):
    """The call of a form, its plan asked for again: the setup, its rows' results and how to check them."""
    what, max_ctx, one_each = F.calls()[form, window]
    s = Setup(**what, seed=7, **more)
    cache = s.cache()
    out = s.attn(cache, s.plan(cache, one_each=one_each, max_ctx=max_ctx))
    cache.check()
    return s, out


def check(s, out, what):
    if s.dtype == torch.bfloat16:
        check_digits(out, s, what=what)
    else:
        s.check(out, what=what)


@pytest.mark.parametrize("form,window", CALLS, ids=[f + (", window" if w else "") for f, w in CALLS])
def test_digits(form, window):
    check(*tried(form, window), form)


@pytest.mark.parametrize("form,window", CALLS, ids=[f + (", window" if w else "") for f, w in CALLS])
def test_every_position_counts_once(form, window):
    """Keys of zeros, so all weights are alike, and a one per position in one of the channels: a result says how many of a channel's
    positions its row sees, up to some hundred, so that one more or less is more than a rounding.  (Of longer caches the positions about
    the borders of pieces, and the first and last ones.)"""
    what, max_ctx, _ = F.calls()[form, window]
    K, h = what["K"], what["h"]
    call = (what["dtype"], K, h, 0 if F.calls()[form, window][2] else 1, len(what["lens"]), sum(what["lens"]) + what.get("rows_behind", 0), max_ctx, what["H"], what["window"], what["sinks"])
    border = 64 * F.plans([call])[0][1]

    s, out = tried(form, window, change=F.ones(K, h, border))
    check(s, out, form)


@pytest.mark.parametrize("form,window", [c for c in CALLS if "once" not in c[0]], ids=[f + (", window" if w else "") for f, w in CALLS if "once" not in f])
def test_a_value_that_is_not_finite_reaches_only_who_sees_it(form, window):
    """An infinite value amid every sample's new rows, and one before them that a window may have left behind: who sees neither is
    what it is without them (they are computed again), and so are the other channels and kv heads of who does."""
    what, max_ctx, one_each = F.calls()[form, window]
    last, before = [b + t // 2 for b, t in zip(what["behind"], what["lens"])], [b // 3 for b in what["behind"]]

    def spoiled(i, x):
        if x.shape[1]:
            x[1, min(last[i], x.shape[1] - 1), 0, 3] = np.inf
            x[1, min(before[i], x.shape[1] - 1), 0, 5] = -np.inf
    s, out = tried(form, window, change=spoiled)
    got = out.float().cpu().double().numpy()[:s.start[-1]]
    clean = Setup(**what, seed=7)
    if s.dtype == torch.bfloat16:
        lo, hi = limits(clean)
    else:
        want = clean.want()
        may = bound(*want, s.h, s.dtype)
        lo, hi = want[0] - may, want[0] + may
    for i, T in enumerate(s.lens):
        if T:
            rows, seen = slice(s.start[i], s.start[i] + T), sees(T, s.behind[i], s.behind[i] + T, s.window, s.sinks)
            for at, ch, value in ((min(last[i], seen.shape[1] - 1), 3, np.inf), (min(before[i], seen.shape[1] - 1), 5, -np.inf)):
                lo[rows, :s.H // s.K, ch] = np.where(seen[:, at, None], value, lo[rows, :s.H // s.K, ch])
                hi[rows, :s.H // s.K, ch] = np.where(seen[:, at, None], value, hi[rows, :s.H // s.K, ch])
    fine = (lo <= got) & (got <= hi)
    assert fine.all(), (form, (~fine).sum(), [int(x) for x in np.argwhere(~fine)[0]], got[tuple(np.argwhere(~fine)[0])])


@pytest.mark.parametrize("form,window", [c for c in CALLS if c[0].startswith("any") or "whole" in c[0]][::2] + [c for c in CALLS if "of many" in c[0]],
                         ids=lambda x: x if isinstance(x, str) else "window" if x else "all")
def test_samples_between_that_take_no_part(form, window):
    """Every third sample is idle, whatever its table: zeros for its rows, the others' as they are without it."""
    what, max_ctx, one_each = F.calls()[form, window]
    s = Setup(**what, seed=8)
    idle = range(1, len(s.lens), 3)
    s.pos[list(idle)] = -1
    table = np.arange(len(s.lens))
    table[list(idle)] = 10 ** 9
    cache = s.cache()
    out = s.attn(cache, s.plan(cache, one_each=one_each, max_ctx=max_ctx, table=dev(table.astype(np.int32))))
    cache.check()
    rows = np.zeros(out.shape[0], bool)
    for i in idle:
        rows[s.start[i]:s.start[i + 1]] = True
    assert (out[dev(rows)] == 0).all()
    if s.dtype == torch.bfloat16:
        check_digits(out, s, what=form, skip=idle)
    else:
        want = s.want()
        seen = np.flatnonzero(~rows[:want[0].shape[0]])
        within(out[dev(seen)], want[0][seen], bound(*want, s.h, s.dtype)[seen], form)


@pytest.mark.parametrize("dtype,H,K,h,n,rows", [(torch.bfloat16, 16, 16, 64, 300000, 300000), (torch.float32, 16, 8, 32, 550000, 550000), (torch.bfloat16, 16, 16, 128, 1800000, 600000)],
                         ids=["bf16", "f32", "bf16, 128"])
def test_more_workgroups_than_a_launch_may_have(dtype, H, K, h, n, rows):
    """Single rows of so many samples that their workgroups go out in several launches: all of them, against 64 bits by samples alike."""
    dev, pt, tables, ctx = "cuda:0", 16, 7, 11
    form = F.form((dtype, K, h, 1, n, rows, ctx, H, 0, 0), pt, F.plans([(dtype, K, h, 1, n, rows, ctx, H, 0, 0)])[0])
    assert form in F.FORMS and "many" in form
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    make = lambda *s: torch.randn(s, generator=g, device=dev).to(dtype)
    data = make(tables, K, 2, pt, h)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    cache = mdi.KvCache(data, torch.arange(tables, dtype=torch.int32, device=dev).unsqueeze(1), err)
    i = torch.arange(n, device=dev)
    start = torch.div((torch.arange(n + 1, device=dev) * rows), n, rounding_mode="floor").to(torch.int32)     # none or one each
    pos, table = (i % ctx).to(torch.int32), (i % tables).to(torch.int32)
    kinds = 5                                                     # different queries, so that rows are of tables * ctx * kinds kinds
    some = make(kinds, H, h)
    mine = torch.repeat_interleave(i, (start[1:] - start[:-1]).long())
    assert mine.shape == (rows,)
    q = some[mine % kinds]
    out = cache.attn(cache.rows(pos, start=start, table=table, n_rows=rows, max_ctx=ctx), q)
    cache.check()
    want = torch.empty((tables, ctx, kinds, H, h), dtype=torch.float64)
    off = torch.empty_like(want)
    host, hq = data.cpu().double().numpy(), some.cpu().double().numpy()
    for t in range(tables):
        for p in range(ctx):
            for j in range(kinds):
                a, b = interval(hq[j:j + 1], host[t, :, 0, :p + 1].transpose(1, 0, 2), host[t, :, 1, :p + 1].transpose(1, 0, 2), p, h ** -0.5, each=PARTS if dtype == torch.bfloat16 else 0.0)
                want[t, p, j], off[t, p, j] = torch.from_numpy(a[0]), torch.from_numpy(b[0])
    at = (mine % tables, mine % ctx, mine % kinds)
    if dtype == torch.float32:
        off += 2.0 ** -24 * want.abs()
    lo, hi = ((want + s * off).to(dtype).to(dev) for s in (-1, 1))
    for a in range(0, rows, 1 << 16):
        part = [x[a:a + (1 << 16)] for x in at]
        got = out[a:a + (1 << 16)]
        assert bool(((lo[part[0], part[1], part[2]] <= got) & (got <= hi[part[0], part[1], part[2]])).all()), a
