"""Pages, table rows and positions outside a cache whose owner asks for no report (err NULL): nothing is written out of place, and
what does not depend on them is right."""
import numpy as np
import pytest
import torch

from kv8_cases import quantise
from kv8_digits import Setup, form_of, interval

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def to_dev(a):
    return torch.from_numpy(np.array(a)).to(DEV)


def right(got, want, off):
    bf16 = lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    got = got.float().cpu().double().numpy()
    return ((bf16(want - off) <= got) & (got <= bf16(want + off))).all()


@pytest.mark.parametrize("report", [False, True], ids=["unreported", "reported"])
@pytest.mark.parametrize("h", [64, 128, 24])
@pytest.mark.parametrize("what", ["page", "negative page", "table", "position"])
def test_what_is_not_of_the_cache(what, h, report):
    s = Setup(4, 2, h, 16, [20, 3], [0, 40], seed=1, stale="inf")
    at = [(i, s.behind[i] + t) for i in (0, 1) for t in range(s.lens[i])]       # sample and position of every row
    bad = {"page": lambda i, p: i == 0 and p >= 16, "negative page": lambda i, p: i == 0 and p < 16, "table": lambda i, p: i == 1,
           "position": lambda i, p: p >= 42}[what]
    spoilt = {"negative page": lambda i, p: i == 0}.get(what, bad)            # rows whose attention meets it
    kv = s.kv
    tables = s.tables.copy()
    if what == "page":
        s.tables[0, 1] = s.codes.shape[0]
    if what == "negative page":
        s.tables[0, 0] = -1
    table = to_dev(np.array([0, 2 if what == "table" else 1], np.int32))
    max_ctx = 42 if what == "position" else s.max_ctx
    q = s.q.to(DEV)
    want = [interval(s.q[s.start[i]:s.start[i + 1]].double().numpy(), kv[i][0], kv[i][1], s.behind[i], h ** -0.5, form_of(h)) for i in (0, 1)]

    cache = s.cache(err=report)
    rows = s.plan(cache, table=table, max_ctx=max_ctx)
    out = cache.attn(rows, q)
    for r, (i, p) in enumerate(at):
        if not spoilt(i, p):
            t = r - s.start[i]
            assert right(out[r], want[i][0][t], want[i][1][t]), ("packed", i, p)
    for i, p in ((0, 15), (0, 19), (1, 41), (1, 42)):
        pos, mine = [19, 40], i
        pos[i] = p
        tokens = cache.rows(to_dev(np.array(pos, np.int32)), table=table, max_ctx=max_ctx)
        t = p - s.behind[i]
        q2 = torch.stack([q[s.start[j] + pos[j] - s.behind[j]] for j in (0, 1)])
        out = cache.attn(tokens, q2)
        if not spoilt(i, p):
            w, off = interval(s.q[s.start[i]:s.start[i + 1]].double().numpy(), kv[i][0], kv[i][1], s.behind[i], h ** -0.5, form_of(h, True))
            assert right(out[mine], w[t], off[t]), ("token", i, p)

    x = torch.randn((2, s.rows, 2, h), device=DEV)
    back = torch.full((2, s.rows, 2, h), 7.0, device=DEV)
    cache.read(rows, back[0], back[1])
    cache.write(rows, x[0], x[1])
    code, scale = quantise(x.cpu().double().numpy())
    codes, scales = s.codes.copy(), s.scales.copy()
    for r, (i, p) in enumerate(at):
        if bad(i, p):
            assert (back[:, r] == 7).all(), ("read", i, p)
            continue
        page, slot = tables[i, p // 16], p % 16
        assert torch.equal(back[:, r].cpu(), torch.from_numpy((s.codes[page, :, :, slot].astype(np.float32) * s.scales[page, :, :, slot][..., None]).transpose(1, 0, 2))), ("read", i, p)
        codes[page, :, :, slot] = code[:, r].transpose(1, 0, 2)
        scales[page, :, :, slot] = scale[:, r].T
    assert np.array_equal(cache.codes.cpu().numpy(), codes)       # the rows that have a place, and nothing else
    assert np.array_equal(cache.scales.cpu().numpy(), scales, equal_nan=True)
    assert not report or int(s.err.cpu()[0]) == 2
