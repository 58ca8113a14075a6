"""Calls of very many samples over the 8-bit cache: what a row or workgroup does to find its sample does not grow with them."""
import numpy as np
import pytest
import torch

from kv8_digits import STEP
from paper_2505_18164_amd import mdi

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def bf16_between(got, out, off):
    lo, hi = (out - off).to(torch.bfloat16), (out + off).to(torch.bfloat16)
    return ((lo <= got) & (got <= hi)).all()


def expected(q, codes, scales, page, pos, scale):
    """Rows q [m, H, h] on one page each, at position pos: attention in 64 bits, and how far off it may be (kv8_digits.interval, whose
    terms these are, all of them at the row's largest score)."""
    x = codes[page].double() * scales[page].double().unsqueeze(-1)                # [m, K, 2, pt, h]
    m, H, h = q.shape
    K, pt = x.shape[1], x.shape[3]
    q = q.double().view(m, K, H // K, 1, h)
    k, v = x[:, :, 0].unsqueeze(2), x[:, :, 1].unsqueeze(2)
    seen = (torch.arange(pt, device=DEV) <= pos.unsqueeze(-1)).view(m, 1, 1, pt)
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    s = torch.where(seen, scale * (q * k).sum(-1), zero - np.inf)
    w = torch.softmax(s, -1).unsqueeze(-1)
    v = torch.where(seen.unsqueeze(-1), v, zero)
    out, mag, total = (w * v).sum(-2), (w * v.abs()).sum(-2), v.abs().sum(-2)
    wrong = (h + 8) * STEP * torch.where(seen, scale * (q.abs() * k.abs()).sum(-1), zero).amax(-1, keepdim=True) + 4 * STEP
    off = (2 * wrong + 66 * STEP) * (mag + out.abs()) + 2.0 ** -11 * (2 * mag + out.abs()) + 2.0 ** -30 * (total + pt * out.abs())
    return out.reshape(m, H, h), 1.01 * off.reshape(m, H, h)


@pytest.mark.parametrize("H,K,h,n,pt", [(4, 2, 64, 70000, 8), (3, 1, 128, 4097, 512), (2, 2, 64, 4096, 512), (8, 1, 64, 65, 512), (4, 4, 128, 384, 512),
                                        (4, 4, 128, 385, 512), (8, 2, 64, 400, 500), (8, 2, 128, 400, 500), (2, 1, 24, 9000, 8)])
def test_packed_samples(H, K, h, n, pt):
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 4, n)
    if n > 1000:
        lens[n // 2:n // 2 + 200] = 0                             # many without rows, and a long one behind them
    lens[n // 2 + 200 if n > 1000 else 40] = pt // 2 + 1
    pos = rng.integers(0, pt - lens.max() + 1, n)
    pos[rng.random(n) < 0.05] = -1
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    rows = int(start[-1])
    order = rng.permutation(n).astype(np.int32)
    codes = torch.randint(-127, 128, (n, K, 2, pt, h), dtype=torch.int8, device=DEV)
    scales = torch.rand((n, K, 2, pt), device=DEV) / 50 + 1e-3
    dev = lambda a: torch.from_numpy(np.array(a)).to(DEV)
    cache = mdi.Kv8Cache(codes, scales, dev(order.reshape(n, 1)), torch.zeros(1, dtype=torch.int32, device=DEV))
    plan = cache.rows(dev(pos.astype(np.int32)), start=dev(start), n_rows=rows + 2)
    which = np.repeat(np.arange(n), lens)
    at = pos[which] + np.arange(rows) - start[which]
    part = dev(pos[which] >= 0)
    page, at = dev(order[which]).long(), dev(at)
    at0 = at.clamp(min=0)
    x = torch.randn((2, rows + 2, K, h), device=DEV)
    cache.write(plan, x[0], x[1])
    back = torch.full((2, rows + 2, K, h), 7.0, device=DEV)
    cache.read(plan, back[0], back[1])
    for side in (0, 1):                                           # half a step
        assert ((back[side, :rows] - x[side, :rows]).abs() <= x[side, :rows].abs().amax(-1, keepdim=True) / 254 * (1 + 2.0 ** -15))[part].all()
        assert (back[side, :rows][~part] == 7).all() and (back[side, rows:] == 7).all()
        want = cache.codes[page, :, side, at0].float() * cache.scales[page, :, side, at0].unsqueeze(-1)
        assert torch.equal(back[side, :rows][part], want[part])
    q = torch.randn((rows + 2, H, h), device=DEV).bfloat16()
    out = torch.full_like(q, 3.0)
    cache.attn(plan, q, out=out)
    assert (out[:rows][~part] == 0).all() and (out[rows:] == 3).all()
    for lo in range(0, rows, 20000 if pt == 8 else 500):
        hi = min(rows, lo + (20000 if pt == 8 else 500))
        want, off = expected(q[lo:hi], cache.codes, cache.scales, page[lo:hi], at0[lo:hi], h ** -0.5)
        assert bf16_between(out[lo:hi][part[lo:hi]], want[part[lo:hi]], off[part[lo:hi]]), lo
    cache.check()


def test_more_workgroups_than_a_launch_may_have():
    """2^18 samples of one row and 32 heads, packed: a workgroup each, of 512 threads, would be 1.004 * 2^32 threads."""
    rng = np.random.default_rng(1)
    n, K, h, pt = 1 << 18, 32, 64, 8
    codes = torch.randint(-127, 128, (16, K, 2, pt, h), dtype=torch.int8, device=DEV)
    scales = torch.rand((16, K, 2, pt), device=DEV) / 50 + 1e-3
    dev = lambda a: torch.from_numpy(np.array(a)).to(DEV)
    cache = mdi.Kv8Cache(codes, scales, dev(np.arange(16, dtype=np.int32).reshape(16, 1)), torch.zeros(1, dtype=torch.int32, device=DEV))
    table, pos = rng.integers(0, 16, n).astype(np.int32), rng.integers(0, pt, n).astype(np.int32)
    plan = cache.rows(dev(pos), start=dev(np.arange(n + 1, dtype=np.int32)), table=dev(table), n_rows=n)
    q = torch.randn((n, K, h), dtype=torch.bfloat16, device=DEV)
    out = torch.full_like(q, 300.0)
    cache.attn(plan, q, out=out)
    cache.check()
    assert (out.abs().amax(-1) < 300).all()                       # every row and head has been written
    some = np.concatenate([np.arange(500), rng.integers(0, n, 3000), np.arange(n - 2000, n)])
    for at in np.array_split(some, 11):
        i = dev(at)
        want, off = expected(q[i], codes, scales, dev(table[at]).long(), dev(pos[at]).long(), h ** -0.5)
        assert bf16_between(out[i], want, off), at
