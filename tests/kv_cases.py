"""The cache in the storage type in 64 bits (numpy), and caches and rows to try its operators on."""
import numpy as np
import torch

from paper_2505_18164_amd import mdi

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of a type, relative
U = 2.0 ** -24


def sees(T, p0, ctx, window=0, sinks=0):
    """[T, ctx]: does the row at position p0 + t see position j."""
    p, j = p0 + np.arange(T)[:, None], np.arange(ctx)[None, :]
    return (j <= p) & ((p - j < window) | (j < sinks) if window else True)


def attention(q, k, v, p0, scale, window=0, sinks=0):
    """q [T, H, h] at positions p0 ..; k, v [ctx, K, h]: (out, sum of w |v|, largest sum of |scale q k| of a row [T, H, 1],
    positions a row sees [T, 1, 1])."""
    T, H, h = q.shape
    G, ctx = H // k.shape[1], k.shape[0]
    seen = sees(T, p0, ctx, window, sinks)
    out, mag, big = np.zeros((T, H, h)), np.zeros((T, H, h)), np.zeros((T, H, 1))
    for i in range(H):
        kk = np.where(seen.any(axis=0)[:, None], k[:, i // G], 0.0)
        vv = np.where(seen.any(axis=0)[:, None], v[:, i // G], 0.0)
        s = np.where(seen, scale * (q[:, i] @ kk.T), -np.inf)
        w = np.where(seen, np.exp(s - s.max(axis=1, keepdims=True)), 0.0)
        w /= w.sum(axis=1, keepdims=True)
        out[:, i], mag[:, i] = w @ vv, w @ np.abs(vv)
        big[:, i, 0] = np.where(seen, np.abs(scale) * (np.abs(q[:, i]) @ np.abs(kk).T), 0.0).max(axis=1)
    return out, mag, big, seen.sum(axis=1)[:, None, None] + np.zeros((T, H, 1))


def bound(out, mag, big, n, h, dtype):
    """How far a result may be from `out`.  Its own rounding: half a step.  A score is a sum of h products (exact, or rounded once) and
    a few factors in fp32, off by (h + 8) 2^-24 of the sum of magnitudes, which moves its weight by that; an exponential
    is good to a few 2^-24, and sums over n positions, in whatever order, add up to n of them; each of these counts above and below
    the line.  With bf16 every weight may be rounded to bf16, 2^-8 of itself, above and below the line."""
    each = (h + 8) * U * big + (n + 16) * U + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    return HALF[dtype] * np.abs(out) + 2.02 * each * mag + 1e-30


def heads(x, pos, g=None, b=None, norm="rms", eps=1e-6, freq=None):
    """Head rows x [rows, heads, h] at positions pos [rows] normalised and rotated: (what they become, how far fp32 arithmetic may be
    from it).  Per channel: a sum of h terms above and below the line, (2 h + 32) 2^-24 of the magnitudes that meet in it; a
    mean that is off moves the deviation's root as well, by as many deviations as the channel is from it; angles are good to a
    few 2^-24 of a turn, of which the two channels of a pair each take their share."""
    x = np.asarray(x, dtype=np.float64)
    h = x.shape[-1]
    mag = np.abs(x)
    if g is not None:
        mean = x.mean(-1, keepdims=True) if norm == "layer" else 0.0
        by = 1.0 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
        away = np.abs(x - mean) * by
        mag = (np.abs(x) + (np.abs(x).mean(-1, keepdims=True) if norm == "layer" else 0.0)) * by * np.abs(g) * (1 + away) + (0 if b is None else np.abs(b))
        x = (x - mean) * by * g + (0 if b is None else b)
    off = (2 * h + 32) * U * mag if g is not None else 0.0 * mag
    if freq is not None and len(freq):
        r = len(freq)
        a = np.asarray(pos, dtype=np.float64)[:, None, None] * np.asarray(freq)
        c, s = np.cos(a), np.sin(a)
        y, both = x.copy(), np.abs(x[..., :r]) + np.abs(x[..., r:2 * r])
        y[..., :r], y[..., r:2 * r] = x[..., :r] * c - x[..., r:2 * r] * s, x[..., r:2 * r] * c + x[..., :r] * s
        more = off[..., :r] + off[..., r:2 * r] + 32 * U * both
        x, off = y, off.copy()
        off[..., :r] = off[..., r:2 * r] = more
    return x, off


def within(got, want, may, what=""):
    got = got.float().cpu().double().numpy() if isinstance(got, torch.Tensor) else got
    off = np.abs(got - want)
    if not (off <= may).all():
        at = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off / np.maximum(may, 1e-300))), off.shape)
        raise AssertionError(f"{what}: at {at}: {got[at]} instead of {want[at]}, may be off by {may[at]:.3g}; {(~(off <= may)).sum()} of {off.size}")


def dev(a):
    return torch.from_numpy(np.array(a)).to("cuda:0")


class Setup:
    """A cache with `behind` earlier positions and `lens` new rows per sample.  What nobody sees of it is NaN (or `stale`), pages that nobody
    sees are not there: their table entries are wild."""

    def __init__(self, H, K, h, pt, lens, behind, dtype=torch.bfloat16, window=0, sinks=0, seed=0, spare=2, stale=float("nan"), k_gain=1.0, v_gain=None,
                 rows_behind=0, change=None):
        rng = np.random.default_rng(seed)
        self.H, self.K, self.h, self.pt, self.lens, self.behind, self.dtype, self.window, self.sinks = H, K, h, pt, lens, behind, dtype, window, sinks
        n = len(lens)
        total = [a + b for a, b in zip(lens, behind)]
        used = [(t + pt - 1) // pt for t in total]
        stride = max(max(used), 1) + spare
        some = [sees(lens[i], behind[i], total[i], window, sinks).any(axis=0) for i in range(n)]
        n_pages = sum(used) + 3
        order = rng.permutation(n_pages)
        self.tables = np.full((n, stride), 2 ** 31 - 7, dtype=np.int32)
        data = np.full((n_pages, K, 2, pt, h), stale, dtype=np.float32)
        self.kv, at = [], 0
        for i in range(n):
            x = rng.standard_normal((2, total[i], K, h)).astype(np.float32)
            x[0] *= k_gain
            if v_gain is not None:
                x[1] *= v_gain(np.arange(total[i]))[:, None, None]
            if change is not None:
                change(i, x)
            x = torch.from_numpy(x).to(dtype).float().numpy()
            self.kv.append(x.astype(np.float64))
            for page in range(used[i]):
                here = np.arange(page * pt, min((page + 1) * pt, total[i]))
                here = here[some[i][here]]
                if len(here):
                    self.tables[i, page] = order[at]
                    data[order[at]][:, :, here - page * pt] = x[:, here].transpose(2, 0, 1, 3)
                    at += 1
        self.data = torch.from_numpy(data).to(dtype)
        self.rows = sum(lens) + rows_behind
        self.start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.pos = np.asarray(behind, dtype=np.int32)
        self.max_ctx = max(max(total), 1)
        q = torch.from_numpy(rng.standard_normal((sum(lens) + min(rows_behind, 3), H, h)).astype(np.float32)).to(dtype)
        self.q = torch.cat([q, torch.zeros((self.rows - q.shape[0], H, h), dtype=dtype)])

    def cache(self, err=True):
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda:0") if err else None
        return mdi.KvCache(self.data.to("cuda:0"), dev(self.tables), self.err)

    def plan(self, cache, one_each=False, **kw):
        kw.setdefault("max_ctx", self.max_ctx)
        return cache.rows(dev(self.pos), start=None if one_each else dev(self.start), n_rows=self.rows, **kw)

    def attn(self, cache, plan, **kw):
        return cache.attn(plan, self.q.to("cuda:0"), window=self.window, sinks=self.sinks, **kw)

    def want(self, scale=None):
        scale = self.h ** -0.5 if scale is None else scale
        q = self.q.double().numpy()
        got = [attention(q[self.start[i]:self.start[i + 1]], self.kv[i][0], self.kv[i][1], self.behind[i], scale, self.window, self.sinks)
               for i in range(len(self.lens)) if self.lens[i]]
        return [np.concatenate(x) for x in zip(*got)]

    def check(self, got, want=None, what=""):
        want = self.want() if want is None else want
        within(got[:want[0].shape[0]], want[0], bound(*want, self.h, self.dtype), what)
