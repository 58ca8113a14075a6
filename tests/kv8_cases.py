"""The 8-bit cache in 64 bits (numpy), and caches and rows to try its operators on."""
import numpy as np
import torch

from paper_2505_18164_amd import mdi

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step of a type, relative


def quantise(x):
    """Codes and scales of rows x [..., h]: scale = max / 127 and c = 127 / max rounded to fp32, the code nearest to x c."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(all="ignore"):
        top = np.max(np.abs(x), axis=-1)
        fine = np.isfinite(x).all(axis=-1)
        some = fine & (top >= 2.0 ** -100)
        t = np.where(some, top, 1.0)
        c = (127.0 / t).astype(np.float32).astype(np.float64)
        scale = np.where(some, (t / 127.0).astype(np.float32), np.where(fine, np.float32(0), np.float32("nan"))).astype(np.float32)
        code = np.where(some[..., None], np.rint(np.where(some[..., None], x, 0.0) * c[..., None]), 0.0).astype(np.int8)
    return code, scale


def attention(q, k, v, p0, scale):
    """q [T, H, h] at positions p0 ..; k, v [ctx, K, h]: (out, sum of w |v|, largest sum of |scale q k| of a row [T, H, 1],
    2^-30 sum of |v| + 2^-36 max |v|)."""
    T, H, h = q.shape
    G = H // k.shape[1]
    out, mag, big, low = np.zeros((T, H, h)), np.zeros((T, H, h)), np.zeros((T, H, 1)), np.zeros((T, H, h))
    for i in range(H):
        kk, vv = k[:, i // G], v[:, i // G]
        s = scale * (q[:, i] @ kk.T)
        seen = np.arange(kk.shape[0])[None, :] <= p0 + np.arange(T)[:, None]
        s = np.where(seen, s, -np.inf)
        w = np.where(seen, np.exp(s - s.max(axis=1, keepdims=True)), 0.0)
        w /= w.sum(axis=1, keepdims=True)
        out[:, i], mag[:, i] = w @ vv, w @ np.abs(vv)
        big[:, i, 0] = np.where(seen, np.abs(scale) * (np.abs(q[:, i]) @ np.abs(kk).T), 0.0).max(axis=1)
        low[:, i] = 2.0 ** -30 * (seen @ np.abs(vv)) + 2.0 ** -36 * np.abs(vv).max()
    return out, mag, big, low


def bound(out, mag, big, low, h):
    """How far a bf16 result may be from `out`: its own rounding; one rounding to bf16 of every weight, of relative size
    2^-8, moves the weighted sum by up to 2^-8 sum w |v|, and the sum of weights likewise where it is taken of rounded ones;
    a score is a sum of h exact products and four factors in fp32, off by (h + 8) 2^-24 of the sum of magnitudes, which moves
    its weight by that, once above and once below the line; exponentials and the sums of up to 2^14 weights add 2^-24 each
    (pairwise or in runs of at most 2^7 by lane, so 2^7 2^-24 bounds them).  Weights that are rounded to fp16 with the
    largest one at 2^6 or more are off by 2^-11 of themselves, as above, or, below 2^-14, by half a step of 2^-24: 2^-31 of the
    largest, each of them, above and below the line; values in fp16 with the largest of a row at 2^12 or more by 2^-11 or
    2^-25 / 2^12 of the largest of any row (which may be a later row's)."""
    delta = (h + 8) * 2.0 ** -24 * big
    return 2.0 ** -8 * np.abs(out) + (2 * 2.0 ** -8 + 2 * delta + 2 * 2.0 ** -17) * mag * 1.01 + low * 1.01 + 1e-30


class Setup:
    """A cache on the GPU with `behind` earlier positions and `lens` new rows per sample, filled by the formula in 64 bits."""

    def __init__(self, H, K, h, pt, lens, behind, seed=0, spare=2, stale="nan", pos_of=None, k_gain=1.0, rows_behind=0, v_gain=None):
        rng = np.random.default_rng(seed)
        self.H, self.K, self.h, self.pt, self.lens, self.behind = H, K, h, pt, lens, behind
        n = len(lens)
        total = [a + b for a, b in zip(lens, behind)]
        used = [(t + pt - 1) // pt for t in total]
        stride = max(max(used), 1) + spare
        n_pages = sum(used) + 3
        order = rng.permutation(n_pages)
        self.tables = np.full((n, stride), 2 ** 31 - 7, dtype=np.int32)      # entries that nothing reaches
        self.codes = rng.integers(-127, 128, (n_pages, K, 2, pt, h)).astype(np.int8)
        self.scales = np.full((n_pages, K, 2, pt), np.nan if stale == "nan" else np.inf, dtype=np.float32)
        self.kv, at = [], 0
        for i in range(n):
            self.tables[i, :used[i]] = order[at:at + used[i]]
            at += used[i]
            x = rng.standard_normal((2, total[i], K, h)).astype(np.float32)
            x[0] *= k_gain
            if v_gain is not None:
                x[1] *= v_gain(np.arange(total[i]))[:, None, None]
            code, scale = quantise(x)
            self.kv.append(code.astype(np.float64) * scale.astype(np.float64)[..., None])
            for p in range(total[i]):
                page, slot = self.tables[i, p // pt], p % pt
                self.codes[page, :, :, slot] = code[:, p].transpose(1, 0, 2)
                self.scales[page, :, :, slot] = scale[:, p].T
        self.rows = sum(lens) + rows_behind
        self.start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.pos = np.asarray(behind, dtype=np.int32)
        self.max_ctx = max(max(total), 1)
        self.q = torch.from_numpy(rng.standard_normal((self.rows, H, h)).astype(np.float32)).bfloat16()

    def cache(self, err=True, **over):
        dev = lambda a: torch.from_numpy(np.array(a)).to("cuda:0")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda:0") if err else None
        return mdi.Kv8Cache(dev(over.get("codes", self.codes)), dev(over.get("scales", self.scales)), dev(over.get("tables", self.tables)), self.err)

    def plan(self, cache, one_each=False, **kw):
        dev = lambda a: torch.from_numpy(np.array(a)).to("cuda:0")
        kw.setdefault("max_ctx", self.max_ctx)
        return cache.rows(dev(self.pos), start=None if one_each else dev(self.start), n_rows=self.rows, **kw)

    def want(self, scale=None):
        scale = self.h ** -0.5 if scale is None else scale
        q = self.q.double().numpy()
        got = [attention(q[self.start[i]:self.start[i + 1]], self.kv[i][0], self.kv[i][1], self.behind[i], scale) for i in range(len(self.lens)) if self.lens[i]]
        return [np.concatenate(x) for x in zip(*got)]


def check(got, want, h, what=""):
    out, mag, big, low = want
    got = got.float().cpu().double().numpy()[:out.shape[0]]
    off, may = np.abs(got - out), bound(out, mag, big, low, h)
    if not (off <= may).all():
        at = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off / may)), off.shape)
        raise AssertionError(f"{what}: row, head, channel {at}: {got[at]} instead of {out[at]}, may be off by {may[at]:.3g}")
