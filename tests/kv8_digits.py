"""Results of the 8-bit cache's attention held to the digits that its products keep: what a bf16 result may be is between the
roundings of the two ends of an interval around the 64-bit value, and the interval is no wider than the arithmetic makes it.
It counts what a row sees, and nothing that lies behind it."""
import numpy as np
import torch

from kv8_cases import Setup

STEP = 2.0 ** -24                                                 # half a step of binary32, relative


def interval(q, k, v, p0, scale, form):
    """q [T, H, h] at positions p0 ..; k, v [ctx, K, h]: the result and how far from it the kernels' sums may lie before they are
    rounded to bf16, both [T, H, h].  With weights w_j, A_j = |scale| sum |q_i k_ji| and n the positions that a row sees:

    * a score is a sum of h exact products and up to eight roundings in binary32, off by (h + 8) 2^-24 A_j, and its exponential by two
      steps more: w_j is off by w_j (exp(that) - 1), above and below the line: times |v_j| + |out|;
    * sums of n terms by several lanes and wavefronts, in runs of at most 64 + n / 4: 2^-24 of the sum of magnitudes each;
    * `tokens`: the product of a weight and a value's scale is cut to 8 digits and what that leaves, less than 2^-7 of it, rounded to
      bf16: 2^-15 w_j |v_j|;
    * `packed` (heads of 64 or 128): weights are cut to fp16, the same ones above and below the line.  A factor that all have in common
      falls out, so what counts is the distance from the middle, 2^-11 w_j (|v_j| + |out|) - or, for weights below 2^-14 where the
      largest has 2^6, the cut of 2^-24, 2^-30 of the sum of weights: 2^-30 (|v_j| + |out|) each; values to fp16, 2^-11 w_j |v_j|;
    * `general`: nothing more."""
    T, H, h = q.shape
    G = H // k.shape[1]
    out, off = np.zeros((T, H, h)), np.zeros((T, H, h))
    for i in range(H):
        kk, vv = k[:, i // G], v[:, i // G]
        seen = np.arange(kk.shape[0])[None, :] <= p0 + np.arange(T)[:, None]
        s = np.where(seen, scale * (q[:, i] @ kk.T), -np.inf)
        top = s.max(axis=1, keepdims=True)
        total = np.exp(s - top).sum(axis=1, keepdims=True)
        w = np.exp(s - top) / total
        o = w @ vv
        wrong = (h + 8) * STEP * abs(scale) * (np.abs(q[:, i]) @ np.abs(kk).T) + 4 * STEP
        dw = np.where(seen, np.exp(np.minimum(s - top + wrong, 700.0)) / total - w, 0.0)
        mag, n = w @ np.abs(vv), seen.sum(axis=1, keepdims=True)
        d = dw @ np.abs(vv) + dw.sum(axis=1, keepdims=True) * np.abs(o) + (64 + n / 4) * STEP * (mag + np.abs(o))
        if form == "tokens":
            d = d + 2.0 ** -15 * mag
        elif form == "packed":
            d = d + 2.0 ** -11 * (2 * mag + np.abs(o)) + 2.0 ** -30 * (seen @ np.abs(vv) + n * np.abs(o))
        out[:, i], off[:, i] = o, 1.01 * d + 2 * STEP * np.abs(o)   # (products of these terms; the way to bf16 by binary32)
    return out, off


def check_digits(got, s, form, scale=None, what=""):
    """got: the call's output for the rows of Setup s."""
    scale = s.h ** -0.5 if scale is None else scale
    q = s.q.double().numpy()
    bf16 = lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    got = got.float().cpu().double().numpy()
    for i, T in enumerate(s.lens):
        if not T:
            continue
        rows = slice(s.start[i], s.start[i] + T)
        out, off = interval(q[rows], s.kv[i][0], s.kv[i][1], s.behind[i], scale, form)
        lo, hi = bf16(out - off), bf16(out + off)
        fine = (lo <= got[rows]) & (got[rows] <= hi)
        if not fine.all():
            at = tuple(np.argwhere(~fine)[0])
            raise AssertionError(f"{what} sample {i}: {(~fine).sum()} of {fine.size}, the first at row, head, channel {at}: {got[rows][at]} "
                                 f"instead of {out[at]}, {lo[at]} to {hi[at]} allowed")


def form_of(h, one_each=False):
    return "general" if h not in (64, 128) else "tokens" if one_each else "packed"


def rekeyed(s, i, positions, sign):
    """Sample i's keys at `positions` get the sign `sign` in every channel (with queries above zero: their scores have it)."""
    for p in positions:
        page, slot = s.tables[i, p // s.pt], p % s.pt
        s.codes[page, :, 0, slot] = sign * np.abs(s.codes[page, :, 0, slot])
        s.kv[i][0, p] = sign * np.abs(s.kv[i][0, p])
    return s


__all__ = ["Setup", "check_digits", "form_of", "interval", "rekeyed"]
