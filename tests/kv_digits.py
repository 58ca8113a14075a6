"""Results of attention over the bf16 cache held to the digits that its products keep: what a result may be is between the roundings of the
two ends of an interval around the 64-bit value, and the interval is no wider than the arithmetic makes it."""
import numpy as np
import torch

from kv_cases import Setup, sees

STEP = 2.0 ** -24                                                 # half a step of binary32, relative
PARTS = 2.0 ** -15                                                # of a weight: 2^-7 of it, at most, are left to its lower digits, and 2^-8 of those is lost


def interval(q, k, v, p0, scale, window=0, sinks=0, each=PARTS):
    """q [T, H, h] at positions p0 ..; k, v [ctx, K, h]: the result and how far from it the kernels' sums may lie before they are
    rounded to bf16, both [T, H, h].  With weights w_j, A_j = |scale| sum |q_i k_ji| and n the positions that a row sees:

    * a score is a sum of h exact products and up to eight roundings in binary32, off by (h + 8) 2^-24 A_j, and its exponential by two
      steps more: w_j is off by w_j (exp(that) - 1), above and below the line: times |v_j| + |out|;
    * sums of n terms by several lanes and wavefronts, in runs of at most 64 + n / 4: 2^-24 of the sum of magnitudes each;
    * the weights that values are multiplied with have lost `each` of themselves, those that are summed have not."""
    T, H, h = q.shape
    G, ctx = H // k.shape[1], k.shape[0]
    seen = sees(T, p0, ctx, window, sinks)
    n = seen.sum(axis=1, keepdims=True)
    out, off = np.zeros((T, H, h)), np.zeros((T, H, h))
    for i in range(H):
        kk, vv = k[:, i // G], v[:, i // G]
        s = np.where(seen, scale * (q[:, i] @ kk.T), -np.inf)
        top = s.max(axis=1, keepdims=True)
        total = np.exp(s - top).sum(axis=1, keepdims=True)
        w = np.exp(s - top) / total
        o, mag = w @ vv, w @ np.abs(vv)
        wrong = (h + 8) * STEP * abs(scale) * (np.abs(q[:, i]) @ np.abs(kk).T) + 4 * STEP
        dw = np.where(seen, w * np.expm1(wrong), 0.0)
        d = dw @ np.abs(vv) + dw.sum(axis=1, keepdims=True) * np.abs(o) + (64 + n / 4) * STEP * (mag + np.abs(o)) + each * mag
        out[:, i], off[:, i] = o, 1.01 * d + 2 * STEP * np.abs(o)   # (products of these terms; the way to bf16 by binary32)
    return out, off


def limits(s, scale=None, skip=()):
    """What results of the rows of Setup s may be, from .. to (64 bits): [rows of samples, H, h]; anything for those of samples `skip`."""
    scale = s.h ** -0.5 if scale is None else scale
    q = s.q.double().numpy()
    bf16 = lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    lo, hi = np.full((2, s.start[-1], s.H, s.h), np.inf)
    lo *= -1
    for i, T in enumerate(s.lens):
        if not T or i in skip:
            continue
        rows = slice(s.start[i], s.start[i] + T)
        out, off = interval(q[rows], s.kv[i][0], s.kv[i][1], s.behind[i], scale, s.window, s.sinks)
        lo[rows], hi[rows] = bf16(out - off), bf16(out + off)
    return lo, hi


def check_digits(got, s, scale=None, what="", skip=()):
    """got: the call's output for the rows of Setup s, those of samples `skip` aside."""
    lo, hi = limits(s, scale, skip)
    got = got.float().cpu().double().numpy()[:s.start[-1]]
    fine = (lo <= got) & (got <= hi)
    for i in skip:
        fine[s.start[i]:s.start[i + 1]] = True
    if not fine.all():
        at = tuple(int(x) for x in np.argwhere(~fine)[0])
        raise AssertionError(f"{what}: {(~fine).sum()} of {fine.size}, the first at row, head, channel {at}: {got[at]}, {lo[at]} to {hi[at]} allowed")


__all__ = ["Setup", "check_digits", "interval", "limits"]
