"""The bound of tests/kv_digits.py tells arithmetic of the digits it counts from arithmetic of fewer: on the CPU, with both worked out."""
import numpy as np
import pytest
import torch

from kv_digits import Setup, check_digits
from kv_forms import ones

bf16 = lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()
upper = lambda w: (w.astype(np.float32).view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32).astype(np.float64)


def attend(s, weigh):
    """Every row with weights weigh(w): those that values are multiplied with, and those that are summed."""
    out = []
    for i, T in enumerate(s.lens):
        k, v = s.kv[i]
        for t in range(T):
            p = s.behind[i] + t
            seen = np.array([j for j in range(p + 1) if not s.window or p - j < s.window or j < s.sinks])
            row = s.q[s.start[i] + t].double().numpy()
            x = np.stack([k[seen, j // (s.H // s.K)] @ row[j] for j in range(s.H)]) * s.h ** -0.5
            w = weigh(np.exp(x - x.max(axis=1, keepdims=True)))
            out.append(np.stack([w[0][j] @ v[seen, j // (s.H // s.K)] for j in range(s.H)]) / w[1].sum(axis=1, keepdims=True))
    return torch.from_numpy(np.stack(out)).to(torch.bfloat16)


@pytest.mark.parametrize("sight", [(0, 0), (20, 3)], ids=["all", "window"])
@pytest.mark.parametrize("weigh,fine", [
    (lambda w: (w, w), True),
    (lambda w: (bf16(w) + bf16(w - bf16(w)), w), True),
    (lambda w: (upper(w) + bf16(w - upper(w)), w), True),
    (lambda w: (bf16(w), w), False),
    (lambda w: (bf16(w), bf16(w)), False),
    (lambda w: (upper(w), w), False),
    (lambda w: (w.astype(np.float16).astype(np.float64), w), False),
], ids=["whole", "two parts", "cut and the rest", "one part", "one part, summed as rounded", "cut", "eleven digits"])
def test_what_the_bound_tells_apart(weigh, fine, sight):
    s = Setup(4, 2, 64, 16, [40, 7], [0, 25], torch.bfloat16, *sight, seed=2)
    got = attend(s, weigh)
    if fine:
        check_digits(got, s)
    else:
        with pytest.raises(AssertionError):
            check_digits(got, s)


def test_a_position_too_few_is_told():
    """In a context of 2000 positions the bound knows a result that lacks one of them."""
    s = Setup(2, 1, 64, 16, [1], [1999], torch.bfloat16, seed=3)
    check_digits(attend(s, lambda w: (w, w)), s)
    for lost in (0, 63, 64, 1024, 1998):
        def without(w):
            w = w.copy()
            w[:, lost] = 0
            return w, w
        with pytest.raises(AssertionError):
            check_digits(attend(s, without), s)


@pytest.mark.parametrize("K,h,ctx", [(2, 24, 2500), (1, 64, 6000), (2, 128, 700)])
def test_a_position_more_or_less_is_told_from_ones(K, h, ctx):
    """Weights that are all alike, every position a one in one channel: any position that is missing, or counted twice."""
    s = Setup(2 * K, K, h, 16, [1], [ctx - 1], torch.bfloat16, seed=3, change=ones(K, h, 64))
    check_digits(attend(s, lambda w: (w, w)), s)
    for p in list(range(0, ctx, 97)) + [63, 64, ctx - 1]:
        for times in (0.0, 2.0):
            def other(w):
                w = w.copy()
                w[:, p] *= times
                return w, w
            with pytest.raises(AssertionError):
                check_digits(attend(s, other), s)
