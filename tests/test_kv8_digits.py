"""The bound of tests/kv8_digits.py tells arithmetic of the digits it counts from arithmetic of fewer: on the CPU, with both worked out."""
import numpy as np
import pytest
import torch

from kv8_digits import Setup, check_digits

bf16 = lambda x: torch.from_numpy(x).to(torch.bfloat16).double().numpy()


def cut_fp16(x):
    """To fp16 towards zero."""
    y = x.astype(np.float16)
    over = np.abs(y.astype(np.float64)) > np.abs(x)
    return np.where(over, np.nextafter(y, np.float16(0)), y).astype(np.float64)


def attend(s, weigh, value):
    """Every row with weights weigh(w), w at most 2^6, and values value(v): [rows, H, h]."""
    out = []
    for i, T in enumerate(s.lens):
        k, v = s.kv[i]
        for t in range(T):
            n = s.behind[i] + t + 1
            row = s.q[s.start[i] + t].double().numpy()
            x = np.stack([k[:n, j // (s.H // s.K)] @ row[j] for j in range(s.H)]) * s.h ** -0.5
            w = weigh(64.0 * np.exp(x - x.max(axis=1, keepdims=True)))
            top = np.stack([w[0][j] @ value(v[:n, j // (s.H // s.K)]) for j in range(s.H)])
            out.append(top / w[1].sum(axis=1, keepdims=True))
    return torch.from_numpy(np.stack(out)).to(torch.bfloat16)


FP16 = lambda v: v.astype(np.float16).astype(np.float64)
SAME = lambda w: (w, w)


@pytest.mark.parametrize("form,weigh,value,fine", [
    ("packed", lambda w: SAME(cut_fp16(w)), FP16, True),
    ("packed", lambda w: SAME(bf16(w)), bf16, False),
    ("packed", lambda w: SAME(bf16(w)), FP16, False),
    ("packed", lambda w: SAME(cut_fp16(w)), bf16, False),
    ("tokens", lambda w: (bf16(w) + bf16(w - bf16(w)), w), lambda v: v, True),
    ("tokens", lambda w: (bf16(w), w), lambda v: v, False),
    ("tokens", lambda w: SAME(cut_fp16(w)), FP16, False),
    ("general", lambda w: SAME(w), lambda v: v, True),
    ("general", lambda w: SAME(w), FP16, False),
], ids=["fp16", "bf16", "bf16 weights", "bf16 values", "two parts", "one part", "tokens in fp16", "binary32", "fp16 values"])
def test_what_the_bound_tells_apart(form, weigh, value, fine):
    s = Setup(4, 2, 64, 16, [40, 7], [0, 25], seed=2)
    got = attend(s, weigh, value)
    if fine:
        check_digits(got, s, form)
    else:
        with pytest.raises(AssertionError):
            check_digits(got, s, form)


def test_what_lies_behind_a_row_is_not_counted():
    """The bound of a row is the same whatever the values behind it are; a row of zeros in their place is told from the right one."""
    from kv8_digits import interval
    s, loud = (Setup(4, 2, 64, 16, [150], [0], seed=2, v_gain=lambda p, g=g: np.where(p >= 100, g, 1.0)) for g in (1.0, 2.0 ** 40))
    q = s.q.double().numpy()
    a, b = (interval(q, x.kv[0][0], x.kv[0][1], 0, s.h ** -0.5, "packed") for x in (s, loud))
    assert all(np.array_equal(x[:100], y[:100]) for x, y in zip(a, b))
    assert (a[1][:100] < 0.01).all()
    got = attend(loud, lambda w: SAME(cut_fp16(w)), lambda v: (v * 2.0 ** -30).astype(np.float16).astype(np.float64) * 2.0 ** 30)
    with pytest.raises(AssertionError):
        check_digits(got, loud, "packed")
