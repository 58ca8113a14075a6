"""Every form of the kernels of the cache in the storage type against 64 bits: digits, and every position counted once."""
import pytest
import torch

import kv_forms as F
from kv_cases import Setup
from kv_digits import check_digits

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
