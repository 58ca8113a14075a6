"""Attention over the bf16 cache keeps sixteen digits of its weights, whichever kernel serves the call: how exact a row is does not depend on how
many others are in its call."""
import pytest
import torch

from kv_digits import Setup, check_digits

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
# Rows of nobody behind the last sample, times heads: so many that the call is taken for a large one.
CROWDS = [0, 30000, 80000, 200000]


@pytest.mark.parametrize("sight", [(0, 0), (50, 3), (200, 70)], ids=["all", "window", "wide window"])
@pytest.mark.parametrize("crowd", CROWDS)
@pytest.mark.parametrize("H,K,h,pt,lens,behind", [
    (4, 2, 64, 16, [1, 17, 64, 65], [0, 0, 0, 90]), (8, 2, 64, 64, [300], [40]), (8, 8, 128, 64, [128, 1, 63], [0, 200, 1]), (6, 2, 128, 7, [70], [59]),
    (16, 2, 128, 128, [300], [300]), (5, 5, 96, 16, [100, 11], [6, 0]), (4, 1, 256, 16, [60], [30])])
def test_packed_rows_keep_sixteen_digits(H, K, h, pt, lens, behind, crowd, sight):
    s = Setup(H, K, h, pt, lens, behind, BF16, *sight, seed=3, rows_behind=crowd // H)
    cache = s.cache()
    check_digits(s.attn(cache, s.plan(cache)), s)
    cache.check()


@pytest.mark.parametrize("sight", [(0, 0), (900, 100)], ids=["all", "window"])
@pytest.mark.parametrize("H,K,h,pt,lens,behind", [
    (32, 4, 128, 64, [100, 64], [1900, 2500]), (32, 2, 128, 24, [90], [2900]), (32, 4, 64, 24, [130, 100], [1500, 2500]), (32, 4, 64, 64, [130, 1], [2500, 30]),
    (8, 2, 128, 64, [3], [2500]), (4, 2, 96, 16, [30], [2100]), (2, 1, 256, 16, [9], [1800])])
def test_pieces_that_are_joined_keep_them(H, K, h, pt, lens, behind, sight):
    s = Setup(H, K, h, pt, lens, behind, BF16, *sight, seed=5, rows_behind=2)
    cache = s.cache()
    check_digits(s.attn(cache, s.plan(cache)), s)
    cache.check()


@pytest.mark.parametrize("sight", [(0, 0), (700, 5)], ids=["all", "window"])
@pytest.mark.parametrize("H,K,h,pt", [(8, 2, 64, 16), (6, 3, 64, 40), (4, 2, 128, 64), (20, 1, 128, 7), (4, 2, 40, 16), (2, 1, 256, 16)])
def test_single_tokens_keep_them(H, K, h, pt, sight):
    s = Setup(H, K, h, pt, [1] * 6, [0, 16, 299, 63, 64, 1700], BF16, *sight, seed=4)
    cache = s.cache()
    check_digits(s.attn(cache, s.plan(cache, one_each=True)), s)
    cache.check()
