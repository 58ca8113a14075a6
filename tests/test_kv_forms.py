"""Every form of the kernels of the cache in the storage type has a call that tests it: the plan itself is asked, on the CPU."""
import random

import kv_forms as F


def test_every_form_is_reached_and_none_besides():
    found = F.calls()
    assert {f for f, _ in found} == set(F.FORMS)
    assert {f for f, window in found if not window} == set(F.FORMS)
    assert set(F.FORMS) - {f for f, window in found if window} == set(F.NO_WINDOW)


def test_pieces_are_as_many_as_the_rows_need():
    """What a row may see, cut as the plan says, is no more pieces than the workspace has places for."""
    rng = random.Random(5)
    calls = []
    while len(calls) < 20000:
        K, G = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 3, 5, 8, 16, 32, 40])
        n, packed = int(2 ** rng.uniform(0, 14)), rng.random() < 0.7
        rows = int(2 ** rng.uniform(0, 18)) if packed else n
        ctx, window = int(2 ** rng.uniform(0, 20)), rng.choice([0, 0, int(2 ** rng.uniform(0, 17))])
        if rows * K * G < 1 << 24 and n * K * G * (ctx // 128 + 3) < 1 << 30:
            calls.append((rng.choice([F.BF16, F.F32]), K, rng.choice([24, 64, 96, 128, 256]), int(packed), n, rows, ctx, K * G, window, rng.choice([0, 4, 700]) if window else 0))
    for call, (kernel, chunk, splits, wgs, groups, rows, _, _) in zip(calls, F.plans(calls)):
        _, K, h, packed, _, _, ctx, H, window, sinks = call
        sh = 0
        while sh < 5 and (H // K) % (2 << sh) == 0:
            sh += 1
        per = (rows >> sh) if kernel == 1 else (16 * groups >> min(sh, 4)) if packed else 1      # positions of a workgroup
        if not window:
            most = -(-ctx // 64)
        elif kernel == 1:                                         # the first positions and a window that begins inside a block, each up to its last block
            most = min(-(-ctx // 64), -(-sinks // 64) + (window + per + 125) // 64)
        else:                                                     # both without the steps of up to 32 positions between them
            most = min(-(-ctx // 64), -(-(sinks + 31 + window + per - 1 + 31) // 64))
        if kernel:
            assert 1 <= splits <= 64 and chunk * splits >= most, (call, chunk, splits, most)
        else:
            assert splits == 1 or wgs == 512
