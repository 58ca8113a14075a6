"""What the 8-bit cache's entry points refuse on the host, before anything reaches a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from kv8_cases import quantise
from paper_2505_18164_amd import mdi

GOOD = dict(codes=4096, scales=8192, tables=64, err=None, n_pages=8, n_kv_head=2, head_dim=64, page_tokens=16, n_tables=2, table_stride=4)
ROWS = dict(table=None, start=16, pos=32, n=2, n_rows=9, max_ctx=64)


def cache(**over):
    f = dict(GOOD, **over)
    return mdi.MdiKv8(*[f[n] for n, _ in mdi.MdiKv8._fields_])


def rows(**over):
    f = dict(ROWS, **over)
    return mdi.MdiKv8Rows(*[f[n] for n, _ in mdi.MdiKv8Rows._fields_])


def bytes_of(c, r, heads=4):
    n = C.c_size_t(77)
    return mdi.lib().mdi_kv8_attn_bytes(C.byref(c) if c else None, C.byref(r) if r else None, heads, C.byref(n)), n.value


def test_sizes():
    assert C.sizeof(mdi.MdiKv8) == 4 * 8 + 6 * 4 and C.sizeof(mdi.MdiKv8Rows) == 3 * 8 + 3 * 4 + 4
    assert bytes_of(cache(), rows()) == (mdi.MDI_OK, 0)                        # short samples are not divided
    st, n = bytes_of(cache(table_stride=1000), rows(n_rows=2, max_ctx=16000, start=None))
    assert st == mdi.MDI_OK and n >= 2 * 4 * 2 * 66 * 4


@pytest.mark.parametrize("over", [dict(codes=None), dict(scales=None), dict(tables=None), dict(codes=4100), dict(scales=8196), dict(n_pages=0), dict(n_kv_head=0),
                                  dict(n_kv_head=1025), dict(head_dim=0), dict(head_dim=60), dict(head_dim=264), dict(page_tokens=0), dict(n_tables=0), dict(table_stride=0),
                                  dict(n_pages=1 << 31), dict(page_tokens=1 << 14, table_stride=16), dict(page_tokens=1, table_stride=(1 << 30) + 1)])
def test_caches_that_are_refused(over):
    assert bytes_of(cache(**over), rows(max_ctx=1))[0] == mdi.MDI_ERR_ARG


@pytest.mark.parametrize("over", [dict(pos=None), dict(start=None), dict(max_ctx=0), dict(max_ctx=65), dict(n_rows=(1 << 24) + 1), dict(n=1 << 31)])
def test_rows_that_are_refused(over):
    assert bytes_of(cache(), rows(**over))[0] == mdi.MDI_ERR_ARG


def test_calls_that_are_refused():
    L, c, r = mdi.lib(), cache(), rows()
    assert bytes_of(None, r)[0] == bytes_of(c, None)[0] == mdi.MDI_ERR_ARG
    for heads in (0, 3, 4098):
        assert bytes_of(c, r, heads)[0] == mdi.MDI_ERR_ARG
    assert L.mdi_kv8_attn_bytes(C.byref(c), C.byref(r), 4, None) == mdi.MDI_ERR_ARG
    for call in (L.mdi_kv8_write, L.mdi_kv8_read):
        for a in ((None, 16, 1, 128, 64), (16, None, 1, 128, 64), (16, 16, 2, 128, 64), (8, 16, 1, 128, 64), (16, 24, 1, 128, 64), (16, 16, 1, 4, 64), (16, 16, 1, 128, 4),
                  (16, 16, 0, 2, 64), (16, 16, 1, 1 << 39, 64)):
            assert call(C.byref(c), C.byref(r), *a, None) == mdi.MDI_ERR_ARG, a
        assert call(None, C.byref(r), 16, 16, 1, 128, 64, None) == mdi.MDI_ERR_ARG
        assert call(C.byref(c), C.byref(rows(n=0, n_rows=0, pos=None)), None, None, 1, 128, 64, None) == mdi.MDI_OK      # nothing to do
    for a in ((None, 256, 4, .1, 16, 256), (16, 256, 4, .1, None, 256), (24, 256, 4, .1, 16, 256), (16, 256, 4, .1, 24, 256), (16, 248, 4, .1, 16, 256), (16, 256, 4, .1, 16, 248),
              (16, 260, 4, .1, 16, 256), (16, 256, 3, .1, 16, 256), (16, 256, 4, float("nan"), 16, 256), (16, 256, 4, float("inf"), 16, 256)):
        assert L.mdi_kv8_attn(C.byref(c), C.byref(r), *a, None, 0, None) == mdi.MDI_ERR_ARG, a
    c, r = cache(table_stride=1000), rows(n_rows=2, max_ctx=16000, start=None)
    assert L.mdi_kv8_attn(C.byref(c), C.byref(r), 16, 256, 4, .1, 16, 256, None, 1 << 30, None) == mdi.MDI_ERR_ARG
    assert L.mdi_kv8_attn(C.byref(c), C.byref(r), 16, 256, 4, .1, 16, 256, 8, 1 << 30, None) == mdi.MDI_ERR_ARG
    assert L.mdi_kv8_attn(C.byref(c), C.byref(r), 16, 256, 4, .1, 16, 256, 16, bytes_of(c, r)[1] - 1, None) == mdi.MDI_ERR_NOMEM


def test_the_formula():
    code, scale = quantise(np.array([[1.0, -1.0, 0.5, 0.0], [0, 0, 0, 0], [2.0 ** -101, 0, 0, 0], [1, np.inf, 0, 0], [127, 0.5, 1.5, -2.5]]))
    assert code.tolist() == [[127, -127, 64, 0], [0] * 4, [0] * 4, [0] * 4, [127, 0, 2, -2]]     # ties to even: 63.5 is 64
    assert scale[1] == scale[2] == 0 and np.isnan(scale[3]) and scale[4] == 1


def test_partitions_with_8_bit_caches():
    from paper_2505_18164_amd import synth as S
    cfg = S.llama3_8b()
    c = mdi.make_config(cfg, max_seqs=16, kv_page_tokens=64, max_prefill=2048)
    plain, small = mdi.partition_bytes(c, 8, 16, 0), mdi.partition_bytes(c, 8, 16, mdi.MDI_KV8)
    rows = 8 * 16 * 8192 * 8 * 2                                              # layers, samples, positions, kv heads, key and value
    saved = rows * (2 * 128) - rows * (128 + 4)
    assert saved * 0.95 < plain - small <= saved
    n = C.c_size_t(0)

    def status(flags, lo=0, hi=2, over=None, **kw):
        c = mdi.make_config(dict(S.tiny(dtype=S.DT_BF16), **(over or {})), max_seqs=2, **kw)
        return mdi.lib().mdi_partition_bytes(C.byref(c), lo, hi, flags, C.byref(n))

    assert status(mdi.MDI_KV8) == mdi.MDI_OK
    assert status(mdi.MDI_KV8 | 1 | 2) == mdi.MDI_OK
    assert status(8) == mdi.MDI_ERR_ARG
    assert status(mdi.MDI_KV8, over=dict(dtype=S.DT_F32)) == mdi.MDI_ERR_ARG
    assert status(mdi.MDI_KV8 | 2, 2, 2) == mdi.MDI_ERR_ARG                   # no blocks, no cache
    assert status(mdi.MDI_KV8, over=dict(max_ctx=(1 << 24) + 1), kv_page_tokens=64) == mdi.MDI_ERR_ARG
    assert mdi.lib().mdi_prefill_batch(None, 1, None, None, None, None) == mdi.MDI_ERR_ARG


def test_limits_of_a_launch():
    big = dict(table_stride=1 << 16, n_kv_head=32, head_dim=128)
    assert bytes_of(cache(**big), rows(n=2, n_rows=(1 << 19) - 1, max_ctx=64), 32)[0] == mdi.MDI_OK
    assert bytes_of(cache(**big), rows(n=2, n_rows=1 << 19, max_ctx=64), 32)[0] == mdi.MDI_ERR_ARG             # 2^24 rows and heads
    assert bytes_of(cache(**big), rows(start=None, n=256, n_rows=256, max_ctx=1 << 20), 512)[0] == mdi.MDI_ERR_ARG      # 2^17 units of 2^13 tiles
    c, r = cache(**big), rows(n=2, n_rows=1 << 21, max_ctx=64)
    for call in (mdi.lib().mdi_kv8_write, mdi.lib().mdi_kv8_read):
        assert call(C.byref(c), C.byref(r), 16, 16, 1, 4096, 128, None) == mdi.MDI_ERR_ARG                      # 2^33 elements
    c, r = cache(), rows()
    assert mdi.lib().mdi_kv8_attn(C.byref(c), C.byref(r), 16, 256, 4, 3e38, 16, 256, None, 0, None) == mdi.MDI_ERR_ARG   # scale * log2 e


def test_what_the_python_calls_refuse():
    z = lambda *shape, dtype=torch.int32, device="cpu": torch.zeros(shape, dtype=dtype, device=device)
    codes, scales, tables = z(3, 2, 2, 16, 64, dtype=torch.int8), z(3, 2, 2, 16, dtype=torch.float32), z(2, 4)
    cache = mdi.Kv8Cache(codes, scales, tables)
    for a in ((codes[:, :, :1], scales, tables), (codes, scales[:2], tables), (codes, scales, tables[0]), (codes.float(), scales, tables),
              (codes, scales.double(), tables), (codes, scales, tables.long()), (codes.transpose(0, 1), scales.transpose(0, 1), tables), (codes, scales, tables.T)):
        with pytest.raises(ValueError):
            mdi.Kv8Cache(*a)
    pos, start = z(2), z(3)
    for a in (dict(pos=pos.long()), dict(pos=pos, start=start), dict(pos=pos, start=z(2), n_rows=4), dict(pos=pos, table=z(3)), dict(pos=pos, n_rows=-1),
              dict(pos=pos, max_ctx=(1 << 32) + 5), dict(pos=z(4)[::2])):
        with pytest.raises(ValueError):
            cache.rows(**a)
    rows = cache.rows(pos, start, n_rows=4)
    x, q = z(4, 2, 64, dtype=torch.bfloat16), z(4, 6, 64, dtype=torch.bfloat16)
    elsewhere = mdi.Kv8Cache(*(t.to("meta") for t in (codes, scales, tables)))
    for call in (cache.write, cache.read):
        for k, v in ((x[:3], x[:3]), (x, x.float()), (x.half(), x.half()), (x, x.transpose(0, 1).contiguous().transpose(0, 1)), (x.to("meta"), x.to("meta")),
                     (x[:, :, ::2], x[:, :, ::2])):
            with pytest.raises(ValueError):
                call(rows, k, v)
    with pytest.raises(ValueError):
        elsewhere.write(rows, x.to("meta"), x.to("meta"))                     # rows of another GPU
    for kw in (dict(q=q[:3]), dict(q=q.float()), dict(q=q[:, ::2]), dict(q=q.to("meta")), dict(q=q, out=q[:, :4]), dict(q=q, out=q.float()),
               dict(q=q, workspace=z(64).to("meta")), dict(q=q, workspace=z(64)[::2])):
        with pytest.raises(ValueError):
            cache.attn(rows, **kw)
    with pytest.raises(ValueError):
        elsewhere.attn(rows, q.to("meta"))


def test_rows_of_a_pass_of_a_partition():
    from paper_2505_18164_amd import synth as S
    n = C.c_size_t(0)

    def status(**kw):
        c = mdi.make_config(S.tiny(dtype=S.DT_BF16, n_head=4, n_kv_head=2, head_dim=64, d_model=256, max_ctx=1 << 22), max_seqs=1, kv_page_tokens=64, **kw)
        return mdi.lib().mdi_partition_bytes(C.byref(c), 0, 1, mdi.MDI_KV8, C.byref(n))

    assert status() == mdi.MDI_ERR_ARG                                        # a first visit of 2^22 rows: 2^24 rows and heads
    assert status(max_prefill=(1 << 22) - 1) == status(max_prefill=1024) == mdi.MDI_OK
