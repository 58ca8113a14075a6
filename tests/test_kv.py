"""What the entry points of the cache in the storage type refuse on the host, before anything reaches a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from kv_cases import attention, heads, sees
from paper_2505_18164_amd import mdi

GOOD = dict(data=4096, tables=64, err=None, dtype=1, n_pages=8, n_kv_head=2, head_dim=64, page_tokens=16, n_tables=2, table_stride=4)
ROWS = dict(table=None, start=16, pos=32, n=2, n_rows=9, max_ctx=64)
PREP = dict(q_g=16, q_b=None, k_g=16, k_b=None, freq=8, eps=1e-6, norm_kind=1, rot=64)


def make(kind, good, **over):
    f = dict(good, **over)
    return kind(*[f[n] for n, _ in kind._fields_])


def cache(**over):
    return make(mdi.MdiKv, GOOD, **over)


def rows(**over):
    return make(mdi.MdiKv8Rows, ROWS, **over)


def prep(**over):
    return make(mdi.MdiQkPrep, PREP, **over)


def ref(x):
    return None if x is None else C.byref(x)


def bytes_of(c, r, heads=4, window=0, sinks=0):
    n = C.c_size_t(77)
    return mdi.lib().mdi_kv_attn_bytes(ref(c), ref(r), heads, window, sinks, C.byref(n)), n.value


def append(c=None, r=None, p=None, **over):
    f = dict(k=16, v=16, row=128, head=64, q=16, q_row=256, q_head=64, n_head=4, out=16, out_row=256)
    f.update(over)
    return mdi.lib().mdi_kv_append(ref(c or cache()), ref(r or rows()), ref(p), f["k"], f["v"], f["row"], f["head"], f["q"], f["q_row"], f["q_head"], f["n_head"],
                                   f["out"], f["out_row"], None)


def attn(c=None, r=None, **over):
    f = dict(q=16, q_row=256, heads=4, scale=.1, window=0, sinks=0, out=16, out_row=256, ws=None, size=0)
    f.update(over)
    return mdi.lib().mdi_kv_attn(ref(c or cache()), ref(r or rows()), f["q"], f["q_row"], f["heads"], f["scale"], f["window"], f["sinks"], f["out"], f["out_row"],
                                 f["ws"], f["size"], None)


def test_sizes():
    assert C.sizeof(mdi.MdiKv) == 3 * 8 + 7 * 4 + 4 and C.sizeof(mdi.MdiQkPrep) == 5 * 8 + 3 * 4 + 4
    assert bytes_of(cache(), rows()) == (mdi.MDI_OK, 0)                        # short samples are not divided
    long = cache(table_stride=1000), rows(n_rows=2, max_ctx=16000, start=None)
    st, n = bytes_of(*long)
    assert st == mdi.MDI_OK and n >= 2 * 4 * 2 * 66 * 4
    assert bytes_of(*long, window=100, sinks=4) == (mdi.MDI_OK, 0)             # nor is a short window
    assert bytes_of(*long, window=0, sinks=1 << 31) == (st, n) == bytes_of(*long, window=(1 << 32) - 1, sinks=(1 << 32) - 1)


@pytest.mark.parametrize("over", [dict(data=None), dict(tables=None), dict(data=4104), dict(dtype=2), dict(n_pages=0), dict(n_kv_head=0), dict(n_kv_head=1025),
                                  dict(head_dim=0), dict(head_dim=60), dict(head_dim=264), dict(page_tokens=0), dict(n_tables=0), dict(table_stride=0),
                                  dict(n_pages=1 << 31), dict(page_tokens=1 << 14, table_stride=16), dict(page_tokens=1, table_stride=(1 << 30) + 1)])
def test_caches_that_are_refused(over):
    c, r = cache(**over), rows(max_ctx=1)
    assert bytes_of(c, r)[0] == append(c, r) == attn(c, r) == mdi.MDI_ERR_ARG


@pytest.mark.parametrize("over", [dict(pos=None), dict(start=None), dict(max_ctx=0), dict(max_ctx=65), dict(n_rows=(1 << 24) + 1), dict(n=1 << 31)])
def test_rows_that_are_refused(over):
    r = rows(**over)
    assert bytes_of(cache(), r)[0] == append(None, r) == attn(None, r) == mdi.MDI_ERR_ARG


@pytest.mark.parametrize("over", [dict(k=None), dict(v=None), dict(k=8), dict(v=24), dict(row=4), dict(head=4), dict(row=1 << 39), dict(head=1 << 39), dict(q=None), dict(out=None),
                                  dict(q=8), dict(out=24), dict(q_row=4), dict(q_head=4), dict(q_row=1 << 39), dict(q_head=1 << 39), dict(out_row=260), dict(out_row=248), dict(out_row=1 << 39),
                                  dict(n_head=3), dict(n_head=4098), dict(n_head=0), dict(n_head=0, q=None), dict(n_head=0, out=None)])
def test_appends_that_are_refused(over):
    assert append(**over) == mdi.MDI_ERR_ARG


@pytest.mark.parametrize("over", [dict(norm_kind=2), dict(rot=72), dict(rot=60), dict(rot=4), dict(freq=None), dict(freq=4), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")),
                                  dict(q_g=8), dict(k_g=24), dict(q_b=8), dict(k_b=4), dict(q_g=None, q_b=16), dict(k_g=None, k_b=16)])
def test_preparations_that_are_refused(over):
    assert append(p=prep(**over)) == mdi.MDI_ERR_ARG


@pytest.mark.parametrize("over", [dict(q=None), dict(out=None), dict(q=24), dict(out=24), dict(q_row=248), dict(out_row=248), dict(q_row=260), dict(out_row=1 << 39), dict(heads=0),
                                  dict(heads=3), dict(heads=4098), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38)])
def test_attentions_that_are_refused(over):
    assert attn(**over) == mdi.MDI_ERR_ARG


def test_workspaces_and_nothing_to_do():
    assert mdi.lib().mdi_kv_attn_bytes(ref(cache()), ref(rows()), 4, 0, 0, None) == mdi.MDI_ERR_ARG
    assert mdi.lib().mdi_kv_attn_bytes(None, ref(rows()), 4, 0, 0, C.byref(C.c_size_t())) == mdi.MDI_ERR_ARG
    assert bytes_of(cache(), None)[0] == mdi.MDI_ERR_ARG
    c, r = cache(table_stride=1000), rows(n_rows=2, max_ctx=16000, start=None)
    assert attn(c, r, size=1 << 30) == attn(c, r, ws=8, size=1 << 30) == mdi.MDI_ERR_ARG
    assert attn(c, r, ws=16, size=bytes_of(c, r)[1] - 1) == mdi.MDI_ERR_NOMEM
    none = rows(n=0, n_rows=0, pos=None)
    assert append(None, none, prep(), k=None, v=None, q=None, out=None) == attn(None, none, q=None, out=None) == mdi.MDI_OK
    assert append(None, none, None, k=None, v=None, q=None, out=None, n_head=0) == mdi.MDI_OK


def test_results_in_the_place_of_queries():
    r = rows(n_rows=4)
    assert attn(cache(), r, q=4096, out=4096) == mdi.MDI_ERR_ARG
    for kw in (dict(out_row=512), dict(q_head=128, q_row=1024, out_row=1024)):                                 # laid out otherwise
        assert append(cache(), r, None, q=4096, out=4096, **{**dict(n_head=4, q_row=256, q_head=64, out_row=256), **kw}) == mdi.MDI_ERR_ARG


def test_limits_of_a_launch():
    big = dict(table_stride=1 << 16, n_kv_head=32, head_dim=128)
    assert bytes_of(cache(**big), rows(n=2, n_rows=(1 << 19) - 1, max_ctx=64), 32)[0] == mdi.MDI_OK
    assert bytes_of(cache(**big), rows(n=2, n_rows=1 << 19, max_ctx=64), 32)[0] == mdi.MDI_ERR_ARG             # 2^24 rows and heads
    assert bytes_of(cache(**big), rows(start=None, n=256, n_rows=256, max_ctx=1 << 20), 512)[0] == mdi.MDI_ERR_ARG      # 2^17 units of 2^13 tiles
    assert append(cache(**big), rows(n_rows=1 << 20), n_head=32, row=4096, head=128, q_row=4096, q_head=128, out_row=4096) == mdi.MDI_ERR_ARG     # 2^33 elements and more


def test_what_the_python_calls_refuse():
    z = lambda *shape, dtype=torch.int32, device="cpu": torch.zeros(shape, dtype=dtype, device=device)
    data, tables = z(3, 2, 2, 16, 64, dtype=torch.bfloat16), z(2, 4)
    cache = mdi.KvCache(data, tables)
    for a in ((data[:, :, :1], tables), (data[0], tables), (data, tables[0]), (data.half(), tables), (data, tables.long()), (data.transpose(0, 1), tables),
              (data, tables.T), (data, tables, z(1).float())):
        with pytest.raises(ValueError):
            mdi.KvCache(*a)
    g, f = z(64, dtype=torch.float32), z(32, dtype=torch.float64)
    for kw in (dict(norm="group"), dict(q_gain=g.double()), dict(k_gain=g[:32]), dict(q_gain=g, q_bias=g.bfloat16()), dict(freq=f.float()), dict(freq=f.unsqueeze(0)),
               dict(freq=z(64, dtype=torch.float64)[::2]), dict(freq=f.to("meta"))):
        with pytest.raises(ValueError):
            cache.prep(**kw)
    rows = cache.rows(z(2), z(3), n_rows=4)
    x, q = z(4, 2, 64, dtype=torch.bfloat16), z(4, 6, 64, dtype=torch.bfloat16)
    elsewhere = mdi.KvCache(data.to("meta"), tables.to("meta"))
    for a in ((x[:3], x[:3]), (x, x.float()), (x.float(), x.float()), (x, x.transpose(0, 1).contiguous().transpose(0, 1)), (x.to("meta"), x.to("meta")), (x[:, :, ::2], x[:, :, ::2]),
              (x, x, q[:3]), (x, x, q.float()), (x, x, q[:, 0]), (x, x, q, None, q[:, :4]), (x, x, q, None, q.float()), (x, x, q, None, z(4, 12, 64, dtype=torch.bfloat16)[:, ::2]),
              (x, x, None, None, q), (x, x, q, elsewhere.prep())):
        with pytest.raises(ValueError):
            cache.append(rows, *a)
    with pytest.raises(ValueError):
        elsewhere.append(rows, x.to("meta"), x.to("meta"))
    for kw in (dict(q=q[:3]), dict(q=q.float()), dict(q=q[:, ::2]), dict(q=q.to("meta")), dict(q=q, out=q[:, :4]), dict(q=q, out=q.float()), dict(q=q, workspace=z(64).to("meta")),
               dict(q=q, workspace=z(64)[::2]), dict(q=q, window=-1), dict(q=q, window=1 << 32), dict(q=q, window=1, sinks=-1)):
        with pytest.raises(ValueError):
            cache.attn(rows, **kw)
    with pytest.raises(ValueError):
        elsewhere.attn(rows, q.to("meta"))
    with pytest.raises(mdi.MdiError):
        cache.workspace(rows, 5)


def test_the_formulas():
    s = sees(3, 4, 7, 3, 1)                                                    # rows at 4, 5, 6: three newest and the first
    assert s.astype(int).tolist() == [[1, 0, 1, 1, 1, 0, 0], [1, 0, 0, 1, 1, 1, 0], [1, 0, 0, 0, 1, 1, 1]]
    assert sees(2, 0, 2).astype(int).tolist() == [[1, 0], [1, 1]]
    q, kv = np.zeros((1, 1, 8)), np.arange(24.0).reshape(3, 1, 8)
    assert np.allclose(attention(q, kv, kv, 2, 1.0, 2)[0][0, 0], kv[1:, 0].mean(axis=0))
    x, off = heads(np.array([[[3.0, 4, 0, 0]]]), [2], g=np.full(4, 2.0), eps=0.0)
    assert np.allclose(x, [[[2.4, 3.2, 0, 0]]]) and (off > 0).any()
    x, _ = heads(np.array([[[3.0, 5, 1, 7]]]), [2], g=np.ones(4), norm="layer", eps=0.0)
    assert np.allclose(x, [[np.array([-1, 1, -3, 3]) / 5 ** 0.5]])
    x, _ = heads(np.array([[[1.0, 0, 0, 5]]]), [3], freq=[np.pi / 6])          # a quarter turn of channels 0 and 1
    assert np.allclose(x, [[[0, 1, 0, 5]]])
    assert mdi.rope_freq(8, 16.0, "cpu").tolist() == [1.0, 0.5, 0.25, 0.125]


def test_a_preparation_for_heads_of_another_size():
    """Gains and biases are as long as a head of the cache that the preparation was made by: the call cannot know."""
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    small, large = (mdi.KvCache(z(3, 2, 2, 16, h), z(2, 4, dtype=torch.int32)) for h in (64, 128))
    for ours, theirs, h in ((large, small, 128), (small, large, 64)):
        g, rows = z(theirs.h, dtype=torch.float32), ours.rows(z(2, dtype=torch.int32), z(3, dtype=torch.int32), n_rows=4)
        x, q = z(4, 2, h), z(4, 6, h)
        for gains in (dict(q_gain=g), dict(k_gain=g, k_bias=g), dict(q_gain=g, k_gain=g, norm="layer")):
            with pytest.raises(ValueError, match=f"heads of {theirs.h}"):
                ours.append(rows, x, x, q, theirs.prep(**gains))


def test_counts_beyond_32_bits_are_not_cut():
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    cache = mdi.KvCache(z(3, 2, 2, 16, 64), z(2, 1000, dtype=torch.int32))
    rows = cache.rows(z(2, dtype=torch.int32), z(3, dtype=torch.int32), n_rows=4)
    for heads, kw in ((4, dict(window=1 << 32)), (4, dict(window=-1)), (4, dict(window=5, sinks=(1 << 32) + 4)), (4, dict(sinks=-1)), ((1 << 32) + 4, {}), (-4, {})):
        with pytest.raises(ValueError, match="32 bits"):
            cache.workspace(rows, heads, **kw)
    many = z(1, 1, 64).expand(4, (1 << 32) + 4, 64)                            # one head in the place of all
    x = z(4, 2, 64)
    with pytest.raises(ValueError, match="32 bits"):
        cache.append(rows, x, x, many)
