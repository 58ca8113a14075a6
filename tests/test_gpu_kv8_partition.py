"""Partitions whose caches are kept in 8 bits, against the oracle reading its keys and values through the same formula."""
import numpy as np
import pytest
import torch

from gpu_util import dev_acts, dev_ids, host, rel_l2_rows, scale_matrices, tol
from kv8_cases import quantise
from oracle import mdi_oracle as O
from paper_2505_18164_amd import mdi, synth as S
from paper_2505_18164_amd.pipeline import RecurrentPipeline

pytestmark = pytest.mark.gpu

SHAPES = {
    "gqa_h64": dict(n_layer=3, d_model=256, n_head=8, n_kv_head=2, head_dim=64, d_ff=320, vocab=97, max_ctx=400, page=16),
    "mha_h128": dict(n_layer=2, d_model=256, n_head=2, n_kv_head=2, head_dim=128, d_ff=512, vocab=97, max_ctx=700, page=40),
    "gpt2_like": dict(n_layer=2, d_model=128, n_head=2, n_kv_head=2, head_dim=64, d_ff=256, vocab=61, max_ctx=200, page=7, norm_kind=S.NORM_LAYERNORM,
                      mlp_kind=S.MLP_GELU_TANH, pos_kind=S.POS_LEARNED, has_bias=1, tie_embed=1),
    "groups_of_3_h16": dict(n_layer=2, d_model=96, n_head=6, n_kv_head=2, head_dim=16, d_ff=128, vocab=61, max_ctx=150, page=64),
}


class Pair:
    """The oracle twice: f(k), whose attention reads the keys and values themselves, and f(q(k)), whose attention reads
    what an 8-bit cache of their bf16 values holds.  A call returns both results.

    The bar.  The partition computes f(q(k')) with keys and values k' that differ from k by the roundings of a bf16 chain.
    |f(q(k')) - f(q(k))|  <=  |f(q(k')) - f(k')|  +  |f(k') - f(k)|  +  |f(k) - f(q(k))|.  The term in the middle is a bf16
    partition's error with an ordinary cache, which tol(cfg) bounds.  The last is the effect of the quantiser, d, and the
    first is the same effect at k': k' moves each value by about as much as a code's step against itself, which gives
    other roundings of the same size, so it is d again.  The bar is tol(cfg) + 2 d, d taken in the worst row."""

    def __init__(self, *a, **kw):
        self.parts = [O.Partition(*a, **kw) for _ in range(2)]

    def __getattr__(self, name):
        def call(*a):
            plain, out = O.causal_attention, []
            for quantised, part in enumerate(self.parts):
                try:
                    if quantised:
                        O.causal_attention = lambda q, k, v, p0: plain(q, through(k), through(v), p0)
                    out.append(getattr(part, name)(*a))
                finally:
                    O.causal_attention = plain
            return out
        return call


def through(x):
    code, scale = quantise(S.round_to_bf16(x.astype(np.float32)))
    return code.astype(np.float64) * scale.astype(np.float64)[..., None]


def check(got, want, cfg, what):
    f, fq = (np.atleast_2d(x) for x in want)
    got = np.atleast_2d(host(got) if isinstance(got, torch.Tensor) else got).reshape(fq.shape)
    bar = tol(cfg) + 2 * rel_l2_rows(f, fq).max()
    assert bar < 0.15, (what, bar)                                # a wrong row, page or scale is off by more
    assert rel_l2_rows(got, fq).max() < bar, (what, rel_l2_rows(got, fq).argmax(), rel_l2_rows(got, fq).max(), bar)


def build(name, embed=True, head=False, lo=0, hi=None, **kw):
    f = dict(SHAPES[name])
    page = f.pop("page")
    cfg = S.tiny(dtype=S.DT_BF16, **f)
    hi = cfg["n_layer"] if hi is None else hi
    w = scale_matrices(S.make_weights(cfg, 31, exercise=True), 4.0)
    o = Pair(cfg, w, lo, hi, has_embed=embed, has_head=head)
    kw.setdefault("max_seqs", 6)
    return cfg, w, o, mdi.Partition(cfg, w, lo, hi, has_embed=embed, has_head=head, kv_page_tokens=page, kv8=True, **kw)


@pytest.mark.parametrize("name", list(SHAPES))
def test_visits_of_a_sample(name):
    cfg, w, o, g = build(name)
    ids = S.make_prompts(cfg, 5, 1, 100)[0]
    check(g.prefill(0, dev_ids(ids[:61])), o.prefill(0, ids[:61]), cfg, "first visit")
    check(g.prefill_chunk(0, dev_ids(ids[61:99])), o.prefill_chunk(0, ids[61:99]), cfg, "its next piece")
    for i in range(20):
        check(g.decode_step(0, dev_ids([ids[i]])), o.decode_step(0, ids[i]), cfg, ("later visit", i))
    assert g.seq_len(0) == 119
    g.seq_reset(0)
    o.reset(0)
    check(g.prefill(0, dev_ids(ids[:1])), o.prefill(0, ids[:1]), cfg, "a prompt of one token")
    check(g.decode_step(0, dev_ids([3])), o.decode_step(0, 3), cfg, "and the next")
    g.sync()


@pytest.mark.parametrize("name", list(SHAPES))
def test_samples_together(name):
    cfg, w, o, g = build(name, max_prefill=90)
    prompts = S.make_prompts(cfg, 6, 6, 60)
    lens = [60, 1, 17, 33, 48, 2]                                 # two passes of at most 90 rows, and a third
    out = g.prefill_batch(list(range(6)), lens, dev_ids(np.concatenate([p[:n] for p, n in zip(prompts, lens)])))
    for s, rows in enumerate(host(out)[a:a + n] for a, n in zip(np.cumsum([0] + lens), lens)):
        check(rows, o.prefill(s, prompts[s][:lens[s]]), cfg, ("first visits together", s))
    for i in range(3):                                            # later visits, in any order
        order = [3, 0, 5, 1][: 4 - i]
        outs = g.decode_batch(order, [dev_ids([7 + s]) for s in order])
        for s, x in zip(order, outs):
            check(x, o.decode_step(s, 7 + s), cfg, ("later visits together", i, s))
    # a piece of a prompt, a single token and a fresh sample side by side
    g.seq_reset(2)
    o.reset(2)
    lens = {4: 20, 0: 1, 2: 9}
    out = host(g.prefill_batch(list(lens), list(lens.values()), dev_ids(np.concatenate([prompts[s][-n:] for s, n in lens.items()]))))
    at = 0
    for s, n in lens.items():
        check(out[at:at + n], o.prefill_chunk(s, prompts[s][-n:]), cfg, ("mixed", s))
        at += n
    out = g.decode_steps([5, 2], [dev_ids([1]), dev_ids([2])])    # one pass each
    for s, t, x in ((5, 1, out[0]), (2, 2, out[1])):
        check(x, o.decode_step(s, t), cfg, ("one after the other", s))
    g.sync()


def test_hidden_states_between_nodes_and_more_samples_than_a_pass_takes():
    cfg, w, o, g = build("gqa_h64", embed=False, lo=1, hi=3, max_seqs=70)
    x = S.make_activations(cfg, 9, 0, 140)
    lens = [2] * 70
    out = host(g.prefill_batch(list(range(70)), lens, dev_acts(x, cfg)))
    y = S.make_activations(cfg, 9, 1, 70)
    outs = g.decode_batch(list(range(70)), [dev_acts(v, cfg) for v in y])
    for s in (0, 1, 33, 63, 64, 69):
        check(out[2 * s:2 * s + 2], o.prefill(s, x[2 * s:2 * s + 2]), cfg, ("first", s))
        check(outs[s], o.decode_step(s, y[s]), cfg, ("later", s))
    assert g.info(0) == 1 and g.info(4) == 64
    g.sync()


def test_long_contexts():
    """Contexts that are divided among workgroups, alone and beside short ones."""
    cfg, w, o, g = build("mha_h128", embed=False, max_seqs=3)
    x = S.make_activations(cfg, 10, 0, 640)
    check(g.prefill(1, dev_acts(x, cfg)), o.prefill(1, x), cfg, "long prompt")
    check(g.prefill(0, dev_acts(x[:3], cfg)), o.prefill(0, x[:3]), cfg, "short prompt")
    y = S.make_activations(cfg, 11, 0, 4)
    check(g.prefill_chunk(1, dev_acts(y[:3], cfg)), o.prefill_chunk(1, y[:3]), cfg, "a few rows behind many")
    outs = g.decode_batch([0, 1], [dev_acts(y[3], cfg)] * 2)
    for s in (0, 1):
        check(outs[s], o.decode_step(s, y[3]), cfg, ("token", s))
    g.sync()


def test_refusals_take_nobody():
    cfg, w, o, g = build("gqa_h64", max_prefill=50, kv_pages=8)   # 128 positions in all
    ids = dev_ids(S.make_prompts(cfg, 5, 1, 400)[0])
    g.prefill_batch([0, 1], [40, 33], ids[:73])                   # six pages

    def refused(status, call, *a):
        with pytest.raises(mdi.MdiError) as e:
            call(*a)
        assert e.value.status == status and [g.seq_len(s) for s in range(3)] == [40, 33, 0]

    refused(mdi.MDI_ERR_STATE, g.prefill, 0, ids[:4])
    refused(mdi.MDI_ERR_ARG, g.prefill_batch, [2, 1, 2], [1, 1, 1], ids[:3])
    refused(mdi.MDI_ERR_ARG, g.prefill_batch, [2, 9], [1, 1], ids[:2])
    refused(mdi.MDI_ERR_ARG, g.prefill_batch, [2, 0], [1, 0], ids[:1])
    refused(mdi.MDI_ERR_ARG, g.prefill_batch, [2], [51], ids[:51])
    refused(mdi.MDI_ERR_NOMEM, g.prefill_batch, [0, 2], [9, 30], ids[:39])
    refused(mdi.MDI_ERR_CTX, g.prefill_batch, [2, 0], [3, 390], ids[:393])
    refused(mdi.MDI_ERR_STATE, g.decode_batch, [0, 2], [ids[:1], ids[:1]])
    refused(mdi.MDI_ERR_STATE, g.decode_step, 2, ids[:1])
    refused(mdi.MDI_ERR_ARG, g.decode_batch, [0, 0], [ids[:1], ids[:1]])
    g.prefill_batch([0, 2], [8, 32], ids[:40])                    # what is left: two pages
    with pytest.raises(mdi.MdiError) as e:
        g.decode_step(0, ids[:1])
    assert e.value.status == mdi.MDI_ERR_NOMEM
    g.sync()


def test_a_token_id_out_of_range_is_reported():
    cfg, w, o, g = build("gqa_h64")
    g.prefill_batch([0, 1], [2, 2], dev_ids([1, 2, cfg["vocab"], 3]))
    with pytest.raises(mdi.MdiError) as e:
        g.sync()
    assert e.value.status == mdi.MDI_ERR_ARG


@pytest.mark.parametrize("dtype", [S.DT_F32, S.DT_BF16], ids=["f32", "bf16"])
def test_first_visits_together_without_an_8_bit_cache_are_the_same_as_alone(dtype):
    cfg = S.tiny(n_layer=2, d_model=64, n_head=4, n_kv_head=2, head_dim=16, d_ff=96, vocab=97, dtype=dtype)
    w = S.make_weights(cfg, 1, exercise=True)
    a, b = (mdi.Partition(cfg, w, 0, 2, has_embed=True, max_seqs=3, kv_page_tokens=8) for _ in range(2))
    ids = S.make_prompts(cfg, 5, 1, 40)[0]
    lens = [9, 1, 30]
    got = a.prefill_batch([2, 0, 1], lens, dev_ids(ids))
    at = 0
    for s, n in zip([2, 0, 1], lens):
        assert torch.equal(got[at:at + n], b.prefill(s, dev_ids(ids[at:at + n])))
        at += n
    assert torch.equal(a.decode_step(1, dev_ids([4])), b.decode_step(1, dev_ids([4])))


def test_a_ring_of_nodes_generates():
    """The driver: one message at a time, and all that wait together with first visits packed."""
    cfg = S.tiny(n_layer=3, d_model=256, n_head=8, n_kv_head=2, head_dim=64, d_ff=320, vocab=97, max_ctx=64, dtype=S.DT_BF16)
    w = scale_matrices(S.make_weights(cfg, 31, exercise=True), 4.0)
    prompts = [S.make_prompts(cfg, 7, 3, 20)[s][:n] for s, n in enumerate((20, 3, 11))]
    got = {}
    for drain in (False, True, "shared"):
        streams = [torch.cuda.Stream() for _ in range(3)]
        parts = [mdi.Partition(cfg, w, i, i + 1, has_embed=i == 0, has_head=i == 2, max_seqs=3, kv_page_tokens=16, stream=streams[i], kv8=True) for i in range(3)]
        toks, logits, _ = RecurrentPipeline(parts).generate([dev_ids(p) for p in prompts], 4, keep_logits=True, drain=drain)
        torch.cuda.synchronize()
        for p in parts:
            p.sync()
        got[drain] = host(logits), toks.cpu().numpy()
    o = Pair(cfg, w, 0, 3, has_embed=True, has_head=True)
    for s, p in enumerate(prompts):
        x = o.prefill(s, p)
        want = [part.logits(y[-1]) for part, y in zip(o.parts, x)]
        for drain, (logits, toks) in got.items():
            check(logits[s, 0], want, cfg, (drain, s))
            assert (toks[s] == logits[s].argmax(-1)).all()        # the tokens are those of the logits it returns


def test_more_rows_than_two_bytes_count():
    """A prompt of 70001 rows in one pass, and in pieces of 8000: what a row's keys and values are does not depend on it."""
    cfg = S.tiny(n_layer=1, d_model=64, n_head=1, n_kv_head=1, head_dim=64, d_ff=64, vocab=61, max_ctx=70001, dtype=S.DT_BF16)
    w = S.make_weights(cfg, 31, exercise=True)
    x = dev_acts(S.make_activations(cfg, 9, 0, 70001), cfg)
    one, pieces = (mdi.Partition(cfg, w, 0, 1, max_seqs=1, kv_page_tokens=64, max_prefill=most, kv8=True) for most in (70001, 8000))
    a = one.prefill(0, x)
    b = torch.cat([pieces.prefill_chunk(0, x[at:at + 8000]) for at in range(0, 70001, 8000)])
    one.sync()
    pieces.sync()
    assert rel_l2_rows(host(a), host(b)).max() < 2 * tol(cfg)         # each is that close to the exact result


def test_inputs_and_outputs_that_lie_anywhere():
    cfg, w, o, g = build("gqa_h64", embed=False)
    x = dev_acts(S.make_activations(cfg, 9, 0, 4), cfg)
    d = cfg["d_model"]
    want = []
    for shift in (0, 1, 4):                                       # elements: 16 bytes, 2, 8
        for s in range(4):
            g.seq_reset(s)
            g.prefill(s, x[:3])
        buf = torch.full((4 * (d + 8) + 8,), -7, dtype=torch.bfloat16, device="cuda:0")
        ins = [buf[s * (d + 8) + shift:][:d] for s in range(4)]
        for s in range(4):
            ins[s].copy_(x[s])
        res = torch.full_like(buf, -7)
        outs = [res[s * (d + 8) + shift:][:d] for s in range(4)]
        g.decode_batch([0, 1, 2, 3], ins, outs)
        g.sync()
        want.append(torch.stack(outs).clone())
        for t in outs:
            t.fill_(-7)
        assert (res == -7).all()                                  # nothing beside them was written
    assert torch.equal(want[0], want[1]) and torch.equal(want[0], want[2])


def test_tables_of_more_entries_than_31_bits_count():
    """2050 samples of up to 2^24 positions in pages of 16: sample 2048's entries start at 2^31."""
    cfg = S.tiny(n_layer=1, d_model=32, n_head=2, n_kv_head=1, head_dim=16, d_ff=64, vocab=61, max_ctx=1 << 24, dtype=S.DT_BF16)
    w = scale_matrices(S.make_weights(cfg, 31, exercise=True), 4.0)
    g = mdi.Partition(cfg, w, 0, 1, max_seqs=2050, kv_page_tokens=16, kv_pages=64, max_prefill=64, kv8=True)
    x = dev_acts(S.make_activations(cfg, 9, 0, 50), cfg)
    for first in (1, 16, 40):                                     # positions of the first visit: a page, and two or three at once
        got = {}
        for s in (0, 2047, 2048, 2049):                           # (others' pages hold other rows)
            g.prefill_chunk(s, x[s % 7:s % 7 + 9])
            g.seq_reset(s)
        for s in (0, 2047, 2048, 2049):
            y = [g.prefill(s, x[:first])] + [g.decode_step(s, x[first + i]).unsqueeze(0) for i in range(8)]
            got[s] = torch.cat(y)
        z = g.decode_batch([2048, 0, 2049], [x[30]] * 3)
        g.sync()
        for s in (2047, 2048, 2049):
            assert torch.equal(got[s], got[0]), (first, s)
        assert torch.equal(z[0], z[1]) and torch.equal(z[0], z[2])
        for s in (0, 2047, 2048, 2049):
            g.seq_reset(s)
