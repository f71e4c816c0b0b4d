"""Attention of one new token over the paged cache on the GPU, against the float64 oracle.

Tolerance, with u = 2^-24, n keys and S = max_j scale sum_d |q_d k_jd|: a logit is a float32 sum of head_dim
products of bf16 values, scaled: within (head_dim + 3) u S; its difference from the maximum, at most 2 S, is rounded (2 u S)
and its exponential good to 4 u more: p_j is off by d = (head_dim + 5) u S + 4 u of itself. Numerator and denominator
are float32 sums of n terms, joined over at most 64 splits: n + 64 roundings each. So o is within
2 (d + (n + 64) u) sum_j p_j |v_j|, plus its rounding to bf16 (2^-8 of the value), and m within the same with
scores for |v| (at most 1). (4 u covers exp2's 1 unit, its argument's product and the conversion to base 2.)"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle as O
from oracle import serving as V
from paper_2604_23996_amd import smoes as S
from paper_2604_23996_amd import workloads as W
from tests.gpu_util import DEV, host, say, t
from tests.test_gpu_kvcache import make, to_device

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def poison(c, table, lens):
    """NaN wherever no position below a length is held: a read of it would show."""
    n_pages, Hkv, page, dh = c["k"].shape
    held = np.zeros((n_pages, page), bool)
    for b in range(len(lens)):
        for j in range(min(max(int(lens[b]), 0), table.shape[1] * page)):
            p = table[b, j // page]
            if 0 <= p < n_pages:
                held[p, j % page] = True
    for n in ("k", "v"):
        x = c[n].transpose(0, 2, 1, 3)
        x[~held] = 0x7fc0 if c["kind"] == "bf16" else 0x7f
        if c["kind"] == "e4m3":
            c[n + "_scale"].transpose(0, 2, 1)[~held] = 255
    if c["m"] is not None:
        c["m"].transpose(0, 2, 1)[~held] = np.nan


def check(c, table, lens, q, o, mh, scale=None):
    ref_o, ref_m, size, av, keys = V.attention_decode(c, table, lens, q, scale)
    dh = q.shape[2]
    d = (dh + 5) * U * size + 4 * U
    rel = 2 * (d + (keys[:, None] + 64) * U)
    tol = rel[..., None] * av
    tol = tol + 2.0 ** -8 * (np.abs(ref_o) + tol)
    err = np.abs(host(o) - ref_o)
    assert np.all(err <= tol), (np.max(err - tol), np.argwhere(err > tol)[:4])
    assert not host(o)[keys == 0].any()
    if mh is not None:
        err = np.abs(host(mh) - ref_m)
        assert np.all(err <= rel[..., None]), np.max(err - rel[..., None])
        assert not host(mh)[keys == 0].any()


def queries(rng, n_seq, H, dh, std=2.0):
    return V.bf16_round(rng.standard_normal((n_seq, H, dh)) * std)


def run(c, table, lens, q, **kw):
    o, mh = S.attention_scores_decode(to_device(c), t(table), t(lens), t(q), **kw)
    torch.cuda.synchronize()
    return o, mh


LENS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 300, 511, 513, 700]


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,Hkv,page", [(4, 4, 16), (8, 2, 32), (6, 1, 256), (20, 1, 16), (40, 2, 64), (17, 1, 128), (33, 1, 16), (70, 1, 32)])
def test_ragged(kind, dh, H, Hkv, page):
    # every length around the tiles, among them 0; stale NaN behind every end; groups over and under 16 heads
    say("decode ragged", kind, dh, H, Hkv, page)
    rng = np.random.default_rng(dh + H + page)
    lens = rng.permutation(LENS).astype(np.int32)
    c, _, table = make(rng, lens, page, Hkv, dh, kind)
    poison(c, table, lens)
    q = queries(rng, len(lens), H, dh)
    check(c, table, lens, q, *run(c, table, lens, q))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 2, 5000])
def test_one_sequence(kind, n):
    say("decode one", kind, n)
    rng = np.random.default_rng(n)
    lens = np.array([n], np.int32)
    c, _, table = make(rng, lens, 64, 2, 128, kind)
    poison(c, table, lens)
    q = queries(rng, 1, 8, 128)
    check(c, table, lens, q, *run(c, table, lens, q))


def test_one_long_among_many_short():
    say("decode long among short")
    rng = np.random.default_rng(11)
    lens = rng.integers(1, 40, 300).astype(np.int32)
    lens[137] = 20011
    lens[[0, 5, 6, 299]] = 0
    c, _, table = make(rng, lens, 16, 1, 64, "bf16")
    q = queries(rng, 300, 4, 64)
    check(c, table, lens, q, *run(c, table, lens, q))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_pages_that_are_not_held(kind):
    # dropped pages in front and in the middle, a sequence without any, lengths past the table and below 0, two
    # sequences that share their first pages
    say("decode pages", kind)
    rng = np.random.default_rng(12)
    lens = np.array([200, 200, 100, 90, 999, -4, 130], np.int32)
    c, _, table = make(rng, np.array([200, 200, 100, 90, 208, 0, 130]), 16, 2, 64, kind)
    table[0, :5] = -1
    table[1, 3], table[1, 7], table[1, 12] = -1, c["k"].shape[0], -(2 ** 31)
    table[2] = -1
    table[6, :6] = table[3, :6]
    table[6, 5] = table[3, 5]
    lens[6] = 96 + 30
    table[6, 6:8] = table[4, 0:2]
    poison(c, table, lens)
    q = queries(rng, 7, 4, 64)
    check(c, table, lens, q, *run(c, table, lens, q))


@pytest.mark.parametrize("scale", [0.0, 0.3, 1e-6, 4.0])
def test_scale(scale):
    # flat and sharp: with 4.0 the running maximum moves often and one key takes nearly all
    say("decode scale", scale)
    rng = np.random.default_rng(13)
    lens = np.array([700, 333], np.int32)
    c, _, table = make(rng, lens, 16, 2, 128, "bf16")
    q = queries(rng, 2, 8, 128)
    check(c, table, lens, q, *run(c, table, lens, q, scale=scale), scale=scale or None)


def test_rising_and_falling_logits():
    # the largest logit first, last, and in the middle, far above the rest
    say("decode order")
    rng = np.random.default_rng(14)
    lens = np.array([600, 600, 600], np.int32)
    c, _, table = make(rng, lens, 16, 1, 64, "bf16")
    q = queries(rng, 3, 2, 64, std=0.01)
    q[:, :, 0] = V.bf16_round(np.full((3, 2), 40.0))
    for b, where in enumerate((np.linspace(30, -30, 600), np.linspace(-30, 30, 600), -np.abs(np.linspace(-30, 30, 600)))):
        for j in range(600):
            c["k"][table[b, j // 16], 0, j % 16, 0] = V.bf16_round(where)[j]
    check(c, table, lens, q, *run(c, table, lens, q))


@pytest.mark.parametrize("H", [16, 40])
def test_infinities_and_nan_in_wide_groups(H):
    # groups over four heads, whose probabilities enter as three bf16 terms: an infinite value stays infinite in its
    # column for every head, a NaN value NaN, and the other columns, sequences and the scores do not see them
    say("decode infinities, wide groups", H)
    rng = np.random.default_rng(23)
    lens = np.array([90, 90, 90], np.int32)
    c, _, table = make(rng, lens, 16, 2, 64, "bf16")
    q = queries(rng, 3, H, 64, std=0.2)
    put = lambda b, j, d, bits: c["v"][table[b, j // 16], 0, j % 16].__setitem__(d, bits)
    for j in (0, 33, 89):  # other tiles, pieces and lanes
        put(0, j, 3, 0x7f80)
        put(0, j, 4, 0xff80)
    put(1, 40, 5, 0x7fc0)
    o, mh = run(c, table, lens, q)
    o, mh, g = host(o), host(mh), H // 2
    assert (o[0, :g, 3] == np.inf).all() and (o[0, :g, 4] == -np.inf).all()
    assert np.isfinite(np.delete(o[0, :g], [3, 4], axis=1)).all() and np.isfinite(o[0, g:]).all()
    assert np.isnan(o[1, :g, 5]).all() and np.isfinite(np.delete(o[1, :g], 5, axis=1)).all()
    assert np.isfinite(o[1, g:]).all() and np.isfinite(o[2]).all() and np.isfinite(mh).all()


def test_infinities_and_nan():
    # a NaN or an infinity in a held row reaches its own sequence and heads, as in the formula, and no other
    say("decode infinities")
    rng = np.random.default_rng(15)
    lens = np.array([90, 90, 90, 90, 90], np.int32)
    c, _, table = make(rng, lens, 16, 2, 64, "bf16")
    q = np.abs(V.bf16_round(rng.uniform(0.5, 1.0, (5, 4, 64))).astype(np.uint16))
    put = lambda n, b, j, bits: c[n][table[b, j // 16], 0, j % 16].__setitem__(3, bits)
    put("k", 0, 40, 0x7fc0)   # NaN key: a NaN logit
    put("v", 1, 40, 0x7fc0)   # NaN value: one column
    put("k", 2, 40, 0xff80)   # -inf key: its probability is 0
    for j in range(90):
        put("k", 3, j, 0xff80)  # every logit -inf: 0 / 0
    put("v", 4, 7, 0x7f80)    # an infinite value
    o, mh = run(c, table, lens, q)
    o, mh = host(o), host(mh)
    assert np.isnan(o[0, :2]).all() and np.isnan(mh[0, :2]).all() and np.isfinite(o[0, 2:]).all()
    assert np.isnan(o[1, :2, 3]).all() and np.isfinite(np.delete(o[1], 3, axis=1)).all() and np.isfinite(mh[1]).all()
    assert np.isfinite(o[2]).all() and np.isfinite(mh[2]).all()
    assert np.isnan(o[3, :2]).all() and np.isnan(mh[3, :2]).all() and np.isfinite(o[3, 2:]).all()
    assert np.isinf(o[4, :2, 3]).all() and np.isfinite(np.delete(o[4], 3, axis=1)).all()
    # the sequence with one key at -inf: as if that key were not there
    sub = V.attention_decode(c, table[2:3], lens[2:3], q[2:3])
    assert np.all(np.abs(o[2] - sub[0][0]) <= 1e-2) and np.all(np.abs(mh[2] - sub[1][0]) <= 1e-4)


@pytest.mark.parametrize("shift,extra", [(0, 64), (1, 0), (3, 5), (8, 8)])
def test_queries_in_a_view_and_no_scores(shift, extra):
    say("decode views", shift, extra)
    rng = np.random.default_rng(16)
    lens = np.array([50, 7, 130], np.int32)
    c, _, table = make(rng, lens, 16, 2, 64, "bf16")
    q = queries(rng, 3, 6, 64)
    width = 6 * 64 + extra
    buf = torch.zeros(3 * width + 16, dtype=torch.bfloat16, device=DEV)
    view = buf[shift:shift + 3 * width].view(3, width)[:, :384].unflatten(1, (6, 64))
    view.copy_(t(q))
    cache = to_device(c)
    o, mh = S.attention_scores_decode(cache, t(table), t(lens), t(q))
    o2, mh2 = S.attention_scores_decode(cache, t(table), t(lens), view)
    bare = S.KVCache(cache.n_pages, 16, 2, 64, device=DEV, scores=False, k=cache.k, v=cache.v)
    o3, mh3 = S.attention_scores_decode(bare, t(table), t(lens), t(q))
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(mh, mh2) and torch.equal(o, o3) and mh3 is None
    assert S.attention_scores_decode(cache, t(table[:0]), t(lens[:0]), view[:0])[0].shape == (0, 6, 64)


def test_far_pages():
    say("decode far pages")
    n_pages, page, Hkv, dh = 70000, 256, 1, 128
    cache = S.KVCache(n_pages, page, Hkv, dh, device=DEV)
    rng = np.random.default_rng(17)
    lens = np.array([300], np.int32)
    c, _, table = make(rng, lens, page, Hkv, dh, "bf16", extra=0)
    far = np.array([[n_pages - 1, 3]], np.int32)
    for n in ("k", "v", "m"):
        for a, b in zip(table[0], far[0]):
            getattr(cache, n)[int(b)] = t(c[n][a])
    q = queries(rng, 1, 3, dh)
    o, mh = S.attention_scores_decode(cache, t(far), t(lens), t(q))
    torch.cuda.synchronize()
    check(c, table, lens, q, o, mh)


def test_reproducible_and_dirty_workspace():
    say("decode reproducible")
    rng = np.random.default_rng(18)
    lens = np.array([3000, 5, 0, 900], np.int32)
    c, _, table = make(rng, lens, 32, 4, 128, "e4m3")
    q = t(queries(rng, 4, 16, 128))
    cache, tb, ln = to_device(c), t(table), t(lens)
    first = None
    for fill in (0, 255, 127):
        ws = torch.full((S.attention_decode_workspace_bytes(cache, 4, 16) + 3,), fill, dtype=torch.uint8, device=DEV)
        o, mh = S.attention_scores_decode(cache, tb, ln, q, workspace=ws[3:] if fill == 127 else ws)
        torch.cuda.synchronize()
        if first is None:
            first = (o, mh)
        assert torch.equal(o, first[0]) and torch.equal(mh, first[1])


def test_two_graphs_share_a_workspace():
    # lengths and tables change between replays; two captured calls on one workspace, replayed in turn with eager work
    say("decode graphs")
    rng = np.random.default_rng(19)
    most = np.array([400, 90, 1500], np.int32)
    calls = []
    for seed in (0, 1):
        c, _, table = make(rng, most, 16, 2, 64, "bf16")
        cache = to_device(c)
        calls.append(dict(c=c, cache=cache, table=table, tb=t(table), ln=t(most.copy()), q=t(queries(rng, 3, 8, 64)),
                          o=torch.empty(3, 8, 64, dtype=torch.bfloat16, device=DEV),
                          m=torch.empty(3, 8, 2, device=DEV)))
    ws = torch.empty(S.attention_decode_workspace_bytes(calls[0]["cache"], 3, 8), dtype=torch.uint8, device=DEV)
    go = lambda a, o, m: S.attention_scores_decode(a["cache"], a["tb"], a["ln"], a["q"], o=o, m_heads=m, workspace=ws)
    graphs = []
    for a in calls:
        go(a, a["o"], a["m"])
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            go(a, a["o"], a["m"])
        graphs.append(g)
    for lens in ([1, 0, 1500], [400, 90, 3], [0, 0, 0], [17, 64, 1025]):
        for a, g in zip(calls, graphs):
            a["ln"].copy_(torch.tensor(lens, dtype=torch.int32))
            want = S.attention_scores_decode(a["cache"], a["tb"], a["ln"], a["q"])
            a["o"].fill_(5.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(a["o"], want[0]) and torch.equal(a["m"], want[1])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_generation_matches_the_whole_sample(kind):
    # prefill (rotary, attention over the samples, cache), then tokens one by one (rotary, cache, decode, score update):
    # the outputs of every generated token are those of the causal attention of the whole samples on what the cache holds
    say("generation", kind)
    rng = np.random.default_rng(20)
    H, Hkv, dh, d, page, steps = 8, 2, 64, 128, 16, 5
    start = np.array([37, 1, 96], np.int32)
    total = start + steps
    plan = S.RotaryPlan(S.RotarySpec(dh, dh, scaling="by_parts", factor=4.0, original_len=64), DEV)
    T = int(total.sum())
    off_all = np.concatenate([[0], total.cumsum()])
    qkv = torch.from_numpy(rng.standard_normal((T, H + 2 * Hkv, dh)).astype(np.float32)).bfloat16().to(DEV)
    x, xa = (torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).bfloat16().to(DEV) for _ in range(2))
    m_in = torch.from_numpy(W.random_soft_scores(rng, T)).to(DEV)
    pos_all = torch.from_numpy(np.concatenate([np.arange(n) for n in total]).astype(np.int32)).to(DEV)
    c, cache, table = make(rng, total, page, Hkv, dh, kind)
    tb = t(table)
    got_o, got_m, rows_of = [], [], []

    def part(idx):
        i = torch.from_numpy(np.asarray(idx)).to(DEV)
        a = qkv[i]
        q, k = S.rotary(plan, a[:, :H], a[:, H:H + Hkv], positions=pos_all[i])
        return i, q, k, a[:, H + Hkv:].contiguous()

    pre = np.concatenate([np.arange(o, o + n) for o, n in zip(off_all, start)])
    off = np.concatenate([[0], start.cumsum()]).astype(np.int32)
    i, q, k, v = part(pre)
    o, mh = S.attention_scores(q, k, v, t(off), m_in[i].contiguous())
    S.kv_write(cache, tb, t(start), k, v, m_in[i].contiguous(), sample_offsets=t(off))
    ln = t(start.copy())
    for s in range(steps):
        ln += 1
        i, q, k, v = part(off_all[:-1] + start + s)
        S.kv_write(cache, tb, ln, k, v, m_in[i].contiguous())
        o, mh = S.attention_scores_decode(cache, tb, ln, q)
        m1 = S.attn_score_update(x[i].contiguous(), xa[i].contiguous(), mh, m_in[i].contiguous())
        got_o.append(host(o)), got_m.append(host(m1)), rows_of.append(off_all[:-1] + start + s)
    kd, vd, md = S.kv_read(cache, tb, ln, sample_offsets=t(off_all.astype(np.int32)), T=T)
    torch.cuda.synchronize()
    assert torch.equal(md, m_in)
    _, q, k, v = part(np.arange(T))
    if kind == "bf16":
        assert torch.equal(kd, k) and torch.equal(vd, v)
    ref_o, ref_a = O.attention_heads(host(q), host(kd), host(vd), off_all, host(m_in))
    ref_m = O.attn_score_update(host(x), host(xa), host(m_in), O.attn_aggregate(ref_a))
    for o, m1, r in zip(got_o, got_m, rows_of):
        # bf16 rounding of the output (2^-8); float32 evaluation far below
        assert np.all(np.abs(o - ref_o[r]) <= 2.0 ** -8 * np.abs(ref_o[r]) + 1e-4)
        assert np.abs(m1 - ref_m[r]).max() <= 1e-5
    # and the same rows through the whole-sample operator, to its tolerance
    whole, _ = S.attention_scores(q, kd, vd, t(off_all.astype(np.int32)), m_in)
    torch.cuda.synchronize()
    for o, r in zip(got_o, rows_of):
        assert np.all(np.abs(o - host(whole)[r]) <= 1e-2 + 2e-2 * np.abs(o))


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_a_captured_step_replayed(kind):
    # one step (rotary, cache, decode, read back) captured with its lengths; every replay, with new rows and eager
    # work between, gives the bits of the eager step on a second cache, across ends of pages and of tiles
    say("captured step", kind)
    rng = np.random.default_rng(21)
    H, Hkv, dh, page, steps = 8, 2, 128, 16, 6
    start = np.array([125, 0, 14, 300], np.int32)
    c, cache, table = make(rng, start + steps, page, Hkv, dh, kind)
    twin = to_device(c)
    tb, n = t(table), len(start)
    plan = S.RotaryPlan(S.RotarySpec(dh, dh), DEV)

    def step(cache, ln, qkv, m_in, ws):
        ln += 1
        q, k = S.rotary(plan, qkv[:, :H], qkv[:, H:H + Hkv], positions=ln - 1)
        S.kv_write(cache, tb, ln, k, qkv[:, H + Hkv:], m_in)
        return S.attention_scores_decode(cache, tb, ln, q, workspace=ws) + S.kv_read(cache, tb, ln)

    ws, ws2 = (torch.empty(S.attention_decode_workspace_bytes(cache, n, H), dtype=torch.uint8, device=DEV) for _ in range(2))
    qkv = torch.zeros((n, H + 2 * Hkv, dh), dtype=torch.bfloat16, device=DEV)
    m_in = torch.zeros((n, 2), device=DEV)
    ln, ln2 = t(start.copy()), t(start.copy())
    step(to_device(c), t(start.copy()), qkv, m_in, ws)  # loads the kernels
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        got = step(cache, ln, qkv, m_in, ws)
    for s in range(steps):
        qkv.copy_(torch.from_numpy(rng.standard_normal(tuple(qkv.shape)).astype(np.float32)))
        m_in.copy_(torch.from_numpy(rng.uniform(0, 1, (n, 2)).astype(np.float32)))
        graph.replay()
        want = step(twin, ln2, qkv, m_in, ws2)
        torch.cuda.synchronize()
        assert torch.equal(ln, ln2) and ln.tolist() == (start + s + 1).tolist()
        for x, y in zip(got, want):
            assert torch.equal(x, y)
    for x, y in zip((cache.k, cache.v, cache.k_scale, cache.m), (twin.k, twin.v, twin.k_scale, twin.m)):
        assert x is None and y is None or torch.equal(x, y)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dh,H,Hkv", [(64, 4, 2), (128, 16, 2), (64, 18, 1)])
def test_more_tiles_than_workgroups(kind, dh, H, Hkv):
    # every workgroup has several tiles, most of more than one (sequence, group)
    say("decode many tiles", kind, dh, H, Hkv)
    rng = np.random.default_rng(21)
    lens = rng.integers(2000, 4100, 26).astype(np.int32)
    lens[[3, 4, 25]] = 0, 1, 128
    c, _, table = make(rng, lens, 32, Hkv, dh, kind)
    poison(c, table, lens)
    q = queries(rng, 26, H, dh)
    check(c, table, lens, q, *run(c, table, lens, q))


@pytest.mark.parametrize("n_seq", [255, 256, 257, 512, 513, 770])
def test_sequences_around_the_blocks_of_the_count(n_seq):
    say("decode sequences", n_seq)
    rng = np.random.default_rng(n_seq)
    lens = rng.integers(0, 200, n_seq).astype(np.int32)
    lens[[0, -1]] = 0, 150
    c, _, table = make(rng, lens, 16, 1, 64, "bf16")
    q = queries(rng, n_seq, 2, 64)
    check(c, table, lens, q, *run(c, table, lens, q))


def test_two_streams_at_once():
    # calls that overlap in time, each with its own workspace, against the same calls one after another
    say("decode streams")
    rng = np.random.default_rng(22)
    calls = []
    for i, lens in enumerate(([3000, 17], [900, 2500])):
        lens = np.array(lens, np.int32)
        c, _, table = make(rng, lens, 16, 2, 128, "bf16")
        calls.append((to_device(c), t(table), t(lens), t(queries(rng, 2, 8, 128))))
    want = [S.attention_scores_decode(*a) for a in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = [[], []]
    for _ in range(5):
        for i, (a, st) in enumerate(zip(calls, streams)):
            with torch.cuda.stream(st):
                got[i].append(S.attention_scores_decode(*a))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for o, m in g:
            assert torch.equal(o, w[0]) and torch.equal(m, w[1])
