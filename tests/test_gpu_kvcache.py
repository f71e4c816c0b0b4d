"""The paged score cache on the GPU against the oracle, bit for bit: codes, scales, scores, and what is read back.
Every array of the cache is compared whole, so that a row written beside its place shows."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import serving as V
from paper_2604_23996_amd import smoes as S
from paper_2604_23996_amd import workloads as W
from tests.gpu_util import DEV, say, t

pytestmark = pytest.mark.gpu


def make(rng, lens, page, Hkv, dh, kind, extra=2, max_pages=None, scores=True):
    """(oracle's cache, framework's cache, block table): stale contents, pages in random order, -1 behind the last."""
    need = [-(-max(int(n), 0) // page) for n in lens]
    n_pages = sum(need) + extra
    max_pages = max_pages or max(1, max(need))
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(lens), max_pages), -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    c = dict(kind=kind, m=rng.uniform(0, 1, (n_pages, 2, page)).astype(np.float32) if scores else None)
    for n in ("k", "v"):
        if kind == "bf16":
            c[n] = V.bf16_round(rng.standard_normal((n_pages, Hkv, page, dh)))
        else:
            c[n] = rng.integers(0, 256, (n_pages, Hkv, page, dh)).astype(np.uint8)
            c[n][(c[n] & 0x7f) == 0x7f] = 0x11
            c[n + "_scale"] = rng.integers(118, 124, (n_pages, Hkv, page)).astype(np.uint8)
    return c, to_device(c), table


def to_device(c):
    n_pages, Hkv, page, dh = c["k"].shape
    return S.KVCache(n_pages, page, Hkv, dh, kind=c["kind"], device=DEV, scores=c["m"] is not None,
                     **{n: t(c[n]) for n in ("k", "v", "k_scale", "v_scale", "m") if c.get(n) is not None})


def same(c, cache):
    torch.cuda.synchronize()
    for n in ("k", "v", "k_scale", "v_scale", "m"):
        if c.get(n) is not None:
            x = getattr(cache, n)
            x = x.view(torch.int16).cpu().numpy().view(np.uint16) if x.dtype == torch.bfloat16 else x.cpu().numpy()
            assert np.array_equal(x, c[n]), n


def rows(rng, T, Hkv, dh, dtype):
    x = rng.standard_normal((T, Hkv, dh)) * 2.0 ** rng.integers(-6, 7, (T, Hkv, 1))
    return V.bf16_round(x) if dtype == "bf16" else x.astype(np.float32)


def read_check(c, cache, table, lens, off, T, dtype):
    n_pages, Hkv, page, dh = c["k"].shape
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, v = (torch.full((T, Hkv, dh), 7.0, dtype=td, device=DEV) for _ in range(2))
    m = torch.full((T, 2), 7.0, device=DEV)
    S.kv_read(cache, t(table), t(lens), sample_offsets=None if off is None else t(off), k=k, v=v, m=m)
    torch.cuda.synchronize()
    rk, rv, rm = np.full((T, Hkv, dh), 7.0), np.full((T, Hkv, dh), 7.0), np.full((T, 2), 7.0)
    V.kv_read(c, table, lens, off, T, rk, rv, rm)
    assert np.array_equal(k.double().cpu().numpy(), rk, equal_nan=True)
    assert np.array_equal(v.double().cpu().numpy(), rv, equal_nan=True)
    assert np.array_equal(m.double().cpu().numpy(), rm)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("page,Hkv,dh", [(16, 1, 64), (32, 3, 128), (64, 8, 64), (4096, 2, 128)])
def test_ragged_append_and_read(kind, dtype, page, Hkv, dh):
    # a first chunk, then a second behind it (empty sequences among them, pages that end inside a chunk, rows of padding)
    say("kv append", kind, dtype, page, Hkv, dh)
    rng = np.random.default_rng(page + Hkv)
    n1, n2 = np.array([5, 0, 40, 1, 17]), np.array([30, 0, 1, 0, 16])
    c, cache, table = make(rng, n1 + n2, page, Hkv, dh, kind)
    for new, total in ((n1, n1), (n2, n1 + n2)):
        off = np.concatenate([[0], new.cumsum()]).astype(np.int32)
        T = int(off[-1]) + 6
        k, v = rows(rng, T, Hkv, dh, dtype), rows(rng, T, Hkv, dh, dtype)
        m = rng.uniform(0, 1, (T, 2)).astype(np.float32)
        lens = total.astype(np.int32)
        S.kv_write(cache, t(table), t(lens), t(k), t(v), t(m), sample_offsets=t(off))
        V.kv_write(c, table, lens, off, k, v, m)
        same(c, cache)
        read_check(c, cache, table, lens, off, T, dtype)
    off = np.concatenate([[0], (n1 + n2).cumsum()]).astype(np.int32)  # the whole context
    read_check(c, cache, table, lens, off, int(off[-1]), "bf16")


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("n_seq", [1, 70, 257])
def test_one_token_each(kind, n_seq):
    say("kv step", kind, n_seq)
    rng = np.random.default_rng(n_seq)
    lens = rng.integers(0, 50, n_seq).astype(np.int32)
    lens[0] = 17
    c, cache, table = make(rng, lens, 16, 2, 128, kind)
    k, v = rows(rng, n_seq, 2, 128, "bf16"), rows(rng, n_seq, 2, 128, "bf16")
    m = rng.uniform(0, 1, (n_seq, 2)).astype(np.float32)
    S.kv_write(cache, t(table), t(lens), t(k), t(v), t(m))
    V.kv_write(c, table, lens, None, k, v, m)
    same(c, cache)
    read_check(c, cache, table, lens, None, n_seq, "bf16")


@pytest.mark.parametrize("kind,dtype", [("bf16", "bf16"), ("e4m3", "f32")])
@pytest.mark.parametrize("n_seq,longest,Hkv,dh", [(1022, 4, 5, 64), (1023, 3, 1, 128), (1024, 9, 3, 64), (1500, 45, 1, 64),
                                                  (37, 130, 8, 128), (3, 1500, 2, 64)])
def test_many_tokens_and_sequences(kind, dtype, n_seq, longest, Hkv, dh):
    # several tokens of different sequences per workgroup (up to 32), offsets that fit its memory and ones that do not
    say("kv many", kind, dtype, n_seq, longest)
    rng = np.random.default_rng(n_seq)
    new = rng.integers(0, longest, n_seq)
    new[n_seq // 2] = 0
    new[n_seq // 3] = longest
    lens = (new + rng.integers(0, 20, n_seq)).astype(np.int32)
    c, cache, table = make(rng, lens, 16, Hkv, dh, kind)
    off = np.concatenate([[0], new.cumsum()]).astype(np.int32)
    T = int(off[-1]) + 3
    k, v = rows(rng, T, Hkv, dh, dtype), rows(rng, T, Hkv, dh, dtype)
    m = rng.uniform(0, 1, (T, 2)).astype(np.float32)
    S.kv_write(cache, t(table), t(lens), t(k), t(v), t(m), sample_offsets=t(off))
    V.kv_write(c, table, lens, off, k, v, m)
    same(c, cache)
    read_check(c, cache, table, lens, off, T, dtype)


def test_places_that_are_not_held():
    # unheld pages (-1 and past the pool), lengths past the table, negative lengths, fewer held than new tokens
    say("kv places")
    rng = np.random.default_rng(5)
    for kind in ("bf16", "e4m3"):
        c, cache, table = make(rng, np.array([40, 20, 33, 16, 10]), 16, 2, 64, kind)
        table[0, 1] = -1
        table[1, 0] = c["k"].shape[0]
        table[2, 2] = 2 ** 31 - 1
        lens = np.array([40, 20, 60, -3, 4], np.int32)
        off = np.array([0, 40, 50, 80, 83, 93], np.int32)  # ten new tokens of the last sequence, four of them held
        k, v = rows(rng, 95, 2, 64, "bf16"), rows(rng, 95, 2, 64, "bf16")
        m = rng.uniform(0, 1, (95, 2)).astype(np.float32)
        S.kv_write(cache, t(table), t(lens), t(k), t(v), t(m), sample_offsets=t(off))
        V.kv_write(c, table, lens, off, k, v, m)
        same(c, cache)
        read_check(c, cache, table, lens, off, 95, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_rows_at_the_edges_of_the_types(kind, dtype):
    say("kv edges", kind, dtype)
    rng = np.random.default_rng(6)
    dh, T = 64, 14
    x = rng.standard_normal((T, 1, dh)).astype(np.float32)
    x[0] = 0.0
    x[1] = -0.0
    x[2, 0, 3], x[2, 0, 4] = np.inf, -np.inf       # infinities and NaN do not set the scale
    x[3, 0, 5] = np.nan
    x[4] = np.nan
    x[5] *= 2.0 ** -130                            # below the smallest scale: denormals
    x[6] *= 2.0 ** 120
    x[7] = np.where(rng.random(dh) < 0.5, 1.75, -1.75)   # exactly 448 * 2^-8
    x[8, 0, 0] = np.float32(3.5) * (1 + 2.0 ** -7) if dtype == "bf16" else np.nextafter(np.float32(3.5), np.float32(4))
    x[8, 0, 1:] *= 0.1                             # a step beyond 448 * 2^-7
    x[9, 0, 1:] = 0.0
    x[10] = np.finfo(np.float32).max if dtype == "f32" else 3.3895e38
    x[11] = 2.0 ** -126
    x[12] = 448.0 * 2.0 ** -117                    # the smallest scale's largest value
    x[13, 0, 0], x[13, 0, 1:] = 448.0, np.resize([17.0, 19.0, -21.0, 2.0 ** -10, 3 * 2.0 ** -10, 1e-9], dh - 1)  # ties
    k = V.bf16_round(x) if dtype == "bf16" else x
    lens, table = np.array([T], np.int32), np.array([[1]], np.int32)
    c, cache, _ = make(rng, lens, 16, 1, dh, kind)
    off, m = np.array([0, T], np.int32), rng.uniform(0, 1, (T, 2)).astype(np.float32)
    S.kv_write(cache, t(table), t(lens), t(k), t(k), t(m), sample_offsets=t(off))
    V.kv_write(c, table, lens, off, k, k, m)
    same(c, cache)
    read_check(c, cache, table, lens, off, T, "f32")
    read_check(c, cache, table, lens, off, T, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_views_at_any_element(kind, dtype):
    # slices of a fused projection that start and step off 16-byte boundaries
    say("kv views", kind, dtype)
    rng = np.random.default_rng(7)
    T, Hkv, dh = 33, 2, 64
    lens, off = np.array([T], np.int32), np.array([0, T], np.int32)
    for shift, width in ((1, 2 * Hkv * dh + 3), (8, 2 * Hkv * dh + 8), (3, 2 * Hkv * dh)):
        c, cache, table = make(rng, lens, 16, Hkv, dh, kind)
        x = rows(rng, T, 2 * Hkv, dh, dtype)
        buf = torch.zeros(T * width + 16, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device=DEV)
        view = buf[shift:shift + T * width].view(T, width)[:, :2 * Hkv * dh].unflatten(1, (2 * Hkv, dh))
        view.copy_(t(x))
        m = rng.uniform(0, 1, (T, 2)).astype(np.float32)
        S.kv_write(cache, t(table), t(lens), view[:, :Hkv], view[:, Hkv:], t(m), sample_offsets=t(off))
        V.kv_write(c, table, lens, off, x[:, :Hkv], x[:, Hkv:], m)
        same(c, cache)


def test_without_scores_and_single_outputs():
    say("kv no scores")
    rng = np.random.default_rng(8)
    lens, off = np.array([20], np.int32), np.array([0, 20], np.int32)
    c, cache, table = make(rng, lens, 16, 2, 64, "e4m3", scores=False)
    k, v = rows(rng, 20, 2, 64, "bf16"), rows(rng, 20, 2, 64, "bf16")
    S.kv_write(cache, t(table), t(lens), t(k), t(v), sample_offsets=t(off))
    V.kv_write(c, table, lens, off, k, v, None)
    same(c, cache)
    k2, v2, m2 = S.kv_read(cache, t(table), t(lens), sample_offsets=t(off), T=20)
    torch.cuda.synchronize()
    assert m2 is None
    # the keys alone, the values alone
    tb, ln, of = t(table), t(lens), t(off)
    for one in ("k", "v"):
        out = torch.zeros(20, 2, 64, dtype=torch.bfloat16, device=DEV)
        S._check(S.lib().smoes_kv_read(cache.desc, tb.data_ptr(), table.shape[1], ln.data_ptr(), 1,
                                       of.data_ptr(), 20, out.data_ptr() if one == "k" else None,
                                       out.data_ptr() if one == "v" else None, S.SMOES_BF16, None, S._stream()), "read")
        torch.cuda.synchronize()
        assert torch.equal(out, k2 if one == "k" else v2)


def test_far_pages():
    # a pool of which a head's rows lie beyond 2^32 bytes: the offsets are 64 bits
    say("kv far pages")
    n_pages, page, Hkv, dh = 70000, 256, 1, 128
    cache = S.KVCache(n_pages, page, Hkv, dh, device=DEV)
    assert cache.k.numel() * 2 > 2 ** 32
    rng = np.random.default_rng(9)
    table = np.array([[n_pages - 1, 3]], np.int32)
    lens, off = np.array([300], np.int32), np.array([0, 300], np.int32)
    k, v = rows(rng, 300, Hkv, dh, "bf16"), rows(rng, 300, Hkv, dh, "bf16")
    m = rng.uniform(0, 1, (300, 2)).astype(np.float32)
    S.kv_write(cache, t(table), t(lens), t(k), t(v), t(m), sample_offsets=t(off))
    k2, v2, m2 = S.kv_read(cache, t(table), t(lens), sample_offsets=t(off), T=300)
    torch.cuda.synchronize()
    assert torch.equal(k2, t(k)) and torch.equal(v2, t(v)) and torch.equal(m2, t(m))
    assert torch.equal(cache.k[n_pages - 1, 0], t(k)[:256, 0]) and torch.equal(cache.v[3, 0, :44], t(v)[256:, 0])
    assert not cache.k[4:n_pages - 1].any() and not cache.v[:3].any()
