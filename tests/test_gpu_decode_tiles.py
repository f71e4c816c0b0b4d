"""The decode with several tiles (128 keys of one sequence and group) a workgroup: tiles that are loaded while others
are worked on, runs that follow each other, runs shared by workgroups, a reference maximum that moves over sums that
are not empty, and whole tiles of which no page is held. The number of workgroups is read off the workspace's size, the
even cut is replayed on the host, and every test asserts what it means to reach.

Tolerance, with u = 2^-24, S = max_j scale sum_d |q_d k_jd|, R = 2 S / ln 2 the range of the exponents: a logit is
within (head_dim + 3) u S. Its weight is a product of exponentials of differences of rising references, whose sum is
at most R: their roundings are 2 u S of the weight together, the logits' own difference 2 u S more. Each factor costs 4 u
(exponential, its argument's product, the product with it): the weight itself, at most R / 8 moves of the running
maximum, one for the wave in its workgroup, W / 32 batches and three more in the join. Sums: a value column of a tile takes at most 3 x 32
additions (three terms of 32 probabilities), a run at most ceil(tiles / W) + 1 tiles, the joins 4 + 4 W / 32 + 16. So
numerator and denominator are off by at most rel / 2 of sum_j p_j |v_j|, and o by rel plus its rounding to bf16 (2^-8 of the value)."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import serving as V
from paper_2604_23996_amd import smoes as S
from tests.gpu_util import DEV, host, say, t
from tests.test_gpu_decode import poison, queries
from tests.test_gpu_kvcache import make, rows, to_device

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TILE = 128


def sets(group):
    """Query heads of a pass over a KV head's rows, and the passes."""
    most = 4 if group <= 4 else 16 if group <= 16 else 32
    return min(group, most), -(-group // most)


def workgroups(cache, n_seq, H):
    """From the size of the workspace: two partial results of head_dim + 4 floats per query head and workgroup, 8 bytes
    for every sequence and 8 more; at most 768 bytes of alignment."""
    per = 8 * sets(H // cache.n_kv_heads)[0] * (cache.head_dim + 4)
    n = (S.attention_decode_workspace_bytes(cache, n_seq, H) - 8 * (1 + n_seq)) // per
    assert n % 256 == 0
    return n


def cut(lens, HR, W):
    """The runs of every workgroup: (sequence, group, first tile, one behind the last, tiles of the sequence)."""
    tiles = [(b, hr, i, -(-int(n) // TILE)) for b, n in enumerate(lens) for hr in range(HR) for i in range(-(-int(n) // TILE))]
    quot, rem = divmod(len(tiles), W)
    out, g = [], 0
    for w in range(W):
        mine, g = tiles[g:g + quot + (w < rem)], g + quot + (w < rem)
        runs = []
        for b, hr, i, nb in mine:
            if runs and runs[-1][:2] == [b, hr]:
                runs[-1][3] = i + 1
            else:
                runs.append([b, hr, i, i + 1, nb])
        out.append(runs)
    return out, len(tiles)


def check(c, table, lens, q, o, mh, W, scale=None):
    ref_o, ref_m, size, av, keys = V.attention_decode(c, table, lens, q, scale)
    H, Hkv, dh = q.shape[1], c["k"].shape[1], q.shape[2]
    tiles = sum(-(-max(int(n), 0) // TILE) for n in lens) * Hkv * sets(H // Hkv)[1]
    factors = 2 * size / math.log(2) / 8 + 5 + W / 32
    adds = 96 * (-(-tiles // W) + 1) + 4 + W / 8 + 16
    rel = 2 * ((dh + 7) * U * size + (4 * factors + adds) * U)
    tol = rel[..., None] * av
    tol = tol + 2.0 ** -8 * (np.abs(ref_o) + tol)
    err = np.abs(host(o) - ref_o)
    assert np.all(err <= tol), (np.max(err - tol), np.argwhere(err > tol)[:4])
    err = np.abs(host(mh) - ref_m)
    assert np.all(err <= rel[..., None]), np.max(err - rel[..., None])
    assert not host(o)[keys == 0].any() and not host(mh)[keys == 0].any()


FORMS = [(64, 8, 4), (128, 8, 2), (64, 32, 4), (128, 16, 2), (64, 36, 2), (128, 20, 1), (64, 40, 1)]


def lengths(rng, cache_of, H, per_seq, least):
    """Long sequences with short and empty ones between, at least `least` tiles a workgroup."""
    Hkv, n_groups = cache_of.n_kv_heads, cache_of.n_kv_heads * sets(H // cache_of.n_kv_heads)[1]
    W = workgroups(cache_of, 1, H)
    lens = []
    while sum(-(-n // TILE) for n in lens) * n_groups < least * W:
        lens += [int(rng.integers(*per_seq)), int(rng.integers(1, 300))]
        if len(lens) % 10 == 0:
            lens += [0, 1, TILE]
    return np.array(lens, np.int32), W, n_groups


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dh,H,Hkv", FORMS)
def test_runs(kind, dh, H, Hkv):
    say("decode tiles", kind, dh, H, Hkv)
    rng = np.random.default_rng(dh + H)
    small = S.KVCache(1, 64, Hkv, dh, kind=kind, device=DEV)
    lens, W, HR = lengths(rng, small, H, (1500, 4200), 3.3)
    runs, tiles = cut(lens, HR, W)
    assert tiles > 3 * W
    assert sum(len(r) > 1 for r in runs) > 10                                # several runs, of other sequences or heads
    assert any(len(r) > 2 for r in runs)
    assert any(x[2] == 0 and x[3] == x[4] > 1 for r in runs for x in r)      # finished by one workgroup
    assert any(x[2] > 0 and x[3] < x[4] for r in runs for x in r)            # the middle of a longer one
    assert any(len(r) > 1 and r[-1][3] < r[-1][4] for r in runs)             # shared, and not its workgroup's first
    c, _, table = make(rng, lens, 64, Hkv, dh, kind)
    b = int(np.argmax(lens))
    table[b, 4:8] = -1   # two whole tiles of the longest sequence
    poison(c, table, lens)
    q = queries(rng, len(lens), H, dh)
    o, mh = S.attention_scores_decode(to_device(c), t(table), t(lens), t(q))
    torch.cuda.synchronize()
    check(c, table, lens, q, o, mh, W)


STEPS = (10.0, 4.0, 8.5, 2.5)  # of the logits from level to level, in powers of two, by head: some move the maximum at
#                                every level, some every second or third (it moves when it is passed by 8)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dh,H,Hkv", FORMS)
def test_the_maximum_moves_over_sums(kind, dh, H, Hkv):
    # dim 0 of a key is its tile's level: rising from tile to tile, falling, in zigzag, drawn for every key
    say("decode maximum", kind, dh, H, Hkv)
    rng = np.random.default_rng(dh + H + 1)
    small = S.KVCache(1, 64, Hkv, dh, kind=kind, device=DEV)
    lens, W, HR = lengths(rng, small, H, (1500, 4200), 3.3)
    level = []
    for b, n in enumerate(lens):
        i = np.arange(n) // TILE
        level.append([i % 16, 15 - i % 16, i % 2 * 8 + i % 5, rng.integers(0, 16, n)][b % 4])
    runs, _ = cut(lens, HR, W)
    moves = {s: 0 for s in STEPS}
    for s in STEPS:
        for b, _, first, last, _ in (x for r in runs for x in r):
            top = -np.inf
            for i in range(first, last):
                here = s * level[b][i * TILE:(i + 1) * TILE].max()
                if here > top + 8:
                    moves[s] += top > -np.inf
                    top = here
    assert all(m > 30 for m in moves.values()), moves
    c, _, table = make(rng, lens, 64, Hkv, dh, kind)
    for b, n in enumerate(lens):
        j = np.arange(n)
        x = rng.standard_normal((n, Hkv, dh)) * 0.1
        x[..., 0] = level[b][:, None]
        at = table[b, j // 64], slice(None), j % 64
        if kind == "bf16":
            c["k"][at] = V.bf16_round(x)
        else:
            c["k"][at] = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
            c["k_scale"][at] = 127
    poison(c, table, lens)
    q = V.widen(queries(rng, len(lens), H, dh, std=0.5))
    q[:, :, 0] = np.resize(STEPS, H) * math.sqrt(dh) * math.log(2)
    q = V.bf16_round(q)
    o, mh = S.attention_scores_decode(to_device(c), t(table), t(lens), t(q))
    torch.cuda.synchronize()
    check(c, table, lens, q, o, mh, W)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dh,H,Hkv", [(64, 4, 1), (128, 8, 2), (64, 16, 1), (128, 40, 2)])
def test_whole_tiles_that_are_not_held(kind, dh, H, Hkv):
    # the first, a middle, the last tiles of a sequence, all but one, and all of several: every tile is a workgroup's
    # own here, so that the join meets partial results of workgroups that saw no key
    say("decode unheld tiles", kind, dh, H, Hkv)
    rng = np.random.default_rng(dh + H + 2)
    lens = np.array([700, 700, 700, 1000, 900, 130, 5, 640], np.int32)
    c, cache, table = make(rng, lens, 16, Hkv, dh, kind)
    table[0, :8] = -1
    table[1, 16:32] = c["k"].shape[0]
    table[2, 32:] = -1
    table[3, :24], table[3, 32:] = -1, -(2 ** 31)
    table[4] = -1
    table[5, :8] = -1
    W = workgroups(cache, len(lens), H)
    runs, tiles = cut(lens, Hkv * sets(H // Hkv)[1], W)
    assert tiles <= W
    poison(c, table, lens)
    q = queries(rng, len(lens), H, dh)
    o, mh = S.attention_scores_decode(to_device(c), t(table), t(lens), t(q))
    torch.cuda.synchronize()
    check(c, table, lens, q, o, mh, W)


def test_every_array_of_a_replayed_8_bit_step():
    # steps captured once and replayed with new rows, eager work between: all five arrays of the cache, and the outputs
    say("decode replayed e4m3 step")
    rng = np.random.default_rng(3)
    Hkv, dh, steps = 3, 64, 4
    start = np.array([30, 127, 500], np.int32)
    c, cache, table = make(rng, start + steps, 16, Hkv, dh, "e4m3")
    twin, tb = to_device(c), t(table)
    k, v, m = (torch.zeros(s, device=DEV, dtype=d) for s, d in
               (((3, Hkv, dh), torch.bfloat16), ((3, Hkv, dh), torch.bfloat16), ((3, 2), torch.float32)))
    q = t(queries(rng, 3, 6, dh))
    ln, ln2 = t(start.copy()), t(start.copy())
    ws, ws2 = (torch.empty(S.attention_decode_workspace_bytes(cache, 3, 6), dtype=torch.uint8, device=DEV) for _ in range(2))

    def step(cache, ln, ws):
        ln += 1
        S.kv_write(cache, tb, ln, k, v, m)
        return S.attention_scores_decode(cache, tb, ln, q, workspace=ws)

    step(to_device(c), t(start.copy()), ws)  # loads the kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(cache, ln, ws)
    for s in range(steps):
        k.copy_(t(rows(rng, 3, Hkv, dh, "bf16")))
        v.copy_(t(rows(rng, 3, Hkv, dh, "bf16")))
        m.copy_(t(rng.uniform(0, 1, (3, 2)).astype(np.float32)))
        graph.replay()
        want = step(twin, ln2, ws2)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        for n in ("k", "v", "k_scale", "v_scale", "m"):
            assert torch.equal(getattr(cache, n), getattr(twin, n)), (s, n)
