"""The probabilities of wide groups (more than four query heads per KV head) enter the value products as three bf16
terms: their sum is the float32 probability in every bit, and no term of a positive one is zero."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import serving as V
from paper_2604_23996_amd import smoes as S
from tests.gpu_util import host, say, t
from tests.test_gpu_decode import run

pytestmark = pytest.mark.gpu

LOG2E = float(np.float32(1.4426950408889634))


def bf16_parts(x):
    """Three bf16 values (as bits) whose sum is the float32 x: its bits cut into eights."""
    parts, x = [], np.asarray(x, dtype=np.float32)
    for _ in range(3):
        u = x.view(np.uint32) & np.uint32(0xffff0000)
        parts.append((u >> 16).astype(np.uint16))
        x = x - u.view(np.float32)
    assert not x.any()
    return parts


def two_keys(kind, n_seq, dh):
    """A cache of n_seq sequences with two keys each: K = 0, and K = 1 in dims 0 .. 2. Values and scores are zeros."""
    c = dict(kind=kind, m=np.zeros((n_seq, 2, 16), np.float32))
    for n in ("k", "v"):
        c[n] = np.zeros((n_seq, 1, 16, dh), np.uint16 if kind == "bf16" else np.uint8)
        c[n + "_scale"] = np.full((n_seq, 1, 16), 127, np.uint8)
    c["k"][:, 0, 1, :3] = bits(kind, 1.0)
    return c, np.arange(n_seq, dtype=np.int32)[:, None], np.full(n_seq, 2, np.int32)


def bits(kind, x):
    """The stored form of values that the kind holds exactly (a row's scale is 1)."""
    x = np.asarray(x, dtype=np.float64)
    if kind == "bf16":
        return V.bf16_round(x)
    codes = np.array([V.kv_quantize([v, 448.0])[0][0] for v in x.ravel()], np.uint8).reshape(x.shape)
    assert np.array_equal(V.E4M3[codes], x)
    return codes


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("H", [4, 16, 32])
def test_no_bit_of_a_probability_is_lost(kind, H):
    # Two keys of weight 1 and p = h + j 2^-24, values -h and 1, scores the same: numerator p - h. p in [1/2, 1) is a
    # multiple of 2^-24, h of 2^-8, every partial sum of the terms' products a multiple of 2^-24 below 1 in size: all
    # are float32 numbers, nothing is rounded before the division, and o is the float32 score rounded to bf16. A term
    # that loses the last bit changes p - h, a few times 2^-24, by a large part of itself.
    say("decode terms", kind, H)
    n = 128 if kind == "bf16" else 8
    h = np.arange(n, 2 * n) / (2.0 * n)
    c, table, lens = two_keys(kind, n, 64)
    c["v"][:, 0, 0, 0], c["v"][:, 0, 1, 0] = bits(kind, -h), bits(kind, 1.0)
    c["m"][:, 0, 0], c["m"][:, 0, 1] = -h, 1.0
    want = h[:, None] + (np.arange(H) - H // 2 + 0.5) * 2.0 ** -24
    q = np.zeros((n, H, 64), np.uint16)
    for d, part in enumerate(bf16_parts(np.log2(want) / LOG2E)):
        q[:, :, d] = part
    o, mh = run(c, table, lens, q, scale=1.0)
    o, mh = host(o)[:, :, 0], mh.cpu().numpy()[:, :, 0]
    # the numerator, to the logit's roundings (|x| <= 1: 2^-24 and 2^-25) and the exponential's (2^-23)
    assert np.all(np.abs(mh * (1 + want) - (want - h[:, None])) <= 4 * 2.0 ** -24)
    assert (mh != 0).mean() > 0.5
    assert np.array_equal(o, host(torch.from_numpy(mh).bfloat16())), np.argwhere(o != host(torch.from_numpy(mh).bfloat16()))[:4]


@pytest.mark.parametrize("H", [4, 16, 32])
def test_an_infinite_value_stays_infinite_at_any_weight(H):
    # weights from 1 down to 2^-125, the smallest normal ones: infinity times a positive number
    say("decode small weights", H)
    down = np.arange(0.0, 126.0)
    n = len(down)
    c, table, lens = two_keys("bf16", n, 64)
    c["v"][:, 0, 0, :] = bits("bf16", 2.0)
    c["v"][:, 0, 1, 3], c["v"][:, 0, 1, 4] = 0x7f80, 0xff80
    q = np.zeros((n, H, 64), np.uint16)
    q[:, :, 0] = V.bf16_round(-down / LOG2E)[:, None]
    o, mh = run(c, table, lens, q, scale=1.0)
    o = host(o)
    assert np.isfinite(host(mh)).all() and np.isfinite(np.delete(o, [3, 4], axis=2)).all()
    bad = np.argwhere((o[:, :, 3] != np.inf) | (o[:, :, 4] != -np.inf))
    assert bad.size == 0, sorted(set(bad[:, 0]))
