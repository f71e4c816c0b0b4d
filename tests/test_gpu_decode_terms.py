"""The probabilities of wide groups (more than four query heads per KV head) enter the value products as three bf16
terms: no term of a positive one is zero."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import serving as V
from tests.gpu_util import host, say
from tests.test_gpu_decode import run

pytestmark = pytest.mark.gpu

LOG2E = float(np.float32(1.4426950408889634))


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
