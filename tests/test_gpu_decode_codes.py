"""The decode over 8-bit caches with what no other test puts there: NaN codes in held rows, and rows whose scales are far
from 1."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import serving as V
from tests.gpu_util import host, say
from tests.test_gpu_decode import U, poison, queries, run
from tests.test_gpu_decode_terms import LOG2E, bf16_parts, bits, two_keys
from tests.test_gpu_kvcache import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("code", [0x7f, 0xff])
@pytest.mark.parametrize("H,dh", [(8, 64), (32, 128), (40, 64)])
def test_nan_codes_reach_their_own_rows(H, dh, code):
    # a NaN key: every output of its sequence and KV head; a NaN value: its column; nothing else
    say("decode NaN codes", H, dh, code)
    rng = np.random.default_rng(H)
    lens = np.array([300, 300, 300], np.int32)
    c, _, table = make(rng, lens, 16, 2, dh, "e4m3")
    g = H // 2
    for j in (0, 17, 46, 200):
        c["k"][table[0, j // 16], 1, j % 16, j % dh] = code
        c["v"][table[1, j // 16], 0, j % 16, 5] = code
    q = queries(rng, 3, H, dh, std=0.2)
    o, mh = run(c, table, lens, q)
    o, mh = host(o), host(mh)
    assert np.isnan(o[0, g:]).all() and np.isnan(mh[0, g:]).all()
    assert np.isfinite(o[0, :g]).all() and np.isfinite(mh[0, :g]).all()
    assert np.isnan(o[1, :g, 5]).all() and np.isfinite(np.delete(o[1, :g], 5, axis=1)).all()
    assert np.isfinite(o[1, g:]).all() and np.isfinite(o[2]).all() and np.isfinite(mh[1:]).all()


@pytest.mark.parametrize("H,dh", [(8, 64), (32, 128), (40, 64)])
def test_scales_far_from_one(H, dh):
    # keys of 2^-100 against queries of 2^100 and the reverse, values of 2^-100, 2^-60, 2^60 and 2^100
    say("decode scales", H, dh)
    rng = np.random.default_rng(H + 1)
    lens = np.array([300, 129, 77, 640], np.int32)
    c, _, table = make(rng, lens, 16, 2, dh, "e4m3")
    q = V.widen(queries(rng, 4, H, dh))
    for b, (ke, ve) in enumerate(((-100, -100), (100, -60), (-100, 60), (100, 100))):
        pages = table[b, :-(-int(lens[b]) // 16)]
        c["k_scale"][pages] += np.uint8(ke % 256)  # modulo 256: the bytes stay between 18 and 224
        c["v_scale"][pages] += np.uint8(ve % 256)
        q[b] *= 2.0 ** -ke
    poison(c, table, lens)
    q = V.bf16_round(q)
    o, mh = run(c, table, lens, q)
    # The bound of tests/test_gpu_decode.py, and what outputs near bf16's smallest numbers cost: an output below 2^-126 is
    # rounded to a multiple of 2^-133, so it is off by up to 2^-134 beside (key codes and queries make the softmax so
    # sharp that an output can be 1e-42); products below 2^-126 are multiples of 2^-149, 640 of them off by 2^-140.
    ref_o, ref_m, size, av, keys = V.attention_decode(c, table, lens, q)
    rel = 2 * ((dh + 5) * U * size + 4 * U + (keys[:, None] + 64) * U)
    tol = rel[..., None] * av + 2.0 ** -140
    tol = tol + 2.0 ** -8 * (np.abs(ref_o) + tol) + 2.0 ** -134
    err = np.abs(host(o) - ref_o)
    assert np.all(err <= tol), (np.max(err - tol), np.argwhere(err > tol)[:4])
    assert np.all(np.abs(host(mh) - ref_m) <= rel[..., None])


@pytest.mark.parametrize("H,dh", [(8, 64), (8, 128), (32, 128), (40, 64)])
def test_large_queries_on_small_keys(H, dh):
    # queries of 2^117 to 2^119 on keys of 2^-119 or so: the products of what is read back are moderate, those of the codes
    # with the queries are beyond float32
    say("decode large queries", H, dh)
    rng = np.random.default_rng(H + 2)
    lens = np.array([300, 70], np.int32)
    c, _, table = make(rng, lens, 16, 2, dh, "e4m3")
    c["k"] = (c["k"] & 0x87) | rng.integers(8, 15, c["k"].shape).astype(np.uint8) << 3  # 2 to 256: no code near zero
    c["k_scale"][:] = 10
    q = V.bf16_round(queries_of(rng, 2, H, dh))
    poison(c, table, lens)
    o, mh = run(c, table, lens, q)
    ref_o, ref_m, size, av, keys = V.attention_decode(c, table, lens, q)
    rel = 2 * ((dh + 5) * U * size + 4 * U + (keys[:, None] + 64) * U)
    # The logits lie thousands apart: weights below 2^-126 of the largest are zero in float32, up to 300 of them on values
    # below 64 (codes of 448 at most, scales of 2^-3), 2^-111 together, all that is left of a column whose largest value is 0.
    tol = rel[..., None] * av + 300 * 2.0 ** -126 * 64
    tol = tol + 2.0 ** -8 * (np.abs(ref_o) + tol)
    assert np.all(np.abs(host(o) - ref_o) <= tol)
    assert np.all(np.abs(host(mh) - ref_m) <= rel[..., None])


def queries_of(rng, n, H, dh):
    return np.where(rng.random((n, H, dh)) < 0.5, -1.0, 1.0) * 2.0 ** rng.integers(117, 120, (n, H, dh))


@pytest.mark.parametrize("H", [4, 16, 32])
@pytest.mark.parametrize("e", [-112, -116])
def test_weights_of_small_values_keep_their_bits(H, e):
    # Two keys of weight 1 and p = h + r, their values -h 2^e and 2^e, scores -h and 1. Every product and sum is a multiple of
    # 2^(e - 24) >= 2^-140 and below 2^e in size: float32 numbers. So the output is the scores' times 2^e, rounded to bf16;
    # r is such that it is a normal number, 2^-126 or more. Were the scale 2^e in the weight before it is cut into bf16
    # terms, what is under 2^-133 of the weight would be lost, up to 2^-8 of these outputs.
    say("decode small 8-bit values", H, e)
    n = 8
    h = np.arange(n, 2 * n) / (2.0 * n)
    c, table, lens = two_keys("e4m3", n, 64)
    c["v"][:, 0, 0, 0], c["v"][:, 0, 1, 0] = bits("e4m3", -h), bits("e4m3", 1.0)
    c["v_scale"][:] = 127 + e
    c["m"][:, 0, 0], c["m"][:, 0, 1] = -h, 1.0
    rng = np.random.default_rng(H - e)
    want = h[:, None] + 2.0 ** (-124 - e + rng.uniform(0, 1, (n, H)))
    assert want.max() < 1
    # the logit in 24 bits, in three bf16 values that meet the key's three ones
    q = np.zeros((n, H, 64), np.uint16)
    for d, part in enumerate(bf16_parts(np.log2(want) / LOG2E)):
        q[:, :, d] = part
    o, mh = run(c, table, lens, q, scale=1.0)
    o, mh = host(o)[:, :, 0], mh.cpu().double()[:, :, 0] * 2.0 ** e
    assert mh.min() >= 2.0 ** -126
    assert np.array_equal(o, host(mh.float().bfloat16())), np.mean(o != host(mh.float().bfloat16()))


@pytest.mark.parametrize("H", [4, 16, 32])
def test_one_key_returns_its_value_at_every_scale(H):
    # every scale byte that a write leaves, 10 to 247, and every code (at 2^120 up to 1.875 * 2^127, the last value below
    # infinity): a weight of 1 over a sum of 1, and the row as it is read back, a bf16 value, bit for bit
    say("decode one key, all scales", H)
    codes = np.concatenate([np.arange(127), np.arange(128, 255)]).astype(np.uint8)
    codes = np.resize(codes, 4 * 64).reshape(4, 64)
    scales = np.repeat(np.arange(10, 248), 4)
    n = len(scales)
    c, table, lens = two_keys("e4m3", n, 64)
    lens[:] = 1
    c["v"][:, 0, 0] = np.tile(codes, (n // 4, 1))
    c["v"][scales == 247] &= 0xf7  # codes of at most 240: below 0x78
    c["v_scale"][:, 0, 0] = scales
    c["k_scale"][:, 0, 0] = scales[::-1]
    c["m"][:, :, 0] = np.random.default_rng(H).uniform(0, 1, (n, 2))
    q = V.bf16_round(np.random.default_rng(H + 1).standard_normal((n, H, 64)))
    o, mh = run(c, table, lens, q)
    want = V.E4M3[c["v"][:, 0, 0]] * 2.0 ** (scales - 127.0)[:, None]
    assert np.abs(want).max() == 1.875 * 2.0 ** 127
    assert np.array_equal(host(o), np.broadcast_to(want[:, None], o.shape))
    assert np.array_equal(mh.cpu().numpy(), np.broadcast_to(c["m"][:, None, :, 0], mh.shape))
