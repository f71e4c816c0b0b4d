"""Pins of the serving oracle (CPU): each against something that is not its own formula."""
import math

import numpy as np
import pytest
import torch

import oracle as O
from oracle import serving as V


def test_e4m3_values_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    ref = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(V.E4M3, ref, equal_nan=True)


def test_quantized_codes_are_torchs_casts_and_the_scale_is_the_smallest():
    rng = np.random.default_rng(0)
    for i in range(60):
        row = (rng.standard_normal(64) * 2.0 ** rng.integers(-100, 100)).astype(np.float32)
        row[:4] *= 2.0 ** -12
        row[5] = 0.0
        codes, e = V.kv_quantize(row)
        top = np.abs(row.astype(np.float64)).max()
        assert top <= 448 * 2.0 ** e and (top > 448 * 2.0 ** (e - 1) or e == -117)
        ref = torch.ldexp(torch.from_numpy(row).double(), torch.tensor(-e)).float().to(torch.float8_e4m3fn)
        assert np.array_equal(codes, ref.view(torch.uint8).numpy())


def test_quantized_ties_go_to_the_even_code():
    # 448 fixes the scale at 1; 17 lies between 16 (code 0x58) and 18 (0x59), 19 between 18 and 20 (0x5a)
    codes, e = V.kv_quantize([448.0, 17.0, 19.0, -17.0, 2.0 ** -10, 3 * 2.0 ** -10, -0.0])
    assert e == 0 and codes.tolist() == [0x7e, 0x58, 0x5a, 0xd8, 0x00, 0x02, 0x80]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_is_a_complex_product(layout):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 12))
    pos = np.array([0, 1, -7, 1000, 2 ** 31 - 1])
    f, a = V.rotary_frequencies(8, "by_parts", 10000.0, 16.0, 2048, 32.0, 1.0)
    y = V.rotary(x, pos, f, a, 8, layout)
    i, j = (np.arange(4), np.arange(4, 8)) if layout == "half" else (np.arange(0, 8, 2), np.arange(1, 8, 2))
    z = (x[..., i] + 1j * x[..., j]) * a * np.exp(1j * pos[:, None] * f)[:, None]
    assert np.allclose(y[..., i], z.real, rtol=0, atol=1e-9) and np.allclose(y[..., j], z.imag, rtol=0, atol=1e-9)
    assert np.array_equal(y[..., 8:], x[..., 8:])
    # the transpose: <R x, g> = <x, R^T g>
    g = rng.standard_normal(x.shape)
    assert math.isclose((y * g).sum(), (x * V.rotary(g, pos, f, a, 8, layout, backward=True)).sum(), rel_tol=1e-10)


def test_rotary_scores_depend_on_the_distance():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    f, _ = V.rotary_frequencies(16, "none", 10000.0, 1.0, 0, 0, 0)
    dot = [float((V.rotary(q, [p + 5], f, 1.0, 16, "half") * V.rotary(k, [p], f, 1.0, 16, "half")).sum()) for p in (0, 3, 777)]
    assert np.allclose(dot, dot[0], atol=1e-12)


def test_rotary_frequencies_limits():
    f, a = V.rotary_frequencies(64, "none", 10000.0, 1.0, 0, 0, 0)
    assert f[0] == 1.0 and a == 1.0 and np.allclose(f[1:] / f[:-1], 10000.0 ** (-1 / 32))
    # linear: all divided; ntk: the first kept, the last divided by the factor; by parts: many turns kept, few divided
    lin, _ = V.rotary_frequencies(64, "linear", 10000.0, 8.0, 0, 0, 0)
    ntk, _ = V.rotary_frequencies(64, "ntk", 10000.0, 8.0, 0, 0, 0)
    part, amp = V.rotary_frequencies(64, "by_parts", 10000.0, 8.0, 4096, 32.0, 1.0)
    assert np.allclose(lin, f / 8) and ntk[0] == 1.0 and math.isclose(ntk[-1], f[-1] / 8, rel_tol=1e-12)
    assert part[0] == f[0] and math.isclose(part[-1], f[-1] / 8) and math.isclose(amp, 1 + 0.1 * math.log(8))


def _cache(rng, n_pages, Hkv, page, dh, kind):
    c = dict(kind=kind, m=np.zeros((n_pages, 2, page), np.float32))
    for n in ("k", "v"):
        c[n] = np.zeros((n_pages, Hkv, page, dh), np.uint16 if kind == "bf16" else np.uint8)
        c[n + "_scale"] = np.zeros((n_pages, Hkv, page), np.uint8)
    return c


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_decode_is_the_last_row_of_the_causal_attention(kind):
    # written in two calls, shuffled pages, then read back whole and given to the oracle of whole samples
    rng = np.random.default_rng(3)
    H, Hkv, dh, page, lens = 4, 2, 64, 16, np.array([37, 0, 16, 1])
    table = np.full((4, 4), -1, np.int32)
    table[0, :3], table[2, :1], table[3, :1] = [5, 0, 3], [1], [4]
    c = _cache(rng, 6, Hkv, page, dh, kind)
    first, second = np.array([30, 0, 10, 0]), np.array([7, 0, 6, 1])
    off1, off2 = np.concatenate([[0], first.cumsum()]), np.concatenate([[0], second.cumsum()])
    for off, l in ((off1, first), (off2, lens)):
        T = int(off[-1])
        k, v = (V.bf16_round(rng.standard_normal((T, Hkv, dh))) for _ in range(2))
        V.kv_write(c, table, l, off, k, v, rng.uniform(0, 1, (T, 2)).astype(np.float32))
    off = np.concatenate([[0], lens.cumsum()])
    T = int(off[-1])
    k, v, m = np.zeros((T, Hkv, dh)), np.zeros((T, Hkv, dh)), np.zeros((T, 2))
    V.kv_read(c, table, lens, off, T, k, v, m)
    q = rng.standard_normal((T, H, dh))
    ref_o, ref_m = O.attention_heads(q, k, v, off, m)
    last = [36, 36, 52, 53]
    o, mh, size, av, keys = V.attention_decode(c, table, lens, q[last])
    assert keys.tolist() == [37, 0, 16, 1] and not o[1].any() and not mh[1].any()
    for b in (0, 2, 3):
        assert np.allclose(o[b], ref_o[last[b]], atol=1e-12) and np.allclose(mh[b], ref_m[last[b]], atol=1e-12)


def test_places():
    table = np.array([[2, -1], [0, 9]], np.int32)
    # lengths past the table, a page that is not held, a negative position, a row behind the last sequence
    got = V.kv_places(table, np.array([18, 40]), np.array([0, 20, 22]), 23, 3, 16)
    assert got[:3] == [None, None, (2, 0)] and got[17] == (2, 15) and got[18] is None and got[19] is None
    assert got[20] is None and got[21] is None and got[22] is False
