"""CPU oracle of the operators of a model that generates with the attention-accumulated score: rotary positions,
the paged cache of keys, values and scores, and the attention of one new token over it (Eq. 3 for a token that is
generated). Plain NumPy in float64, one row or one (sequence, head) at a time, on the exact stored input values.

A cache is a dict: k, v [n_pages, n_kv_heads, page, head_dim] (uint16 bf16 bits or uint8 e4m3 codes), k_scale,
v_scale [n_pages, n_kv_heads, page] uint8 (e4m3), m [n_pages, 2, page] float32, and kind."""
from __future__ import annotations

import math
from typing import Optional

import numpy as np

from .smoes_oracle import widen

# every e4m3 code's value: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN
E4M3 = np.array([math.nan if (c & 0x7f) == 0x7f else
                 (-1.0) ** (c >> 7) * (((c & 7) + 8) * 2.0 ** (((c >> 3) & 15) - 10) if (c >> 3) & 15
                                       else (c & 7) * 2.0 ** -9) for c in range(256)])


def rotary_frequencies(rot_dim: int, scaling: str, base: float, factor: float, original_len: float,
                       beta_fast: float, beta_slow: float):
    """Radians per position of each pair, and the amplitude."""
    f = []
    if scaling == "ntk" and rot_dim > 2:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    for i in range(rot_dim // 2):
        x = base ** (-2.0 * i / rot_dim)
        if scaling == "linear":
            x = x / factor
        if scaling == "by_parts":
            turns = original_len * x / (2 * math.pi)
            g = min(1.0, max(0.0, (turns - beta_slow) / (beta_fast - beta_slow)))
            x = g * x + (1 - g) * x / factor
        f.append(x)
    return np.array(f), 1 + 0.1 * math.log(factor) if scaling == "by_parts" else 1.0


def rotary(x, positions, freqs, amplitude: float, rot_dim: int, layout: str, backward: bool = False) -> np.ndarray:
    """[T, H, head_dim] at its positions; backward: the transpose."""
    y = np.array(widen(x), dtype=np.float64)
    x = y.copy()
    w = np.asarray(positions, dtype=np.float64)[:, None] * freqs[None, :]
    c, s = np.cos(w), np.sin(w)
    for i in range(rot_dim // 2):
        a, b = (i, i + rot_dim // 2) if layout == "half" else (2 * i, 2 * i + 1)
        ci, si = c[:, i, None], s[:, i, None] * (-1.0 if backward else 1.0)
        y[:, :, a] = amplitude * (x[:, :, a] * ci - x[:, :, b] * si)
        y[:, :, b] = amplitude * (x[:, :, a] * si + x[:, :, b] * ci)
    return y


def kv_quantize(row):
    """One row's e4m3 codes and scale exponent e (value = E4M3[code] * 2^e): e the smallest integer >= -117 with
    max |x| <= 448 * 2^e over the finite values, 0 for a row of zeros; nearest code, ties to the even code; but never
    one past 1.875 * 2^127, the last value on the grid below float32's infinity."""
    x = np.asarray(row, dtype=np.float64)
    fin = np.abs(x[np.isfinite(x)])
    top = fin.max() if fin.size else 0.0
    e = 0
    if top > 0:
        e = -117
        while top > 448.0 * 2.0 ** e:
            e += 1
    codes = np.zeros(x.shape, np.uint8)
    grid = E4M3[:127]
    for i, v in enumerate(x):
        sign = 0x80 if math.copysign(1.0, v) < 0 else 0
        if not math.isfinite(v):
            codes[i] = 0x7f | sign
            continue
        a = min(abs(v), 1.875 * 2.0 ** 127) * 2.0 ** -e
        hi = min(int(np.searchsorted(grid, a)), 126)
        lo = max(hi - 1, 0)
        if a >= grid[hi]:
            c = hi
        elif a - grid[lo] != grid[hi] - a:
            c = lo if a - grid[lo] < grid[hi] - a else hi
        else:
            c = lo if lo % 2 == 0 else hi
        codes[i] = c | sign
    return codes, e


def bf16_round(x) -> np.ndarray:
    """float32 values to bf16 bits, nearest even (NaN kept quiet)."""
    u = np.ascontiguousarray(np.asarray(x, dtype=np.float32)).view(np.uint32)
    r = ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where((u & 0x7fffffff) > 0x7f800000, ((u >> 16) | 0x40).astype(np.uint16), r)


def kv_places(block_table, seq_lens, sample_offsets, T: int, n_pages: int, page: int):
    """Per token: (page, slot), None (no place), or False (a row behind the last sequence)."""
    n_seq, max_pages = block_table.shape
    out = []
    for t in range(T):
        if sample_offsets is None:
            b, n, j = t, 1, 0
        else:
            if t >= sample_offsets[n_seq]:
                out.append(False)
                continue
            b = max(i for i in range(n_seq) if sample_offsets[i] <= t < sample_offsets[i + 1])
            n, j = int(sample_offsets[b + 1] - sample_offsets[b]), t - int(sample_offsets[b])
        pos = int(seq_lens[b]) - n + j
        if pos < 0 or pos >= max_pages * page:
            out.append(None)
            continue
        p = int(block_table[b, pos // page])
        out.append((p, pos % page) if 0 <= p < n_pages else None)
    return out


def kv_write(cache, block_table, seq_lens, sample_offsets, k, v, m) -> None:
    """Appends rows k, v [T, n_kv_heads, head_dim] and m [T, 2] to the dict, in place."""
    n_pages, Hkv, page, _ = cache["k"].shape
    for t, at in enumerate(kv_places(block_table, seq_lens, sample_offsets, k.shape[0], n_pages, page)):
        if not at:
            continue
        p, s = at
        for name, x in (("k", k), ("v", v)):
            for h in range(Hkv):
                if cache["kind"] == "e4m3":
                    codes, e = kv_quantize(widen(x[t, h]))
                    cache[name][p, h, s] = codes
                    cache[name + "_scale"][p, h, s] = e + 127
                else:
                    cache[name][p, h, s] = x[t, h] if x.dtype == np.uint16 else bf16_round(x[t, h])
        if m is not None:
            cache["m"][p, :, s] = m[t]


def kv_row(cache, name: str, p: int, h: int, s) -> np.ndarray:
    """The float64 values of rows s of page p, head h."""
    x = cache[name][p, h, s]
    if cache["kind"] == "e4m3":
        return E4M3[x] * 2.0 ** (cache[name + "_scale"][p, h, s].astype(np.float64) - 127)[..., None]
    return widen(x)


def kv_read(cache, block_table, seq_lens, sample_offsets, T: int, k, v, m) -> None:
    """Reads T rows into float64 arrays k, v and m, in place."""
    n_pages, Hkv, page, _ = cache["k"].shape
    for t, at in enumerate(kv_places(block_table, seq_lens, sample_offsets, T, n_pages, page)):
        if at is False:
            continue
        for h in range(Hkv):
            for name, y in (("k", k), ("v", v)):
                y[t, h] = 0.0 if at is None else kv_row(cache, name, at[0], h, at[1])
        m[t] = 0.0 if at is None else cache["m"][at[0], :, at[1]]


def attention_decode(cache, block_table, seq_lens, q, scale: Optional[float] = None):
    """Per sequence and head: (o, m, and what an error bound of a float32 evaluation needs: the largest
    sum_d |q_d k_jd| * scale, sum_j p_j |v_j|, the number of keys)."""
    Q = widen(q)
    n_seq, H, dh = Q.shape
    n_pages, Hkv, page, _ = cache["k"].shape
    sc = 1.0 / math.sqrt(dh) if scale is None else float(scale)
    o, m = np.zeros((n_seq, H, dh)), np.zeros((n_seq, H, 2))
    size, av, keys = np.zeros((n_seq, H)), np.zeros((n_seq, H, dh)), np.zeros(n_seq, int)
    for b in range(n_seq):
        n = min(max(int(seq_lens[b]), 0), block_table.shape[1] * page)
        held = [(int(block_table[b, a // page]), min(page, n - a)) for a in range(0, n, page)]
        held = [(p, c) for p, c in held if 0 <= p < n_pages]
        keys[b] = sum(c for _, c in held)
        if keys[b] == 0:
            continue
        score = None if cache["m"] is None else np.concatenate([cache["m"][p, :, :c] for p, c in held], 1).astype(np.float64)
        for hk in range(Hkv):
            K = np.concatenate([kv_row(cache, "k", p, hk, slice(0, c)) for p, c in held])
            V = np.concatenate([kv_row(cache, "v", p, hk, slice(0, c)) for p, c in held])
            for h in range(hk * (H // Hkv), (hk + 1) * (H // Hkv)):
                x = (K @ Q[b, h]) * sc
                e = np.exp(x - x.max())
                e = e / e.sum()
                o[b, h] = e @ V
                av[b, h] = e @ np.abs(V)
                size[b, h] = (np.abs(K) @ np.abs(Q[b, h])).max() * sc
                if score is not None:
                    m[b, h] = score @ e
    return o, m, size, av, keys
