"""Cache and rotary kernels whose workgroups go over their rows more than once: a trip is 64 rows of the cache, 512
pieces of heads of the rotation; the last trip is part full.

Cache rows are drawn from a set of distinct ones, so that the oracle quantises each once; every array of the cache
and everything that is read back is compared whole, bit for bit."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import serving as V
from paper_2604_23996_amd import smoes as S
from tests.gpu_util import DEV, host, say, t
from tests.test_gpu_kvcache import make, rows, same
from tests.test_gpu_rotary import _check

pytestmark = pytest.mark.gpu

SET = 97


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dh,Hkv,new,page", [
    (128, 33, [3, 0, 4], 16),              # one token a workgroup: 66 rows
    (64, 70, [40, 1], 32),                 # 140 rows
    (64, 8, [9000, 1, 0, 7300, 99], 64),   # 16 tokens a workgroup when writing: 256 rows; the last 16 short
    (128, 5, [7001, 3000], 256),           # 9 and 7 tokens, 90 and 70 rows
])
def test_cache_rows(kind, dtype, dh, Hkv, new, page):
    say("row loops, cache", kind, dtype, dh, Hkv)
    rng = np.random.default_rng(dh + Hkv)
    new = np.array(new)
    lens = (new + rng.integers(0, 30, len(new))).astype(np.int32)
    c, cache, table = make(rng, lens, page, Hkv, dh, kind)
    off = np.concatenate([[0], new.cumsum()]).astype(np.int32)
    T = int(off[-1]) + 3
    m = rng.uniform(0, 1, (T, 2)).astype(np.float32)
    at = V.kv_places(table, lens, off, T, c["k"].shape[0], page)
    held = np.array([i for i, a in enumerate(at) if a])
    page_of, slot_of = np.array([at[i] for i in held]).T
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, out, want = {}, {}, {}
    for n, step in (("k", 5), ("v", 11)):
        base = rows(rng, SET, 1, dh, dtype)[:, 0]
        which = (np.arange(T)[:, None] * step + np.arange(Hkv) * 3) % SET
        x[n] = t(base[which])
        if kind == "e4m3":
            codes, e = zip(*(V.kv_quantize(V.widen(r)) for r in base))
            codes, e = np.stack(codes), np.array(e)
            c[n][page_of, :, slot_of] = codes[which[held]]
            c[n + "_scale"][page_of, :, slot_of] = (e + 127)[which[held]]
            back = V.E4M3[codes] * 2.0 ** e[:, None]
        else:
            stored = base if base.dtype == np.uint16 else V.bf16_round(base)
            c[n][page_of, :, slot_of] = stored[which[held]]
            back = V.widen(stored)
        want[n] = np.full((T, Hkv, dh), 7.0)
        want[n][held] = back[which[held]]
        out[n] = torch.full((T, Hkv, dh), 7.0, dtype=td, device=DEV)
    assert len(held) == off[-1]
    c["m"][page_of, :, slot_of] = m[held]
    out["m"] = torch.full((T, 2), 7.0, device=DEV)
    S.kv_write(cache, t(table), t(lens), x["k"], x["v"], t(m), sample_offsets=t(off))
    same(c, cache)
    S.kv_read(cache, t(table), t(lens), sample_offsets=t(off), **out)
    torch.cuda.synchronize()
    for n in ("k", "v"):
        assert np.array_equal(host(out[n]), want[n]), n
    assert np.array_equal(out["m"].cpu().numpy()[:-3], m[:-3]) and bool((out["m"][-3:] == 7.0).all())


ROTARY = [  # T, H, Hkv, head_dim, rot_dim, layout, dtype
    (5, 40, 8, 128, 66, "half", torch.bfloat16),          # moved-back last pieces in both halves and the rest
    (3, 12, 5, 512, 512, "half", torch.float32),
    (7, 30, 3, 100, 50, "half", torch.float32),
    (4, 20, 9, 128, 70, "interleaved", torch.float32),
    (6, 32, 8, 256, 242, "interleaved", torch.bfloat16),
    (2060, 20, 2, 128, 66, "half", torch.bfloat16),   # two tokens a workgroup
    (3081, 8, 3, 64, 64, "interleaved", torch.float32),
]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("case", ROTARY, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_rotary_pieces(case, backward):
    T, H, Hkv, dh, r, layout, dt = case
    say("row loops, rotary", case, backward)
    V_ = 8 if dt == torch.bfloat16 else 4
    pairs = -(-(r // 2) // (V_ // 2 if layout == "interleaved" else V_))
    per_token = (H + Hkv) * (pairs + -(-(dh - r) // V_))
    tokens = max(1, min(-(-512 // per_token), T // 1024, 16))
    assert tokens * per_token > 512
    g = torch.Generator().manual_seed(T + dh)
    spec = S.RotarySpec(dh, r, layout=layout, scaling="by_parts", factor=8.0)
    plan = S.RotaryPlan(spec, DEV)
    q, k = (torch.randn(T, h, dh, generator=g).to(dt).to(DEV) for h in (H, Hkv))
    pos = torch.randint(-5, 200000, (T,), generator=g, dtype=torch.int32)
    qo, ko = S.rotary(plan, q, k, positions=pos.to(DEV), backward=backward)
    torch.cuda.synchronize()
    _check(spec, q, qo, pos.numpy(), backward)
    _check(spec, k, ko, pos.numpy(), backward)
    S.rotary(plan, q, k, positions=pos.to(DEV), backward=backward, q_out=q, k_out=k)
    torch.cuda.synchronize()
    assert torch.equal(q, qo) and torch.equal(k, ko)
