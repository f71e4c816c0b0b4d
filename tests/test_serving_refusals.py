"""What the rotary, cache and decode entry points refuse on the host, before anything touches a GPU."""
import ctypes
import math
import os

import pytest
import torch

from paper_2604_23996_amd import smoes as S

pytestmark = pytest.mark.skipif(not os.path.exists(S.LIB_PATH), reason="libsmoes.so not built")

FAKE = ctypes.c_void_p(0x1000)  # never dereferenced: every call below returns before a launch
ARG, SHAPE, WS, OK = S.SMOES_ERR_ARG, S.SMOES_ERR_SHAPE, S.SMOES_ERR_WORKSPACE, S.SMOES_OK


def _rot(**kw):
    return S.SmoesRotary(*[{**dict(head_dim=64, rot_dim=32, layout=0, scaling=0, base=1e4, factor=1.0,
                                   original_len=4096.0, beta_fast=32.0, beta_slow=1.0), **kw}[n]
                           for n, _ in S.SmoesRotary._fields_])


def _apply(T=10, dt=1, backward=0, q=FAKE, qs=128, H=2, qo=FAKE, qos=128, k=FAKE, ks=64, Hkv=1, ko=FAKE, kos=64,
           rot=None, freqs=FAKE, amplitude=1.0):
    return S.lib().smoes_rotary_apply(_rot() if rot is None else rot, freqs, amplitude, None, T, dt, backward, q, qs,
                                      H, qo, qos, k, ks, Hkv, ko, kos, None)


def test_rotary_frequencies():
    out, amp = (ctypes.c_double * 256)(), ctypes.c_float()
    f = lambda **kw: S.lib().smoes_rotary_frequencies(_rot(**kw), out, ctypes.byref(amp))
    assert f() == OK and out[0] == 1.0 and amp.value == 1.0
    for kw in (dict(head_dim=1), dict(head_dim=513), dict(rot_dim=0), dict(rot_dim=33), dict(rot_dim=66)):
        assert f(**kw) == SHAPE, kw
    for kw in (dict(layout=2), dict(scaling=4), dict(scaling=-1), dict(base=0.0), dict(base=math.nan),
               dict(base=math.inf), dict(scaling=1, factor=0.5), dict(scaling=2, factor=math.nan),
               dict(scaling=3, original_len=0.0), dict(scaling=3, beta_fast=1.0), dict(scaling=3, beta_slow=-1.0)):
        assert f(**kw) == ARG, kw
    assert f(factor=0.5) == OK  # an unscaled spec does not read the factor
    assert f(rot_dim=2, scaling=2, factor=8.0) == OK and out[0] == 1.0
    assert S.lib().smoes_rotary_frequencies(None, out, ctypes.byref(amp)) == ARG
    assert S.lib().smoes_rotary_frequencies(_rot(), None, ctypes.byref(amp)) == ARG
    with pytest.raises(ValueError):
        S.rotary_frequencies(S.RotarySpec(64, 32, layout="other"))
    with pytest.raises(S.SmoesError):
        S.rotary_frequencies(S.RotarySpec(64, 31))


def test_rotary_apply():
    assert _apply(T=0, q=None, k=None, qo=None, ko=None, freqs=None) == OK
    assert _apply(T=-1) == SHAPE and _apply(T=1 << 24) == SHAPE and _apply(T=1 << 31) == SHAPE
    assert _apply(H=0) == SHAPE and _apply(Hkv=-1) == SHAPE and _apply(H=70000) == SHAPE
    assert _apply(H=40000, Hkv=40000, qs=1 << 30, qos=1 << 30, ks=1 << 30, kos=1 << 30) == SHAPE
    assert _apply(qs=127) == SHAPE and _apply(qos=127) == SHAPE and _apply(ks=63) == SHAPE and _apply(kos=0) == SHAPE
    assert _apply(rot=_rot(rot_dim=7)) == SHAPE
    assert _apply(dt=2) == ARG and _apply(backward=2) == ARG and _apply(amplitude=math.nan) == ARG
    assert _apply(rot=_rot(layout=5)) == ARG and _apply(freqs=None) == ARG
    assert _apply(q=None) == ARG and _apply(qo=None) == ARG and _apply(k=None) == ARG and _apply(ko=None) == ARG
    # in place with another stride would overwrite rows that are still to be read
    assert _apply(qs=128, qos=256) == ARG and _apply(qos=128, ks=64, kos=128) == ARG


def _cache(**kw):
    d = dict(n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, kind=1, k=0x1000, v=0x1000, k_scale=0x1000,
             v_scale=0x1000, m=0x1000)
    d.update(kw)
    return S.SmoesKvCache(*[d[n] for n, _ in S.SmoesKvCache._fields_])


def _write(cache=None, bt=FAKE, max_pages=3, lens=FAKE, n_seq=2, off=FAKE, T=5, k=FAKE, ks=128, v=FAKE, vs=128, dt=1,
           m=FAKE):
    return S.lib().smoes_kv_write(_cache() if cache is None else cache, bt, max_pages, lens, n_seq, off, T, k, ks, v,
                                  vs, dt, m, None)


def _read(cache=None, bt=FAKE, max_pages=3, lens=FAKE, n_seq=2, off=FAKE, T=5, k=FAKE, v=FAKE, dt=1, m=FAKE):
    return S.lib().smoes_kv_read(_cache() if cache is None else cache, bt, max_pages, lens, n_seq, off, T, k, v, dt,
                                 m, None)


def _decode(cache=None, bt=FAKE, max_pages=3, lens=FAKE, n_seq=2, q=ctypes.c_void_p(0x2000), qs=256, H=4, scale=0.0, o=FAKE, m=FAKE,
            ws=FAKE, n=1 << 40):
    return S.lib().smoes_attention_scores_decode(_cache() if cache is None else cache, bt, max_pages, lens, n_seq, q,
                                                 qs, H, scale, o, m, ws, n, None)


@pytest.mark.parametrize("call", [_write, _read, _decode])
def test_cache_sizes(call):
    for kw in (dict(n_pages=0), dict(n_pages=1 << 31), dict(page_size=8), dict(page_size=48), dict(page_size=8192),
               dict(page_size=0), dict(page_size=-16), dict(n_kv_heads=0), dict(head_dim=96), dict(head_dim=0)):
        assert call(cache=_cache(**kw)) == SHAPE, kw
    assert call(cache=_cache(kind=2)) == ARG and call(cache=_cache(kind=-1)) == ARG
    assert call(max_pages=0) == SHAPE and call(max_pages=(1 << 30) // 16 + 1) == SHAPE and call(n_seq=-1) == SHAPE
    # arrays: present, aligned, scales only where the kind has them
    for kw in (dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None), dict(k=0x1008), dict(v=0x1002),
               dict(k_scale=0x1002), dict(m=0x1004)):
        assert call(cache=_cache(**kw)) == ARG, kw
    assert call(bt=None) == ARG and call(lens=None) == ARG


def test_write_and_read():
    for call in (_write, _read):
        assert call(T=0) == OK and call(n_seq=0, T=3) == OK
        assert call(T=-1) == SHAPE and call(T=1 << 24) == SHAPE
        assert call(off=None, T=5) == SHAPE  # one token per sequence
        assert call(dt=2) == ARG
    assert _write(ks=127) == SHAPE and _write(vs=0) == SHAPE
    assert _write(k=None) == ARG and _write(v=None) == ARG
    # scores are written exactly when the cache keeps them
    assert _write(m=None) == ARG and _write(cache=_cache(m=None)) == ARG
    assert _read(cache=_cache(m=None)) == ARG
    assert _read(k=None, v=None, m=None) == OK  # nothing wanted


def test_decode():
    assert _decode(n_seq=0) == OK
    assert _decode(H=3) == SHAPE and _decode(H=0) == SHAPE and _decode(qs=255) == SHAPE
    assert _decode(n_seq=1 << 20, H=16) == SHAPE  # 2^24 workgroups
    assert _decode(o=FAKE, q=FAKE) == ARG  # in place
    assert _decode(scale=math.nan) == ARG and _decode(q=None) == ARG and _decode(o=None) == ARG
    assert _decode(m=None) == ARG and _decode(cache=_cache(m=None)) == ARG
    need = S.lib().smoes_attention_decode_workspace_size(_cache(), 2, 4)
    assert need > 0
    assert _decode(n=need - 1) == WS and _decode(ws=None) == WS
    size = S.lib().smoes_attention_decode_workspace_size
    assert size(_cache(), 2, 3) == 0 and size(_cache(), -1, 4) == 0 and size(_cache(head_dim=80), 2, 4) == 0
    assert size(None, 2, 4) == 0


def test_binding_checks():
    c = S.KVCache(4, 16, 2, 64, device="cpu")
    table, lens = torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    row = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    m = torch.zeros(3, 2)
    with pytest.raises(ValueError, match="GPU"):
        S.kv_write(c, table, lens, row, row, m)
    with pytest.raises(ValueError, match="GPU"):
        S.kv_read(c, table, lens)
    with pytest.raises(ValueError, match="GPU"):
        S.attention_scores_decode(c, table, lens, torch.zeros(3, 4, 64, dtype=torch.bfloat16))
    for bad in (dict(table=table.long()), dict(lens=lens.float()), dict(table=table[:2]), dict(k=row[:, :1]),
                dict(k=row.transpose(1, 2)), dict(v=row.float()), dict(m=m[:2]), dict(m=m.double()),
                dict(k=row[:1].expand(3, 2, 64)), dict(offsets=torch.zeros(3, dtype=torch.int32))):
        a = {**dict(table=table, lens=lens, k=row, v=row, m=m, offsets=None), **bad}
        with pytest.raises((ValueError, TypeError)) as e:
            S.kv_write(c, a["table"], a["lens"], a["k"], a["v"], a["m"], sample_offsets=a["offsets"])
        assert "GPU" not in str(e.value), bad
    for bad in (torch.zeros(3, 4, 64), torch.zeros(2, 4, 64, dtype=torch.bfloat16),
                torch.zeros(3, 4, 128, dtype=torch.bfloat16), torch.zeros(3, 256, dtype=torch.bfloat16)):
        with pytest.raises((ValueError, TypeError)) as e:
            S.attention_scores_decode(c, table, lens, bad)
        assert "GPU" not in str(e.value)
    with pytest.raises(ValueError):
        S.KVCache(4, 16, 2, 64, kind="int8", device="cpu")
    with pytest.raises(ValueError):
        S.KVCache(4, 16, 2, 64, device="cpu", k=torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        S.kv_read(c, table, lens, sample_offsets=torch.zeros(4, dtype=torch.int32))
    plan = S.RotaryPlan(S.RotarySpec(64, 32), "cpu")
    with pytest.raises(ValueError, match="GPU"):
        S.rotary(plan, row)
    with pytest.raises(ValueError):
        S.rotary(plan, torch.zeros(3, 2, 32))
    with pytest.raises(ValueError):
        S.rotary(plan, row, positions=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        S.rotary(plan, row, positions=torch.zeros(3))
    with pytest.raises(TypeError):
        S.rotary(plan, row, row.float())
