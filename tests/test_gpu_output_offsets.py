"""kv_read's rows and the decode's outputs written into dense slices that start at any element: the bits of the call
with outputs of its own, and nothing beside the slice."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2604_23996_amd import smoes as S
from tests.gpu_util import DEV, say, t
from tests.test_gpu_decode import queries
from tests.test_gpu_kvcache import make

pytestmark = pytest.mark.gpu


def slice_at(shift, shape, dtype):
    """A dense tensor `shift` elements into a larger one of sevens, and the larger one."""
    n = int(np.prod(shape))
    buf = torch.full((shift + n + 9,), 7.0, dtype=dtype, device=DEV)
    return buf[shift:shift + n].view(shape), buf


def beside(buf, shift, n):
    return bool((buf[:shift] == 7.0).all() and (buf[shift + n:] == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind,dh", [("bf16", 64), ("bf16", 128), ("e4m3", 64), ("e4m3", 128)])
def test_rows_read_back(kind, dh, dtype):
    say("kv_read offsets", kind, dh, dtype)
    rng = np.random.default_rng(dh)
    lens, off = np.array([37, 5], np.int32), np.array([0, 37, 42], np.int32)
    _, cache, table = make(rng, lens, 16, 3, dh, kind)
    want = S.kv_read(cache, t(table), t(lens), sample_offsets=t(off), T=42, dtype=dtype)
    for shift in (1, 2, 3, 5, 8):
        (k, kb), (v, vb) = slice_at(shift, (42, 3, dh), dtype), slice_at(shift + 2, (42, 3, dh), dtype)
        m, mb = slice_at(shift, (42, 2), torch.float32)
        S.kv_read(cache, t(table), t(lens), sample_offsets=t(off), k=k, v=v, m=m)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((k, v, m), want)), shift
        assert beside(kb, shift, k.numel()) and beside(vb, shift + 2, v.numel()) and beside(mb, shift, m.numel())


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("dh,H,Hkv", [(64, 6, 2), (128, 16, 1), (64, 20, 1)])
def test_outputs_of_the_decode(kind, dh, H, Hkv):
    # sequences that one workgroup finishes, that several share, and an empty one
    say("decode offsets", kind, dh, H, Hkv)
    rng = np.random.default_rng(H)
    lens = np.array([40, 0, 700], np.int32)
    c, cache, table = make(rng, lens, 16, Hkv, dh, kind)
    q = t(queries(rng, 3, H, dh))
    want = S.attention_scores_decode(cache, t(table), t(lens), q)
    for shift in (1, 2, 3, 5, 8):
        (o, ob), (m, mb) = slice_at(shift, (3, H, dh), torch.bfloat16), slice_at(shift, (3, H, 2), torch.float32)
        S.attention_scores_decode(cache, t(table), t(lens), q, o=o, m_heads=m)
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(m, want[1]), shift
        assert beside(ob, shift, o.numel()) and beside(mb, shift, m.numel())
