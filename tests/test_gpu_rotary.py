"""Rotary positions on the GPU against the float64 oracle.

Tolerance of a pair (x, y): the float32 angle in half turns is rounded once (pi 2^-24 radians at most), sine and
cosine are good to 2^-22, two products, a sum and the amplitude are rounded (4 2^-24): 12 2^-24 a (|x| + |y|)
covers them; bf16 results add half a step, 2^-8 of the value. The float64 angle of a position below 2^31 is good
to 2^31 3 2^-53 < 8 2^-24."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import serving as V
from paper_2604_23996_amd import smoes as S
from tests.gpu_util import DEV, host, say

pytestmark = pytest.mark.gpu


def _f64(t):
    return t.double().cpu().numpy()


def _check(spec, x, y, pos, backward=False):
    f, a = V.rotary_frequencies(spec.rot_dim, spec.scaling, spec.base, spec.factor, spec.original_len, spec.beta_fast,
                                spec.beta_slow)
    X = _f64(x)
    ref = V.rotary(X, pos, f, a, spec.rot_dim, spec.layout, backward)
    r = spec.rot_dim
    i, j = (slice(0, r // 2), slice(r // 2, r)) if spec.layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    size = np.zeros(X.shape)
    size[..., i] = size[..., j] = a * (np.abs(X[..., i]) + np.abs(X[..., j]))
    far = 8 * 2.0 ** -24 if np.abs(np.asarray(pos)).max(initial=0) > 2 ** 27 else 0.0
    tol = (12 * 2.0 ** -24 + far) * size
    if y.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    tol[..., r:] = 0.0
    assert np.all(np.abs(_f64(y) - ref) <= tol), np.max(np.abs(_f64(y) - ref) - tol)


CASES = [  # T, H, Hkv, head_dim, rot_dim, layout, scaling, dtype
    (1, 16, 16, 128, 128, "half", "none", torch.bfloat16),
    (5, 32, 8, 128, 128, "interleaved", "by_parts", torch.bfloat16),
    (67, 4, 1, 64, 32, "half", "linear", torch.float32),
    (33, 5, 5, 64, 64, "interleaved", "ntk", torch.float32),
    (130, 3, 1, 80, 34, "half", "none", torch.bfloat16),        # pairs that no 16-byte piece divides
    (19, 2, 2, 80, 34, "interleaved", "by_parts", torch.float32),
    (9, 1, 0, 6, 2, "half", "ntk", torch.bfloat16),
    (7, 2, 1, 512, 512, "half", "none", torch.float32),
    (12, 7, 3, 96, 48, "interleaved", "linear", torch.bfloat16),
    (300, 40, 2, 128, 64, "half", "by_parts", torch.bfloat16),
    (2, 3, 2, 512, 16, "interleaved", "none", torch.bfloat16),
    (1200, 3, 1, 128, 66, "half", "none", torch.bfloat16),      # a last piece that shares values with the one before
    (1100, 2, 1, 128, 66, "interleaved", "linear", torch.float32),
    (40, 2, 1, 20, 18, "half", "none", torch.bfloat16),         # halves and a rest shorter or little longer than a piece
    (40, 2, 1, 20, 18, "interleaved", "none", torch.float32),
    (11, 1, 1, 12, 12, "half", "none", torch.bfloat16),
    (3, 2, 2, 7, 6, "half", "none", torch.float32),
    (3, 2, 2, 31, 30, "interleaved", "none", torch.bfloat16),
    (2051, 3, 2, 64, 64, "half", "none", torch.bfloat16),        # two and more tokens of a workgroup, the last one short
    (5003, 2, 1, 128, 96, "interleaved", "ntk", torch.bfloat16),
    (17001, 1, 1, 64, 22, "half", "none", torch.float32),
    (16411, 1, 0, 8, 6, "interleaved", "linear", torch.bfloat16),
]


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_rotary(case, backward):
    T, H, Hkv, dh, r, layout, scaling, dt = case
    say("rotary", case, backward)
    g = torch.Generator().manual_seed(T + dh)
    spec = S.RotarySpec(dh, r, layout=layout, scaling=scaling, factor=1.0 if scaling == "none" else 8.0)
    plan = S.RotaryPlan(spec, DEV)
    q = torch.randn(T, H, dh, generator=g).to(dt).to(DEV)
    k = torch.randn(T, Hkv, dh, generator=g).to(dt).to(DEV) if Hkv else None
    pos = torch.randint(-5, 200000, (T,), generator=g, dtype=torch.int32)
    qo, ko = S.rotary(plan, q, k, positions=pos.to(DEV), backward=backward)
    torch.cuda.synchronize()
    _check(spec, q, qo, pos.numpy(), backward)
    if Hkv:
        _check(spec, k, ko, pos.numpy(), backward)
    else:
        assert ko is None
    # in place: the same bits, and the values behind rot_dim untouched
    q2, k2 = q.clone(), None if k is None else k.clone()
    S.rotary(plan, q2, k2, positions=pos.to(DEV), backward=backward, q_out=q2, k_out=k2)
    torch.cuda.synchronize()
    assert torch.equal(q2, qo) and (k is None or torch.equal(k2, ko))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [0, 1, 8])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_views_at_any_element(dt, shift, layout):
    # slices of a fused projection, its start and stride off the wide accesses' boundaries: the same bits
    T, H, Hkv, dh = 21, 4, 2, 64
    say("rotary views", dt, shift, layout)
    plan = S.RotaryPlan(S.RotarySpec(dh, 32, layout=layout), DEV)
    for extra in (0, 3, 8):
        width = (H + 2 * Hkv) * dh + extra
        buf = torch.randn(T * width + 16, device=DEV).to(dt)
        rows = buf[shift:shift + T * width].view(T, width)
        q = rows[:, :H * dh].unflatten(1, (H, dh))
        k = rows[:, H * dh:(H + Hkv) * dh].unflatten(1, (Hkv, dh))
        before = buf.clone()
        qd, kd = S.rotary(plan, q.contiguous(), k.contiguous())
        qv, kv = S.rotary(plan, q, k)
        S.rotary(plan, q, k, q_out=q, k_out=k)
        torch.cuda.synchronize()
        assert torch.equal(qd, qv) and torch.equal(kd, kv) and torch.equal(q, qd) and torch.equal(k, kd)
        q.copy_(before[shift:shift + T * width].view(T, width)[:, :H * dh].unflatten(1, (H, dh)))
        k.copy_(before[shift:shift + T * width].view(T, width)[:, H * dh:(H + Hkv) * dh].unflatten(1, (Hkv, dh)))
        assert torch.equal(buf, before)  # nothing beside q and k was written


def test_rotary_positions():
    # none given: the token index; far positions; T = 0
    say("rotary positions")
    spec = S.RotarySpec(64, 64)
    plan = S.RotaryPlan(spec, DEV)
    q = torch.randn(40, 2, 64, device=DEV)
    qo, _ = S.rotary(plan, q)
    _check(spec, q, qo, np.arange(40))
    far = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, 123456789] * 10, np.int64)
    qo, _ = S.rotary(plan, q, positions=torch.from_numpy(far).to(torch.int32).to(DEV))
    _check(spec, q, qo, far)
    e, _ = S.rotary(plan, q[:0])
    assert e.shape == (0, 2, 64)


def test_rotary_gradient_is_the_derivative():
    # d/dx_e <rotary(x), g> by central differences (the rotation is linear: a step of 1 loses nothing to truncation) is
    # rotary(g, backward) at e; float32 sums of 2 head_dim values below 4: 2^-24 * 16 * 4 each
    say("rotary gradient")
    T, H, dh = 3, 2, 16
    for layout in ("half", "interleaved"):
        plan = S.RotaryPlan(S.RotarySpec(dh, 8, layout=layout, scaling="by_parts", factor=4.0), DEV)
        pos = torch.tensor([5, 900, 77], dtype=torch.int32, device=DEV)
        x, g = torch.randn(T, H, dh, device=DEV), torch.randn(T, H, dh, device=DEV)
        dx, _ = S.rotary(plan, g, positions=pos, backward=True)
        for e in range(dh):
            step = torch.zeros_like(x)
            step[..., e] = 1.0
            up, _ = S.rotary(plan, x + step, positions=pos)
            dn, _ = S.rotary(plan, x - step, positions=pos)
            fd = ((up.double() - dn.double()) * g.double()).sum(-1) / 2
            assert torch.all((fd - dx[..., e].double()).abs() <= 2.0 ** -24 * 16 * 4 * 4)


def test_rotary_in_a_graph_and_on_a_side_stream():
    say("rotary graph")
    plan = S.RotaryPlan(S.RotarySpec(128, 128), DEV)
    q, k = (torch.randn(50, h, 128, device=DEV).bfloat16() for h in (8, 2))
    pos = torch.arange(50, dtype=torch.int32, device=DEV)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        S.rotary(plan, q, k, positions=pos, q_out=qo, k_out=ko)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.rotary(plan, q, k, positions=pos, q_out=qo, k_out=ko)
    for step in (0, 3, 100):
        pos.copy_(torch.arange(50, dtype=torch.int32, device=DEV) + step)
        want = S.rotary(plan, q, k, positions=pos)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
