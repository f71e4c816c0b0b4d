"""The angle of a rotation keeps its float64 bits: near a zero of the sine or the cosine, rounding it to float32 would be the
whole error."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import serving as V
from paper_2604_23996_amd import smoes as S
from tests.gpu_util import DEV, host, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_small_sines_and_cosines(layout, backward):
    # Pairs (1, 0) give the cosine and the sine themselves. Positions where one of the first pair's (frequency 1) is below
    # 1e-4: its error is that of sine and cosine of the float32 part of the angle (4 units of 2^-24 of the value), of the
    # remainder's products and sum (3 more) and of the float64 angle, 2 pi * 2^22 turns * 3 * 2^-53 < 2^-26 (position / 2 pi
    # below 2^22). Rounded to float32 the angle alone would be off by up to pi 2^-25.
    say("rotary angles", layout, backward)
    p = np.arange(1, 2 ** 24, dtype=np.float64)
    near = p[np.minimum(np.abs(np.sin(p)), np.abs(np.cos(p))) < 1e-4].astype(np.int64)
    near = np.concatenate([near, -near])
    assert len(near) > 1000
    plan = S.RotaryPlan(S.RotarySpec(4, 4, layout=layout), DEV)
    x = torch.zeros(len(near), 1, 4, device=DEV)
    x[:, :, 0] = 1.0
    y, _ = S.rotary(plan, x, positions=torch.from_numpy(near).to(torch.int32).to(DEV), backward=backward)
    torch.cuda.synchronize()
    f, _ = V.rotary_frequencies(4, "none", 10000.0, 1.0, 0, 0, 0)
    ref = V.rotary(x.double().cpu().numpy(), near, f, 1.0, 4, layout, backward)
    err = np.abs(host(y) - ref)[:, 0]
    tol = 7 * 2.0 ** -24 * np.abs(ref[:, 0]) + 2.0 ** -26
    small = np.abs(ref[:, 0]) < 1e-4
    assert (small & (ref[:, 0] != 0)).sum() >= len(near)
    assert np.all(err[small] <= tol[small]), (np.max(err[small]), (err > tol).mean())
