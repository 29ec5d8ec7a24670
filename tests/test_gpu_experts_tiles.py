"""The experts' first product where a workgroup takes several tiles: tiles of 256 and of 128 rows, full ones followed
by others, whose results are still on their way when the next tile's first steps are multiplied.  (The
second product: test_gpu_experts_sums.py, value for value.)"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2510_03293_amd import binding as B
from tests import products as P
from tests import ways

pytestmark = pytest.mark.gpu

F32, BF16 = B.DTYPE_F32, B.DTYPE_BF16

# T, H, F, E, k, total, first; the way of a bf16 call
SHAPES = [
    (2600, 1160, 2184, 4, 2, 4, 0, "256"),   # steps, rows and columns with a rest
    (5120, 1152, 2048, 1, 1, 1, 0, "256"),   # none, every tile full
    (3000, 1224, 2056, 4, 2, 6, 1, "256"),   # a share of the experts
    (2600, 264, 2184, 4, 2, 4, 0, "128"),    # five steps
    (2600, 64, 2184, 4, 2, 4, 0, "128"),     # one
    (2600, 128, 2176, 4, 2, 4, 0, "128"),    # two
    (5120, 192, 2048, 1, 1, 1, 0, "128"),    # every tile full
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T%d_H%d_F%d_E%d_k%d" % s[:5])
def test_up(shape):
    T, H, F, E, k, total, first, way = shape
    rng = np.random.default_rng(70)
    ids = P.random_ids(rng, T, k, total, 0.1)
    perm, offs = P.tables(ids, total)
    assert ways.experts("up", T, H, F, E, k, False, offs, first) == way
    hidden = P.rounded(rng, (T, H), 1.0, BF16)
    w_up = P.rounded(rng, (E, 2 * F, H), 2.0 / np.sqrt(H), BF16)
    act = P.run_up(hidden, w_up, perm, offs, k, BF16, first)
    pos, want, tol = P.up_reference(hidden, w_up, perm, offs, k, first, BF16)
    got = P.f64(act)
    P.assert_within(got[pos], want, tol, f"up {shape}")
    assert (np.delete(got, pos, axis=0) == 776.0).all()
    # and again, other work in between: the same bits
    again = P.run_up(hidden, w_up, perm, offs, k, BF16, first)
    assert torch.equal(again.view(torch.int16), act.view(torch.int16))


# T, H, F; the way
GATES = [(4, 8, 16, "few"), (40, 64, 72, "64"), (300, 64, 72, "128"), (5120, 1152, 2048, "256")]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,H,F,way", GATES, ids=[g[3] for g in GATES])
def test_large_gates(T, H, F, way, dtype):
    """exp(-g) overflows for very negative gates, and very positive ones pass through, whichever way a call goes."""
    assert dtype == F32 or ways.experts("up", T, H, F, 1, 1, False, None, 0) == way
    values = np.array([1.0, 300.0, -300.0, 0.0, -30.0, 30.0, -80.0, 80.0, 1e18, -1e18])
    hidden = torch.zeros(T, H, dtype=P.TORCH[dtype])
    hidden[:, 0] = torch.from_numpy(values[np.arange(T) % len(values)]).to(P.TORCH[dtype])
    w_up = torch.zeros(1, 2 * F, H, dtype=P.TORCH[dtype])
    w_up[0, :, 0] = 1.0
    act = P.f64(P.run_up(hidden, w_up, None, None, 1, dtype))
    g = P.f64(hidden)[:, :1]
    with np.errstate(over="ignore"):
        want = P.silu(g) * g
    # (one product and zeros: g is exact; what is left is the sigmoid, as in up_reference)
    tol = ((np.abs(g) + 12) * 2 * P.U + P.HALF_STEP[dtype]) * np.abs(want) * 1.01 + 1e-30
    P.assert_within(act, np.broadcast_to(want, act.shape), np.broadcast_to(tol, act.shape), "gates")
    assert (act[2::10] == 0.0).all() and (act[9::10] == 0.0).all() and (act[3::10] == 0.0).all()
