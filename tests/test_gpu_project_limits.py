"""Infinities, NaN and values near the types' limits in a row's own adapter: whichever way a call goes,
they come out as the formula gives them in fp32."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2510_03293_amd import binding as B
from tests import products as P

pytestmark = pytest.mark.gpu

F32, BF16 = B.DTYPE_F32, B.DTYPE_BF16

# T, H, N, R
SHAPES = [
    (20, 136, 64, 16),       # thin
    (1, 72, 5, 8),
    (600, 1032, 130, 24),    # slices of the contraction axis
    (700, 136, 64, 16),      # a gate in one launch, adapters of one block ...
    (700, 264, 33, 32),      # ... two
    (900, 136, 61, 56),      # ... and four
    (600, 136, 130, 16),     # tiles of 64 x 64
    (600, 1480, 600, 128),   # ... behind inner values in slices
    (2100, 136, 1100, 40),   # tiles of 128 x 128
    (4200, 136, 2056, 8),    # tiles of 256 x 256
]


def limits(T, H, N, R, dtype):
    """Rows in turn with adapters 0 .. 3; x is positive and begins with 1 in every row."""
    rng = np.random.default_rng(50)
    x = np.abs(rng.standard_normal((T, H))) + 0.1
    x[:, 0] = 1.0
    down = np.abs(rng.standard_normal((4, R, H))) / H
    down[2:, :, :] = 0.0
    down[2:, :, 0] = 1.0                     # inner values of exactly 1 ...
    down[3, 1::2, 0] = 1.0 / 3               # ... and some with more digits than one piece holds
    up = rng.standard_normal((4, N, R)) * 0.2
    sign = np.where(np.arange(N) % 2, -1.0, 1.0)[:, None]
    up[1] = (np.abs(up[1]) + 0.01) * sign    # infinite inner values of one sign: an infinity, not NaN
    up[2] = 2.0 ** -100 * sign               # inner values of 3.4e38: finite in fp32, above the largest bf16
    up[3, 0, 0] = np.inf
    up[3, 1 % N, R - 1] = -np.inf
    up[3, 2 % N, 1] = np.nan
    up[3, 3 % N, 1] = np.inf                 # two infinities of opposite signs
    up[3, 3 % N, R // 2] = -np.inf
    scales = np.array([1.0, np.inf, 3.4e38, 0.7], dtype=np.float32)
    t = P.TORCH[dtype]
    cuts = np.linspace(0, T, 13).astype(np.int32)
    which = (np.arange(12) % 4).astype(np.int32)
    return dict(x=torch.from_numpy(x.astype(np.float32)).to(t), w=P.rounded(rng, (N, H), 0.05, dtype),
                a_down=torch.from_numpy(down.astype(np.float32)).to(t), a_up=torch.from_numpy(up.astype(np.float32)).to(t),
                scales=scales, cuts=cuts, which=which)


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, F32), (BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T%d_H%d_N%d_R%d" % s)
def test_limits(shape, dtype, out_dtype):
    T, N, R = shape[0], shape[2], shape[3]
    i = limits(*shape, dtype)
    got = P.f64(P.run_project(**i, out_dtype=out_dtype, dtype=dtype))
    finite = dict(i, which=np.where(np.isin(i["which"], (0, 2)), i["which"], -1))
    with np.errstate(all="ignore"):
        want, tol = P.project_reference(**finite, out_dtype=out_dtype, dtype=dtype)
    for q, m in enumerate(i["which"]):
        a, b = int(i["cuts"][q]), int(i["cuts"][q + 1])
        if m == 1:
            assert (got[a:b] == np.where(np.arange(N) % 2, -np.inf, np.inf)).all(), "infinite inner values"
        elif m == 3:
            # (inner values are positive: an entry of up decides the sign)
            up = P.f64(i["a_up"][3])
            with np.errstate(all="ignore"):
                ends = up.sum(axis=1)
            special = ~np.isfinite(ends)
            assert np.array_equal(got[a:b][:, special], np.broadcast_to(ends[special], (b - a, special.sum())),
                                  equal_nan=True), "infinite entries of up"
            assert np.isfinite(got[a:b][:, ~special]).all()
        else:
            P.assert_within(got[a:b], want[a:b], tol[a:b], f"adapter {m}")
