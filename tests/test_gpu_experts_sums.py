"""The sums of the experts' second product, value for value.

Operands are small whole numbers, weights powers of two, so that every product, every partial sum in any
order and every weighted summand is a multiple of 1/2 below 2^23 and has no rounding in 32 bits.  `base`
takes nearly all of the sum away, so that out is the exact remainder rounded once to its type.  There is no
tolerance: a summand that is held in fewer than 32 bits anywhere on the way shows.
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2510_03293_amd import binding as B
from tests import products as P
from tests import ways

pytestmark = pytest.mark.gpu

F32, BF16 = B.DTYPE_F32, B.DTYPE_BF16


def whole_numbers(T, H, F, E, k, total, first, dtype, seed):
    """act, w_down, tables, weights, base, and the exact sum."""
    rng = np.random.default_rng(seed)
    ids = P.random_ids(rng, T, k, total, 0.3)
    perm, offs = P.tables(ids, total)
    act = torch.from_numpy(rng.integers(0, 8, (T * k, F)).astype(np.float32))
    w = torch.from_numpy(rng.integers(0, 8, (E, H, F)).astype(np.float32))
    weights = rng.choice([0.5, 1.0, 2.0], (T, k)).astype(np.float32)
    total_sum = torch.zeros(T, H)  # (fp32 is exact here, on the CPU as well)
    for e in range(E):
        a, b = int(offs[first + e]), int(offs[first + e + 1])
        if a == b:
            continue
        slots = perm[a:b].astype(np.int64)
        z = (act[a:b] @ w[e].T) * torch.from_numpy(weights.reshape(-1)[slots])[:, None]
        total_sum.index_add_(0, torch.from_numpy(slots // k), z)
    assert float(total_sum.abs().max()) < 2 ** 23
    base = (-total_sum).to(P.TORCH[dtype])
    left = total_sum + base.float()
    return act.to(P.TORCH[dtype]), w.to(P.TORCH[dtype]), perm, offs, ids, weights, base, left.to(P.TORCH[dtype]), total_sum


# T, H, F, E, k, total, first; the way of a bf16 and of an fp32 call
SHAPES = [
    (1, 256, 1416, 8, 2, 8, 0, "few", "few"),
    (4, 136, 1032, 5, 3, 9, 2, "few", "few"),
    (3, 72, 9000, 2, 2, 2, 0, "few", "few"),
    (300, 136, 1160, 3, 2, 3, 0, "slices", "slices"),
    (1100, 392, 1032, 1, 1, 1, 0, "slices", "slices"),
    (64, 1544, 264, 64, 6, 64, 0, "64", "64"),
    (300, 264, 328, 16, 2, 16, 0, "64", "32"),
    (300, 2056, 328, 8, 2, 32, 8, "128", "64"),
    (2000, 1032, 520, 4, 2, 4, 0, "128", "64"),
    (2600, 4360, 264, 4, 2, 4, 0, "128", "64"),   # more tiles than workgroups
    (2600, 4360, 1160, 4, 2, 4, 0, "256", "64"),  # ... of 256 rows
    (2600, 4360, 1160, 4, 2, 12, 5, "256", "64"),  # a share of the experts
    (5120, 2048, 1152, 1, 1, 1, 0, "256", "64"),  # ... all of them full
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T%d_H%d_F%d_E%d_k%d" % s[:5])
def test_sums_that_cancel_are_exact(shape, dtype):
    T, H, F, E, k, total, first = shape[:7]
    act, w, perm, offs, ids, weights, base, left, whole = whole_numbers(T, H, F, E, k, total, first, dtype, 40)
    assert ways.experts("down", T, H, F, E, k, dtype == F32, offs, first) == shape[7 if dtype == BF16 else 8]
    out = P.run_down(act, w, perm, offs, ids, weights, base, k, T, dtype, first).cpu()
    differ = int((out != left).sum())
    assert differ == 0, f"{differ} of {out.numel()} values"
    out = P.run_down(act, w, perm, offs, ids, weights, None, k, T, dtype, first).cpu()
    differ = int((out != whole.to(P.TORCH[dtype])).sum())
    assert differ == 0, f"{differ} of {out.numel()} values without a base"
