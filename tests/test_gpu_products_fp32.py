"""fp32 products: how long the chains of roundings are.

One product of 2^26 comes first, 2^-1 each behind it.  At 2^26 a step is 8, so that a chain which adds the small
ones one by one, or four by four, loses every one of them.  Bound: 32 products, a step of a tile, are summed by
themselves (at most 32 roundings), the steps' sums one after the other (n / 32), and what cuts the axis adds at
most 16 slices, a weight and a base (18); each is off by at most 2^-24 of a sum no larger than that of the
magnitudes.  (Wavefronts that take shares of the axis have shorter chains yet: 80 products of a thin
call, 32 of a few tokens, half a step of a gate.)
"""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2510_03293_amd import binding as B
from tests import products as P
from tests import ways

pytestmark = pytest.mark.gpu

F32 = B.DTYPE_F32
N = 2052            # (no multiple of a step, so that the rows are walked from their beginning)
SUM = 2.0 ** 26 + (N - 1) / 2
TOL = (32 + N / 32 + 18) * P.U * SUM


def rows(n):
    x = torch.ones(n, N)
    x[:, 0] = 2.0 ** 13
    return x


def weights(*shape):
    w = torch.full((*shape, N), 0.5)
    w[..., 0] = 2.0 ** 13
    return w


@pytest.mark.parametrize("T,H,E,k,way", [(3, 72, 2, 1, "few"), (40, 136, 2, 1, "slices"), (150, 1024, 16, 2, "32"),
                                         (150, 2048, 16, 2, "64")])
def test_down(T, H, E, k, way):
    ids = P.random_ids(np.random.default_rng(1), T, k, E)
    perm, offs = P.tables(ids, E)
    assert ways.experts("down", T, H, N, E, k, True, offs, 0) == way
    out = P.f64(P.run_down(rows(T * k), weights(E, H), perm, offs, ids, None, None, k, T, F32))
    P.assert_within(out, np.full((T, H), k * SUM), np.full((T, H), k * (TOL + P.U * k * SUM)), way)


@pytest.mark.parametrize("T,F,E,way", [(3, 72, 2, "few"), (40, 136, 2, "32"), (300, 1024, 16, "64")])
def test_up(T, F, E, way):
    ids = P.random_ids(np.random.default_rng(2), T, 1, E)
    perm, offs = P.tables(ids, E)
    assert ways.experts("up", T, N, F, E, 1, True, offs, 0) == way
    w = weights(E, 2 * F)
    w[:, :F] = 0.0
    w[:, :F, 1] = 8.0                          # the gate is exactly 8
    act = P.f64(P.run_up(rows(T), w, perm, offs, 1, F32))
    gate = P.silu(8.0)
    tol = gate * TOL + (8 + 12) * 2 * P.U * gate * SUM + P.U * gate * SUM
    P.assert_within(act, np.full((T, F), gate * SUM), np.full((T, F), tol), way)


@pytest.mark.parametrize("T,columns,way", [(20, 64, "thin"), (700, 130, "slices"), (9000, 33, "gate"), (2100, 1100, "64")])
def test_project(T, columns, way):
    assert ways.project(T, N, columns, 8, 0, True) == way
    out = P.f64(P.run_project(rows(T), weights(columns), None, None, None, None, np.zeros(0, np.int32), F32, F32))
    P.assert_within(out, np.full((T, columns), SUM), np.full((T, columns), TOL), way)
