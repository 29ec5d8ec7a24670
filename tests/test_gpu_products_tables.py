"""Tables with entries out of range on every way a call of the products can go: values are unspecified then, but
nothing outside the arrays is read or written, the call ends, and the arrays' neighbours are untouched."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2510_03293_amd import binding as B
from tests import products as P
from tests import ways

pytestmark = pytest.mark.gpu

F32, BF16 = B.DTYPE_F32, B.DTYPE_BF16
EDGE = 64   # rows before and behind an array


class Guarded:
    """Rows between rows of a mark, and whether the marks are still there."""

    def __init__(self, rows, columns, dtype):
        self.all = torch.full((rows + 2 * EDGE, columns), 777.0, dtype=dtype, device="cuda")
        self.mark = self.all[0, 0].item()
        self.rows = self.all[EDGE:EDGE + rows]

    def untouched(self):
        return bool((self.all[:EDGE] == self.mark).all()) and bool((self.all[EDGE + len(self.rows):] == self.mark).all())


class Workspace:
    def __init__(self, nbytes):
        self.all = torch.full((nbytes + 2048,), 77, dtype=torch.uint8, device="cuda")
        self.bytes = self.all[1024:1024 + nbytes]

    def untouched(self):
        return bool((self.all[:1024] == 77).all()) and bool((self.all[1024 + len(self.bytes):] == 77).all())


def bad_tables(rng, slots, E):
    lowest, highest = -2 ** 31, 2 ** 31 - 1
    even = np.linspace(0, slots, E + 1).astype(np.int32)
    straight = np.arange(slots, dtype=np.int32)
    wild = rng.choice(np.array([0, -1, 7, slots, slots - 1, slots // 2, highest, lowest, -5], dtype=np.int64), E + 1)
    yield rng.integers(lowest, highest, slots).astype(np.int32), even          # slots out of range
    yield np.zeros(slots, dtype=np.int32), even                               # one slot for all positions
    yield straight, even[::-1].copy()                                         # descending
    yield straight, wild.astype(np.int32)                                     # anything
    yield straight, np.array([0, highest] * E, dtype=np.int32)[:E + 1]        # every other expert has all rows


# T, H, F, E, k; the ways of up and of down (bf16; with tables in order)
EXPERTS = [
    (3, 520, 520, 5, 4, "few", "few"),
    (40, 136, 136, 5, 2, "64", "64"),
    (70, 136, 1544, 4, 2, "64", "slices"),
    (300, 136, 136, 4, 2, "128", "128"),
    (700, 1160, 1160, 2, 2, "128", "slices"),
    (2600, 1160, 2184, 4, 2, "256", "128"),
    (2600, 4360, 1160, 4, 2, "256", "256"),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", EXPERTS, ids=lambda s: "T%d_H%d_F%d_E%d_k%d" % s[:5])
def test_dispatch_tables(shape, dtype):
    T, H, F, E, k, up_way, down_way = shape
    rng = np.random.default_rng(80)
    order = np.linspace(0, T * k, E + 1).astype(np.int32)
    if dtype == BF16:
        assert ways.experts("up", T, H, F, E, k, False, order, 0) == up_way
        assert ways.experts("down", T, H, F, E, k, False, order, 0) == down_way
    g = torch.Generator(device="cuda")
    g.manual_seed(80)

    def normal(*shape, std=1.0):
        return torch.empty(*shape, dtype=P.TORCH[dtype], device="cuda").normal_(0, std, generator=g)

    hidden, w_up, w_down, act = normal(T, H), normal(E, 2 * F, H, std=0.05), normal(E, H, F, std=0.05), normal(T * k, F)
    weights = torch.rand(T, k, generator=g, device="cuda")
    ids = torch.randint(-3, E + 3, (T, k), generator=g, device="cuda", dtype=torch.int32)
    params = B.make_experts_params(k, dtype=dtype)
    for perm, offs in bad_tables(rng, T * k, E):
        p, o = torch.from_numpy(perm).cuda(), torch.from_numpy(offs).cuda()
        up, out = Guarded(T * k, F, P.TORCH[dtype]), Guarded(T, H, P.TORCH[dtype])
        ws = Workspace(B.laser_experts_workspace_bytes(T, H, F, E, params))
        B.laser_experts_up(hidden, w_up, T, H, F, E, params, p, o, up.rows)
        torch.cuda.synchronize()
        B.laser_experts_down(act, w_down, T, H, F, E, params, p, o, ids, weights, None, out.rows, ws.bytes)
        torch.cuda.synchronize()
        assert up.untouched() and out.untouched() and ws.untouched()


# T, H, N, R, requests; the way
PROJECTIONS = [
    (100, 136, 64, 16, 3, "thin"),
    (100, 136, 64, 16, 300, "thin"),
    (700, 1032, 130, 24, 200, "slices"),
    (1500, 136, 64, 16, 20, "gate"),
    (9000, 72, 33, 40, 130, "gate"),
    (700, 136, 130, 16, 3, "64"),
    (700, 136, 64, 16, 1000, "64"),
    (2100, 136, 1100, 128, 70, "128"),
    (4200, 136, 2056, 8, 700, "256"),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", PROJECTIONS, ids=lambda s: "T%d_H%d_N%d_R%d_q%d" % s[:5])
def test_request_tables(shape, dtype):
    T, H, N, R, requests, way = shape
    M = 3
    assert dtype == F32 or ways.project(T, H, N, R, requests, False) == way
    rng = np.random.default_rng(81)
    g = torch.Generator(device="cuda")
    g.manual_seed(81)

    def normal(*shape, std=1.0):
        return torch.empty(*shape, dtype=P.TORCH[dtype], device="cuda").normal_(0, std, generator=g)

    x, w, down, up = normal(T, H), normal(N, H, std=0.05), normal(M, R, H, std=0.1), normal(M, N, R, std=0.1)
    scales = torch.rand(M, generator=g, device="cuda")
    params = B.make_adapter_params(R, M, requests, dtype=dtype)
    lowest, highest = -2 ** 31, 2 ** 31 - 1
    order = np.linspace(0, T, requests + 1).astype(np.int64)
    cuts = [order[::-1], rng.integers(lowest, highest, requests + 1),
            rng.choice(np.array([0, 1, -1, T, T + 1, highest, lowest, T // 2]), requests + 1), order * 3 - T,
            np.full(requests + 1, lowest), np.full(requests + 1, highest)]
    which = [rng.choice(np.array([0, 1, 2, -1, 3, highest, lowest]), requests), np.full(requests, highest)]
    for i, c in enumerate(cuts):
        q, m = (torch.from_numpy(np.ascontiguousarray(t).astype(np.int32)).cuda() for t in (c, which[i % 2]))
        out = Guarded(T, N, P.TORCH[dtype])
        ws = Workspace(B.laser_project_workspace_bytes(T, H, N, params))
        B.laser_project_adapted(x, w, T, H, N, params, down, up, scales, q, m, out.rows, ws.bytes)
        torch.cuda.synchronize()
        assert out.untouched() and ws.untouched() and bool(torch.isfinite(out.rows).all())
