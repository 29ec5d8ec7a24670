"""The ends of the products' size ranges: rows of one load, one row against very many columns, more slots than 2^24,
empty calls."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2510_03293_amd import binding as B
from tests import products as P
from tests import ways

pytestmark = pytest.mark.gpu

F32, BF16 = B.DTYPE_F32, B.DTYPE_BF16


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,H,F,E,k", [(700, 8, 8, 3, 2), (5, 8, 8, 64, 16), (40, 8, 4000, 9, 1), (5000, 4000, 8, 2, 1),
                                       (5000, 8, 4000, 2, 1), (5, 16, 16, 1, 1), (1, 8, 70000, 2, 2), (1, 8000, 8, 2, 2)])
def test_short_rows_of_the_experts(T, H, F, E, k, dtype):
    rng = np.random.default_rng(100)
    ids = P.random_ids(rng, T, k, E)
    perm, offs = P.tables(ids, E)
    hidden, w_up = P.rounded(rng, (T, H), 1.0, dtype), P.rounded(rng, (E, 2 * F, H), 1.0 / np.sqrt(H), dtype)
    act = P.run_up(hidden, w_up, perm, offs, k, dtype)
    pos, want, tol = P.up_reference(hidden, w_up, perm, offs, k, 0, dtype)
    P.assert_within(P.f64(act)[pos], want, tol, "up")
    a, w_down = P.rounded(rng, (T * k, F), 1.0, dtype), P.rounded(rng, (E, H, F), 1.0 / np.sqrt(F), dtype)
    weights = rng.random((T, k)).astype(np.float32)
    out = P.run_down(a, w_down, perm, offs, ids, weights, None, k, T, dtype)
    want, tol = P.down_reference(a, w_down, perm, offs, ids, weights, None, k, 0, T, dtype)
    P.assert_within(P.f64(out), want, tol, "down")


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, F32), (BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("T,H,N,R,lengths", [(1, 72, 70001, 8, [1]), (5, 264, 20000, 16, [1, 3]), (1, 8, 65536, 8, [1]),
                                             (65, 8, 2000, 128, [30, 35]), (3000, 8, 1, 8, [2999]), (513, 136, 129, 8, [1] * 513)])
def test_few_rows_or_columns_of_a_projection(T, H, N, R, lengths, dtype, out_dtype):
    rng = np.random.default_rng(101)
    M = 3
    cuts = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    which = rng.integers(-1, M, len(lengths)).astype(np.int32)
    which[0] = 1
    given = dict(x=P.rounded(rng, (T, H), 1.0, dtype), w=P.rounded(rng, (N, H), 0.05, dtype),
                 a_down=P.rounded(rng, (M, R, H), 1 / np.sqrt(H), dtype), a_up=P.rounded(rng, (M, N, R), 0.2, dtype),
                 scales=(rng.random(M) * 2).astype(np.float32), cuts=cuts, which=which, out_dtype=out_dtype, dtype=dtype)
    want, tol = P.project_reference(**given)
    P.assert_within(P.f64(P.run_project(**given)), want, tol, "projection")


def test_more_slots_than_24_bits():
    """17.6 million slots: positions are kept apart by another rule there, and summands lie beyond 2^29 bytes."""
    T, H, F, E, k = 1_100_000, 8, 8, 64, 16
    assert T * k > 1 << 24
    g = torch.Generator(device="cuda")
    g.manual_seed(102)
    ids = torch.rand(T, E, generator=g, device="cuda").topk(k, dim=1)[1].int()
    flat = ids.reshape(-1)
    perm = torch.sort(flat, stable=True)[1].int()
    offs = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offs[1:] = torch.cumsum(torch.bincount(flat, minlength=E), 0).int()
    hidden = torch.empty(T, H, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    w_up = torch.empty(E, 2 * F, H, dtype=torch.bfloat16, device="cuda").normal_(0, 0.5, generator=g)
    w_down = torch.empty(E, H, F, dtype=torch.bfloat16, device="cuda").normal_(0, 0.5, generator=g)
    weights = torch.rand(T, k, generator=g, device="cuda")
    params = B.make_experts_params(k)
    assert ways.experts("up", T, H, F, E, k, False, offs.cpu().numpy(), 0) == "128"
    act = torch.full((T * k, F), 777.0, dtype=torch.bfloat16, device="cuda")
    B.laser_experts_up(hidden, w_up, T, H, F, E, params, perm, offs, act)
    ws = torch.empty(B.laser_experts_workspace_bytes(T, H, F, E, params), dtype=torch.uint8, device="cuda")
    out = torch.full((T, H), 777.0, dtype=torch.bfloat16, device="cuda")
    B.laser_experts_down(act, w_down, T, H, F, E, params, perm, offs, ids, weights, hidden, out, ws)
    torch.cuda.synchronize()
    # every row near, by the plain form in fp32, some to the bound
    at = torch.empty(T * k, dtype=torch.long, device="cuda")
    at[perm.long()] = torch.arange(T * k, device="cuda")
    for e in range(E):
        a, b = int(offs[e]), int(offs[e + 1])
        z = hidden[(perm[a:b] // k).long()].float() @ w_up[e].float().t()
        want = z[:, :F] * torch.sigmoid(z[:, :F]) * z[:, F:]
        assert bool(((act[a:b].float() - want).abs() <= 2.0 ** -7 * want.abs() + 1e-4).all())
    some = torch.cat([torch.arange(300, device="cuda"), torch.randint(0, T, (300,), generator=g, device="cuda"),
                      torch.arange(T - 300, T, device="cuda")])
    n = len(some)
    mine = ids[some].cpu().numpy()
    p2, o2 = P.tables(mine, E)
    rows = act[at[(some[:, None] * k + torch.arange(k, device="cuda")).reshape(-1)]].cpu()[p2.astype(np.int64)]
    want, tol = P.down_reference(rows, w_down, p2, o2, mine, weights[some].cpu().numpy(), hidden[some], k, 0, n, BF16)
    P.assert_within(P.f64(out[some]), want, tol, "some rows")


def test_empty_calls_on_another_stream():
    side = torch.cuda.Stream()

    def ones(*shape, dtype=torch.bfloat16):
        return torch.ones(*shape, dtype=dtype, device="cuda")

    layer = B.experts(ones(0, 64), ones(1, 32, 64), ones(1, 64, 16), None, stream=side)
    assert layer.out.shape == (0, 64)
    bare = (ones(0, 8, 64), ones(0, 5, 8), None, 0 * ones(1, dtype=torch.int32), ones(0, dtype=torch.int32))
    x, w = ones(3, 64), ones(5, 64)
    torch.cuda.synchronize()
    assert B.project_adapted(x[:0], w, *bare, stream=side).shape == (0, 5)
    out = B.project_adapted(x, w, *bare, stream=side)
    side.synchronize()
    assert bool((out == 64.0).all())
