"""The experts' products over the dispatch tables against their definition in 64 bits."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2510_03293_amd import binding as B
from tests import products as P

pytestmark = pytest.mark.gpu

F32, BF16 = B.DTYPE_F32, B.DTYPE_BF16

# T, H, F, E, k, total, first, skew
SHAPES = [
    (1, 8, 8, 1, 1, 1, 0, 0.0),            # the smallest there is
    (1, 2048, 1408, 64, 6, 64, 0, 1.1),    # a single token
    (1, 256, 264, 8, 2, 8, 0, 0.0),
    (2, 136, 72, 3, 3, 3, 0, 0.0),         # rows that end inside a step
    (3, 64, 40, 64, 16, 64, 0, 0.0),       # more experts than a token reaches
    (17, 128, 128, 1, 1, 1, 0, 0.0),       # one row more than a block
    (64, 512, 200, 64, 6, 64, 0, 1.1),
    (65, 520, 104, 8, 2, 8, 0, 0.3),
    (100, 72, 1000, 33, 3, 33, 0, 0.0),
    (129, 192, 136, 2, 1, 2, 0, 3.0),
    (257, 328, 248, 5, 2, 5, 0, 2.0),      # an expert that takes nearly everything
    (300, 256, 64, 16, 6, 64, 16, 1.1),    # a share of the experts
    (300, 256, 64, 3, 2, 64, 61, 1.1),     # ... the last ones, hardly any row
    (1000, 136, 264, 7, 4, 9, 2, 0.5),
    (1500, 320, 392, 6, 3, 6, 0, 0.3),
    (2600, 256, 272, 4, 2, 4, 0, 0.1),     # hundreds of rows per expert
    (4, 312, 288, 13, 3, 21, 4, 0.0),      # the most tokens that go one by one, a share of the experts
    (4, 64, 3000, 40, 16, 40, 0, 0.5),     # ... and the most slots
    (5, 1032, 520, 4, 4, 4, 0, 0.0),
    (1400, 1160, 136, 4, 2, 4, 0, 0.3),    # the widest tiles: rows of many steps, with a rest ...
    (700, 136, 1208, 3, 2, 3, 0, 0.0),
    (900, 1152, 1216, 2, 1, 2, 0, 1.0),    # ... and without
    (1000, 1216, 1152, 4, 4, 32, 8, 0.0),  # a share with fewer rows than the tables hold for as many experts
    (515, 2048, 1280, 1, 1, 1, 0, 0.0),
    (3, 72, 2504, 21, 8, 24, 2, 0.0),      # few tokens whose rows are short and many
    (2, 2088, 72, 30, 9, 30, 0, 0.0),
]


def _case(T, H, F, E, k, total, first, skew, dtype, seed=0):
    rng = np.random.default_rng(1000 + seed)
    ids = P.random_ids(rng, T, k, total, skew)
    perm, offs = P.tables(ids, total)
    hidden = P.rounded(rng, (T, H), 1.0, dtype)
    w_up = P.rounded(rng, (E, 2 * F, H), 2.0 / np.sqrt(H), dtype)
    return rng, ids, perm, offs, hidden, w_up


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T%d_H%d_F%d_E%d_k%d" % s[:5])
def test_up(shape, dtype):
    T, H, F, E, k, total, first, skew = shape
    _, ids, perm, offs, hidden, w_up = _case(*shape, dtype)
    act = P.run_up(hidden, w_up, perm, offs, k, dtype, first)
    pos, want, tol = P.up_reference(hidden, w_up, perm, offs, k, first, dtype)
    P.assert_within(P.f64(act)[pos], want, tol, f"up {shape}")
    others = np.setdiff1d(np.arange(T * k), pos)
    assert (P.f64(act)[others] == 777.0 if dtype == F32 else P.f64(act)[others] == 776.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "T%d_H%d_F%d_E%d_k%d" % s[:5])
def test_down(shape, dtype):
    T, H, F, E, k, total, first, skew = shape
    rng, ids, perm, offs, _, _ = _case(*shape, dtype)
    act = P.rounded(rng, (T * k, F), 1.0, dtype)
    w_down = P.rounded(rng, (E, H, F), 1.0 / np.sqrt(F), dtype)
    weights = rng.random((T, k)).astype(np.float32)
    for base in (None, P.rounded(rng, (T, H), 1.0, dtype)):
        out = P.run_down(act, w_down, perm, offs, ids, weights, base, k, T, dtype, first)
        want, tol = P.down_reference(act, w_down, perm, offs, ids, weights, base, k, first, T, dtype)
        P.assert_within(P.f64(out), want, tol, f"down {shape}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [
    (69, 248, 2760, 5, 1, 5, 0, 0.3),
    (5, 72, 8200, 2, 2, 2, 0, 0.0),
    (40, 264, 1544, 6, 3, 24, 12, 0.5),     # a share of the experts
    (333, 136, 1032, 3, 2, 3, 0, 2.0),      # an expert that takes nearly everything
    (6, 8, 4096, 64, 16, 64, 0, 0.0),       # steps without a rest
    (700, 264, 1160, 1, 1, 1, 0, 0.0),
], ids=lambda s: "T%d_H%d_F%d_E%d_k%d" % s[:5])
def test_down_in_slices(shape, dtype):
    """Few rows and a long way along the contraction axis."""
    test_down(shape, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [
    (2600, 1032, 1160, 4, 2, 4, 0, 0.1),    # the widest tiles
    (1500, 1032, 1160, 12, 1, 12, 0, 0.0),  # tiles for which those would be too few
], ids=lambda s: "T%d_H%d_F%d_E%d_k%d" % s[:5])
def test_down_in_tiles(shape, dtype):
    """Rows enough not to go in slices, of many steps."""
    test_down(shape, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_expert_for_every_token(dtype):
    """Without tables: a shared expert; its output is the base of the routed ones, in place."""
    rng = np.random.default_rng(7)
    T, H, F, E, k = 77, 264, 136, 8, 2
    hidden = P.rounded(rng, (T, H), 1.0, dtype)
    w_up, w_down = P.rounded(rng, (1, 2 * F, H), 0.1, dtype), P.rounded(rng, (1, H, F), 0.1, dtype)
    one, offs1 = np.arange(T, dtype=np.int32), np.array([0, T], dtype=np.int32)
    act = P.run_up(hidden, w_up, None, None, 1, dtype)
    pos, want, tol = P.up_reference(hidden, w_up, one, offs1, 1, 0, dtype)
    P.assert_within(P.f64(act), want, tol, "shared up")
    shared = P.run_down(act, w_down, None, None, None, None, hidden, 1, T, dtype)
    want, tol = P.down_reference(act, w_down, one, offs1, None, None, hidden, 1, 0, T, dtype)
    P.assert_within(P.f64(shared), want, tol, "shared down")
    ids = P.random_ids(rng, T, k, E)
    perm, offs = P.tables(ids, E)
    act2 = P.rounded(rng, (T * k, F), 1.0, dtype)
    w2 = P.rounded(rng, (E, H, F), 0.1, dtype)
    weights = rng.random((T, k)).astype(np.float32)
    base = shared.clone().cpu()
    out = P.run_down(act2, w2, perm, offs, ids, weights, shared, k, T, dtype, in_place=True)
    want, tol = P.down_reference(act2, w2, perm, offs, ids, weights, base, k, 0, T, dtype)
    P.assert_within(P.f64(out), want, tol, "in place")


@pytest.mark.parametrize("T,H,F,E,k", [(40, 72, 40, 6, 2), (700, 200, 136, 3, 2), (1, 136, 72, 4, 2)])
def test_what_does_not_belong_to_a_row_does_not_reach_it(T, H, F, E, k):
    """Infinities and NaN in other tokens' rows, in an expert without rows and in the weights of
    slots of other GPUs: the rest comes out bit for bit as without them."""
    rng, ids, perm, offs, hidden, w_up = _case(T, H, F, E, k, E, 0, 0.0, BF16, seed=3)
    empty = E - 1
    ids = np.where(ids == empty, (ids.max(axis=1, keepdims=True) + 1) % E, ids)
    ids = P.random_ids(rng, T, k, E - 1)                      # nobody takes the last expert
    perm, offs = P.tables(ids, E)
    clean = P.run_up(hidden, w_up, perm, offs, k, BF16)
    bad_h, bad_w = hidden.clone(), w_up.clone()
    bad_w[empty] = float("nan")
    hit = T // 2 if T > 1 else None
    if hit is not None:
        bad_h[hit] = float("inf")
    act = P.run_up(bad_h, bad_w, perm, offs, k, BF16)
    keep = np.array([p for p in range(T * k) if perm[p] // k != hit])
    assert torch.equal(act.cpu()[keep].view(torch.int16), clean.cpu()[keep].view(torch.int16))

    w_down = P.rounded(rng, (E, H, F), 0.2, BF16)
    weights = rng.random((T, k)).astype(np.float32)
    a = P.rounded(rng, (T * k, F), 1.0, BF16)
    clean = P.run_down(a, w_down, perm, offs, ids, weights, None, k, T, BF16)
    bad_a, bad_w = a.clone(), w_down.clone()
    bad_w[empty] = float("nan")
    if hit is not None:
        bad_a[np.nonzero(perm // k == hit)[0]] = float("nan")
    out = P.run_down(bad_a, bad_w, perm, offs, ids, weights, None, k, T, BF16)
    keep = np.array([t for t in range(T) if t != hit])
    assert torch.equal(out.cpu()[keep].view(torch.int16), clean.cpu()[keep].view(torch.int16))
    # only the first two experts are here: the others' weights are not looked at
    share_w = weights.copy()
    share_w[ids >= 2] = np.nan
    got = P.run_down(a, w_down[:2], perm, offs, ids, share_w, None, k, T, BF16)
    want, tol = P.down_reference(a, w_down[:2], perm, offs, ids, weights, None, k, 0, T, BF16)
    P.assert_within(P.f64(got), want, tol, "share")


def test_large_gates():
    """exp(-g) overflows for very negative gates; very positive ones pass through."""
    H, F, T = 8, 16, 4
    hidden = torch.zeros(T, H, dtype=torch.bfloat16)
    hidden[:, 0] = torch.tensor([1.0, 300.0, -300.0, 0.0])
    w_up = torch.zeros(1, 2 * F, H, dtype=torch.bfloat16)
    w_up[0, :F, 0] = 1.0
    w_up[0, F:, 0] = 1.0
    act = P.f64(P.run_up(hidden, w_up, None, None, 1, BF16))
    assert np.all(act[1] == 90112.0)                          # 300 * 300 = 90000, a step is 512
    assert np.all(act[2] == 0.0) and np.all(act[3] == 0.0)
    w32, h32 = w_up.float(), hidden.float()
    act = P.f64(P.run_up(h32, w32, None, None, 1, F32))
    assert np.all(act[1] == 90000.0) and np.all(act[2] == 0.0) and np.all(act[3] == 0.0)


def test_tables_out_of_range_stay_inside_the_arrays():
    """Whatever the tables hold, nothing outside the arrays is read or written: entries are
    brought into range before they are used, so the call ends and its neighbours are untouched."""
    T, H, F, E, k = 70, 64, 64, 4, 2
    rng = np.random.default_rng(5)
    hidden, w_up = P.rounded(rng, (T, H), 1.0, BF16), P.rounded(rng, (E, 2 * F, H), 0.2, BF16)
    w_down = P.rounded(rng, (E, H, F), 0.2, BF16)
    weights = rng.random((T, k)).astype(np.float32)
    ids = P.random_ids(rng, T, k, E)
    for perm, offs in ((rng.integers(-2**31, 2**31, T * k).astype(np.int32), np.array([0, 30, 60, 100, T * k], np.int32)),
                       (np.arange(T * k, dtype=np.int32), np.array([-5, 2**31 - 1, 7, -2**31, 2**31 - 1], np.int32)),
                       (np.arange(T * k, dtype=np.int32), np.array([140, 100, 60, 30, 0], np.int32))):
        guard = torch.full((T * k + 64, F), 777.0, dtype=torch.bfloat16, device="cuda")
        params = B.make_experts_params(k)
        dev = [torch.from_numpy(t).cuda() for t in (perm, offs, ids, weights)]
        B.laser_experts_up(hidden.cuda(), w_up.cuda(), T, H, F, E, params, dev[0], dev[1], guard[32:])
        out = torch.full((T + 64, H), 777.0, dtype=torch.bfloat16, device="cuda")
        ws = torch.zeros(B.laser_experts_workspace_bytes(T, H, F, E, params), dtype=torch.uint8, device="cuda")
        B.laser_experts_down(guard[32:], w_down.cuda(), T, H, F, E, params, *dev, None, out[32:], ws)
        torch.cuda.synchronize()
        assert (guard[:32] == 776.0).all() and (guard[32 + T * k:] == 776.0).all()
        assert (out[:32] == 776.0).all() and (out[32 + T:] == 776.0).all()


def test_rows_beyond_four_gigabytes():
    """Byte offsets of hidden and act beyond 2^32."""
    T, H, F, E = 300_000, 8192, 8, 1
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    hidden = torch.empty(T, H, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    w_up = torch.empty(1, 2 * F, H, dtype=torch.bfloat16, device="cuda").normal_(0, 0.02, generator=g)
    act = torch.full((T, F), 777.0, dtype=torch.bfloat16, device="cuda")
    perm = torch.arange(T - 1, -1, -1, dtype=torch.int32, device="cuda")
    offs = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    B.laser_experts_up(hidden, w_up, T, H, F, E, B.make_experts_params(1), perm, offs, act)
    some = np.array([0, 1, 63, 64, 1000, 37_856, 37_857, 150_000, T - 2, T - 1])
    rows = hidden[torch.from_numpy(T - 1 - some).cuda()].cpu()
    pos, want, tol = P.up_reference(rows, w_up, np.arange(len(some)), np.array([0, len(some)]), 1, 0, BF16)
    P.assert_within(P.f64(act[torch.from_numpy(some).cuda()]), want, tol, "far rows")
    del hidden
    F = 8192
    far = torch.empty(T, F, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    w_down = torch.empty(1, 8, F, dtype=torch.bfloat16, device="cuda").normal_(0, 0.02, generator=g)
    params = B.make_experts_params(1)
    ws = torch.empty(B.laser_experts_workspace_bytes(T, 8, F, 1, params), dtype=torch.uint8, device="cuda")
    out = torch.full((T, 8), 777.0, dtype=torch.bfloat16, device="cuda")
    B.laser_experts_down(far, w_down, T, 8, F, 1, params, perm, offs, None, None, None, out, ws)
    want, tol = P.down_reference(far[torch.from_numpy(some).cuda()], w_down, np.arange(len(some), dtype=np.int32),
                                 np.array([0, len(some)]), None, None, None, 1, 0, len(some), BF16)
    P.assert_within(P.f64(out[torch.from_numpy(T - 1 - some).cuda()]), want, tol, "far act")


def _layer(T, H, F, E, k, seed, dtype=BF16):
    """A routed layer: gate logits routed by the library, then both products."""
    rng = np.random.default_rng(seed)
    hidden = P.rounded(rng, (T, H), 1.0, dtype).cuda()
    w_gate = P.rounded(rng, (E, H), 0.05, dtype).cuda()
    w_up = P.rounded(rng, (E, 2 * F, H), 0.05, dtype).cuda()
    w_down = P.rounded(rng, (E, H, F), 0.05, dtype).cuda()
    return hidden, w_gate, w_up, w_down, B.make_params(k, min(k + 2, E), 0.4, 0.8, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1, 64, 500])
def test_behind_the_routing_call(T, dtype):
    H, F, E, k = 256, 136, 16, 4
    hidden, w_gate, w_up, w_down, params = _layer(T, H, F, E, k, 11, dtype)
    loads = torch.zeros(E, dtype=torch.int32, device="cuda")
    routed = B.route(hidden, w_gate, params, loads)
    layer = B.experts(hidden, w_up, w_down, routed, base=hidden)
    torch.cuda.synchronize()
    perm, offs, ids = (t.cpu().numpy() for t in (routed.permutation, routed.expert_offsets, routed.expert_ids))
    pos, act, tol = P.up_reference(hidden, w_up, perm, offs, k, 0, dtype)
    P.assert_within(P.f64(layer.act), act, tol, "layer up")
    want, tol = P.down_reference(layer.act, w_down, perm, offs, ids, routed.weights.cpu().numpy(), hidden, k, 0, T,
                                 dtype)
    P.assert_within(P.f64(layer.out), want, tol, "layer down")


def test_shares_of_the_experts_add_up():
    """Four GPUs with a quarter of the experts each: the sum of their outputs is the layer's."""
    T, H, F, E, k = 150, 128, 72, 16, 3
    hidden, w_gate, w_up, w_down, params = _layer(T, H, F, E, k, 12, F32)
    routed = B.route(hidden, w_gate, params, torch.zeros(E, dtype=torch.int32, device="cuda"))
    whole = B.experts(hidden, w_up, w_down, routed)
    total = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    for first in range(0, E, 4):
        part = B.experts(hidden, w_up[first:first + 4], w_down[first:first + 4], routed, first_expert=first)
        total += part.out.double()
    perm, offs, ids = (t.cpu().numpy() for t in (routed.permutation, routed.expert_offsets, routed.expert_ids))
    want, tol = P.down_reference(whole.act, w_down, perm, offs, ids, routed.weights.cpu().numpy(), None, k, 0, T, F32)
    P.assert_within(P.f64(whole.out), want, tol, "whole")
    # (the shares are rounded once more each: at most four roundings of no more than the terms' magnitudes)
    P.assert_within(P.f64(total), want, 4 * tol, "sum of shares")


def test_calls_replayed_from_a_graph_and_other_streams():
    """route -> up -> down captured once and replayed on new inputs, eager work in between;
    then the same on a stream of its own; every run as the eager one, bit for bit."""
    T, H, F, E, k = 96, 256, 200, 16, 4
    hidden, w_gate, w_up, w_down, params = _layer(T, H, F, E, k, 13)
    loads = torch.zeros(E, dtype=torch.int32, device="cuda")
    routed = B.RouteBuffers(T, H, E, params)
    layer = B.ExpertBuffers(T, H, F, E, k, hidden.dtype)

    def step():
        loads.zero_()
        B.route(hidden, w_gate, params, loads, routed)
        B.experts(hidden, w_up, w_down, routed, base=hidden, buffers=layer)

    def eager(x):
        hidden.copy_(x)
        step()
        torch.cuda.synchronize()
        return layer.out.clone()

    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    inputs = [torch.empty_like(hidden).normal_(0, 1, generator=g) for _ in range(4)]
    want = [eager(x) for x in inputs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, w in zip(inputs + inputs, want + want):
        hidden.copy_(x)
        layer.out.fill_(777.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.out, w)
        eager(inputs[0])
    side = torch.cuda.Stream()
    hidden.copy_(inputs[2])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(layer.out, want[2])


def test_two_layers_at_once_on_two_streams():
    """Calls with their own buffers side by side."""
    T, H, F, E, k = 400, 256, 264, 8, 2
    a = _layer(T, H, F, E, k, 21)
    b = _layer(T, H, F, E, k, 22)
    alone, both = [], []
    for hidden, w_gate, w_up, w_down, params in (a, b):
        routed = B.route(hidden, w_gate, params, torch.zeros(E, dtype=torch.int32, device="cuda"))
        alone.append((routed, B.experts(hidden, w_up, w_down, routed).out.clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [B.ExpertBuffers(T, H, F, E, k, torch.bfloat16) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for i, (hidden, w_gate, w_up, w_down, params) in enumerate((a, b)):
            B.experts(hidden, w_up, w_down, alone[i][0], buffers=outs[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i].out, alone[i][1])


def test_smaller_calls_run_in_larger_buffers():
    T, H, F, E, k = 200, 128, 72, 8, 2
    hidden, w_gate, w_up, w_down, params = _layer(T, H, F, E, k, 31)
    ep = B.make_experts_params(k)
    assert B.laser_experts_workspace_bytes(T, H, F, E, ep) >= B.laser_experts_workspace_bytes(T - 1, H, F, E, ep)
    ws = torch.empty(B.laser_experts_workspace_bytes(T, H, F, E, ep), dtype=torch.uint8, device="cuda")
    for n in (T, 33, 1):
        routed = B.route(hidden[:n], w_gate, params, torch.zeros(E, dtype=torch.int32, device="cuda"))
        want = B.experts(hidden[:n], w_up, w_down, routed)
        out = torch.full((n, H), 777.0, dtype=torch.bfloat16, device="cuda")
        B.laser_experts_down(want.act, w_down, n, H, F, E, ep, routed.permutation, routed.expert_offsets,
                             routed.expert_ids, routed.weights, None, out, ws)
        assert torch.equal(out, want.out)


def test_nothing_to_do():
    params = B.make_experts_params(2)
    one = torch.zeros(1, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(4, 16, 64, dtype=torch.bfloat16, device="cuda")
    offs = torch.zeros(5, dtype=torch.int32, device="cuda")
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    B.laser_experts_up(None, w, 0, 64, 8, 4, params, None, offs, None)
    B.laser_experts_down(None, w, 0, 64, 8, 4, params, None, offs, None, None, None, None, ws)
    # no assignment for any of the call's experts: act untouched, out the base
    act = torch.full((2, 8), 777.0, dtype=torch.bfloat16, device="cuda")
    perm = torch.zeros(2, dtype=torch.int32, device="cuda")
    ids = torch.full((1, 2), 9, dtype=torch.int32, device="cuda")
    B.laser_experts_up(one, w, 1, 64, 8, 4, params, perm, offs, act)
    out = torch.full((1, 64), 777.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((B.laser_experts_workspace_bytes(1, 64, 8, 4, params),), 255, dtype=torch.uint8, device="cuda")
    B.laser_experts_down(act, w.reshape(4, 64, 16)[:, :, :8].contiguous(), 1, 64, 8, 4, params, perm, offs, ids, None,
                         one + 3, out, ws)
    torch.cuda.synchronize()
    assert (act == 776.0).all() and (out == 3.0).all()
