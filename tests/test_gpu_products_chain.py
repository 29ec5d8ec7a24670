"""A whole layer of adapted requests: gate with adapters -> laser_route_from_logits -> both products of the experts,
eager, from a graph, and on another stream."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2510_03293_amd import binding as B
from tests import products as P

pytestmark = pytest.mark.gpu

BF16 = B.DTYPE_BF16


@pytest.mark.parametrize("T,H,E,F,lengths", [(3, 256, 16, 136, [1, 1, 1]), (200, 256, 16, 72, [50, 1, 149]),
                                             (1500, 520, 64, 200, [700, 0, 700]), (900, 2056, 33, 264, [1] * 20 + [880])])
def test_captured_layer(T, H, E, F, lengths):
    k, M, R = 4, 3, 16
    rng = np.random.default_rng(90)
    x, w = P.rounded(rng, (T, H), 1.0, BF16).cuda(), P.rounded(rng, (E, H), 0.05, BF16).cuda()
    down, up = P.rounded(rng, (M, R, H), 1 / np.sqrt(H), BF16).cuda(), P.rounded(rng, (M, E, R), 0.2, BF16).cuda()
    w_up, w_down = P.rounded(rng, (E, 2 * F, H), 0.05, BF16).cuda(), P.rounded(rng, (E, H, F), 0.05, BF16).cuda()
    scales = torch.from_numpy((rng.random(M) * 2).astype(np.float32)).cuda()
    cuts = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).cuda()
    which = torch.from_numpy(rng.integers(-1, M, len(lengths)).astype(np.int32)).cuda()
    params = B.make_params(k, 6, 0.4, 0.8)
    loads = torch.zeros(E, dtype=torch.int32, device="cuda")
    gate = B.ProjectBuffers(T, H, E, B.make_adapter_params(R, M, len(lengths), out_dtype=B.DTYPE_F32))
    routed = B.RouteBuffers(T, 0, E, params)
    layer = B.ExpertBuffers(T, H, F, E, k, x.dtype)

    def step(stream=None):
        if stream is None:
            loads.zero_()
        else:
            with torch.cuda.stream(stream):
                loads.zero_()
        logits = B.project_adapted(x, w, down, up, scales, cuts, which, out_dtype=torch.float32, buffers=gate, stream=stream)
        B.route_from_logits(logits, params, loads, routed, stream=stream)
        B.experts(x, w_up, w_down, routed, base=x, buffers=layer, stream=stream)

    def eager(new):
        x.copy_(new)
        step()
        torch.cuda.synchronize()
        return layer.out.clone(), gate.out.clone(), routed.expert_ids.clone()

    def same(want):
        return all(torch.equal(a, b) for a, b in zip((layer.out, gate.out, routed.expert_ids), want))

    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    inputs = [torch.empty_like(x).normal_(0, 1, generator=g) for _ in range(3)]
    want = [eager(new) for new in inputs]
    P.assert_within(P.f64(gate.out), *P.project_reference(inputs[2], w, down, up, scales.cpu().numpy(), cuts.cpu().numpy(),
                                                          which.cpu().numpy(), B.DTYPE_F32, BF16), "logits")
    perm, offs, ids = (t.cpu().numpy() for t in (routed.permutation, routed.expert_offsets, routed.expert_ids))
    P.assert_within(P.f64(layer.out), *P.down_reference(layer.act, w_down, perm, offs, ids, routed.weights.cpu().numpy(), x, k, 0,
                                                        T, BF16), "layer")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for new, w_ in zip(inputs + inputs, want + want):
        x.copy_(new)
        layer.out.fill_(777.0)
        graph.replay()
        torch.cuda.synchronize()
        assert same(w_)
        eager(inputs[0])
    side = torch.cuda.Stream()
    x.copy_(inputs[1])
    torch.cuda.synchronize()
    step(side)
    side.synchronize()
    assert same(want[1])
    # a captured call whose work goes to a stream of its own, forked from the capturing one and joined again
    forked = torch.cuda.CUDAGraph()
    with torch.cuda.graph(forked):
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        torch.cuda.current_stream().wait_stream(side)
    for new, w_ in zip(inputs, want):
        x.copy_(new)
        layer.out.fill_(777.0)
        forked.replay()
        torch.cuda.synchronize()
        assert same(w_)
