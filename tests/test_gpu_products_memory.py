"""Calls of the products on a stream of their own whose tensors are dropped right behind them: the memory
is not handed out again before the call has run."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2510_03293_amd import binding as B
from tests import products as P

pytestmark = pytest.mark.gpu

BF16 = B.DTYPE_BF16
LAYER = dict(T=300, H=256, F=264, E=8, k=2)


class Tables:
    """A routed call's tables as tensors of their own."""

    def __init__(self, T, E, k, seed):
        rng = np.random.default_rng(seed)
        ids = P.random_ids(rng, T, k, E)
        perm, offs = P.tables(ids, E)
        self.k = k
        self.permutation, self.expert_offsets, self.expert_ids = (torch.from_numpy(t).cuda() for t in (perm, offs, ids))
        self.weights = torch.from_numpy(rng.random((T, k)).astype(np.float32)).cuda()


def operands(seed=60):
    T, H, F, E, k = LAYER.values()
    rng = np.random.default_rng(seed)
    return (P.rounded(rng, (T, H), 1.0, BF16).cuda(), P.rounded(rng, (E, 2 * F, H), 0.1, BF16).cuda(),
            P.rounded(rng, (E, H, F), 0.1, BF16).cuda(), Tables(T, E, k, seed))


def busy_stream():
    """A stream that has some milliseconds of work before what comes next."""
    side, big = torch.cuda.Stream(), torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(8):
            big.add_(1.0)
    return side, big


def overwrite(sizes):
    """Every block of these sizes that the current stream can have by now."""
    return [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]


def nbytes(*tensors):
    return [t.numel() * t.element_size() for t in tensors]


@pytest.mark.parametrize("own_buffers", [False, True])
def test_dropped_operands_of_the_experts(own_buffers):
    hidden, w_up, w_down, routed = operands()
    want = B.experts(hidden, w_up, w_down, routed, base=hidden).out.clone()
    side, big = busy_stream()
    h, u, d, r = operands()                   # (these copies come from pageable memory: they are there when it returns)
    base = hidden.clone()
    buf = B.ExpertBuffers(*LAYER.values(), torch.bfloat16) if own_buffers else None
    torch.cuda.current_stream().synchronize()
    sizes = nbytes(h, u, d, base, r.permutation, r.expert_offsets, r.expert_ids, r.weights)
    if own_buffers:
        sizes += nbytes(buf.act, buf.workspace)
    got = B.experts(h, u, d, r, base=base, buffers=buf, stream=side).out
    del h, u, d, r, base, buf
    other = overwrite(sizes)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(bool((t == 255).all()) for t in other)


@pytest.mark.parametrize("own_buffers", [False, True])
def test_dropped_operands_of_the_projection(own_buffers):
    T, H, N, R, M = 700, 264, 200, 16, 3

    def made():
        rng = np.random.default_rng(61)
        return [t.cuda() for t in (P.rounded(rng, (T, H), 1.0, BF16), P.rounded(rng, (N, H), 0.05, BF16),
                                   P.rounded(rng, (M, R, H), 0.1, BF16), P.rounded(rng, (M, N, R), 0.2, BF16),
                                   torch.rand(M, generator=torch.Generator().manual_seed(1)),
                                   torch.tensor([0, 300, 300, 650], dtype=torch.int32),
                                   torch.tensor([2, 1, 0], dtype=torch.int32))]

    want = B.project_adapted(*made(), out_dtype=torch.float32).clone()
    side, big = busy_stream()
    given = made()
    buf = B.ProjectBuffers(T, H, N, B.make_adapter_params(R, M, 3, out_dtype=B.DTYPE_F32)) if own_buffers else None
    torch.cuda.current_stream().synchronize()
    sizes = nbytes(*given) + (nbytes(buf.workspace) if own_buffers else [])
    got = B.project_adapted(*given, out_dtype=torch.float32, buffers=buf, stream=side)
    del given, buf
    other = overwrite(sizes)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and all(bool((t == 255).all()) for t in other)


def test_dropped_results():
    """A result that the current stream is still reading when it is dropped, and the next call on the other
    stream, which could be given its memory."""
    hidden, w_up, w_down, routed = operands(62)
    other = operands(63)
    want = B.experts(hidden, w_up, w_down, routed).out.clone()
    side, big = torch.cuda.Stream(), torch.zeros(1 << 28, device="cuda")
    torch.cuda.synchronize()
    layer = B.experts(hidden, w_up, w_down, routed, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(8):
        big.add_(1.0)
    seen = layer.out + 0
    del layer
    for _ in range(3):
        B.experts(*other, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(seen, want)
