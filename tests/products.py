"""What the tests of the products share: inputs, routing tables and the definitions in 64 bits
with the bounds on a correct result's distance from them.

Bounds.  A sum of n products held in fp32 is off by at most (n + 1) 2^-24 times the sum of the
products' magnitudes, whatever its order (each of its n roundings is off by half a step of a partial
sum that is no larger; bf16 products are exact, fp32 products round once more).  A value stored
in bf16 is off by 2^-8 of itself, in fp32 by 2^-24.
"""
from __future__ import annotations

import numpy as np
import torch

from paper_2510_03293_amd import binding as B

TORCH = {B.DTYPE_F32: torch.float32, B.DTYPE_BF16: torch.bfloat16}
HALF_STEP = {B.DTYPE_F32: 2.0 ** -24, B.DTYPE_BF16: 2.0 ** -8}
U = 2.0 ** -24


def rounded(rng, shape, std, dtype):
    """Normal values already rounded to the type, as a CPU tensor of it."""
    return torch.from_numpy((rng.standard_normal(shape) * std).astype(np.float32)).to(TORCH[dtype])


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def tables(ids, total):
    """permutation [T*k], offsets [total+1] of expert ids [T,k] (numpy)."""
    flat = ids.reshape(-1)
    perm = np.argsort(flat, kind="stable").astype(np.int32)
    offs = np.zeros(total + 1, dtype=np.int32)
    offs[1:] = np.cumsum(np.bincount(flat, minlength=total))
    return perm, offs


def random_ids(rng, T, k, total, skew=0.0):
    """k distinct experts per token, popularity falling like rank^-skew."""
    p = (np.arange(total) + 1.0) ** -skew
    score = np.log(p)[rng.permutation(total)] + rng.gumbel(size=(T, total))
    return np.argsort(-score, axis=1)[:, :k].astype(np.int32)


def product_bound(x, w, dtype):
    """x [r,n] times w [c,n] transposed in fp64, and how far an fp32 sum may be from it."""
    n = x.shape[1] + (x.shape[1] if dtype == B.DTYPE_F32 else 0)
    return x @ w.T, (n + 1) * U * (np.abs(x) @ np.abs(w).T)


def silu(g):
    return g / (1.0 + np.exp(-g))


def up_reference(hidden, w_up, perm, offs, k, first, dtype):
    """(positions, act, bound) of the experts' rows in fp64."""
    h, w = f64(hidden), f64(w_up)
    E, F2, _ = w.shape
    F = F2 // 2
    pos, val, tol = [], [], []
    for e in range(E):
        a, b = int(offs[first + e]), int(offs[first + e + 1])
        if a == b:
            continue
        z, bz = product_bound(h[perm[a:b] // k], w[e], dtype)
        g, u, dg, du = z[:, :F], z[:, F:], bz[:, :F], bz[:, F:]
        y = silu(g) * u
        # |silu'| < 1.1.  The sigmoid itself: exp2's argument is rounded (2^-24 of itself, so
        # |g| 2^-24 in the exponential and no more in the sigmoid), then exp2, sum, reciprocal and
        # two products, each within two steps
        own = (np.abs(g) + 12) * 2 * U * np.abs(y)
        pos.append(np.arange(a, b))
        val.append(y)
        tol.append((1.1 * dg * np.abs(u) + np.abs(silu(g)) * du + 1.1 * dg * du + own) * 1.01
                   + HALF_STEP[dtype] * np.abs(y) * 1.01 + 1e-37)
    if not pos:
        return np.zeros(0, np.int64), np.zeros((0, F)), np.zeros((0, F))
    return np.concatenate(pos), np.concatenate(val), np.concatenate(tol)


def down_reference(act, w_down, perm, offs, ids, weights, base, k, first, T, dtype):
    """(out, bound) in fp64."""
    a64, w = f64(act), f64(w_down)
    E, H, _ = w.shape
    out, tol, size = np.zeros((T, H)), np.zeros((T, H)), np.zeros((T, H))
    if base is not None:
        out += f64(base)
        size += np.abs(out)
    for e in range(E):
        a, b = int(offs[first + e]), int(offs[first + e + 1])
        if a == b:
            continue
        slots = perm[a:b]
        z, bz = product_bound(a64[a:b], w[e], dtype)
        wt = np.ones(b - a) if weights is None else weights.reshape(-1)[slots].astype(np.float64)
        np.add.at(out, slots // k, z * wt[:, None])
        np.add.at(tol, slots // k, (bz + U * np.abs(z)) * np.abs(wt)[:, None])
        np.add.at(size, slots // k, np.abs(z * wt[:, None]))
    # bf16: a summand may be held in fp16 after a power of two has brought the largest of its row's 64
    # columns to 2^14 or more.  fp16 values have 11 significant bits, so rounding is off by half of
    # 2^-10 of the value, 2^-11; below 2^-14 it is off by half of its step of 2^-24, which is 2^-25 / 2^14 =
    # 2^-39 of the largest.
    if dtype == B.DTYPE_BF16:
        own = size if base is None else size - np.abs(f64(base))
        tol += 2.0 ** -11 * own + 2.0 ** -39 * own.max(axis=1, keepdims=True) * k
    # k additions (and the base's) of partial sums no larger than the sum of magnitudes
    return out, (tol + (k + 1) * U * size) * 1.01 + HALF_STEP[dtype] * np.abs(out) * 1.01 + 1e-37


def project_reference(x, w, a_down, a_up, scales, cuts, which, out_dtype, dtype):
    """(out, bound) in fp64."""
    x64 = f64(x)
    out, tol = product_bound(x64, f64(w), dtype)
    M = 0 if a_down is None else a_down.shape[0]
    for q, m in enumerate(which):
        a, b = int(cuts[q]), int(cuts[q + 1])
        if a >= b or not 0 <= m < M:
            continue
        s = 1.0 if scales is None else float(scales[m])
        v, bv = product_bound(x64[a:b], f64(a_down[m]), dtype)
        up = f64(a_up[m])
        y = v @ up.T
        size = np.abs(v) @ np.abs(up).T
        R = up.shape[1]
        # the inner sum's error through the second product; the scale's rounding; the second
        # sum, whose products are not exact here, so two roundings a term and three for an
        # inner value that is held in pieces of the storage type
        out[a:b] += s * y
        tol[a:b] += abs(s) * (bv @ np.abs(up).T + (2 * R + 8) * U * size)
    return out, (tol + 2 * U * np.abs(out)) * 1.01 + HALF_STEP[out_dtype] * np.abs(out) * 1.01 + 1e-37


def assert_within(got, want, tol, label=""):
    got = np.asarray(got, dtype=np.float64)
    off = np.abs(got - want)
    bad = ~(off <= tol)
    if bad.any():
        at = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{label}: {bad.sum()} of {bad.size} outside the bound, first at {at}: got {got[at]}, "
                             f"want {want[at]}, off by {off[at]}, bound {tol[at]}")


def run_up(hidden, w_up, perm, offs, k, dtype, first=0, fill=None):
    """laser_experts_up on CPU tensors / numpy tables; act on the GPU, pre-filled with `fill`."""
    T, H = hidden.shape
    E, F2, _ = w_up.shape
    act = torch.full((T * k, F2 // 2), 777.0 if fill is None else fill, dtype=TORCH[dtype], device="cuda")
    p = None if perm is None else torch.from_numpy(perm).cuda()
    o = None if offs is None else torch.from_numpy(offs).cuda()
    params = B.make_experts_params(k, dtype=dtype, first_expert=first)
    B.laser_experts_up(hidden.cuda(), w_up.cuda(), T, H, F2 // 2, E, params, p, o, act)
    torch.cuda.synchronize()
    return act


def run_down(act, w_down, perm, offs, ids, weights, base, k, T, dtype, first=0, in_place=False):
    E, H, F = w_down.shape
    params = B.make_experts_params(k, dtype=dtype, first_expert=first)
    ws = torch.full((B.laser_experts_workspace_bytes(T, H, F, E, params),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((T, H), 777.0, dtype=TORCH[dtype], device="cuda")
    dev = [None if t is None else torch.from_numpy(t).cuda() for t in (perm, offs, ids, weights)]
    bd = None if base is None else base.cuda()
    if in_place:
        out = bd
    B.laser_experts_down(act.cuda(), w_down.cuda(), T, H, F, E, params, *dev, bd, out, ws)
    torch.cuda.synchronize()
    return out


def run_project(x, w, a_down, a_up, scales, cuts, which, out_dtype, dtype):
    T, H = x.shape
    N = w.shape[0]
    M, R = (0, 8) if a_down is None else a_down.shape[:2]
    params = B.make_adapter_params(R, M, len(which), dtype=dtype, out_dtype=out_dtype)
    ws = torch.full((B.laser_project_workspace_bytes(T, H, N, params),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((T, N), 777.0, dtype=TORCH[out_dtype], device="cuda")
    up = [None if t is None else (torch.from_numpy(t) if isinstance(t, np.ndarray) else t).cuda()
          for t in (a_down, a_up, scales, cuts, which)]
    B.laser_project_adapted(x.cuda(), w.cuda(), T, H, N, params, *up, out, ws)
    torch.cuda.synchronize()
    return out
