"""Which way a call of the products goes: the library's rules once more, so that a test that is meant for
one kernel says so and notices when the rules change under it."""
from __future__ import annotations

import numpy as np
import torch


def compute_units():
    return torch.cuda.get_device_properties(0).multi_processor_count


def ceil(a, b):
    return -(-a // b)


def experts(op, T, H, F, E, k, f32, offs, first, units=None):
    """few, slices, 32 (fp32), 64, 128 or 256 (rows of a tile), of op "up" or "down"."""
    units = compute_units() if units is None else units
    slots, size = T * k, 4 if f32 else 2
    up = op == "up"
    K, out = (H if up else F) * size, F if up else H
    steps = ceil(K, 128)
    if T <= 4 and slots <= 64 and F <= 1 << 17 and (K >= 1024 or slots * (2 * F if up else H) <= 1 << 15):
        return "few"

    def tiles(bm, bn):
        return min(slots, slots // bm + min(E, slots)) * ceil(out, bn // 2 if up else bn)

    if not up and min(16, (512 if slots >= 32 * E else 256) // tiles(64, 128), steps // 8) > 1:
        return "slices"
    if f32:
        return "32" if tiles(64, 128) < units else "64"
    if slots < 56 * E:
        return "64"
    if steps < 18:
        return "128"
    counts = np.diff(np.asarray(offs, dtype=np.int64)[first:first + E + 1]) if offs is not None else np.array([slots])

    def cost(side, per_unit, step, once):
        whole = int(ceil(counts, side).sum()) * ceil(out, side // 2 if up else side)
        return ceil(whole, per_unit * units) * (step * steps + 120) + once

    return "256" if cost(256, 1, 25, 120) <= cost(128, 2, 19, 0) else "128"


def project(T, H, N, R, requests, f32):
    """thin, slices (joined by a second launch), gate (one launch), or 64, 128, 256 (rows of a tile)."""
    if T <= 512 and T * N <= 1 << 16:
        return "thin"
    rows = ceil(T, 64)
    tiles = rows * ceil(N, 128)
    gate = N <= 64 and R <= 64 and (requests <= 32 or requests <= T // 64)
    steps = ceil(H * (4 if f32 else 2), 128)
    if tiles + rows <= 256 and steps >= 16 and T * N * R <= 1 << 25:
        slices = max(1, min(8, (256 if tiles + rows <= 128 else 512) // (tiles + rows), steps))
        if not gate or steps * (2 if R > 16 else 1) * (slices - 1) > 18 * slices:
            return "slices"
    if gate:
        return "gate"
    if not f32:
        for side in (256, 128):
            if ceil(T, side) * ceil(N, side) >= 128:
                return str(side)
    return "64"
