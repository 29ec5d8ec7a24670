"""What the products' entry points refuse, before any device work (no GPU needed: fake non-null
addresses are never used)."""
import ctypes

import pytest
import torch

from paper_2510_03293_amd import binding as B

FAKE = ctypes.c_void_p(0x1000)
WS = ctypes.c_void_p(0x10000)
lib = B._lib


def up(p=None, T=8, H=64, F=64, E=4, hidden=FAKE, w=FAKE, perm=FAKE, offs=FAKE, act=FAKE):
    p = B.make_experts_params(2) if p is None else p
    return lib.laser_experts_up(hidden, w, T, H, F, E, ctypes.byref(p), perm, offs, act, None)


def down(p=None, T=8, H=64, F=64, E=4, act=FAKE, w=FAKE, perm=FAKE, offs=FAKE, ids=FAKE, wt=FAKE, base=FAKE, out=FAKE,
         ws=WS, wsz=1 << 30):
    p = B.make_experts_params(2) if p is None else p
    return lib.laser_experts_down(act, w, T, H, F, E, ctypes.byref(p), perm, offs, ids, wt, base, out, ws, wsz, None)


def project(p=None, T=8, H=64, N=5, x=FAKE, w=FAKE, a=FAKE, b=FAKE, s=FAKE, cuts=FAKE, which=FAKE, out=FAKE, ws=WS,
            wsz=1 << 30):
    p = B.make_adapter_params(8, 2, 3) if p is None else p
    return lib.laser_project_adapted(x, w, T, H, N, ctypes.byref(p), a, b, s, cuts, which, out, ws, wsz, None)


ODD = ctypes.c_void_p(0x1008)


@pytest.mark.parametrize("call", [up, down])
def test_experts(call):
    assert call(T=-1) == -2 and call(H=0) == -2 and call(F=0) == -2 and call(E=0) == -2
    assert call(B.make_experts_params(0)) == -2
    assert call(B.make_experts_params(2, first_expert=-1)) == -2
    assert call(B.make_experts_params(2, dtype=7)) == -2
    assert call(B.make_experts_params(2), T=1 << 30) == -2              # T * k beyond 2^31
    assert call(B.make_experts_params(17)) == -5
    assert call(E=65) == -5
    assert call(B.make_experts_params(2, first_expert=61)) == -5
    assert call(H=60) == -3 and call(F=60) == -3
    assert call(B.make_experts_params(2, dtype=B.DTYPE_F32), H=62) == -3
    assert call(w=ODD) == -3 and call(act=ODD) == -3
    assert call(w=None) == -1 and call(act=None) == -1
    assert call(perm=None) == -1 and call(offs=None) == -1
    assert call(perm=None, offs=None) == -1                             # k = 2, E = 4: tables are needed
    assert call(B.make_experts_params(1), E=2, perm=None, offs=None) == -1
    bad = B.make_experts_params(2)
    bad.struct_bytes = 12
    assert call(bad) == -6
    assert call(T=0) == 0                                               # nothing to do, nothing launched


def test_experts_up_and_down_alone():
    assert up(hidden=None) == -1 and up(hidden=ODD) == -3
    assert down(out=None) == -1 and down(out=ODD) == -3 and down(base=ODD) == -3
    assert down(ws=None) == -1 and down(ws=ctypes.c_void_p(0x10010)) == -3
    need = B.laser_experts_workspace_bytes(8, 64, 64, 4, B.make_experts_params(2))
    assert need > 0 and down(wsz=need - 1) == -4
    assert lib.laser_experts_up(FAKE, FAKE, 8, 64, 64, 4, None, FAKE, FAKE, FAKE, None) == -1
    assert B.laser_experts_workspace_bytes(8, 60, 64, 4, B.make_experts_params(2)) == 0
    assert B.laser_experts_workspace_bytes(0, 64, 64, 4, B.make_experts_params(2)) > 0


def test_project():
    assert project(T=-1) == -2 and project(H=0) == -2 and project(N=0) == -2
    assert project(B.make_adapter_params(0, 2, 3)) == -2
    assert project(B.make_adapter_params(8, -1, 3)) == -2
    assert project(B.make_adapter_params(8, 2, -1)) == -2
    assert project(B.make_adapter_params(8, 2, 3, dtype=5)) == -2
    assert project(B.make_adapter_params(8, 2, 3, dtype=B.DTYPE_F32, out_dtype=B.DTYPE_BF16)) == -2
    assert project(B.make_adapter_params(136, 2, 3)) == -5
    assert project(B.make_adapter_params(12, 2, 3)) == -3
    assert project(H=60) == -3
    for name in ("x", "w", "a", "b", "out"):
        assert project(**{name: ODD}) == -3, name
    for name in ("x", "w", "a", "b", "out", "cuts", "which", "ws"):
        assert project(**{name: None}) == -1, name
    need = B.laser_project_workspace_bytes(8, 64, 5, B.make_adapter_params(8, 2, 3))
    assert need > 0 and project(wsz=need - 1) == -4
    assert project(ws=ctypes.c_void_p(0x10010)) == -3
    bad = B.make_adapter_params(8, 2, 3)
    bad.struct_bytes = 8
    assert project(bad) == -6
    assert project(T=0) == 0
    assert project(B.make_adapter_params(8, 2, (1 << 28) + 1)) == -2
    assert B.laser_project_workspace_bytes(8, 60, 5, B.make_adapter_params(8, 2, 3)) == 0


def test_python_wrappers_check_their_tensors():
    T, H, F, E, k = 4, 64, 32, 4, 2
    h = torch.zeros(T, H, dtype=torch.bfloat16)
    up_w, down_w = torch.zeros(E, 2 * F, H, dtype=torch.bfloat16), torch.zeros(E, H, F, dtype=torch.bfloat16)

    class Routed:
        permutation = torch.zeros(T * k, dtype=torch.int32)
        expert_offsets = torch.zeros(E + 1, dtype=torch.int32)
        expert_ids = torch.zeros(T, k, dtype=torch.int32)
        weights = torch.zeros(T, k)

    Routed.k = k
    ok = dict(hidden=h, w_up=up_w, w_down=down_w, routed=Routed)
    for bad in (dict(hidden=h[:3]), dict(hidden=h.float()), dict(hidden=h.t().contiguous().t()),
                dict(w_up=up_w[:, :-1]), dict(w_down=down_w[:3]), dict(w_down=down_w.transpose(1, 2)),
                dict(base=h[:, :8]), dict(base=h.float()), dict(hidden=h.half())):
        with pytest.raises(ValueError):
            B.experts(**{**ok, **bad})
    with pytest.raises(ValueError):
        B.experts(**ok)                                     # tensors that are not on a GPU
    x, w = torch.zeros(T, H, dtype=torch.bfloat16), torch.zeros(8, H, dtype=torch.bfloat16)
    a, b = torch.zeros(2, 8, H, dtype=torch.bfloat16), torch.zeros(2, 8, 8, dtype=torch.bfloat16)
    cuts, which = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    ok = dict(x=x, w=w, a_down=a, a_up=b, scales=torch.ones(2), request_offsets=cuts, request_adapters=which)
    for bad in (dict(w=w[:, :32]), dict(a_down=a[:1]), dict(a_up=b[:, :4]), dict(scales=torch.ones(3)),
                dict(scales=torch.ones(2, dtype=torch.float64)), dict(request_offsets=cuts[:2]),
                dict(request_offsets=cuts.long()), dict(out_dtype=torch.float16), dict(x=x.float())):
        with pytest.raises(ValueError):
            B.project_adapted(**{**ok, **bad})
    with pytest.raises(ValueError):
        B.project_adapted(**ok)
