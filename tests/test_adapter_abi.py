"""CPU-side checks of the adapters' and the gradients' entry points: sizes, refusals before anything touches the device."""
import ctypes

import pytest

import paper_2411_19460_amd as pk
from paper_2411_19460_amd import binding

NULL, SHAPE, DIVISIBILITY, DTYPE, WORKSPACE, ARG = -1, -2, -3, -4, -5, -8
P = 1 << 20          # stands for an aligned device pointer: nothing is launched in a refused call


def shape(**kw):
    base = dict(rows=40, in_dim=64, out_dim=72, rank=16, nadapters=3, x_row_stride=0, out_row_stride=0, dx_row_stride=0)
    base.update(kw)
    return pk.ssd_adapter_shape_t(**base)


def fwd(s, x=P, w=P, a=P, b=P, scale=P, plan=P, out=P, hidden=None, ws=P, nbytes=1 << 40):
    return binding.lib().ssd_adapter_linear_fwd(ctypes.byref(s) if s else None, x, w, a, b, scale, plan, out, hidden, ws, nbytes, None)


def bwd(s, x=P, w=P, a=P, b=P, scale=P, plan=P, dout=P, hidden=None, dx=P, da=P, db=P, ws=P, nbytes=1 << 40, flags=0):
    return binding.lib().ssd_adapter_linear_bwd(ctypes.byref(s) if s else None, x, w, a, b, scale, plan, dout, hidden, dx, da, db, ws, nbytes, flags, None)


BAD_SHAPES = [(dict(rows=-1), SHAPE), (dict(rows=(1 << 30) + 1), SHAPE), (dict(in_dim=0), SHAPE), (dict(out_dim=-8), SHAPE), (dict(in_dim=60), DIVISIBILITY),
              (dict(out_dim=70), DIVISIBILITY), (dict(rank=0), SHAPE), (dict(rank=264), SHAPE), (dict(rank=12), DIVISIBILITY), (dict(nadapters=0), SHAPE),
              (dict(nadapters=16385), SHAPE), (dict(x_row_stride=56), SHAPE), (dict(x_row_stride=68), SHAPE), (dict(out_row_stride=64), SHAPE),
              (dict(dx_row_stride=8), SHAPE)]


@pytest.mark.parametrize("bad,code", BAD_SHAPES)
def test_shapes_that_are_refused(bad, code):
    s = shape(**bad)
    assert fwd(s) == code and bwd(s) == code
    assert binding.lib().ssd_adapter_workspace_bytes(ctypes.byref(s), 0) == 0 and binding.lib().ssd_adapter_workspace_bytes(ctypes.byref(s), 1) == 0


def test_pointers_that_are_refused():
    s = shape()
    assert fwd(None) == NULL and bwd(None) == NULL
    for k in ("x", "w", "a", "b", "scale", "plan", "out"):
        assert fwd(s, **{k: None}) == NULL, k
        assert fwd(s, **{k: P + 2}) == ARG, k
    assert fwd(s, hidden=P + 8) == ARG
    for k in ("x", "w", "a", "b", "scale", "plan", "dout"):
        assert bwd(s, **{k: None}) == NULL, k
        assert bwd(s, **{k: P + 2}) == ARG, k
    assert bwd(s, da=None) == NULL and bwd(s, db=None) == NULL and bwd(s, da=P + 4) == ARG and bwd(s, dx=P + 8) == ARG
    assert bwd(s, flags=1) == ARG and bwd(s, flags=64) == ARG
    for call, i in ((fwd, 0), (bwd, 1)):
        need = binding.lib().ssd_adapter_workspace_bytes(ctypes.byref(s), i)
        assert need > 0 and call(s, ws=None) == WORKSPACE and call(s, ws=P + 16) == WORKSPACE and call(s, nbytes=need - 1) == WORKSPACE
    assert fwd(shape(rows=0), x=None, plan=None, out=None, ws=None) == 0
    assert bwd(s, dx=None, da=None, db=None) == 0          # nothing is asked for


def test_plan_sizes_and_refusals():
    L = binding.lib()
    assert L.ssd_adapter_plan_bytes(0, 1) > 0 and L.ssd_adapter_plan_bytes(-1, 1) == 0 and L.ssd_adapter_plan_bytes(8, 0) == 0
    assert L.ssd_adapter_plan_bytes((1 << 30) + 1, 1) == 0 and L.ssd_adapter_plan_bytes(8, 16385) == 0
    need = L.ssd_adapter_plan_bytes(1000, 7)
    assert L.ssd_adapter_plan(1000, 0, P, P, need, None) == SHAPE
    assert L.ssd_adapter_plan(1000, 7, None, P, need, None) == NULL and L.ssd_adapter_plan(1000, 7, P, None, need, None) == NULL
    assert L.ssd_adapter_plan(1000, 7, P + 2, P, need, None) == ARG
    assert L.ssd_adapter_plan(1000, 7, P, P + 16, need, None) == WORKSPACE and L.ssd_adapter_plan(1000, 7, P, P, need - 1, None) == WORKSPACE
    # what a plan of the longest batch takes does for shorter ones
    sizes = [L.ssd_adapter_plan_bytes(r, 7) for r in (1, 100, 1000, 10000, 100000)]
    assert sizes == sorted(sizes)


def test_gradient_lists():
    L = binding.lib()
    T = pk.ssd_grad_tensor_t

    def plan(*tensors, plan=P, nbytes=1 << 40, pieces=True):
        arr, n = (T * max(1, len(tensors)))(*tensors), ctypes.c_int64()
        return L.ssd_grad_plan(len(tensors), arr, plan, nbytes, ctypes.byref(n) if pieces else None, None)

    ok = T(P, P, 100, 0, 0)
    assert plan(ok, plan=None) == NULL and plan(ok, pieces=False) == NULL
    assert plan(T(None, P, 100, 0, 0)) == NULL and plan(T(P, None, 100, 0, 0)) == NULL
    assert plan(T(P, P, -1, 0, 0)) == SHAPE and plan(T(P, P, 1, 2, 0)) == DTYPE and plan(T(P, P, 1, 0, 7)) == DTYPE
    assert plan(T(P + 2, P, 1, 0, 0)) == ARG and plan(T(P, P + 1, 1, 1, 1)) == ARG and plan(T(P, P, 1, 0, 1)) == ARG
    arr = (T * 2)(ok, T(P, P, 100000, 1, 1))
    need = L.ssd_grad_plan_bytes(2, arr)
    assert need > L.ssd_grad_plan_bytes(1, arr) > 0 and L.ssd_grad_plan_bytes(-1, arr) == 0 and L.ssd_grad_plan_bytes(1, None) == 0
    assert plan(ok, plan=P + 128) == WORKSPACE and plan(ok, nbytes=16) == WORKSPACE
    assert L.ssd_grad_norm(None, 1, P, None) == NULL and L.ssd_grad_norm(P, 1, None, None) == NULL and L.ssd_grad_norm(P, -1, P, None) == ARG
    assert L.ssd_grad_norm(P, 1, P + 4, None) == ARG and L.ssd_grad_norm(P + 16, 1, P, None) == ARG
    f = ctypes.c_float
    assert L.ssd_grad_clip(None, 1, None, f(1.0), None, None) == NULL and L.ssd_grad_clip(P, -1, None, f(1.0), None, None) == ARG
    for m in (-1.0, float("nan")):
        assert L.ssd_grad_clip(P, 1, None, f(m), None, None) == ARG
    assert L.ssd_grad_clip(P, 1, P + 4, f(1.0), None, None) == ARG and L.ssd_grad_clip(P, 1, None, f(1.0), P + 2, None) == ARG
