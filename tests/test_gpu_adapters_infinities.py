"""An infinity in one operand, in a row or an adapter that meets it: every result is what the formula gives, infinite with its sign or NaN at
the same places as in fp64, and unchanged (bounds of test_gpu_adapters.py) where the infinity does not come in."""
import numpy as np
import pytest
import torch

import paper_2411_19460_amd as pk
from oracle import adapter_ref
from test_gpu_adapters import bounds, dev, draw, host, inside
from test_gpu_adapters_parts import SHAPES

pytestmark = pytest.mark.gpu


def as_formula(name, got, ref, clean, off):
    wild = ~np.isfinite(ref)
    assert np.array_equal(got[wild], ref[wild], equal_nan=True), f"{name}: {np.sum(~((got == ref) | (np.isnan(got) & np.isnan(ref)))[wild])} of {wild.sum()} that are not finite"
    inside(name, got[~wild], clean[~wild], off[~wild])


# along the axis that is summed over, whose end the kernels fill up
PLACES = [(*s, "middle") for s in SHAPES] + [(*s, p) for s in SHAPES for p in ("first", "last") if s[0] * s[1] * s[2] < 3e7]


@pytest.mark.parametrize("T,I,O,R,place", PLACES)
@pytest.mark.parametrize("where", ["x", "dout", "a", "b"])
def test_an_infinity(where, T, I, O, R, place):
    n = 3
    ops = dict(zip(("x", "w", "a", "b", "scale", "ids", "dout"), draw(T + O, T, I, O, R, n, np.arange(T) * 2 % n)))
    clean, off = bounds(**ops)
    t = min(T - 1, 1)
    along = lambda size, middle: {"middle": middle, "first": 0, "last": size - 1}[place]
    at = {"x": (t, along(I, I // 2)), "dout": (t, along(O, O // 3)), "a": (ops["ids"][t], R // 2, along(I, I // 3)),
          "b": (ops["ids"][t], along(O, O // 2), R // 3)}[where]
    ops[where] = ops[where].copy()
    ops[where][at] = -np.inf if T % 2 else np.inf
    with np.errstate(all="ignore"):
        *most, dout = ops.values()
        ref = {**adapter_ref.adapter_fwd(*most), **adapter_ref.adapter_bwd(*most, dout)}
    plan = pk.ssd_adapter_plan(torch.from_numpy(ops["ids"].astype(np.int32)).cuda(), n)
    args = (*(dev(ops[k]) for k in ("x", "w", "a", "b")), dev(ops["scale"], torch.float32), plan)
    f = pk.ssd_adapter_linear_fwd(*args, want_hidden=True)
    g = pk.ssd_adapter_linear_bwd(*args, dev(ops["dout"]), hidden=f["hidden"])
    for name, got in {**f, **g}.items():
        as_formula(name, host(got), ref[name], clean[name], off[name])


@pytest.mark.parametrize("T,I,O,R", SHAPES + [(1, 10248, 520, 16), (2, 6152, 264, 24), (3, 1288, 776, 16), (9, 72, 136, 8)])
@pytest.mark.parametrize("place", [0, 5, -1, -6])
def test_an_infinity_in_a_row_without_an_adapter(place, T, I, O, R):
    """The projection alone: every result of the row is infinite, with the sign of its weight."""
    n, t = 2, min(T - 1, 1)
    x, w, a, b, scale, ids, dout = draw(T + O, T, I, O, R, n, np.arange(T) % n)
    ids[t] = -1
    x[t, place], dout[t, place] = np.inf, -np.inf
    plan = pk.ssd_adapter_plan(torch.from_numpy(ids.astype(np.int32)).cuda(), n)
    args = dev(x), dev(w), dev(a), dev(b), dev(scale, torch.float32), plan
    out = host(pk.ssd_adapter_linear_fwd(*args)["out"])
    dx = host(pk.ssd_adapter_linear_bwd(*args, dev(dout), want_dab=False)["dx"])
    assert np.array_equal(out[t], np.inf * w[:, place], equal_nan=True)
    assert np.array_equal(dx[t], -np.inf * w[place], equal_nan=True)
    rest = np.arange(T) != t
    assert np.isfinite(out[rest]).all() and np.isfinite(dx[rest]).all()
