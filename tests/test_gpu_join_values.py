"""The join's gradients where values are not finite: a dropped element adds nothing to any sum, whatever it and its gradient hold; a kept one does, also where
its gate is zero.  The same in rows that a workgroup holds in registers and in wider ones."""
import numpy as np
import pytest
import torch

import paper_2411_19460_amd as pk
from join_bounds import gradient_bounds
from oracle import join_ref as ref
from test_gpu_join import EPS, TYPES, dev, draw, near, rng_of

pytestmark = pytest.mark.gpu
WIDTHS = [8200, 8196, 10243]
NARROW = [7, 8, 264, 512, 2560, 2561, 4104, 8191, 8192]


def backward(d, dtype, stream, T, gate_rows, s, ds, p, f=None, x=True):
    params = {k: dev(d[k]) for k in ("post_w", "gate", "alpha", "pre_w")}
    return pk.ssd_join_bwd(s, dev(d["f"], dtype) if f is None else f, dev(d["dout"], dtype), ds=ds, x=dev(d["x"], stream) if x else None, **params,
                           gate_rows=gate_rows, eps=EPS, p=p, rng=rng_of(1, 2))


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("D", NARROW + WIDTHS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("post", [True, False])
def test_a_gradient_of_a_dropped_element(dtype, stream, D, value, post):
    """ds that is not finite where elements are dropped: dx has it there, and nothing else knows of it but dalpha's columns."""
    T, p, gate_rows = 9, 0.3, 4
    d = draw(D, dtype, stream, T, D, post=post, gate_rows=gate_rows)
    keep = ref.mask(T, D, p, 1, 2)
    dropped = [np.argwhere(keep[r] == 0)[:, 0] for r in range(T)]
    places = [(r, int(dropped[r][k % len(dropped[r])])) for r, k in ((0, 0), (3, -1), (4, 7), (8, 20)) if len(dropped[r])]
    assert places
    params = {k: dev(d[k]) for k in ("post_w", "gate", "alpha", "pre_w")}
    s = pk.ssd_join_fwd(dev(d["x"], stream), dev(d["f"], dtype), **params, gate_rows=gate_rows, eps=EPS, p=p, rng=rng_of(1, 2))["s"]
    ds = dev(d["ds"], stream)
    for r, c in places:
        ds[r, c] = value
        d["ds"][r, c] = 0.0
    q = backward(d, dtype, stream, T, gate_rows, s, ds, p)
    sh = s.double().cpu().numpy()
    gates = ref._gates(d["gate"], T, gate_rows)
    g = ref.backward(sh, d["f"], d["dout"], d["ds"], d["x"], d["post_w"], d["gate"], gate_rows, d["alpha"], d["pre_w"], keep, EPS)
    b = gradient_bounds(sh, d["f"], d["dout"], d["ds"], d["x"], d["post_w"], gates, d["alpha"], d["pre_w"], keep, EPS, g, T)
    b["dgate"] = np.stack([b["dgate rows"][k:k + gate_rows].sum(0) for k in range(0, T, gate_rows)])
    for name in ("df", "dgate", "dpre_w") + (("dpost_w",) if post else ()):
        near(q[name], g[name], b[name], dtype if name == "df" else "f32", name)
    rows, cols = (list(t) for t in zip(*places))
    assert not bool(torch.isfinite(q["dx"][rows, cols]).any()) and not bool(torch.isfinite(q["dalpha"][cols]).any())
    finite = torch.ones((T, D), dtype=torch.bool, device="cuda")
    finite[rows, cols] = False
    assert bool(torch.isfinite(q["dx"][finite]).all())
    others = torch.ones(D, dtype=torch.bool, device="cuda")
    others[cols] = False
    assert bool(torch.isfinite(q["dalpha"][others]).all())


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("D", [1, 5, *NARROW, *WIDTHS])
@pytest.mark.parametrize("which", ["ds", "dout"])
def test_where_everything_is_dropped(dtype, stream, D, which):
    """Nothing of f enters the stream, so its gradient and those of its norm and gate are zero, whatever the gradients of the results."""
    T = 5
    d = draw(D, dtype, stream, T, D, gate_rows=2)
    d[which][1, D // 2], d[which][4, 0] = np.inf, np.nan
    q = backward(d, dtype, stream, T, 2, dev(d["x"], stream), dev(d["ds"], stream), 1.0)
    for name in ("df", "dgate", "dpost_w"):
        assert bool((q[name] == 0).all()), name


@pytest.mark.parametrize("D", [264, *WIDTHS])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_a_kept_value_behind_a_closed_gate(D, value, p):
    """du = 0 times an fhat that is not finite is not a number, and dpost_w says so; where the element is dropped as well, it is not asked."""
    T, c = 9, 20
    d = draw(D, "bf16", "bf16", T, D, gate_rows=0, alpha=False, pre=False)
    d["gate"][:, c] = 0.0
    keep = ref.mask(T, D, p, 1, 2) if p else np.ones((T, D))
    row = int(np.argwhere(keep[:, c] > 0)[0, 0])
    f = dev(d["f"], "bf16")
    f[row, c] = value
    q = pk.ssd_join_bwd(dev(d["x"], "bf16"), f, None, ds=dev(d["ds"], "bf16"), post_w=dev(d["post_w"]), gate=dev(d["gate"]), eps=EPS, p=p, rng=rng_of(1, 2))
    assert bool(torch.isnan(q["dpost_w"][c])) and bool(torch.isnan(q["dgate"][0, c]))
