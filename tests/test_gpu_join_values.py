"""The join's gradients where values are not finite, the same in rows that a workgroup holds in registers and in wider ones."""
import numpy as np
import pytest
import torch

import paper_2411_19460_amd as pk
from oracle import join_ref as ref
from test_gpu_join import EPS, dev, draw, rng_of

pytestmark = pytest.mark.gpu
WIDTHS = [8200, 8196, 10243]


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
