"""An infinite max_norm asks for the norm alone: nothing is scaled, also where the norm is infinite or a NaN (the step that a caller is to drop)."""
import math

import pytest
import torch

import paper_2411_19460_amd as pk
from oracle import adapter_ref

pytestmark = pytest.mark.gpu


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(nan=0.0), b.nan_to_num(nan=0.0))


@pytest.mark.parametrize("odd", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [999, 1_000_003])        # one workgroup does both passes; a launch for each
@pytest.mark.parametrize("given", [False, True])          # the sum of squares handed in
def test_nothing_is_scaled(odd, dtype, size, given):
    g = [torch.randn(size, generator=torch.Generator().manual_seed(size)).to(dtype).cuda(), torch.ones(5, dtype=dtype, device="cuda")]
    g[0][size // 3] = odd
    keep = [t.clone() for t in g]
    plan = pk.ssd_grad_plan(g)
    norm = float(pk.ssd_grad_clip(plan, math.inf, pk.ssd_grad_norm(plan) if given else None))
    ref, want = adapter_ref.clip([t.double().cpu().numpy() for t in keep], math.inf)
    assert math.isnan(norm) if math.isnan(odd) else norm == math.inf == ref
    assert all(same(t, k) for t, k in zip(g, keep))
    outs = [torch.zeros(t.shape, device="cuda") for t in g]
    pk.ssd_grad_clip(pk.ssd_grad_plan(g, outs), math.inf)
    assert all(same(o, k.float()) and same(o.double(), torch.from_numpy(w).cuda()) for o, k, w in zip(outs, keep, want))
