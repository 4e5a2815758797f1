"""A call of the gated recurrence with more workgroups than one launch takes."""
import pytest
import torch

import paper_2411_19460_amd as pk
from test_gpu_gated_scan_long import both, inputs

pytestmark = pytest.mark.gpu


def test_more_workgroups_than_a_launch_takes():
    """65535 sequences of one channel: 16.8 million chunks backward, the last ones in a second launch.  Every sequence as when it is alone, bit for bit, and dlam is
    the sum over the batch's halves: each is rounded to fp32 once (2^-24 of itself), from fp64 sums of the same chunks' shares, before its two products with
    the factor of lam, so that the halves' sum is off by 6 such steps of the sum of their absolute values."""
    B, L = 65535, 64 * 256 + 1
    x, zr, zi, dout, lam, init = inputs(B, L, 1)
    got = both(x, zr, zi, dout, lam, init)
    for b in (0, 1, 32767, 65278, 65279, 65533, 65534):
        s = slice(b, b + 1)
        alone = both(*(t[s].contiguous() for t in (x, zr, zi, dout)), lam, init[s].contiguous())
        for i in (0, 1, 2, 3, 4, 5, 7):
            assert torch.equal(got[i][s], alone[i]), (b, i)
    assert all(bool(torch.isfinite(t).all()) for t in got)
    halves = [both(*(t[s] for t in (x, zr, zi, dout)), lam, init[s])[6] for s in (slice(0, 30000), slice(30000, B))]
    assert float((got[6] - (halves[0] + halves[1])).abs()) <= 6 * 2.0 ** -24 * float(halves[0].abs() + halves[1].abs())
    acc = torch.full_like(lam, 2.0)
    states = got[2]
    pk.ssd_gated_scan_bwd(x, zr, zi, lam, states, dout, dfinal_state=init, dlam=acc, flags=pk.SSD_FLAG_ACCUM_PARAM)
    assert torch.equal(acc, got[6] + 2.0)
