"""Calls of the gated recurrence with more workgroups than a launch takes along a dimension."""
import pytest
import torch

import paper_2411_19460_amd as pk
from test_gpu_gated_scan_long import both, inputs

pytestmark = pytest.mark.gpu


def test_more_workgroups_than_a_line_holds():
    """65535 sequences of one channel: 16.8 million chunks backward.  Every sequence as when it is alone, bit for bit, and dlam is
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


def test_more_tiles_than_a_line_holds():
    """65535 sequences of one token: 16.8 million tiles of one chunk each."""
    B, C = 65535, 257 * 64
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((B, 1, C), generator=g, device="cuda").bfloat16()
    lam = torch.randn(C, generator=g, device="cuda") - 4
    f = pk.ssd_gated_scan_fwd(x, x, x, lam)
    for s in (slice(0, 2), slice(32767, 32768), slice(65270, 65280), slice(65533, B)):
        part = pk.ssd_gated_scan_fwd(*(x[s],) * 3, lam)
        assert all(torch.equal(f[k][s], part[k]) for k in f), s
    q = pk.ssd_gated_scan_bwd(x, x, x, lam, f["states"], x)
    for s in (slice(0, 2), slice(32767, 32768), slice(65270, 65280), slice(65533, B)):
        part = pk.ssd_gated_scan_bwd(*(x[s],) * 3, lam, f["states"][s], x[s])
        assert all(torch.equal(q[k][s], part[k]) for k in ("dx", "dgate_r", "dgate_i", "dinit_state")), s
    assert all(bool(torch.isfinite(t).all()) for t in (f["out"], q["dx"], q["dgate_r"], q["dgate_i"], q["dlam"]))
