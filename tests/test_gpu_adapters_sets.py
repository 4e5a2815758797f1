"""Sets of many adapters of which few have rows, adapters of several units beside them, and rows that lie far apart.  Bounds as in
test_gpu_adapters.py."""
import numpy as np
import pytest
import torch

import paper_2411_19460_amd as pk
from test_gpu_adapters import bounds, dev, draw, host, inside

pytestmark = pytest.mark.gpu


def run(x, w, a, b, scale, ids, dout, n, **out):
    plan = pk.ssd_adapter_plan(torch.from_numpy(np.asarray(ids)).int().cuda(), n)
    f = pk.ssd_adapter_linear_fwd(x, w, a, b, scale, plan, want_hidden=True, out=out.get("out"))
    return {**f, **pk.ssd_adapter_linear_bwd(x, w, a, b, scale, plan, dout, hidden=f["hidden"], dx=out.get("dx"))}


def check(case, ids, n):
    x, w, a, b, scale, _, dout = case
    ref, off = bounds(x, w, a, b, scale, ids, dout)
    got = run(dev(x), dev(w), dev(a), dev(b), dev(scale, torch.float32), ids, dev(dout), n)
    for name in ("hidden", "out", "dx", "da", "db"):
        inside(name, host(got[name]), ref[name], off[name])


def test_few_of_the_most_adapters():
    """The same bits as with the adapters that have rows alone, zeros for the others."""
    T, I, O, R, n = 3000, 520, 72, 8, 16384
    used = np.array([0, 63, 64, 9000, n - 1])
    r = np.random.default_rng(3)
    mine = r.integers(-1, len(used), T)
    ids = np.where(mine < 0, -1, used[mine])
    x, w, a, b, scale, _, dout = draw(1, T, I, O, R, len(used), mine)
    x, w, dout = dev(x), dev(w), dev(dout)
    few = [dev(a), dev(b), dev(scale, torch.float32)]
    at = torch.from_numpy(used).cuda()
    all_ = [torch.full((n, *t.shape[1:]), float("nan"), dtype=t.dtype, device="cuda") for t in few]
    for big, small in zip(all_, few):
        big[at] = small
    ref, got = run(x, w, *few, mine, dout, len(used)), run(x, w, *all_, ids, dout, n)
    for name in ("hidden", "out", "dx"):
        assert torch.equal(ref[name], got[name]), name
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[at] = False
    for name in ("da", "db"):
        assert torch.equal(ref[name], got[name][at]), name
        assert not bool(got[name][rest].any()), name


def test_several_hundred_adapters_with_rows():
    T, n = 2100, 300
    ids = np.random.default_rng(4).permutation(np.arange(T) % n)
    check(draw(2, T, 72, 520, 40, n, ids), ids, n)


@pytest.mark.parametrize("own", [(3,), (3, 40), (0, 1, 49), (48, 49, 5, 6, 7)])
def test_adapters_of_several_units_among_others(own):
    T, n = 6000, 50
    r = np.random.default_rng(5)
    ids = np.where(r.random(T) < 0.95, np.array(own)[r.integers(0, len(own), T)], r.integers(-1, n, T))
    check(draw(3, T, 136, 72, 16, n, ids), ids, n)


@pytest.mark.parametrize("T", [3, 16, 40, 300, 700])
def test_rows_far_apart(T):
    """A row stride whose byte offsets inside one tile pass 32 bits."""
    I, O, R, n, ld = 136, 200, 16, 3, (1 << 22) + 8
    ids = np.random.default_rng(6).integers(-1, n, T)
    x, w, a, b, scale, _, dout = draw(4, T, I, O, R, n, ids)
    ref, off = bounds(x, w, a, b, scale, ids, dout)

    def far(t, cols):
        v = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda").view(T, ld)[:, :cols]
        return v if t is None else v.copy_(dev(t))

    got = run(far(x, I), dev(w), dev(a), dev(b), dev(scale, torch.float32), ids, far(dout, O), n, out=far(None, O), dx=far(None, I))
    for name in ("hidden", "out", "dx", "da", "db"):
        inside(name, host(got[name]), ref[name], off[name])
