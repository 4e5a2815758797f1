"""Global gradient norm and clipping against the fp64 oracle.  Bounds: S is an fp64 sum of exact fp64 squares of the fp32 values (off by
2^-44 of itself at a million elements), the norm is rounded to fp32 once, the factor and each product once, a bf16 result once more."""
import math

import numpy as np
import pytest
import torch

import paper_2411_19460_amd as pk
from oracle import adapter_ref

pytestmark = pytest.mark.gpu
U, BF = 2.0 ** -24, 2.0 ** -8
F32, B16 = torch.float32, torch.bfloat16


def draw(seed, sizes, dtypes):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(s, generator=g) * 10.0 ** (i % 4 - 2)).to(dtypes[i % len(dtypes)]).cuda() for i, s in enumerate(sizes)]


def check(grads, outs, norm, max_norm, before=None):
    src = [t.double().cpu().numpy() for t in (before or grads)]
    n, ref = adapter_ref.clip(src, max_norm)
    assert norm.shape == (1,) and norm.dtype == F32
    assert abs(float(norm) - n) <= 2 * U * n
    for o, r in zip(outs, ref):
        got = o.double().cpu().numpy()
        off = (3 * U + (1.01 * BF if o.dtype == B16 else 0.0)) * np.abs(r) + (2.0 ** -149 if o.dtype == F32 else 2.0 ** -133)
        assert got.shape == r.shape and (np.abs(got - r) <= off).all()


SIZES = [(1,), (0,), (7,), (8,), (8191,), (8192,), (8193,), (3, 5, 7), (129, 127), (1 << 18,)]


@pytest.mark.parametrize("sizes", [[(1,)], [(5,)], SIZES, SIZES * 20], ids=["one", "five", "mixed", "many"])
@pytest.mark.parametrize("src", [(F32,), (B16,), (F32, B16)], ids=["f32", "bf16", "both"])
@pytest.mark.parametrize("dst", [(F32,), (B16,), (B16, F32)], ids=["f32", "bf16", "both"])
def test_norm_and_clip(sizes, src, dst):
    grads = draw(len(sizes), sizes, src)
    outs = [torch.full(t.shape, float("nan"), dtype=dst[i % len(dst)], device="cuda") for i, t in enumerate(grads)]
    before = [t.clone() for t in grads]
    plan = pk.ssd_grad_plan(grads, outs)
    for max_norm in (0.5, 1e9, 0.0):
        check(grads, outs, pk.ssd_grad_clip(plan, max_norm), max_norm)
    assert all(torch.equal(t, v) for t, v in zip(grads, before))


@pytest.mark.parametrize("dtype", [F32, B16])
def test_in_place(dtype):
    grads = draw(3, SIZES, (dtype,))
    before = [t.clone() for t in grads]
    plan = pk.ssd_grad_plan(grads)
    check(grads, grads, pk.ssd_grad_clip(plan, 1e9), 1e9, before)
    assert all(torch.equal(t, v) for t, v in zip(grads, before))
    check(grads, grads, pk.ssd_grad_clip(plan, 2.0), 2.0, before)


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("shift", [1, 2, 3])
def test_unaligned(dtype, shift):
    """Slices that begin at any element, results at others: nothing beside them is written."""
    base = draw(5, [(20011,), (9,), (8200,)], (dtype,))
    grads = [t[shift:] for t in base]
    to = [torch.full((t.numel() + 8,), float("nan"), dtype=F32, device="cuda") for t in grads]
    outs = [t[5 - shift:5 - shift + g.numel()] for t, g in zip(to, grads)]
    check(grads, outs, pk.ssd_grad_clip(pk.ssd_grad_plan(grads, outs), 0.7), 0.7)
    for t, g in zip(to, grads):
        assert bool(torch.isnan(t[:5 - shift]).all()) and bool(torch.isnan(t[5 - shift + g.numel():]).all())


def test_range_of_the_sum():
    """Squares beyond what fp32 holds, and below: the norm is still theirs."""
    for size in (1e25, 1e-25):
        g = [torch.full((1000,), size, device="cuda"), torch.full((24,), -size, device="cuda")]
        o = [torch.empty_like(t) for t in g]
        norm = pk.ssd_grad_clip(pk.ssd_grad_plan(g, o), 1.0)
        n = math.sqrt(1024 * float(g[0][0].double()) ** 2)
        assert abs(float(norm) - n) <= 4 * U * n
        ref = float(g[0][0].double()) * min(1.0, 1.0 / (n + 1e-6))
        assert abs(float(o[0][0]) - ref) <= 4 * U * ref


def test_not_finite():
    g = [torch.tensor([float("inf"), 1.0, -2.0], device="cuda"), torch.ones(5, device="cuda")]
    o = [torch.empty_like(t) for t in g]
    assert math.isinf(float(pk.ssd_grad_clip(pk.ssd_grad_plan(g, o), 1.0)))
    assert bool(torch.isnan(o[0][0])) and not o[0][1:].any() and not o[1].any()
    g[1][2] = float("nan")
    assert math.isnan(float(pk.ssd_grad_clip(pk.ssd_grad_plan(g, o), 1.0)))
    assert all(bool(torch.isnan(t).all()) for t in o)


def test_zero_gradients_and_norm_alone():
    g = [torch.zeros(100, device="cuda"), torch.zeros(0, device="cuda")]
    assert float(pk.ssd_grad_clip(pk.ssd_grad_plan(g), 1.0)) == 0.0 and not g[0].any()
    h = draw(8, [(999,)], (F32,))
    keep = h[0].clone()
    norm = pk.ssd_grad_clip(pk.ssd_grad_plan(h), math.inf)
    assert torch.equal(h[0], keep) and abs(float(norm) - float(keep.double().norm())) <= 2 * U * float(norm)
    assert float(pk.ssd_grad_clip(pk.ssd_grad_plan([torch.empty(0, device="cuda")]), 1.0)) == 0.0


def test_sum_over_several_lists():
    """What several devices do: their sums added up, each scaled by the factor of all."""
    g = draw(9, SIZES, (F32, B16))
    a, b = pk.ssd_grad_plan(g[:4]), pk.ssd_grad_plan(g[4:])
    before = [t.clone() for t in g]
    s = pk.ssd_grad_norm(a) + pk.ssd_grad_norm(b)
    n1, n2 = pk.ssd_grad_clip(a, 0.3, s), pk.ssd_grad_clip(b, 0.3, s)
    assert torch.equal(n1, n2)
    check(g, g, n1, 0.3, before)


def test_same_bits_again_and_in_a_graph():
    g = draw(10, SIZES * 40, (F32, B16))
    outs = [torch.empty_like(t) for t in g]
    plan = pk.ssd_grad_plan(g, outs)
    s = pk.ssd_grad_norm(plan)
    norm = pk.ssd_grad_clip(plan, 1.0)
    want = [t.clone() for t in outs]
    for _ in range(5):
        assert torch.equal(pk.ssd_grad_norm(plan), s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = pk.ssd_grad_clip(plan, 1.0)
    for k in range(3):
        for t in outs:
            t.fill_(float(k))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, norm) and all(torch.equal(t, v) for t, v in zip(outs, want))
        assert torch.equal(pk.ssd_grad_norm(plan), s)


def test_refusals():
    g = torch.zeros(8, device="cuda")
    for bad in (lambda: pk.ssd_grad_plan([]), lambda: pk.ssd_grad_plan([g], []), lambda: pk.ssd_grad_plan([g.double()]), lambda: pk.ssd_grad_plan([g.cpu()]),
                lambda: pk.ssd_grad_plan([g[::2]]), lambda: pk.ssd_grad_plan([g], [g[:4]]), lambda: pk.ssd_grad_clip(pk.ssd_grad_plan([g]), -1.0),
                lambda: pk.ssd_grad_clip(pk.ssd_grad_plan([g]), float("nan")), lambda: pk.ssd_grad_clip(pk.ssd_grad_plan([g]), 1.0, torch.zeros(1, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
