"""GPU parity of the low-rank adapters beside a shared projection, element by element against the fp64 oracle.

Bounds, all derived from what is rounded where (u = 2^-24, a sum of n fp32 terms is taken to be off by (8 + sqrt n) u of the sum of their
magnitudes; bf16, of eight significant bits, rounds by up to 2^-8 of a value):
  hidden   the sum over in_dim
  out, dx  one rounding to bf16, the term's low-rank operand once more to bf16, the sums
  da, db   the sum over the rows of products whose low-rank operand is a sum over out_dim or in_dim; nothing in bf16
"""
import numpy as np
import pytest
import torch

import paper_2411_19460_amd as pk
from oracle import adapter_ref
from paper_2411_19460_amd import synth

pytestmark = pytest.mark.gpu
U, BF = 2.0 ** -24, 2.0 ** -8


def summed(n):
    return (8 + np.sqrt(n)) * U


def bf16(a):
    return np.asarray(synth.round_bf16(a), dtype=np.float64)


def dev(a, dtype=torch.bfloat16):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(dtype)


def host(t):
    return t.double().cpu().numpy()


def draw(seed, T, I, O, R, n, ids):
    r = np.random.default_rng(7000 + seed)
    f = r.standard_normal
    x, w = bf16(f((T, I))), bf16(f((O, I)) / np.sqrt(I))
    a, b = bf16(f((n, R, I)) / np.sqrt(I)), bf16(f((n, O, R)) / np.sqrt(R))
    scale = np.float32(0.5 + 1.5 * r.random(n)).astype(np.float64)
    return x, w, a, b, scale, ids, bf16(0.1 * f((T, O)))


def bounds(x, w, a, b, scale, ids, dout):
    """Magnitudes of the sums -> how far each result may be off."""
    I, O, R, T = x.shape[1], w.shape[0], a.shape[1], max(len(x), 1)
    f = adapter_ref.adapter_fwd(x, w, a, b, scale, ids)
    g = adapter_ref.adapter_bwd(x, w, a, b, scale, ids, dout)
    m = [np.abs(v) for v in (x, w, a, b, scale)]
    mf = adapter_ref.adapter_fwd(*m, ids)
    mg = adapter_ref.adapter_bwd(*m, ids, np.abs(dout))
    low, up = mf["out"] - m[0] @ m[1].T, mg["dx"] - np.abs(dout) @ m[1]
    off = {"hidden": summed(I) * mf["hidden"],
           "out": BF * np.abs(f["out"]) + 1.01 * BF * low + (summed(I) + summed(R)) * mf["out"] * 1.01,
           "dx": BF * np.abs(g["dx"]) + 1.01 * BF * up + (summed(O) + summed(R)) * mg["dx"] * 1.01,
           "da": (summed(T) + summed(O) + 2 * U) * mg["da"],
           "db": (summed(T) + summed(I) + 2 * U) * mg["db"]}
    return {**f, **g}, off


def inside(name, got, ref, off):
    assert got.shape == ref.shape, name
    bad = ~(np.abs(got - ref) <= off + 1e-30)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} outside, worst {np.max(np.abs(got - ref) / (off + 1e-30)):.2f} of the bound"


def wide(t, cols, col0):
    """t as a column slice of a wider tensor whose other columns are NaN."""
    v = torch.full((t.shape[0], cols), float("nan"), dtype=t.dtype, device=t.device)
    v[:, col0:col0 + t.shape[1]] = t
    return v[:, col0:col0 + t.shape[1]]


def untouched(view, col0):
    w = view._base
    keep = torch.ones(w.shape[1], dtype=torch.bool)
    keep[col0:col0 + view.shape[1]] = False
    assert bool(torch.isnan(w[:, keep.to(w.device)]).all())


def segments(seed, T, n, pieces, bare=0.0):
    r = np.random.default_rng(seed)
    cuts = np.sort(r.choice(np.arange(1, T), min(pieces - 1, max(T - 1, 0)), replace=False)) if T > 1 and pieces > 1 else []
    ids = np.zeros(T, dtype=np.int64)
    for k, (s, e) in enumerate(zip([0, *cuts], [*cuts, T])):
        ids[s:e] = -1 if r.random() < bare else r.integers(0, n)
    return ids


def scattered(seed, T, n):
    return np.random.default_rng(seed).integers(-1, n, T)


CASES = [
    # rows, in, out, rank, adapters, ids
    (1, 2560, 10576, 16, 8, "scattered"),
    (1, 8, 8, 8, 1, "one"),
    (2, 264, 136, 24, 3, "scattered"),
    (3, 5120, 2560, 64, 5, "scattered"),
    (5, 520, 72, 8, 2, "none"),
    (16, 2560, 3352, 32, 16, "scattered"),
    (16, 6184, 520, 16, 4, "scattered"),     # rows of more pieces than a workgroup has waves
    (17, 768, 1544, 40, 30, "scattered"),
    (33, 1000, 264, 128, 3, "segments"),
    (64, 2560, 1032, 256, 40, "scattered"),
    (65, 1024, 4384, 8, 64, "scattered"),
    (128, 5120, 2560, 32, 3, "segments"),
    (200, 136, 200, 96, 7, "scattered"),
    (256, 2560, 264, 16, 1, "one"),
    (257, 768, 3352, 24, 300, "scattered"),  # more adapters than rows of a tile
    (600, 1024, 4384, 8, 3, "segments"),
    (700, 72, 2056, 72, 2, "alternating"),
    (1905, 5120, 2560, 8, 6, "segments"),
    (2100, 2560, 1544, 64, 3, "segments"),
    (9001, 264, 520, 16, 5, "segments"),     # units of the gradients of more than 512 rows
]


def ids_of(kind, T, n):
    return {"scattered": lambda: scattered(T, T, n), "one": lambda: np.full(T, n - 1), "none": lambda: np.full(T, -1),
            "segments": lambda: segments(T, T, n, 6, 0.2), "alternating": lambda: np.arange(T) % n}[kind]()


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
@pytest.mark.parametrize("sliced", [False, True])
def test_forward_and_backward(case, sliced):
    T, I, O, R, n, kind = case
    d = draw(T + R, T, I, O, R, n, ids_of(kind, T, n))
    ref, off = bounds(*d)
    x, w, a, b = (dev(v) for v in d[:4])
    scale, dout = dev(d[4], torch.float32), dev(d[6])
    plan = pk.ssd_adapter_plan(torch.from_numpy(d[5].astype(np.int32)).cuda(), n)
    out, dx = None, None
    if sliced:
        x, dout = wide(x, I + 24, 8), wide(dout, O + 40, 16)
        out, dx = wide(torch.empty((T, O), dtype=torch.bfloat16, device="cuda"), O + 40, 24), wide(torch.empty_like(x), I + 8, 0)
    f = pk.ssd_adapter_linear_fwd(x, w, a, b, scale, plan, out=out, want_hidden=True)
    inside("hidden", host(f["hidden"]), ref["hidden"], off["hidden"])
    inside("out", host(f["out"]), ref["out"], off["out"])
    again = pk.ssd_adapter_linear_fwd(x, w, a, b, scale, plan)
    assert again["hidden"] is None and torch.equal(again["out"], f["out"])
    g = pk.ssd_adapter_linear_bwd(x, w, a, b, scale, plan, dout, hidden=f["hidden"], dx=dx)
    for k in ("dx", "da", "db"):
        inside(k, host(g[k]), ref[k], off[k])
    if sliced:
        untouched(f["out"], 24)
        untouched(g["dx"], 0)
    # without the forward call's hidden values, and one result alone: the same bits
    g2 = pk.ssd_adapter_linear_bwd(x, w, a, b, scale, plan, dout, want_dx=False)
    assert g2["dx"] is None and torch.equal(g2["da"], g["da"]) and torch.equal(g2["db"], g["db"])
    g3 = pk.ssd_adapter_linear_bwd(x, w, a, b, scale, plan, dout, want_dab=False)
    assert g3["da"] is None and torch.equal(g3["dx"], g["dx"])


def test_gradients_are_added_to_what_is_there():
    T, n = 1300, 4
    d = draw(1, T, 264, 136, 16, n, np.minimum(np.arange(T) // 600, 1) * 2)     # adapters 1 and 3 have no rows
    ref, off = bounds(*d)
    x, w, a, b = (dev(v) for v in d[:4])
    scale, dout = dev(d[4], torch.float32), dev(d[6])
    plan = pk.ssd_adapter_plan(torch.from_numpy(d[5].astype(np.int32)).cuda(), n)
    da, db = torch.full(a.shape, 2.0, device="cuda"), torch.full(b.shape, -3.0, device="cuda")
    g = pk.ssd_adapter_linear_bwd(x, w, a, b, scale, plan, dout, da=da, db=db, flags=pk.SSD_FLAG_ACCUM_PARAM)
    inside("da", host(g["da"]), ref["da"] + 2.0, off["da"] + 2 * U * (np.abs(ref["da"]) + 2))
    inside("db", host(g["db"]), ref["db"] - 3.0, off["db"] + 2 * U * (np.abs(ref["db"]) + 3))
    assert bool((da[1] == 2.0).all()) and bool((db[3] == -3.0).all())
    g = pk.ssd_adapter_linear_bwd(x, w, a, b, scale, plan, dout, da=da, db=db)
    assert not da[1].any() and not db[3].any()
    inside("da", host(g["da"]), ref["da"], off["da"])


@pytest.mark.parametrize("T", [2, 13, 40, 300])
def test_nothing_of_another_adapter_or_row_reaches_a_row(T):
    """An adapter of infinities and NaN, and a row of them: the other rows' bits do not change."""
    I, O, R, n = 264, 520, 24, 3
    x, w, a, b, scale, ids, dout = draw(T, T, I, O, R, n, np.arange(T) % (n + 1) - 1)
    plan = pk.ssd_adapter_plan(torch.from_numpy(ids.astype(np.int32)).cuda(), n)
    sc = dev(scale, torch.float32)

    def both(x, a, b, dout):
        f = pk.ssd_adapter_linear_fwd(dev(x), dev(w), dev(a), dev(b), sc, plan, want_hidden=True)
        g = pk.ssd_adapter_linear_bwd(dev(x), dev(w), dev(a), dev(b), sc, plan, dev(dout), hidden=f["hidden"])
        return f["out"], f["hidden"], g["dx"], g["da"], g["db"]

    clean = both(x, a, b, dout)
    a2, b2 = a.copy(), b.copy()
    a2[1], b2[1] = np.inf, np.nan
    b2[1, ::2] = -np.inf
    other = torch.from_numpy(ids != 1).cuda()
    for u, v in zip(both(x, a2, b2, dout)[:3], clean[:3]):
        assert torch.equal(u[other], v[other])
    for u, v in zip(both(x, a2, b2, dout)[3:], clean[3:]):
        assert torch.equal(u[0], v[0]) and torch.equal(u[2], v[2])
    x2, d2 = x.copy(), dout.copy()
    x2[1], d2[1] = np.nan, np.inf          # a row of adapter 0
    other = torch.arange(T, device="cuda") != 1
    bad = both(x2, a, b, d2)
    for u, v in zip(bad[:3], clean[:3]):
        assert torch.equal(u[other], v[other])
    for u, v in zip(bad[3:], clean[3:]):
        assert torch.equal(u[1:], v[1:])


def test_no_rows():
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    w, a, b = (torch.ones(s, dtype=torch.bfloat16, device="cuda") for s in ((72, 64), (2, 8, 64), (2, 72, 8)))
    scale = torch.ones(2, device="cuda")
    plan = pk.ssd_adapter_plan(torch.empty(0, dtype=torch.int32, device="cuda"), 2)
    assert pk.ssd_adapter_linear_fwd(x, w, a, b, scale, plan)["out"].shape == (0, 72)
    g = pk.ssd_adapter_linear_bwd(x, w, a, b, scale, plan, torch.empty((0, 72), dtype=torch.bfloat16, device="cuda"))
    assert g["dx"].shape == (0, 64) and not g["da"].any() and not g["db"].any()


def test_adapters_outside_the_list_are_none():
    T, n = 40, 3
    d = draw(3, T, 136, 72, 8, n, np.where(np.arange(T) % 3 == 0, -1, np.arange(T) % 3))
    odd = np.where(d[5] < 0, np.array([-7, n, 2 ** 31 - 1, -2 ** 31])[np.arange(T) % 4], d[5])
    x, w, a, b = (dev(v) for v in d[:4])
    scale = dev(d[4], torch.float32)
    one, two = (pk.ssd_adapter_linear_fwd(x, w, a, b, scale, pk.ssd_adapter_plan(torch.from_numpy(i.astype(np.int32)).cuda(), n))["out"]
                for i in (d[5], odd))
    assert torch.equal(one, two)


def test_on_another_stream_and_in_a_graph():
    T, I, O, R, n = 24, 520, 264, 16, 5
    d = draw(4, T, I, O, R, n, scattered(4, T, n))
    x, w, a, b = (dev(v) for v in d[:4])
    scale, dout = dev(d[4], torch.float32), dev(d[6])
    plan = pk.ssd_adapter_plan(torch.from_numpy(d[5].astype(np.int32)).cuda(), n)
    out, dx = torch.empty_like(dout), torch.empty_like(x)
    da, db = (torch.empty(t.shape, device="cuda") for t in (a, b))
    hid = torch.empty((T, R), device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def step():
        pk.ssd_adapter_linear_fwd(x, w, a, b, scale, plan, out=out, hidden=hid)
        pk.ssd_adapter_linear_bwd(x, w, a, b, scale, plan, dout, hidden=hid, dx=dx, da=da, db=db, workspace=ws)

    step()
    want = [t.clone() for t in (out, hid, dx, da, db)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        for t in (out, hid, dx, da, db):
            t.fill_(float(k))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, v) for t, v in zip((out, hid, dx, da, db), want))
        x.mul_(1.0)     # eager work between the replays


def test_refusals():
    x, w, a, b = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((4, 64), (72, 64), (2, 8, 64), (2, 72, 8)))
    scale, dout = torch.ones(2, device="cuda"), torch.zeros((4, 72), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    plan = pk.ssd_adapter_plan(ids, 2)
    fwd, bwd = pk.ssd_adapter_linear_fwd, pk.ssd_adapter_linear_bwd
    for bad in (lambda: fwd(x[:3], w, a, b, scale, plan), lambda: fwd(x, w.float(), a, b, scale, plan), lambda: fwd(x, w, a[:1], b, scale, plan),
                lambda: fwd(x, w, a, b[:, :64], scale, plan), lambda: fwd(x, w, a, b, scale.double(), plan), lambda: fwd(x, w, a, b, scale, None),
                lambda: fwd(x, w, a, b, scale, pk.ssd_adapter_plan(ids, 3)), lambda: fwd(x, w, a, b, scale, plan, out=x),
                lambda: fwd(x, w, a, b, scale, plan, hidden=torch.zeros((4, 16), device="cuda")), lambda: fwd(x, w, a.cpu(), b, scale, plan),
                lambda: bwd(x, w, a, b, scale, plan, dout[:, :64]), lambda: bwd(x, w, a, b, scale, plan, dout, da=torch.zeros(a.shape, device="cuda")),
                lambda: bwd(x, w, a, b, scale, plan, dout, dx=dout), lambda: pk.ssd_adapter_plan(ids.long(), 2), lambda: pk.ssd_adapter_plan(ids.cpu(), 2)):
        with pytest.raises(ValueError):
            bad()
    odd = torch.zeros((2, 12, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 72, 12), dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: fwd(x, w, *odd, scale, plan), lambda: bwd(x, w, a, b, scale, plan, dout, flags=1), lambda: pk.ssd_adapter_plan(ids, 0),
                lambda: fwd(x, w, a, b, scale, plan, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(pk.SSDError):
            bad()
