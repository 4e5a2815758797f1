"""The kernels of the wide products, each at a shape that takes it.  Long batches: 128 x 128 tiles, 256-row tiles of each width, of two widths
in one launch, with and without the other factor packed, and K in slices, forward and for the input's gradient; a few rows whose products
go by in several turns.  Bounds as in test_gpu_adapters.py."""
import numpy as np
import pytest
import torch

from test_gpu_adapters import dev, draw, ids_of, untouched, wide
from test_gpu_adapters_sets import check, run

pytestmark = pytest.mark.gpu

CASES = [
    # rows, in, out, rank, adapters, ids; what runs forward | for the input's gradient (256-row tiles: their columns)
    (4700, 72, 5128, 16, 4, "segments"),       # 256 and 192 | slices, 128
    (4700, 72, 5128, 40, 4, "scattered"),      # the same, packed
    (4900, 72, 3352, 24, 3, "segments"),       # 192 and 128 | 64 x 64
    (4900, 72, 3352, 64, 70, "scattered"),     # the same, packed, more adapters than lanes
    (2500, 72, 4872, 8, 5, "segments"),        # 256 |
    (2500, 136, 1544, 48, 70, "scattered"),    # 128, packed |
    (5003, 136, 1544, 128, 3, "segments"),     # 192, packed |
    (2500, 1544, 136, 16, 4, "scattered"),     # | 128
    (5003, 1544, 136, 40, 300, "scattered"),   # | 256
    (700, 72, 2056, 24, 9, "scattered"),       # 128 x 128 |
    (700, 2056, 72, 24, 9, "scattered"),       # | 128 x 128
    (37, 10248, 2056, 16, 5, "scattered"),     # slices, 128 |
    (300, 5120, 4384, 8, 3, "segments"),       # slices, 192 |
    (100, 10248, 5640, 16, 6, "scattered"),    # slices, 256 | slices, 256
    (512, 5120, 2560, 24, 4, "segments"),      # slices, 128 | 128 x 128
    (9001, 72, 4104, 24, 5, "segments"),       # gradients of ranks 17 to 32 in a workgroup of one part
    (1, 10248, 520, 16, 2, "one"),             # a row of more pieces than a workgroup has waves
    (2, 6152, 264, 24, 3, "scattered"),
    (2, 1288, 12808, 8, 2, "one"),
    (3, 1288, 32776, 16, 3, "scattered"),      # three to eight rows against very many outputs: few waves, several turns
    (6, 2048, 32776, 40, 2, "scattered"),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_forward_and_backward(case):
    T, I, O, R, n, kind = case
    ids = ids_of(kind, T, n)
    check(draw(T + R, T, I, O, R, n, ids), ids, n)


@pytest.mark.parametrize("case", [CASES[1], CASES[2], CASES[7], CASES[9], CASES[11]], ids=lambda c: "x".join(map(str, c)))
def test_column_slices(case):
    """Inputs and results as column slices of wider tensors of NaN: the bits of dense ones, and nothing beside them is written."""
    T, I, O, R, n, kind = case
    ids = ids_of(kind, T, n)
    x, w, a, b, scale, _, dout = (dev(v) if v.ndim > 1 else v for v in draw(T, T, I, O, R, n, ids))
    scale = dev(scale, torch.float32)
    dense = run(x, w, a, b, scale, ids, dout, n)
    out, dx = wide(torch.empty_like(dout), O + 40, 24), wide(torch.empty_like(x), I + 8, 0)
    got = run(wide(x, I + 24, 8), w, a, b, scale, ids, wide(dout, O + 16, 16), n, out=out, dx=dx)
    for name in ("hidden", "out", "dx", "da", "db"):
        assert torch.equal(got[name], dense[name]), name
    untouched(out, 24)
    untouched(dx, 0)


@pytest.mark.parametrize("T,I,O,R", [(700, 72, 2056, 24), (700, 2056, 72, 24), (2500, 136, 1544, 48), (2500, 1544, 136, 16), (5003, 136, 1544, 16),
                                     (5003, 1544, 136, 40), (2500, 72, 4872, 8), (4700, 72, 5128, 40), (4900, 72, 3352, 24), (37, 10248, 2056, 16),
                                     (40, 2568, 5640, 16), (100, 10248, 5640, 16)])
def test_nothing_of_another_adapter_or_row_reaches_a_row(T, I, O, R):
    """An adapter of infinities and NaN, and a row of them, among the rows of each of these tiles: the other rows' bits do not change."""
    n = 3
    x, w, a, b, scale, ids, dout = draw(T + 1, T, I, O, R, n, np.arange(T) % (n + 1) - 1)
    x, w, a, b, scale, dout = dev(x), dev(w), dev(a), dev(b), dev(scale, torch.float32), dev(dout)
    clean = run(x, w, a, b, scale, ids, dout, n)
    a2, b2 = a.clone(), b.clone()
    a2[1], b2[1], b2[1, ::2] = np.inf, np.nan, -np.inf
    other = torch.from_numpy(ids != 1).cuda()
    got = run(x, w, a2, b2, scale, ids, dout, n)
    for name in ("hidden", "out", "dx"):
        assert torch.equal(got[name][other], clean[name][other]), name
    for name in ("da", "db"):
        assert torch.equal(got[name][0], clean[name][0]) and torch.equal(got[name][2], clean[name][2]), name
    x2, d2 = x.clone(), dout.clone()
    x2[1], d2[1] = np.nan, np.inf          # a row of adapter 0
    other = torch.arange(T, device="cuda") != 1
    got = run(x2, w, a, b, scale, ids, d2, n)
    for name in ("hidden", "out", "dx"):
        assert torch.equal(got[name][other], clean[name][other]), name
    for name in ("da", "db"):
        assert torch.equal(got[name][1:], clean[name][1:]), name
