"""The join where a workgroup walks several rows and gates end inside its rows, against the fp64 oracle: forward, backward and every parameter's sums.

Rows are cut into parts of equal length, forward and backward each in its own way; the lengths that the cases give are named beside them.  The sums of the
parameters run over the rows of a part one after another (32 at most here), then over the parts, 2048 at most: 128 additions one after another in each of sixteen
waves and 16 more.  That is less than the 512 + 80 roundings that the bounds of `compare` allow for."""
import pytest

import paper_2411_19460_amd as pk
from test_gpu_join import TYPES, compare, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,D,gate_rows", [
    (4097, 72, 3), (4097, 72, 7),           # forward 2 rows a part, backward 5: gates begin inside both
    (5000, 72, 3), (5000, 72, 7),
    (9000, 72, 7), (9000, 71, 4),           # 3 and 8
    (20000, 72, 3), (20000, 72, 7), (20000, 72, 1001), (20000, 69, 13),     # 5 and 10, eight parts a compute unit backward
    (40000, 72, 10001), (40000, 72, 0),     # 10 and 20
    (2100, 1032, 4), (2100, 1032, 1),       # three waves a row: 2 and 4
    (1100, 2561, 4), (1100, 2561, 0),       # six waves, off the vectors: 3 and 4
    (700, 4104, 7), (700, 4104, 2), (700, 4104, 0)])                        # nine waves, a part a compute unit: 3 and 3
def test_gates_inside_parts(T, D, gate_rows):
    flags = pk.SSD_FLAG_ACCUM_PARAM if gate_rows in (1, 2, 3, 10001) else 0
    compare(draw(T + D + gate_rows, "bf16", "bf16", T, D, gate_rows=gate_rows), "bf16", "bf16", gate_rows, 0.1, flags=flags)


@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("alpha", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.2])
def test_gates_inside_parts_of_every_type(dtype, stream, alpha, p):
    compare(draw(1, dtype, stream, 4500, 136, gate_rows=7, alpha=alpha), dtype, stream, 7, p)
    compare(draw(2, dtype, stream, 2100, 513, post=False, gate_rows=11, alpha=alpha), dtype, stream, 11, p)


@pytest.mark.parametrize("gate_rows,flags", [(0, 0), (1, 0), (2, pk.SSD_FLAG_ACCUM_PARAM), (4, 0), (7, pk.SSD_FLAG_ACCUM_PARAM), (299, 0)])
def test_wide_rows(gate_rows, flags):
    """More than 8192 values: three rows a part; gates end inside one, begin in one and go on behind it, and lie in several."""
    compare(draw(gate_rows, "bf16", "bf16", 600, 8200, gate_rows=gate_rows), "bf16", "bf16", gate_rows, 0.1, flags=flags)


@pytest.mark.parametrize("dtype,stream", TYPES)
def test_wide_rows_of_every_type(dtype, stream):
    compare(draw(3, dtype, stream, 520, 8195, gate_rows=7), dtype, stream, 7, 0.2, pad=(1, 2))        # three rows a part


@pytest.mark.parametrize("T,D,gate_rows", [(65536, 100, 1001), (16384, 512, 0), (5000, 1024, 700)])
def test_sums_of_many_rows(T, D, gate_rows):
    compare(draw(T, "bf16", "bf16", T, D, gate_rows=gate_rows), "bf16", "bf16", gate_rows, 0.1)
