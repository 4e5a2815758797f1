"""Ranks that leave the last block of a workgroup's ranks in part empty, at widths where the waves' groups of k end with the projection's
output: what a lane asks for beyond its rows must not be used, nor lie beyond the adapters.  Bounds as in test_gpu_adapters.py."""
import pytest

from test_gpu_adapters import draw, ids_of
from test_gpu_adapters_sets import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,I,O,R,n", [(4100, 264, 2048, 8, 3), (4100, 136, 2048, 24, 5), (4100, 136, 2048, 96, 2), (4100, 264, 1024, 72, 4),
                                       (2000, 136, 2048, 40, 8), (5000, 72, 768, 40, 3), (300, 72, 2640, 8, 2), (4200, 72, 10576, 72, 2)])
def test_partly_empty_blocks_of_ranks(T, I, O, R, n):
    ids = ids_of("segments", T, n)
    check(draw(T + R, T, I, O, R, n, ids), ids, n)
