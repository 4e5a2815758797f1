"""The longest batch that the adapters' calls take, and the first that they refuse (CPU: nothing is launched)."""
import ctypes

import pytest

from paper_2411_19460_amd import binding
from test_adapter_abi import P, SHAPE, WORKSPACE, bwd, fwd, shape

MOST = 1 << 27


def test_the_longest_batch():
    L = binding.lib()
    need = L.ssd_adapter_plan_bytes(MOST, 3)
    assert need >= 2 * 4 * MOST                                   # two numbers a row at least
    assert L.ssd_adapter_plan(MOST, 3, P, P, need - 1, None) == WORKSPACE
    s = shape(rows=MOST)
    for call, i in ((fwd, 0), (bwd, 1)):
        need = L.ssd_adapter_workspace_bytes(ctypes.byref(s), i)
        assert need >= 4 * MOST * s.rank                          # the narrow product in two bf16 parts
        assert call(s, nbytes=need - 1) == WORKSPACE


@pytest.mark.parametrize("rows", [MOST + 1, MOST + 256, 1 << 28, (1 << 31) - 1])
def test_longer_ones_are_refused(rows):
    L = binding.lib()
    assert L.ssd_adapter_plan_bytes(rows, 3) == 0
    assert L.ssd_adapter_plan(rows, 3, P, P, 1 << 40, None) == SHAPE
    s = shape(rows=rows)
    assert L.ssd_adapter_workspace_bytes(ctypes.byref(s), 0) == 0 and L.ssd_adapter_workspace_bytes(ctypes.byref(s), 1) == 0
    assert fwd(s) == SHAPE and bwd(s) == SHAPE
