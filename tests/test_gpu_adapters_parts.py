"""How many bits of the narrow products reach the wide ones: a projection of zeros, so that the results are the low-rank terms alone.  h and g
come in two bf16 parts, 16 bits, so a result is off by its own rounding to bf16 (2^-8 of it at most), 2^-16 of the magnitudes of the term's
products, and the fp32 sums ((8 + sqrt n) 2^-24 of their magnitudes each).  With h and g in one bf16 part the second bound would be 2^-8."""
import numpy as np
import pytest
import torch

import paper_2411_19460_amd as pk
from oracle import adapter_ref
from test_gpu_adapters import BF, dev, draw, host, inside, summed

pytestmark = pytest.mark.gpu

# rows, in, out, rank: each of the kernels that take such a term, forward or for the input's gradient
SHAPES = [(1, 264, 520, 16), (2, 520, 264, 40), (5, 264, 520, 24), (16, 2568, 136, 64), (17, 264, 136, 8), (33, 72, 4384, 40), (33, 72, 10576, 16),
          (33, 5128, 72, 24), (300, 264, 264, 96), (700, 72, 2056, 24), (700, 2056, 72, 16), (2500, 136, 1544, 48), (2500, 1544, 136, 16),
          (5003, 136, 1544, 128), (5003, 1544, 136, 40), (2500, 72, 4872, 8), (4700, 72, 5128, 16), (4700, 72, 5128, 40), (4900, 72, 3352, 24),
          (40, 10248, 2056, 16), (40, 2568, 5640, 72)]


@pytest.mark.parametrize("T,I,O,R", SHAPES)
def test_sixteen_bits_of_the_narrow_products(T, I, O, R):
    n = 3
    x, w, a, b, scale, ids, dout = draw(T + I, T, I, O, R, n, np.arange(T) * 2 % n)
    w[:] = 0
    zero, m = np.zeros_like(w), [np.abs(v) for v in (x, w, a, b, scale)]
    out = adapter_ref.adapter_fwd(x, zero, a, b, scale, ids)["out"]
    dx = adapter_ref.adapter_bwd(x, zero, a, b, scale, ids, dout)["dx"]
    low, up = adapter_ref.adapter_fwd(*m, ids)["out"], adapter_ref.adapter_bwd(*m, ids, np.abs(dout))["dx"]
    plan = pk.ssd_adapter_plan(torch.from_numpy(ids.astype(np.int32)).cuda(), n)
    args = dev(x), dev(w), dev(a), dev(b), dev(scale, torch.float32), plan
    inside("out", host(pk.ssd_adapter_linear_fwd(*args)["out"]), out, BF * np.abs(out) + 1.02 * (2.0 ** -16 + summed(I) + summed(R)) * low)
    got = host(pk.ssd_adapter_linear_bwd(*args, dev(dout), want_dab=False)["dx"])
    inside("dx", got, dx, BF * np.abs(dx) + 1.02 * (2.0 ** -16 + summed(O) + summed(R)) * up)
