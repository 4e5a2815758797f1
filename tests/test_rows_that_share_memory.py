"""Rows at a distance of zero (a broadcast row) are refused by every call that takes rows with a stride, before anything is launched: the C ABI
takes 0 as dense and would read, or write, rows that are not there.  The tensors are stand-ins: nothing here needs a device."""
import pytest
import torch

from paper_2411_19460_amd import binding


class Rows:
    """What the checks look at, of a device tensor that the CPU cannot hold."""
    is_cuda = True

    def __init__(self, rows, dim, stride, dtype=torch.bfloat16):
        self.shape, self.strides, self.dtype, self.device = torch.Size((rows, dim)), stride, dtype, torch.device("cuda", 0)

    def dim(self):
        return 2

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def get_device(self):
        return 0

    def is_contiguous(self):
        return self.strides == (self.shape[1], 1) or self.shape[0] <= 1

    def data_ptr(self):
        raise AssertionError("a refused call looks at no address")


def dense(rows, dim, **kw):
    return Rows(rows, dim, (dim, 1), **kw)


def broadcast(rows, dim, **kw):
    return Rows(rows, dim, (0, 1), **kw)


def test_rows_with_a_stride_of_their_own_are_taken():
    assert binding._rows_view(dense(5, 64), "x") == 64 and binding._rows_view(Rows(5, 64, (200, 1)), "x") == 200
    assert binding._rows_view(broadcast(1, 64), "x") == 64 and binding._rows_view(Rows(0, 64, (0, 1)), "x") == 64
    s = binding._norm_shape(Rows(5, 64, (72, 1)), Rows(5, 64, (200, 1)), 1, 1e-5)
    assert (s.y_row_stride, s.z_row_stride) == (72, 200)
    assert binding._norm_shape(dense(5, 64), None, 1, 1e-5).z_row_stride == 64


@pytest.mark.parametrize("t", [broadcast(2, 64), broadcast(40, 64), Rows(3, 64, (8, 1))])
def test_rows_that_share_memory_are_refused(t):
    rows, w = t.shape[0], dense(72, 64)
    calls = [lambda: binding._rows_view(t, "x"), lambda: binding.ssd_linear_fwd(t, w), lambda: binding.ssd_linear_bwd(t, w, dense(rows, 72)),
             lambda: binding.ssd_linear_bwd(dense(rows, 72), dense(64, 72), t), lambda: binding._norm_shape(t, None, 1, 1e-5),
             lambda: binding._norm_shape(dense(rows, 64), t, 1, 1e-5), lambda: binding.ssd_gated_norm_fwd(t, None, None)]
    for call in calls:
        with pytest.raises(ValueError, match="share memory"):
            call()


@pytest.mark.parametrize("which", ["x", "out", "dout", "dx"])
def test_adapters_refuse_them(which):
    T, I, O, R, n = 4, 64, 72, 8, 2

    class Dense(Rows):
        def __init__(self, *shape, dtype=torch.bfloat16):
            super().__init__(4, 4, None, dtype)
            self.shape, self.strides = torch.Size(shape), torch.empty(shape, device="meta").stride()

        def dim(self):
            return len(self.shape)

        def is_contiguous(self):
            return True

    plan = binding.AdapterPlan(Dense(64, dtype=torch.uint8), T, n)
    t = {"x": dense(T, I), "out": None, "dout": dense(T, O), "dx": None}
    t[which] = broadcast(T, I if which in ("x", "dx") else O)
    fixed = (Dense(O, I), Dense(n, R, I), Dense(n, O, R), Dense(n, dtype=torch.float32), plan)
    with pytest.raises(ValueError, match="share memory"):
        if which in ("x", "out"):
            binding.ssd_adapter_linear_fwd(t["x"], *fixed, out=t["out"])
        else:
            binding.ssd_adapter_linear_bwd(t["x"], *fixed, t["dout"], dx=t["dx"])
