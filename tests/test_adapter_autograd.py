"""The differentiable face of the adapters (CPU): what it has no gradient for is refused, not left without one."""
import pytest
import torch

import paper_2411_19460_amd as pk
from paper_2411_19460_amd import binding


def operands():
    shapes = dict(x=(4, 64), w=(72, 64), a=(2, 8, 64), b=(2, 72, 8))
    return {**{k: torch.zeros(s, dtype=torch.bfloat16) for k, s in shapes.items()}, "scale": torch.ones(2), "plan": None}


@pytest.mark.parametrize("name", ["w", "scale"])
def test_constants_that_require_a_gradient(name):
    t = operands()
    t[name].requires_grad_()
    with pytest.raises(ValueError, match=f"{name} requires a gradient"):
        pk.adapter_linear(**t)
    # nothing is recorded here, so nothing is lost: the call gets as far as its next check (of the plan)
    with torch.no_grad(), pytest.raises(ValueError, match="plan"):
        pk.adapter_linear(**t)


@pytest.fixture
def on_cpu(monkeypatch):
    """One adapter that every row has, computed by torch in place of the C ABI's calls."""
    def fwd(x, w, a, b, scale, plan, want_hidden=False):
        h = scale[0] * (x.float() @ a[0].float().t())
        return {"out": (x.float() @ w.float().t() + h @ b[0].float().t()).bfloat16(), "hidden": h if want_hidden else None}

    def bwd(x, w, a, b, scale, plan, dout, hidden=None, want_dx=True, want_dab=True):
        d, x = dout.float(), x.float()
        g = scale[0] * (d @ b[0].float())
        h = scale[0] * (x @ a[0].float().t())
        return {"dx": (d @ w.float() + g @ a[0].float()).bfloat16() if want_dx else None, "da": (g.t() @ x)[None] if want_dab else None,
                "db": (d.t() @ h)[None] if want_dab else None}

    monkeypatch.setattr(binding, "ssd_adapter_linear_fwd", fwd)
    monkeypatch.setattr(binding, "ssd_adapter_linear_bwd", bwd)


def test_a_gradient_of_a_gradient_is_an_error(on_cpu):
    """out is bilinear in x and a: d(dx)/da is not zero, and it was taken to be."""
    r = lambda *s: torch.randn(s, generator=torch.Generator().manual_seed(sum(s))).bfloat16()
    x, a, b = r(4, 64).requires_grad_(), r(1, 8, 64).requires_grad_(), r(1, 72, 8).requires_grad_()
    out = pk.adapter_linear(x, r(72, 64), a, b, torch.ones(1), None)
    (dx,) = torch.autograd.grad(out.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="differentiate twice"):
        dx.float().square().sum().backward()


@pytest.mark.parametrize("begin", [0, 1, 3, 8])
def test_gradients_that_begin_anywhere(on_cpu, monkeypatch, begin):
    """out joined with something else: its gradient is a piece of the whole one, at any element."""
    seen, plain = [], binding.ssd_adapter_linear_bwd

    def bwd(x, w, a, b, scale, plan, dout, *args, **kw):
        seen.append((dout.data_ptr() % 16, dout.is_contiguous()))
        return plain(x, w, a, b, scale, plan, dout, *args, **kw)

    monkeypatch.setattr(binding, "ssd_adapter_linear_bwd", bwd)
    r = lambda *s: torch.randn(s, generator=torch.Generator().manual_seed(sum(s))).bfloat16()
    x, w, a, b, one = r(4, 64).requires_grad_(), r(72, 64), r(1, 8, 64), r(1, 72, 8), torch.ones(1)
    dout = r(begin + 4 * 72)
    torch.cat([torch.zeros(begin, dtype=torch.bfloat16), pk.adapter_linear(x, w, a, b, one, None).flatten()]).backward(dout)
    assert seen == [(0, True)]
    assert torch.equal(x.grad, plain(x, w, a, b, one, None, dout[begin:].view(4, 72))["dx"])


def test_gradients_are_added_to_what_is_given_alone():
    """Without da and db the sums would be added to memory that nobody has written."""
    t = operands()
    with pytest.raises(ValueError, match="SSD_FLAG_ACCUM_PARAM"):
        pk.ssd_adapter_linear_bwd(**t, dout=torch.zeros((4, 72), dtype=torch.bfloat16), flags=pk.SSD_FLAG_ACCUM_PARAM)
