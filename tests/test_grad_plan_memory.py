"""A plan of gradients keeps the memory alive whose addresses it holds, whatever the tensors are given afterwards (CPU: nothing is launched)."""
import weakref

import torch

from paper_2411_19460_amd import binding


class Memory:
    """Stands for a tensor's storage."""


class Gradient:
    """A tensor whose memory can be exchanged."""

    def __init__(self):
        self.memory = Memory()

    def untyped_storage(self):
        return self.memory


def test_memory_that_the_tensors_let_go_of():
    grads, outs = [Gradient(), Gradient()], [Gradient(), Gradient()]
    was = [weakref.ref(t.memory) for t in (*grads, *outs)]
    plan = binding.GradPlan(None, 2, grads, outs)
    for t in (*grads, *outs):
        t.memory = Memory()                       # what t.data = ... does
    assert all(m() is not None for m in was)
    del plan
    assert all(m() is None for m in was)


def test_memory_of_tensors():
    """The same with real ones: the plan's storages are the first, not the tensors' present ones."""
    g = [torch.arange(8.0), torch.ones(5)]
    first = [t.data_ptr() for t in g]
    plan = binding.GradPlan(None, 2, g, g)
    for t in g:
        t.data = torch.zeros_like(t)
    assert [m.data_ptr() for m in plan._memory] == first and all(t.data_ptr() not in first for t in g)
