"""Scalar arguments of the operators around the mixer: their value at the call counts, whatever object holds it."""
import numpy as np
import pytest

import paper_2602_01744_amd as sla
from paper_2602_01744_amd import binding


class _Seen(list):
    def __call__(self, call, t, params, *rest):
        self.append(params._obj)


@pytest.fixture
def seen(monkeypatch):
    """The parameter blocks that reach the library, in place of the calls (there is no GPU here)."""
    s = _Seen()
    monkeypatch.setattr(binding, "_run", s)
    return s


def _calls():
    import torch

    x, w, f = torch.zeros(2, 3, 2, 64), torch.ones(64), torch.ones(32, dtype=torch.float64)
    a = torch.zeros(5, 64)
    return [("magnitude", lambda v: sla.rotary(x, None, f, magnitude=v)), ("magnitude", lambda v: sla.rotary_backward(x, None, f, magnitude=v)),
            ("eps", lambda v: sla.norm_gate(x, x, w, eps=v)), ("eps", lambda v: sla.norm_gate_backward(x, x, w, x, eps=v)),
            ("eps", lambda v: sla.join_norm(a, a, w, eps=v)), ("eps", lambda v: sla.join_norm_backward(a, a, w, a, eps=v)),
            ("scale", lambda v: sla.join_norm(a, a, w, scale=v)), ("scale", lambda v: sla.join_norm_backward(a, a, w, a, scale=v))]


@pytest.mark.parametrize("i", range(8))
def test_a_scalar_changed_in_place_is_read_again(seen, i):
    """A learned scale that an optimiser's step changes in its place: tensors hash by identity."""
    import torch

    name, call = _calls()[i]
    for holder in (torch.tensor(0.5), torch.nn.Parameter(torch.tensor(0.5, dtype=torch.float64))):
        for value in (0.5, 2.0, 0.25):
            with torch.no_grad():
                holder.fill_(value)
            call(holder)
            assert getattr(seen[-1], name) == value
    for value in (0.5, np.float32(2.0), np.float64(0.25), np.array(0.125), 1):
        call(value)
        assert getattr(seen[-1], name) == float(value)


def test_what_is_no_number_is_refused(seen):
    for _, call in _calls():
        for bad in ("half", [0.5], object()):
            with pytest.raises((ValueError, TypeError)):
                call(bad)
    assert not seen


def test_caches_hold_no_tensor(seen):
    """A parameter that a call was given can be freed afterwards."""
    import gc
    import weakref

    import torch

    for _, call in _calls():
        s = torch.tensor(0.75)
        gone = weakref.ref(s)
        call(s)
        del s
        gc.collect()
        assert gone() is None


def test_a_scale_that_changes_every_step_asks_for_the_workspace_once(monkeypatch, seen):
    import torch

    asked = []
    query = binding.sla_join_norm_backward_workspace_bytes
    monkeypatch.setattr(binding, "sla_join_norm_backward_workspace_bytes", lambda p, packed: asked.append(p) or query(p, packed))
    binding._workspace_size.cache_clear()
    a, w = torch.zeros(5, 64), torch.ones(64)
    for step in range(4):
        sla.join_norm_backward(a, a, w, a, scale=1.0 + step)
    assert len(asked) == 1
