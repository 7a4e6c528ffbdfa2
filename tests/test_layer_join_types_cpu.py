"""The type that a caller asks of the join's norm: given where nothing else decides it, refused where it contradicts what does."""
import pytest

import paper_2602_01744_amd as sla
from paper_2602_01744_amd import binding


def test_a_contradicted_y_dtype_is_refused(monkeypatch):
    import torch

    ran = []
    monkeypatch.setattr(binding, "_run", lambda *a: ran.append(a))  # there is no GPU here
    f32, bf16 = torch.float32, torch.bfloat16
    x, w = torch.zeros(4, 64), torch.ones(64)
    h = {t: torch.zeros(4, 64, dtype=t) for t in (f32, bf16)}
    for bad in (lambda: sla.join_norm(x, h[bf16], w, y_dtype=f32), lambda: sla.join_norm(x, h[f32], w, y_dtype=bf16),
                lambda: sla.join_norm(x, None, w, y=torch.zeros_like(h[bf16]), y_dtype=f32),
                lambda: sla.join_norm(x, h[bf16], w, y=torch.zeros_like(h[bf16]), y_dtype=f32)):
        with pytest.raises(ValueError):
            bad()
    assert not ran
    for t in (f32, bf16):
        assert sla.join_norm(x, h[t], w, y_dtype=t)[1].dtype is t and sla.join_norm(x, h[t], w)[1].dtype is t
        assert sla.join_norm(x, None, w, y_dtype=t)[1].dtype is t
        y = torch.zeros_like(h[t])
        assert sla.join_norm(x, None, w, y=y, y_dtype=t)[1] is y and sla.join_norm(x, None, w, y=y)[1] is y
    assert sla.join_norm(x, None, w)[1].dtype is f32
    assert sla.join_norm(x, h[bf16], None, y_dtype=f32)[1] is None  # there is no y
