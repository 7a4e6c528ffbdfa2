"""The gates of the read-out and their slopes over the whole range that fp32 holds, against values formed without cancellation in 64
bits."""
import numpy as np
import pytest

from layer_util import K, numpy64, rounded, tensor, within

pytestmark = pytest.mark.gpu


def _gate(g, kind):
    """act(g), act'(g), and the sum of the absolute terms of act'(g): e / (1 + e)^2 for the sigmoid, with e = exp(-|g|)."""
    e = np.exp(-np.abs(g))
    p = np.where(g >= 0, 1.0, e) / (1.0 + e)
    rest = np.where(g >= 0, e, 1.0) / (1.0 + e)  # 1 - p
    if kind == "sigmoid":
        return p, p * rest, p * rest
    return g * p, p * (1.0 + g * rest), p * (1.0 + np.abs(g) * rest)


def _case(dtype, kind, seed):
    import paper_2602_01744_amd as sla

    r = np.random.default_rng(seed)
    g = rounded(np.concatenate([np.linspace(-85, 85, 768), np.linspace(-20, 20, 768)]).reshape(1, 6, 4, 64), dtype)
    x, dy = rounded(r.standard_normal(g.shape), dtype), rounded(1 + r.random(g.shape), dtype)
    w = (1 + 0.25 * r.standard_normal(64)).astype(np.float32)
    y = sla.norm_gate(tensor(x, dtype), tensor(g, dtype), tensor(w), gate=kind)
    got = sla.norm_gate_backward(tensor(x, dtype), tensor(g, dtype), tensor(w), tensor(dy, dtype), gate=kind)
    x, g, dy = (t.astype(np.float64) for t in (x, g, dy))
    n = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + 1e-5)
    return y, got["dg"], n * w, dy, g


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["sigmoid", "silu"])
def test_slopes_of_open_and_closed_gates(dtype, kind):
    """dg relative to the slope itself: e^-|g| where the sigmoid is nearly open or nearly closed."""
    _, dg, nw, dy, g = _case(dtype, kind, 1)
    _, slope, terms = _gate(g, kind)
    t = np.abs(dy * nw)
    # K for the norm, 2 |g| for the exponential
    within("dg", dg, dy * nw * slope, t * terms * (1 + 2 * np.abs(g) / K), dtype)
