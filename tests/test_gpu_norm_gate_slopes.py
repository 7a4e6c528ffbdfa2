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


@pytest.mark.parametrize("kind", ["sigmoid", "silu"])
def test_exponentials_of_far_gates_in_fp32(kind):
    """The exponential's error does not grow with |g|.  Rows of ones and eps = 0 make the norm exact, so what is left is the gate's:
    2 steps each for exp2 and the reciprocal, one each for the exponent's correction, 1 + e and every product; 12 in all, and 16 in
    the slopes, whose terms are a product more."""
    import torch
    import paper_2602_01744_amd as sla

    g = np.linspace(-86, 86, 64 * 256).astype(np.float32).reshape(1, 64, 4, 64)
    gt = tensor(g)
    one = torch.ones_like(gt)
    y = sla.norm_gate(one, gt, None, gate=kind, eps=0.0)
    dg = sla.norm_gate_backward(one, gt, None, one, gate=kind, eps=0.0)["dg"]
    act, slope, terms = _gate(g.astype(np.float64), kind)
    within("y", y, act, np.abs(act), "f32", steps=12)
    within("dg", dg, slope, terms, "f32", steps=16)


def test_infinite_gates():
    """The limits where they exist: closed and open sigmoids, an open SiLU; NaN stays in its place."""
    import torch
    import paper_2602_01744_amd as sla

    inf = float("inf")
    for dtype in (torch.float32, torch.bfloat16):
        g = torch.tensor([inf, -inf, float("nan"), 3e38, -3e38, 0.0, 90.0, -90.0], device="cuda").repeat(8).view(1, 1, 1, 64).to(dtype).contiguous()
        one = torch.ones_like(g)
        y = sla.norm_gate(one, g, None, gate="sigmoid", eps=0.0)[0, 0, 0, :8].float().tolist()
        assert y[:2] == [1.0, 0.0] and np.isnan(y[2]) and y[3:7] == [1.0, 0.0, 0.5, 1.0] and 0 <= y[7] < 1e-38
        d = sla.norm_gate_backward(one, g, None, one, gate="sigmoid", eps=0.0)["dg"][0, 0, 0, :8].float().tolist()
        assert d[:2] == [0.0, 0.0] and np.isnan(d[2]) and d[3:6] == [0.0, 0.0, 0.25] and max(d[6:]) < 1e-38
        y = sla.norm_gate(one, g, None, gate="silu", eps=0.0)[0, 0, 0, :8].float().tolist()
        assert y[0] == inf and np.isnan(y[2]) and y[3] == float(g[0, 0, 0, 3]) and y[4] == 0 and y[5:7] == [0.0, 90.0]
        d = sla.norm_gate_backward(one, g, None, one, gate="silu", eps=0.0)["dg"][0, 0, 0, :8].float().tolist()
        assert np.isnan(d[2]) and d[3:6] == [1.0, 0.0, 0.5] and d[6] == 1.0 and abs(d[7]) < 1e-36
