"""Norms without an epsilon of vectors whose mean square lies under fp32's normal range, in the read-out and the join."""
import numpy as np
import pytest

from layer_util import K, STEP, numpy64, rounded, tensor, within
from oracle import sla_layer as ol

pytestmark = pytest.mark.gpu

# root mean squares: 1.08e-19 is the border of mean squares in the normal range; squares are held to 2^-149
SIZES = [3e-19, 1.2e-19, 1.0e-19, 3e-20, 1e-20, 1e-21]


def _steps(x):
    """A vector's error in steps of 2^-24: K, and from squares (and their mean) that are off by half of 2^-149 each, of which the
    root takes half.  |x| in [1/2, 3/2] of its size, so no square vanishes beside the others."""
    ms = np.mean(x.astype(np.float64) ** 2, -1, keepdims=True)
    return K + 2.0 ** -149 / ms / STEP


def _vectors(seed, lead, width, dtype):
    r = np.random.default_rng(seed)
    x = (0.5 + r.random((len(SIZES),) + lead + (width,))) * np.where(r.random((len(SIZES),) + lead + (width,)) < 0.5, -1, 1)
    return rounded(x * np.array(SIZES).reshape((-1,) + (1,) * (len(lead) + 1)), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,dv", [(4, 64), (1, 256), (3, 40)])
def test_read_out(dtype, H, dv):
    import paper_2602_01744_amd as sla

    x = _vectors(dv, (3, H), dv, dtype)
    r = np.random.default_rng(1)
    g, dy = rounded(r.standard_normal(x.shape), dtype), rounded(1e-12 * r.standard_normal(x.shape), dtype)
    w = (1 + 0.25 * r.standard_normal(dv)).astype(np.float32)
    y = sla.norm_gate(tensor(x, dtype), tensor(g, dtype), tensor(w), eps=0.0)
    want = ol.norm_gate(x, g, w, eps=0.0)
    within("y", y, want, np.abs(want) * (_steps(x) + 2 * np.abs(g)), dtype, steps=1)
    got = sla.norm_gate_backward(tensor(x, dtype), tensor(g, dtype), tensor(w), tensor(dy, dtype), eps=0.0)
    want = ol.norm_gate_backward(x, g, w, dy, eps=0.0)
    x64, dy64 = x.astype(np.float64), dy.astype(np.float64)
    s = np.sqrt(np.mean(x64 * x64, -1, keepdims=True))
    act, _ = ol._gate(g.astype(np.float64), "silu")
    n, dn = x64 / s, np.abs(dy64 * w * act)
    within("dx", got["dx"], want["dx"], (dn + np.abs(n) * np.mean(np.abs(n) * dn, -1, keepdims=True)) / s * (3 * _steps(x) + 2 * np.max(np.abs(g))), dtype, steps=1)


@pytest.mark.parametrize("types", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("D", [64, 1000, 8200])
def test_join(types, D):
    """The norm of the stream alone, and a tiny block's output behind its own norm."""
    import torch
    import paper_2602_01744_amd as sla

    ht, xt = types
    el = torch.bfloat16 if ht == "bf16" else torch.float32
    x = _vectors(D, (2,), D, xt)
    w = (1 + 0.25 * np.random.default_rng(2).standard_normal(D)).astype(np.float32)
    _, y = sla.join_norm(tensor(x, xt), None, tensor(w), eps=0.0, y_dtype=el)
    _, want = ol.join_norm(x, None, w, eps=0.0)
    within("y", y, want, np.abs(want) * _steps(x), ht, steps=1)
    h = _vectors(D + 1, (2,), D, ht)
    xo, _ = sla.join_norm(torch.zeros(h.shape, device="cuda", dtype=torch.bfloat16 if xt == "bf16" else torch.float32), tensor(h, ht), None,
                          w_after=tensor(w), eps=0.0)
    want, _ = ol.join_norm(np.zeros(h.shape), h, None, w_after=w, eps=0.0)
    within("x_out", xo, want, np.abs(want) * _steps(h), xt, steps=1)
    dy = rounded(1e-12 * np.random.default_rng(3).standard_normal(x.shape), ht)
    got = sla.join_norm_backward(tensor(x, xt), None, tensor(w), tensor(dy, ht), eps=0.0)
    want = ol.join_norm_backward(x, None, w, dy, eps=0.0)
    x64 = x.astype(np.float64)
    s = np.sqrt(np.mean(x64 * x64, -1, keepdims=True))
    n, dn = np.abs(x64 / s), np.abs(dy.astype(np.float64) * w)
    within("dx", got["dx"], want["dx"], (dn + n * np.mean(n * dn, -1, keepdims=True)) / s * 3 * _steps(x), xt, steps=1)


def test_rows_of_zeros_without_an_epsilon_stay_undefined_and_to_themselves():
    """0 / 0: NaN there as in the formula, and in no other row."""
    import torch
    import paper_2602_01744_amd as sla

    x = torch.randn(5, 3, 64, device="cuda")
    x[2, 1] = 0.0
    y = sla.norm_gate(x, None, None, gate="none", eps=0.0)
    bad = torch.isnan(y).any(-1)
    assert bool(torch.isnan(y[2, 1]).all()) and int(bad.sum()) == 1
