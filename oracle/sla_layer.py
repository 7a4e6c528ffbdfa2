"""Oracle statements for what stands around the SLA mixer inside a layer, and their gradients, fp64 numpy.  TEST
INFRASTRUCTURE ONLY: the GPU library never imports this module and shares no code with it.

* rotary positions on head vectors: pairs turned by position * frequency (RetNet's queries and keys, Sec. 5.1's baseline);
* the read-out: every head vector over its root mean square, weighted and gated;
* the residual stream's join with a block's output and the norm for the next block.

Every function is the definition written out; gradients are the chain rule line by line, pinned by finite differences.
"""
from __future__ import annotations

import numpy as np


def _f64(a):
    return None if a is None else np.asarray(a, dtype=np.float64)


def rotary(x, positions, frequencies, *, adjacent=False, magnitude=1.0, inverse=False):
    """x [..., H, d] with positions [...] (one for every token): pairs (i, i + r/2), or (2i, 2i+1), of the first
    r = 2 len(frequencies) elements turned by position * frequency (back with inverse) and scaled by magnitude."""
    x = _f64(x)
    f = _f64(frequencies)
    r = 2 * len(f)
    th = _f64(positions)[..., None, None] * f * (-1.0 if inverse else 1.0)
    a = np.arange(0, r, 2) if adjacent else np.arange(r // 2)
    b = a + (1 if adjacent else r // 2)
    y = x.copy()
    y[..., a] = magnitude * (x[..., a] * np.cos(th) - x[..., b] * np.sin(th))
    y[..., b] = magnitude * (x[..., a] * np.sin(th) + x[..., b] * np.cos(th))
    return y


def _sigmoid(g):
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1.0, e) / (1.0 + e)


def _gate(g, kind):
    """(act(g), act'(g))"""
    if kind == "none":
        return 1.0, 0.0
    p = _sigmoid(g)
    return (g * p, p + g * p * (1.0 - p)) if kind == "silu" else (p, p * (1.0 - p))


def _rms(x, eps):
    return np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)


def _rms_backward(x, dn, eps):
    """Gradient of n = x / rms(x) for the cotangent dn of n."""
    s = _rms(x, eps)
    return dn / s - x * np.mean(dn * x, axis=-1, keepdims=True) / s ** 3


def norm_gate(x, g, w, *, gate="silu", eps=1e-5):
    """x, g [..., H, dv]; w [dv], [H,dv] or None."""
    x, g, w = _f64(x), _f64(g), _f64(w)
    return x / _rms(x, eps) * (1.0 if w is None else w) * _gate(g, gate)[0]


def norm_gate_backward(x, g, w, dy, *, gate="silu", eps=1e-5):
    x, g, w, dy = _f64(x), _f64(g), _f64(w), _f64(dy)
    act, dact = _gate(g, gate)
    wt = 1.0 if w is None else w
    n = x / _rms(x, eps)
    dw = None
    if w is not None:
        t = dy * n * act
        dw = t.reshape((-1,) + w.shape).sum(0)
    return {"dx": _rms_backward(x, dy * wt * act, eps), "dg": None if gate == "none" else dy * n * wt * dact, "dw": dw}


def join_norm(x, h, w_before, *, w_after=None, channel_scale=None, scale=1.0, eps=1e-5):
    x, h, wb, wa, c = (_f64(t) for t in (x, h, w_before, w_after, channel_scale))
    if h is not None:
        u = h if wa is None else h / _rms(h, eps) * wa
        x = x + scale * (u if c is None else c * u)
    return x, None if wb is None else x / _rms(x, eps) * wb


def join_norm_backward(x_out, h, w_before, dy, dx_out=None, *, w_after=None, channel_scale=None, scale=1.0, eps=1e-5):
    x, h, wb, wa, c, dy, dxo = (_f64(t) for t in (x_out, h, w_before, w_after, channel_scale, dy, dx_out))
    g = dict.fromkeys(("dx", "dh", "dw_after", "dchannel_scale", "dw_before"))
    dX = np.zeros_like(x) if dxo is None else dxo
    total = lambda t: t.reshape(-1, x.shape[-1]).sum(0)
    if wb is not None:
        g["dw_before"] = total(dy * x / _rms(x, eps))
        dX = dX + _rms_backward(x, dy * wb, eps)
    g["dx"] = dX
    if h is None:
        return g
    u = h if wa is None else h / _rms(h, eps) * wa
    du = scale * dX
    if c is not None:
        g["dchannel_scale"] = total(du * u)
        du = du * c
    if wa is not None:
        g["dw_after"] = total(du * h / _rms(h, eps))
        du = _rms_backward(h, du * wa, eps)
    g["dh"] = du
    return g
