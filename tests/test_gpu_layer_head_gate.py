"""What the norms behind the mixer leave of the read gate G^Q, which multiplies every head's output vector: a norm over each head
divides it out, a norm over all heads of a token keeps the heads' ratios."""
import numpy as np
import pytest

import oracle
import sla_inputs as si
from gpu_util import RETNET, TOL, rel_err
from layer_util import numpy64, tensor
from oracle import sla_layer as ol

pytestmark = pytest.mark.gpu

B, T, H, DK, DV = 2, 41, 4, 64, 128


def _mixer(seed=5):
    d = si.custom(RETNET, "f32", B=B, T=T, H=H, dk=DK, dv=DV, seed=seed)
    g, _ = si.to_device(d, "f32", RETNET)
    r = np.random.default_rng(seed)
    w, dy = (1 + 0.1 * r.standard_normal(DV)).astype(np.float32), r.standard_normal((B, T, H, DV)).astype(np.float32)
    return d, g, w, dy


def test_a_norm_over_each_head_divides_the_read_gate_out():
    """Two read gates, one read-out (eps = 0), and no gradient for the gate's logits.  Tolerances: the mixer's 1e-4 of the largest value,
    four of them where the norm divides by a head's own size."""
    import torch
    import paper_2602_01744_amd as sla

    d, g, w, dy = _mixer()
    outs, reads = [], []
    for ql in (g["q_logits"], torch.flip(g["q_logits"], dims=(-1,)).contiguous()):
        out, _ = sla.forward(sla.RETNET, g["q"], g["k"], g["v"], ql, g["k_logits"], g["log_decay"])
        outs.append(out)
        reads.append(sla.norm_gate(out, None, tensor(w), gate="none", eps=0.0))
    assert rel_err(numpy64(outs[1]), numpy64(outs[0])) > 0.1
    assert rel_err(numpy64(reads[1]), numpy64(reads[0])) <= 4 * TOL["f32"]
    dx = sla.norm_gate_backward(outs[0], None, tensor(w), tensor(dy), gate="none", eps=0.0)["dx"]
    grads = sla.backward(sla.RETNET, g["q"], g["k"], g["v"], g["q_logits"], g["k_logits"], g["log_decay"], dx)
    terms = (numpy64(dx) * numpy64(outs[0]))
    assert np.max(np.abs(numpy64(grads["dq_head_logits"]))) <= 4 * TOL["f32"] * np.max(np.abs(terms).sum(-1))
    assert np.max(np.abs(numpy64(grads["dk_head_logits"]))) > 1e-2 * np.max(np.abs(terms).sum(-1))


def test_a_norm_over_all_heads_keeps_the_read_gate():
    """join_norm over the H dv values of a token: outputs and gradients, those of both gates' logits among them."""
    import paper_2602_01744_amd as sla

    d, g, w, dy = _mixer(6)
    wide = np.tile(w, H)
    out, _ = sla.forward(sla.RETNET, g["q"], g["k"], g["v"], g["q_logits"], g["k_logits"], g["log_decay"])
    _, y = sla.join_norm(out.view(B, T, H * DV), None, tensor(wide))
    dx = sla.join_norm_backward(out.view(B, T, H * DV), None, tensor(wide), tensor(dy).view(B, T, H * DV))["dx"]
    got = sla.backward(sla.RETNET, g["q"], g["k"], g["v"], g["q_logits"], g["k_logits"], g["log_decay"], dx.view(B, T, H, DV))
    args = [d[n] for n in ("q", "k", "v", "q_logits", "k_logits", "log_decay")]
    O, _ = oracle.forward(RETNET, *args)
    _, Y = ol.join_norm(O.reshape(B, T, -1), None, wide)
    DX = ol.join_norm_backward(O.reshape(B, T, -1), None, wide, dy.reshape(B, T, -1))["dx"]
    want = oracle.backward(RETNET, *args, DX.reshape(B, T, H, DV))
    assert rel_err(numpy64(y), Y.reshape(B, T, -1)) <= 3 * TOL["f32"]
    for n in ("dq", "dk", "dv", "dq_head_logits", "dk_head_logits"):
        e = rel_err(numpy64(got[n]), want[n.replace("_head", "")])
        print(f"[head gate] {n} {e:.2e}", flush=True)
        assert e <= 3 * TOL["f32"], n
    assert np.max(np.abs(want["dq_logits"])) > 0.1 * np.max(np.abs(want["dk_logits"]))
