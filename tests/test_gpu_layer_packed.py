"""Packed batches of very many sequences through the operators around the mixer: what they compute does not depend on where
sequences end (rotary positions apart), so every result is that of one row of all tokens."""
import numpy as np
import pytest

from layer_util import numpy64, tensor, within
from oracle import sla_layer as ol

pytestmark = pytest.mark.gpu


def _offsets(rng, T, B):
    """cu_seqlens of B sequences over T tokens, most of them of a few tokens and many of them empty."""
    cuts = np.sort(rng.integers(0, T + 1, size=B - 1))
    return np.concatenate([[0], cuts, [T]]).astype(np.int32)


# B * T past 2^30, 2^31 and 2^32
@pytest.mark.parametrize("T,B", [(65536, 16385), (65536, 40001), (65600, 131072)])
@pytest.mark.parametrize("weight", ["shared", "heads"])
def test_read_out(T, B, weight):
    import torch
    import paper_2602_01744_amd as sla

    rng = np.random.default_rng(B)
    cu = torch.from_numpy(_offsets(rng, T, B)).cuda()
    x, g, dy = (torch.randn(T, 4, 16, device="cuda").bfloat16() for _ in range(3))
    w = 1 + 0.1 * torch.randn(*((4, 16) if weight == "heads" else (16,)), device="cuda")
    assert torch.equal(sla.norm_gate(x, g, w, cu_seqlens=cu), sla.norm_gate(x[None], g[None], w)[0])
    got, want = sla.norm_gate_backward(x, g, w, dy, cu_seqlens=cu), sla.norm_gate_backward(x[None], g[None], w, dy[None])
    assert torch.equal(got["dw"], want["dw"])
    for n in ("dx", "dg"):
        assert torch.equal(got[n], want[n][0]), n
    p = sla.SlaNormGateParams(sla.BF16, B, T, 4, 16, 1, sla.FLAG_HEAD_WEIGHTS if weight == "heads" else 0, 1e-5)
    need = sla.sla_norm_gate_backward_workspace_bytes(p, packed=True)
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")  # a margin that must stay
    again = sla.norm_gate_backward(x, g, w, dy, cu_seqlens=cu, workspace=ws[:need])
    assert torch.equal(again["dw"], want["dw"]) and bool((ws[need:] == 0x5a).all())


@pytest.mark.parametrize("T,B,D", [(65536, 16385, 64), (65600, 131072, 520)])
def test_join(T, B, D):
    import torch
    import paper_2602_01744_amd as sla

    rng = np.random.default_rng(B + D)
    cu = torch.from_numpy(_offsets(rng, T, B)).cuda()
    x, dxo = (torch.randn(T, D, device="cuda") for _ in range(2))
    h, dy = (torch.randn(T, D, device="cuda").bfloat16() for _ in range(2))
    wb, wa, c = (1 + 0.1 * torch.randn(D, device="cuda") for _ in range(3))
    kw = dict(w_after=wa, channel_scale=c, scale=0.5)
    got, want = sla.join_norm(x, h, wb, cu_seqlens=cu, **kw), sla.join_norm(x, h, wb, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    xo = want[0]
    got, want = sla.join_norm_backward(xo, h, wb, dy, dxo, cu_seqlens=cu, **kw), sla.join_norm_backward(xo, h, wb, dy, dxo, **kw)
    assert all(torch.equal(got[n], want[n]) for n in want)
    p = sla.SlaJoinNormParams(sla.BF16, sla.F32, B, T, D, 0.5, 1e-5)
    need = sla.sla_join_norm_backward_workspace_bytes(p, packed=True)
    ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    again = sla.join_norm_backward(xo, h, wb, dy, dxo, cu_seqlens=cu, workspace=ws[:need], **kw)
    assert all(torch.equal(again[n], want[n]) for n in want) and bool((ws[need:] == 0x5a).all())


def test_rotary():
    """Positions count from every sequence's start; fp32 bound as for few sequences: 8 steps of the terms."""
    import torch
    import paper_2602_01744_amd as sla

    T, B, r = 65600, 131072, 16
    rng = np.random.default_rng(5)
    cu = _offsets(rng, T, B)
    x = rng.standard_normal((T, 2, 16)).astype(np.float32)
    f = 10000.0 ** (-2.0 * np.arange(r // 2) / r)
    at = np.zeros(T, np.int64)
    for b in range(B):
        at[cu[b]:cu[b + 1]] = np.arange(cu[b + 1] - cu[b])
    y, _ = sla.rotary(tensor(x), None, torch.from_numpy(f).cuda(), cu_seqlens=torch.from_numpy(cu).cuda())
    terms = np.abs(x[..., :r // 2]) + np.abs(x[..., r // 2:])
    within("q", numpy64(y), ol.rotary(x, at, f), 9 * np.concatenate([terms, terms], -1).astype(np.float64), "f32", steps=1)
