"""The gated read-out norm and its gradients on the GPU against the oracle."""
import numpy as np
import pytest

from layer_util import K, numpy64, rounded, sequences, tensor, within
from oracle import sla_layer as ol

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _inputs(seed, lead, H, dv, gate, weight, dtype):
    r = np.random.default_rng(seed)
    x = rounded(r.standard_normal(lead + (H, dv)) * np.exp(r.standard_normal(lead + (H, 1)) - 2.0), dtype)
    g = None if gate == "none" else rounded(r.standard_normal(lead + (H, dv)) * 1.5, dtype)
    dy = rounded(r.standard_normal(lead + (H, dv)), dtype)
    w = {"none": None, "shared": 1 + 0.25 * r.standard_normal(dv), "heads": 1 + 0.25 * r.standard_normal((H, dv))}[weight]
    return x, g, None if w is None else w.astype(np.float32), dy


def _steps(g):
    return K if g is None else K + 2 * np.max(np.abs(g))


def _check_backward(got, x, g, w, dy, gate, dtype, eps=EPS):
    want = ol.norm_gate_backward(x, g, w, dy, gate=gate, eps=eps)
    x, dy = x.astype(np.float64), dy.astype(np.float64)
    s = np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
    act, dact = ol._gate(None if g is None else g.astype(np.float64), gate)
    wt = 1.0 if w is None else w.astype(np.float64)
    n, dn = x / s, np.abs(dy * wt * act)
    # dx is a difference: the terms of both parts, those of the mean with their absolute values
    within("dx", got["dx"], want["dx"], (dn + np.abs(n) * np.mean(np.abs(n) * dn, -1, keepdims=True)) / s, dtype, 2 * _steps(g))
    if g is not None:
        g = g.astype(np.float64)
        p = ol._sigmoid(g)  # SiLU's derivative is a sum whose terms cancel near -1.28
        slope = p * (1 + np.abs(g) * (1 - p)) if gate == "silu" else p
        within("dg", got["dg"], want["dg"], np.abs(dy * n * wt) * slope, dtype, _steps(g))
    else:
        assert got["dg"] is None
    if w is not None:
        t = np.abs(dy * n * act)
        rows = t.size // w.size
        # a term's own error, and one step an addition: a lane's rows, the 32 to 256 slots of a workgroup, 16 partial sums a
        # thread, 6 halvings
        within("dw", got["dw"], want["dw"], t.reshape((-1,) + w.shape).sum(0), "f32", _steps(g) + min(rows, 64) + 256 + 22)
    else:
        assert got["dw"] is None


SHAPES = [  # lead, H, dv
    ((2, 37), 4, 128), ((1, 1), 1, 64), ((64, 1), 16, 128), ((1, 203), 5, 64), ((3, 11), 12, 256), ((1, 130), 3, 8), ((2, 5), 7, 40),
    ((1, 19), 2, 512), ((1, 9), 1, 504), ((1, 700), 64, 16), ((2, 3), 1, 96),
    ((1, 2500), 64, 16), ((1, 2300), 4, 256)]  # more tokens than the gradients' workgroups take at a time


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lead,H,dv", SHAPES)
@pytest.mark.parametrize("gate,weight", [("silu", "shared"), ("sigmoid", "heads"), ("none", "shared"), ("silu", "none"), ("none", "heads")])
def test_parity(dtype, lead, H, dv, gate, weight):
    import paper_2602_01744_amd as sla

    x, g, w, dy = _inputs(H * dv + lead[1], lead, H, dv, gate, weight, dtype)
    xt, gt, wt, dyt = tensor(x, dtype), tensor(g, dtype), tensor(w), tensor(dy, dtype)
    y = sla.norm_gate(xt, gt, wt, gate=gate, eps=EPS)
    want = ol.norm_gate(x, g, w, gate=gate, eps=EPS)
    within("y", y, want, np.abs(want), dtype, _steps(g))
    _check_backward(sla.norm_gate_backward(xt, gt, wt, dyt, gate=gate, eps=EPS), x, g, w, dy, gate, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,H,dv", [(2, 33, 4, 128), (3, 17, 5, 64), (1, 70, 1, 256), (4, 1, 6, 40), (2, 2600, 16, 64)])
@pytest.mark.parametrize("weight", ["shared", "heads"])
def test_head_major(dtype, B, T, H, dv, weight):
    """x as sla_forward leaves it in its head-major layout, everything else token-major: bits as from the other layout."""
    import torch
    import paper_2602_01744_amd as sla

    x, g, w, dy = _inputs(T + dv, (B, T), H, dv, "silu", weight, dtype)
    xt, gt, wt, dyt = tensor(x, dtype), tensor(g, dtype), tensor(w), tensor(dy, dtype)
    xh = xt.transpose(1, 2).contiguous()
    assert torch.equal(sla.norm_gate(xh, gt, wt, head_major=True), sla.norm_gate(xt, gt, wt))
    a, b = sla.norm_gate_backward(xh, gt, wt, dyt, head_major=True), sla.norm_gate_backward(xt, gt, wt, dyt)
    assert torch.equal(a["dx"].transpose(1, 2), b["dx"]) and torch.equal(a["dg"], b["dg"]) and torch.equal(a["dw"], b["dw"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weight", ["shared", "heads"])
@pytest.mark.parametrize("n,T,pad", [(1, 9, 0), (5, 150, 7), (64, 2100, 3), (3, 40, 20)])
def test_packed_leaves_the_rest_alone(dtype, weight, n, T, pad):
    """Rows outside every sequence hold NaN: they are not counted in dw, and their outputs stay as they were."""
    import torch
    import paper_2602_01744_amd as sla
    from paper_2602_01744_amd import binding

    H, dv = 3, 64
    x, g, w, dy = _inputs(n + T, (T,), H, dv, "silu", weight, dtype)
    cu = sequences(np.random.default_rng(n), n, T, pad)
    inside = slice(int(cu[0]), int(cu[-1]))
    poison = lambda a: np.concatenate([np.full_like(a[:cu[0]], np.nan), a[inside], np.full_like(a[cu[-1]:], np.nan)])
    xt, gt, dyt, wt = tensor(poison(x), dtype), tensor(poison(g), dtype), tensor(poison(dy), dtype), tensor(w)
    cut = torch.from_numpy(cu).cuda()
    y = torch.full_like(xt, 7.0)
    sla.norm_gate(xt, gt, wt, cu_seqlens=cut, out=y)
    want = ol.norm_gate(x, g, w)
    within("y", numpy64(y)[inside], want[inside], np.abs(want[inside]), dtype, _steps(g))
    dx, dg, dw = torch.full_like(xt, 7.0), torch.full_like(xt, 7.0), torch.full_like(wt, 7.0)
    p = sla.SlaNormGateParams(sla.BF16 if dtype == "bf16" else sla.F32, n, T, H, dv, 1, sla.FLAG_HEAD_WEIGHTS if weight == "heads" else 0, EPS)
    need = sla.sla_norm_gate_backward_workspace_bytes(p, packed=True)
    ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")  # NaN before, and a margin that must stay
    rc = sla.sla_norm_gate_backward(p, xt.data_ptr(), gt.data_ptr(), wt.data_ptr(), dyt.data_ptr(), cut.data_ptr(), dx.data_ptr(),
                                    dg.data_ptr(), dw.data_ptr(), ws.data_ptr(), need, binding._stream(xt))
    assert rc == 0
    for t in (y, dx, dg):
        assert bool((t[:cu[0]] == 7.0).all()) and bool((t[int(cu[-1]):] == 7.0).all())
    assert bool((ws[need:] == 0xff).all())
    got = {"dx": numpy64(dx)[inside], "dg": numpy64(dg)[inside], "dw": dw}
    if inside.start < inside.stop:
        _check_backward(got, x[inside], g[inside], w, dy[inside], "silu", dtype)
    else:
        assert bool((dw == 0).all())


def test_empty_batches_give_zero_weight_gradients():
    import torch
    import paper_2602_01744_amd as sla

    w = torch.ones(64, device="cuda")
    for shape in ((0, 4, 2, 64), (2, 0, 2, 64), (0, 2, 64)):
        x = torch.empty(shape, device="cuda")
        assert sla.norm_gate(x, x, w).shape == shape
        got = sla.norm_gate_backward(x, x, w, x)
        assert got["dx"].shape == shape and bool((got["dw"] == 0).all())
    x = torch.ones(5, 2, 64, device="cuda")
    for cu in ([0], [5, 5]):
        cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
        assert bool((sla.norm_gate_backward(x, x, w, x, cu_seqlens=cu)["dw"] == 0).all())


def test_silent_heads():
    """A head whose read gate is zero is a row of zeros: y and dg are zero, dx is dy w act / sqrt(eps), dw takes nothing from it."""
    import torch
    import paper_2602_01744_amd as sla

    x, g, w, dy = _inputs(3, (1, 9), 4, 64, "silu", "shared", "f32")
    x[:, :, 1] = 0.0
    x[:, 4] = 0.0
    y = sla.norm_gate(tensor(x), tensor(g), tensor(w), eps=1e-6)
    assert bool((y[:, :, 1] == 0).all())
    got = sla.norm_gate_backward(tensor(x), tensor(g), tensor(w), tensor(dy), eps=1e-6)
    assert bool((got["dg"][:, :, 1] == 0).all()) and bool(torch.isfinite(got["dx"]).all())
    _check_backward(got, x, g, w, dy, "silu", "f32", eps=1e-6)


@pytest.mark.parametrize("gate", ["silu", "sigmoid"])
def test_far_gates(gate):
    """Gates far out: closed ones give 0, open ones 1 (times g), slopes 0 or 1; an infinite or NaN value stays in its place."""
    import torch
    import paper_2602_01744_amd as sla

    g = torch.tensor([-200.0, -95.0, -89.0, -20.0, 20.0, 89.0, 200.0, 0.0], device="cuda").repeat(8).view(1, 1, 1, 64).contiguous()
    x = torch.ones_like(g)
    y = sla.norm_gate(x, g, None, gate=gate, eps=0.0)
    d = sla.norm_gate_backward(x, g, None, x, gate=gate, eps=0.0)["dg"]
    act, slope = ol._gate(numpy64(g), gate)
    # exp2's argument is rounded to |g| 2^-24; results under the normal range are flushed
    assert np.all(np.abs(numpy64(y) - act) <= np.abs(act) * (K + 400) * 2.0 ** -24 + 3e-36)
    assert np.all(np.abs(numpy64(d) - slope) <= (np.abs(slope) + (np.abs(numpy64(g)) < 30) * 20) * (K + 400) * 2.0 ** -24 + 3e-36)
    g[..., 5] = float("nan")
    y = sla.norm_gate(x, g, None, gate=gate, eps=0.0)
    assert bool(torch.isnan(y[..., 5]).all()) and int(torch.isnan(y).sum()) == 1


def test_no_epsilon_and_no_rows_beyond_the_last():
    """eps = 0: lanes without a row divide by zero, which must not reach dw."""
    import paper_2602_01744_amd as sla

    x, g, w, dy = _inputs(8, (1, 5), 3, 8, "silu", "shared", "f32")
    _check_backward(sla.norm_gate_backward(tensor(x), tensor(g), tensor(w), tensor(dy), eps=0.0), x, g, w, dy, "silu", "f32", eps=0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_repeatable(dtype):
    import torch
    import paper_2602_01744_amd as sla

    x, g, w, dy = _inputs(9, (3, 401), 4, 128, "silu", "shared", dtype)
    xt, gt, wt, dyt = tensor(x, dtype), tensor(g, dtype), tensor(w), tensor(dy, dtype)
    y = sla.norm_gate(xt, gt, wt)
    a, b = (sla.norm_gate_backward(xt, gt, wt, dyt) for _ in range(2))
    assert all(torch.equal(a[n], b[n]) for n in a)
    for out in (xt.clone(), gt.clone()):
        on_x = bool(torch.equal(out, xt))
        got = sla.norm_gate(out if on_x else xt, gt if on_x else out, wt, out=out)
        assert torch.equal(got, y)


def test_gradients_against_differences():
    """Central differences of the GPU's own forward in fp32: steps of 2^-6 make a truncation of about 1e-4 and a rounding of 1e-5
    relative to the largest gradient."""
    import torch
    import paper_2602_01744_amd as sla

    x, g, w, dy = _inputs(10, (1, 3), 2, 16, "silu", "heads", "f32")
    x = (x / np.sqrt(np.mean(x * x, -1, keepdims=True))).astype(np.float32)  # curvature of order one
    args = [tensor(x), tensor(g), tensor(w)]
    got = sla.norm_gate_backward(*args, tensor(dy))
    d64 = torch.from_numpy(dy.astype(np.float64)).cuda()
    for i, name in enumerate(("dx", "dg", "dw")):
        num = torch.zeros(args[i].numel(), dtype=torch.float64)
        for j in range(args[i].numel()):
            v = []
            for sign in (1, -1):
                moved = [t.clone() for t in args]
                moved[i].view(-1)[j] += sign * 2.0 ** -6
                v.append(float((sla.norm_gate(*moved).double() * d64).sum()))
            num[j] = (v[0] - v[1]) * 32.0
        ref = got[name].double().cpu().view(-1)
        assert float((num - ref).abs().max()) <= 2e-3 * float(ref.abs().max()), name
