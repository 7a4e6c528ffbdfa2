"""The residual join with its norms, and its gradients, on the GPU against the oracle."""
import itertools

import numpy as np
import pytest

from layer_util import K, numpy64, rounded, sequences, tensor, within
from oracle import sla_layer as ol

pytestmark = pytest.mark.gpu
EPS = 1e-5
TYPES = {"f32": ("f32", "f32"), "bf16": ("bf16", "bf16"), "mixed": ("bf16", "f32")}  # blocks, stream


def _inputs(seed, lead, D, types, after, channel):
    ht, xt = TYPES[types]
    r = np.random.default_rng(seed)
    loud = np.where(r.random(D) < 0.02, 12.0, 1.5)
    x, dxo = rounded(r.standard_normal(lead + (D,)) * loud, xt), rounded(r.standard_normal(lead + (D,)), xt)
    h, dy = rounded(0.5 * r.standard_normal(lead + (D,)), ht), rounded(r.standard_normal(lead + (D,)), ht)
    vec = lambda: (1 + 0.25 * r.standard_normal(D)).astype(np.float32)
    return x, h, vec(), vec() if after else None, vec() if channel else None, dy, dxo


def _check_forward(xo, y, x, h, wb, wa, c, scale, types, eps=EPS):
    ht, xt = TYPES[types]
    want_x, want_y = ol.join_norm(x, h, wb, w_after=wa, channel_scale=c, scale=scale, eps=eps)
    x = x.astype(np.float64)
    part = np.abs(want_x) if h is None else np.abs(x) + np.abs(want_x - x)  # the join is a sum: its terms
    if h is not None:
        within("x_out", xo, want_x, part, xt)
    if wb is not None:
        rms = np.sqrt(np.mean(want_x ** 2, -1, keepdims=True) + eps)
        # y's error from x': its own, and through the mean of its squares
        spread = np.sqrt(np.mean(part ** 2, -1, keepdims=True) + eps) / rms
        within("y", y, want_y, (part + np.abs(want_x) * spread) / rms * np.abs(wb), ht, 2 * K)


def _check_backward(got, xo, h, wb, dy, dxo, wa, c, scale, types, eps=EPS):
    ht, xt = TYPES[types]
    want = ol.join_norm_backward(xo, h, wb, dy, dxo, w_after=wa, channel_scale=c, scale=scale, eps=eps)
    a = np.zeros(xo.shape) if dxo is None else np.abs(dxo.astype(np.float64))
    rows = xo.size // xo.shape[-1]
    adds = min(rows, 128) + 4 + 16 + 6  # a wave's rows, the workgroup's rows, partial sums a thread, halvings
    if wb is not None:
        x = xo.astype(np.float64)
        s = np.sqrt(np.mean(x * x, -1, keepdims=True) + eps)
        n, dn = np.abs(x / s), np.abs(dy.astype(np.float64) * wb)
        a = a + (dn + n * np.mean(n * dn, -1, keepdims=True)) / s
        within("dx", got["dx"], want["dx"], a, xt, 2 * K)
        within("dw_before", got["dw_before"], want["dw_before"], np.abs(dy * n).reshape(-1, x.shape[-1]).sum(0), "f32", K + adds)
    if h is None:
        assert got["dh"] is None
        return
    h = h.astype(np.float64)
    rh = np.sqrt(np.mean(h * h, -1, keepdims=True) + eps) if wa is not None else 1.0
    m, du = np.abs(h / rh), scale * a
    for name, other in (("dw_after", c), ("dchannel_scale", wa)):
        if want[name] is not None:
            t = (du * m).reshape(-1, h.shape[-1]).sum(0) * (1.0 if other is None else np.abs(other))
            within(name, got[name], want[name], t, "f32", 3 * K + adds)
        else:
            assert got[name] is None
    du = du * (1.0 if c is None else np.abs(c))
    if wa is not None:
        du = du * np.abs(wa)
        du = (du + m * np.mean(m * du, -1, keepdims=True)) / rh
    within("dh", got["dh"], want["dh"], du, ht, 4 * K)


def _both(x, h, wb, wa, c, dy, dxo, scale, types, **kw):
    import paper_2602_01744_amd as sla

    ht, xt = TYPES[types]
    xo, y = sla.join_norm(tensor(x, xt), tensor(h, ht), tensor(wb), w_after=tensor(wa), channel_scale=tensor(c), scale=scale, **kw)
    _check_forward(xo, y, x, h, wb, wa, c, scale, types, kw.get("eps", EPS))
    stored = numpy64(xo).astype(np.float32)
    got = sla.join_norm_backward(xo, tensor(h, ht), tensor(wb), tensor(dy, ht) if wb is not None else None, tensor(dxo, xt),
                                 w_after=tensor(wa), channel_scale=tensor(c), scale=scale, **kw)
    _check_backward(got, stored, h, wb, dy, dxo, wa, c, scale, types, kw.get("eps", EPS))


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("lead,D", [((1, 1), 1024), ((2, 37), 1024), ((3, 5), 2048), ((7,), 8), ((130,), 264), ((2, 3), 4104), ((5,), 8192),
                                    ((3,), 16384), ((2, 701), 520), ((4,), 1536),
                                    # more rows than the gradients' workgroups take at a time
                                    ((9001,), 64), ((1100,), 4096), ((300,), 8192), ((300,), 8200)])
@pytest.mark.parametrize("after,channel", [(0, 0), (1, 1)])
def test_parity(types, lead, D, after, channel):
    x, h, wb, wa, c, dy, dxo = _inputs(D + lead[0], lead, D, types, after, channel)
    _both(x, h, wb, wa, c, dy, dxo, 0.5 if after else 1.0, types)


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("after,channel,norm,later,join", itertools.product([0, 1], repeat=5))
def test_every_part_alone_and_together(types, after, channel, norm, later, join):
    import torch
    import paper_2602_01744_amd as sla

    if not (norm or later) or (not join and (after or channel or not norm)):
        return
    x, h, wb, wa, c, dy, dxo = _inputs(31, (2, 21), 776, types, after, channel)
    if join:
        _both(x, h, wb if norm else None, wa, c, dy, dxo if later else None, 0.25, types)
        return
    ht, xt = TYPES[types]
    xs = tensor(x, xt)
    same, y = sla.join_norm(xs, None, tensor(wb), y_dtype=torch.bfloat16 if ht == "bf16" else torch.float32)
    assert same is xs and y.dtype is (torch.bfloat16 if ht == "bf16" else torch.float32)
    _check_forward(None, y, x, None, wb, None, None, 1.0, types)
    got = sla.join_norm_backward(xs, None, tensor(wb), tensor(dy, ht), tensor(dxo, xt) if later else None)
    _check_backward(got, x, None, wb, dy, dxo if later else None, None, None, 1.0, types)


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("D", [512, 3000])
@pytest.mark.parametrize("n,T,pad", [(1, 9, 0), (5, 150, 7), (64, 1100, 3), (3, 40, 20)])
def test_packed_leaves_the_rest_alone(types, D, n, T, pad):
    import torch
    import paper_2602_01744_amd as sla
    from paper_2602_01744_amd import binding

    ht, xt = TYPES[types]
    x, h, wb, wa, c, dy, dxo = _inputs(n + T, (T,), D, types, 1, 1)
    cu = sequences(np.random.default_rng(n), n, T, pad)
    inside = slice(int(cu[0]), int(cu[-1]))
    poison = lambda a, t: tensor(np.concatenate([np.full_like(a[:cu[0]], np.nan), a[inside], np.full_like(a[cu[-1]:], np.nan)]), t)
    X, H, DY, DXO = poison(x, xt), poison(h, ht), poison(dy, ht), poison(dxo, xt)
    WB, WA, C = tensor(wb), tensor(wa), tensor(c)
    cut = torch.from_numpy(cu).cuda()
    xo, y = torch.full_like(X, 7.0), torch.full_like(H, 7.0)
    sla.join_norm(X, H, WB, w_after=WA, channel_scale=C, scale=0.5, cu_seqlens=cut, x_out=xo, y=y)
    dx, dh = torch.full_like(X, 7.0), torch.full_like(H, 7.0)
    sums = [torch.full_like(WB, 7.0) for _ in range(3)]
    p = sla.SlaJoinNormParams(sla.F32 if ht == "f32" else sla.BF16, sla.F32 if xt == "f32" else sla.BF16, n, T, D, 0.5, EPS)
    need = sla.sla_join_norm_backward_workspace_bytes(p, packed=True)
    ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")
    a = [t.data_ptr() for t in (xo, H, WA, C, WB, DY, DXO, cut, dx, dh, *sums, ws)]
    assert sla.sla_join_norm_backward(p, *a, need, binding._stream(X)) == 0
    for t in (xo, y, dx, dh):
        assert bool((t[:cu[0]] == 7.0).all()) and bool((t[int(cu[-1]):] == 7.0).all())
    assert bool((ws[need:] == 0xff).all())
    if inside.start == inside.stop:
        assert all(bool((s == 0).all()) for s in sums)
        return
    cut64 = lambda t: numpy64(t)[inside]
    _check_forward(cut64(xo), cut64(y), x[inside], h[inside], wb, wa, c, 0.5, types)
    got = {"dx": cut64(dx), "dh": cut64(dh), "dw_after": sums[0], "dchannel_scale": sums[1], "dw_before": sums[2]}
    _check_backward(got, cut64(xo).astype(np.float32), h[inside], wb, dy[inside], dxo[inside], wa, c, 0.5, types)


def test_empty_batches_give_zero_weight_gradients():
    import torch
    import paper_2602_01744_amd as sla

    w = torch.ones(64, device="cuda")
    x = torch.empty(0, 3, 64, device="cuda")
    xo, y = sla.join_norm(x, x, w, w_after=w, channel_scale=w)
    assert xo.shape == y.shape == x.shape
    g = sla.join_norm_backward(x, x, w, x, x, w_after=w, channel_scale=w)
    assert all(bool((g[n] == 0).all()) and g[n].shape == (64,) for n in ("dw_after", "dchannel_scale", "dw_before"))
    x = torch.ones(5, 64, device="cuda")
    for cu in ([0], [5, 5]):
        cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
        g = sla.join_norm_backward(x, x, w, x, x, w_after=w, channel_scale=w, cu_seqlens=cu)
        assert all(bool((g[n] == 0).all()) for n in ("dw_after", "dchannel_scale", "dw_before"))


@pytest.mark.parametrize("D", [64, 1032, 4096])
def test_rows_of_zeros_and_no_epsilon(D):
    """A block that adds nothing (h = 0) behind a norm; and eps = 0 with workgroups whose last rows are not there."""
    x, h, wb, wa, c, dy, dxo = _inputs(4, (5,), D, "f32", 1, 1)
    _both(x, h, wb, wa, c, dy, dxo, 1.0, "f32", eps=0.0)
    h[1] = 0.0
    x[3] = 0.0
    _both(x, h, wb, wa, c, dy, dxo, 1.0, "f32", eps=1e-6)


@pytest.mark.parametrize("types", list(TYPES))
@pytest.mark.parametrize("D", [1024, 6000])
def test_in_place_and_repeatable(types, D):
    import torch
    import paper_2602_01744_amd as sla
    from paper_2602_01744_amd import binding

    ht, xt = TYPES[types]
    x, h, wb, wa, c, dy, dxo = _inputs(6, (301,), D, types, 1, 1)
    X, H, WB, DY, DXO = tensor(x, xt), tensor(h, ht), tensor(wb), tensor(dy, ht), tensor(dxo, xt)
    kw = dict(w_after=tensor(wa), channel_scale=tensor(c), scale=0.5)
    xo, y = sla.join_norm(X, H, WB, **kw)
    a, b = (sla.join_norm_backward(xo, H, WB, DY, DXO, **kw) for _ in range(2))
    assert all(torch.equal(a[n], b[n]) for n in a)
    X2, H2 = X.clone(), H.clone()
    sla.join_norm(X2, H2, WB, x_out=X2, y=H2, **kw)
    assert torch.equal(X2, xo) and torch.equal(H2, y)
    p = sla.SlaJoinNormParams(sla.F32 if ht == "f32" else sla.BF16, sla.F32 if xt == "f32" else sla.BF16, 1, 301, D, 0.5, EPS)
    need = sla.sla_join_norm_backward_workspace_bytes(p)
    ws, sums = torch.empty(need, dtype=torch.uint8, device="cuda"), [torch.empty_like(WB) for _ in range(3)]
    for onto in ("dy", "h"):
        dxo2, dy2, h2 = DXO.clone(), DY.clone(), H.clone()
        target = dy2 if onto == "dy" else h2
        args = [t.data_ptr() for t in (xo, h2, kw["w_after"], kw["channel_scale"], WB, dy2, dxo2)] + [0] + [
            t.data_ptr() for t in (dxo2, target, *sums, ws)]
        assert sla.sla_join_norm_backward(p, *args, need, binding._stream(X)) == 0
        assert torch.equal(dxo2, a["dx"]) and torch.equal(target, a["dh"])


def test_what_a_row_holds_stays_in_it():
    import torch
    import paper_2602_01744_amd as sla

    x = torch.randn(9, 1000, device="cuda")
    h, w = torch.randn_like(x), torch.ones(1000, device="cuda")
    x[4, 7], h[6, 3] = float("nan"), float("inf")
    xo, y = sla.join_norm(x, h, w, w_after=w)
    bad = torch.isnan(y).any(-1)
    assert bad.tolist() == [False] * 4 + [True, False, True, False, False]


def test_gradients_against_differences():
    """Central differences of the GPU's own forward in fp32 with steps of 2^-6: see the read-out's."""
    import torch
    import paper_2602_01744_amd as sla

    x, h, wb, wa, c, dy, dxo = _inputs(12, (3,), 16, "f32", 1, 1)
    x = (x / 3).astype(np.float32)
    h = (h * 2).astype(np.float32)
    args = [tensor(t) for t in (x, h, wb, wa, c)]
    run = lambda x, h, wb, wa, c: sla.join_norm(x, h, wb, w_after=wa, channel_scale=c, scale=0.5)
    xo, _ = run(*args)
    got = sla.join_norm_backward(xo, args[1], args[2], tensor(dy), tensor(dxo), w_after=args[3], channel_scale=args[4], scale=0.5)
    dy64, dx64 = tensor(dy).double(), tensor(dxo).double()
    for i, name in enumerate(("dx", "dh", "dw_before", "dw_after", "dchannel_scale")):
        num = torch.zeros(args[i].numel(), dtype=torch.float64)
        for j in range(args[i].numel()):
            v = []
            for sign in (1, -1):
                moved = [t.clone() for t in args]
                moved[i].view(-1)[j] += sign * 2.0 ** -6
                a, b = run(*moved)
                v.append(float((a.double() * dx64).sum() + (b.double() * dy64).sum()))
            num[j] = (v[0] - v[1]) * 32.0
        ref = got[name].double().cpu().view(-1)
        assert float((num - ref).abs().max()) <= 2e-3 * float(ref.abs().max()), name
