"""The operators around the mixer together with it, as a layer runs them: a training step against the oracles' composition, token
by token against the whole sequence, captured into graphs, on another stream."""
import numpy as np
import pytest

import oracle
import sla_inputs as si
from gpu_util import GLA, RETNET, TOL, rel_err
from layer_util import numpy64, tensor
from oracle import sla_layer as ol

pytestmark = pytest.mark.gpu

B, T, H, DK, DV, D = 2, 53, 4, 64, 128, 512


def _layer(seed):
    r = np.random.default_rng(seed)
    n = lambda *s: r.standard_normal(s).astype(np.float32)
    w = {m: n(D, H * d) / np.float32(np.sqrt(D)) for m, d in (("q", DK), ("k", DK), ("v", DV), ("g", DV))}
    w["o"] = n(H * DV, D) / np.float32(np.sqrt(H * DV))
    w.update(before=1 + 0.1 * n(D), after=1 + 0.1 * n(D), out=1 + 0.1 * n(DV), channel=0.5 + 0.1 * n(D), next=1 + 0.1 * n(D))
    x, ql, kl = 2 * n(B, T, D), n(B, T, H), n(B, T, H)
    decay = np.log1p(-np.exp2(-5.0 - np.arange(H))).astype(np.float32)
    return w, x, ql, kl, decay, n(B, T, D), n(B, T, D)


def test_training_step_of_a_layer():
    """RetNet's layer in fp32: norm, projections, rotary positions, mixer, read-out, output projection, join with both norms; the
    gradients of the input, of every weight of the new operators and of the projections.  Tolerance: the mixer's own 1e-4, twice in
    a gradient's way (forward and backward), and fp32 products of 512 terms."""
    import torch
    import paper_2602_01744_amd as sla

    w, x, ql, kl, decay, dy, dxo = _layer(1)
    t = {k: tensor(v) for k, v in w.items()}
    X, QL, KL, LD = tensor(x), tensor(ql), tensor(kl), tensor(decay)
    f, m = sla.rotary_frequencies(DK)
    f64 = f.cpu().numpy()
    heads = lambda a, d: a.view(B, T, H, d)
    _, a = sla.join_norm(X, None, t["before"])
    proj = {n: heads(a @ t[n], d) for n, d in (("q", DK), ("k", DK), ("v", DV), ("g", DV))}
    q, k = sla.rotary(proj["q"], proj["k"], f, magnitude=m)
    out, _ = sla.forward(sla.RETNET, q, k, proj["v"], QL, KL, LD)
    z = sla.norm_gate(out, proj["g"], t["out"])
    h = z.view(B, T, H * DV) @ t["o"]
    xo, y = sla.join_norm(X, h, t["next"], w_after=t["after"], channel_scale=t["channel"], scale=0.5)
    # and back
    gj = sla.join_norm_backward(xo, h, t["next"], tensor(dy), tensor(dxo), w_after=t["after"], channel_scale=t["channel"], scale=0.5)
    dz = (gj["dh"] @ t["o"].t()).view(B, T, H, DV)
    gz = sla.norm_gate_backward(out, proj["g"], t["out"], dz)
    gm = sla.backward(sla.RETNET, q, k, proj["v"], QL, KL, LD, gz["dx"])
    dq, dk = sla.rotary_backward(gm["dq"], gm["dk"], f, magnitude=m)
    da = sum(d.reshape(B, T, -1) @ t[n].t() for n, d in (("q", dq), ("k", dk), ("v", gm["dv"]), ("g", gz["dg"])))
    g0 = sla.join_norm_backward(X, None, t["before"], da, gj["dx"])
    torch.cuda.synchronize()

    _, A = ol.join_norm(x, None, w["before"])
    P = {n: (A @ w[n]).reshape(B, T, H, d) for n, d in (("q", DK), ("k", DK), ("v", DV), ("g", DV))}
    pos = np.broadcast_to(np.arange(T), (B, T))
    Q, Kk = (ol.rotary(P[n], pos, f64, magnitude=m) for n in "qk")
    O, _ = oracle.forward(RETNET, Q, Kk, P["v"], ql, kl, decay)
    Z = ol.norm_gate(O, P["g"], w["out"])
    Hh = Z.reshape(B, T, -1) @ w["o"]
    kw = dict(w_after=w["after"], channel_scale=w["channel"], scale=0.5)
    XO, Y = ol.join_norm(x, Hh, w["next"], **kw)
    GJ = ol.join_norm_backward(XO, Hh, w["next"], dy, dxo, **kw)
    DZ = (GJ["dh"] @ w["o"].T).reshape(B, T, H, DV)
    GZ = ol.norm_gate_backward(O, P["g"], w["out"], DZ)
    GM = oracle.backward(RETNET, Q, Kk, P["v"], ql, kl, decay, GZ["dx"])
    DQ, DKk = (ol.rotary(GM[n], pos, f64, magnitude=m, inverse=True) for n in ("dq", "dk"))
    DA = sum(d.reshape(B, T, -1) @ w[n].T for n, d in (("q", DQ), ("k", DKk), ("v", GM["dv"]), ("g", GZ["dg"])))
    G0 = ol.join_norm_backward(x, None, w["before"], DA, GJ["dx"])
    for name, got, want in (("y", y, Y), ("x_out", xo, XO), ("dx", g0["dx"], G0["dx"]), ("dw_before", g0["dw_before"], G0["dw_before"]),
                            ("dw_out", gz["dw"], GZ["dw"]), ("dw_after", gj["dw_after"], GJ["dw_after"]),
                            ("dchannel", gj["dchannel_scale"], GJ["dchannel_scale"]), ("dw_next", gj["dw_before"], GJ["dw_before"]),
                            ("dW_q", A.reshape(-1, D).T @ numpy64(dq).reshape(B * T, -1), A.reshape(-1, D).T @ DQ.reshape(B * T, -1)),
                            ("dW_g", A.reshape(-1, D).T @ numpy64(gz["dg"]).reshape(B * T, -1), A.reshape(-1, D).T @ GZ["dg"].reshape(B * T, -1))):
        e = rel_err(got if isinstance(got, np.ndarray) else numpy64(got), want)
        print(f"[layer] {name} {e:.2e}", flush=True)
        assert e <= 3 * TOL["f32"], name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_by_token_is_the_whole_sequence(dtype):
    """A prompt at once, then the same tokens one at a time with their positions: rotary, decode step, read-out."""
    import torch
    import paper_2602_01744_amd as sla

    n = 12
    d = si.custom(GLA, dtype, B=3, T=n, H=4, dk=128, dv=128, seed=71)
    g, el = si.to_device(d, dtype, GLA)
    gate, w = torch.randn(3, n, 4, 128, device="cuda").to(el), 1 + 0.1 * torch.randn(128, device="cuda")
    f, m = sla.rotary_frequencies(128, scaling="blend", factor=4.0)
    start = torch.tensor([0, 5000, 99], dtype=torch.int32, device="cuda")
    q, k = sla.rotary(g["q"], g["k"], f, start=start, magnitude=m)
    out, fin = sla.forward(GLA, q, k, g["v"], g["q_logits"], g["k_logits"], g["log_decay"])
    y = sla.norm_gate(out, gate, w)
    state = torch.zeros(3, 4, 128, 128, device="cuda")
    steps = []
    for t in range(n):
        one = lambda a: a[:, t].contiguous()
        qt, kt = sla.rotary(one(g["q"]), one(g["k"]), f, start=start + t, magnitude=m)
        assert torch.equal(qt, q[:, t]) and torch.equal(kt, k[:, t])
        o = sla.decode_step(GLA, qt, kt, one(g["v"]), one(g["q_logits"]), one(g["k_logits"]), one(g["log_decay"]), None, state)
        steps.append(sla.norm_gate(o, one(gate), w))
    # the mixer's two forms agree to its tolerance; the norm divides by a head's own size
    assert rel_err(numpy64(torch.stack(steps, 1)), numpy64(y)) <= 4 * TOL[dtype]
    assert rel_err(numpy64(state), numpy64(fin)) <= TOL[dtype]


def test_packed_chain_is_each_sequence_alone():
    import torch
    import paper_2602_01744_amd as sla

    lens, n = [5, 0, 33, 1], 39
    cu = torch.tensor([0, 5, 5, 38, 39], dtype=torch.int32, device="cuda")
    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()
    q, k, x, g = r(n, 4, 64), r(n, 2, 64), r(n, 4, 64), r(n, 4, 64)
    h, s, w = r(n, 256), torch.randn(n, 256, device="cuda"), torch.ones(256, device="cuda")
    f, _ = sla.rotary_frequencies(64)
    qo, ko = sla.rotary(q, k, f, cu_seqlens=cu)
    y = sla.norm_gate(x, g, None, cu_seqlens=cu)
    xo, z = sla.join_norm(s, h, w, w_after=w, cu_seqlens=cu)
    at = 0
    for length in lens:
        c = slice(at, at + length)
        at += length
        a, b = sla.rotary(q[c][None].contiguous(), k[c][None].contiguous(), f)
        assert torch.equal(a[0], qo[c]) and torch.equal(b[0], ko[c])
        assert torch.equal(sla.norm_gate(x[c], g[c], None) if length else y[c], y[c])
        u, v = sla.join_norm(s[c], h[c], w, w_after=w)
        assert torch.equal(u, xo[c]) and torch.equal(v, z[c])


def test_captured_chain_replays_identically():
    """Forward and gradients of all three operators captured as one graph with its own workspaces; replayed on changed inputs with
    eager calls of the same operators, other sizes, and synchronisations between the replays."""
    import torch
    import paper_2602_01744_amd as sla

    torch.manual_seed(3)
    r = lambda *s: torch.randn(*s, device="cuda")
    f, _ = sla.rotary_frequencies(128)
    start = torch.tensor([17, 40], dtype=torch.int32, device="cuda")
    t = {"q": r(2, 300, 4, 128).bfloat16(), "k": r(2, 300, 4, 128).bfloat16(), "x": r(2, 300, 4, 128).bfloat16(),
         "g": r(2, 300, 4, 128).bfloat16(), "dy": r(2, 300, 4, 128).bfloat16(), "w": 1 + 0.1 * r(128),
         "s": r(2, 300, 1024), "h": r(2, 300, 1024).bfloat16(), "wb": 1 + 0.1 * r(1024), "wa": 1 + 0.1 * r(1024), "dz": r(2, 300, 1024).bfloat16(),
         "ds": r(2, 300, 1024)}

    def chain():
        q, k = sla.rotary(t["q"], t["k"], f, start=start)
        dq, dk = sla.rotary_backward(q, k, f, start=start)
        y = sla.norm_gate(t["x"], t["g"], t["w"])
        gz = sla.norm_gate_backward(t["x"], t["g"], t["w"], t["dy"])
        xo, z = sla.join_norm(t["s"], t["h"], t["wb"], w_after=t["wa"])
        gj = sla.join_norm_backward(xo, t["h"], t["wb"], t["dz"], t["ds"], w_after=t["wa"])
        return [q, k, dq, dk, y, xo, z] + [v for g in (gz, gj) for v in g.values() if v is not None]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        kept = chain()
    for rep in range(4):
        for n in ("q", "x", "dy", "s", "dz"):
            t[n].copy_(torch.randn_like(t[n].float()))
        want = chain()
        sla.norm_gate_backward(t["x"][:, :7].contiguous(), t["g"][:, :7].contiguous(), t["w"], t["dy"][:, :7].contiguous())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(kept, want)), f"replay {rep}"


@pytest.mark.parametrize("D", [8192, 16384])
def test_captured_wide_rows(D):
    """Rows wide enough that the gradients' kernel asks for more LDS than a launch gets by itself."""
    import torch
    import paper_2602_01744_amd as sla

    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()
    xo, h, dy, dxo = (r(70, D) for _ in range(4))
    w = [1 + 0.1 * torch.randn(D, device="cuda") for _ in range(3)]
    run = lambda: sla.join_norm_backward(xo, h, w[0], dy, dxo, w_after=w[1], channel_scale=w[2])
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        kept = run()
    for rep in range(3):
        for t in (xo, h, dy, dxo):
            t.copy_(r(70, D))
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(kept[n], want[n]) for n in want), f"replay {rep}"


def test_host_tensors_workspaces_and_outputs_are_checked():
    """What only a machine with a GPU can be asked: tensors of two devices, a workspace that is too small or elsewhere, an output on
    an input that is laid out differently."""
    import torch
    import paper_2602_01744_amd as sla

    x = torch.ones(2, 4, 4, 64, device="cuda")
    w, f = torch.ones(64, device="cuda"), torch.ones(32, dtype=torch.float64)
    for call in (lambda: sla.rotary(x, x, f), lambda: sla.norm_gate(x, x.cpu(), w), lambda: sla.norm_gate(x, x, w.cpu()),
                 lambda: sla.norm_gate(x, x, w, head_major=True, out=x), lambda: sla.join_norm(x, x.cpu(), w),
                 lambda: sla.norm_gate_backward(x, x, w, x, workspace=torch.empty(1 << 20, dtype=torch.uint8)),
                 lambda: sla.rotary(x, x, f.cuda(), q_out=x), lambda: sla.rotary(x, x.clone(), f.cuda(), q_out=x, k_out=x)):
        with pytest.raises(ValueError):
            call()
    small = torch.empty(16, dtype=torch.uint8, device="cuda")
    for call in (lambda: sla.norm_gate_backward(x, x, w, x, workspace=small), lambda: sla.join_norm_backward(x, x, w, x, workspace=small)):
        with pytest.raises(sla.SlaError) as e:
            call()
        assert e.value.status == -6


def test_offsets_past_32_bits():
    """Tensors of more than 2^32 bytes: their last rows come out as those of small ones, in the outputs and the gradients."""
    import torch
    import paper_2602_01744_amd as sla

    if torch.cuda.mem_get_info()[0] < 40 * 2 ** 30:
        pytest.skip("not enough memory")
    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()
    w = 1 + 0.1 * torch.randn(16384, device="cuda")
    rows, tail = 135000, [r(5, 16384) for _ in range(4)]  # 4.4 GB a tensor
    big = [torch.zeros(rows, 16384, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    for a, b in zip(big, tail):
        a[-5:] = b
    got, want = (sla.join_norm(t[0], t[1], w, w_after=w) for t in (big, tail))
    assert all(torch.equal(a[-5:], b) for a, b in zip(got, want))
    got, want = (sla.join_norm_backward(t[0], t[1], w, t[2], t[3], w_after=w) for t in (big, tail))
    assert torch.equal(got["dx"][-5:], want["dx"]) and torch.equal(got["dh"][-5:], want["dh"])
    assert rel_err(numpy64(got["dw_before"]), numpy64(want["dw_before"])) <= 1e-6  # zero rows add nothing; another order
    del got, want
    heads = [t.view(1, -1, 32, 512) for t in big[:3]]
    small = [t.view(1, -1, 32, 512) for t in tail[:3]]
    n = small[0].shape[1]
    v = w[:512].contiguous()
    assert torch.equal(sla.norm_gate(heads[0], heads[1], v)[:, -n:], sla.norm_gate(small[0], small[1], v))
    got, want = (sla.norm_gate_backward(t[0], t[1], v, t[2]) for t in (heads, small))
    assert torch.equal(got["dx"][:, -n:], want["dx"]) and torch.equal(got["dg"][:, -n:], want["dg"])


def test_offsets_of_sequences_are_clamped():
    """No content of cu_seqlens makes a kernel leave the tensors: offsets under 0, past the last token, and out of order."""
    import torch
    import paper_2602_01744_amd as sla

    T = 12
    x, g, w = torch.randn(T, 4, 64, device="cuda"), torch.randn(T, 4, 64, device="cuda"), torch.ones(64, device="cuda")
    f, _ = sla.rotary_frequencies(64)
    for cu in ([-3, 5, 99], [0, 9, 2, 12], [7, 3], [50, 60], [-9, -2]):
        lo = min(max(cu[0], 0), T)
        hi = max(min(max(cu[-1], 0), T), lo)
        c = torch.tensor(cu, dtype=torch.int32, device="cuda")
        y = torch.full_like(x, 7.0)
        sla.norm_gate(x, g, w, cu_seqlens=c, out=y)
        want = torch.full_like(x, 7.0)
        if hi > lo:
            want[lo:hi] = sla.norm_gate(x[lo:hi].contiguous(), g[lo:hi].contiguous(), w)
        assert torch.equal(y, want), cu
        q = torch.full_like(x, 7.0)
        sla.rotary(x, None, f, cu_seqlens=c, start=torch.zeros(len(cu) - 1, dtype=torch.int32, device="cuda"), q_out=q)
        assert bool((q[:lo] == 7.0).all()) and bool((q[hi:] == 7.0).all()) and bool(torch.isfinite(q).all())
        v, ones = x.view(T, 256), torch.ones(256, device="cuda")
        a, b = torch.full_like(v, 7.0), torch.full_like(v, 7.0)
        sla.join_norm(v, g.view(T, 256), ones, cu_seqlens=c, x_out=a, y=b)
        sla.join_norm_backward(v, g.view(T, 256), ones, v, v, cu_seqlens=c)
        assert bool((a[:lo] == 7.0).all()) and bool((b[hi:] == 7.0).all())
        assert hi == lo or torch.equal(a[lo:hi], (v + g.view(T, 256))[lo:hi])


def test_two_streams_at_once():
    """Calls on a stream of their own run there: after work that is queued on it, beside calls on another stream."""
    import torch
    import paper_2602_01744_amd as sla

    streams = [torch.cuda.Stream() for _ in range(2)]
    x = torch.randn(2, 4096, 2048, device="cuda").bfloat16()
    w = 1 + 0.1 * torch.randn(2048, device="cuda")
    torch.cuda.synchronize()
    got = []
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            a = x[i] * 2
            for _ in range(3):
                a = a + 1  # work that the calls have to wait for
            xo, y = sla.join_norm(a, x[i], w, w_after=w)
            got.append((a, xo, y, sla.join_norm_backward(xo, x[i], w, y, w_after=w)))
    torch.cuda.synchronize()
    for i in range(2):
        a = x[i] * 2 + 1 + 1 + 1
        xo, y = sla.join_norm(a, x[i], w, w_after=w)
        g = sla.join_norm_backward(xo, x[i], w, y, w_after=w)
        assert torch.equal(got[i][1], xo) and torch.equal(got[i][2], y)
        assert all(torch.equal(got[i][3][n], g[n]) for n in g if g[n] is not None)
