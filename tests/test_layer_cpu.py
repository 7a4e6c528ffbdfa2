"""The operators around the mixer without a GPU: their oracle pinned by finite differences and by properties, what the C
entry points and the binding refuse, and the host code under sanitizers."""
import itertools
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2602_01744_amd as sla
from oracle import sla_layer as ol

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20  # a 16-byte aligned address that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sla.library_path()):
        from paper_2602_01744_amd import build

        build.build()
    return sla.load_library()


# ---------------------------------------------------------------------------------------------------------------- oracle

def _differences(f, x, dy_of):
    """d sum(f(x) * dy) / dx by central differences, whose error at step 1e-5 is about 1e-10 for values of order one."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = 1e-5
        g[i] = (dy_of(f(x + e)) - dy_of(f(x - e))) / 2e-5
    return g


@pytest.mark.parametrize("adjacent", [False, True])
def test_rotary_oracle(adjacent):
    r = np.random.default_rng(1)
    x, f, pos = r.standard_normal((2, 3, 2, 10)), np.array([1.0, 0.3, 0.01]), np.array([[0, 1, 2], [7, -3, 100000]])
    y = ol.rotary(x, pos, f, adjacent=adjacent, magnitude=1.25)
    assert np.array_equal(y[..., 6:], x[..., 6:])  # what is not turned is copied
    assert np.allclose(y[0, 0, :, :6], 1.25 * x[0, 0, :, :6])  # position 0: no turn
    assert np.allclose(np.sum(y[..., :6] ** 2, -1), 1.25 ** 2 * np.sum(x[..., :6] ** 2, -1))
    dy = r.standard_normal(x.shape)
    dx = ol.rotary(dy, pos, f, adjacent=adjacent, magnitude=1.25, inverse=True)
    num = _differences(lambda v: ol.rotary(v, pos, f, adjacent=adjacent, magnitude=1.25), x, lambda v: np.sum(v * dy))
    dx[..., 6:] = dy[..., 6:]
    assert np.max(np.abs(dx - num)) < 1e-8
    # the product of a turned query and a turned key depends on the distance alone
    q, k = r.standard_normal((1, 1, 6)), r.standard_normal((1, 1, 6))
    dot = lambda a, b: np.sum(ol.rotary(q, np.array([a]), f, adjacent=adjacent) * ol.rotary(k, np.array([b]), f, adjacent=adjacent))
    assert abs(dot(5, 2) - dot(1005, 1002)) < 1e-9


@pytest.mark.parametrize("gate,weight", itertools.product(["silu", "sigmoid", "none"], [None, "shared", "heads"]))
def test_norm_gate_oracle(gate, weight):
    r = np.random.default_rng(2)
    x, dy = r.standard_normal((2, 3, 4)), r.standard_normal((2, 3, 4))
    g = None if gate == "none" else r.standard_normal((2, 3, 4))
    w = {None: None, "shared": r.standard_normal(4), "heads": r.standard_normal((3, 4))}[weight]
    y = ol.norm_gate(x, g, w, gate=gate, eps=0.0)
    act = 1.0 if g is None else y * 0 + (g / (1 + np.exp(-g)) if gate == "silu" else 1 / (1 + np.exp(-g)))
    n = y / act / (1.0 if w is None else w)
    assert np.allclose(np.mean(n * n, -1), 1.0)
    got = ol.norm_gate_backward(x, g, w, dy, gate=gate, eps=0.1)
    run = lambda x, g, w: np.sum(ol.norm_gate(x, g, w, gate=gate, eps=0.1) * dy)
    one = lambda v: v
    assert np.max(np.abs(got["dx"] - _differences(lambda v: run(v, g, w), x, one))) < 1e-8
    if g is not None:
        assert np.max(np.abs(got["dg"] - _differences(lambda v: run(x, v, w), g, one))) < 1e-8
    if w is not None:
        assert np.max(np.abs(got["dw"] - _differences(lambda v: run(x, g, v), w, one))) < 1e-8


@pytest.mark.parametrize("after,channel,norm,later", itertools.product([0, 1], [0, 1], [0, 1], [0, 1]))
def test_join_norm_oracle(after, channel, norm, later):
    if not norm and not later:
        return
    r = np.random.default_rng(3)
    x, h, dy, dxo = (r.standard_normal((3, 5)) for _ in range(4))
    wa = r.standard_normal(5) if after else None
    c = r.standard_normal(5) if channel else None
    wb = r.standard_normal(5) if norm else None
    kw = dict(scale=0.7, eps=0.1)

    def loss(x, h, wa, c, wb):
        xo, y = ol.join_norm(x, h, wb, w_after=wa, channel_scale=c, **kw)
        return (np.sum(y * dy) if norm else 0.0) + (np.sum(xo * dxo) if later else 0.0)

    xo, _ = ol.join_norm(x, h, wb, w_after=wa, channel_scale=c, **kw)
    got = ol.join_norm_backward(xo, h, wb, dy if norm else None, dxo if later else None, w_after=wa, channel_scale=c, **kw)
    args = {"dx": x, "dh": h, "dw_after": wa, "dchannel_scale": c, "dw_before": wb}
    names = list(args)
    for i, n in enumerate(names):
        if args[n] is None:
            assert got[n] is None
            continue
        num = _differences(lambda v: loss(*[v if j == i else args[m] for j, m in enumerate(names)]), args[n], lambda v: v)
        assert np.max(np.abs(got[n] - num)) < 1e-8, n


# ---------------------------------------------------------------------------------------------------------- frequencies

def test_rotary_frequencies():
    f, m = sla.rotary_frequencies(64, device="cpu")
    i = np.arange(32)
    assert m == 1.0 and np.max(np.abs(f.numpy() / 10000.0 ** (-i / 32) - 1)) < 1e-15
    lin, m = sla.rotary_frequencies(64, scaling="linear", factor=4.0, device="cpu")
    assert m == 1.0 and np.allclose(lin.numpy(), f.numpy() / 4, rtol=1e-15)
    base, m = sla.rotary_frequencies(64, scaling="base", factor=4.0, device="cpu")
    assert m == 1.0 and base[0] == 1.0 and abs(base[-1] / f[-1] - 0.25) < 1e-12  # the slowest pair slowed by the factor
    blend, m = sla.rotary_frequencies(64, scaling="blend", factor=4.0, original_length=2048, device="cpu")
    turns = 2048 * f.numpy() / (2 * np.pi)
    ratio = blend.numpy() / f.numpy()
    assert np.all(ratio[turns >= 32] == 1.0) and np.allclose(ratio[turns <= 1], 0.25) and np.all(np.diff(ratio) <= 0)
    assert abs(m - (0.1 * np.log(4.0) + 1)) < 1e-15
    for bad in (dict(width=7), dict(width=0), dict(width=8, scaling="dynamic"), dict(width=8, scaling="linear", factor=0.0),
                dict(width=8, scaling="blend", factor=0.5), dict(width=8, scaling="blend", factor=2.0, fast=1.0)):
        with pytest.raises(ValueError):
            sla.rotary_frequencies(**bad)


# -------------------------------------------------------------------------------------------------------------- refusals

def _rp(**kw):
    d = dict(dtype=sla.BF16, B=2, T=16, Hq=4, Hk=4, d=64, rotary=64, flags=0, magnitude=1.0)
    d.update(kw)
    return sla.SlaRotaryParams(**d)


@pytest.mark.parametrize("call", [sla.sla_rotary, sla.sla_rotary_backward])
def test_rotary_rejects_bad_calls(lib, call):
    assert call(_rp(), A, A, A, 0, 0, A, A, 0) in (0, -5)  # valid: reaches the launch (no device here)
    assert call(None, A, A, A, 0, 0, A, A, 0) == -1
    assert call(_rp(B=0), 0, 0, 0, 0, 0, 0, 0, 0) == 0 and call(_rp(T=0), 0, 0, 0, 0, 0, 0, 0, 0) == 0
    for kw, rc in ((dict(dtype=2), -3), (dict(flags=8), -3), (dict(B=-1), -2), (dict(T=-1), -2), (dict(Hq=0), -2), (dict(Hq=1025), -2),
                   (dict(Hk=-1), -2), (dict(d=60), -2), (dict(d=520), -2), (dict(d=0), -2), (dict(rotary=0), -2), (dict(rotary=63), -2),
                   (dict(rotary=66), -2), (dict(B=1 << 16, T=1 << 16), -2)):
        assert call(_rp(**kw), A, A, A, 0, 0, A, A, 0) == rc, kw
    assert call(_rp(flags=sla.FLAG_HEAD_MAJOR), A, A, A, 0, A, A, A, 0) == -3    # packed batches have one layout
    assert call(_rp(flags=sla.FLAG_TOKEN_POSITIONS), A, A, A, 0, 0, A, A, 0) == -1
    for i in (0, 1, 2, 5, 6):
        a = [A, A, A, 0, 0, A, A]
        a[i] = 0
        assert call(_rp(), *a, 0) == -1, i
    assert call(_rp(Hk=0), A, A, A, 0, 0, A, A, 0) == -1 and call(_rp(Hk=0), A, 0, A, 0, 0, A, 0, 0) in (0, -5)
    for i, off in ((0, 8), (1, 8), (2, 4), (3, 2), (4, 2), (5, 8), (6, 8)):
        a = [A, A, A, A, A, A, A]
        a[i] = A + off
        assert call(_rp(), *a, 0) == -4, i


def _np(**kw):
    d = dict(dtype=sla.BF16, B=2, T=16, H=4, dv=64, gate=1, flags=0, eps=1e-5)
    d.update(kw)
    return sla.SlaNormGateParams(**d)


def test_norm_gate_rejects_bad_calls(lib):
    f, b = sla.sla_norm_gate, sla.sla_norm_gate_backward
    n = sla.sla_norm_gate_backward_workspace_bytes(_np())
    assert n > 0 and n % (64 * 4) == 0
    assert f(_np(), A, A, A, 0, A, 0) in (0, -5) and b(_np(), A, A, A, A, 0, A, A, A, A, n, 0) in (0, -5)
    assert f(None, A, A, A, 0, A, 0) == -1 and b(None, A, A, A, A, 0, A, A, A, A, n, 0) == -1
    assert f(_np(B=0), 0, 0, 0, 0, 0, 0) == 0 and b(_np(T=0), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0) == 0
    for kw, rc in ((dict(dtype=5), -3), (dict(gate=3), -3), (dict(gate=-1), -3), (dict(flags=4), -3), (dict(B=-1), -2), (dict(H=0), -2),
                   (dict(H=1025), -2), (dict(dv=4), -2), (dict(dv=100), -2), (dict(dv=520), -2), (dict(eps=-1.0), -2),
                   (dict(eps=float("nan")), -2), (dict(B=1 << 16, T=1 << 16), -2)):
        assert f(_np(**kw), A, A, A, 0, A, 0) == rc and b(_np(**kw), A, A, A, A, 0, A, A, A, A, n, 0) == rc, kw
        assert sla.sla_norm_gate_backward_workspace_bytes(_np(**kw)) == (n if kw.get("gate") else 0), kw
    assert f(_np(gate=0), A, A, A, 0, A, 0) == -1 and f(_np(), A, 0, A, 0, A, 0) == -1  # gate and g go together
    assert f(_np(flags=sla.FLAG_HEAD_MAJOR), A, A, A, A, A, 0) == -3
    assert f(_np(flags=sla.FLAG_HEAD_WEIGHTS), A, A, 0, 0, A, 0) == -1
    for i in (0, 4):
        a = [A, A, A, 0, A]
        a[i] = 0
        assert f(_np(), *a, 0) == -1
    for i in (0, 3, 5, 6, 7):  # x, dy, dx, dg, dw
        a = [A, A, A, A, 0, A, A, A]
        a[i] = 0
        assert b(_np(), *a, A, n, 0) == -1, i
    assert b(_np(), A, A, 0, A, 0, A, A, A, A, n, 0) == -1                           # dw without w
    assert b(_np(), A, A, A, A, 0, A, A, A, A, n - 1, 0) == -6 and b(_np(), A, A, A, A, 0, A, A, A, 0, n, 0) == -6
    for i, off in ((0, 8), (1, 8), (2, 8), (3, 2), (4, 8)):
        a = [A, A, A, A, A]
        a[i] += off
        assert f(_np(), *a, 0) == -4, i
    for i in range(9):
        a = [A] * 9
        a[i] += 2
        assert b(_np(), *a, n, 0) == -4, i


def _jp(**kw):
    d = dict(dtype=sla.BF16, x_dtype=sla.F32, B=2, T=16, D=64, scale=1.0, eps=1e-5)
    d.update(kw)
    return sla.SlaJoinNormParams(**d)


def test_join_norm_rejects_bad_calls(lib):
    f, b = sla.sla_join_norm, sla.sla_join_norm_backward
    n = sla.sla_join_norm_backward_workspace_bytes(_jp())
    assert n > 0 and n % (2 * 64 * 4) == 0
    full_f, full_b = [A, A, A, A, A, 0, A, A], [A, A, A, A, A, A, A, 0, A, A, A, A, A]
    assert f(_jp(), *full_f, 0) in (0, -5) and b(_jp(), *full_b, A, n, 0) in (0, -5)
    assert f(None, *full_f, 0) == -1 and b(None, *full_b, A, n, 0) == -1
    assert f(_jp(B=0), *[0] * 8, 0) == 0 and b(_jp(T=0), *[0] * 13, 0, 0, 0) == 0
    for kw, rc in ((dict(dtype=5), -3), (dict(x_dtype=5), -3), (dict(dtype=sla.F32, x_dtype=sla.BF16), -3), (dict(B=-1), -2), (dict(D=4), -2),
                   (dict(D=68), -2), (dict(D=16392), -2), (dict(eps=-1.0), -2), (dict(eps=float("nan")), -2), (dict(B=1 << 16, T=1 << 16), -2)):
        assert f(_jp(**kw), *full_f, 0) == rc and b(_jp(**kw), *full_b, A, n, 0) == rc, kw
        assert sla.sla_join_norm_backward_workspace_bytes(_jp(**kw)) == 0
    put = lambda full, zero: [0 if i in zero else a for i, a in enumerate(full)]
    # x; h without x_out and the other way round; a norm's weight without y and the other way round; weights of h without h
    for zero in ((0,), (1,), (6,), (4,), (7,), (1, 6), (1, 6, 2), (1, 6, 3)):
        assert f(_jp(), *put(full_f, zero), 0) == -1, zero
    assert f(_jp(), *put(full_f, (1, 2, 3, 6)), 0) in (0, -5)   # the norm alone
    assert f(_jp(), *put(full_f, (4, 7)), 0) in (0, -5)         # the join alone
    assert f(_jp(), *put(full_f, (1, 2, 3, 4, 6, 7)), 0) == -1  # nothing
    # x_out, h, w_after, channel, w_before, dy, dx_out, cu, dx, dh, dw_after, dchannel, dw_before
    for zero in ((0,), (1,), (2,), (3,), (4,), (5,), (8,), (9,), (10,), (11,), (12,)):
        assert b(_jp(), *put(full_b, zero), A, n, 0) == -1, zero
    assert b(_jp(), *put(full_b, (6,)), A, n, 0) in (0, -5)
    assert b(_jp(), *put(full_b, (4, 5, 8, 12)), A, n, 0) in (0, -5)          # the join alone
    assert b(_jp(), *put(full_b, (4, 5, 6, 8, 12)), A, n, 0) == -1            # and nothing flows in
    assert b(_jp(), *put(full_b, (1, 2, 3, 9, 10, 11)), A, n, 0) in (0, -5)   # the norm alone
    assert b(_jp(), *full_b, A, n - 1, 0) == -6 and b(_jp(), *full_b, 0, n, 0) == -6
    for i in range(8):
        a = [A] * 5 + [0] + [A] * 2
        a[i] = A + 2
        assert f(_jp(), *a, 0) == -4, i
    for i in range(14):
        a = [A] * 14
        a[i] += 2
        assert b(_jp(), *a, n, 0) == -4, i


def test_workspace_sizes_follow_the_batch(lib):
    for T in (1, 3, 64, 1000, 100000):
        n = sla.sla_norm_gate_backward_workspace_bytes(_np(B=1, T=T))
        assert n <= 1024 * 64 * 4 and n == sla.sla_norm_gate_backward_workspace_bytes(_np(B=7, T=T), packed=True)
        n = sla.sla_join_norm_backward_workspace_bytes(_jp(B=1, T=T))
        assert n <= 1024 * 2 * 64 * 4 and n == sla.sla_join_norm_backward_workspace_bytes(_jp(B=7, T=T), packed=True)
    assert sla.sla_norm_gate_backward_workspace_bytes(_np(B=0)) == 0 and sla.sla_join_norm_backward_workspace_bytes(_jp(T=0)) == 0


def test_binding_refuses_what_the_library_cannot_see(lib):
    """Types, shapes, orders and devices; every refusal is a ValueError raised before the library is called."""
    import torch

    q, f = torch.zeros(2, 8, 4, 64), torch.ones(32, dtype=torch.float64)
    w, D = torch.ones(64), torch.zeros(2, 8, 64)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    bad = [
        lambda: sla.rotary(q, q, f),                                       # host tensors
        lambda: sla.rotary(q.half(), q.half(), f),
        lambda: sla.rotary(q, q.bfloat16(), f),
        lambda: sla.rotary(q, q[:, :4], f),
        lambda: sla.rotary(q.transpose(1, 2), q, f),
        lambda: sla.rotary(q, q, f.float()),
        lambda: sla.rotary(q, q, f, start=i32(3)),
        lambda: sla.rotary(q, q, f, start=torch.zeros(2, dtype=torch.int64)),
        lambda: sla.rotary(q, q, f, positions=i32(2, 9)),
        lambda: sla.rotary(q, q, f, positions=i32(2, 8), start=i32(2)),
        lambda: sla.rotary(q, q, f, cu_seqlens=i32(3)),
        lambda: sla.rotary(q[0], q[0], f, cu_seqlens=i32(3).long()),
        lambda: sla.rotary(q[0], q[0], f, head_major=True),
        lambda: sla.rotary(q, None, f, k_out=q),
        lambda: sla.rotary(q, q, f, q_out=q.bfloat16()),
        lambda: sla.rotary(q, q.clone(), f, q_out=q, k_out=q),
        lambda: sla.rotary(q, q, f, q_out=q),
        lambda: sla.norm_gate(q, q, w),
        lambda: sla.norm_gate(q, None, w),
        lambda: sla.norm_gate(q, q, w, gate="none"),
        lambda: sla.norm_gate(q, q, w, gate="relu"),
        lambda: sla.norm_gate(q, q[:, :4], w),
        lambda: sla.norm_gate(q, q, w[:32]),
        lambda: sla.norm_gate(q, q, torch.ones(3, 64)),
        lambda: sla.norm_gate(q, q, w.double()),
        lambda: sla.norm_gate(q, q.bfloat16(), w),
        lambda: sla.norm_gate(q, q, w, cu_seqlens=i32(3)),
        lambda: sla.norm_gate(q, q, w, head_major=True, out=q),            # the output is [B,T,H,dv]
        lambda: sla.norm_gate(torch.zeros(1, 4, 4, 64), torch.zeros(1, 4, 4, 64), w, head_major=True, out=torch.zeros(1, 4, 4, 64)),
        lambda: sla.norm_gate_backward(q, q, w, q[:, :4]),
        lambda: sla.join_norm(D, D, w),
        lambda: sla.join_norm(D, D[:, :4], w),
        lambda: sla.join_norm(D, D, w[:32]),
        lambda: sla.join_norm(D, D, w, w_after=w[:32]),
        lambda: sla.join_norm(D, None, None),
        lambda: sla.join_norm(D, None, w, w_after=w),
        lambda: sla.join_norm(D, D.half(), w),
        lambda: sla.join_norm(D, D, None, y=D),
        lambda: sla.join_norm(D, D, w, cu_seqlens=i32(3)),
        lambda: sla.join_norm(D, D, w, x_out=D.bfloat16()),
        lambda: sla.join_norm(D.transpose(0, 1), D.transpose(0, 1), w),
        lambda: sla.join_norm(D, D.clone(), w, y=D),
        lambda: sla.join_norm(D, None, w, y=D),
        lambda: sla.join_norm(D, w.expand(2, 8, 64).contiguous(), w, x_out=D, y=D),
        lambda: (lambda h: sla.join_norm(D, h, w, x_out=h))(D.clone()),
        lambda: sla.join_norm_backward(D, D, w, None),
        lambda: sla.join_norm_backward(D, D, None, None),
        lambda: sla.join_norm_backward(D, None, w, D, w_after=w),
        lambda: sla.join_norm_backward(D, D, w, D.bfloat16()),
        lambda: sla.join_norm_backward(D, D, w, D, D[:, :4]),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {i} was not refused")


def test_calls_run_on_their_tensors_device(monkeypatch):
    """Tensors of another GPU than the current one: the call is made with theirs current, on their current stream."""
    import contextlib

    import torch
    from paper_2602_01744_amd import binding

    current = [0]

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], int(d)
        yield
        current[0] = before

    class Tensor:
        def __init__(self, d):
            self.d, self.device = d, f"cuda:{d}"

        def get_device(self):
            return self.d

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 1000 + d, raising=False)
    seen = []
    for d in (0, 1):
        binding._run(lambda *a: seen.append((current[0],) + a) or 0, Tensor(d), 7)
    assert seen == [(0, 7, 1000), (1, 7, 1001)] and current == [0]
    with pytest.raises(ValueError):
        binding._run(lambda *a: pytest.fail("called"), Tensor(-1), 7)


def test_host_code_under_sanitizers(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "layer_san")
    host = [x for f in ("address", "undefined") for x in ("-Xarch_host", f"-fsanitize={f}")] + ["-Xarch_host", "-fno-sanitize-recover=all"]
    csrc = os.path.join(ROOT, "paper_2602_01744_amd", "csrc")
    cmd = [hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17"] + host + [
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
        "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "sanitize", "layer_main.cpp")] + [
        os.path.join(csrc, f) for f in ("sla_rotary.hip", "sla_norm_gate.hip", "sla_join_norm.hip")] + ["-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env)
    assert res.returncode == 0 and "0 failures" in res.stdout, res.stdout + res.stderr
