"""Workspaces of the gradients around the mixer on packed batches of many sequences: T is the whole batch there, so the number of
sequences has no say in what is asked for, and a call with less is refused."""
import os
import shutil
import subprocess

import pytest

import paper_2602_01744_amd as sla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20  # a 16-byte aligned address that is never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(sla.library_path()):
        from paper_2602_01744_amd import build

        build.build()
    return sla.load_library()


def _gate(B, T, flags=0):
    return sla.SlaNormGateParams(dtype=sla.BF16, B=B, T=T, H=4, dv=64, gate=1, flags=flags, eps=1e-5)


def _join(B, T):
    return sla.SlaJoinNormParams(dtype=sla.BF16, x_dtype=sla.F32, B=B, T=T, D=2048, scale=1.0, eps=1e-5)


# B * T on both sides of 2^30, and past 2^31 and 2^32
@pytest.mark.parametrize("T,B", [(1 << 20, 1024), (1 << 20, 1025), (1 << 20, 4097), (1 << 16, 16384), (1 << 16, 16385), (1 << 16, 1 << 17),
                                 (1 << 30, 1), (1 << 30, 2), (1 << 30, 2 ** 31 - 1), (7, 2 ** 31 - 1)])
def test_packed_sizes_do_not_depend_on_the_number_of_sequences(lib, T, B):
    for flags in (0, sla.FLAG_HEAD_WEIGHTS):
        one = sla.sla_norm_gate_backward_workspace_bytes(_gate(1, T, flags), packed=True)
        assert one > 0 and sla.sla_norm_gate_backward_workspace_bytes(_gate(B, T, flags), packed=True) == one
        assert one == sla.sla_norm_gate_backward_workspace_bytes(_gate(1, T, flags))  # as one row of T tokens
    one = sla.sla_join_norm_backward_workspace_bytes(_join(1, T), packed=True)
    assert one > 0 and sla.sla_join_norm_backward_workspace_bytes(_join(B, T), packed=True) == one
    assert one == sla.sla_join_norm_backward_workspace_bytes(_join(1, T))


@pytest.mark.parametrize("T,B", [(1 << 20, 1024), (1 << 20, 1025), (1 << 16, 16385), (1 << 30, 2)])
def test_packed_gradients_refuse_less_workspace_than_they_write(lib, T, B):
    """-6, and never a launch; no call here has the room it needs."""
    gate = sla.sla_norm_gate_backward_workspace_bytes(_gate(1, T), packed=True)
    join = sla.sla_join_norm_backward_workspace_bytes(_join(1, T), packed=True)
    for size in (0, 16, gate - 1):
        assert sla.sla_norm_gate_backward(_gate(B, T), A, A, A, A, A, A, A, A, A, size, 0) == -6, size
    assert sla.sla_norm_gate_backward(_gate(B, T), A, A, A, A, A, A, A, A, 0, gate, 0) == -6
    for size in (0, 16, join - 1):
        assert sla.sla_join_norm_backward(_join(B, T), A, A, A, A, A, A, A, A, A, A, A, A, A, A, size, 0) == -6, size
    assert sla.sla_join_norm_backward(_join(B, T), A, A, A, A, A, A, A, A, A, A, A, A, A, 0, join, 0) == -6


def test_rectangular_batches_past_the_limit_have_no_size(lib):
    """What a call refuses asks for nothing; a packed batch of the same numbers is a call."""
    for B, T in ((1025, 1 << 20), (2, 1 << 30), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert sla.sla_norm_gate_backward_workspace_bytes(_gate(B, T)) == 0
        assert sla.sla_join_norm_backward_workspace_bytes(_join(B, T)) == 0
        assert sla.sla_norm_gate_backward(_gate(B, T), A, A, A, A, 0, A, A, A, A, 1 << 30, 0) == -2
        assert sla.sla_join_norm_backward(_join(B, T), A, A, A, A, A, A, A, 0, A, A, A, A, A, A, 1 << 30, 0) == -2
    T = (1 << 30) + 1  # more tokens than a packed batch may have
    assert sla.sla_norm_gate_backward_workspace_bytes(_gate(1, T), packed=True) == 0
    assert sla.sla_join_norm_backward_workspace_bytes(_join(1, T), packed=True) == 0
    assert sla.sla_norm_gate_backward(_gate(1, T), A, A, A, A, A, A, A, A, A, 1 << 30, 0) == -2
    assert sla.sla_join_norm_backward(_join(1, T), A, A, A, A, A, A, A, A, A, A, A, A, A, A, 1 << 30, 0) == -2


def test_binding_asks_for_the_packed_size(lib):
    from paper_2602_01744_amd import binding

    T, B = 1 << 20, 2048
    gate = (sla.SlaNormGateParams, sla.BF16, B, T, 4, 64, 1, 0, 1e-5)
    join = (sla.SlaJoinNormParams, sla.BF16, sla.F32, B, T, 2048, 1.0, 1e-5)
    assert binding._workspace_size(*gate, packed=True) == sla.sla_norm_gate_backward_workspace_bytes(_gate(1, T))
    assert binding._workspace_size(*join, packed=True) == sla.sla_join_norm_backward_workspace_bytes(_join(1, T))


def test_packed_host_code_under_sanitizers(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("hipcc not available")
    import torch

    if torch.cuda.is_available():
        pytest.skip("valid calls end at their launch only where there is no GPU")
    exe = str(tmp_path / "layer_packed_san")
    host = [x for f in ("address", "undefined") for x in ("-Xarch_host", f"-fsanitize={f}")] + ["-Xarch_host", "-fno-sanitize-recover=all"]
    csrc = os.path.join(ROOT, "paper_2602_01744_amd", "csrc")
    cmd = [hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17"] + host + [
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
        "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "sanitize", "layer_packed_main.cpp")] + [
        os.path.join(csrc, f) for f in ("sla_rotary.hip", "sla_norm_gate.hip", "sla_join_norm.hip")] + ["-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([exe], capture_output=True, text=True, env=env)
    assert res.returncode == 0 and "0 failures" in res.stdout, res.stdout + res.stderr
