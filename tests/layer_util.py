"""Inputs and error bounds shared by the tests of the operators around the mixer.

Bounds count roundings: one to the output's type is at most half a step, `finfo.eps / 2` of the value; what the kernels do in
fp32 is at most K steps of 2^-24 of the terms that a value is the sum of.  K: a sum of squares over a row is at most 8 V
additions in a lane, 6 exchanges between lanes and 16 waves (8 * 4 + 22 = 54 for a row of 16384), halved by the root, 3 for
the root and the mean, 2 for the products with it and the weight; the gate's exp2 argument is rounded to |g| 2^-24 relative
to the result twice, and exp2, reciprocal and the additions around them make 6.  K = 64 + 2 |g|.
"""
from __future__ import annotations

import numpy as np

STEP = 2.0 ** -24
K = 64


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24


def rounded(a, dtype):
    import sla_inputs as si

    a = np.ascontiguousarray(a, dtype=np.float32)
    return si.round_to_bf16(a) if dtype == "bf16" else a


def tensor(a, dtype="f32"):
    import torch

    if a is None:
        return None
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()


def numpy64(t):
    return t.float().cpu().numpy().astype(np.float64)


def within(name, got, want, terms, dtype, steps=K):
    """|got - want| <= half a step of the type at want, and `steps` fp32 steps of `terms` (1e-37: results that leave the
    normal range are flushed)."""
    got = numpy64(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == want.shape, (name, got.shape, want.shape)
    bound = half_step(dtype) * np.abs(want) * (1 + 2.0 ** -8) + steps * STEP * terms * 1.01 + 1e-37
    bad = ~(np.abs(got - want) <= bound)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) / bound, 0)), want.shape)
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.size} out of bounds, worst at {i}: got {got[i]!r}, want "
                             f"{want[i]!r}, bound {bound[i]!r}")


def sequences(r, n, T, pad):
    """cu_seqlens of n sequences (one of them empty) over T tokens, the first and the last `pad` tokens outside."""
    cuts = np.sort(r.integers(pad, T - pad + 1, size=n - 1)) if n > 1 else np.zeros(0, np.int64)
    cu = np.concatenate([[pad], cuts, [T - pad]])
    if n > 2:
        cu[2] = cu[1]
    return cu.astype(np.int32)
