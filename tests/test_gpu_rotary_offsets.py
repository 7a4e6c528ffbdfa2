"""Rotary positions on packed batches whose offsets leave the tensors: a sequence begins at its clamped start, as for the mixer's
packed calls."""
import numpy as np
import pytest

from layer_util import STEP, numpy64, rounded, tensor, within
from oracle import sla_layer as ol

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("adjacent,r", [(False, 64), (True, 48), (False, 22)])
@pytest.mark.parametrize("cu", [[-3, 5, 99], [-2147483648, 2147483647], [-7, -2, 4, 12], [-5, -5, 0, 12], [-1, 13], [2, 20, 30], [-4, -1]])
def test_positions_count_from_the_clamped_start(dtype, adjacent, r, cu):
    import torch
    import paper_2602_01744_amd as sla

    T, H, d = 12, 3, 64
    rng = np.random.default_rng(r + len(cu))
    x = rounded(rng.standard_normal((T, H, d)), dtype)
    f = 10000.0 ** (-2.0 * np.arange(r // 2) / r)
    start = rng.integers(0, 1000, size=len(cu) - 1).astype(np.int32)
    inside, at, seq = np.zeros(T, bool), np.zeros(T, np.int64), np.zeros(T, np.int64)
    for b in range(len(cu) - 1):
        lo = min(max(cu[b], 0), T)
        hi = min(max(cu[b + 1], lo), T)
        inside[lo:hi], at[lo:hi], seq[lo:hi] = True, np.arange(hi - lo), b
    c, ft = torch.tensor(cu, dtype=torch.int32, device="cuda"), torch.from_numpy(f).cuda()
    for call, inverse in ((sla.rotary, False), (sla.rotary_backward, True)):
        for name, where, kw in (("zero", at, {}), ("start", at + start[seq], {"start": torch.from_numpy(start).cuda()})):
            out = torch.full_like(tensor(x, dtype), 7.0)
            call(tensor(x, dtype), None, ft, cu_seqlens=c, adjacent=adjacent, **{"dq" if inverse else "q_out": out}, **kw)
            got = numpy64(out)
            assert np.all(got[~inside] == 7.0)
            if not inside.any():
                continue
            want = ol.rotary(x[inside], where[inside], f, adjacent=adjacent, inverse=inverse)
            a = np.arange(0, r, 2) if adjacent else np.arange(r // 2)
            b = a + (1 if adjacent else r // 2)
            terms = np.zeros_like(want)
            # 8 fp32 steps of both terms (sine and cosine, the products), and the angle's 2^-51 of itself, which is under 2^-41
            pair = np.abs(x[inside][..., a].astype(np.float64)) + np.abs(x[inside][..., b])
            terms[..., a] = terms[..., b] = (8 + 2.0 ** -41 / STEP) * pair
            within(name, got[inside], want, terms, dtype, steps=1)


def test_more_than_2_30_sequences():
    """The search for a token's sequence halves ranges whose ends add to more than 2^31; all sequences but two are empty."""
    import torch
    import paper_2602_01744_amd as sla

    B, T = (1 << 30) + 5, 9
    if torch.cuda.mem_get_info()[0] < 12 * 2 ** 30:
        pytest.skip("not enough memory")
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    cu[-2], cu[-1], start[-2], start[-1] = 4, T, 70, 100000
    x = torch.randn(T, 2, 64, device="cuda")
    f, _ = sla.rotary_frequencies(64)
    y, _ = sla.rotary(x, None, f, cu_seqlens=cu, start=start)
    at = torch.tensor([70, 71, 72, 73, 100000, 100001, 100002, 100003, 100004], dtype=torch.int32, device="cuda")
    want, _ = sla.rotary(x[None], None, f, positions=at[None])
    assert torch.equal(y, want[0])
