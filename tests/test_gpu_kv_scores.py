"""Attention over the 4-bit cache where scores are large and close together.

Scores are exact in fp32: a key's only values are a constant in dim 5 and one of
0 .. 6 in dim 40 (another block), so a score is level + step times that value.
With scale 1 and u the half step of q's type, o the exact value,
spread = sum w |v - o| / sum w, the bound of one output value is
  u |o|                 the output's own rounding
  u_w spread            the weights' rounding: u, or u^2 where a weight is the
                        sum of two numbers
  2 ds spread           exponents off by ds at most.  They are at most 18 in
                        magnitude where weights count (scores 12 apart, log2 e),
                        so one rounding of one is 2^-20; the scale's two are
                        2^-23 of 18; the exponential's function 2^-21; a weight
                        is made by one of them and moved by at most 6 others
                        (references of its wave, waves, runs): ds = 7 * 2^-18
  (n + 8) 2^-23 max|v|  sums over n positions in fp32
  n 2^-30 max|v|        f16 weights below its normal range
  2^-25                 f16 outputs below it
and none of them depends on the level."""
import numpy as np
import pytest
import torch

import kv_model as M
from kv_gpu import DEV, DT, pair, up
from paper_2606_00021_amd import sense

pytestmark = pytest.mark.gpu


def exact(q, k, v, end, scale=1.0):
    """o and spread [d] of a row q [d] over the first `end` positions."""
    s = k[:end] @ q * scale
    w = np.exp(s - s.max())
    w /= w.sum()
    o = w @ v[:end]
    return o, w @ np.abs(v[:end] - o)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,rows,heads", [(64, 1, 4), (128, 1, 4), (128, 7, 4), (256, 1, 4),
                                          (64, 30, 4), (128, 40, 4), (256, 20, 4), (64, 100, 4)])
def test_large_scores_that_lie_close_together(dtype, d, rows, heads):
    """Levels of 2^14 to 2^21, scores up to 12 apart; every page has a largest
    one of its own, so that waves and runs have different references."""
    print(f"[kv scores] close {dtype} d={d} rows={rows}", flush=True)
    rng = np.random.default_rng(d + rows)
    lens = [2300, 700, 130]
    kvc, m = pair(rng, lens, page=32, heads=1, d=d)
    m.codes[:, :, 0] = 0
    shape = m.codes[:, :, 0, :, :, 2].shape
    m.codes[:, :, 0, :, :, 2] = 6 << 4                      # dim 5: 4 units of 2^8
    cap = rng.integers(1, 9, shape[1])[None, :, None, None]  # dim 40: units of 1
    m.codes[:, :, 0, :, :, 20] = rng.integers(0, 8, shape) % cap + 8 * rng.integers(0, 2, shape)
    m.scales[:, :, 0, :, 0] = 127 + 8
    m.scales[:, :, 0, :, 1] = 127
    kvc = up(m)
    q = torch.zeros((3, rows, heads, d), dtype=DT[dtype], device=DEV)
    q[..., 5] = torch.tensor([2.0 ** 4, 1.5 * 2.0 ** 7, -1.25 * 2.0 ** 9, 2.0 ** 11]).to(DEV)
    q[..., 40] = 1.0
    u = torch.finfo(q.dtype).eps / 2
    out = sense.sense_kv_attention(kvc, 0, q, softmax_scale=1.0).double().cpu().numpy()
    qd = q.double().cpu().numpy()
    for i, n in enumerate(lens):
        k, v = m.rows(0, i, 0, n)[:, :, 0]
        for h in range(heads):
            for j in {0, rows // 2, rows - 1}:
                end = n - rows + j + 1
                o, spread = exact(qd[i, j, h], k, v, end)
                u_w = u * u if rows * heads <= 64 else u
                tol = (u * np.abs(o) + (u_w + 2 * 7 * 2.0 ** -18) * spread
                       + ((n + 8) * 2.0 ** -23 + n * 2.0 ** -30) * np.abs(v).max() + 2.0 ** -25)
                off = np.abs(out[i, j, h] - o) / tol
                assert (off <= 1).all(), (i, h, j, float(off.max()))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("d,rows", [(64, 1), (128, 9), (128, 70)])
def test_references_on_both_sides_of_2_to_the_24(dtype, sign, d, rows):
    """Exponents (score times scale times log2 e) around 2^24, where fp32 goes
    from steps of 1 to 2: some pages' largest lie below, others beyond."""
    print(f"[kv scores] border {dtype} d={d} rows={rows} {sign}", flush=True)
    rng = np.random.default_rng(d + rows)
    lens = [1500, 333]
    kvc, m = pair(rng, lens, page=32, heads=1, d=d)
    m.codes[:, :, 0] = 0
    shape = m.codes[:, :, 0, :, :, 2].shape
    m.codes[:, :, 0, :, :, 2] = 6 << 4                       # dim 5: 2^10
    cap = rng.integers(1, 5, shape[1])[None, :, None, None]  # dim 40: 0 .. 3/8
    m.codes[:, :, 0, :, :, 20] = rng.integers(0, 4, shape) % cap
    m.scales[:, :, 0, :, 0] = 127 + 8
    m.scales[:, :, 0, :, 1] = 127 - 2
    kvc = up(m)
    q = torch.zeros((2, rows, 1, d), dtype=DT[dtype], device=DEV)
    q[..., 5], q[..., 40] = sign * 2.0 ** 10, 1.0             # scores sign 2^20 + 0 .. 3/8
    scale = float(np.float32(2.0 ** 24 / (np.log2(np.e) * (2.0 ** 20 + sign * 0.1875))))
    u = torch.finfo(q.dtype).eps / 2
    out = sense.sense_kv_attention(kvc, 0, q, softmax_scale=scale).double().cpu().numpy()
    qd = q.double().cpu().numpy()
    for i, n in enumerate(lens):
        k, v = m.rows(0, i, 0, n)[:, :, 0]
        for j in {0, rows // 2, rows - 1}:
            o, spread = exact(qd[i, j, 0], k, v, n - rows + j + 1, scale)
            u_w = u * u if rows <= 64 else u
            tol = (u * np.abs(o) + (u_w + 2 * 7 * 2.0 ** -18) * spread
                   + ((n + 8) * 2.0 ** -23 + n * 2.0 ** -30) * np.abs(v).max() + 2.0 ** -25)
            off = np.abs(out[i, j, 0] - o) / tol
            assert (off <= 1).all(), (i, j, float(off.max()))
