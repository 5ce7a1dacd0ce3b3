"""How many bits the weights of the cache's attention carry.

Scores are exact in fp32 (a key's only value is in dim 5) and sequences short,
so that weights' rounding is the largest error besides the result's, and that is
small where the exact value o is small beside the spread p |v - o| (p the
normalised weights).  Over the values of an entry of at most a 16th of their
spread, with R the root of the sum of (round(o) - o)^2 and E that of
(got - o)^2:  E <= 1.05 R + W + S, where
  W  the weights' rounding: off by at most u_w each and in either direction, a
     value is off by u_w sqrt(sum p^2 (v - o)^2)
  S  scores and sums: an exponent is at most 9 (scores 6 apart), so its fma is
     off by 2^-21, the scale's two roundings by 9 * 2^-23, the function by
     2^-22: 2^-19 in all, twice (numerator and sum) of the spread; and n + 8
     sums, each off by at most 2^-23 of p |v|
  1.05  where the result is rounded after being off by W and S, its own rounding
     is another one, of the same distribution.
The test first shows that weights rounded once to q's type would not pass."""
import numpy as np
import pytest
import torch

import kv_model as M
from kv_gpu import DEV, DT, ints, pair, up
from paper_2606_00021_amd import sense

pytestmark = pytest.mark.gpu
SCALE = 0.5


def short_cache(rng, lens, heads, d, page=32):
    _, m = pair(rng, lens, page=page, heads=heads, d=d)
    m.codes[:, :, 0] = 0
    m.codes[:, :, 0, :, :, 2] = rng.integers(0, 16, m.codes[:, :, 0, :, :, 2].shape) << 4
    m.scales[:, :, 0] = 127
    m.scales[:, :, 1] = rng.integers(126, 128, m.scales[:, :, 1].shape)
    return up(m), m


def levels(rng, shape, dtype):
    """Queries of which only dim 5 is not 0: 1, 1/2, -1 or -1/2."""
    q = torch.zeros(shape, dtype=DT[dtype])
    q[..., 5] = torch.tensor(rng.choice([1.0, 0.5, -1.0, -0.5], shape[:-1])).to(q.dtype)
    return q.to(DEV)


def judge(got, q, kv, see, u_w, coarse):
    """got and q [rows, heads, d]; kv [2, n, kv_heads, d]; see [rows, n].
    `coarse`: the type to which weights rounded once have to fail."""
    rows, heads, d = q.shape
    n, group = kv.shape[1], heads // kv.shape[2]
    qd, gd = q.double().cpu().numpy(), got.double().cpu().numpy()
    o, w2, s2, spread = (np.zeros((rows, heads, d)) for _ in range(4))
    once = np.zeros((rows, heads, d))
    for j in range(rows):
        for h in range(heads):
            k, v = kv[0, see[j], h // group], kv[1, see[j], h // group]
            s = k @ qd[j, h] * SCALE
            p = np.exp(s - s.max())
            r = torch.tensor(p).to(coarse).double().numpy()
            once[j, h] = (r @ v) / r.sum()
            p /= p.sum()
            o[j, h] = p @ v
            off = np.abs(v - o[j, h])
            w2[j, h] = (p ** 2) @ off ** 2
            spread[j, h] = p @ off
            s2[j, h] = (2 * 2.0 ** -19 * (p @ off) + (n + 8) * 2.0 ** -23 * (p @ np.abs(v))) ** 2

    small = np.abs(o) <= spread / 16
    o, w2, s2, once, gd = o[small], w2[small], s2[small], once[small], gd[small]

    def rounded(x):
        return torch.tensor(x).to(q.dtype).double().numpy()

    def root(x):
        return float(np.sqrt((x ** 2).sum()))
    most = 1.05 * root(rounded(o) - o) + u_w * np.sqrt(w2.sum()) + np.sqrt(s2.sum())
    assert root(rounded(once) - o) > 1.05 * most, "weights rounded once would pass"
    assert root(gd - o) <= most, (root(gd - o) / most, root(rounded(once) - o) / most)


def causal(m, n):
    return np.arange(n)[None] <= n - m + np.arange(m)[:, None]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,rows,heads,kv", [(64, 1, 12, 2), (128, 4, 8, 2), (128, 3, 16, 2),
                                             (256, 2, 8, 1), (64, 5, 24, 2), (128, 8, 8, 1),
                                             (256, 8, 8, 1)])
def test_few_rows_are_off_by_the_results_rounding(dtype, d, rows, heads, kv):
    print(f"[kv weights] few {dtype} d={d} rows={rows}x{heads}/{kv}", flush=True)
    rng = np.random.default_rng(d + rows + heads)
    lens = [31, 20, 26]
    kvc, m = short_cache(rng, lens, kv, d)
    q = levels(rng, (3, rows, heads, d), dtype)
    out = sense.sense_kv_attention(kvc, 0, q, softmax_scale=SCALE)
    for i, n in enumerate(lens):
        judge(out[i], q[i], m.rows(0, i, 0, n), causal(rows, n),
              (torch.finfo(q.dtype).eps / 2) ** 2, q.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,heads", [(64, 16), (128, 8), (256, 8)])
def test_entries_of_few_rows_are_so_beside_any_other(dtype, d, heads):
    """Single tokens and small trees in one call with a long chunk."""
    print(f"[kv weights] beside {dtype} d={d}", flush=True)
    rng = np.random.default_rng(d)
    lens, counts = [31, 150, 24, 29], [1, 150, 4, 3]
    kvc, m = short_cache(rng, lens, 1, d)
    q = levels(rng, (4, 150, heads, d), dtype)
    out = sense.sense_kv_attention(kvc, 0, q, row_len=ints(counts), softmax_scale=SCALE)
    for i in (0, 2, 3):
        c, n = counts[i], lens[i]
        judge(out[i, :c], q[i, :c], m.rows(0, i, 0, n), causal(c, n),
              (torch.finfo(q.dtype).eps / 2) ** 2, q.dtype)


@pytest.mark.parametrize("d,rows,heads,kv", [(64, 10, 32, 2), (64, 6, 22, 1), (128, 6, 32, 2),
                                             (256, 9, 16, 1), (128, 15, 32, 1)])
def test_many_rows_of_bf16_have_weights_of_11_bits(d, rows, heads, kv):
    print(f"[kv weights] many d={d} rows={rows}x{heads}/{kv}", flush=True)
    rng = np.random.default_rng(d + rows)
    lens = [31, 20, 26]
    kvc, m = short_cache(rng, lens, kv, d)
    q = levels(rng, (3, rows, heads, d), "bf16")
    mask = np.tril(np.ones((3, rows, rows), np.uint8))
    mask[:, rows // 2:, 1] = 0
    out = sense.sense_kv_attention(kvc, 0, q, mask=torch.tensor(mask, device=DEV),
                                   softmax_scale=SCALE)
    for i, n in enumerate(lens):
        see = causal(rows, n)
        see[rows // 2:, n - rows + 1] = False
        judge(out[i], q[i], m.rows(0, i, 0, n), see, 2.0 ** -11, torch.bfloat16)


@pytest.mark.parametrize("d,rows,heads", [(64, 3, 24), (64, 3, 48), (128, 4, 40), (256, 5, 16),
                                          (128, 2, 24)])
def test_values_of_any_size(d, rows, heads):
    """bf16: values from 2^-60 to 2^60, beside each other, among tiny, huge and
    empty blocks: sizes that f16 holds or does not.  Bound: the result's and the
    weights' rounding (2^-11) of each value, and sums of n in fp32."""
    print(f"[kv weights] sizes d={d} rows={rows}x{heads}", flush=True)
    rng = np.random.default_rng(d + heads)
    lens = [300, 77, 40]
    kvc, m = pair(rng, lens, page=16, heads=1, d=d)
    kinds = [(104, 141), (103, 105), (140, 142), (67, 188), (90, 150)]
    for page in range(m.refs.size):
        lo, hi = kinds[page % len(kinds)]
        m.scales[:, page, 1] = rng.integers(lo, hi, m.scales[:, page, 1].shape)
    m.scales[:, ::3, 1, :, 0, ::2] = 0                          # tiny units with zeros only
    codes = m.codes[:, ::3, 1, :, ::2]
    codes[..., :16] &= 0x88
    m.scales[:, ::4, 1, :, -1, 3] = 250
    m.codes[:, ::4, 1, :, 3, -16:] &= 0x88
    kvc = up(m)
    q = torch.tensor(rng.standard_normal((3, rows, heads, d))).to(torch.bfloat16).to(DEV)
    out = sense.sense_kv_attention(kvc, 0, q).double().cpu().numpy()
    qd = q.double().cpu().numpy()
    for i, n in enumerate(lens):
        k, v = m.rows(0, i, 0, n)[:, :, 0]
        for j in range(rows):
            end = n - rows + j + 1
            for h in range(heads):
                s = k[:end] @ qd[i, j, h] * d ** -0.5
                size = (np.abs(k[:end]) @ np.abs(qd[i, j, h])).max() * d ** -0.5
                p = np.exp(s - s.max())
                p /= p.sum()
                o = p @ v[:end]
                ds = (d + 4) * 2.0 ** -23 * size + 2.0 ** -21
                big = p @ np.abs(v[:end])
                tol = (2.0 ** -8 * np.abs(o) + (2.0 ** -11 + 2 * ds) * (p @ np.abs(v[:end] - o))
                       + (n + 8) * 2.0 ** -23 * big
                       + n * 2.0 ** -30 * np.abs(v[:end]).max(0) + 2.0 ** -120)
                assert (np.abs(out[i, j, h] - o) <= tol).all(), (i, j, h)


@pytest.mark.parametrize("d,rows,heads", [(64, 1, 4), (128, 4, 4), (128, 3, 16), (128, 4, 40),
                                          (256, 5, 16)])
def test_values_just_below_2_to_the_80(d, rows, heads):
    """bf16, over long sequences: sums of weights times values stay finite.
    Bound as above."""
    print(f"[kv weights] huge values d={d} rows={rows}x{heads}", flush=True)
    rng = np.random.default_rng(d + heads)
    lens = [1300, 40]
    kvc, m = pair(rng, lens, page=64, heads=1, d=d)
    m.scales[:, :, 1] = 127 + 77
    m.codes[:, :, 1] = rng.choice([0x66, 0x77, 0x75], m.codes[:, :, 1].shape)   # 4 and 6, 3
    kvc = up(m)
    q = torch.tensor(rng.standard_normal((2, rows, heads, d))).to(torch.bfloat16).to(DEV)
    for bound in (0, 1024):
        out = sense.sense_kv_attention(kvc, 0, q, max_kv=bound).double().cpu().numpy()
        for i, n in enumerate(lens):
            k, v = m.rows(0, i, 0, n)[:, :, 0]
            for j in range(rows):
                end = n - rows + j + 1
                s = k[:end] @ q[i, j].double().cpu().numpy().T * d ** -0.5     # [end, heads]
                p = np.exp(s - s.max(0))
                p /= p.sum(0)
                o = p.T @ v[:end]
                size = np.abs(k[:end]) @ np.abs(q[i, j].double().cpu().numpy()).T * d ** -0.5
                ds = ((d + 4) * 2.0 ** -23 * size.max(0) + 2.0 ** -21)[:, None]
                spread = np.stack([p[:, h] @ np.abs(v[:end] - o[h]) for h in range(heads)])
                tol = (2.0 ** -8 * np.abs(o) + (2.0 ** -11 + 2 * ds) * spread
                       + ((n + 8) * 2.0 ** -23 + n * 2.0 ** -30) * np.abs(v).max())
                assert (np.abs(out[i, j] - o) <= tol).all(), (i, j)
