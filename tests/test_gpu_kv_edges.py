"""The cache's attention where an entry has more rows than positions.  Bounds as
in test_gpu_kv_attention."""
import numpy as np
import pytest
import torch

from kv_gpu import DEV, pair
from paper_2606_00021_amd import sense
from test_gpu_kv_attention import queries, reference, sees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,rows,n,heads", [(64, 6, 3, 1), (128, 6, 0, 4), (128, 20, 7, 4),
                                            (64, 40, 33, 4), (256, 12, 11, 8), (128, 90, 60, 2),
                                            (64, 90, 17, 8)])
def test_rows_of_positions_below_zero_see_nothing(dtype, d, rows, n, heads):
    """The last n rows have the n positions; the others become 0, whatever their
    row of a mask names, also where the output is the queries' own memory."""
    print(f"[kv edges] below 0 {dtype} d={d} rows={rows} n={n}", flush=True)
    rng = np.random.default_rng(d + rows + n)
    kvc, m = pair(rng, [n, n + 5], page=16, heads=1, d=d)
    q = queries(rng, (2, rows, heads, d), dtype)
    mask = np.ones((2, rows, rows), np.uint8)
    mask[1] = rng.random((rows, rows)) < 0.5
    for given in (None, torch.tensor(mask, device=DEV)):
        out = sense.sense_kv_attention(kvc, 0, q, mask=given)
        for i, length in enumerate((n, n + 5)):
            below = max(rows - length, 0)
            assert (out[i, :below] == 0).all()
            see = sees(rows, length, None if given is None else mask[i])
            see[:below] = False
            ref, tol = reference(q[i], m.rows(0, i, 0, length), d ** -0.5, see)
            assert ((out[i].double().cpu() - ref).abs() <= tol).all(), i
        own = q.clone()
        assert sense.sense_kv_attention(kvc, 0, own, mask=given, out=own) is own
        assert torch.equal(own, out)


def test_a_long_chunk_of_more_rows_than_positions():
    """Cut into runs and joined: rows in front of the sequence are 0."""
    print("[kv edges] below 0, cut", flush=True)
    rng = np.random.default_rng(5)
    rows, n, d = 1500, 1300, 64
    kvc, m = pair(rng, [n], page=64, heads=1, d=d)
    q = queries(rng, (1, rows, 1, d), "bf16")
    mask = np.ones((1, rows, rows), np.uint8)
    assert sense.sense_kv_attention_workspace_size(kvc, 1, rows, 1) > 0
    for given in (None, torch.tensor(mask, device=DEV)):
        out = sense.sense_kv_attention(kvc, 0, q, mask=given)
        assert (out[0, :rows - n] == 0).all()
        at = [rows - n, rows - n + 1, rows - 700, rows - 1]
        see = sees(rows, n, None if given is None else mask[0])[at]
        ref, tol = reference(q[0, at], m.rows(0, 0, 0, n), d ** -0.5, see)
        assert ((out[0, at].double().cpu() - ref).abs() <= tol).all()
