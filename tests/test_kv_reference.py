"""The two references of the cache's attention against each other (CPU): the one
with bounds (test_gpu_kv_attention) and the model's, row by row (kv_model)."""
import numpy as np
import pytest
import torch

import kv_model as M
from test_gpu_kv_attention import reference, sees


@pytest.mark.parametrize("m,n,heads,kv,d", [(1, 1, 1, 1, 64), (3, 20, 4, 2, 64), (7, 5, 2, 1, 128),
                                            (4, 0, 2, 2, 64)])
def test_references_agree(m, n, heads, kv, d):
    rng = np.random.default_rng(m + n)
    q = torch.tensor(rng.standard_normal((m, heads, d))).to(torch.bfloat16)
    held = rng.standard_normal((2, n, kv, d))
    masks = rng.random((m, m)) < 0.5
    masks[0] = False
    for see in (sees(m, n), sees(m, n, masks)):
        see[:max(m - n, 0)] = False                  # rows of positions below 0
        o, tol = reference(q, held, d ** -0.5, see)
        want = M.attention(q.double().numpy(), held[0], held[1], d ** -0.5, see)
        assert np.abs(o.numpy() - want).max() < 1e-12
        assert (tol > 0).all()


def test_the_model_spreads_nan_as_far_as_the_row_sees_it():
    q, k, v = np.ones((3, 1, 64)), np.zeros((3, 1, 64)), np.ones((3, 1, 64))
    k[2, 0, 5] = np.nan
    v[1, 0, 32:] = np.nan
    out = M.attention(q, k, v, 1.0, np.tril(np.ones((3, 3), bool)))
    assert np.isfinite(out[0]).all()
    assert np.isfinite(out[1, 0, :32]).all() and np.isnan(out[1, 0, 32:]).all()
    assert np.isnan(out[2]).all()
