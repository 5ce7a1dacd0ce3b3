"""A cache built, grown, written and attended beside the numpy model, with values
that are not finite among those written.  Bounds as in test_gpu_kv_attention."""
import numpy as np
import pytest
import torch

import kv_model as M
from kv_gpu import DEV, DT, empty, ints, same_rows, same_tables
from paper_2606_00021_amd import sense
from test_gpu_kv_attention import queries, reference, sees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,heads,kv", [(64, 4, 2), (128, 3, 1), (256, 2, 1), (128, 40, 1)])
def test_steps_from_an_empty_cache(dtype, d, heads, kv):
    print(f"[kv model] steps {dtype} d={d} {heads}/{kv}", flush=True)
    rng = np.random.default_rng(d + heads)
    seqs, pages, page = 3, 24, 16
    kvc = empty(n_layers=2, n_pages=pages, page_size=page, n_kv_heads=kv, head_dim=d, n_seqs=seqs,
                max_pages=8)
    m = M.Cache(2, pages, page, kv, d, seqs, 8)
    for counts in ([5, 33, 0], [4, 1, 20], [7, 7, 7]):
        status = sense.sense_kv_reserve(kvc, ints(counts))
        assert status.cpu().tolist() == m.reserve(list(range(seqs)), counts)
        rows = max(counts)
        x = torch.tensor(rng.standard_normal((2, seqs, rows, kv, d))).to(DT[dtype])
        x[1, 1, 0, 0, d - 1] = float("nan")          # a value of sequence 1
        x[0, 0, counts[0] - 1, kv - 1, 3] = float("inf")     # a key of sequence 0
        x = x.to(DEV)
        sense.sense_kv_write(kvc, 1, x[0], x[1], row_len=ints(counts))
        for s in range(seqs):
            for j in range(counts[s]):
                for w in (0, 1):
                    for h in range(kv):
                        m.write(1, s, int(m.lens[s]) - counts[s] + j, w, h,
                                x[w, s, j, h].double().cpu().numpy())
        same_tables(kvc, m)
        same_rows(kvc, m)
        q = queries(rng, (seqs, rows, heads, d), dtype)
        out = sense.sense_kv_attention(kvc, 1, q, row_len=ints(counts))
        nan = 0
        for s, c in enumerate(counts):
            n = int(m.lens[s])
            held, see = m.rows(1, s, 0, n), sees(c, n)
            want = M.attention(q[s, :c].double().cpu().numpy(), held[0], held[1], d ** -0.5, see)
            got = out[s, :c].double().cpu().numpy()
            assert np.array_equal(np.isnan(got), np.isnan(want)), s
            _, tol = reference(q[s, :c], np.nan_to_num(held), d ** -0.5, see)
            ok = ~np.isnan(want)
            assert (np.abs(got - want)[ok] <= tol.numpy()[ok]).all(), s
            nan += int((~ok).sum())
        assert nan > 0
