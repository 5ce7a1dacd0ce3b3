"""Rows into the 4-bit cache and back (sense_kv_write, sense_kv_read).

Both are exact by definition (one rounding to the nearest code, none on the
way back in a type that holds the values), so bytes and values must equal the
model's."""
import numpy as np
import pytest
import torch

import kv_model as M
from kv_gpu import DEV, DT, ints, pair, same_rows
from paper_2606_00021_amd import sense

pytestmark = pytest.mark.gpu


def rows(rng, shape, dtype):
    """Values of many magnitudes, zeros, and ties of the grid."""
    x = rng.standard_normal(shape) * np.exp(2 * rng.standard_normal(shape[:-1] + (1,)))
    x[rng.random(shape) < 0.05] = 0.0
    tie = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5, -0.25, -2.5, 4.0], shape)
    x = np.where(rng.random(shape) < 0.3, tie, x)
    return torch.tensor(x, dtype=torch.float32).to(DT[dtype]).to(DEV)


def model_write(m, layer, s, rows_k, rows_v, first):
    for w, x in ((0, rows_k), (1, rows_v)):
        x = x.double().cpu().numpy()
        for j in range(x.shape[0]):
            for h in range(x.shape[1]):
                m.write(layer, s, first + j, w, h, x[j, h])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("d,page,heads,q", [(64, 16, 3, 1), (64, 128, 1, 37), (128, 16, 2, 5),
                                            (128, 32, 8, 1), (128, 64, 5, 33), (256, 16, 1, 17),
                                            (256, 32, 3, 2)])
def test_written_rows_equal_the_model(dtype, d, page, heads, q):
    print(f"[kv rows] {dtype} d={d} page={page} heads={heads} q={q}", flush=True)
    rng = np.random.default_rng(d + page + q)
    lens = [q, q + 1, q + page - 1, 3 * page + q]
    kv, m = pair(rng, lens, layers=2, page=page, heads=heads, d=d)
    k, v = rows(rng, (4, q, heads, d), dtype), rows(rng, (4, q, heads, d), dtype)
    sense.sense_kv_write(kv, 1, k, v)
    for s in range(4):
        model_write(m, 1, s, k[s], v[s], lens[s] - q)
    same_rows(kv, m)
    # nothing else changed
    assert np.array_equal(kv["codes"].cpu().numpy(), m.codes)
    assert np.array_equal(kv["scales"].cpu().numpy(), m.scales)
    gk, gv = torch.full_like(k, 9), torch.full_like(v, 9)
    sense.sense_kv_read(kv, 1, gk, gv)
    for s in range(4):
        want = m.rows(1, s, lens[s] - q, lens[s])
        for got, w in ((gk, want[0]), (gv, want[1])):
            assert torch.equal(got[s].cpu(), torch.tensor(w).to(DT[dtype]))


def test_extreme_blocks():
    """Blocks of zeros, subnormals, the largest values, NaN and infinities."""
    print("[kv rows] extremes", flush=True)
    rng = np.random.default_rng(1)
    kv, m = pair(rng, [6], d=64, heads=1)
    x = torch.zeros((1, 6, 1, 64))
    x[0, 1, 0, :4] = torch.tensor([1e-45, -3e-45, 2.0 ** -127, 0.0])
    x[0, 1, 0, 32:36] = torch.tensor([-0.0, 1.17e-38, 5e-39, -1e-38])
    x[0, 2, 0, :3] = torch.tensor([3.4e38, -3.4028235e38, 1e37])
    x[0, 3, 0, 7] = float("nan")
    x[0, 4, 0, 40] = float("inf")
    x[0, 5, 0, 3] = -float("inf")
    x = x.to(DEV)
    sense.sense_kv_write(kv, 0, x, x)
    model_write(m, 0, 0, x[0], x[0], 0)
    same_rows(kv, m)
    got, _ = sense.sense_kv_read(kv, 0, torch.empty_like(x), torch.empty_like(x))
    want = m.rows(0, 0, 0, 6)[0]
    assert np.array_equal(got[0].cpu().double().numpy(), want, equal_nan=True)


def test_ragged_strided_rows_of_listed_sequences():
    """Rows cut out of a wider tensor, sequences out of order, empty entries,
    entries of no sequence, a sequence named twice, rows beyond the tensor."""
    print("[kv rows] ragged", flush=True)
    rng = np.random.default_rng(2)
    heads, d = 2, 128
    kv, m = pair(rng, [40, 3, 77, 50], heads=heads, d=d, page=32)
    fused = rows(rng, (30, 6, d), "bf16")                      # [q q | k k | v v] heads
    k, v = fused[:, 2:4], fused[:, 4:6]
    seqs, start, count = [2, 0, 9, 1, 2, -1, 3], [0, 5, 6, 11, 14, 0, 28], [5, 0, 2, 7, 3, 2, 4]
    sense.sense_kv_write(kv, 0, k, v, seqs=ints(seqs), row_start=ints(start), row_len=ints(count),
                         max_rows=6)
    model_write(m, 0, 2, k[0:5], v[0:5], 77 - 5)
    # 7 rows are cut to max_rows = 6, of which positions below 0 do not exist
    model_write(m, 0, 1, k[14:17], v[14:17], 0)
    model_write(m, 0, 3, k[28:30], v[28:30], 46)               # the tensor ends at row 30
    assert np.array_equal(kv["codes"].cpu().numpy(), m.codes)
    assert np.array_equal(kv["scales"].cpu().numpy(), m.scales)
    out = torch.full((30, 6, d), 7.0, dtype=torch.float32, device=DEV)
    sense.sense_kv_read(kv, 0, out[:, 2:4], out[:, 4:6], seqs=ints([3, 1]), row_start=ints([2, 20]),
                        row_len=ints([3, 99]), max_rows=5)
    want = np.full((30, 6, d), 7.0)
    want[2:5, 2:4], want[2:5, 4:6] = m.rows(0, 3, 47, 50)
    # 5 rows of a sequence of 3: the first two have no position
    want[22:25, 2:4], want[22:25, 4:6] = m.rows(0, 1, 0, 3)
    assert np.array_equal(out.cpu().double().numpy(), want)


def test_layers_in_one_call_and_pages_that_are_none():
    print("[kv rows] layers, bad pages", flush=True)
    rng = np.random.default_rng(4)
    kv, m = pair(rng, [20, 20], layers=4, heads=2, d=64)
    k, v = rows(rng, (3, 2, 18, 2, 64), "f16"), rows(rng, (3, 2, 18, 2, 64), "f16")
    for bad in (-1, 1 << 30, -(1 << 31)):
        kv["page_table"][1, 1] = bad
        sense.sense_kv_write(kv, 1, k, v)
        got = sense.sense_kv_read(kv, 1, torch.full_like(k, 3), torch.full_like(v, 3))
        for layer in range(3):
            model_write(m, 1 + layer, 0, k[layer, 0], v[layer, 0], 2)
            model_write(m, 1 + layer, 1, k[layer, 1, :14], v[layer, 1, :14], 2)
            for i in (0, 1):
                assert torch.equal(got[i][layer, 0].cpu(),
                                   torch.tensor(m.rows(1 + layer, 0, 2, 20)[i]).half())
                assert torch.equal(got[i][layer, 1, :14].cpu(),
                                   torch.tensor(m.rows(1 + layer, 1, 2, 16)[i]).half())
                assert (got[i][layer, 1, 14:] == 0).all()
        assert np.array_equal(kv["codes"].cpu().numpy(), m.codes)


def test_offsets_beyond_32_bits():
    """The last page of the last layer of a cache of more than 4 GiB."""
    print("[kv rows] large", flush=True)
    layers, pages, page, heads, d = 9, 4096, 128, 8, 128
    kv = {"codes": torch.zeros((layers, pages, 2, heads, page, d // 2), dtype=torch.uint8, device=DEV),
          "scales": torch.zeros((layers, pages, 2, heads, d // 32, page), dtype=torch.uint8, device=DEV),
          "page_table": ints([[pages - 1]]), "seq_len": ints([page]),
          "page_refs": torch.zeros(pages, dtype=torch.int32, device=DEV)}
    assert kv["codes"].numel() > 1 << 32
    rng = np.random.default_rng(5)
    k, v = rows(rng, (1, page, heads, d), "bf16"), rows(rng, (1, page, heads, d), "bf16")
    sense.sense_kv_write(kv, layers - 1, k, v)
    gk, gv = sense.sense_kv_read(kv, layers - 1, torch.empty_like(k), torch.empty_like(v))
    tail = kv["codes"][-1, -1].cpu().numpy()
    c, s = M.quantise_row(v[0, -1, -1].double().cpu().numpy())
    assert np.array_equal(tail[1, -1, -1], c)
    assert torch.equal(gv[0, -1, -1].cpu().double(), torch.tensor(M.values(c, s)))
    c, s = M.quantise_row(k[0, 0, 0].double().cpu().numpy())
    assert torch.equal(gk[0, 0, 0].cpu().double(), torch.tensor(M.values(c, s)))
    assert int(kv["codes"][:-1].count_nonzero()) == 0
    assert int(kv["codes"][-1, :-1].count_nonzero()) == 0
