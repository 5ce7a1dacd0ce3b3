"""Helpers of the GPU tests of the 4-bit cache: caches filled from numpy, and
the model beside them."""
import numpy as np
import torch

import kv_model as M
from paper_2606_00021_amd import sense

DEV = "cuda"
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def pair(rng, lens, layers=1, page=16, heads=2, d=64, spare=4, extra_seqs=0, fill=True):
    """A cache on the GPU and its model: sequences of the given lengths in
    shuffled pages, random codes and scales (also in slots nobody uses)."""
    held = [-(-n // page) for n in lens]
    total = sum(held) + spare
    cap = max(held + [1]) + spare
    m = M.Cache(layers, total, page, heads, d, len(lens) + extra_seqs, cap)
    if fill:
        m.codes[:] = rng.integers(0, 256, m.codes.shape)
        m.scales[:] = rng.integers(122, 128, m.scales.shape)
    order = rng.permutation(total)
    at = 0
    for s, n in enumerate(held):
        m.table[s, :n] = order[at:at + n]
        m.refs[order[at:at + n]] = 1
        m.lens[s] = lens[s]
        at += n
    return up(m), m


def up(m):
    return {"codes": torch.from_numpy(m.codes.copy()).to(DEV),
            "scales": torch.from_numpy(m.scales.copy()).to(DEV),
            "page_table": ints(m.table), "seq_len": ints(m.lens), "page_refs": ints(m.refs)}


def same_tables(kv, m):
    assert np.array_equal(kv["page_table"].cpu().numpy(), m.table)
    assert np.array_equal(kv["seq_len"].cpu().numpy(), m.lens)
    assert np.array_equal(kv["page_refs"].cpu().numpy(), m.refs)


def same_rows(kv, m, lens=None):
    """Every position of every sequence (of its first lens) holds the model's
    bytes."""
    codes, scales = kv["codes"].cpu().numpy(), kv["scales"].cpu().numpy()
    for s, n in enumerate(m.lens if lens is None else lens):
        pos = np.arange(n)
        page, slot = m.table[s, pos // m.page], pos % m.page
        assert np.array_equal(codes[:, page, :, :, slot], m.codes[:, page, :, :, slot]), s
        assert np.array_equal(scales[:, page, :, :, :, slot], m.scales[:, page, :, :, :, slot]), s


def empty(**kw):
    return sense.sense_build_kv_cache(device=DEV, **kw)
