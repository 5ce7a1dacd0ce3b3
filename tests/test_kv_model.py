"""The numpy model of the 4-bit cache against its definition (CPU)."""
import numpy as np
import pytest

import kv_model as M


def test_codes_are_the_nearest_and_ties_go_to_the_even_code():
    unit = 2.0 ** -3
    x = np.zeros(32)
    x[0] = 4 * unit * 1.5                       # the largest: the unit is 2^-3
    ties = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    want = [0, 2, 2, 4, 4, 6, 6]                # even codes
    x[1:8] = np.array(ties) * unit
    x[8:15] = -np.array(ties) * unit
    codes, scale = M.quantise_block(x)
    assert scale == 127 - 3
    assert codes[1:8].tolist() == want
    assert codes[8:15].tolist() == [c | 8 for c in want]


@pytest.mark.parametrize("top,unit", [(4.0, 1.0), (7.99, 1.0), (8.0, 2.0), (3.99, 0.5),
                                      (2.0 ** -149, 2.0 ** -127), (3.4e38, 2.0 ** 125)])
def test_unit_of_a_block(top, unit):
    x = np.zeros(32)
    x[5] = -top
    _, scale = M.quantise_block(x)
    assert 2.0 ** (scale - 127) == unit


def test_rows_survive_a_second_quantisation():
    rng = np.random.default_rng(3)
    x = rng.standard_normal(128) * np.exp(rng.standard_normal(128))
    c, s = M.quantise_row(x)
    held = M.values(c, s)
    # half a grid step at most, and the clip of [6, 8) units to 6
    step = np.repeat(2.0 ** (s.astype(float) - 127), 32)
    assert (np.abs(held - x) <= 2 * step).all()
    c2, s2 = M.quantise_row(held)
    assert (M.values(c2, s2) == held).all()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_a_block_that_is_not_finite_is_nan(bad):
    x = np.ones(64)
    x[40] = bad
    v = M.values(*M.quantise_row(x))
    assert (v[:32] == 1).all() and np.isnan(v[32:]).all()


def test_page_operations_balance():
    rng = np.random.default_rng(0)
    c = M.Cache(1, 40, 16, 1, 64, 6, 8)
    for _ in range(300):
        op = rng.integers(4)
        seqs = [int(s) for s in rng.permutation(6)[:3]]
        if op == 0:
            c.truncate(seqs, [int(v) for v in rng.integers(0, 100, 3)])
        elif op == 1:
            c.fork(seqs[:1], seqs[1:2])
        elif op == 2:
            c.reserve(seqs, [int(v) for v in rng.integers(0, 30, 3)])
        else:
            tails = [int(rng.integers(0, c.lens[s] + 1)) for s in seqs]
            c.compact(seqs, tails, [sorted(set(rng.integers(0, max(t, 1), 4).tolist()))
                                    for t in tails])
        held = np.bincount(c.table[c.table >= 0], minlength=40)
        assert (held == c.refs).all()
        assert [(row >= 0).sum() for row in c.table] == [c.pages(int(n)) for n in c.lens]
