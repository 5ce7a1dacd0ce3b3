"""Page operations of the 4-bit cache against the model that serves one entry
after the other: tables, lengths, counts, statuses and the rows' bytes are
integers and must be equal."""
import numpy as np
import pytest
import torch

import kv_model as M
from kv_gpu import DEV, ints, pair, same_rows, same_tables, up
from paper_2606_00021_amd import sense

pytestmark = pytest.mark.gpu


def check(kv, m, status, want):
    assert status.tolist() == want
    same_tables(kv, m)
    same_rows(kv, m)


def grow(kv, m, seqs, counts):
    """A reserve on both sides.  New positions hold nothing in particular, so
    the rows in front of them are compared, and something is written there."""
    old = m.lens.copy()
    got, want = sense.sense_kv_reserve(kv, ints(counts), ints(seqs)), m.reserve(seqs, counts)
    assert got.tolist() == want
    same_tables(kv, m)
    same_rows(kv, m, old)
    for s, n in enumerate(old):
        for p in range(n, m.lens[s]):
            page, slot = m.cell(s, p)
            m.codes[:, page, :, :, slot] = p % 251
            m.scales[:, page, :, :, :, slot] = s
    kv["codes"].copy_(torch.from_numpy(m.codes))
    kv["scales"].copy_(torch.from_numpy(m.scales))


def test_reserve_serves_in_order_until_pages_run_out():
    print("[kv pages] reserve", flush=True)
    rng = np.random.default_rng(0)
    kv, m = pair(rng, [0, 5, 16, 31, 33, 100], spare=6)
    for seqs, counts in (([3, 1, 0], [1, 11, 0]), ([2, 2, -1, 9, 4], [1, 1, 1, 1, -2]),
                         ([0, 5, 1], [16 * 30, 0, 1]),         # beyond max_pages
                         ([0, 2, 5, 3], [60, 1, 20, 0]),       # the pool ends at the second or third
                         ([3, 4, 0], [1, 40, 1])):
        grow(kv, m, seqs, counts)


def test_forks_share_and_copy_before_they_grow():
    print("[kv pages] fork", flush=True)
    rng = np.random.default_rng(1)
    kv, m = pair(rng, [37, 32, 1, 0], layers=3, heads=3, d=128, spare=40, extra_seqs=9)
    src, dst = [0, 0, 0, 1, 2, 3, 0, 7, 5], [4, 5, 6, 7, 8, 9, 4, 10, 5]
    check(kv, m, sense.sense_kv_fork(kv, ints(src), ints(dst)), m.fork(src, dst))
    # to a sequence that holds tokens, from and to none
    check(kv, m, sense.sense_kv_fork(kv, ints([1, 77, 1, 1]), ints([2, 11, -1, 11])),
          m.fork([1, 77, 1, 1], [2, 11, -1, 11]))
    # all sharers of a partly filled page grow: the last in the list keeps it
    seqs, counts = [5, 0, 6, 4, 7, 1, 8, 2], [1, 1, 0, 20, 1, 1, 1, 16]
    grow(kv, m, seqs, counts)
    grow(kv, m, [6], [3])


def test_truncate_releases_what_nobody_else_holds():
    print("[kv pages] truncate", flush=True)
    rng = np.random.default_rng(2)
    kv, m = pair(rng, [64, 17, 80, 5], spare=10, extra_seqs=3)
    sense.sense_kv_fork(kv, ints([0, 2]), ints([4, 5]))
    m.fork([0, 2], [4, 5])
    for seqs, lens in (([0, 4, 1], [33, 16, 17]), ([2, 2, 2], [70, 3, 40]), ([9, 3, -3, 5], [0, -1, 2, 0]),
                       ([0, 1, 2, 3, 4, 5, 6], [0] * 7)):
        check(kv, m, sense.sense_kv_truncate(kv, ints(lens), ints(seqs)), m.truncate(seqs, lens))
    assert (m.refs == 0).all()
    kv, m = pair(rng, [64, 17])
    check(kv, m, sense.sense_kv_truncate(kv), m.truncate([0, 1], [0, 0]))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 64])
def test_compact_keeps_the_path(d, page):
    print(f"[kv pages] compact d={d} page={page}", flush=True)
    rng = np.random.default_rng(d + page)
    lens = [1, 30, 150, 200, 90, 48, 20, 300]
    kv, m = pair(rng, lens, layers=3, page=page, heads=2, d=d)
    tails = [1, 30, 140, 64, 91, 0, -1, 260]
    ld, rows = 200, 3
    keep = np.full((8, rows, ld), -7, np.int32)
    count = np.zeros((8, rows), np.int32)
    pick = np.array([0, 2, 1, 0, 0, 1, 2, 2], np.int32)
    paths = [[0], [1, 3, 4, 29], list(range(1, 140, 2)), [5, 9, 9, 12], [0], [], [0],
             sorted(rng.permutation(260)[:200].tolist())]
    for i, p in enumerate(paths):
        keep[i, pick[i], :len(p)] = p
        count[i, pick[i]] = len(p)
    got = sense.sense_kv_compact(kv, ints(tails), ints(keep), ints(count), ints(pick))
    want = m.compact(list(range(8)), tails, paths)
    assert want[4] == want[6] == M.REFUSED and want[7] == M.DONE
    check(kv, m, got, want)


def test_compact_refuses_shared_pages_and_odd_lists():
    print("[kv pages] compact refusals", flush=True)
    rng = np.random.default_rng(5)
    kv, m = pair(rng, [40, 40, 40, 40], spare=20, extra_seqs=1)
    sense.sense_kv_fork(kv, ints([1]), ints([4]))
    m.fork([1], [4])
    seqs, tails = [1, 0, 0, 3, 7, 2, 4], [20, 20, 20, 20, 20, 20, 20]
    paths = [[3, 5], [3, 5], [1], [0, 1, 2], [1], None, [0, 1, 2, 3]]
    keep = np.full((7, 2, 5), 1 << 20, np.int32)
    count = np.zeros((7, 2), np.int32)
    pick = [1, 0, 0, 1, 0, 2, 0]                               # 2 is no row
    for i, p in enumerate(paths):
        if p is not None:
            keep[i, pick[i], :len(p)] = p
            count[i, pick[i]] = 99 if i == 3 else len(p)       # clamped to the row, then cut
    got = sense.sense_kv_compact(kv, ints(tails), ints(keep), ints(count), ints(pick),
                                 seqs=ints(seqs))
    want = m.compact(seqs, tails, paths)
    assert want == [M.REFUSED, M.DONE, M.REFUSED, M.DONE, M.REFUSED, M.REFUSED, M.DONE]
    check(kv, m, got, want)


@pytest.mark.parametrize("seed", range(4))
def test_random_operations(seed):
    print(f"[kv pages] random {seed}", flush=True)
    rng = np.random.default_rng(seed)
    page = [16, 32, 64, 128][seed]
    kv, m = pair(rng, [0, 20, 70, 5, 33, 1], layers=2, page=page, spare=12, extra_seqs=6)
    for _ in range(60):
        op = rng.integers(5)
        n = int(rng.integers(1, 7))
        seqs = [int(s) for s in rng.integers(-1, 13, n)]
        if op == 0:
            lens = [int(v) for v in rng.integers(-1, 90, n)]
            check(kv, m, sense.sense_kv_truncate(kv, ints(lens), ints(seqs)), m.truncate(seqs, lens))
        elif op == 1:
            dst = [int(s) for s in rng.integers(-1, 13, n)]
            check(kv, m, sense.sense_kv_fork(kv, ints(seqs), ints(dst)), m.fork(seqs, dst))
        elif op <= 3:
            counts = [int(v) for v in rng.integers(-1, 50, n)]
            grow(kv, m, seqs, counts)
        else:
            tails = [int(rng.integers(0, m.lens[s] + 2)) if 0 <= s < 12 else 3 for s in seqs]
            paths = [sorted(set(rng.integers(0, max(t, 1) + 1, 6).tolist())) for t in tails]
            keep = np.zeros((n, 8), np.int32)
            for i, p in enumerate(paths):
                keep[i, :len(p)] = p
            got = sense.sense_kv_compact(kv, ints(tails), ints(keep), ints([len(p) for p in paths]),
                                         seqs=ints(seqs))
            check(kv, m, got, m.compact(seqs, tails, paths))


def test_large_pools_and_lists():
    """More pages than a workgroup scans at once, few of them free; the largest
    list of entries."""
    print("[kv pages] large pool", flush=True)
    rng = np.random.default_rng(8)
    n, pages = 4096, 21_003
    m = M.Cache(1, pages, 16, 1, 64, n, 4)
    free = np.sort(rng.choice(pages, 3000, replace=False))
    m.refs[:] = 1
    m.refs[free] = rng.integers(-1, 1, 3000)
    kv = up(m)
    seqs = rng.permutation(n).tolist()
    counts = rng.integers(0, 30, n).tolist()
    got = sense.sense_kv_reserve(kv, ints(counts), ints(seqs))
    want = m.reserve(seqs, counts)
    assert M.DONE in want and M.NO_PAGES in want
    assert got.tolist() == want
    same_tables(kv, m)


def test_tables_that_make_no_sense_stay_in_bounds():
    """Lengths beyond the capacity and below 0, page ids that are none: the
    calls end, and what is sound elsewhere stays as it was."""
    print("[kv pages] broken tables", flush=True)
    rng = np.random.default_rng(9)
    kv, m = pair(rng, [40, 40, 40, 40], spare=8)
    kv["seq_len"][1] = 1 << 30
    kv["seq_len"][2] = -5
    kv["page_table"][3, 1:] = ints([1 << 30, -9] + [-1] * (kv["page_table"].shape[1] - 3))
    keep = ints([[1, 2, 3]] * 4)
    sense.sense_kv_compact(kv, ints([20] * 4), keep, ints([3] * 4))
    sense.sense_kv_reserve(kv, ints([5] * 4))
    sense.sense_kv_truncate(kv, ints([10] * 4))
    torch.cuda.synchronize()
    m.compact([0], [20], [[1, 2, 3]])
    m.reserve([0], [5])
    m.truncate([0], [10])
    assert kv["seq_len"][0].item() == 10 and kv["seq_len"][1].item() == 10
    assert np.array_equal(kv["page_table"][0].cpu().numpy(), m.table[0])


def test_offsets_beyond_32_bits():
    """A copy and a path at the end of a cache of more than 4 GiB."""
    print("[kv pages] large", flush=True)
    layers, pages, page, heads, d, n = 9, 4096, 128, 8, 128, 100
    old, new = pages - 1, pages - 2
    kv = {"codes": torch.zeros((layers, pages, 2, heads, page, d // 2), dtype=torch.uint8, device=DEV),
          "scales": torch.zeros((layers, pages, 2, heads, d // 32, page), dtype=torch.uint8, device=DEV),
          "page_table": ints([[old], [-1]]), "seq_len": ints([n, 0]),
          "page_refs": torch.ones(pages, dtype=torch.int32, device=DEV)}
    assert kv["codes"].numel() > 1 << 32
    kv["page_refs"][new] = 0                                  # the one free page
    for name, hi in (("codes", 256), ("scales", 255)):
        t = kv[name][:, old]
        t.copy_(torch.randint(0, hi, t.shape, dtype=torch.uint8, device=DEV))
    codes, scales = kv["codes"][:, old].clone(), kv["scales"][:, old].clone()
    assert sense.sense_kv_fork(kv, ints([0]), ints([1])).tolist() == [0]
    assert sense.sense_kv_reserve(kv, ints([1]), ints([1])).tolist() == [0]
    assert kv["page_table"].tolist() == [[old], [new]] and kv["seq_len"].tolist() == [n, n + 1]
    assert kv["page_refs"][[old, new]].tolist() == [1, 1]
    assert torch.equal(kv["codes"][:, new, :, :, :n], codes[:, :, :, :n])
    assert torch.equal(kv["scales"][:, new, :, :, :, :n], scales[..., :n])
    keep = [0, 3, 4, 18]
    assert sense.sense_kv_compact(kv, ints([20]), ints([keep]), ints([4]), seqs=ints([1])).tolist() == [0]
    base = n + 1 - 20
    at = list(range(base)) + [base + u for u in keep]
    assert kv["seq_len"].tolist() == [n, base + 4]
    assert torch.equal(kv["codes"][:, new, :, :, :base + 4], codes[:, :, :, at])
    assert torch.equal(kv["scales"][:, new, :, :, :, :base + 4], scales[..., at])
    assert torch.equal(kv["codes"][:, old], codes) and torch.equal(kv["scales"][:, old], scales)
    assert int(kv["codes"][:, :new].count_nonzero()) == int(kv["scales"][:, :new].count_nonzero()) == 0
