"""Attention over the 4-bit cache against the definition in 64 bits.

Bound of one output value, with u the half step of q's type (bf16 2^-8,
f16 2^-11), o the exact value and spread = sum w |v - o| / sum w:
  u |o|                 the output's own rounding
  u spread              every weight is rounded once, and normalised by the sum
                        of the rounded ones (u^2 spread where it is the sum of
                        two numbers, the second the first one's rounding)
  2 ds spread           scores off by ds at most change weights by a factor
                        within 1 +- 2 ds (ds < 1/4); a score is a sum of d
                        products in fp32 and one product with the scale:
                        ds = (d + 4) 2^-23 scale sum |q k|, and 2^-21 for the
                        exponent's function
  (n + 8) 2^-23 max|v|  sums over n positions in fp32
  n 2^-30 max|v|        f16 weights below its normal range (their step is
                        2^-24 where the largest is 2^7 or more)
  2^-25                 f16 outputs below the normal range
doubled nowhere: each is a bound, not an estimate."""
import math

import numpy as np
import pytest
import torch

import kv_model as M
from kv_gpu import DEV, DT, ints, pair, up
from paper_2606_00021_amd import sense

pytestmark = pytest.mark.gpu


def reference(q, kv, scale, see, once=True):
    """Exact values and bounds; q [m, heads, d] tensor, kv [2, L, kv_heads, d]
    float64, see [m, L] bool."""
    m, heads, d = q.shape
    u = torch.finfo(q.dtype).eps / 2
    qd = q.double().cpu()
    kd = torch.tensor(kv)
    group = heads // kd.shape[2]
    n = kd.shape[1]
    see = torch.as_tensor(see)
    out = torch.zeros((m, heads, d), dtype=torch.float64)
    tol = torch.full((m, heads, d), 2.0 ** -25, dtype=torch.float64)
    for h in range(kd.shape[2]):
        k, v = kd[0, :, h], kd[1, :, h]
        for g in range(h * group, (h + 1) * group):
            s = qd[:, g] @ k.t() * scale
            size = (qd[:, g].abs() @ k.abs().t() * scale)
            s = torch.where(see, s, torch.tensor(-math.inf, dtype=torch.float64))
            top = s.amax(1, keepdim=True) if n else torch.zeros((m, 1))
            w = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
            w = torch.where(see, w, 0.0)
            total = w.sum(1, keepdim=True)
            w = w / torch.where(total > 0, total, 1.0)
            o = w @ v
            spread = (w[:, :, None] * (v[None] - o[:, None]).abs()).sum(1)
            ds = ((d + 4) * 2.0 ** -23 * torch.where(see, size, 0.0).amax(1, keepdim=True)
                  + 2.0 ** -21) if n else torch.zeros((m, 1))
            assert (ds < 0.25).all()
            big = v.abs().amax() if n else 0.0
            out[:, g] = o
            tol[:, g] += (u * o.abs() + ((u if once else u * u) + 2 * ds) * spread
                          + ((n + 8) * 2.0 ** -23 + n * 2.0 ** -30) * big)
    return out, tol


def sees(m, n, mask=None):
    """[m, n] visibility of m rows that are the last of n positions."""
    p, j = np.arange(n)[None], np.arange(m)[:, None]
    base = n - m
    if mask is None:
        return p <= base + j
    out = np.broadcast_to(p < base, (m, n)).copy()
    for u in range(m):
        if base + u >= 0:
            out[:, base + u] = mask[:m, u] != 0
    return out


def queries(rng, shape, dtype, gain=1.0):
    return torch.tensor(rng.standard_normal(shape) * gain).to(DT[dtype]).to(DEV)


def compare(out, q, m, layer, seqs, counts, scale=None, masks=None, where=None):
    """Rows of each entry against the reference; `where` gives their tensors."""
    d = q.shape[-1]
    for i, (s, c) in enumerate(zip(seqs, counts)):
        n = int(m.lens[s])
        qi = q[i, :c] if where is None else where(q, i)
        oi = out[i, :c] if where is None else where(out, i)
        ref, tol = reference(qi, m.rows(layer, s, 0, n), scale or d ** -0.5,
                             sees(c, n, None if masks is None else masks[i]))
        got = oi.double().cpu()
        bad = (got - ref).abs() > tol
        assert not bad.any(), (i, s, n, c, float(((got - ref).abs() / tol).max()))
        assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,page,heads,kv", [(64, 16, 2, 2), (64, 64, 14, 2), (128, 16, 8, 1),
                                             (128, 32, 7, 1), (128, 128, 16, 2), (256, 16, 2, 2),
                                             (256, 64, 20, 1), (64, 32, 32, 1), (128, 16, 40, 1)])
def test_single_tokens(dtype, d, page, heads, kv):
    print(f"[kv attention] token {dtype} d={d} page={page} heads={heads}/{kv}", flush=True)
    rng = np.random.default_rng(d + page + heads)
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 127, 128, 129, 255, 256, 257, 300]
    kvc, m = pair(rng, lens, layers=2, page=page, heads=kv, d=d)
    q = queries(rng, (len(lens), 1, heads, d), dtype)
    out = sense.sense_kv_attention(kvc, 1, q)
    compare(out, q, m, 1, range(len(lens)), [1] * len(lens))
    # the bound on the lengths changes nothing but the launches
    for bound in (300, 256, 1):
        short = sense.sense_kv_attention(kvc, 1, q, max_kv=bound)
        compare(short, q, m, 1, range(len(lens)), [1] * len(lens))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,heads,kv", [(64, 6, 2), (128, 8, 2), (256, 4, 1), (128, 3, 3)])
def test_prompt_chunks(dtype, d, heads, kv):
    print(f"[kv attention] chunk {dtype} d={d} heads={heads}/{kv}", flush=True)
    rng = np.random.default_rng(d + heads)
    lens, counts = [70, 70, 200, 333, 5, 1, 64], [70, 1, 33, 100, 0, 1, 17]
    kvc, m = pair(rng, lens, page=32, heads=kv, d=d)
    q = queries(rng, (len(lens), 100, heads, d), dtype)
    out = torch.full_like(q, 7)
    sense.sense_kv_attention(kvc, 0, q, row_len=ints(counts), out=out)
    compare(out, q, m, 0, range(len(lens)), counts)
    for i, c in enumerate(counts):
        assert (out[i, c:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,heads,kv,nodes", [(64, 4, 2, 5), (128, 8, 2, 61), (256, 2, 1, 40),
                                              (128, 4, 1, 130)])
def test_trees(dtype, d, heads, kv, nodes):
    """Random masks; a row that sees nothing at all, one that sees one node."""
    print(f"[kv attention] tree {dtype} d={d} nodes={nodes}", flush=True)
    rng = np.random.default_rng(nodes)
    counts = [nodes, nodes // 2, nodes, 1]
    lens = [nodes, nodes // 2 + 3, nodes + 290, 1]
    kvc, m = pair(rng, lens, page=16, heads=kv, d=d)
    masks = (rng.random((4, nodes, nodes + 3)) < 0.3).astype(np.uint8) * 200
    masks[0, 1] = 0                                            # and no prefix: nothing seen
    masks[0, 2] = 0
    masks[0, 2, 0] = 1
    masks[3] = 0
    q = queries(rng, (4, nodes, heads, d), dtype)
    gmask = torch.tensor(masks, device=DEV)[:, :, :nodes + 1]
    out = sense.sense_kv_attention(kvc, 0, q, mask=gmask, row_len=ints(counts))
    compare(out, q, m, 0, range(4), counts, masks=masks)
    assert (out[0, 1] == 0).all() and (out[3, 0] == 0).all()
    as_bool = sense.sense_kv_attention(kvc, 0, q, mask=gmask.ne(0), row_len=ints(counts))
    for i, c in enumerate(counts):
        assert torch.equal(out[i, :c], as_bool[i, :c])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,heads,kv,q_len", [(128, 8, 1, 1), (64, 4, 2, 1), (256, 4, 2, 3),
                                              (128, 6, 2, 9), (128, 4, 1, 30)])
def test_long_sequences_are_cut_and_joined(dtype, d, heads, kv, q_len):
    print(f"[kv attention] long {dtype} d={d} q={q_len}", flush=True)
    rng = np.random.default_rng(q_len + d)
    lens = [5003, 40, 2000]
    kvc, m = pair(rng, lens, page=64, heads=kv, d=d)
    q = queries(rng, (3, q_len, heads, d), dtype)
    out = sense.sense_kv_attention(kvc, 0, q)
    compare(out, q, m, 0, range(3), [q_len] * 3)
    again = sense.sense_kv_attention(kvc, 0, q)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scores_that_climb_and_fall(dtype):
    """Scores over a range of thousands, rising, falling and alternating along
    the sequence, so that the reference moves often, late or never."""
    print(f"[kv attention] steep {dtype}", flush=True)
    rng = np.random.default_rng(11)
    d, n = 64, 700
    kvc, m = pair(rng, [n] * 4, page=16, heads=1, d=d)
    ramp = np.linspace(0, 6, n)
    shapes = [ramp, ramp[::-1], 3 + 3 * np.sin(np.arange(n)), np.where(np.arange(n) == 350, 6, 0)]
    for s, level in enumerate(shapes):
        for p in range(n):
            pg, slot = m.cell(s, p)
            c, sc = M.quantise_row(np.full(d, level[p]))
            m.codes[0, pg, 0, 0, slot], m.scales[0, pg, 0, 0, :, slot] = c, sc
    kvc = up(m)
    q = torch.full((4, 1, 3, d), 4.0, dtype=DT[dtype], device=DEV)
    q[:, :, 1] = -4.0
    q[:, :, 2] = 0.0
    out = sense.sense_kv_attention(kvc, 0, q, softmax_scale=1.0)
    compare(out, q, m, 0, range(4), [1] * 4, scale=1.0)


def test_listed_sequences_ragged_rows_and_strides():
    """Sequences out of order and named twice, no such sequence, rows cut out
    of a wider tensor, rows beyond its end, an output in place."""
    print("[kv attention] ragged", flush=True)
    rng = np.random.default_rng(3)
    d, heads, kv = 128, 6, 2
    kvc, m = pair(rng, [90, 33, 260, 7], page=32, heads=kv, d=d)
    fused = queries(rng, (60, heads + 2 * kv, d), "bf16")
    before = fused.clone()
    seqs, start, count = [2, 0, 9, 2, 3, 1, -1], [0, 10, 20, 25, 40, 57, 2], [7, 8, 3, 1, 99, 6, 1]
    q = fused[:, :heads]
    args = dict(seqs=ints(seqs), row_start=ints(start), row_len=ints(count), max_rows=8)
    out = sense.sense_kv_attention(kvc, 0, q, **args, out=torch.full_like(fused, 5)[:, :heads])
    used = np.zeros(60, bool)
    for s, a, c in ((2, 0, 7), (0, 10, 8), (2, 25, 1), (3, 40, 8), (1, 57, 6)):
        n = int(m.lens[s])
        rows = min(c, 60 - a)
        ref, tol = reference(q[a:a + rows], m.rows(0, s, 0, n), d ** -0.5, sees(c, n)[:rows])
        assert ((out[a:a + rows].double().cpu() - ref).abs() <= tol).all(), (s, a)
        used[a:a + rows] = True
    assert (out[torch.tensor(~used, device=DEV)] == 5).all()
    got = sense.sense_kv_attention(kvc, 0, q, **args, out=q)
    keep = torch.tensor(used, device=DEV)
    assert torch.equal(got[keep], out[keep]) and torch.equal(fused[~keep], before[~keep])
    assert torch.equal(fused[:, heads:], before[:, heads:])


def test_many_entries():
    """More entries than a wave has lanes, most of them short, some empty."""
    print("[kv attention] many", flush=True)
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 50, 333).tolist()
    lens[100], lens[332] = 900, 450
    kvc, m = pair(rng, lens, page=16, heads=2, d=64)
    q = queries(rng, (333, 1, 4, 64), "bf16")
    out = sense.sense_kv_attention(kvc, 0, q)
    for i in (0, 1, 63, 64, 100, 101, 332, *rng.integers(0, 333, 40).tolist()):
        compare(out[i:i + 1], q[i:i + 1], m, 0, [i], [1])
    for i, n in enumerate(lens):
        if n == 0:
            assert (out[i] == 0).all()
    # whole units (a bound that cuts none), and sequences in another order
    assert torch.equal(sense.sense_kv_attention(kvc, 0, q, max_kv=900)[5], out[5])
    order = rng.permutation(333)
    perm = torch.tensor(order, device=DEV)
    whole = sense.sense_kv_attention(kvc, 0, q[perm], seqs=ints(order), max_kv=900)
    for i in (0, 64, 332, int(np.nonzero(order == 100)[0][0])):
        compare(whole[i:i + 1], q[order[i]:order[i] + 1], m, 0, [int(order[i])], [1])


def test_many_chunks():
    """More than 64 entries of many rows each, some without any."""
    print("[kv attention] many chunks", flush=True)
    rng = np.random.default_rng(14)
    counts = rng.integers(0, 50, 70).tolist()
    counts[3], counts[69] = 0, 50
    lens = [c + int(e) for c, e in zip(counts, rng.integers(0, 200, 70))]
    lens[20] += 1500
    kvc, m = pair(rng, lens, page=32, heads=2, d=64)
    q = queries(rng, (70, 50, 6, 64), "f16")
    out = torch.full_like(q, 3)
    sense.sense_kv_attention(kvc, 0, q, row_len=ints(counts), out=out)
    for i in (0, 3, 20, 63, 64, 65, 69):
        compare(out[i:i + 1], q[i:i + 1], m, 0, [i], [counts[i]])
        assert (out[i, counts[i]:] == 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_what_a_row_does_not_see_does_not_touch_it(dtype, d):
    """NaN blocks in slots behind the end, in unseen tree nodes, in pages that
    are none; and in positions that some rows see, which become NaN there."""
    print(f"[kv attention] unseen NaN {dtype} d={d}", flush=True)
    rng = np.random.default_rng(d)
    nodes, lens = 40, [40, 301, 77]
    kvc, m = pair(rng, lens, page=64, heads=2, d=d)
    masks = np.tril((rng.random((3, nodes, nodes)) < 0.5)).astype(np.uint8)
    masks[:, np.arange(nodes), np.arange(nodes)] = 1
    clean = sense.sense_kv_attention(kvc, 0, q := queries(rng, (3, nodes, 4, d), dtype),
                                     mask=torch.tensor(masks, device=DEV))
    compare(clean, q, m, 0, range(3), [nodes] * 3, masks=masks)
    dirty = {k: v.clone() for k, v in kvc.items()}
    # slots behind every sequence's end, and every page that no sequence holds
    used = set()
    for s, n in enumerate(lens):
        used |= set(m.table[s][m.table[s] >= 0].tolist())
        if n % 64:
            dirty["scales"][:, int(m.table[s, n // 64]), :, :, :, n % 64:] = 255
    for p in set(range(m.refs.size)) - used:
        dirty["scales"][:, p] = 255
    assert torch.equal(sense.sense_kv_attention(dirty, 0, q, mask=torch.tensor(masks, device=DEV)),
                       clean)
    # node 3's value (head 0, its last block) and node 5's key (head 1)
    for s, n in enumerate(lens):
        (p3, s3), (p5, s5) = m.cell(s, n - nodes + 3), m.cell(s, n - nodes + 5)
        dirty["scales"][0, int(p3), 1, 0, -1, int(s3)] = 255
        dirty["scales"][0, int(p5), 0, 1, 0, int(s5)] = 255
    got = sense.sense_kv_attention(dirty, 0, q, mask=torch.tensor(masks, device=DEV))
    for i in range(3):
        want = torch.zeros((nodes, 4, d), dtype=torch.bool)
        want[masks[i][:, 3] != 0, 0:2, d - 32:] = True
        want[masks[i][:, 5] != 0, 2:4] = True
        assert torch.equal(torch.isnan(got[i]).cpu(), want)
        assert torch.equal(got[i].cpu()[~want], clean[i].cpu()[~want])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,nodes", [(64, 3), (128, 40), (256, 9)])
def test_unseen_positions_may_hold_anything(dtype, d, nodes):
    """Any byte as a code or scale behind the end and in free pages, and tree
    nodes of the largest scales that most rows do not see."""
    print(f"[kv attention] unseen bytes {dtype} d={d} nodes={nodes}", flush=True)
    rng = np.random.default_rng(d + nodes)
    lens = [nodes, 301, 77 + nodes]
    kvc, m = pair(rng, lens, page=32, heads=1, d=d)
    masks = np.repeat(np.eye(nodes, dtype=np.uint8)[None], 3, 0)
    masks[:, -1, 0] = 1
    gmask = torch.tensor(masks, device=DEV)
    q = queries(rng, (3, nodes, 4, d), dtype)
    clean = sense.sense_kv_attention(kvc, 0, q, mask=gmask)
    dirty = {k: v.clone() for k, v in kvc.items()}
    free = torch.ones(m.refs.size, dtype=torch.bool, device=DEV)
    for s, n in enumerate(lens):
        free[torch.tensor(m.table[s][m.table[s] >= 0], device=DEV).long()] = False
        if n % 32:
            tail = dirty["scales"][:, int(m.table[s, n // 32]), :, :, :, n % 32:]
            tail.copy_(torch.randint(0, 256, tail.shape, device=DEV))
        pg, slot = m.cell(s, n - nodes + 1)
        dirty["scales"][0, int(pg), :, :, :, int(slot)] = 254
        dirty["codes"][0, int(pg), :, :, int(slot)] = 0xF7
    dirty["scales"][:, free] = 254
    dirty["codes"][:, free] = 0x77
    got = sense.sense_kv_attention(dirty, 0, q, mask=gmask)
    rows = [u for u in range(nodes) if u != 1]                 # node 1 sees itself
    assert torch.equal(got[:, rows], clean[:, rows])


def test_seen_nan_in_the_prefix_reaches_every_row():
    print("[kv attention] seen NaN", flush=True)
    rng = np.random.default_rng(6)
    kvc, m = pair(rng, [300, 300], page=16, heads=1, d=64)
    q = queries(rng, (2, 1, 2, 64), "bf16")
    clean = sense.sense_kv_attention(kvc, 0, q)
    pg, slot = m.cell(0, 77)
    kvc["scales"][0, int(pg), 1, 0, 1, int(slot)] = 255
    got = sense.sense_kv_attention(kvc, 0, q)
    assert torch.isnan(got[0, :, :, 32:]).all()
    assert torch.equal(got[0, :, :, :32], clean[0, :, :, :32]) and torch.equal(got[1], clean[1])


def test_pages_that_are_none_and_lengths_that_cannot_be():
    print("[kv attention] broken tables", flush=True)
    rng = np.random.default_rng(7)
    kvc, m = pair(rng, [64, 64, 64, 64], page=16, heads=1, d=64)
    q = queries(rng, (4, 2, 2, 64), "f16")
    kvc["page_table"][0, 1] = -1
    kvc["page_table"][1, 2] = 1 << 30
    kvc["seq_len"][2] = -3
    kvc["seq_len"][3] = 1 << 30                                # the capacity, mostly without pages
    out = sense.sense_kv_attention(kvc, 0, q)
    for s, lo, hi in ((0, 16, 32), (1, 32, 48)):
        see = sees(2, 64)
        see[:, lo:hi] = False
        ref, tol = reference(q[s], m.rows(0, s, 0, 64), 64 ** -0.5, see)
        assert ((out[s].double().cpu() - ref).abs() <= tol).all()
    assert (out[2] == 0).all()
    ref, tol = reference(q[3], m.rows(0, 3, 0, 64), 64 ** -0.5, np.ones((2, 64), bool))
    assert ((out[3].double().cpu() - ref).abs() <= tol).all()
    # no page at all, and more rows than positions
    kvc["page_table"][:] = -1
    assert (sense.sense_kv_attention(kvc, 0, q) == 0).all()
    kvc, m = pair(rng, [3], page=16, heads=1, d=64)
    q = queries(rng, (1, 6, 1, 64), "bf16")
    out = sense.sense_kv_attention(kvc, 0, q)
    assert (out[0, :3] == 0).all()
    ref, tol = reference(q[0], m.rows(0, 0, 0, 3), 64 ** -0.5, sees(6, 3))
    assert ((out[0].double().cpu() - ref).abs() <= tol).all()


def test_offsets_beyond_32_bits():
    print("[kv attention] large", flush=True)
    rng = np.random.default_rng(8)
    layers, pages, page, heads, d = 9, 4096, 128, 8, 128
    kvc = {"codes": torch.full((layers, pages, 2, heads, page, d // 2), 0x77, dtype=torch.uint8,
                               device=DEV),
           "scales": torch.full((layers, pages, 2, heads, d // 32, page), 130, dtype=torch.uint8,
                                device=DEV),
           "page_table": ints([[pages - 1, pages - 2, 0]]), "seq_len": ints([200]),
           "page_refs": torch.zeros(pages, dtype=torch.int32, device=DEV)}
    m = M.Cache(1, 3, page, heads, d, 1, 3)
    m.table[0], m.lens[0] = [2, 1, 0], 200
    m.codes[:] = rng.integers(0, 256, m.codes.shape)
    m.scales[:] = rng.integers(122, 128, m.scales.shape)
    kvc["codes"][-1, -2:] = torch.from_numpy(m.codes[0, 1:]).to(DEV)
    kvc["scales"][-1, -2:] = torch.from_numpy(m.scales[0, 1:]).to(DEV)
    assert kvc["codes"].numel() > 1 << 32
    q = queries(rng, (1, 2, 16, d), "bf16")
    out = sense.sense_kv_attention(kvc, layers - 1, q)
    compare(out, q, m, 0, [0], [2])


def test_other_streams_and_replays():
    """A named stream; a captured call that follows the cache as it grows, two
    of them on one workspace, eager work in between."""
    print("[kv attention] streams", flush=True)
    rng = np.random.default_rng(9)
    kvc, m = pair(rng, [700, 90], page=16, heads=2, d=64, spare=30)
    q = queries(rng, (2, 1, 8, 64), "bf16")
    first = sense.sense_kv_attention(kvc, 0, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        got = sense.sense_kv_attention(kvc, 0, q, stream=stream)
        side.synchronize()
        assert torch.equal(got, first)
    size = sense.sense_kv_attention_workspace_size(kvc, 2, 1, 8)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(q) for _ in range(2)]
    other = queries(rng, q.shape, "bf16")
    graphs = []
    torch.cuda.synchronize()
    for qi, o in ((q, outs[0]), (other, outs[1])):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sense.sense_kv_attention(kvc, 0, qi, workspace=ws, out=o)
        graphs.append(g)
    for turn in range(4):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for qi, o in ((q, outs[0]), (other, outs[1])):
            assert torch.equal(o, sense.sense_kv_attention(kvc, 0, qi))
        compare(outs[1], other, m, 0, [0, 1], [1, 1])
        grown = ints([40 * (turn + 1), 3])
        sense.sense_kv_reserve(kvc, grown)
        m.reserve([0, 1], grown.tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("rows,heads", [(1, 2), (9, 3), (40, 4)])
def test_scores_beyond_what_their_differences_resolve(dtype, d, rows, heads):
    """Scores that are exact in fp32 and differ by far more than weights reach
    (or not at all), up to 2^144: a row is the mean of its best positions'
    values.  Bound: weights are 0 or equal, so the output's rounding and the
    sums' alone."""
    print(f"[kv attention] huge scores {dtype} d={d} rows={rows}", flush=True)
    rng = np.random.default_rng(d + rows)
    lens = [2500, 700, 300]
    kvc, m = pair(rng, lens, page=32, heads=1, d=d)
    # A key is its code's value in dim 5 and 0 elsewhere; scales as they are.
    m.codes[:, :, 0] = 0
    m.codes[:, :, 0, :, :, 2] = rng.integers(0, 16, m.codes[:, :, 0, :, :, 2].shape) << 4
    kvc = up(m)
    gains = torch.tensor([2.0 ** 14, -(2.0 ** 13), 3.0, 0.0])[:heads]
    q = torch.zeros((3, rows, heads, d), dtype=DT[dtype], device=DEV)
    q[..., 5] = gains.to(DEV)
    u = torch.finfo(q.dtype).eps / 2
    held = [m.rows(0, i, 0, n)[:, :, 0] for i, n in enumerate(lens)]
    for scale in (2.0 ** 12, 3.0 * 2.0 ** 15, 2.0 ** 127):
        out = sense.sense_kv_attention(kvc, 0, q, softmax_scale=scale).double().cpu()
        for i, n in enumerate(lens):
            k, v = held[i]
            for h in range(heads):
                s = k[:, 5] * float(gains[h])
                for j in range(rows):
                    end = n - rows + j + 1
                    best = s[:end] == s[:end].max()
                    ref = torch.tensor(v[:end][best].mean(0))
                    tol = u * ref.abs() + 2.0 ** -25 + (n + 8) * 2.0 ** -23 * np.abs(v).max()
                    off = (out[i, j, h] - ref).abs()
                    assert (off <= tol).all(), (scale, i, h, j, float((off / tol).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,rows,heads,kv", [(64, 1, 6, 2), (128, 4, 8, 2), (128, 3, 16, 2),
                                             (256, 2, 4, 1), (64, 9, 14, 2), (128, 16, 4, 1),
                                             (256, 7, 8, 2)])
def test_units_of_few_rows_round_only_the_result(dtype, d, rows, heads, kv):
    """Up to 64 rows of a key head: weights are sums of two numbers."""
    print(f"[kv attention] two numbers {dtype} d={d} rows={rows}", flush=True)
    rng = np.random.default_rng(d + rows + heads)
    lens = [1400, 300, 77]
    kvc, m = pair(rng, lens, page=32, heads=kv, d=d)
    q = queries(rng, (3, rows, heads, d), dtype)
    out = sense.sense_kv_attention(kvc, 0, q).double().cpu()
    for i, n in enumerate(lens):
        ref, tol = reference(q[i], m.rows(0, i, 0, n), d ** -0.5, sees(rows, n), once=False)
        assert ((out[i] - ref).abs() <= tol).all(), (i, float(((out[i] - ref).abs() / tol).max()))
