"""One speculative step of several streams, the calls together: retrieval,
loose trie, room and rows for the tree, attention under the trie's mask,
verification through the trie, the accepted path kept; then the next token."""
import numpy as np
import pytest
import torch

from kv_gpu import DEV, ints, pair, same_rows
from paper_2606_00021_amd import sense, synth
from test_gpu_kv_attention import compare, queries, reference, sees

pytestmark = pytest.mark.gpu


def streams(seed, groups, heads, kv, d, page, layers):
    rng = np.random.default_rng(seed)
    w = synth.scaled(synth.WORKLOADS["store-1m-d4096"], n=4000, d=256, n_clusters=64, vocab=700,
                     k=6, span=4)
    ds = synth.make_datastore(w, seed, torch.device(DEV))
    hidden, _ = synth.make_queries(w, ds, seed, n_queries=groups)
    index = sense.sense_build_index(ds.keys, ds.spans)
    lens = rng.integers(1, 400, groups).tolist()
    kvc, m = pair(rng, lens, layers=layers, page=page, heads=kv, d=d, spare=8 * groups)
    return rng, w, index, hidden, lens, kvc, m


@pytest.mark.parametrize("heads,kv,d,page,dtype", [(8, 2, 128, 16, "bf16"), (14, 2, 64, 32, "f16")])
def test_a_step(heads, kv, d, page, dtype):
    print(f"[kv step] heads={heads}/{kv} d={d} page={page} {dtype}", flush=True)
    groups, layers = 3, 2
    rng, w, index, hidden, lens, kvc, m = streams(heads, groups, heads, kv, d, page, layers)
    _, _, drafts, dlen = sense.sense_retrieve(index, hidden, w.k)
    c = groups * w.k
    trie = sense.sense_build_loose_trie(drafts.view(c, w.span), dlen.view(c), n_groups=groups,
                                        want_mask=True)
    nodes = w.k * w.span
    counts = trie["tree_len"]

    # room for the trees, and their rows in every layer
    assert sense.sense_kv_reserve(kvc, counts).tolist() == [0] * groups
    m.reserve(list(range(groups)), counts.tolist())
    k = queries(rng, (layers, groups, nodes, kv, d), dtype)
    v = queries(rng, (layers, groups, nodes, kv, d), dtype)
    sense.sense_kv_write(kvc, 0, k, v, row_len=counts)
    for layer in range(layers):
        for s in range(groups):
            for u in range(int(counts[s])):
                for h in range(kv):
                    for i, x in ((0, k), (1, v)):
                        m.write(layer, s, lens[s] + u, i, h,
                                x[layer, s, u, h].double().cpu().numpy())
    same_rows(kvc, m)

    # every layer's attention under the trie's mask
    masks = trie["mask"].cpu().numpy()
    for layer in range(layers):
        q = queries(rng, (groups, nodes, heads, d), dtype)
        out = torch.zeros_like(q)
        sense.sense_kv_attention(kvc, layer, q, mask=trie["mask"], row_len=counts, out=out)
        compare(out, q, m, layer, range(groups), counts.tolist(), masks=masks)

    # logits of the tree's rows, sharp towards each node's first child
    logits = torch.randn((groups, 1 + nodes, w.vocab), device=DEV)
    logits[:, 1:, :] += (out.float().flatten(2) @ torch.randn((heads * d, w.vocab), device=DEV)
                         ) * 0.01
    for g in range(groups):
        for u in range(int(counts[g]) - 1, -1, -1):
            logits[g, 1 + int(trie["tree_parent"][g, u]), int(trie["tree_tokens"][g, u])] += 8.0
    res = sense.sense_soft_gate_verify_tree(logits, trie, n_groups=groups)

    # the accepted path stays, in all layers
    gamma, best, accept = trie["gamma"], res["best"], res["accept_len"]
    status = sense.sense_kv_compact(kvc, counts, gamma, accept, best)
    rows = [g * w.k + int(best[g]) for g in range(groups)]
    paths = [gamma[r, :int(accept[r])].tolist() for r in rows]
    assert max(len(p) for p in paths) > 0
    tails = counts.tolist()
    assert status.tolist() == m.compact(list(range(groups)), tails, paths) == [0] * groups
    same_rows(kvc, m)
    assert kvc["seq_len"].tolist() == [n + len(p) for n, p in zip(lens, paths)]

    # a chain written token by token holds the same
    for s, path in enumerate(paths):
        if not path:
            continue
        at = torch.tensor(path, device=DEV)
        gk, gv = (torch.empty((layers, 1, len(path), kv, d), dtype=k.dtype, device=DEV)
                  for _ in range(2))
        sense.sense_kv_read(kvc, 0, gk, gv, seqs=ints([s]))
        fresh = sense.sense_build_kv_cache(layers, 8, page, kv, d, 1, 8)
        for j in range(len(path)):
            sense.sense_kv_reserve(fresh, ints([1]))
            sense.sense_kv_write(fresh, 0, k[:, s:s + 1, at[j:j + 1]].contiguous(),
                                 v[:, s:s + 1, at[j:j + 1]].contiguous())
        fk, fv = torch.empty_like(gk), torch.empty_like(gv)
        sense.sense_kv_read(fresh, 0, fk, fv)
        assert torch.equal(gk, fk) and torch.equal(gv, fv)

    # the next token, over prefix and path
    sense.sense_kv_reserve(kvc, ints([1] * groups))
    m.reserve(list(range(groups)), [1] * groups)
    k1, v1 = queries(rng, (groups, 1, kv, d), dtype), queries(rng, (groups, 1, kv, d), dtype)
    sense.sense_kv_write(kvc, 1, k1, v1)
    for s in range(groups):
        for h in range(kv):
            for i, x in ((0, k1), (1, v1)):
                m.write(1, s, int(m.lens[s]) - 1, i, h, x[s, 0, h].double().cpu().numpy())
    q = queries(rng, (groups, 1, heads, d), dtype)
    compare(sense.sense_kv_attention(kvc, 1, q), q, m, 1, range(groups), [1] * groups)
    index.close()


def test_a_tree_row_is_its_chain():
    """A tree row's result is what the chain of its ancestors gives on its
    own, in a sequence that shares the prefix's pages."""
    print("[kv step] chains", flush=True)
    rng = np.random.default_rng(5)
    kvc, m = pair(rng, [83], page=16, heads=2, d=128, spare=60, extra_seqs=7)
    parent = [-1, 0, 1, 0, -1, 4, 4]
    mask = np.zeros((7, 7), np.uint8)
    for u, p in enumerate(parent):
        if p >= 0:
            mask[u] = mask[p]
        mask[u, u] = 1
    k, v = queries(rng, (1, 7, 2, 128), "bf16"), queries(rng, (1, 7, 2, 128), "bf16")
    q = queries(rng, (1, 7, 4, 128), "bf16")
    # one sequence a node, forked off the prefix, before the tree grows
    dst = ints(range(1, 8))
    assert sense.sense_kv_fork(kvc, ints([0] * 7), dst).tolist() == [0] * 7
    depth = mask.sum(1).tolist()
    assert sense.sense_kv_reserve(kvc, ints([7] + depth)).tolist() == [0] * 8
    sense.sense_kv_write(kvc, 0, k, v, seqs=ints([0]))
    tree = sense.sense_kv_attention(kvc, 0, q, mask=torch.tensor(mask[None], device=DEV),
                                    seqs=ints([0]))
    for u in range(7):
        chain = torch.tensor(np.nonzero(mask[u])[0], device=DEV)
        sense.sense_kv_write(kvc, 0, k[:, chain].contiguous(), v[:, chain].contiguous(),
                             seqs=dst[u:u + 1])
    for u in range(7):
        got = sense.sense_kv_attention(kvc, 0, q[:, u:u + 1].contiguous(), seqs=dst[u:u + 1])
        held = torch.empty((1, 83 + depth[u], 2, 128), device=DEV), \
            torch.empty((1, 83 + depth[u], 2, 128), device=DEV)
        sense.sense_kv_read(kvc, 0, *held, seqs=dst[u:u + 1])
        rows = torch.stack([h[0] for h in held]).double().cpu().numpy()
        n = rows.shape[1]
        ref, tol = reference(q[0, u:u + 1], rows, 128 ** -0.5, sees(1, n))
        for x in (got[0], tree[0, u:u + 1]):
            assert ((x.double().cpu() - ref).abs() <= tol).all(), u


def test_a_captured_step_follows_the_cache():
    """Room, rows, attention and the path kept, captured once: every replay
    works on what the cache holds then, as the same calls do eagerly on a
    second cache."""
    print("[kv step] captured", flush=True)
    rng = np.random.default_rng(6)
    lens = [40, 7, 130]
    kvc, _ = pair(rng, lens, layers=2, page=16, heads=2, d=64, spare=60)
    twin = {name: t.clone() for name, t in kvc.items()}
    nodes = 9
    k, v = (queries(rng, (2, 3, nodes, 2, 64), "bf16") for _ in range(2))
    q = queries(rng, (3, nodes, 4, 64), "bf16")
    mask = torch.tensor(np.tril(rng.random((3, nodes, nodes)) < 0.6), device=DEV)
    counts, keep, kept = ints([9, 5, 9]), ints([[0, 2, 4, 8]] * 3), ints([2, 4, 3])
    size = sense.sense_kv_attention_workspace_size(kvc, 3, nodes, 4)
    ws = torch.empty(max(size, 1 << 20), dtype=torch.uint8, device=DEV)

    def step(cache, out):
        sense.sense_kv_reserve(cache, counts, workspace=ws)
        sense.sense_kv_write(cache, 0, k, v, row_len=counts)
        sense.sense_kv_attention(cache, 1, q, mask=mask, row_len=counts, workspace=ws, out=out)
        sense.sense_kv_compact(cache, counts, keep, kept, workspace=ws)

    out, want = torch.zeros_like(q), torch.zeros_like(q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(kvc, out)
    for turn in range(5):
        g.replay()
        torch.cuda.synchronize()
        step(twin, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), turn
        for name in kvc:
            assert torch.equal(kvc[name], twin[name]), (turn, name)
        k.normal_()
        v.mul_(-1.5)
