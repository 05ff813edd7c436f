"""Speculative steps over pages in which verification accepts and kv_keep moves, by construction: along the way from the root to a tree's
last row the target's logits leave no token but the next row's, so that this row is accepted for certain (the target's probability is
above the draft's) and its elder siblings are not (theirs is zero); the last row never lies where it has to go.  What the pages
hold afterwards is held against the appended rows, and a plain token's attention against the plain form (tests/serving.py)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from serving import HALF, attend_plain, compare, page_table, rounds_weights, visible_rows

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    return m


@pytest.mark.parametrize("dtype,Hq,Hkv,d", [(BF16, 8, 2, 128), (F32, 4, 4, 64)])
def test_accepted_rows_move_and_are_attended_to(dy, dtype, Hq, Hkv, d):
    dev, page, V = "cuda", 16, 600
    g = torch.Generator(device=dev).manual_seed(11)
    randn = lambda *sh: torch.randn(sh, generator=g, device=dev)
    table, pool = page_table([400, 400], page, 9)
    cache = dy.PagedCache(*(torch.full((pool, page, Hkv, d), math.nan, dtype=dtype, device=dev) for _ in range(2)), torch.from_numpy(table).to(dev))
    scale, context = 1.0 / math.sqrt(d), [0, 0]
    record = [[torch.zeros((0, Hkv, d), dtype=dtype)] * 2 for _ in range(2)]                     # [sequence] -> k, v

    def append(sizes, rel):
        batch = dy.Batch.from_sizes(sizes, context)
        k, v = randn(sum(sizes), Hkv, d).to(dtype), randn(sum(sizes), Hkv, d).to(dtype)
        dy.kv_append(k, v, batch, cache, rel_pos=rel)
        return batch, k.cpu(), v.cpu()

    def keep_on_record(s, k, v):
        record[s] = [torch.cat([r, x]) for r, x in zip(record[s], (k, v))]
        context[s] += k.shape[0]

    _, k, v = append([37, 150], None)
    keep_on_record(0, k[:37], v[:37]), keep_on_record(1, k[37:], v[37:])
    moved = 0
    for step in range(4):
        sizes = [48, 30]
        draft = randn(sum(sizes), V) * 2
        built = dy.build_tree(draft, dy.Batch.from_sizes(sizes, context), 0.8, 300 + step)
        batch, k, v = append(sizes, built.tree.depth)
        target, parent, token = draft.clone(), built.tree.parent.tolist(), built.tree.token.tolist()
        ways = []
        for s, n in enumerate(sizes):
            a, way = int(batch.node_offset[s]), [n - 1]
            while way[0] > 0:
                way.insert(0, parent[a + way[0]])
            for up, row in zip(way, way[1:]):
                target[a + up, token[a + row]] += 500.0              # over 0.8: no other token is left in fp32
            ways.append(way[1:])
        res = dy.verify(draft, target, batch, built.tree, 0.8, 0.8, 400 + step)
        dy.kv_keep(cache, batch, res.accepted_nodes, res.n_accepted)
        counts, nodes = res.n_accepted.tolist(), res.accepted_nodes.cpu().numpy()
        for s in range(2):
            a = int(batch.node_offset[s])
            path = [int(x) for x in nodes[a:a + counts[s]]]
            assert path == ways[s]
            moved += sum(x != i + 1 for i, x in enumerate(path))
            rows = [a] + [a + x for x in path]
            keep_on_record(s, k[rows], v[rows])
            at = [(int(table[s, j // page]), j % page) for j in range(context[s])]
            pages, places = torch.tensor([p for p, _ in at]), torch.tensor([r for _, r in at])
            assert torch.equal(cache.k.cpu()[pages, places], record[s][0]) and torch.equal(cache.v.cpu()[pages, places], record[s][1])
        one, k, v = append([1, 1], None)
        q = randn(2, Hq, d).to(dtype)
        out = dy.paged_attn(q, one, cache, scale).double().cpu().numpy()
        for s in range(2):
            keep_on_record(s, k[s:s + 1], v[s:s + 1])
            want, bound = attend_plain(q[s:s + 1].double().cpu().numpy(), *(x.double().numpy() for x in record[s]), visible_rows(1, context[s] - 1), scale,
                                       rounds_weights(dtype, d), HALF[dtype])
            compare(out[s:s + 1], want, bound, f"step {step}, sequence {s}")
    assert moved >= 8                                            # the last row of each tree at least
