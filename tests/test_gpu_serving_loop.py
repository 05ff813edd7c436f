"""The paged cache's calls as a server makes them: prompts, draft trees built, attended to, verified and kept, single tokens; on
streams, in graphs, several at once.  Attention over pages is compared with the library's dense calls and with the plain form."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from serving import HALF, Paged, attend_plain, compare, page_table, random_mask, rounds_weights, visible_rows

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    m.init()
    return m


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype is BF16 else torch.int32)


@pytest.mark.parametrize("dtype,Hq,Hkv,d", [(BF16, 8, 2, 128), (F32, 4, 4, 64)])
def test_prompts_then_trees_then_tokens(dy, dtype, Hq, Hkv, d):
    """Three speculative steps of two sequences over one cache of two layers.  A record of every token's rotated key and value is
    kept beside; each attention is checked against the plain form over that record."""
    dev, L, page, V = "cuda", 2, 16, 600
    g = torch.Generator(device=dev).manual_seed(5)
    randn = lambda *sh: torch.randn(sh, generator=g, device=dev)
    prompts, room = [37, 150], 400
    table, pool = page_table([room, room], page, 9)
    k_pages, v_pages = (torch.full((L, pool, page, Hkv, d), math.nan, dtype=dtype, device=dev) for _ in range(2))
    cache = dy.PagedCache(k_pages, v_pages, torch.from_numpy(table).to(dev))
    layers = [cache.layer(l) for l in range(L)]
    freq = torch.from_numpy((10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)).to(dev)
    scale, wh, oh = 1.0 / math.sqrt(d), rounds_weights(dtype, d), HALF[dtype]
    record = [[[torch.zeros((0, Hkv, d), dtype=dtype)] * 2 for _ in range(2)] for _ in range(L)]        # [layer][sequence] -> k, v
    context = [0, 0]

    def attend(l, batch, mask, rel):
        """Appends random rows, attends, checks; returns the keys and values as the cache has them."""
        total = batch.total_nodes
        q, k, v = randn(total, Hq + 2 * Hkv, d).to(dtype).split([Hq, Hkv, Hkv], dim=1)
        turned = torch.empty((total, Hkv, d), dtype=dtype, device=dev)
        q = dy.kv_append(k, v, batch, layers[l], q=q, rel_pos=rel, inv_freq=freq, k_out=turned)
        out = dy.paged_attn(q, batch, layers[l], scale, anc_mask=mask)
        got, words = out.double().cpu().numpy(), None if mask is None else mask.cpu().numpy().view(np.uint64)
        for s in range(2):
            a, b = int(batch.node_offset[s]), int(batch.node_offset[s + 1])
            keys, values = (torch.cat([r, t[a:b].cpu()]).double().numpy() for r, t in zip(record[l][s], (turned, v)))
            want, bound = attend_plain(q[a:b].double().cpu().numpy(), keys, values, visible_rows(b - a, context[s], None if words is None else words[a:b]), scale, wh, oh)
            compare(got[a:b], want, bound, f"layer {l}, sequence {s}")
        return q, out, turned, v

    def extend(l, s, k, v):
        record[l][s] = [torch.cat([r, x.cpu()]) for r, x in zip(record[l][s], (k, v))]

    batch = dy.Batch.from_sizes(prompts, context)
    for l in range(L):
        q, out, k, v = attend(l, batch, None, None)
        whole = dy.prompt_attn(q, k, v, batch, scale)                     # the same prompts, never in pages
        assert float((whole.float() - out.float()).abs().max()) <= (4 * 2 ** -8 if dtype is BF16 else 1e-5) * float(v.float().abs().max())
        for s in range(2):
            a, b = int(batch.node_offset[s]), int(batch.node_offset[s + 1])
            extend(l, s, k[a:b], v[a:b])
    context = list(prompts)
    for step in range(3):
        sizes = [48, 30]
        batch = dy.Batch.from_sizes(sizes, context)
        draft = randn(sum(sizes), V) * 2
        built = dy.build_tree(draft, batch, 0.8, 100 + step)
        rows = []
        for l in range(L):
            q, out, k, v = attend(l, batch, built.anc_mask, built.tree.depth)
            rows.append((k, v))
            dense = [torch.cat([record[l][s][i] for s in range(2)]).to(dev) for i in range(2)]
            other = dy.tree_attn(q, dense[0], dense[1], k, v.contiguous(), built.anc_mask, batch, scale)
            assert float((other.float() - out.float()).abs().max()) <= (4 * 2 ** -8 if dtype is BF16 else 1e-5) * 5.0
        res = dy.verify(draft, draft + 0.3 * randn(sum(sizes), V), batch, built.tree, 0.8, 0.8, 200 + step)
        dy.kv_keep(cache, batch, res.accepted_nodes, res.n_accepted)
        n_acc, nodes = res.n_accepted.tolist(), res.accepted_nodes.cpu().numpy()
        for s in range(2):
            a = int(batch.node_offset[s])
            path = [a] + [a + int(x) for x in nodes[a:a + n_acc[s]]]
            for l in range(L):
                extend(l, s, rows[l][0][path], rows[l][1][path])
            context[s] += 1 + n_acc[s]
        assert sum(n_acc) > 0 or step < 2 or context != prompts
        one = dy.Batch.from_sizes([1, 1], context)                        # and a plain token each
        for l in range(L):
            _, _, k, v = attend(l, one, None, None)
            for s in range(2):
                extend(l, s, k[s:s + 1], v[s:s + 1])
        context = [c + 1 for c in context]


def cases(seed):
    return [Paged((1, 1, 1), (3000, 40, 700), 16, 2, 128, BF16, 16, seed), Paged((1,), (1500,), 8, 8, 64, F32, 16, seed + 1),
            Paged((64,), (900,), 16, 2, 128, BF16, 16, seed + 2, mask=random_mask((64,), seed)[0]),
            Paged((400, 1), (100, 2000), 8, 2, 128, BF16, 32, seed + 3)]


def test_replays_of_a_recorded_step_equal_the_eager_step(dy):
    s = torch.cuda.Stream()
    cs = cases(50)
    eager = [dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev) for c in cs]
    g = torch.Generator(device="cuda").manual_seed(1)
    p = torch.randn((300, 12, 128), generator=g, device="cuda").to(BF16)
    lengths = dy.Batch.from_sizes([200, 100])
    eager_prompt = dy.prompt_attn(p[:, :8], p[:, 8:10], p[:, 10:], lengths, 0.1)
    c0 = cs[3]
    k, v = (torch.randn((401, 2, 128), generator=g, device="cuda").to(BF16) for _ in range(2))
    torch.cuda.synchronize()
    outs = [torch.empty_like(c.q_dev) for c in cs]
    prompt_out = torch.empty_like(eager_prompt)
    spare = dy.PagedCache(c0.cache.k.clone(), c0.cache.v.clone(), c0.cache.page_table)
    want = dy.PagedCache(spare.k.clone(), spare.v.clone(), spare.page_table)
    accepted = torch.arange(401, dtype=torch.int32, device="cuda") * 2 + 5
    count = torch.tensor([6, 0], dtype=torch.int32, device="cuda")
    dy.kv_append(k, v, c0.batch, want), dy.kv_keep(want, c0.batch, accepted, count)
    with torch.cuda.stream(s):
        calls = [dy.paged_attn_call(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, out=o, stream=s) for c, o in zip(cs, outs)]
        calls.append(dy.prompt_attn_call(p[:, :8], p[:, 8:10], p[:, 10:], lengths, 0.1, out=prompt_out, stream=s))
        calls.append(dy.kv_append_call(k, v, c0.batch, spare, stream=s))
        for call in calls:
            call()
        dy.kv_keep(spare, c0.batch, accepted, count)
        s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        for call in calls:
            call()
        dy.kv_keep(spare, c0.batch, accepted, count)
        inside = dy.paged_attn(cs[0].q_dev, cs[0].batch, cs[0].cache, cs[0].scale)        # a plain call, recorded
    for rep in range(4):
        for t in outs + [prompt_out, spare.k, spare.v, inside]:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for o, e in zip(outs + [prompt_out, inside], eager + [eager_prompt, eager[0]]):
            assert torch.equal(bits(o), bits(e)), f"replay {rep}"
        at = [c0.place(0, 100 + j) for j in (0, 1, 5, 60)]
        for pg, r in at:
            assert torch.equal(bits(spare.k[pg, r]), bits(want.k[pg, r])) and torch.equal(bits(spare.v[pg, r]), bits(want.v[pg, r]))
        other = dy.paged_attn(cs[2].q_dev, cs[2].batch, cs[2].cache, cs[2].scale)
        assert torch.isfinite(other.float().sum()).item()


def test_graphs_and_streams_beside_each_other(dy):
    """Two graphs recorded on one stream and replayed on two, eager calls of other streams among them: nobody's workspace is
    another's."""
    cs = cases(70)
    eager = [dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev) for c in cs]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graphs, outs = [], []
    for c in cs[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs.append(dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(20):
        for graph, t in zip(graphs, streams):
            with torch.cuda.stream(t):
                graph.replay()
        with torch.cuda.stream(streams[2]):
            third = dy.paged_attn(cs[2].q_dev, cs[2].batch, cs[2].cache, cs[2].scale, anc_mask=cs[2].mask_dev)
        fourth = dy.paged_attn(cs[0].q_dev, cs[0].batch, cs[0].cache, cs[0].scale, stream=streams[2])
        torch.cuda.synchronize()
        assert torch.equal(bits(outs[0]), bits(eager[0])) and torch.equal(bits(outs[1]), bits(eager[1]))
        assert torch.equal(bits(third), bits(eager[2])) and torch.equal(bits(fourth), bits(eager[0]))


def test_a_call_gives_the_same_bits_every_time(dy):
    cs = cases(90)
    for c in cs:
        first = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev)
        for _ in range(10):
            assert torch.equal(bits(dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev)), bits(first))


def test_rows_behind_the_last_token_are_left(dy):
    """`out` longer memory: nothing is written before or behind it."""
    c = Paged((3, 70), (100, 9), 8, 2, 128, BF16, 16, 4)
    room = torch.full((73 + 16, 8, 128), 3.0, dtype=BF16, device="cuda")
    dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, out=room[8:81])
    assert bool((room[:8] == 3).all()) and bool((room[81:] == 3).all())
    c.check(room[8:81])
