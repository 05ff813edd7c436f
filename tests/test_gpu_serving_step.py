"""A server's step from its parts, as they are used together: pages by the lengths, keys into them, attention with capped scores and
windows, filtered tables through the builder and the verification, the kept path, drawn tokens."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle
from helpers import DECISION_MARGIN, compare_trees, f32, oracle_trees
from sampling import plain_row
from scored import scored_plain, visible_rows
from serving import HALF

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


@pytest.mark.parametrize("top_k,top_p,min_p", [(20, 1.0, 0.0), (0, 0.8, 0.0), (0, 1.0, 0.05), (60, 0.95, 0.01)])
@pytest.mark.parametrize("bf16", [False, True])
def test_filtered_tables_through_builder_and_verification(dy, top_k, top_p, min_p, bf16):
    """The builder and the verification on filtered tables are the oracle's on the same tables; no token comes from what was taken out."""
    nodes, V, temps = (60, 33), 1500, [0.7, 1.1]
    g = torch.Generator(device="cuda").manual_seed(top_k + 7)
    randn = lambda *sh: torch.randn(sh, generator=g, device="cuda")
    draft = randn(sum(nodes), V) * 2
    target = draft + 0.5 * randn(sum(nodes), V)
    if bf16:
        draft, target = draft.to(BF16), target.to(BF16)
    batch = dy.Batch.from_sizes(nodes)
    draft, target = (dy.filter_logits(x, batch, temps, top_k=top_k, top_p=top_p, min_p=min_p) for x in (draft, target))
    wide = [x.float() for x in (draft, target)]                    # (the builder reads fp32)
    built = dy.build_tree(wide[0], batch, temps, 11)
    full = compare_trees(built, batch, oracle_trees(wide[0].cpu().numpy(), nodes, temps, 11))
    assert full >= 1 or bf16                                       # (equal logits make decisions that are too close to be compared)
    parent, token = built.tree.parent.cpu().numpy(), built.tree.token.cpu().numpy()
    kept = torch.isfinite(wide[0]).cpu().numpy()
    for s, (a, b) in enumerate(zip(batch.node_offset[:-1], batch.node_offset[1:])):
        for j in range(a + 1, b):
            assert parent[j] < 0 or kept[a + parent[j], token[j]]
    res = dy.verify(draft, target, batch, built.tree, temps, temps, 5)
    t = {k: getattr(built.tree, k).cpu().numpy() for k in ("token", "first_child", "next_sibling")}
    sure = 0
    for s, (a, b) in enumerate(zip(batch.node_offset[:-1], batch.node_offset[1:])):
        want = oracle.verify(wide[0][a:b].cpu().numpy(), wide[1][a:b].cpu().numpy(), t["token"][a:b], t["first_child"][a:b], t["next_sibling"][a:b],
                             f32(temps[s]), f32(temps[s]), 5, seq=s)
        n = int(res.n_accepted[s])
        path = [0] + res.accepted_nodes[a:a + n].tolist()
        last = int(res.final_token[s])
        assert last < 0 or bool(torch.isfinite(wide[1][a + path[-1], last]))
        if want.min_accept_margin >= DECISION_MARGIN:
            sure += 1
            assert res.accepted_nodes[a:a + n].tolist() == want.accepted_nodes.tolist()
    assert sure > 0


@pytest.mark.parametrize("dtype,Hq,Hkv,d", [(BF16, 8, 2, 128), (F32, 4, 4, 64)])
def test_steps_of_a_server(dy, dtype, Hq, Hkv, d):
    """Two requests over a pool that never has much to spare, two layers: one capped with a window, one capped.  Prompts, then steps of
    a draft tree, filtered and verified, then a drawn token each; lengths stay on the device.  Attention is checked against the plain
    form over a record of what went in, pages against the lengths."""
    dev, page, V, cap, window = "cuda", 16, 700, 8.0, 40
    g = torch.Generator(device=dev).manual_seed(3)
    randn = lambda *sh: torch.randn(sh, generator=g, device=dev)
    n_pages = 2 * 12
    pool = dy.PagePool.full(n_pages, page, dev)
    table = torch.full((2, 20), -1, dtype=torch.int32, device=dev)
    k_pages, v_pages = (torch.full((2, n_pages, page, Hkv, d), math.nan, dtype=dtype, device=dev) for _ in range(2))
    cache = dy.PagedCache(k_pages, v_pages, table)
    layers = [cache.layer(l) for l in range(2)]
    scale, exact = 1 / math.sqrt(d), dtype is F32
    record = [[[torch.zeros((0, Hkv, d), dtype=dtype)] * 2 for _ in range(2)] for _ in range(2)]
    held, context = torch.zeros(2, dtype=torch.int32, device=dev), [0, 0]
    settings = dict(top_k=[0, 30], top_p=[0.9, 1.0], min_p=0.01)
    temps = [0.8, 1.0]

    def room(new):
        """Pages for the new tokens, and where they go."""
        nonlocal held
        slots = torch.full((sum(new),), -1, dtype=torch.int64, device=dev)
        wanted = torch.tensor([c + n for c, n in zip(context, new)], dtype=torch.int32, device=dev)
        held = dy.page_plan(pool, table, held, wanted, slots=slots, slots_from=torch.tensor(context, dtype=torch.int32, device=dev))
        assert held.tolist() == wanted.tolist()
        used = [-(-x // page) for x in wanted.tolist()]
        assert pool.state[1].item() == n_pages - sum(used)
        t = table.cpu().numpy()
        assert len({int(p) for s in range(2) for p in t[s, :used[s]]}) == sum(used) and all((t[s, used[s]:] == -1).all() for s in range(2))
        return slots

    def attend(l, batch, slots, mask=None, rel=None):
        total = batch.total_nodes
        q, k, v = (randn(total, Hq + 2 * Hkv, d) * 2).to(dtype).split([Hq, Hkv, Hkv], dim=1)
        q = dy.kv_append(k, v, batch, layers[l], q=q, rel_pos=rel)
        flat = k_pages[l].flatten(0, 1)[slots], v_pages[l].flatten(0, 1)[slots]
        assert torch.equal(flat[0], k) and torch.equal(flat[1], v)
        w = window if l == 0 else 0
        out = dy.paged_attn(q, batch, layers[l], scale, anc_mask=mask, cap=cap, window=w or None, rel_pos=rel)
        if mask is None and sum(context) == 0:                     # the same prompts, never in pages
            whole = dy.prompt_attn(q, k, v, batch, scale, cap=cap, window=w or None)
            assert float((whole.float() - out.float()).abs().max()) <= (8 * 2 ** -8 if dtype is BF16 else 1e-5) * float(v.float().abs().max())
        got, words = out.double().cpu().numpy(), None if mask is None else mask.cpu().numpy().view(np.uint64)
        for s in range(2):
            a, b = int(batch.node_offset[s]), int(batch.node_offset[s + 1])
            keys, values = (torch.cat([r, x[a:b].cpu()]).double().numpy() for r, x in zip(record[l][s], (k, v)))
            see = visible_rows(b - a, context[s], None if words is None else words[a:b], w, None if rel is None else rel[a:b].cpu().numpy())
            want, bound = scored_plain(q[a:b].double().cpu().numpy(), keys, values, see, scale, cap, 0.0 if exact else HALF[BF16], HALF[dtype], exact)
            assert (np.abs(got[a:b] - want) <= bound).all(), (l, s)
        return k, v

    def extend(l, s, k, v):
        record[l][s] = [torch.cat([r, x.cpu()]) for r, x in zip(record[l][s], (k, v))]

    prompts = [37, 80]
    batch, slots = dy.Batch.from_sizes(prompts, context), room(prompts)
    for l in range(2):
        k, v = attend(l, batch, slots)
        for s in range(2):
            extend(l, s, k[batch.node_offset[s]:batch.node_offset[s + 1]], v[batch.node_offset[s]:batch.node_offset[s + 1]])
    context = list(prompts)
    accepted = 0
    for step in range(3):
        sizes = [48, 20]
        batch, slots = dy.Batch.from_sizes(sizes, context), room(sizes)
        draft = randn(sum(sizes), V) * 2
        target = dy.filter_logits(draft + 0.3 * randn(sum(sizes), V), batch, temps, **settings)
        draft = dy.filter_logits(draft, batch, temps, out=draft, **settings)
        built = dy.build_tree(draft, batch, temps, 40 + step)
        rows = [attend(l, batch, slots, built.anc_mask, built.tree.depth) for l in range(2)]
        res = dy.verify(draft, target, batch, built.tree, temps, temps, 90 + step)
        dy.kv_keep(cache, batch, res.accepted_nodes, res.n_accepted)
        n_acc = res.n_accepted.tolist()
        accepted += sum(n_acc)
        for s in range(2):
            a = int(batch.node_offset[s])
            path = [a] + [a + int(x) for x in res.accepted_nodes[a:a + n_acc[s]]]
            for l in range(2):
                extend(l, s, rows[l][0][path], rows[l][1][path])
        context = [c + 1 + n for c, n in zip(context, n_acc)]
        one = dy.Batch.from_sizes([1, 1], context)
        slots = room([1, 1])                                       # what the path did not keep goes back to the pool
        for l in range(2):
            k, v = attend(l, one, slots)
            for s in range(2):
                extend(l, s, k[s:s + 1], v[s:s + 1])
        logits, u = randn(2, V) * 3, torch.rand(2, generator=g, device=dev)
        got = dy.sample(logits, dy.Batch.from_sizes([1, 1]), u, temps, **settings)
        for s in range(2):
            kept, token, prob, _ = plain_row(logits[s].double().cpu().numpy(), u[s].item(), temps[s], settings["top_k"][s], settings["top_p"][s], settings["min_p"])
            assert got.token[s].item() == token and got.n_kept[s].item() == kept.sum() and abs(got.prob[s].item() - prob) <= 1e-6
        context = [c + 1 for c in context]
    assert accepted > 0
    context = [0, 0]
    held = dy.page_plan(pool, table, held, torch.zeros(2, dtype=torch.int32, device=dev))
    assert held.tolist() == [0, 0] and pool.state[1].item() == n_pages and bool((table == -1).all())
    assert sorted(pool.ring.tolist()) == list(range(n_pages))
