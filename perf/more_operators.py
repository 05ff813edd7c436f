"""What a serving step needs beside its cache and its trees, operator by operator: pages are dealt out by the requests' lengths,
attention scores are capped or kept to a window, logits are filtered, tokens are drawn.

A case is a dict of plain values; `kind` says which call it times:

  pages    page_plan: page tables and slot maps follow the requests' lengths, pages taken from the pool and given back to it
  attend   paged_attn with capped scores, a window, or both, over pages
  prompt   prompt_attn with the same
  filter   filter_logits: what top-k, top-p and min-p take out becomes -inf
  sample   sample: a token a row, after the same filters, from given random numbers

Sizes per sequence are comma-separated (`new`, `context`, and the settings of filter and sample).  With `own` false the operators
are computed by elementary torch operations in 32 bits (weights that are summed and compared with a border in 64), rounded once.
"""
import math

import numpy as np
import torch

own = False
DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# contexts of a serving batch of 64 requests, some young, some old: no size a multiple of a page
AGES = ",".join(str(500 + (i * 2477) % 7499) for i in range(64))
YOUNG = ",".join(str(200 + (i * 577) % 1801) for i in range(64))
# settings of 64 requests: greedy ones, plain temperatures, top-k, top-p, min-p, all at once
TEMPERATURES = ",".join(("0", "0.6", "1.0", "0.8", "1.2", "0.7", "0.3", "0.9")[i % 8] for i in range(64))
TOP_KS = ",".join(("0", "0", "0", "50", "0", "200", "0", "40")[i % 8] for i in range(64))
TOP_PS = ",".join(("1.0", "0.9", "1.0", "1.0", "1.0", "0.95", "0.8", "0.92")[i % 8] for i in range(64))
MIN_PS = ",".join(("0", "0", "0", "0", "0.1", "0", "0", "0.02")[i % 8] for i in range(64))


def listed():
    return [
        # one decode step of 64 requests: a token each, a few of them cross into a new page.  The smallest: latency
        dict(name="pages_decode", kind="pages", held=YOUNG, wanted=",".join(str(int(x) + 1) for x in YOUNG.split(",")), page=16, max_pages=256, spare=100),
        # requests come with prompts, others end and give everything back, the rest take room for a draft tree
        dict(name="pages_churn", kind="pages", held=",".join("0" if i % 4 == 0 else x for i, x in enumerate(AGES.split(","))),
             wanted=",".join("0" if i % 4 == 1 else str(int(x) + 64) for i, x in enumerate(AGES.split(","))), page=16, max_pages=512, spare=9000),
        # one request's next token, capped scores: latency
        dict(name="attend_capped_1", kind="attend", new="1", context="1024", q_heads=32, kv_heads=32, head_dim=128, dtype="bf16", page=16, tree=False, cap=50.0, window=0),
        # one token each of 64 requests, capped: the pages' stream from memory is the work
        dict(name="attend_capped_64", kind="attend", new=",".join(["1"] * 64), context=AGES, q_heads=64, kv_heads=8, head_dim=128, dtype="bf16", page=16, tree=False,
             cap=50.0, window=0),
        # the same requests in a layer that looks back 1024 positions
        dict(name="attend_window_64", kind="attend", new=",".join(["1"] * 64), context=AGES, q_heads=64, kv_heads=8, head_dim=128, dtype="bf16", page=16, tree=False,
             cap=0.0, window=1024),
        # the draft tree of the headline shape, verified with capped scores over a window of half its context
        dict(name="attend_capped_tree", kind="attend", new="512", context="4096", q_heads=64, kv_heads=8, head_dim=128, dtype="bf16", page=16, tree=True, cap=50.0,
             window=2048),
        # prompts, from one token to thousands, capped and with a window: the largest
        dict(name="prompt_capped", kind="prompt", new="5000,1,1290,333", q_heads=32, kv_heads=8, head_dim=128, dtype="bf16", cap=50.0, window=2048),
        # small fp32 prompts, grouped heads of 64
        dict(name="prompt_capped_f32", kind="prompt", new="300,1,85,641", q_heads=8, kv_heads=4, head_dim=64, dtype="f32", cap=30.0, window=100),
        # the target's rows of one draft tree, filtered before they are verified: bound by memory
        dict(name="filter_tree", kind="filter", rows="512", vocab=32000, dtype="f32", temperature="0.6", top_k="0", top_p="0.9", min_p="0"),
        # ... of a serving batch of eight trees, each with settings of its own
        dict(name="filter_ragged8", kind="filter", rows="754,102,259,334,466,351,156,95", vocab=32000, dtype="bf16", temperature="0.6,1.0,0.8,0.7,1.2,0,0.9,1.0",
             top_k="0,50,0,200,0,0,1000,0", top_p="0.9,1.0,0.95,0.8,1.0,1.0,0.9,0.99", min_p="0,0,0.02,0,0.1,0,0,0.001"),
        # one request's next token: latency
        dict(name="sample_1", kind="sample", rows="1", vocab=32000, dtype="f32", temperature="0.7", top_k="50", top_p="0.9", min_p="0"),
        # a decode step's 64, each with settings of its own
        dict(name="sample_64", kind="sample", rows=",".join(["1"] * 64), vocab=32000, dtype="bf16", temperature=TEMPERATURES, top_k=TOP_KS, top_p=TOP_PS, min_p=MIN_PS),
    ]


def draw(rng):
    def size(lo, hi):                       # spread over the logarithm, odd values among them
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def sizes(n, lo, hi):
        return [size(lo, hi) for _ in range(n)]

    text = lambda xs: ",".join(str(x) for x in xs)
    kind = rng.choice(["pages", "attend", "attend", "attend", "prompt", "prompt", "filter", "filter", "sample", "sample"])
    n_seq = rng.choice([1, 1, 2, 4, 8, 24, 64])
    if kind == "pages":
        page = rng.choice([8, 16, 16, 32, 64, 256])
        held = [rng.choice([0, x, x, x]) for x in sizes(n_seq, 1, 8000)]
        step = rng.choice(["token", "tree", "churn"])
        wanted = [h + 1 if step == "token" else h + size(2, 768) if step == "tree" else rng.choice([0, h, h + size(1, 4000), max(0, h - size(1, 4000))]) for h in held]
        most = max(1, max(-(-x // page) for x in held + wanted))
        need = sum(max(0, -(-w // page) - -(-h // page)) for h, w in zip(held, wanted))
        return dict(kind=kind, held=text(held), wanted=text(wanted), page=page, max_pages=most + rng.choice([0, 3, 100]),
                    spare=need // 2 if rng.random() < 0.2 else need + rng.randint(1, 500))
    if kind in ("filter", "sample"):
        vocab = rng.choice([32000, 32000, 32768, size(50, 32768), size(50, 32768), 50001, 131072])
        most = max(1, 6_000_000 // vocab)
        if kind == "filter" or rng.random() < 0.3:
            rows = sizes(n_seq, 1, max(2, min(768, most // n_seq)))
        else:
            rows = [1] * n_seq
        which = [rng.choice(["greedy", "plain", "top_k", "top_p", "min_p", "all"]) for _ in rows]
        return dict(kind=kind, rows=text(rows), vocab=vocab, dtype=rng.choice(["f32", "bf16"]),
                    temperature=text("0" if w == "greedy" else round(rng.uniform(0.2, 1.5), 3) for w in which),
                    top_k=text(size(1, 2000) if w in ("top_k", "all") else 0 for w in which),
                    top_p=text(round(rng.uniform(0.3, 0.999), 4) if w in ("top_p", "all") else 1.0 for w in which),
                    min_p=text(round(rng.uniform(0.001, 0.3), 4) if w in ("min_p", "all") else 0 for w in which))
    f32 = rng.random() < 0.25
    q_heads, kv_heads = rng.choice([(8, 8), (8, 4), (16, 2)] if f32 else [(32, 32), (40, 40), (64, 8), (32, 8)])
    heads = dict(q_heads=q_heads, kv_heads=kv_heads, head_dim=rng.choice([64, 64, 128, 96]) if f32 else rng.choice([128, 128, 64]), dtype="f32" if f32 else "bf16")
    form = rng.choice(["cap", "window", "both", "both"])
    scores = dict(cap=0.0 if form == "window" else round(rng.uniform(5, 100), 2), window=0 if form == "cap" else size(16, 4000))
    if kind == "prompt":
        most = 1000 if f32 else 5000
        return dict(kind=kind, new=text(sizes(n_seq, 1, max(most // n_seq, 2) if n_seq < 8 else 400)), **heads, **scores)
    shape = rng.choice(["decode", "decode", "tree", "tree", "chunk"])
    if shape == "decode":
        new, context = [1] * n_seq, sizes(n_seq, 16, 1000 if f32 else 16000 if n_seq < 24 else 6000)
    else:
        n_seq = min(n_seq, 8)
        new = sizes(n_seq, 2, 100 if f32 else 768 if shape == "tree" else 1500 // n_seq + 100)
        context = sizes(n_seq, 16, 1000 if f32 else 5000)
    return dict(kind=kind, new=text(new), context=text(context), page=rng.choice([8, 16, 16, 32, 64, 256]), tree=shape == "tree", **heads, **scores)


# ---------------------------------------------------------------------------------------- inputs

def ints(text):
    return [int(x) for x in str(text).split(",")]


def floats(text):
    return [float(x) for x in str(text).split(",")]


class Bag:
    """The state of a case: what a program holds before the call."""

    def __init__(self, **kw):
        self.__dict__.update(kw)


def trees(sizes, rng):
    """Random trees, a row of each pointing to an earlier one: (ancestor bits [sum, words] int64, depth [sum] int32)."""
    words = max(1, -(-max(sizes) // 64))
    masks, depths = [], []
    for n in sizes:
        bits, depth = np.zeros((n, words), np.uint64), np.zeros(n, np.int32)
        for j in range(n):
            if j:
                up = int(j * rng.random() ** 1.5)
                bits[j], depth[j] = bits[up], depth[up] + 1
            bits[j, j // 64] |= np.uint64(1) << np.uint64(j % 64)
        masks.append(bits)
        depths.append(depth)
    return np.concatenate(masks).view(np.int64), np.concatenate(depths)


def page_table(lengths, page, columns, spare, rng):
    """A pool with pages to spare, its pages dealt out in no order: (table [n_seq, columns] int32, the free pages, pages of the pool)."""
    need = [-(-n // page) for n in lengths]
    pool = sum(need) + spare
    order = rng.permutation(pool).astype(np.int32)
    table = np.full((len(need), columns), -1, np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, order[at:], pool


def put(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEVICE)


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    kind = case["kind"]
    if kind == "pages":
        held, wanted = ints(case["held"]), ints(case["wanted"])
        table, free, pool = page_table(held, case["page"], case["max_pages"], case["spare"], rng)
        ring = np.full(pool, -1, np.int32)                                               # free pages from `head` on, round the end
        head = int(rng.integers(pool))
        ring[(head + np.arange(len(free))) % pool] = free
        growth = max(sum(max(0, b - a) for a, b in zip(*x)) for x in ((held, wanted), (wanted, held)))
        # a pass goes from one set of lengths to the other, the next one back
        lengths = (put(np.asarray(held, np.int32)), put(np.asarray(wanted, np.int32)))
        return Bag(kind=kind, page=case["page"], table=put(table), ring=put(ring), state=put(np.asarray([head, len(free), 0, 0], np.int32)),
                   lengths=lengths, held=lengths[0], turn=0, slots=put(np.full(max(1, growth), -1, np.int64)), pool=None)
    dtype = DTYPES[case["dtype"]]
    randn = lambda *shape: torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)
    if kind in ("filter", "sample"):
        rows, vocab = ints(case["rows"]), case["vocab"]
        total = sum(rows)
        s = Bag(kind=kind, rows=rows, batch=None, temperature=floats(case["temperature"]), top_k=ints(case["top_k"]), top_p=floats(case["top_p"]), min_p=floats(case["min_p"]))
        # a language model's logits: most tokens far below a few, rows of different sharpness
        s.logits = (randn(total, vocab) * 2.0 - 2.0 + (2.0 + randn(total, 1).abs() * 3.0) * (torch.rand((total, vocab), generator=gen, device=DEVICE) < 0.002)).to(dtype)
        s.uniform = torch.rand(total, generator=gen, device=DEVICE)
        # the plain form looks its settings up row by row; as a program's own 32-bit numbers
        row_of = np.repeat(np.arange(len(rows)), rows)
        s.by_row = [put(np.asarray(x, t)[row_of])[:, None] for x, t in ((s.temperature, np.float32), (s.top_k, np.int64), (s.top_p, np.float32), (s.min_p, np.float32))]
        return s
    new, hkv, d = ints(case["new"]), case["kv_heads"], case["head_dim"]
    total = sum(new)
    s = Bag(kind=kind, new=new, context=[0] * len(new), batch=None, cache=None, mask=None, depth=None, scale=1.0 / math.sqrt(d), cap=case["cap"], window=case["window"])
    s.local = put(np.concatenate([np.arange(n) for n in new]))                          # a token's place in its sequence's new ones
    s.owner = put(np.repeat(np.arange(len(new)), new))                                  # its sequence
    s.new_of, s.context_of = put(np.asarray(new)), put(np.asarray(s.context))
    # queries larger than keys, so that scores reach into the cap's bend
    if kind == "prompt":                                                                # views of what one projection wrote
        qkv = randn(total, case["q_heads"] + 2 * hkv, d)
        qkv[:, :case["q_heads"]] *= 4.0
        s.q, s.k, s.v = qkv.to(dtype).split([case["q_heads"], hkv, hkv], dim=1)
        return s
    s.context = ints(case["context"])
    s.context_of = put(np.asarray(s.context))
    s.page = case["page"]
    lengths = [c + n for c, n in zip(s.context, new)]
    table, _, pool = page_table(lengths, s.page, max(1, max(-(-n // s.page) for n in lengths)), 3, rng)
    s.table = put(table)
    s.k_pages, s.v_pages = randn(pool, s.page, hkv, d).to(dtype), randn(pool, s.page, hkv, d).to(dtype)
    if case["tree"]:
        mask, depth = trees(new, rng)
        s.mask, s.depth = put(mask), put(depth)
    s.q = (randn(total, case["q_heads"], d) * 4.0).to(dtype)
    return s


# ---------------------------------------------------------------------------------------- the calls

def run(s):
    if own:
        return run_own(s)
    if s.kind == "pages":
        return plain_pages(s)
    if s.kind == "filter":
        return plain_filter(s)
    if s.kind == "sample":
        return plain_sample(s)
    return plain_attend(s)


def next_lengths(s):
    """The lengths that this pass is to bring the requests to."""
    s.turn ^= 1
    return s.lengths[s.turn]


def run_own(s):
    import paper_2410_11744_amd as dy
    if s.kind == "pages":
        if s.pool is None:                  # a program has one pool for as long as it runs
            s.pool = dy.PagePool(s.ring, s.state, s.page)
        s.held = dy.page_plan(s.pool, s.table, s.held, next_lengths(s), slots=s.slots)
        return s.table, s.held, s.slots, s.ring, s.state
    if s.kind in ("filter", "sample"):
        if s.batch is None:                 # ... and describes its step once
            s.batch = dy.Batch.from_sizes(s.rows)
        if s.kind == "filter":
            return dy.filter_logits(s.logits, s.batch, s.temperature, top_k=s.top_k, top_p=s.top_p, min_p=s.min_p)
        got = dy.sample(s.logits, s.batch, s.uniform, s.temperature, top_k=s.top_k, top_p=s.top_p, min_p=s.min_p)
        return got.token, got.prob, got.n_kept
    if s.batch is None:
        s.batch = dy.Batch.from_sizes(s.new, s.context)
        s.cache = None if s.kind == "prompt" else dy.PagedCache(s.k_pages, s.v_pages, s.table)
    cap, window = s.cap or None, s.window or None
    if s.kind == "attend":
        return dy.paged_attn(s.q, s.batch, s.cache, s.scale, anc_mask=s.mask, cap=cap, window=window, rel_pos=s.depth)
    return dy.prompt_attn(s.q, s.k, s.v, s.batch, s.scale, cap=cap, window=window)


# ---------------------------------------------------------------------------------------- plain forms

def plain_pages(s):
    """Everything by columns of the table: a place's page comes from the ring, or goes behind its last free one."""
    pool, columns, page = s.ring.numel(), s.table.shape[1], s.page
    head, count = s.state[0].long(), s.state[1].long()
    a, b = s.held.long(), next_lengths(s).long()
    before, after = (a + page - 1) // page, (b + page - 1) // page
    right = (a >= 0) & (b >= 0) & (before <= columns) & (after <= columns)
    need = torch.where(right, (after - before).clamp(min=0), 0)
    fits = need.cumsum(0) <= count
    taken = torch.where(fits, need, 0)
    back = torch.where(right, (before - after).clamp(min=0), 0)
    column = torch.arange(columns, device=DEVICE)
    new = (column >= before[:, None]) & (column < (before + taken)[:, None])
    left = (column >= after[:, None]) & (column < (after + back)[:, None])
    source = head + (taken.cumsum(0) - taken)[:, None] + column - before[:, None]
    target = head + count + (back.cumsum(0) - back)[:, None] + column - after[:, None]
    fresh = s.ring[source % pool]
    longer = torch.cat((s.ring, s.ring[:1]))                                             # (one place more: what does not go back)
    longer[torch.where(left, target % pool, pool).flatten()] = s.table.flatten()
    s.ring.copy_(longer[:pool])
    s.table.copy_(torch.where(new, fresh, torch.where(left, -1, s.table)))
    s.state[0], s.state[1] = (head + taken.sum()) % pool, count - taken.sum() + back.sum()
    grows = torch.where(right, (b - a).clamp(min=0), 0)
    ends = grows.cumsum(0)
    token = torch.arange(s.slots.numel(), device=DEVICE)
    owner = torch.searchsorted(ends, token, right=True)
    some = owner < ends.numel()
    owner = torch.where(some, owner, 0)
    place = a[owner] + token - (ends - grows)[owner]
    spot = s.table[owner, (place // page).clamp(0, columns - 1)].long() * page + place % page
    s.slots.copy_(torch.where(some, torch.where(fits[owner] | (need[owner] == 0), spot, -1), s.slots))
    s.held = torch.where(right, torch.where(fits | (need == 0), b, a), -1).int()
    return s.table, s.held, s.slots, s.ring, s.state


def plain_weights(s):
    """Weights against the row's largest, and which tokens the filters keep, [rows, vocab] in 64 bits."""
    temperature, top_k, top_p, min_p = s.by_row
    x = s.logits.double()
    vocab = x.shape[1]
    weight = torch.exp((x - x.amax(1, keepdim=True)) / torch.where(temperature > 0, temperature, 1.0).double())
    _, order = torch.sort(x, dim=1, descending=True, stable=True)
    down = torch.gather(weight, 1, order)
    rank = torch.arange(vocab, device=DEVICE)
    keep = rank < torch.where(top_k > 0, top_k, vocab)
    down = torch.where(keep, down, 0.0)
    total = down.cumsum(1)
    keep &= (total - down < top_p.double() * total[:, -1:]) | (top_p >= 1.0)
    keep &= down >= min_p.double()
    keep = torch.where(temperature > 0, keep, rank == 0)
    return weight, torch.zeros_like(keep).scatter_(1, order, keep)


def plain_filter(s):
    return torch.where(plain_weights(s)[1], s.logits, -math.inf)


def plain_sample(s):
    weight, keep = plain_weights(s)
    weight = torch.where(keep, weight, 0.0)
    upto = weight.cumsum(1)
    token = (upto <= s.uniform.double()[:, None] * upto[:, -1:]).sum(1)
    prob = torch.gather(weight, 1, token[:, None])[:, 0] / upto[:, -1]
    return token.int(), prob.float(), keep.sum(1).int()


def plain_attend(s):
    """Every sequence padded to the longest; scores in full."""
    n_seq, most = len(s.new), max(s.new)
    total, hq, d = s.q.shape
    keys = max(c + n for c, n in zip(s.context, s.new))
    key, query = torch.arange(keys, device=DEVICE), torch.arange(most, device=DEVICE)
    in_use = key < (s.context_of + s.new_of)[:, None]
    if s.kind == "prompt":
        start = torch.cumsum(s.new_of, 0) - s.new_of
        at = torch.where(in_use, start[:, None] + key, 0)
        k, v = s.k[at].float(), s.v[at].float()
    else:
        where = torch.where(in_use, key, 0)
        at = s.table[torch.arange(n_seq, device=DEVICE)[:, None], where // s.page].long(), where % s.page
        k, v = s.k_pages[at].float(), s.v_pages[at].float()                             # [n_seq, keys, Hkv, d]
    since = key - s.context_of[:, None]                                                 # a key's row among the new tokens
    if s.mask is None:
        seen = since[:, None, :] <= query[None, :, None]
    else:
        words = torch.zeros((n_seq, most, s.mask.shape[1]), dtype=torch.int64, device=DEVICE)
        words[s.owner, s.local] = s.mask
        bit = since.clamp(min=0)
        word = (bit // 64).clamp(max=s.mask.shape[1] - 1)
        seen = (torch.gather(words, 2, word[:, None, :].expand(-1, most, -1)) >> (bit % 64)[:, None, :]) & 1 == 1
        seen |= since[:, None, :] < 0
    seen &= in_use[:, None, :]
    if s.window:                                                                        # positions relative to the context's end
        row_at, key_at = query.expand(n_seq, -1), since
        if s.depth is not None:
            row_at = torch.zeros((n_seq, most), dtype=torch.int64, device=DEVICE)
            row_at[s.owner, s.local] = s.depth.long()
            key_at = torch.where(since < 0, since, torch.gather(row_at, 1, since.clamp(0, most - 1)))
        seen &= key_at[:, None, :] > row_at[:, :, None] - s.window
    hkv = k.shape[2]
    q = torch.zeros((n_seq, most, hq, d), dtype=torch.float32, device=DEVICE)
    q[s.owner, s.local] = s.q.float() * s.scale
    q = q.view(n_seq, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n_seq, hkv, -1, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).view(n_seq, hkv, hq // hkv, most, keys)
    if s.cap:
        score = score.div_(s.cap).tanh_().mul_(s.cap)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)      # a row that sees nothing: all zeros
    weight = score.exp_()
    total_weight = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.view(n_seq, hkv, -1, keys), v.permute(0, 2, 1, 3).contiguous()).view(n_seq, hkv, hq // hkv, most, d)
    out = torch.where(total_weight > 0, out / total_weight, 0.0)
    return out.permute(0, 3, 1, 2, 4)[s.owner, s.local].reshape(total, hq, d).to(s.q.dtype)


# ---------------------------------------------------------------------------------------- cost and truth

def visible_pairs(new, context, window, tree):
    """Pairs of a row and a key that it sees; of a tree's rows among themselves: each its own."""
    pairs = 0
    for n, c in zip(new, context):
        back = (np.zeros(n, np.int64) if tree else np.arange(n)) + c + 1                 # keys up to the row's own
        pairs += int(np.minimum(back, window or 1 << 40).sum())
    return pairs


def work(case):
    """Inputs read once, outputs written once; products of visible pairs only."""
    kind = case["kind"]
    if kind == "pages":
        held, wanted, page = ints(case["held"]), ints(case["wanted"]), case["page"]
        moved = sum(abs(-(-b // page) - -(-a // page)) for a, b in zip(held, wanted))
        return dict(bytes=12 * len(held) + 8 * moved + 8 * sum(max(0, b - a) for a, b in zip(held, wanted)), flops=0)
    size = 4 if case["dtype"] == "f32" else 2
    if kind in ("filter", "sample"):
        n = sum(ints(case["rows"]))
        return dict(bytes=size * n * case["vocab"] * (2 if kind == "filter" else 1) + 16 * n, flops=4 * n * case["vocab"])
    new, hq, hkv, d = ints(case["new"]), case["q_heads"], case["kv_heads"], case["head_dim"]
    context = [0] * len(new) if kind == "prompt" else ints(case["context"])
    window = case["window"] or 1 << 40
    keys = sum(min(c, window - 1) + n if n else 0 for n, c in zip(new, context))
    return dict(bytes=size * (2 * sum(new) * hq + 2 * keys * hkv) * d, flops=4 * hq * d * visible_pairs(new, context, case["window"], case.get("tree")))


def exact_pages(s):
    """Sequence by sequence, on the host."""
    (a, b), page = (x.tolist() for x in s.lengths), s.page
    table, ring, slots = s.table.cpu().numpy(), s.ring.cpu().numpy(), s.slots.cpu().numpy()
    head, free = int(s.state[0]), int(s.state[1])
    tail, at, asked, taken, granted = head + free, 0, 0, 0, []
    returned = []
    for q, (x, y) in enumerate(zip(a, b)):
        before, after = -(-x // page), -(-y // page)
        asked += max(0, after - before)
        ok = after <= before or asked <= free
        granted.append(y if ok else x)
        for column in range(before, after if ok else before):
            table[q, column] = ring[(head + taken) % len(ring)]
            taken += 1
        for column in range(after, before):
            returned.append((tail + len(returned), int(table[q, column])))
            table[q, column] = -1
        for place in range(x, y):
            slots[at] = int(table[q, place // page]) * page + place % page if ok else -1
            at += 1
    for to, number in returned:
        ring[to % len(ring)] = number
    state = np.asarray([(head + taken) % len(ring), free - taken + len(returned), 0, 0], np.int32)
    return put(table), put(np.asarray(granted, np.int32)), put(slots), put(ring), put(state)


def exact_rows(s):
    """Row by row on the host: tokens are taken, largest first, until one of the filters says stop."""
    settings = [np.repeat(np.asarray(x, np.float32).astype(np.float64), s.rows) for x in (s.temperature, s.top_k, s.top_p, s.min_p)]
    logits, uniform = s.logits.double().cpu().numpy(), s.uniform.double().cpu().numpy()
    filtered, tokens, probs, counts = np.full(logits.shape, -np.inf), [], [], []
    for r, x in enumerate(logits):
        temperature, top_k, top_p, min_p = (y[r] for y in settings)
        order = np.argsort(-x, kind="stable")
        if temperature == 0:
            kept, share = order[:1], np.ones(1)
        else:
            best = order[:int(top_k)] if top_k > 0 else order
            share = np.exp((x[best] - x[best[0]]) / temperature)
            n = len(best)
            if top_p < 1:
                n = min(n, 1 + int(np.searchsorted(np.cumsum(share), top_p * share.sum(), side="left")))
            n = min(n, int(np.count_nonzero(share >= min_p)))
            kept, share = best[:n], share[:n]
        filtered[r, kept] = x[kept]
        by_index = np.argsort(kept)
        sums = np.cumsum(share[by_index])
        i = int(np.searchsorted(sums, uniform[r] * sums[-1], side="right"))
        tokens.append(kept[by_index[i]])
        probs.append(share[by_index[i]] / sums[-1])
        counts.append(len(kept))
    if s.kind == "filter":
        return put(filtered)
    return put(np.asarray(tokens, np.int32)), put(np.asarray(probs)), put(np.asarray(counts, np.int32))


def exact(case, seed):
    """From the definitions, sequence by sequence, in 64 bits."""
    s = prepare(case, seed)
    if s.kind == "pages":
        return exact_pages(s)
    if s.kind in ("filter", "sample"):
        return exact_rows(s)
    out = torch.zeros(s.q.shape, dtype=torch.float64, device=DEVICE)
    ends = np.cumsum(s.new)
    for b, end in enumerate(ends):
        n, c = s.new[b], s.context[b]
        span = slice(int(end) - n, int(end))
        if s.kind == "prompt":
            k, v = s.k[span], s.v[span]
        else:
            pages = s.table[b, :-(-(c + n) // s.page)].long()
            k, v = (p[pages].flatten(0, 1)[:c + n] for p in (s.k_pages, s.v_pages))
        places = torch.arange(n, device=DEVICE)
        if s.mask is None:
            among = torch.ones(n, n, dtype=torch.bool, device=DEVICE).tril()
        else:
            among = ((s.mask[span][:, places // 64] >> (places % 64)) & 1).bool()
        hidden = torch.cat((torch.zeros(n, c, dtype=torch.bool, device=DEVICE), ~among), dim=1)
        if s.window:
            new_at = c + (places if s.depth is None else s.depth[span].long())
            key_at = torch.cat((torch.arange(c, device=DEVICE), new_at))
            hidden |= new_at[:, None] - key_at >= s.window
        for h in range(s.q.shape[1]):
            g = h * k.shape[1] // s.q.shape[1]
            x = (s.q[span, h].double() @ k[:, g].double().t()).mul_(s.scale)
            if s.cap:
                x = s.cap * torch.tanh(x / s.cap)
            x = x.masked_fill_(hidden, -math.inf)
            out[span, h] = x.sub_(torch.logsumexp(x, dim=1, keepdim=True)).exp_().nan_to_num_(nan=0.0) @ v[:, g].double()
    return out
