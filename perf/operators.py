"""The serving path around a speculative step, operator by operator: keys and values go into a paged cache, chunks of new
tokens and draft trees attend to it, the accepted path is kept, whole prompts attend to themselves.

A case is a dict of plain values; `kind` says which call it times:

  append   kv_append: the new tokens' keys (rotated) and values into the pages, their rotated queries beside
  attend   paged_attn: new tokens that are in the pages already attend to everything before them, or by an ancestor mask
  keep     kv_keep: the accepted path's rows move up behind the root's, in every layer
  prompt   prompt_attn: packed prompts, causal, keys and values as the projection wrote them

`new` and `context` are comma-separated sizes, one per sequence: its new tokens, and the tokens that the cache holds before them.
With `own` false the operators are computed by elementary torch operations in 32 bits (angles in 64), rounded once at the end.
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


def listed():
    return [
        # one decode step's keys and values of 64 requests: latency, a few hundred KB
        dict(name="append_decode", kind="append", new=",".join(["1"] * 64), context=YOUNG, q_heads=64, kv_heads=8, head_dim=128, dtype="bf16", page=16,
             rotary=128, interleaved=False, tree=False),
        # four prompts (or pieces of prompts) through the 40-head shape: bound by memory
        dict(name="append_prompts", kind="append", new="1531,706,2048,37", context="0,512,100,0", q_heads=40, kv_heads=40, head_dim=128, dtype="bf16", page=64,
             rotary=128, interleaved=False, tree=False),
        # the smallest: a tree of 32 rows, fp32, neighbouring pairs rotated, half of the head, positions by depth
        dict(name="append_tree_f32", kind="append", new="32", context="128", q_heads=8, kv_heads=8, head_dim=64, dtype="f32", page=16,
             rotary=32, interleaved=True, tree=True),
        # after the verification of one tree: 9 rows of 80 layers
        dict(name="keep_70b", kind="keep", new="512", context="67", kv_heads=8, head_dim=128, dtype="bf16", page=16, layers=80, accepted="9"),
        # ... of a serving batch of eight trees, one of which accepted nothing
        dict(name="keep_ragged8", kind="keep", new="754,102,259,334,466,351,156,95", context="83,6,118,65,43,47,55,30", kv_heads=8, head_dim=128, dtype="bf16",
             page=32, layers=16, accepted="12,3,1,7,0,5,4,2"),
        # one request, one token: latency
        dict(name="attend_decode_1", kind="attend", new="1", context="1024", q_heads=32, kv_heads=32, head_dim=128, dtype="bf16", page=16, tree=False),
        # one token each of 64 requests: the pages' stream from memory is the work
        dict(name="attend_decode_64", kind="attend", new=",".join(["1"] * 64), context=AGES, q_heads=64, kv_heads=8, head_dim=128, dtype="bf16", page=16, tree=False),
        # the draft tree of the headline shape, verified over pages: bound by the matrix cores
        dict(name="attend_tree_70b", kind="attend", new="512", context="4096", q_heads=64, kv_heads=8, head_dim=128, dtype="bf16", page=16, tree=True),
        # pieces of two prompts beside requests that decode, the way a server fills its step
        dict(name="attend_mixed", kind="attend", new="700,1,1,331,1,5,1,0", context="2500,1801,77,0,4600,1203,2999,640", q_heads=64, kv_heads=8, head_dim=128,
             dtype="bf16", page=64, tree=False),
        # a long prompt of the headline shape: the largest
        dict(name="prompt_8k", kind="prompt", new="8192", q_heads=64, kv_heads=8, head_dim=128, dtype="bf16"),
        # a packed batch of prompts, from one token to over a thousand, ungrouped heads
        dict(name="prompt_packed", kind="prompt", new="1,517,1300,64,129,33,903,260,2,750,127,411", q_heads=32, kv_heads=32, head_dim=128, dtype="bf16"),
        # small fp32 prompts, grouped heads of 64
        dict(name="prompt_packed_f32", kind="prompt", new="300,1,85,641", q_heads=8, kv_heads=4, head_dim=64, dtype="f32"),
    ]


def draw(rng):
    def size(lo, hi):                       # spread over the logarithm, odd values among them
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def sizes(n, lo, hi):
        return [size(lo, hi) for _ in range(n)]

    text = lambda xs: ",".join(str(x) for x in xs)
    kind = rng.choice(["append", "append", "attend", "attend", "attend", "attend", "keep", "prompt", "prompt"])
    f32 = rng.random() < 0.25
    q_heads, kv_heads = rng.choice([(8, 8), (8, 4), (16, 2)] if f32 else [(32, 32), (40, 40), (64, 8), (32, 8)])
    head_dim = rng.choice([64, 64, 128, 96]) if f32 else rng.choice([128, 128, 64])
    heads = dict(q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, dtype="f32" if f32 else "bf16")
    page = rng.choice([8, 16, 16, 32, 64, 256])
    n_seq = rng.choice([1, 1, 2, 4, 8, 24, 64])
    if kind == "append":
        most = 6000 // n_seq
        new = [1] * n_seq if rng.random() < 0.4 else sizes(n_seq, 1, max(most, 2))
        rotary = rng.choice([head_dim, head_dim, head_dim // 2])
        return dict(kind=kind, new=text(new), context=text(sizes(n_seq, 1, 1500)), page=page, rotary=rotary, interleaved=rng.random() < 0.3,
                    tree=max(new) > 1 and max(new) <= 768 and rng.random() < 0.4, **heads)
    if kind == "keep":
        n_seq = rng.choice([1, 2, 4, 8])
        new = sizes(n_seq, 40, 600)
        return dict(kind=kind, new=text(new), context=text(sizes(n_seq, 1, 200)), kv_heads=kv_heads, head_dim=head_dim, dtype=heads["dtype"], page=page,
                    layers=rng.choice([1, 8, 16]), accepted=text([rng.randint(0, 12) for _ in new]))
    if kind == "prompt":
        most = 1000 if f32 else 6000
        new = sizes(n_seq, 1, max(most // n_seq, 2) if n_seq < 8 else 400)
        return dict(kind=kind, new=text(new), **heads)
    shape = rng.choice(["decode", "decode", "tree", "tree", "chunk"])
    if shape == "decode":
        new = [1] * n_seq
        context = sizes(n_seq, 16, 1000 if f32 else 16000 if n_seq < 24 else 6000)
    else:
        n_seq = min(n_seq, 8)
        new = sizes(n_seq, 2, 100 if f32 else 768 if shape == "tree" else 1500 // n_seq + 100)
        context = sizes(n_seq, 16, 1000 if f32 else 5000)
    return dict(kind=kind, new=text(new), context=text(context), page=page, tree=shape == "tree", **heads)


# ---------------------------------------------------------------------------------------- inputs

def ints(text):
    return [int(x) for x in str(text).split(",")]


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


def page_table(lengths, page, rng):
    """A pool with a few pages to spare, its pages dealt out in no order: (table [n_seq, most] int32, pages of the pool)."""
    need = [-(-n // page) for n in lengths]
    pool = sum(need) + 3
    order = rng.permutation(pool).astype(np.int32)
    table = np.zeros((len(need), max(1, max(need))), np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table, pool


def paths(sizes, accepted, rng):
    """Accepted rows as a verification lists them: per sequence, from its first row on, ascending.  They lie behind the
    places they move to, so that the call can be repeated."""
    rows = np.full(sum(sizes), -1, np.int32)
    at = 0
    for n, a in zip(sizes, accepted):
        rows[at:at + a] = np.sort(rng.choice(np.arange(a + 1, n), a, replace=False))
        at += n
    return rows


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype, kind = DTYPES[case["dtype"]], case["kind"]
    randn = lambda *shape: torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32).to(dtype)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEVICE)
    new, hkv, d = ints(case["new"]), case["kv_heads"], case["head_dim"]
    total = sum(new)
    s = Bag(kind=kind, new=new, context=[0] * len(new), batch=None, cache=None, mask=None, scale=1.0 / math.sqrt(d))
    s.local = put(np.concatenate([np.arange(n) for n in new]))                          # a token's place in its sequence's new ones
    s.owner = put(np.repeat(np.arange(len(new)), new))                                  # its sequence
    s.new_of, s.context_of = put(np.asarray(new)), put(np.asarray(s.context))
    if kind == "prompt":                                                                # views of what one projection wrote
        qkv = randn(total, case["q_heads"] + 2 * hkv, d)
        s.q, s.k, s.v = qkv.split([case["q_heads"], hkv, hkv], dim=1)
        return s
    s.context = ints(case["context"])
    s.context_of = put(np.asarray(s.context))
    s.page = case["page"]
    table, pool = page_table([c + n for c, n in zip(s.context, new)], s.page, rng)
    s.table = put(table)
    layers = [case["layers"]] if kind == "keep" else []
    s.k_pages, s.v_pages = randn(*layers, pool, s.page, hkv, d), randn(*layers, pool, s.page, hkv, d)
    if kind == "keep":
        accepted = ints(case["accepted"])
        s.rows, s.n_rows = put(paths(new, accepted, rng)), put(np.asarray(accepted, np.int32))
        s.first_row = put(np.concatenate([[0], np.cumsum(new)[:-1]]))
        s.most = max(accepted)
        return s
    if case["tree"]:
        mask, depth = trees(new, rng)
        s.mask, s.depth = put(mask), put(depth)
    if kind == "attend":
        s.q = randn(total, case["q_heads"], d)
        return s
    s.q, s.k, s.v = randn(total, case["q_heads"] + 2 * hkv, d).split([case["q_heads"], hkv, hkv], dim=1)
    half = case["rotary"] // 2
    s.inv_freq = (10000.0 ** (-torch.arange(half, device=DEVICE, dtype=torch.float64) / half)).float()
    s.interleaved = case["interleaved"]
    s.rel_pos = s.depth if case["tree"] else None
    return s


# ---------------------------------------------------------------------------------------- the calls

def run(s):
    if own:
        return run_own(s)
    if s.kind == "append":
        return plain_append(s)
    if s.kind == "keep":
        return plain_keep(s)
    return plain_attend(s)


def run_own(s):
    import paper_2410_11744_amd as dy
    if s.batch is None:                     # a program describes its step once, and calls every layer with that
        s.batch = dy.Batch.from_sizes(s.new, s.context)
        s.cache = None if s.kind == "prompt" else dy.PagedCache(s.k_pages, s.v_pages, s.table)
    if s.kind == "append":
        q = dy.kv_append(s.k, s.v, s.batch, s.cache, q=s.q, rel_pos=s.rel_pos, inv_freq=s.inv_freq, interleaved=s.interleaved)
        return q, s.k_pages, s.v_pages
    if s.kind == "keep":
        dy.kv_keep(s.cache, s.batch, s.rows, s.n_rows)
        return s.k_pages, s.v_pages
    if s.kind == "attend":
        return dy.paged_attn(s.q, s.batch, s.cache, s.scale, anc_mask=s.mask)
    return dy.prompt_attn(s.q, s.k, s.v, s.batch, s.scale)


# ---------------------------------------------------------------------------------------- plain forms

def place(s, sequence, position):
    """Page and row of tokens in the pool."""
    return s.table[sequence, position // s.page].long(), position % s.page


def plain_rotate(x, position, inv_freq, interleaved):
    half = inv_freq.numel()
    angle = position.double()[:, None, None] * inv_freq.double()
    cos, sin = angle.cos().float(), angle.sin().float()
    x = x.float()
    turned, rest = x[..., :2 * half], x[..., 2 * half:]
    if interleaved:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    else:
        a, b = turned[..., :half], turned[..., half:]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    return torch.cat((turned, rest), dim=-1)


def plain_append(s):
    first = s.context_of[s.owner]
    position = first + (s.local if s.rel_pos is None else s.rel_pos)
    at = place(s, s.owner, first + s.local)
    s.k_pages[at] = plain_rotate(s.k, position, s.inv_freq, s.interleaved).to(s.k_pages.dtype)
    s.v_pages[at] = s.v
    return plain_rotate(s.q, position, s.inv_freq, s.interleaved).to(s.q.dtype), s.k_pages, s.v_pages


def plain_keep(s):
    step = torch.arange(s.most, device=DEVICE)
    sequence, step = torch.nonzero(step < s.n_rows[:, None], as_tuple=True)
    row = s.rows[s.first_row[sequence] + step].long()
    root = s.context_of[sequence]
    old, there = place(s, sequence, root + row), place(s, sequence, root + 1 + step)
    s.k_pages[:, there[0], there[1]] = s.k_pages[:, old[0], old[1]]
    s.v_pages[:, there[0], there[1]] = s.v_pages[:, old[0], old[1]]
    return s.k_pages, s.v_pages


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
        at = place(s, torch.arange(n_seq, device=DEVICE)[:, None], torch.where(in_use, key, 0))
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
    hkv = k.shape[2]
    q = torch.zeros((n_seq, most, hq, d), dtype=torch.float32, device=DEVICE)
    q[s.owner, s.local] = s.q.float() * s.scale
    q = q.view(n_seq, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(n_seq, hkv, -1, d)
    score = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).view(n_seq, hkv, hq // hkv, most, keys)
    score.masked_fill_(~seen[:, None, None], -math.inf)
    score -= score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)      # a row that sees nothing: all zeros
    weight = score.exp_()
    total_weight = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.view(n_seq, hkv, -1, keys), v.permute(0, 2, 1, 3).contiguous()).view(n_seq, hkv, hq // hkv, most, d)
    out = torch.where(total_weight > 0, out / total_weight, 0.0)
    return out.permute(0, 3, 1, 2, 4)[s.owner, s.local].reshape(total, hq, d).to(s.q.dtype)


# ---------------------------------------------------------------------------------------- cost and truth

def work(case):
    """Inputs read once, outputs written once; products of visible pairs only (of a tree's rows among themselves: each its own)."""
    new, context = ints(case["new"]), ints(case.get("context", "0"))
    size = 4 if case["dtype"] == "f32" else 2
    hkv, d, total = case["kv_heads"], case["head_dim"], sum(new)
    if case["kind"] == "append":
        hq = case["q_heads"]
        return dict(bytes=2 * size * total * (hq + 2 * hkv) * d, flops=3 * total * (hq + hkv) * case["rotary"])
    if case["kind"] == "keep":
        return dict(bytes=4 * size * sum(ints(case["accepted"])) * hkv * d * case["layers"], flops=0)
    hq = case["q_heads"]
    if case["kind"] == "prompt":
        context = [0] * len(new)
    alone = case.get("tree")
    pairs = sum(n * c + (n if alone else n * (n + 1) // 2) for n, c in zip(new, context))
    keys = sum((c + n) if n else 0 for n, c in zip(new, context))
    return dict(bytes=size * (2 * total * hq + 2 * keys * hkv) * d, flops=4 * hq * d * pairs)


def exact(case, seed):
    """From the definitions, sequence by sequence, in 64 bits."""
    s = prepare(case, seed)
    ends = np.cumsum(s.new)
    if s.kind in ("append", "keep"):
        k, v, table = s.k_pages.double(), s.v_pages.double(), s.table.cpu().numpy()
        spot = lambda b, p: (int(table[b, p // s.page]), p % s.page)
        if s.kind == "keep":
            rows, count = s.rows.cpu().numpy(), s.n_rows.cpu().numpy()
            for b, end in enumerate(ends):
                for i in range(int(count[b])):
                    (pa, ra), (pb, rb) = spot(b, s.context[b] + int(rows[end - s.new[b] + i])), spot(b, s.context[b] + 1 + i)
                    k[:, pb, rb], v[:, pb, rb] = k[:, pa, ra].clone(), v[:, pa, ra].clone()
            return k, v

        def turned(x, pos):                                            # pairs as complex numbers, times exp(i angle)
            half, y = s.inv_freq.numel(), x.double().clone()
            a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s.interleaved else (slice(0, half), slice(half, 2 * half))
            turn = torch.polar(torch.ones(len(pos), half, dtype=torch.float64, device=DEVICE), torch.outer(pos, s.inv_freq.double()))
            z = torch.complex(y[..., a].contiguous(), y[..., b].contiguous()) * turn[:, None]
            y[..., a], y[..., b] = z.real, z.imag
            return y

        q = torch.empty(s.q.shape, dtype=torch.float64, device=DEVICE)
        for b, end in enumerate(ends):
            span = slice(int(end) - s.new[b], int(end))
            rel = torch.arange(s.new[b], device=DEVICE) if s.rel_pos is None else s.rel_pos[span]
            pos = (s.context[b] + rel).double()
            q[span] = turned(s.q[span], pos)
            flat = torch.arange(s.context[b], s.context[b] + s.new[b], device=DEVICE)
            at = (s.table[b][flat // s.page].long(), flat % s.page)
            k[at], v[at] = turned(s.k[span], pos), s.v[span].double()
        return q, k, v
    out = torch.zeros(s.q.shape, dtype=torch.float64, device=DEVICE)
    hq = s.q.shape[1]
    for b, end in enumerate(ends):
        n, c = s.new[b], s.context[b]
        if n == 0:
            continue
        span = slice(int(end) - n, int(end))
        if s.kind == "prompt":
            k, v = s.k[span], s.v[span]
        else:
            pages = s.table[b, :-(-(c + n) // s.page)].long()
            k, v = (p[pages].flatten(0, 1)[:c + n] for p in (s.k_pages, s.v_pages))
        if s.mask is None:
            among = torch.ones(n, n, dtype=torch.bool, device=DEVICE).tril()
        else:
            places = torch.arange(n, device=DEVICE)
            among = ((s.mask[span][:, places // 64] >> (places % 64)) & 1).bool()
        hidden = torch.cat((torch.zeros(n, c, dtype=torch.bool, device=DEVICE), ~among), dim=1)
        for h in range(hq):
            g = h * k.shape[1] // hq
            x = (s.q[span, h].double() @ k[:, g].double().t()).mul_(s.scale).masked_fill_(hidden, -math.inf)
            norm = torch.logsumexp(x, dim=1, keepdim=True)
            out[span, h] = x.sub_(norm).exp_().nan_to_num_(nan=0.0) @ v[:, g].double()
    return out
