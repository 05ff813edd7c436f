"""dyspec_kv_append and dyspec_kv_keep against the plain forms in 64 bits (tests/serving.py)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from serving import Paged, compare, page_table, random_mask, rotate_plain

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    return m


def frequencies(n, base=10000.0):
    return (base ** (-np.arange(n) / max(n, 1))).astype(np.float32)


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype is BF16 else torch.int32)


# new, context, Hq, Hkv, d, dtype, page, n_freq, interleaved
APPENDS = [
    ((1,), (0,), 4, 4, 64, F32, 8, 32, False),
    ((1, 1, 1), (7, 8, 500), 8, 2, 128, BF16, 16, 64, False),
    ((5, 0, 33), (30, 4, 0), 8, 8, 128, BF16, 16, 64, True),
    ((300, 1), (1, 900), 4, 2, 64, BF16, 32, 16, False),
    ((300, 1), (1, 900), 4, 2, 64, F32, 32, 16, True),
    ((700, 600), (3, 0), 3, 1, 96, BF16, 64, 48, False),
    ((9, 40), (15, 16), 6, 2, 96, BF16, 16, 12, False),         # frequencies that no 16-byte piece holds
    ((9, 40), (15, 16), 6, 2, 96, F32, 16, 5, True),
    ((20,), (0,), 4, 2, 100, BF16, 8, 50, False),
    ((20,), (0,), 4, 2, 100, BF16, 8, 50, True),
    ((20,), (11,), 4, 2, 4, F32, 8, 1, False),
    ((12,), (11,), 5, 5, 256, F32, 8, 128, False),
    ((12,), (11,), 4, 2, 128, BF16, 8, 0, False),               # nothing rotated: a copy
]


@pytest.mark.parametrize("strided", [False, True], ids=["dense", "fused"])
@pytest.mark.parametrize("case", APPENDS, ids=str)
def test_new_tokens_go_into_the_pages(dy, case, strided):
    new, context, Hq, Hkv, d, dtype, page, n_freq, interleaved = case
    print("case", case, strided, flush=True)
    c = Paged(new, context, Hq, Hkv, d, dtype, page, 3, both_in_one=strided)
    g = torch.Generator().manual_seed(17)
    qkv = torch.randn((c.total, Hq + 2 * Hkv, d), generator=g).to(dtype)
    q, k, v = qkv.cuda().split([Hq, Hkv, Hkv], dim=1)
    if not strided:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    rel = np.random.default_rng(2).integers(0, 50, c.total).astype(np.int32) if strided else np.concatenate([np.arange(n) for n in new]).astype(np.int32)
    freq = frequencies(n_freq)
    before_k, before_v = c.cache.k.clone(), c.cache.v.clone()
    k_out = torch.empty((c.total, Hkv, d), dtype=dtype, device="cuda")
    out = dy.kv_append(k, v, c.batch, c.cache, q=q, rel_pos=torch.from_numpy(rel).cuda() if strided else None,
                       inv_freq=torch.from_numpy(freq).cuda() if n_freq else None, interleaved=interleaved, k_out=k_out)
    position = np.repeat(np.asarray(context), new) + rel
    want_q, bound_q = rotate_plain(qkv[:, :Hq], position, freq, interleaved)
    want_k, bound_k = rotate_plain(qkv[:, Hq:Hq + Hkv], position, freq, interleaved)
    compare(out.double().cpu().numpy(), want_q, bound_q, "queries")
    compare(k_out.double().cpu().numpy(), want_k, bound_k, "keys")
    at = [c.place(s, context[s] + j) for s, n in enumerate(new) for j in range(n)]
    pages, rows = torch.tensor([p for p, _ in at]), torch.tensor([r for _, r in at])
    assert torch.equal(bits(c.cache.k.cpu()[pages, rows]), bits(k_out.cpu()))
    assert torch.equal(bits(c.cache.v.cpu()[pages, rows]), bits(qkv[:, Hq + Hkv:]))
    # every other row of the pool is as it was
    before_k[pages, rows], before_v[pages, rows] = c.cache.k[pages, rows], c.cache.v[pages, rows]
    assert torch.equal(bits(before_k), bits(c.cache.k)) and torch.equal(bits(before_v), bits(c.cache.v))


def test_in_place_and_without_queries(dy):
    c = Paged((40, 3), (5, 90), 4, 2, 128, BF16, 16, 6)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((43, h, 128), generator=g).to(BF16).cuda() for h in (4, 2, 2))
    freq = torch.from_numpy(frequencies(64)).cuda()
    apart = torch.empty_like(k)
    want = dy.kv_append(k, v, c.batch, c.cache, q=q, inv_freq=freq, k_out=apart)
    q2, k2 = q.clone(), k.clone()
    assert dy.kv_append(k2, v, c.batch, c.cache, q=q2, inv_freq=freq, out=q2, k_out=k2) is q2
    assert torch.equal(bits(q2), bits(want)) and torch.equal(bits(k2), bits(apart))
    c.cache.k.zero_()
    assert dy.kv_append(k, v, c.batch, c.cache, inv_freq=freq) is None
    p, r = c.place(1, 92)
    assert torch.equal(bits(c.cache.k[p, r]), bits(apart[42]))


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_keep_their_angle(dy, interleaved):
    """Position 10^6 and beyond: the angle of the first pair is a million radians, its sine still right to fp32."""
    context, d, page = 1_048_000, 64, 65536
    table = torch.zeros((1, 17), dtype=torch.int32, device="cuda")        # the far pages, all one
    k_pages = torch.zeros((1, page, 1, d), device="cuda")
    cache = dy.PagedCache(k_pages, torch.zeros_like(k_pages), table)
    x = torch.randn((3, 1, d), generator=torch.Generator().manual_seed(2))
    freq = frequencies(32)
    out = dy.kv_append(x.cuda(), x.cuda(), dy.Batch.from_sizes([3], [context]), cache, q=x.cuda(), inv_freq=torch.from_numpy(freq).cuda(), interleaved=interleaved)
    want, bound = rotate_plain(x, context + np.arange(3), freq, interleaved)
    compare(out.double().cpu().numpy(), want, bound, "far")


def test_a_page_outside_the_pool_is_not_written(dy):
    c = Paged((20,), (10,), 2, 2, 64, F32, 16, 6)
    before_k, before_v = c.cache.k.clone(), c.cache.v.clone()
    for bad in (-1, int(c.cache.k.shape[0]), 2 ** 30, -2 ** 31):
        table = c.cache.page_table.clone()
        table[0, 1] = bad
        x = torch.randn((20, 2, 64), device="cuda")
        dy.kv_append(x, x, c.batch, dy.PagedCache(c.cache.k, c.cache.v, table))
        p0 = int(c.table[0, 0])
        assert torch.equal(c.cache.k[p0, 10:], x[:6])
        before_k[p0, 10:], before_v[p0, 10:] = x[:6], x[:6]
        assert torch.equal(before_k, c.cache.k) and torch.equal(before_v, c.cache.v)
        dy.kv_keep(dy.PagedCache(c.cache.k, c.cache.v, table), c.batch, torch.full((20,), 15, dtype=torch.int32, device="cuda"),
                   torch.tensor([1], dtype=torch.int32, device="cuda"))
        assert torch.equal(before_k, c.cache.k)                            # row 25 lies in the bad page: nothing moves


def test_places_behind_four_gigabytes(dy):
    """A pool whose last pages lie beyond 2^32 bytes (and 2^31 elements)."""
    page, Hkv, d = 64, 8, 128
    n_pages = 2 ** 31 // (page * Hkv * d) + 700
    k, v = (torch.empty((n_pages, page, Hkv, d), dtype=BF16, device="cuda") for _ in range(2))
    c = Paged((70, 1), (200, 130), 16, 8, 128, BF16, page, 8)
    far = torch.from_numpy(c.table).cuda()
    far = torch.where(far >= 0, n_pages - 1 - far, far).int()
    used = sorted(set(int(x) for x in c.table.ravel() if x >= 0))
    for p in used:
        k[n_pages - 1 - p].copy_(c.k[p]), v[n_pages - 1 - p].copy_(c.v[p])
    cache = dy.PagedCache(k, v, far)
    out = dy.paged_attn(c.q_dev, c.batch, cache, c.scale)
    c.check(out)
    x = torch.randn((71, 8, 128), device="cuda").to(BF16)
    dy.kv_append(x, x, c.batch, cache)
    p, r = c.place(0, 269)
    assert torch.equal(k[n_pages - 1 - p, r], x[69]) and torch.equal(v[n_pages - 1 - p, r], x[69])
    dy.kv_keep(cache, c.batch, torch.full((71,), 69, dtype=torch.int32, device="cuda"), torch.tensor([1, 0], dtype=torch.int32, device="cuda"))
    p, r = c.place(0, 201)
    assert torch.equal(k[n_pages - 1 - p, r], x[69])


# ---- keep

def keep_plain(pages, c, accepted, counts):
    want = pages.clone()
    at = 0
    for s, n in enumerate(c.new):
        for i in range(counts[s]):
            a = accepted[at + i]
            if i < a < n and i < n - 1:
                p, r = c.place(s, c.context[s] + int(a))
                p2, r2 = c.place(s, c.context[s] + 1 + i)
                want[..., p2, r2, :, :] = pages[..., p, r, :, :]
        at += n
    return want


@pytest.mark.parametrize("dtype,Hkv,d", [(F32, 2, 64), (BF16, 8, 128), (BF16, 1, 4), (BF16, 40, 128), (BF16, 3, 20)])
@pytest.mark.parametrize("layers", [0, 1, 5])
@pytest.mark.parametrize("apart", [False, True], ids=["dense", "in_turns"])
def test_the_accepted_path_moves_up(dy, dtype, Hkv, d, layers, apart):
    new, context = (40, 0, 7, 1, 200, 2), (3, 5, 0, 16, 100, 31)
    c = Paged(new, context, 2 * Hkv, Hkv, d, dtype, 16, 3, layers=layers, both_in_one=apart)
    rng = np.random.default_rng(4)
    accepted = np.full(c.total, -5, np.int32)
    counts = []
    at = 0
    for n in new:
        m = int(rng.integers(0, min(n, 30))) if n > 1 else 0
        counts.append(m)
        accepted[at:at + m] = np.sort(rng.choice(np.arange(1, n), m, replace=False)) if m else []
        at += n
    counts[4] = max(counts[4], 19)
    accepted[c.row0[4]:c.row0[4] + counts[4]] = np.sort(rng.choice(np.arange(1, 60), counts[4], replace=False))     # rows that make way for each other
    dy.kv_keep(c.cache, c.batch, torch.from_numpy(accepted).cuda(), torch.tensor(counts, dtype=torch.int32, device="cuda"))
    assert torch.equal(bits(c.cache.k.cpu()), bits(keep_plain(c.k, c, accepted, counts)))
    assert torch.equal(bits(c.cache.v.cpu()), bits(keep_plain(c.v, c, accepted, counts)))


def test_lists_that_no_verification_writes(dy):
    """Counts past the tree or below zero, rows outside it or before their place, one row twice: what is not a move is none."""
    new, context = (20, 6, 9, 5), (0, 3, 8, 1)
    c = Paged(new, context, 2, 2, 64, F32, 8, 3)
    accepted = np.zeros(c.total, np.int32)
    accepted[:4] = [7, 7, 0, 25]
    accepted[20:26] = [5, 5, 5, 5, 5, 5]
    accepted[26:29] = [-3, 2 ** 31 - 1, 8]
    counts = [4, 60, 3, -2]
    dy.kv_keep(c.cache, c.batch, torch.from_numpy(accepted).cuda(), torch.tensor(counts, dtype=torch.int32, device="cuda"))
    want = keep_plain(c.k, c, accepted, [4, 5, 3, 0])
    assert torch.equal(c.cache.k.cpu(), want)
