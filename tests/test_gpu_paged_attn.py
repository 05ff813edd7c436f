"""dyspec_paged_attn and dyspec_prompt_attn against the plain form in 64 bits (tests/serving.py: formulas and bounds)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from serving import HALF, Paged, attend_plain, compare, random_mask, rounds_weights, visible_rows

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    return m


# new, context, Hq, Hkv, d, dtype, page
SHAPES = [
    ((1,), (0,), 1, 1, 64, F32, 8),
    ((1,), (0,), 8, 8, 128, BF16, 16),
    ((1,), (1000,), 8, 8, 64, F32, 16),
    ((1,), (1023,), 32, 8, 128, BF16, 16),
    ((1,), (31,), 6, 2, 128, BF16, 8),
    ((1, 1, 1, 1, 1), (7, 64, 0, 513, 2050), 16, 2, 128, BF16, 32),
    ((1, 1, 0, 1, 1), (7, 64, 9, 513, 1), 4, 4, 64, BF16, 16),
    ((3, 0, 17, 1), (5, 8, 0, 300), 8, 2, 64, F32, 8),
    ((5,), (77,), 8, 8, 128, BF16, 16),
    ((33,), (95,), 8, 1, 128, BF16, 64),
    ((64,), (64,), 8, 8, 64, BF16, 8),
    ((200, 1, 70), (130, 600, 0), 8, 2, 128, BF16, 16),
    ((129, 31), (0, 1), 4, 4, 128, BF16, 16),
    ((513,), (300,), 16, 2, 128, BF16, 256),
    ((300, 7), (1111, 45), 12, 4, 64, BF16, 32),
    ((150,), (33,), 6, 3, 96, F32, 16),
    ((40, 2), (100, 3), 4, 2, 4, F32, 8),
    ((20,), (50,), 4, 2, 256, F32, 16),
    ((65,), (40,), 4, 1, 192, F32, 16),
    ((20, 1), (50, 200), 4, 2, 256, BF16, 16),
    ((70, 1), (31, 90), 4, 4, 80, BF16, 16),
    ((9,), (31,), 3, 1, 100, BF16, 8),
    ((1,), (260,), 20, 1, 36, BF16, 8),
]


@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_new_tokens_attend_to_the_pages(dy, shape, tree):
    new, context, Hq, Hkv, d, dtype, page = shape
    print("case", shape, tree, flush=True)
    mask = random_mask(new, 5)[0] if tree else None
    c = Paged(new, context, Hq, Hkv, d, dtype, page, 11, mask=mask, both_in_one=len(new) % 2 == 0)
    out = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev)
    torch.cuda.synchronize()
    c.check(out)


@pytest.mark.parametrize("dtype,d", [(F32, 64), (BF16, 128), (BF16, 64)])
@pytest.mark.parametrize("n", [40, 300])
def test_rows_without_a_key_are_zeros_and_bits_above_the_diagonal_do_not_count(dy, dtype, d, n):
    new, context = (n, n), (0, 50)
    mask = random_mask(new, 3)[0]
    mask[::3] = 0                                            # nothing, not even the row itself
    mask[1::3, 0] |= np.uint64(0xffffffff00000000)           # bits above the diagonal in rows below 32
    c = Paged(new, context, 8, 2, d, dtype, 16, 4, mask=mask)
    out = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev)
    c.check(out)
    assert not out[:n][::3].any()


@pytest.mark.parametrize("dtype,d,new,context", [(F32, 64, 40, 20), (BF16, 128, 40, 20), (BF16, 128, 300, 90), (BF16, 64, 3, 700), (BF16, 128, 200, 0), (BF16, 80, 30, 9)])
@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
def test_unseen_keys_may_hold_anything(dy, dtype, d, new, context, tree):
    """Infinities and NaN in later tokens, in keys that the mask hides, and in the rows behind the last token."""
    mask = random_mask((new, 5), 8)[0] if tree else None
    c = Paged((new, 5), (context, 30), 4, 2, d, dtype, 16, 21, mask=mask)
    for s, position, what, bad in [(0, context + new // 2, "v", math.nan), (0, context + new - 1, "k", math.inf), (0, context + new - 1, "v", math.inf),
                                   (0, context + new - 2, "v", -math.inf), (1, 33, "k", math.nan)]:
        p, r = c.place(s, position)
        getattr(c, what)[p, r, :, 1] = bad
    k_dev, v_dev = c.k.clone(), c.v.clone()
    for s, n in enumerate(c.new):                            # behind the last token
        p, r = c.place(s, c.context[s] + n - 1)
        k_dev[p, r + 1:] = math.nan
        v_dev[p, r + 1:] = math.inf
    c.cache.k.copy_(k_dev), c.cache.v.copy_(v_dev)
    out = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev).double().cpu().numpy()
    wh, seen_nan = rounds_weights(dtype, d), 0
    for s, n in enumerate(c.new):
        a = c.row0[s]
        k, v = c.rows(s)
        vis = visible_rows(n, c.context[s], None if mask is None else mask[a:a + n])
        bad_key = ~(np.isfinite(k).all((1, 2)) & np.isfinite(v).all((1, 2)))
        touched = (vis & bad_key[None]).any(1)
        clean_k, clean_v = np.where(bad_key[:, None, None], 0.0, k), np.where(bad_key[:, None, None], 0.0, v)
        want, bound = attend_plain(c.q[a:a + n].double().numpy(), clean_k, clean_v, vis & ~bad_key[None], c.scale, wh, HALF[dtype])
        compare(out[a:a + n][~touched], want[~touched], bound[~touched], f"sequence {s}")
        seen_nan += int((~np.isfinite(out[a:a + n][touched]).all((1, 2))).sum())
    assert seen_nan > 0                                      # rows that do see them come out as what they are


def test_every_walk_in_one_piece_without_a_workspace(dy):
    """The C call with no workspace, with one too small, and with one: within the bound each."""
    import ctypes
    c = Paged((1, 1), (3000, 900), 8, 2, 128, BF16, 16, 5)
    lib, cb = dy.load_library(), c.batch._c()
    need = lib.dyspec_paged_attn_workspace_bytes(ctypes.byref(cb), 8, 2, 128, dy.BF16)
    assert need > 16384
    stream = torch.cuda.current_stream().cuda_stream
    for nbytes in (0, 16384, need):
        ws = torch.zeros(max(nbytes, 16), dtype=torch.uint8, device="cuda")
        out = torch.full_like(c.q_dev, math.nan)
        st = lib.dyspec_paged_attn(c.q_dev.data_ptr(), c.cache._ref, ctypes.byref(cb), None, 8, 2, 128, dy.BF16, c.scale, out.data_ptr(),
                                   ws.data_ptr() if nbytes else None, nbytes, stream)
        torch.cuda.synchronize()
        assert st == 0
        c.check(out)
        assert not ws[:16384].any()


def test_scores_of_any_size(dy):
    """Large scores, far apart and all of one sign: the running maximum, not the size of the scores, decides."""
    for dtype, d in ((F32, 64), (BF16, 128)):
        for add in (0.0, 30.0, -30.0):
            c = Paged((1, 90), (500, 20), 4, 2, d, dtype, 16, 9)
            c.q = ((c.q.float() * 4 + add).to(dtype))
            c.k = (c.k.float() * 3 + abs(add) / 10).to(dtype)
            c.cache.k.copy_(c.k)
            out = dy.paged_attn(c.q.cuda(), c.batch, c.cache, c.scale)
            c.check(out)


PROMPTS = [
    ((1,), 4, 4, 64, F32), ((1,), 8, 1, 128, BF16), ((0, 2, 0), 8, 8, 128, BF16), ((17, 1, 64), 4, 2, 64, F32), ((65, 300), 8, 2, 64, F32),
    ((1, 517, 33, 129), 8, 8, 128, BF16), ((700, 64, 0, 63), 16, 2, 128, BF16), ((1025,), 4, 4, 128, BF16), ((260, 1, 90), 8, 4, 64, BF16),
    ((128, 127, 256), 8, 8, 64, BF16), ((40, 9), 4, 2, 96, BF16), ((50,), 3, 3, 20, F32), ((2000,), 2, 1, 128, BF16),
]


@pytest.mark.parametrize("fused", [False, True], ids=["dense", "fused"])
@pytest.mark.parametrize("shape", PROMPTS, ids=str)
def test_prompts_attend_to_themselves(dy, shape, fused):
    new, Hq, Hkv, d, dtype = shape
    print("case", shape, fused, flush=True)
    g = torch.Generator().manual_seed(7)
    qkv = torch.randn((sum(new), Hq + 2 * Hkv, d), generator=g).to(dtype)
    dev = qkv.cuda()
    q, k, v = dev.split([Hq, Hkv, Hkv], dim=1)
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    out = dy.prompt_attn(q, k, v, dy.Batch.from_sizes(new), 0.2)
    got, at = out.double().cpu().numpy(), 0
    for s, n in enumerate(new):
        if n:
            x = qkv[at:at + n].double().numpy()
            want, bound = attend_plain(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], visible_rows(n, 0), 0.2, rounds_weights(dtype, d), HALF[dtype])
            compare(got[at:at + n], want, bound, f"prompt {s}")
        at += n


@pytest.mark.parametrize("dtype,d,n", [(F32, 64, 100), (BF16, 128, 300), (BF16, 128, 40), (BF16, 64, 129)])
def test_a_prompts_later_tokens_may_hold_anything(dy, dtype, d, n):
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((n, 4, d), generator=g).to(dtype) for _ in range(3))
    at = 2 * n // 3
    v[at, 2, 5], k[at + 1, 1, 0] = math.inf, math.nan
    out = dy.prompt_attn(q.cuda(), k.cuda(), v.cuda(), dy.Batch.from_sizes([n]), 0.1).double().cpu().numpy()
    want, bound = attend_plain(*(x[:at].double().numpy() for x in (q, k, v)), visible_rows(at, 0), 0.1, rounds_weights(dtype, d), HALF[dtype])
    compare(out[:at], want, bound, "rows before")
    assert not np.isfinite(out[at, 2, 5]) and np.isfinite(out[at:, 3]).all() and np.isnan(out[at + 1:, 1]).all()


def test_rows_that_are_no_sixteen_bytes_apart(dy):
    """bf16 rows at 8-byte places and odd strides: another kernel, the same results."""
    g = torch.Generator().manual_seed(13)
    wide = torch.randn((150, 3 * 4 * 128 + 4), generator=g).to(BF16).cuda()
    q, k, v = (wide.as_strided((150, 4, 128), (1540, 128, 1), 4 + 512 * i) for i in range(3))
    out = dy.prompt_attn(q, k, v, dy.Batch.from_sizes([90, 60]), 0.1)
    same = dy.prompt_attn(q.contiguous(), k.contiguous(), v.contiguous(), dy.Batch.from_sizes([90, 60]), 0.1)
    for a, n in ((0, 90), (90, 60)):
        want, bound = attend_plain(*(x[a:a + n].double().cpu().numpy() for x in (q, k, v)), visible_rows(n, 0), 0.1, 2.0 ** -8, 2.0 ** -8)
        compare(out[a:a + n].double().cpu().numpy(), want, bound, "strided")
        compare(same[a:a + n].double().cpu().numpy(), want, bound, "dense")


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
def test_a_full_batch_of_sequences_of_every_kind(dy, dtype, d, tree):
    """64 sequences: without a new token, with one, with a few, with hundreds; without a context, with thousands."""
    rng = np.random.default_rng(17)
    new = [int(x) for x in rng.choice([0, 1, 1, 1, 2, 7, 33, 150, 260], 64)]
    context = [int(x) for x in rng.choice([0, 1, 15, 64, 200, 1000, 2500], 64)]
    c = Paged(new, context, 4, 2, d, dtype, 16, 23, mask=random_mask(new, 6)[0] if tree else None)
    out = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev)
    c.check(out)


@pytest.mark.parametrize("dtype,new,context", [(BF16, (1,), (150_001,)), (BF16, (70,), (60_003,)), (BF16, (300, 1), (33_000, 90_000)), (F32, (1, 3), (50_000, 7))])
def test_long_contexts(dy, dtype, new, context):
    c = Paged(new, context, 2, 1, 64 if dtype is F32 else 128, dtype, 256, 29)
    c.check(dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale))


@pytest.mark.parametrize("new,context,Hq,Hkv,d", [((500, 1, 2), (400, 2000, 1500), 64, 8, 128), ((1, 1000), (3000, 100), 32, 32, 64),
                                                  ((544,), (1000,), 64, 8, 128)], ids=str)
def test_whole_walks_beside_walks_in_parts(dy, new, context, Hq, Hkv, d):
    """More row blocks than CUs: single tokens' long walks are cut beside them, or what is left after a round of workgroups."""
    c = Paged(new, context, Hq, Hkv, d, BF16, 16, 37, mask=random_mask(new, 8)[0])
    assert dy.load_library().dyspec_paged_attn_workspace_bytes(c.batch._c(), Hq, Hkv, d, dy.BF16) > 0
    c.check(dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev))


def test_a_long_prompt(dy):
    """20001 tokens: rows from all over it against the plain form."""
    n, g = 20001, torch.Generator().manual_seed(31)
    q, k, v = (torch.randn((n, 2, 128), generator=g).to(BF16) for _ in range(3))
    out = dy.prompt_attn(q.cuda(), k.cuda(), v.cuda(), dy.Batch.from_sizes([n]), 0.1).double().cpu().numpy()
    rows = np.unique(np.concatenate([np.arange(70), np.random.default_rng(1).integers(0, n, 60), np.arange(n - 70, n)]))
    seen = np.arange(n)[None] <= rows[:, None]
    want, bound = attend_plain(q[rows].double().numpy(), k.double().numpy(), v.double().numpy(), seen, 0.1, 2.0 ** -8, 2.0 ** -8)
    compare(out[rows], want, bound, "rows")


@pytest.mark.parametrize("dtype,d,new", [(BF16, 128, 300), (BF16, 128, 20), (BF16, 64, 200), (F32, 64, 100)])
def test_a_row_that_is_no_number_leaves_the_others_alone(dy, dtype, d, new):
    c = Paged((new, 3), (100, 40), 4, 2, d, dtype, 16, 41)
    c.q[new // 2, 1, 7] = math.nan
    c.q[new // 3, 2] = math.inf
    out = dy.paged_attn(c.q.cuda(), c.batch, c.cache, c.scale)
    assert torch.isnan(out[new // 2, 1]).all() and torch.isnan(out[new // 3, 2]).all()
    c.q[new // 2, 1], c.q[new // 3, 2] = 0, 0
    out[new // 2, 1] = dy.paged_attn(c.q.cuda(), c.batch, c.cache, c.scale)[new // 2, 1]
    out[new // 3, 2] = dy.paged_attn(c.q.cuda(), c.batch, c.cache, c.scale)[new // 3, 2]
    c.check(out)


@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
@pytest.mark.parametrize("dtype,d,new,context", [(BF16, 128, 300, 200), (BF16, 128, 20, 700), (BF16, 64, 1, 5000), (F32, 64, 100, 50), (BF16, 80, 9, 40)])
def test_what_every_row_sees_stays_in_its_dims(dy, dtype, d, new, context, tree):
    """A NaN and an infinity in V, and a NaN in K, of a context: in the rows' results where the formula has them, nowhere else."""
    c = Paged((new, 2, 40), (context, context, 33), 4, 2, d, dtype, 16, 43, mask=random_mask((new, 2, 40), 3)[0] if tree else None)
    p, r = c.place(0, 5)
    c.v[p, r, 0, 3], c.v[p, r, 1, d - 1] = 0, 0              # what the other dims are held against
    v_dev = c.v.clone()
    v_dev[p, r, 0, 3], v_dev[p, r, 1, d - 1] = math.nan, math.inf
    p, r = c.place(1, context - 1)
    c.k[p, r, 1, 2] = math.nan
    c.cache.k.copy_(c.k), c.cache.v.copy_(v_dev)
    out = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev)
    first, second = out[:new], out[new:new + 2]
    assert torch.isnan(first[:, :2, 3]).all() and (first[:, 2:, d - 1] == math.inf).all()
    assert torch.isnan(second[:, 2:]).all() and torch.isfinite(second[:, :2]).all()
    c.cache.v.copy_(c.v)
    clean = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev)
    first[:, :2, 3], first[:, 2:, d - 1] = clean[:new, :2, 3], clean[:new, 2:, d - 1]
    c.check(out, only=(0, 2))
