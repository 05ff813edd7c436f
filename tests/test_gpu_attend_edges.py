"""Attention over pages and of prompts at the edges of its numbers: a score far above all before it, infinities and NaN that some rows see
and others do not, queries that are no numbers, a scale of nearly nothing.  Every kernel, whole and in parts (test_gpu_attend_forms.py),
against the plain form in 64 bits (tests/serving.py: formulas and bounds)."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from serving import HALF, Paged, attend_plain, compare, random_mask, visible_rows
from test_gpu_attend_forms import FORMS, check, in_form, weight_half, with_forms, workspace

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    return m


def prompt_in_form(dy, form, q, k, v, lengths, scale):
    lib, ws, out = dy.load_library(), workspace(), torch.full_like(q, 7.0)
    b = dy.Batch.from_sizes(lengths)
    f, p, I = (ctypes.c_int32 * 3)(*form), lambda t: ctypes.c_void_p(t.data_ptr()), ctypes.c_int64
    Hq, Hkv, d = q.shape[1], k.shape[1], q.shape[2]
    st = lib.dyspec_prompt_attn_in_form(f, p(q), I(Hq * d), p(k), I(Hkv * d), p(v), I(Hkv * d), ctypes.byref(b._c()), Hq, Hkv, d, dy.F32 if q.dtype is F32 else dy.BF16,
                                        ctypes.c_float(scale), p(out), p(ws), ctypes.c_size_t(ws.numel()), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert st == 0 and not ws[:16384].any()
    return out


# ---- a score far above all before it

def one_direction(q, k, at, nats, scale):
    """Every query shares a direction that key `at` alone has: its score lies about `nats` above the others."""
    q[..., 0], k[..., 0] = 40.0, 0.0
    k[at, :, 0] = nats / (40.0 * scale)


@pytest.mark.parametrize("nats", [100, 300])
@pytest.mark.parametrize("seen_by", ["all", "some"])
@pytest.mark.parametrize("form,dtype,d", with_forms((BF16, 128), (BF16, 64), (F32, 64)), ids=str)
def test_a_key_far_above_those_before_it(dy, form, dtype, d, seen_by, nats):
    """What was summed before it no longer counts in the rows that see it; the others keep it.  The key lies behind the first of
    every walk, whole or in parts: place 356 of the context, or a new token from the 36th to the 60th."""
    print("form", form, dtype, d, seen_by, nats, flush=True)
    n, context = 90, 500
    mask = random_mask((n,), 12)[0]
    seen = visible_rows(n, context, mask)
    at = 356 if seen_by == "all" else context + 35 + int(seen[:, context + 35:context + 60].sum(0).argmax())
    assert seen[:, at].all() if seen_by == "all" else 3 < seen[:, at].sum() < n - 40
    c = Paged((n,), (context,), 4, 2, d, dtype, 16, 35, mask=mask)
    c.q[..., 0], c.k[..., 0] = 40.0, 0.0
    p, r = c.place(0, at)
    c.k[p, r, :, 0] = nats / (40.0 * c.scale)
    c.q_dev.copy_(c.q), c.cache.k.copy_(c.k)
    st, out = in_form(dy, form, c)
    assert st == 0
    check(c, out, form)


@pytest.mark.parametrize("form,dtype,Hq,Hkv,d", with_forms((BF16, 4, 1, 128), (BF16, 2, 2, 64), (F32, 2, 1, 64)), ids=str)
def test_a_prompts_key_far_above_those_before_it(dy, form, dtype, Hq, Hkv, d):
    """Keys 100 of each prompt: the rows before them sum others, later rows those and, 150 nats above, these."""
    print("form", form, dtype, Hq, Hkv, d, flush=True)
    lengths, g = (450, 64, 129, 230), torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((sum(lengths), h, d), generator=g).to(dtype) for h in (Hq, Hkv, Hkv))
    one_direction(q, k, [100, 614, 743], 150, 0.1)                # (row 614: the third prompt's)
    out, at = prompt_in_form(dy, form, q.cuda(), k.cuda(), v.cuda(), lengths, 0.1).double().cpu().numpy(), 0
    for s, n in enumerate(lengths):
        want, bound = attend_plain(*(t[at:at + n].double().numpy() for t in (q, k, v)), visible_rows(n, 0), 0.1, weight_half(form, dtype), HALF[dtype])
        compare(out[at:at + n], want, bound, f"prompt {s}")
        at += n


# ---- infinities that the last token sees

FORMS_OF_EACH = with_forms((BF16, 128), (BF16, 64), (F32, 64), (F32, 192)) + [(form, BF16, 80) for form in FORMS if form[0] >= 4]


@pytest.mark.parametrize("form,dtype,d", FORMS_OF_EACH, ids=str)
def test_an_infinity_in_the_newest_value(dy, form, dtype, d):
    """One token each, causal: its own value's infinities come out as they are whether its place ends a block of keys or not, a second
    sequence (which has none) as if they were not there."""
    for context in (0, 30, 31, 63, 99, 127, 200, 511):
        print("form", form, dtype, d, context, flush=True)
        c = Paged((1, 1), (context, 77), 4, 2, d, dtype, 16, 45)
        p, r = c.place(0, context)
        c.v[p, r, 0, 3], c.v[p, r, 1, d - 1] = 0, 0               # what the other dims are held against
        v = c.v.clone()
        v[p, r, 0, 3], v[p, r, 1, d - 1] = math.inf, -math.inf
        c.cache.v.copy_(v)
        st, out = in_form(dy, form, c)
        assert st == 0
        assert (out[0, :2, 3] == math.inf).all() and (out[0, 2:, d - 1] == -math.inf).all()
        c.cache.v.copy_(c.v)
        st, clean = in_form(dy, form, c)
        out[0, :2, 3], out[0, 2:, d - 1] = clean[0, :2, 3], clean[0, 2:, d - 1]
        check(c, out, form)


@pytest.mark.parametrize("form,dtype,d", with_forms((BF16, 128), (BF16, 64), (F32, 64)), ids=str)
def test_an_infinity_in_a_prompts_last_value(dy, form, dtype, d):
    """The same of a prompt, whose last row block may hold the last token alone (65 tokens of two heads)."""
    for n in (1, 33, 64, 65, 129, 450):
        print("form", form, dtype, d, n, flush=True)
        g = torch.Generator().manual_seed(3)
        q, k, v = (torch.randn((n, h, d), generator=g).to(dtype) for h in (4, 2, 2))
        v[n - 1, 0, 3], v[n - 1, 1, d - 1] = 0, 0
        bad = v.clone()
        bad[n - 1, 0, 3], bad[n - 1, 1, d - 1] = math.inf, -math.inf
        out = prompt_in_form(dy, form, q.cuda(), k.cuda(), bad.cuda(), (n,), 0.1).double().cpu().numpy()
        assert (out[n - 1, :2, 3] == math.inf).all() and (out[n - 1, 2:, d - 1] == -math.inf).all()
        want, bound = attend_plain(*(x.double().numpy() for x in (q, k, v)), visible_rows(n, 0), 0.1, weight_half(form, dtype), HALF[dtype])
        out[n - 1, :2, 3], out[n - 1, 2:, d - 1] = want[n - 1, :2, 3], want[n - 1, 2:, d - 1]
        compare(out, want, bound, "the rest")


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64), (BF16, 80)])
def test_an_infinity_in_the_newest_value_of_each_of_many(dy, dtype, d):
    """As the library chooses the kernels: 20 sequences of one token, contexts of any size."""
    context = [int(x) for x in np.random.default_rng(8).integers(0, 900, 20)]
    c = Paged([1] * 20, context, 4, 2, d, dtype, 16, 47)
    v = c.v.clone()
    for s in range(20):
        p, r = c.place(s, context[s])
        c.v[p, r, 1, 5], v[p, r, 1, 5] = 0, math.inf
    c.cache.v.copy_(v)
    out = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale)
    assert (out[:, 2:, 5] == math.inf).all()
    c.cache.v.copy_(c.v)
    out[:, 2:, 5] = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale)[:, 2:, 5]
    c.check(out)


# ---- queries that are no numbers

@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("form,dtype,d", with_forms((BF16, 128), (BF16, 64), (F32, 64)), ids=str)
@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
def test_a_query_that_is_no_number_is_no_matter_to_other_rows(dy, form, dtype, d, tree, bad):
    """Not in one bit: rows are taken 32 at a time (those beside it may go by another reference), and no others are done again."""
    print("form", form, dtype, d, tree, bad, flush=True)
    n, context = 90, 700
    c = Paged((n,), (context,), 4, 2, d, dtype, 16, 51, mask=random_mask((n,), 12)[0] if tree else None)
    st, clean = in_form(dy, form, c)
    assert st == 0
    c.q_dev[20, 1, 7], c.q_dev[50, 0, 3] = bad, bad               # rows 41 and 100 of the first KV head
    st, out = in_form(dy, form, c)
    assert st == 0 and torch.isnan(out[20, 1]).all() and torch.isnan(out[50, 0]).all()
    rows = (torch.arange(n)[:, None] * 2 + torch.arange(4)[None] % 2) // 32
    others = (torch.arange(4)[None] >= 2) | ((rows != 41 // 32) & (rows != 100 // 32))
    whole = torch.int16 if dtype is BF16 else torch.int32
    assert others.sum() > 200 and torch.equal(out.cpu()[others].view(whole), clean.cpu()[others].view(whole))


# ---- tokens that overflowed

@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
@pytest.mark.parametrize("form,dtype,d", FORMS_OF_EACH + [(form, BF16, 256) for form in FORMS if form[0] >= 4], ids=str)
def test_every_infinity_and_nan_stays_with_the_rows_that_see_it(dy, form, dtype, d, tree):
    """Six values hold something that is no number, some in the context, some in new tokens: a dim of a row is what the formula gives
    for the keys that the row sees, and all other dims and rows are as if there were none."""
    print("form", form, dtype, d, tree, flush=True)
    n, context = 75, 341
    mask = random_mask((n,), 12)[0] if tree else None
    c = Paged((n,), (context,), 4, 2, d, dtype, 16, 53, mask=mask)
    odd = [(17, 0, 1, math.inf), (context + 3, 0, d - 1, math.nan), (context + 18, 0, 1, -math.inf), (context + 18, 1, 2, math.inf),
           (context + 40, 1, d // 2, math.inf), (context + n - 1, 0, 3, math.nan)]
    for at, h, dim, _ in odd:                                    # what the rest is held against
        p, r = c.place(0, at)
        c.v[p, r, h, dim] = 0
    v = c.v.clone()
    for at, h, dim, x in odd:
        p, r = c.place(0, at)
        v[p, r, h, dim] = x
    c.cache.v.copy_(v)
    st, out = in_form(dy, form, c)
    assert st == 0
    got, seen = out.double().cpu().numpy(), visible_rows(n, context, mask)
    add = np.zeros((n, 4, d))
    for at, h, dim, x in odd:
        with np.errstate(invalid="ignore"):                      # inf - inf is a NaN, as in the sum
            add[:, 2 * h:2 * h + 2, dim] += np.where(seen[:, at], x, 0.0)[:, None]
    assert np.isnan(add).any() and np.isinf(add).any()
    assert np.array_equal(np.isnan(got), np.isnan(add)) and np.array_equal(np.where(np.isinf(got), got, 0), np.where(np.isinf(add), add, 0))
    want, bound = attend_plain(c.q.double().numpy(), *c.rows(0), seen, c.scale, weight_half(form, dtype), HALF[dtype])
    fine = np.isfinite(add)
    compare(got[fine], want[fine], bound[fine], "the rest")


def test_one_token_that_overflowed_does_not_hold_up_the_call(dy):
    """The rows beside it are done again, once more over their keys, not a row and a key at a time: 2.0 ms in place of 0.09 for a tree,
    2.9 in place of 1.0 for a prompt (it was 60, and 98)."""
    def time_of(call):
        best, a, b = math.inf, torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for _ in range(4):
            a.record(), call(), b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    c = Paged((512,), (4096,), 64, 8, 128, BF16, 16, 3, mask=random_mask((512,), 3)[0])
    tree = lambda: dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev)
    clean = time_of(tree)
    p, r = c.place(0, 4096 + 300)
    c.cache.v[p, r, :, 3] = math.nan
    assert time_of(tree) < 100 * clean
    q, k, v = (torch.randn((8192, h, 128), device="cuda").to(BF16) for h in (64, 8, 8))
    prompt = lambda: dy.prompt_attn(q, k, v, dy.Batch.from_sizes([8192]), 0.1)
    clean = time_of(prompt)
    v[8190, :, 3] = math.nan
    assert time_of(prompt) < 15 * clean


@pytest.mark.parametrize("form,dtype,d", with_forms((BF16, 128), (BF16, 64), (F32, 64)), ids=str)
def test_a_nan_that_all_rows_see_is_not_looked_for_again(dy, form, dtype, d):
    """One token whose own value has a NaN, its keys whole blocks: the other dims have the same bits as without it."""
    for context in (63, 127, 511):
        print("form", form, dtype, d, context, flush=True)
        c = Paged((1,), (context,), 4, 2, d, dtype, 16, 57)
        p, r = c.place(0, context)
        c.cache.v[p, r, :, 3] = 0
        st, clean = in_form(dy, form, c)
        c.cache.v[p, r, :, 3] = math.nan
        st2, out = in_form(dy, form, c)
        assert st == st2 == 0 and torch.isnan(out[0, :, 3]).all()
        whole = torch.int16 if dtype is BF16 else torch.int32
        rest = [x for x in range(d) if x != 3]
        assert torch.equal(out[..., rest].contiguous().view(whole), clean[..., rest].contiguous().view(whole))


@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
@pytest.mark.parametrize("form,dtype,d", with_forms((BF16, 128), (BF16, 64), (F32, 64)), ids=str)
def test_a_scale_of_nearly_nothing(dy, form, dtype, d, tree):
    """All weights alike, beside a query that is no number: no running reference is ever passed by much."""
    print("form", form, dtype, d, tree, flush=True)
    n, context = 90, 130
    c = Paged((n,), (context,), 4, 2, d, dtype, 16, 59, mask=random_mask((n,), 12)[0] if tree else None)
    c.scale = 1e-38
    c.q_dev[20, 1, 7] = math.nan
    st, out = in_form(dy, form, c)
    assert st == 0 and torch.isnan(out[20, 1]).all()
    c.q_dev[20, 1, 7] = 0
    out[20, 1] = in_form(dy, form, c)[1][20, 1]
    check(c, out, form)
