"""Every kernel behind dyspec_paged_attn and dyspec_prompt_attn, with walks in one piece, in parts and some of each, on cases whose sizes would
choose another: masks, empty rows, unseen infinities and NaN, ragged ends (tests/serving.py: formulas and bounds)."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from serving import HALF, Paged, attend_plain, compare, random_mask, visible_rows

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
FORMS = [(k, share, whole) for k in range(6) for share, whole in ((0, 0), (128, 0), (384, 0), (128, 3))]


def with_forms(*shapes):
    """Every form a shape (its type first) has: kernels 0 .. 3 are for bf16."""
    return [(form, *shape) for shape in shapes for form in FORMS if shape[0] is BF16 or form[0] >= 4]


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    return m


def weight_half(form, dtype):
    return HALF[BF16] if form[0] < 4 else 0.0                # kernels 4 and 5 keep weights in fp32


def workspace():
    return torch.zeros(96 << 20, dtype=torch.uint8, device="cuda")


def in_form(dy, form, c):
    lib, ws, out = dy.load_library(), workspace(), torch.full_like(c.q_dev, 7.0)
    f = (ctypes.c_int32 * 3)(*form)
    mask = None if c.mask_dev is None else ctypes.c_void_p(c.mask_dev.data_ptr())
    p = lambda t: ctypes.c_void_p(t.data_ptr())
    st = lib.dyspec_paged_attn_in_form(f, p(c.q_dev), c.cache._ref, ctypes.byref(c.batch._c()), mask, c.Hq, c.Hkv, c.d, c.cache._code,
                                       ctypes.c_float(c.scale), p(out), p(ws), ctypes.c_size_t(ws.numel()),
                                       ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert not ws[:16384].any(), "the counters are zero again"
    return st, out


def check(c, out, form):
    got = out.double().cpu().numpy()
    for s, n in enumerate(c.new):
        if n:
            a = c.row0[s]
            k, v = c.rows(s)
            want, bound = attend_plain(c.q[a:a + n].double().numpy(), k, v, visible_rows(n, c.context[s], None if c.mask is None else c.mask[a:a + n]), c.scale,
                                       weight_half(form, c.dtype), HALF[c.dtype])
            compare(got[a:a + n], want, bound, f"sequence {s}")


@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
@pytest.mark.parametrize("form,dtype,Hq,Hkv,d,page", with_forms((BF16, 8, 2, 128, 16), (BF16, 3, 3, 64, 8), (F32, 8, 2, 64, 32), (F32, 3, 1, 96, 8)), ids=str)
def test_paged(dy, form, dtype, Hq, Hkv, d, page, tree):
    print("form", form, dtype, Hq, Hkv, d, page, tree, flush=True)
    new, context = (1, 0, 37, 200, 5, 64), (700, 30, 0, 129, 1023, 64)
    mask = None
    if tree:
        mask = random_mask(new, 9)[0]
        mask[10:20] = 0
    c = Paged(new, context, Hq, Hkv, d, dtype, page, 19, mask=mask, both_in_one=tree)
    st, out = in_form(dy, form, c)
    assert st == 0
    check(c, out, form)


@pytest.mark.parametrize("form,dtype,d", with_forms((BF16, 128), (BF16, 64), (F32, 64)), ids=str)
def test_unseen_keys_may_hold_anything(dy, form, dtype, d):
    print("form", form, dtype, d, flush=True)
    n, context = 90, 500
    mask = random_mask((n,), 12)[0]
    c = Paged((n,), (context,), 4, 2, d, dtype, 16, 33, mask=mask)
    at = n // 2
    p, r = c.place(0, context + at)
    c.v[p, r, 0, 3], c.v[p, r, 1, d - 1], c.k[p, r, 1, 0] = math.inf, math.nan, math.nan
    c.cache.k.copy_(c.k), c.cache.v.copy_(c.v)
    st, out = in_form(dy, form, c)
    assert st == 0
    seen = visible_rows(n, context, mask)
    free = ~seen[:, context + at]
    k, v = c.rows(0)
    k[context + at], v[context + at] = 0, 0
    want, bound = attend_plain(c.q.double().numpy(), k, v, seen, c.scale, weight_half(form, dtype), HALF[dtype])
    got = out.double().cpu().numpy()
    compare(got[free], want[free], bound[free], "rows that do not see it")
    assert free.sum() > n // 2 and not np.isfinite(got[at, 0, 3]) and not np.isfinite(got[at, 2]).any()


@pytest.mark.parametrize("form,dtype,Hq,Hkv,d", with_forms((BF16, 4, 1, 128), (BF16, 2, 2, 64), (F32, 2, 1, 64)), ids=str)
def test_prompts(dy, form, dtype, Hq, Hkv, d):
    print("form", form, dtype, Hq, Hkv, d, flush=True)
    new = (1, 450, 0, 64, 129, 31)
    g = torch.Generator().manual_seed(3)
    host = [torch.randn((sum(new), h, d), generator=g).to(dtype) for h in (Hq, Hkv, Hkv)]
    q, k, v = (t.cuda() for t in host)
    lib, ws, out = dy.load_library(), workspace(), torch.full_like(q, 7.0)
    b = dy.Batch.from_sizes(new)
    f, p = (ctypes.c_int32 * 3)(*form), lambda t: ctypes.c_void_p(t.data_ptr())
    I = ctypes.c_int64
    st = lib.dyspec_prompt_attn_in_form(f, p(q), I(Hq * d), p(k), I(Hkv * d), p(v), I(Hkv * d), ctypes.byref(b._c()), Hq, Hkv, d, dy.F32 if dtype is F32 else dy.BF16,
                                        ctypes.c_float(0.1), p(out), p(ws), ctypes.c_size_t(ws.numel()), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert st == 0 and not ws[:16384].any()
    at = 0
    for s, n in enumerate(new):
        if n:
            want, bound = attend_plain(*(t[at:at + n].double().numpy() for t in host), visible_rows(n, 0), 0.1, weight_half(form, dtype), HALF[dtype])
            compare(out[at:at + n].double().cpu().numpy(), want, bound, f"prompt {s}")
        at += n


def test_forms_that_there_are_not(dy):
    c = Paged((5,), (300,), 4, 2, 64, F32, 16, 2)
    for form in ((0, 0, 0), (3, 0, 0), (6, 0, 0), (-1, 0, 0), (4, 100, 0), (4, -128, 0), (4, 128, -1)):
        assert in_form(dy, form, c)[0] == -3, form
