"""Attention over pages and of prompts where one key decides: its score lies far above all before it.  Every kernel, whole and in
parts (test_gpu_attend_forms.py), against the plain form in 64 bits (tests/serving.py: formulas and bounds)."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from serving import HALF, Paged, attend_plain, compare, random_mask, visible_rows
from test_gpu_attend_forms import check, in_form, weight_half, with_forms, workspace

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
