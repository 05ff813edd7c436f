"""What the paged cache's calls and prompt attention refuse, on the host, before anything is launched: fake addresses are enough
and no GPU is needed."""
import ctypes

import numpy as np
import pytest

from paper_2410_11744_amd import binding

A = 0x7f0000001000
BAD_ARG, BAD_SHAPE, UNSUPPORTED = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def cache(k=A, v=A, table=A, n_pages=100, page=16, max_pages=10, stride=10, page_stride=16 * 2 * 128):
    return binding._PagedKV(k, v, table, n_pages, page, max_pages, stride, page_stride)


def batch(new=(3, 1), context=(20, 100)):
    return binding.Batch.from_sizes(new, context)._c()


def attn(lib, c=None, b=None, q=A, out=A + 0x10000, mask=None, Hq=8, Hkv=2, d=128, dtype=binding.BF16, scale=0.1, ws=None, nbytes=0):
    return lib.dyspec_paged_attn(q, ctypes.byref(c or cache()), ctypes.byref(b or batch()), mask, Hq, Hkv, d, dtype, scale, out, ws, nbytes, None)


def append(lib, c=None, b=None, q=A, qs=1024, k=A, ks=256, v=A, vs=256, rel=None, freq=A, n_freq=64, Hq=8, Hkv=2, d=128, dtype=binding.BF16,
           q_out=A + 0x10000, k_out=None):
    return lib.dyspec_kv_append(q, qs, k, ks, v, vs, ctypes.byref(c or cache()), ctypes.byref(b or batch()), rel, freq, n_freq, 0, Hq, Hkv, d, dtype,
                                q_out, k_out, None)


def keep(lib, c=None, b=None, layers=1, stride=0, nodes=A, count=A, Hkv=2, d=128, dtype=binding.BF16):
    return lib.dyspec_kv_keep(ctypes.byref(c or cache()), layers, stride, ctypes.byref(b or batch()), nodes, count, Hkv, d, dtype, None)


def prompt(lib, b=None, q=A, qs=1024, k=A, ks=256, v=A, vs=256, Hq=8, Hkv=2, d=128, dtype=binding.BF16, scale=0.1, out=A + 0x10000):
    return lib.dyspec_prompt_attn(q, qs, k, ks, v, vs, ctypes.byref(b or batch((3, 1), (0, 0))), Hq, Hkv, d, dtype, scale, out, None)


def test_caches(lib):
    for call in (attn, append, keep):
        for bad in (dict(k=None), dict(v=None), dict(table=None), dict(k=A + 8), dict(v=A + 8), dict(table=A + 2)):
            assert call(lib, c=cache(**bad)) == BAD_ARG, (call.__name__, bad)
        for page in (0, 1, 4, 12, 24, -16, 131072):
            assert call(lib, c=cache(page=page, page_stride=1 << 26)) == UNSUPPORTED, (call.__name__, page)
        # a table too narrow for 101 tokens of 16 a page, no pool, pages closer than their rows, pages at no 16-byte distance
        for bad in (dict(max_pages=6), dict(stride=9), dict(n_pages=0), dict(page_stride=16 * 2 * 128 - 8), dict(page_stride=16 * 2 * 128 + 4)):
            assert call(lib, c=cache(**bad)) == BAD_SHAPE, (call.__name__, bad)


def test_batches(lib):
    too_long = binding.Batch(np.array([0, (1 << 20) + 1], np.int32), np.array([0], np.int32), np.zeros(2, np.int64))._c()
    falling = binding.Batch(np.array([0, 5, 3], np.int32), np.zeros(2, np.int32), np.zeros(3, np.int64))._c()
    late = binding.Batch(np.array([1, 5], np.int32), np.zeros(1, np.int32), np.zeros(2, np.int64))._c()
    negative = binding.Batch(np.array([0, 5], np.int32), np.array([-1], np.int32), np.zeros(2, np.int64))._c()
    far = binding.Batch(np.array([0, 5], np.int32), np.array([1 << 30], np.int32), np.zeros(2, np.int64))._c()
    for call in (attn, append, keep, prompt):
        for b in (too_long, falling, late, negative, far, binding.Batch.from_sizes([1] * 65)._c()):
            assert call(lib, b=b) == BAD_SHAPE, call.__name__
    assert prompt(lib, b=batch((3, 1), (0, 4))) == BAD_SHAPE                 # a prompt has nothing before it
    # 2^23 + 1 new tokens in all; 2^23 with 17 heads, more than 2^27 rows
    many = binding.Batch(np.array([min(i << 20, (1 << 23) + 1) for i in range(10)], np.int32), np.zeros(9, np.int32), np.zeros(10, np.int64))._c()
    wide = dict(max_pages=1 << 17, stride=1 << 17)
    assert append(lib, c=cache(**wide), b=many) == keep(lib, c=cache(**wide), b=many) == attn(lib, c=cache(**wide), b=many) == prompt(lib, b=many) == BAD_SHAPE
    rows = binding.Batch(np.array([i << 20 for i in range(9)] + [(1 << 23)], np.int32), np.zeros(9, np.int32), np.zeros(10, np.int64))._c()
    assert attn(lib, c=cache(page_stride=16 * 17 * 64, **wide), b=rows, Hq=17, Hkv=17, d=64) == BAD_SHAPE
    assert prompt(lib, b=rows, Hq=17, Hkv=17, d=64, qs=17 * 64, ks=17 * 64, vs=17 * 64) == BAD_SHAPE
    # under a mask, trees of up to 2048 rows
    wide = cache(max_pages=200, stride=200)
    assert attn(lib, c=wide, b=batch((2049,), (0,)), mask=A) == BAD_SHAPE
    assert lib.dyspec_paged_attn(A, ctypes.byref(cache()), None, None, 8, 2, 128, binding.BF16, 0.1, A + 64, None, 0, None) == BAD_ARG
    assert lib.dyspec_paged_attn(A, None, ctypes.byref(batch()), None, 8, 2, 128, binding.BF16, 0.1, A + 64, None, 0, None) == BAD_ARG


def test_heads_and_types(lib):
    for call in (attn, prompt):
        assert call(lib, Hq=7) == BAD_SHAPE and call(lib, Hkv=0) == BAD_SHAPE and call(lib, Hq=0) == BAD_SHAPE and call(lib, Hq=-8) == BAD_SHAPE
        for scale in (0.0, -1.0, float("nan"), float("inf"), 3e38):
            assert call(lib, scale=scale) == BAD_ARG
    for call in (attn, prompt, append, keep):
        for d in (0, 2, 66, 260, -4):
            assert call(lib, d=d) == UNSUPPORTED, (call.__name__, d)
        assert call(lib, dtype=binding.BF16_WAVE) == UNSUPPORTED and call(lib, dtype=7) == UNSUPPORTED
    # rows times heads per KV head squared past 32 bits
    assert prompt(lib, b=batch((1 << 20,), (0,)), Hq=128, Hkv=1, qs=128 * 128) == BAD_SHAPE


def test_addresses(lib):
    assert attn(lib, q=None) == BAD_ARG and attn(lib, out=None) == BAD_ARG and attn(lib, out=A) == BAD_ARG
    for bad in (dict(q=A + 8), dict(out=A + 0x10008), dict(mask=A + 4), dict(ws=A + 8, nbytes=1 << 30)):
        assert attn(lib, **bad) == BAD_ARG, bad
    assert prompt(lib, out=A) == BAD_ARG
    for bad in (dict(q=A + 4), dict(k=A + 4), dict(v=A + 2), dict(out=A + 0x10004), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(qs=1026), dict(ks=258)):
        assert prompt(lib, **bad) == BAD_ARG, bad
    for bad in (dict(qs=1020), dict(ks=252), dict(vs=0), dict(vs=1 << 23)):
        assert prompt(lib, **bad) == BAD_SHAPE, bad
    for bad in (dict(q=A + 1), dict(k=A + 1), dict(k=None), dict(v=None), dict(freq=None), dict(freq=A + 2), dict(rel=A + 2), dict(q_out=None), dict(q=None),
                dict(Hq=0), dict(q=A, q_out=A, qs=1032), dict(k_out=A, ks=264)):
        assert append(lib, **bad) == BAD_ARG, bad
    for bad in (dict(n_freq=65), dict(n_freq=-1), dict(qs=1016), dict(ks=0), dict(vs=255)):
        assert append(lib, **bad) == BAD_SHAPE, bad
    for bad in (dict(nodes=None), dict(count=None), dict(nodes=A + 2), dict(count=A + 1)):
        assert keep(lib, **bad) == BAD_ARG, bad
    for bad in (dict(layers=0), dict(layers=32768), dict(stride=-8), dict(layers=2, stride=4)):
        assert keep(lib, **bad) == BAD_SHAPE, bad


def test_workspace_sizes(lib):
    size = lambda new, context, Hq=8, Hkv=2, d=128, t=binding.BF16: lib.dyspec_paged_attn_workspace_bytes(ctypes.byref(batch(new, context)), Hq, Hkv, d, t)
    assert size((1,), (0,)) == 0 and size((0, 0), (500, 9)) == 0
    assert size((1,), (4000,)) > binding.PAGED_COUNTER_BYTES
    assert size((1,), (4000,), Hq=7) == 0 and size((1,), (4000,), d=3) == 0 and size((1,), (4000,), t=9) == 0


def test_no_token_is_no_call(lib):
    """A batch whose sequences have no new token launches nothing and is no error."""
    none = batch((0, 0), (5, 0))
    assert attn(lib, b=none) == 0 and append(lib, b=none) == 0 and keep(lib, b=none) == 0 and prompt(lib, b=batch((0, 0), (0, 0))) == 0


def test_host_tensors_are_refused():
    import torch
    z = torch.zeros((4, 8, 2, 64))
    with pytest.raises(ValueError):
        binding.PagedCache(z, z, torch.zeros((1, 4), dtype=torch.int32))
    with pytest.raises(ValueError):
        binding.prompt_attn(torch.zeros((4, 2, 64)), torch.zeros((4, 2, 64)), torch.zeros((4, 2, 64)), binding.Batch.from_sizes([4]), 0.1)
