"""What dyspec_sample and dyspec_filter_logits refuse, on the host, before anything is launched: fake addresses are enough and no GPU
is needed.  And the plain form that they are compared with, on rows worked out by hand."""
import ctypes

import numpy as np
import pytest

from paper_2410_11744_amd import binding
from sampling import plain_row

A = 0x7f0000001000
FAR = 0x7f1000000000
BAD_ARG, BAD_SHAPE, UNSUPPORTED = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def settings(n, t=1.0, k=0, p=1.0, m=0.0):
    return (ctypes.c_float * n)(*[t] * n), (ctypes.c_int32 * n)(*[k] * n), (ctypes.c_float * n)(*[p] * n), (ctypes.c_float * n)(*[m] * n)


def sample(lib, logits=A, dtype=0, vocab=100, stride=100, b=None, u=A, token=A, prob=A, kept=A, **s):
    c = (b or binding.Batch.from_sizes([2, 1]))._c()
    return lib.dyspec_sample(logits, dtype, vocab, stride, ctypes.byref(c), *settings(max(c.n_seq, 1), **s), u, token, prob, kept, None)


def keep(lib, logits=A, dtype=0, vocab=100, stride=100, b=None, out=FAR, out_stride=100, **s):
    c = (b or binding.Batch.from_sizes([2, 1]))._c()
    return lib.dyspec_filter_logits(logits, dtype, vocab, stride, ctypes.byref(c), *settings(max(c.n_seq, 1), **s), out, out_stride, None)


def test_settings(lib):
    nan, inf = float("nan"), float("inf")
    for call in (sample, keep):
        for bad in [dict(t=x) for x in (-1.0, nan, inf)] + [dict(k=-1)] + [dict(p=x) for x in (0.0, -0.5, 1.5, nan)] + [dict(m=x) for x in (-0.1, 1.1, nan)]:
            assert call(lib, **bad) == BAD_ARG, (call.__name__, bad)


def test_tables(lib):
    for call in (sample, keep):
        assert call(lib, logits=None) == BAD_ARG and call(lib, logits=A + 2) == BAD_ARG and call(lib, logits=A + 1, dtype=1) == BAD_ARG
        assert call(lib, dtype=7) == UNSUPPORTED and call(lib, vocab=(1 << 18) + 1, stride=1 << 19) == UNSUPPORTED
        assert call(lib, vocab=0) == BAD_SHAPE and call(lib, vocab=-4) == BAD_SHAPE and call(lib, stride=99) == BAD_SHAPE
    for name in ("u", "token", "prob", "kept"):
        assert sample(lib, **{name: None}) == BAD_ARG and sample(lib, **{name: A + 2}) == BAD_ARG, name
    assert keep(lib, out=None) == BAD_ARG and keep(lib, out=FAR + 2) == BAD_ARG and keep(lib, out_stride=99) == BAD_SHAPE
    # in place with the same rows, or apart
    for shift in (4, 400, 299 * 4, -4, -299 * 4):
        assert keep(lib, out=A + shift) == BAD_ARG, shift
    assert keep(lib, out=A, out_stride=104) == BAD_ARG


def test_batches(lib):
    falling = binding.Batch(np.array([0, 5, 3], np.int32), np.zeros(2, np.int32), np.zeros(3, np.int64))
    late = binding.Batch(np.array([1, 5], np.int32), np.zeros(1, np.int32), np.zeros(2, np.int64))
    for call in (sample, keep):
        for b in (falling, late, binding.Batch.from_sizes([1] * 65), binding.Batch.from_sizes([(1 << 21) + 1])):
            assert call(lib, b=b) == BAD_SHAPE
    one = settings(1)
    assert lib.dyspec_sample(A, 0, 9, 9, None, *one, A, A, A, A, None) == BAD_ARG
    assert lib.dyspec_sample(A, 0, 9, 9, ctypes.byref(binding.Batch.from_sizes([1])._c()), None, *one[1:], A, A, A, A, None) == BAD_ARG
    # no row: nothing is launched, no error; filters may be missing
    none = ctypes.byref(binding.Batch.from_sizes([0])._c())
    assert lib.dyspec_sample(A, 0, 9, 9, none, one[0], None, None, None, A, A, A, A, None) == 0
    assert lib.dyspec_filter_logits(A, 0, 9, 9, none, one[0], None, None, None, FAR, 9, None) == 0


def given(settings):
    return [None if b is None else np.frombuffer(b, t).tolist() for b, t in zip(settings, (np.float32, np.int32, np.float32, np.float32))]


def test_wrong_numbers_of_settings():
    b = binding.Batch.from_sizes([1, 1])
    for bad in ([1.0], [1.0] * 3, np.ones(3)):
        with pytest.raises(ValueError):
            binding._settings(b, bad, None, None, None)
    t, k, p, m = given(binding._settings(b, np.float32([0.5, 1.0]), 7, [0.25, 0.5], None))
    assert t == [0.5, 1.0] and k == [7, 7] and p == [0.25, 0.5] and m is None


def test_settings_of_other_kinds():
    """Numbers as arrays' elements, and what does not fit 32 bits: refused, not taken for another number."""
    b = binding.Batch.from_sizes([1, 1])
    t, k, p, m = given(binding._settings(b, np.float64(0.7), np.int64(40), np.array(0.5), None))
    assert t == [np.float32(0.7)] * 2 and k == [40, 40] and p == [0.5, 0.5] and m is None
    assert given(binding._settings(b, 1.0, [np.int32(3), 2**31 - 1], None, None))[1] == [3, 2**31 - 1]
    for bad in (2**31, 2**32 + 1, [5, -2**31 - 1], 1 << 70, 1.5, [2, 2.5]):
        with pytest.raises(ValueError):
            binding._settings(b, 1.0, bad, None, None)
    assert given(binding._settings(b, 1e39, None, None, None))[0] == [float("inf")] * 2      # (refused by the call)


def test_settings_that_are_not_on_the_host():
    """Refused by name: tensors of a device, which numpy cannot read (here one without data, and one whose gradient is wanted)."""
    import torch
    b = binding.Batch.from_sizes([1, 1])
    for bad in (torch.ones(2, device="meta"), torch.ones(2, requires_grad=True)):
        for at, name in enumerate(("temperature", "top_k", "top_p", "min_p")):
            with pytest.raises(ValueError, match=name):
                binding._settings(b, *[bad if at == x else 1.0 if x == 0 else None for x in range(4)])
    assert given(binding._settings(b, torch.tensor([0.5, 1.0]), torch.tensor([3, 4]), torch.tensor(0.5), None))[:3] == [[0.5, 1.0], [3, 4], [0.5, 0.5]]


def test_the_plain_form_by_hand():
    x = np.log(np.array([1.0, 4.0, 2.0, 1.0]))                # weights 1/4, 1, 1/2, 1/4 of the largest
    for args, kept, token in [((0.0, 1.0), [0, 1, 2, 3], 0), ((0.2, 1.0), [0, 1, 2, 3], 1), ((0.99, 1.0), [0, 1, 2, 3], 3), ((0.5, 0.0), [1], 1),
                              ((0.99, 1.0, 2), [1, 2], 2), ((0.99, 1.0, 3), [0, 1, 2], 2), ((0.99, 1.0, 0, 0.6), [1, 2], 2), ((0.99, 1.0, 0, 0.4), [1], 1),
                              ((0.99, 1.0, 0, 1.0, 0.4), [1, 2], 2), ((0.99, 1.0, 2, 0.6), [1], 1)]:
        got, t, prob, _ = plain_row(x, *args)
        assert np.nonzero(got)[0].tolist() == kept and t == token, args
        assert args[1] == 0 or abs(prob - np.exp(x[t]) / np.exp(x[kept]).sum()) < 1e-15
    assert plain_row(np.array([np.nan, 1.0]), 0.5, 1.0)[1] == -1 and plain_row(np.array([-np.inf, -np.inf]), 0.5, 0.0)[1] == -1
