"""What the calls with capped scores and windows refuse, on the host, before anything is launched: fake addresses are enough and no GPU
is needed.  And their plain form on rows worked out by hand."""
import ctypes
import math

import numpy as np
import pytest

from paper_2410_11744_amd import binding
from scored import scored_plain, visible_rows

A = 0x7f0000001000
BAD_ARG = -1


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def attn(lib, cap=0.0, window=0, rel=None, scale=0.1, new=(3, 1), context=(20, 100)):
    c = binding._PagedKV(A, A, A, 100, 16, 10, 10, 16 * 2 * 128)
    b = binding.Batch.from_sizes(new, context)._c()
    x = binding._Scores(cap, window, rel)
    return lib.dyspec_paged_attn_scored(A, ctypes.byref(c), ctypes.byref(b), None, 8, 2, 128, binding.BF16, scale, ctypes.byref(x), A + 0x10000, None, 0, None)


def prompt(lib, cap=0.0, window=0, rel=None, scale=0.1, new=(3, 1)):
    b = binding.Batch.from_sizes(new)._c()
    x = binding._Scores(cap, window, rel)
    return lib.dyspec_prompt_attn_scored(A, 1024, A, 256, A, 256, ctypes.byref(b), 8, 2, 128, binding.BF16, scale, ctypes.byref(x), A + 0x10000, None)


def test_scores(lib):
    for call in (attn, prompt):
        for cap in (-1.0, float("nan"), float("inf"), 2e30, 1e-31):
            assert call(lib, cap=cap) == BAD_ARG, cap
        assert call(lib, cap=1e30, scale=1e-10) == BAD_ARG and call(lib, cap=1e-20, scale=1e30) == BAD_ARG
        assert call(lib, window=-1) == BAD_ARG and call(lib, window=5, rel=A + 2) == BAD_ARG
        assert call(lib, scale=0.0, cap=5.0) == BAD_ARG and call(lib, scale=float("nan"), window=5) == BAD_ARG
        none = dict(new=(0, 0))
        assert call(lib, cap=5.0, window=7, rel=A, **none) == 0                      # no token: nothing is launched


def test_the_ends_of_caps(lib):
    """1e-30 .. 1e30, at scales whose ratio to them is in range."""
    none = dict(new=(0, 0))
    for call in (attn, prompt):
        for cap, scale in ((1e-31, 1e-20), (9.99e-31, 1e-20), (1.001e30, 1.0)):
            assert call(lib, cap=cap, scale=scale) == BAD_ARG and call(lib, cap=cap, scale=scale, **none) == BAD_ARG, cap
        for cap, scale in ((1.001e-30, 1e-20), (9.99e29, 1.0)):
            assert call(lib, cap=cap, scale=scale, **none) == 0, cap
        # the ratio's ends
        assert call(lib, cap=1.0, scale=1.3e-38, **none) == 0 and call(lib, cap=1.0, scale=1.1e-38, **none) == BAD_ARG
        assert call(lib, cap=0.01, scale=9.9e34, **none) == 0 and call(lib, cap=0.01, scale=1.1e35, **none) == BAD_ARG


def test_workspaces(lib):
    b = ctypes.byref(binding.Batch.from_sizes((1,), (100000,))._c())
    size = lambda x: lib.dyspec_paged_attn_scored_workspace_bytes(b, 8, 2, 128, binding.BF16, x)
    plain = lib.dyspec_paged_attn_workspace_bytes(b, 8, 2, 128, binding.BF16)
    assert plain > 0 and size(None) == size(binding._Scores(0.0, 0, None)) == size(binding._Scores(50.0, 0, None)) == plain
    assert size(binding._Scores(0.0, 64, None)) == 0                                 # a walk that short is in one piece
    assert size(binding._Scores(-1.0, 0, None)) == 0


def test_binding():
    for bad in (dict(cap=0.0), dict(cap=-3), dict(cap=float("nan")), dict(window=0), dict(window=-5)):
        with pytest.raises(ValueError):
            binding._scores(bad.get("cap"), bad.get("window"), None, 4, 0)
    x = binding._scores(None, 1 << 40, None, 4, 0)
    assert x.window == (1 << 31) - 1 and x.cap == 0.0


def test_caps_of_no_32_bits():
    """A cap that rounds to zero would be none at all: refused.  The smallest that does not goes on to the call, which says what it takes."""
    for bad in (1e-46, 7e-46, 1e-300, 5e-324, -1e-50):
        with pytest.raises(ValueError):
            binding._scores(bad, None, None, 4, 0)
    assert binding._scores(1.5e-45, None, None, 4, 0).cap > 0 and binding._scores(50, None, None, 4, 0).cap == 50.0


def test_the_plain_form_by_hand():
    assert visible_rows(3, 2, None, 2).tolist() == [[False, True, True, False, False], [False, False, True, True, False], [False, False, False, True, True]]
    # a tree: rows 1 and 2 are children of row 0, at depth 1
    mask = np.array([[1], [3], [5]], np.uint64)
    assert visible_rows(3, 2, mask, 2, [0, 1, 1]).tolist() == [[False, True, True, False, False], [False, False, True, True, False], [False, False, True, False, True]]
    q, k, v = np.ones((1, 1, 1)), np.array([[[1.0]], [[-2.0]]]), np.array([[[1.0]], [[0.0]]])
    out, _ = scored_plain(q, k, v, np.ones((1, 2), bool), 3.0, 2.0, 0.0, 0.0, True)
    a, b = 2 * math.tanh(1.5), 2 * math.tanh(-3.0)
    assert abs(out.item() - math.exp(a) / (math.exp(a) + math.exp(b))) < 1e-15
