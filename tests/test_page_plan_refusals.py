"""What dyspec_page_plan refuses, on the host, before anything is launched: fake addresses are enough and no GPU is needed."""
import ctypes

import pytest

from paper_2410_11744_amd import binding

A = 0x7f0000001000
BAD_ARG, BAD_SHAPE, UNSUPPORTED = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def plan(lib, ring=A, state=A + 0x1000, n_pages=100, page=16, table=A + 0x2000, max_pages=10, stride=10, held=A + 0x3000, wanted=A + 0x4000, n_seq=4,
         granted=A + 0x5000, slots=A + 0x6000, n_slots=100, slots_from=None):
    return lib.dyspec_page_plan(ctypes.byref(binding._PagePool(ring, state, n_pages, page)), table, max_pages, stride, held, wanted, n_seq, granted, slots, n_slots, slots_from, None)


def test_addresses(lib):
    for name in ("ring", "state", "table", "held", "wanted", "granted"):
        assert plan(lib, **{name: None}) == BAD_ARG, name
        assert plan(lib, **{name: A + 2}) == BAD_ARG, name
    assert plan(lib, slots_from=A + 2) == BAD_ARG and plan(lib, slots_from=A + 0x5008) == BAD_ARG
    assert plan(lib, slots=A + 4) == BAD_ARG and plan(lib, slots=None) == BAD_ARG
    assert lib.dyspec_page_plan(None, A, 1, 1, A, A, 1, A, None, 0, None, None) == BAD_ARG
    # granted is written while lengths are read
    for shift in (0, 4, 12, -12):
        assert plan(lib, granted=A + 0x3000 + shift) == BAD_ARG and plan(lib, granted=A + 0x4000 + shift) == BAD_ARG, shift


def test_shapes(lib):
    for page in (0, 1, 4, 12, 24, -16, 131072):
        assert plan(lib, page=page) == UNSUPPORTED, page
    for bad in (dict(n_seq=0), dict(n_seq=65), dict(n_seq=-1), dict(n_pages=0), dict(n_pages=-5), dict(max_pages=-1), dict(stride=9), dict(n_slots=-1)):
        assert plan(lib, **bad) == BAD_SHAPE, bad


def test_host_tensors_are_refused():
    import torch
    with pytest.raises(ValueError):
        binding.PagePool(torch.zeros(5, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), 16)
