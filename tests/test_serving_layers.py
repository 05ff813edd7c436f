"""dyspec_kv_keep refuses layers whose pages lie on top of each other, on the host, before anything is launched (no GPU needed)."""
import pytest

from paper_2410_11744_amd import binding
from test_serving_refusals import BAD_SHAPE, cache, keep


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def test_layers_that_overlap(lib):
    """A layer moves its own rows, beside the others: one row moved by two of them would be read after it was overwritten."""
    page = 16 * 2 * 128                                      # elements of a page
    for layers in (2, 80):
        for stride in (0, 8, page - 8):
            assert keep(lib, layers=layers, stride=stride) == BAD_SHAPE, (layers, stride)
    # ... whatever lies between the pages (a second page between two)
    assert keep(lib, c=cache(page_stride=2 * page), layers=2, stride=page - 8) == BAD_SHAPE
