"""Tree attention in bf16 where one key's score lies far above all before it in the walk, against the fp64 oracle: what was summed before
no longer counts in the rows that see it, and stays in the others."""
import math

import numpy as np
import pytest

from helpers import ATTN_TOL, attn_in_form, oracle_attention_rows
from test_gpu_tree_attn import make_case

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    return m


def far_case(d, seen_by, nats, prefix=1500, n=130):
    q, kp, vp, kt, vt, mask = make_case((n,), (prefix,), 4, 2, d, "bf16", 77)
    for k in (kp, kt):
        k[..., 0] = 0.0
    q[..., 0] = 40.0
    far = nats * math.sqrt(d) / 40.0
    if seen_by == "all":
        kp[356, :, 0] = far                       # behind the first keys of every walk
    else:
        viewers = [int(((mask[:, 0] >> np.uint64(i)) & np.uint64(1)).sum()) for i in range(35, 60)]
        kt[35 + int(np.argmax(viewers)), :, 0] = far
        assert 10 < max(viewers) < n - 60
    return q, kp, vp, kt, vt, mask


def compare_with_oracle(q, kp, vp, kt, vt, mask, batch, d, out):
    rj, rh = np.divmod(np.arange(q.shape[0] * 4), 4)
    want = oracle_attention_rows(*[t.float().numpy() for t in (q, kp, vp, kt, vt)], mask, batch, 0, 1.0 / math.sqrt(d), rj, rh)
    assert np.abs(out.float().cpu().numpy()[rj, rh] - want).max() <= ATTN_TOL["bf16"]


@pytest.mark.parametrize("nats", [100, 300])
@pytest.mark.parametrize("seen_by", ["all", "some"])
@pytest.mark.parametrize("form", [(0, 1, 0), (0, 7, 1), (4, 1, 0), (8, 1, 0)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_a_key_far_above_those_before_it(dy, d, form, seen_by, nats):
    print("form", form, d, seen_by, nats, flush=True)
    case = far_case(d, seen_by, nats)
    batch = dy.Batch.from_sizes([130], [1500])
    dev = [t.cuda() for t in case[:5]]
    out = attn_in_form(dy, form, *dev, torch.from_numpy(case[5].view(np.int64)).cuda(), batch, 1.0 / math.sqrt(d))
    compare_with_oracle(*case, batch, d, out)


@pytest.mark.parametrize("seen_by", ["all", "some"])
@pytest.mark.parametrize("d", [64, 128])
def test_in_the_call_as_it_is(dy, d, seen_by):
    case = far_case(d, seen_by, 150, prefix=3000, n=600)
    batch = dy.Batch.from_sizes([600], [3000])
    out = dy.tree_attn(*[t.cuda() for t in case[:5]], torch.from_numpy(case[5].view(np.int64)).cuda(), batch, 1.0 / math.sqrt(d))
    compare_with_oracle(*case, batch, d, out)
