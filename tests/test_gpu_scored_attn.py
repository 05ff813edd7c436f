"""paged_attn and prompt_attn with capped scores, windows and both: every kernel behind them, in one piece and in parts, single tokens,
chunks and trees, odd keys outside the window (tests/scored.py: formulas and bounds)."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from scored import scored_plain, visible_rows
from serving import HALF, Paged, page_table, random_mask

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SCORES = [(50.0, 0), (0.0, 100), (5.0, 700), (30.0, 1), (0.0, 65)]
FORMS = [(k, share, whole) for k in range(6) for share, whole in ((0, 0), (128, 0), (128, 3))]


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    return m


def halves(form, dtype, d, cap):
    """(weights', whether scores are exact) of a kernel."""
    cores = form[0] < 4 if form else dtype is BF16 and d in (64, 128) and cap <= 256
    return HALF[BF16] if cores else 0.0, not cores


_known = {}


def check(c, got, cap, window, rel=None, form=None, key=None):
    """Every sequence's rows against the plain form; rows that see something odd are left to other tests.  Largest share of the bound.
    key: names the inputs, for which the plain form is then computed once."""
    got, worst = got.double().cpu().numpy(), 0.0
    weight, exact = halves(form, c.dtype, c.d, cap)
    for s, n in enumerate(c.new):
        if n == 0:
            continue
        a = c.row0[s]
        k, v = c.rows(s)
        see = visible_rows(n, c.context[s], None if c.mask is None else c.mask[a:a + n], window, None if rel is None else rel[a:a + n])
        known = _known.get((key, s, weight, exact)) if key else None
        want, bound = known or scored_plain(c.q[a:a + n].double().numpy(), k, v, see, c.scale, cap, weight, HALF[c.dtype], exact)
        if key:
            _known[key, s, weight, exact] = want, bound
        fine = np.isfinite(want)
        assert np.isfinite(got[a:a + n][fine]).all(), f"sequence {s}: odd values in rows that see none"
        share = np.abs(got[a:a + n][fine] - want[fine]) / bound[fine]
        worst = max(worst, float(share.max()) if share.size else 0.0)
        assert worst <= 1.0, f"sequence {s}: {worst:.2f} of the bound"
    return worst


def dev(rel):
    return None if rel is None else torch.from_numpy(np.ascontiguousarray(rel, np.int32)).cuda()


def in_form(dy, form, c, cap, window, rel):
    from paper_2410_11744_amd import binding
    lib, out = dy.load_library(), torch.full_like(c.q_dev, 7.0)
    ws = torch.zeros(96 << 20, dtype=torch.uint8, device="cuda")
    f = (ctypes.c_int32 * 3)(*form)
    p = lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())
    positions = dev(rel)
    x = binding._Scores(cap, window, 0 if rel is None else positions.data_ptr())
    st = lib.dyspec_paged_attn_scored_in_form(f, p(c.q_dev), c.cache._ref, ctypes.byref(c.batch._c()), p(c.mask_dev), c.Hq, c.Hkv, c.d, c.cache._code,
                                              ctypes.c_float(c.scale), ctypes.byref(x), p(out), p(ws), ctypes.c_size_t(ws.numel()),
                                              ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    assert not ws[:16384].any(), "the counters are zero again"
    return st, out


@pytest.mark.parametrize("kind", ["causal", "tree", "positions"])
@pytest.mark.parametrize("form,dtype,Hq,Hkv,d,page", [(f, *s) for s in ((BF16, 8, 2, 128, 16), (BF16, 3, 3, 64, 8), (F32, 8, 2, 64, 32), (F32, 3, 1, 96, 8))
                                                      for f in FORMS if s[0] is BF16 or f[0] >= 4], ids=str)
def test_every_kernel(dy, form, dtype, Hq, Hkv, d, page, kind):
    print("form", form, dtype, Hq, Hkv, d, page, kind, flush=True)
    new, context = (1, 0, 37, 200, 5, 64, 300), (700, 30, 0, 129, 1023, 64, 2000)
    mask, rel = random_mask(new, 3) if kind != "causal" else (None, None)
    c = Paged(new, context, Hq, Hkv, d, dtype, page, 11, mask=mask if kind == "tree" else None)
    c.q_dev *= 4
    c.q = c.q_dev.cpu()
    for cap, window in SCORES:
        st, out = in_form(dy, form, c, cap, window, rel)
        assert st == 0
        check(c, out, cap, window, rel, form, (dtype, Hq, Hkv, d, page, kind, cap, window))


@pytest.mark.parametrize("dtype,Hq,Hkv,d", [(BF16, 8, 2, 128), (BF16, 4, 4, 64), (F32, 4, 2, 64), (BF16, 2, 2, 80), (F32, 2, 1, 256)], ids=str)
@pytest.mark.parametrize("window", [1, 2, 31, 63, 64, 65, 127, 128, 129, 1000, 1 << 30, (1 << 31) - 1])
def test_windows(dy, dtype, Hq, Hkv, d, window):
    new, context = (1, 130, 1, 77), (1500, 333, 0, 64)
    c = Paged(new, context, Hq, Hkv, d, dtype, 16, window % 997)
    check(c, dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, window=window), 0.0, window)
    check(c, dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, window=window, cap=20), 20.0, window)


@pytest.mark.parametrize("cap", [1e-3, 0.5, 5, 50, 255, 257, 1e4, 1e9])
@pytest.mark.parametrize("dtype,Hq,Hkv,d", [(BF16, 8, 2, 128), (BF16, 4, 4, 64), (F32, 4, 2, 64), (BF16, 2, 2, 96)], ids=str)
def test_caps(dy, dtype, Hq, Hkv, d, cap):
    """Scores far below the cap, far beyond it, and (for caps that no score comes near) as good as without."""
    new, context = (1, 90, 3), (1100, 200, 31)
    for factor in (0.05, 1.0, 40.0):
        c = Paged(new, context, Hq, Hkv, d, dtype, 32, 7)
        c.q_dev *= factor
        c.q = c.q_dev.cpu()
        check(c, dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, cap=cap), cap, 0)


@pytest.mark.parametrize("window", [1, 3, 8, 20, 47, 48, 400])
@pytest.mark.parametrize("dtype,Hq,Hkv,d", [(BF16, 16, 2, 128), (BF16, 4, 4, 64), (F32, 4, 2, 64)], ids=str)
def test_deep_trees_in_short_windows(dy, dtype, Hq, Hkv, d, window):
    """Windows that end inside the tree: an ancestor is seen by its depth, not by its row."""
    new, context = (48, 300, 130, 1), (10, 700, 0, 55)
    mask, depth = random_mask(new, 5)
    c = Paged(new, context, Hq, Hkv, d, dtype, 16, 3, mask=mask)
    check(c, dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, window=window, rel_pos=dev(depth)), 0.0, window, depth)
    check(c, dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, window=window, cap=9.0, rel_pos=dev(depth)), 9.0, window, depth)
    check(c, dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, window=window), 0.0, window)          # by row


def test_positions_outside_the_tree_count_as_the_nearest(dy):
    new, context = (40,), (100,)
    mask, depth = random_mask(new, 5)
    c = Paged(new, context, 4, 2, 128, BF16, 16, 3, mask=mask)
    wild = depth.copy()
    wild[::3] = 1 << 30
    wild[1::3] = -(1 << 30)
    out = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, window=30, rel_pos=dev(wild))
    check(c, out, 0.0, 30, np.clip(wild, 0, 39))


@pytest.mark.parametrize("dtype,Hq,Hkv,d", [(BF16, 8, 2, 128), (BF16, 8, 8, 64), (F32, 4, 2, 64), (BF16, 2, 2, 32)], ids=str)
@pytest.mark.parametrize("cap,window", SCORES + [(0.0, 64), (12.0, 333)])
def test_prompts(dy, dtype, Hq, Hkv, d, cap, window):
    lengths = [1, 700, 64, 0, 129, 1500, 33]
    g = torch.Generator().manual_seed(9)
    p = torch.randn((sum(lengths), Hq + 2 * Hkv, d), generator=g)
    p[:, :Hq] *= 4
    p = p.to(dtype).cuda()
    q, k, v = p.split([Hq, Hkv, Hkv], dim=1)
    out = dy.prompt_attn(q, k, v, dy.Batch.from_sizes(lengths), 1 / math.sqrt(d), cap=cap or None, window=window or None)
    weight, exact = halves(None, dtype, d, cap)
    at = 0
    for n in lengths:
        if n:
            qs, ks, vs = (x[at:at + n].double().cpu().numpy() for x in (q, k, v))
            want, bound = scored_plain(qs, ks, vs, visible_rows(n, 0, None, window), 1 / math.sqrt(d), cap, weight, HALF[dtype], exact)
            share = np.abs(out[at:at + n].double().cpu().numpy() - want) / bound
            assert share.max() <= 1.0, (n, share.max())
        at += n


@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("form", [None] + [(k, s, 0) for k in range(6) for s in (0, 128)], ids=str)
@pytest.mark.parametrize("dtype,d", [(BF16, 128), (BF16, 64), (F32, 64)], ids=str)
def test_odd_keys_outside_the_window(dy, dtype, d, form, odd):
    """Infinities and NaN in K and V of keys that are behind the window, in the next tile or in the same, do not matter to the rows that
    do not see them; rows that see one in V have it."""
    if form and form[0] < 4 and dtype is F32:
        pytest.skip("kernels 0 .. 3 are for bf16")
    print("form", form, dtype, d, odd, flush=True)
    new, context, window = (1, 140, 20), (900, 500, 40), 70
    c = Paged(new, context, 4, 2, d, dtype, 16, 21)
    for s, at in ((0, 100), (0, 829), (0, 830), (1, 400), (1, 431), (1, 500), (1, 520), (2, 0), (2, 3)):
        page, row = c.place(s, at)
        for t in (c.k, c.v, c.cache.k, c.cache.v):
            t[page, row] = odd
    cap = 10.0 if d == 64 else 0.0
    out = in_form(dy, form, c, cap, window, None)[1] if form else dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, window=window, cap=cap or None)
    check(c, out, cap, window, None, form, ("odd", dtype, d, odd))
    assert bool(torch.isfinite(out[0]).all())                      # (row 900 sees keys 831 .. 900)


def test_rows_that_see_nothing_are_zero(dy):
    """An ancestor mask without the row's own bit, and a window that hides the context."""
    new, context = (70, 5), (300, 20)
    mask, depth = random_mask(new, 8)
    for j in range(75):
        local = j if j < 70 else j - 70
        mask[j, local // 64] &= ~(np.uint64(1) << np.uint64(local % 64))
    for dtype, d in ((BF16, 128), (F32, 64)):
        c = Paged(new, context, 8, 2, d, dtype, 16, 2, mask=mask)
        rel = np.maximum(depth, 0)
        out = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, window=1, rel_pos=dev(rel))
        assert bool((out == 0).all())
        out = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, window=4, cap=3.0, rel_pos=dev(rel))
        check(c, out, 3.0, 4, rel)


def test_only_the_window_is_read(dy):
    """Page numbers of keys before the window lie outside the pool and are not looked at: what they stand for does not show."""
    new, context, window, page = (1, 33), (3000, 1000), 256, 16
    for dtype, d in ((BF16, 128), (F32, 64)):
        c = Paged(new, context, 8, 2, d, dtype, page, 5)
        want = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, window=window)
        table = c.cache.page_table.clone()
        for s in range(2):
            table[s, :(context[s] - window - 64) // page] = -1
        got = dy.paged_attn(c.q_dev, c.batch, dy.PagedCache(c.cache.k, c.cache.v, table), c.scale, window=window)
        assert torch.equal(got, want)
        check(c, got, 0.0, window)


def test_pages_behind_the_window_given_away(dy):
    """Every page whose keys are all behind the window is gone, those that a walk begins with among them; what is read in their place holds
    NaN.  A tree's positions, single tokens, and several."""
    new, context, window, page = (1, 33, 1), (3000, 1000, 777), 256, 16
    for dtype, d in ((BF16, 128), (BF16, 64), (F32, 64)):
        c = Paged(new, context, 8, 2, d, dtype, page, 6)
        k, v = (torch.cat([x, torch.full_like(x[:1], math.nan)]) for x in (c.cache.k, c.cache.v))
        for rel in (None, np.concatenate([np.minimum(np.arange(n), 3) for n in new]).astype(np.int32)):
            table = c.cache.page_table.clone()
            for s in range(3):
                table[s, :(context[s] + 1 - window) // page] = -1
            out = dy.paged_attn(c.q_dev, c.batch, dy.PagedCache(k, v, table), c.scale, window=window, rel_pos=None if rel is None else dev(rel))
            check(c, out, 0.0, window, rel)


def test_graphs_and_streams(dy):
    """Prepared calls of capped and windowed layers, recorded and replayed beside eager ones of other streams."""
    mask, depth = random_mask((64,), 1)
    cs = [(Paged((1, 1, 1), (3000, 40, 700), 16, 2, 128, BF16, 16, 1), dict(cap=50.0)), (Paged((1,), (1500,), 8, 8, 64, F32, 16, 2), dict(window=500)),
          (Paged((64,), (900,), 16, 2, 128, BF16, 16, 3, mask=mask), dict(cap=20.0, window=300, rel_pos=dev(depth))),
          (Paged((400, 1), (100, 2000), 8, 2, 128, BF16, 32, 4), dict(window=128))]
    eager = [dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, **x) for c, x in cs]
    torch.cuda.synchronize()
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [torch.empty_like(c.q_dev) for c, _ in cs]
    calls = [dy.paged_attn_call(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, out=o, stream=s, **x) for (c, x), o in zip(cs, outs)]
    graph = torch.cuda.CUDAGraph()
    dy.init()
    with torch.cuda.graph(graph, stream=s):
        for call in calls:
            call()
    for rep in range(4):
        for o in outs:
            o.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        beside = [dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, stream=other, **x) for c, x in cs]
        torch.cuda.synchronize()
        for o, b, e in zip(outs, beside, eager):
            assert torch.equal(o, e) and torch.equal(b, e), rep


def test_empty_batches(dy):
    c = Paged((1,), (20,), 4, 2, 64, F32, 16, 1)
    none = dy.Batch.from_sizes([0, 0], [5, 6])
    z = torch.zeros((0, 4, 64), device="cuda")
    table = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    assert dy.paged_attn(z, none, dy.PagedCache(c.cache.k, c.cache.v, table), 0.1, cap=5, window=3).shape == (0, 4, 64)
    assert dy.prompt_attn(z, z[:, :2], z[:, :2], dy.Batch.from_sizes([0]), 0.1, cap=5).shape == (0, 4, 64)


@pytest.mark.parametrize("kind", ["causal", "tree", "positions", "near"])
@pytest.mark.parametrize("form,dtype,Hq,Hkv,d", [(f, *s) for s in ((BF16, 4, 4, 128), (BF16, 8, 2, 64), (F32, 4, 2, 64)) for f in FORMS if s[0] is BF16 or f[0] >= 4], ids=str)
def test_a_scale_of_nearly_nothing(dy, form, dtype, Hq, Hkv, d, kind):
    """All weights alike, so that no running reference is ever passed by much, in rows that first sit through keys only others see: those
    of a window, or (near) of masks whose rows see two tokens and no context.  Beside a query that is no number, whose row alone is none."""
    print("form", form, dtype, Hq, Hkv, d, kind, flush=True)
    new, context = (300, 1, 90), (0, 0, 0) if kind == "near" else (130, 2000, 0)
    mask, rel = random_mask(new, 12) if kind in ("tree", "positions") else (None, None)
    if kind == "near":
        mask, at = np.zeros((sum(new), 5), np.uint64), 0
        for n in new:
            for j in range(n):
                for see in (j, j - j % 7):
                    mask[at + j, see // 64] |= np.uint64(1) << np.uint64(see % 64)
            at += n
    c = Paged(new, context, Hq, Hkv, d, dtype, 16, 59, mask=mask if kind in ("tree", "near") else None)
    c.scale = 1e-38
    window = 0 if kind == "near" else 40
    rel = rel if kind == "positions" else None
    st, want = in_form(dy, form, c, 0.0, window, rel)
    assert st == 0
    check(c, want, 0.0, window, rel, form)
    c.q_dev[20, 1, 7] = math.nan
    out = in_form(dy, form, c, 0.0, window, rel)[1]
    assert bool(torch.isnan(out[20, 1]).all())
    out[20, 1] = want[20, 1]
    check(c, out, 0.0, window, rel, form)


def test_positions_are_looked_at_whether_they_are_read_or_not(dy):
    """rel_pos of another size, type or device is refused by calls without a window too; one that fits changes nothing there."""
    new, context = (40, 3), (100, 20)
    mask, depth = random_mask(new, 5)
    c = Paged(new, context, 4, 2, 64, F32, 16, 3, mask=mask)
    k, v = (torch.randn((43, 2, 64), device="cuda") for _ in range(2))
    prompts = dy.Batch.from_sizes(new)
    for scores in (dict(), dict(cap=9.0), dict(window=20)):
        calls = [lambda f, rel: f(c.q_dev, c.batch, c.cache, c.scale, anc_mask=c.mask_dev, rel_pos=rel, **scores), lambda f, rel: f(c.q_dev, k, v, prompts, c.scale, rel_pos=rel, **scores)]
        for call, fs in zip(calls, ((dy.paged_attn, dy.paged_attn_call), (dy.prompt_attn, dy.prompt_attn_call))):
            for f in fs:
                for bad in (dev(depth[:-1]), dev(depth).long(), dev(depth).cpu(), torch.zeros(86, dtype=torch.int32, device="cuda")[::2]):
                    with pytest.raises(ValueError, match="rel_pos"):
                        call(f, bad)
            if "window" not in scores:
                assert torch.equal(call(fs[0], dev(depth)), call(fs[0], None)) and torch.equal(call(fs[1], dev(depth))(), call(fs[0], None))


def test_workspaces_go_by_the_numbers(dy):
    """What a batch remembers of a call is its cap and window, not the objects that hold them: a cap in a tensor that is written anew, or in
    another tensor, is taken as it stands."""
    c = Paged((1, 1), (9000, 40), 8, 2, 128, BF16, 16, 4)
    cap = torch.tensor(300.0)                                      # (fp32 throughout; 50: the bf16 matrix cores)
    first = dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, cap=cap)
    assert torch.equal(first, dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, cap=300.0))
    cap.fill_(50.0)
    want = dy.paged_attn(c.q_dev, dy.Batch.from_sizes((1, 1), (9000, 40)), c.cache, c.scale, cap=50.0)
    assert torch.equal(dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, cap=cap), want)
    known = len(c.batch._memo())
    for _ in range(5):
        assert torch.equal(dy.paged_attn(c.q_dev, c.batch, c.cache, c.scale, cap=torch.tensor(50.0)), want)
    assert len(c.batch._memo()) == known
