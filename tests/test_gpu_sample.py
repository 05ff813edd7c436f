"""dyspec_sample and dyspec_filter_logits against the plain form in 64 bits: every filter by itself and all at once, vocabularies
of 1 to 2^18, ties, masks, odd rows and strides, graphs and streams."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from sampling import plain_rows

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
# (temperature, top_k, top_p, min_p)
SETTINGS = [(0, 0, 1, 0), (1, 0, 1, 0), (0.6, 0, 0.9, 0), (0.8, 50, 1, 0), (1.2, 0, 1, 0.1), (0.7, 40, 0.9, 0.02), (1, 1, 1, 0), (1, 0, 1e-6, 0), (1, 0, 1, 1),
            (0.01, 0, 0.5, 0), (30, 1000, 0.99, 0.001), (1e-30, 0, 1, 0), (1e30, 7, 0.5, 0), (1, 1 << 30, 1 - 2.0 ** -24, 1e-30), (2, 300, 0.5, 1e-4)]


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    m.init()
    return m


def columns(settings):
    return [list(c) for c in zip(*settings)]


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype is BF16 else torch.int32)


def check(dy, logits, rows, uniform, settings, batch=None, least=0.9):
    """Both calls on a device table against the plain form."""
    t, k, p, m = columns(settings)
    batch = batch or dy.Batch.from_sizes(rows)
    t = [float(x) for x in t]
    filtered = dy.filter_logits(logits, batch, t, top_k=k, top_p=p, min_p=m)
    got = dy.sample(logits, batch, uniform, t, top_k=k, top_p=p, min_p=m)
    out, tokens, probs, counts, fine = plain_rows(logits, rows, uniform.cpu().numpy(), t, k, p, m)
    assert fine.mean() >= least
    assert np.array_equal(filtered.double().cpu().numpy()[fine], out[fine])
    assert np.array_equal(got.token.cpu().numpy()[fine], tokens[fine])
    assert np.array_equal(got.n_kept.cpu().numpy()[fine], counts[fine])
    # two exact sums, weights within 2^-46 of the largest, one rounding to fp32
    close = np.abs(got.prob.double().cpu().numpy() - probs)[fine] <= 2.0 ** -24 * probs[fine] + logits.shape[1] * 2.0 ** -45
    assert close.all()
    return got, filtered


def table(rows, vocab, dtype, seed, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, vocab), generator=g, device="cuda") * spread
    x += 6 * (torch.rand((rows, vocab), generator=g, device="cuda") < 0.003)
    return x.to(dtype), torch.rand(rows, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [1, 2, 3, 4, 5, 7, 8, 9, 63, 64, 100, 257, 1000, 4095, 4097, 8193, 32000, 32767, 32768, 32769, 50001, 131072, 262143, 262144])
def test_every_setting_at_every_size(dy, vocab, dtype):
    rows = [1, 2, 1] * 5 if vocab < 40000 else [1] * 15
    logits, uniform = table(sum(rows), vocab, dtype, vocab)
    check(dy, logits, rows, uniform, SETTINGS)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_tree_of_rows(dy, dtype):
    rows = [300, 0, 17, 0]
    logits, uniform = table(317, 5000, dtype, 3)
    check(dy, logits, rows, uniform, [(0.6, 0, 0.9, 0), (0, 1, 0.5, 1), (1.1, 64, 0.95, 0.01), (1, 0, 1, 0)])


@pytest.mark.parametrize("vocab", [40, 2000, 32000, 70000])
def test_ties(dy, vocab):
    """Equal logits: the smallest indices are kept, and the draw goes by index.  Whole rows of one value, of two, zeros of both signs,
    a few values many times over (more of them than are looked at one by one)."""
    i = torch.arange(vocab, device="cuda")
    rows = [torch.zeros(vocab, device="cuda"), torch.where(i % 3 == 0, 1.0, 1.0 - 2 ** -20), torch.where(i % 2 == 0, 0.0, -0.0),
            torch.round(torch.randn(vocab, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 2), torch.where(i == vocab - 1, 3.0, -3.0),
            (i // 5).float().neg() / 64, torch.where(i < vocab // 2, -5.0, 5.0)]
    for settings in [(1, 0, 0.5, 0), (1, vocab // 2, 1, 0), (1, 3, 1, 0), (1, 17, 0.4, 0), (0, 0, 1, 0), (1, 0, 1, 0.5), (0.5, vocab - 1, 0.999, 0)]:
        logits = torch.stack(rows)
        uniform = torch.tensor([0.5, 0.25, 0.0, 0.75, 0.3, 0.9, 0.6], device="cuda")
        check(dy, logits, [1] * 7, uniform, [settings] * 7, least=0.5)
        check(dy, logits.to(BF16), [1] * 7, uniform, [settings] * 7, least=0.5)


def test_equal_weights_by_hand(dy):
    """Four equal logits: half of the mass is two tokens; u = 0.5 falls on the third of four."""
    x = torch.zeros((1, 4), device="cuda")
    b = dy.Batch.from_sizes([1])
    got = dy.sample(x, b, torch.tensor([0.5], device="cuda"), 1.0)
    assert (got.token.item(), got.n_kept.item(), got.prob.item()) == (2, 4, 0.25)
    got = dy.sample(x, b, torch.tensor([0.5], device="cuda"), 1.0, top_p=0.5)
    assert (got.token.item(), got.n_kept.item(), got.prob.item()) == (1, 2, 0.5)
    got = dy.sample(x, b, torch.tensor([0.999], device="cuda"), 1.0, top_k=3)
    assert (got.token.item(), got.n_kept.item()) == (2, 3)
    assert dy.filter_logits(x, b, 0.0).tolist() == [[0.0, -np.inf, -np.inf, -np.inf]]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [30, 3001, 40000])
def test_masked_logits(dy, vocab, dtype):
    """-inf and the type's lowest value in most places, in all but one, far apart values, values whose difference overflows."""
    lowest = torch.finfo(dtype).min
    logits, uniform = table(12, vocab, F32, 5)
    i = torch.arange(vocab, device="cuda")
    for r in range(4):
        logits[r, i % 7 != r] = -np.inf if r < 2 else lowest
    logits[4], logits[5] = -np.inf, lowest
    logits[4, vocab // 2] = logits[5, vocab - 1] = -3.0
    logits[6] = lowest
    logits[7, ::2], logits[7, 1::2] = lowest, -lowest
    logits[8] *= 1e30
    logits[9] *= 1e-38
    logits[10] = -np.inf
    logits[10, 0] = lowest
    logits = logits.to(dtype)
    for settings in SETTINGS:
        check(dy, logits, [1] * 12, uniform, [settings] * 12, least=0.5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [9, 2050, 33000])
def test_rows_without_a_distribution(dy, vocab, dtype):
    logits, uniform = table(8, vocab, dtype, 11)
    logits[0, vocab - 1] = np.nan
    logits[1, 0] = np.inf
    logits[2] = -np.inf
    logits[3] = np.nan
    logits[4, vocab // 2], logits[4, 0] = -np.nan, np.inf
    for settings in SETTINGS[:6]:
        got, filtered = check(dy, logits, [1] * 8, uniform, [settings] * 8)
        assert got.token[:5].tolist() == [-1] * 5 and got.n_kept[:5].tolist() == [0] * 5 and got.prob[:5].tolist() == [0.0] * 5
        assert bool((filtered[:5] == -np.inf).all()) and bool((got.token[5:] >= 0).all())


def test_random_numbers_at_the_ends(dy):
    vocab = 1000
    logits, _ = table(8, vocab, F32, 2)
    logits[:, 0] = -np.inf                                   # no weight: not drawn, not by 0 either
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 1.0, -1.0, np.nan, np.inf, -np.inf, 1e-40], device="cuda")
    for s in [(1, 0, 1, 0), (0.7, 20, 0.8, 0)]:
        got, _ = check(dy, logits, [8], u, [s], least=0.0)
        first = torch.stack([got.token[i] for i in (0, 3, 4, 6, 7)])
        kept = [torch.nonzero(torch.isfinite(x))[:, 0] for x in dy.filter_logits(logits, dy.Batch.from_sizes([8]), s[0], top_k=s[1], top_p=s[2])]
        assert [int(x) for x in first] == [int(kept[i][0]) for i in (0, 3, 4, 6, 7)]
        assert all(int(got.token[i]) == int(kept[i][-1]) or s[1] == 0 for i in (1, 2, 5))


def test_draws_follow_the_weights(dy):
    """2^16 evenly spaced numbers: every token comes as often as its weight says, to one."""
    logits, _ = table(1, 300, F32, 8)
    n = 1 << 16
    u = ((torch.arange(n, device="cuda").double() + 0.5) / n).float()
    got = dy.sample(logits.expand(n, 300).contiguous(), dy.Batch.from_sizes([n]), u, 0.9, top_k=100)
    w = torch.exp((logits[0].double() - logits.max()) / np.float32(0.9))
    w[torch.sort(logits[0], descending=True, stable=True)[1][100:]] = 0
    assert float((torch.bincount(got.token.long(), minlength=300) - n * w / w.sum()).abs().max()) <= 1.0 + 1e-2


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("shift,vocab,width", [(0, 999, 1000), (1, 1000, 1003), (3, 32000, 32007), (5, 33333, 33340)])
def test_slices_of_wider_tables(dy, dtype, shift, vocab, width):
    """Rows that begin at any element; what lies beside them is neither used nor written."""
    rows = 6
    wide, uniform = table(rows, width, dtype, 31)
    wide[:, :shift] = wide[:, shift + vocab:] = np.nan
    logits = wide[:, shift:shift + vocab]
    s = [(0.8, 100, 0.9, 0.0)] * rows
    got, filtered = check(dy, logits, [1] * rows, uniform, s)
    dense = dy.sample(logits.contiguous(), dy.Batch.from_sizes([1] * rows), uniform, 0.8, top_k=100, top_p=0.9)
    assert torch.equal(dense.token, got.token) and torch.equal(dense.prob, got.prob)
    room = torch.full((rows, width + 2), 7.0, dtype=dtype, device="cuda")
    out = room[:, 2 - shift % 2:2 - shift % 2 + vocab]
    assert dy.filter_logits(logits, dy.Batch.from_sizes([1] * rows), 0.8, top_k=100, top_p=0.9, out=out) is out
    assert torch.equal(bits(out), bits(filtered))
    assert bool((room[:, :2 - shift % 2] == 7).all()) and bool((room[:, 2 - shift % 2 + vocab:] == 7).all())
    dy.filter_logits(logits, dy.Batch.from_sizes([1] * rows), 0.8, top_k=100, top_p=0.9, out=logits)
    assert torch.equal(bits(logits), bits(filtered)) and bool(torch.isnan(wide[:, :shift]).all()) and bool(torch.isnan(wide[:, shift + vocab:]).all())


def test_numbers_for_all_sequences_and_one_each(dy):
    logits, uniform = table(4, 500, F32, 6)
    b = dy.Batch.from_sizes([1, 2, 1], [5, 6, 7])            # (contexts are of no matter here)
    one = dy.sample(logits, b, uniform, 0.9, top_k=5, top_p=0.9, min_p=0.01)
    each = dy.sample(logits, b, uniform, np.full(3, 0.9), top_k=(5, 5, 5), top_p=[0.9] * 3, min_p=[0.01] * 3)
    assert torch.equal(one.token, each.token) and torch.equal(one.prob, each.prob) and torch.equal(one.n_kept, each.n_kept)
    none = dy.sample(logits[:0], dy.Batch.from_sizes([0, 0]), uniform[:0], 1.0)
    assert none.token.numel() == 0 and dy.filter_logits(logits[:0], dy.Batch.from_sizes([0, 0]), 1.0).shape == (0, 500)


def test_the_same_bits_every_time_and_in_graphs(dy):
    s = torch.cuda.Stream()
    rows, vocab = 40, 32000
    logits, uniform = table(rows, vocab, BF16, 17)
    logits[3] = 0.0
    b = dy.Batch.from_sizes([1] * rows)
    t, k, p, m = columns([SETTINGS[i % len(SETTINGS)] for i in range(rows)])
    want = dy.sample(logits, b, uniform, [float(x) for x in t], top_k=k, top_p=p, min_p=m)
    kept = dy.filter_logits(logits, b, [float(x) for x in t], top_k=k, top_p=p, min_p=m)
    torch.cuda.synchronize()
    out, table_out = dy.Sampled.empty(rows, "cuda"), torch.empty_like(logits)
    call = dy.sample_call(logits, b, uniform, [float(x) for x in t], top_k=k, top_p=p, min_p=m, out=out, stream=s)
    other = dy.filter_logits_call(logits, b, [float(x) for x in t], top_k=k, top_p=p, min_p=m, out=table_out, stream=s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call()
        other()
    kept_logits = logits.clone()
    for rep in range(5):
        out.token.fill_(-9), out.prob.fill_(-9), out.n_kept.fill_(-9), table_out.fill_(9)
        if rep == 3:
            logits.copy_(kept_logits.roll(1, 0))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if rep >= 3:
            want = dy.sample(logits, b, uniform, [float(x) for x in t], top_k=k, top_p=p, min_p=m)
            kept = dy.filter_logits(logits, b, [float(x) for x in t], top_k=k, top_p=p, min_p=m)
        for x, y in ((out.token, want.token), (out.prob, want.prob), (out.n_kept, want.n_kept)):
            assert torch.equal(x, y), rep
        assert torch.equal(bits(table_out), bits(kept))


def test_streams_beside_each_other(dy):
    streams = [torch.cuda.Stream() for _ in range(3)]
    sets = [table(20, 20000 + 999 * i, F32, 40 + i) for i in range(3)]
    b = dy.Batch.from_sizes([20])
    want = [dy.sample(x, b, u, 0.8, top_p=0.9) for x, u in sets]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [dy.sample(x, b, u, 0.8, top_p=0.9, stream=s) for (x, u), s in zip(sets, streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g.token, w.token) and torch.equal(g.prob, w.prob)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [1, 5, 300, 9000, 32768, 33000])
def test_more_rows_than_the_chip_has_places(dy, vocab, dtype):
    """Many rows share the chip in other workgroups than few do: the same bits."""
    rows, per = 300, 20
    logits, uniform = table(rows, vocab, dtype, vocab + 1)
    logits[7, 0] = np.nan
    logits[8] = 1.5
    settings = [SETTINGS[i % len(SETTINGS)] for i in range(rows // per)]
    t, k, p, m = columns(settings)
    t = [float(x) for x in t]
    many = dy.filter_logits(logits, dy.Batch.from_sizes([per] * len(settings)), t, top_k=k, top_p=p, min_p=m)
    for s in range(len(settings)):
        some = dy.filter_logits(logits[s * per:(s + 1) * per], dy.Batch.from_sizes([per]), t[s], top_k=k[s], top_p=p[s], min_p=m[s])
        assert torch.equal(bits(many[s * per:(s + 1) * per]), bits(some)), settings[s]
    check(dy, logits[:20], [20], uniform[:20], settings[:1], least=0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [70, 5000, 40000])
def test_min_p_cuts_next_to_zero(dy, vocab, dtype):
    """Settings whose cut is the difference of two near numbers: it lies next to a logit of zero, where floats are far denser than what the
    difference is known to.  Logits on both sides of it, 1e-5 and more away."""
    for top, temperature, min_p in [(0.0866413191, 0.0650000051, 0.263699979), (1.79451227, 0.782053828, 0.100800216), (3.0, 1.0, float(np.exp(-3.0))),
                                    (-2.0, 1.0, 0.5), (2.5, 1e-30, 0.3), (1.0, 1e30, 1.0)]:
        g = torch.Generator(device="cuda").manual_seed(vocab)
        x = torch.rand((3, vocab), generator=g, device="cuda") * 3 - 2.9
        x[:, :8] = torch.tensor([1e-5, -1e-5, 1e-3, -1e-3, 0.05, -0.05, 1e-4, -1e-4], device="cuda")
        x = torch.minimum(x, torch.tensor(top, device="cuda")).to(dtype)
        x[:, vocab // 2] = torch.tensor(top).to(dtype)
        x = torch.minimum(x, x[:, vocab // 2:vocab // 2 + 1])
        check(dy, x, [1, 1, 1], torch.tensor([0.1, 0.5, 0.9], device="cuda"), [(temperature, 0, 1, min_p), (temperature, 20, 1, min_p), (temperature, 0, 0.9, min_p)], least=0.5)
