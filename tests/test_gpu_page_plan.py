"""dyspec_page_plan against a plain form on the host: tables, slots, the ring of free pages, over lengths that grow and shrink."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2410_11744_amd as m
    m.load_library()
    return m


class Plain:
    """The pool, the table and the rules, page by page."""

    def __init__(self, n_seq, columns, page, free, pool, head=0):
        self.page, self.table = page, np.full((n_seq, columns), -1, np.int32)
        self.ring = np.full(pool, -7, np.int32)
        self.ring[(head + np.arange(len(free))) % pool] = free
        self.head, self.count = head, len(free)

    def plan(self, held, wanted, slots, slots_from=None):
        columns, pool = self.table.shape[1], len(self.ring)
        pages = lambda n: -(-n // self.page)
        granted, asked, taken, returned, at = [], 0, [], [], 0
        head, tail, free = self.head, self.head + self.count, self.count
        for s, (x, y) in enumerate(zip(held, wanted)):
            if x < 0 or y < 0 or max(x, y) > 1 << 30 or max(pages(x), pages(y)) > columns:
                granted.append(-1)
                continue
            a, b = pages(x), pages(y)
            asked += max(0, b - a)
            ok = b <= a or asked <= free
            granted.append(y if ok else x)
            if ok:
                for c in range(a, b):
                    self.table[s, c] = self.ring[(head + len(taken)) % pool]
                    taken.append(self.table[s, c])
            for c in range(b, a):
                returned.append(self.table[s, c])
                self.table[s, c] = -1
            for place in range(x if slots_from is None else max(0, slots_from[s]), y):
                if at < len(slots):
                    slots[at] = self.table[s, place // self.page] * self.page + place % self.page if ok else -1
                at += 1
        for i, p in enumerate(returned[:pool - free]):
            self.ring[(tail + i) % pool] = p
        self.head = (head + len(taken)) % pool
        self.count = free - len(taken) + min(len(returned), pool - free)
        return np.asarray(granted, np.int32)


def on_device(dy, plain, extra_columns=0):
    """(pool, table) as the plain form has them; the table may be a slice of a wider one."""
    wide = np.full((plain.table.shape[0] + 1, plain.table.shape[1] + extra_columns), 99, np.int32)
    wide[:-1, :plain.table.shape[1]] = plain.table
    dev = torch.from_numpy(wide).cuda()
    pool = dy.PagePool(torch.from_numpy(plain.ring.copy()).cuda(), torch.tensor([plain.head, plain.count, 0, 0], dtype=torch.int32, device="cuda"), plain.page)
    return pool, dev[:, :plain.table.shape[1]], dev


def check(plain, pool, table, granted, want, slots, slots_want):
    assert np.array_equal(granted.cpu().numpy(), want)
    n = plain.table.shape[0]
    assert np.array_equal(table.cpu().numpy()[:n], plain.table)
    assert pool.state.tolist() == [plain.head, plain.count, 0, 0]
    assert np.array_equal(pool.ring.cpu().numpy(), plain.ring)
    assert np.array_equal(slots.cpu().numpy(), slots_want)


@pytest.mark.parametrize("n_seq,page,pages,columns", [(1, 16, 40, 20), (2, 8, 30, 9), (7, 32, 200, 33), (63, 16, 900, 40), (64, 64, 700, 64), (64, 8, 20000, 1100)])
@pytest.mark.parametrize("extra", [0, 5])
def test_many_steps(dy, n_seq, page, pages, columns, extra):
    """A server's life: lengths grow by a token, by a tree, by a prompt, shrink, end; the pool runs short now and then.  Every step
    equals the plain form's, whole arrays compared, and no page has two owners."""
    rng = np.random.default_rng(n_seq * 1000 + page + extra)
    plain = Plain(n_seq, columns, page, rng.permutation(pages).astype(np.int32), pages, head=int(rng.integers(pages)))
    pool, table, whole = on_device(dy, plain, extra)
    held = np.zeros(n_seq, np.int32)
    denied = 0
    for step in range(40):
        grow = [1, 0, int(rng.integers(2, 100)), int(rng.integers(1, columns * page))]
        wanted = np.array([int(rng.choice([0, h, max(0, h - grow[2]), min(h + grow[0], columns * page), min(h + grow[2], columns * page), min(h + grow[3], columns * page)]))
                           for h in held], np.int32)
        room = int(rng.choice([0, 1, int(np.maximum(wanted - held, 0).sum()), 5000]))
        slots = torch.full((room,), -5, dtype=torch.int64, device="cuda")
        slots_want = np.full(room, -5, np.int64)
        since = None if step % 3 else (held * rng.random(n_seq)).astype(np.int32) - (rng.random(n_seq) < 0.1)      # inside what is held, or before it
        granted = dy.page_plan(pool, table, torch.from_numpy(held).cuda(), torch.from_numpy(wanted).cuda(), slots=slots if room or step % 2 else None,
                               slots_from=None if since is None else torch.from_numpy(since.astype(np.int32)).cuda())
        want = plain.plan(held.tolist(), wanted.tolist(), slots_want, None if since is None else since.tolist())
        check(plain, pool, table, granted, want, slots, slots_want)
        denied += int((want != wanted).sum())
        free = plain.ring[(plain.head + np.arange(plain.count)) % pages]
        used = plain.table[plain.table >= 0]
        assert sorted(np.concatenate([free, used]).tolist()) == list(range(pages))
        held = want
    assert bool((whole[-1] == 99).all()) and bool((whole[:, columns:] == 99).all())          # a row and columns beside: left
    assert denied > 0 or n_seq * columns < 2 * pages                      # (where the pool can run short, it did)


def test_lengths_that_cannot_be(dy):
    """Negative lengths, lengths past the table, past 2^30: -1, nothing of the sequence is changed, the others go on."""
    plain = Plain(7, 10, 16, np.arange(100, dtype=np.int32), 100)
    pool, table, _ = on_device(dy, plain)
    start = np.array([20, 20, 20, 20, 20, 20, 20], np.int32)
    plain.plan([0] * 7, start.tolist(), [])
    dy.page_plan(pool, table, torch.zeros(7, dtype=torch.int32, device="cuda"), torch.from_numpy(start).cuda())
    held = [20, -1, 20, 20, (1 << 30) + 5, 2147483647, 20]
    wanted = [50, 30, -2147483648, 161, 30, 2147483647, 160]
    slots, slots_want = torch.full((400,), -5, dtype=torch.int64, device="cuda"), np.full(400, -5, np.int64)
    granted = dy.page_plan(pool, table, torch.tensor(held, dtype=torch.int32, device="cuda"), torch.tensor(wanted, dtype=torch.int32, device="cuda"), slots=slots)
    want = plain.plan(held, wanted, slots_want)
    assert want.tolist() == [50, -1, -1, -1, -1, -1, 160]
    check(plain, pool, table, granted, want, slots, slots_want)


def test_pages_given_back_twice_stay_inside_the_ring(dy):
    """A caller that gives back what the pool already has: what does not fit is dropped."""
    plain = Plain(2, 8, 8, np.arange(4, dtype=np.int32), 6, head=5)
    pool, table, _ = on_device(dy, plain)
    slots = torch.zeros(0, dtype=torch.int64, device="cuda")
    held, wanted = [64, 64], [0, 1]
    granted = dy.page_plan(pool, table, torch.tensor(held, dtype=torch.int32, device="cuda"), torch.tensor(wanted, dtype=torch.int32, device="cuda"), slots=slots)
    want = plain.plan(held, wanted, [])
    check(plain, pool, table, granted, want, slots, np.zeros(0, np.int64))
    assert plain.count == 6


def test_a_state_that_is_no_state_reads_and_writes_inside_the_ring(dy):
    plain = Plain(1, 8, 8, np.arange(6, dtype=np.int32), 6)
    for head, count, as_if in ((-1, 6, 6), (100, 1000, 6), (3, -9, 0)):
        pool, table, whole = on_device(dy, plain, 3)
        pool.state.copy_(torch.tensor([head, count, 0, 0], dtype=torch.int32))
        granted = dy.page_plan(pool, table, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([30], dtype=torch.int32, device="cuda"))
        assert granted.item() == (30 if as_if else 0)
        got = whole.cpu().numpy()
        assert (got[-1] == 99).all() and (got[:, 8:] == 99).all() and ((got[0, :4] >= 0) & (got[0, :4] < 6)).all() == bool(as_if)
        assert 0 <= pool.state[0].item() < 6 and 0 <= pool.state[1].item() <= 6


def test_a_cache_uses_what_was_planned(dy):
    """Rows appended through a planned table lie where the slots say."""
    n_pages, page, Hkv, d = 30, 16, 2, 64
    pool = dy.PagePool.full(n_pages, page, "cuda")
    table = torch.full((3, 8), -1, dtype=torch.int32, device="cuda")
    k_pages, v_pages = (torch.zeros((n_pages, page, Hkv, d), device="cuda") for _ in range(2))
    held = torch.zeros(3, dtype=torch.int32, device="cuda")
    new = [5, 40, 17]
    for context in ([0, 0, 0], new):
        wanted = torch.tensor([c + n for c, n in zip(context, new)], dtype=torch.int32, device="cuda")
        slots = torch.full((sum(new),), -1, dtype=torch.int64, device="cuda")
        held = dy.page_plan(pool, table, held, wanted, slots=slots)
        assert held.tolist() == wanted.tolist()
        k, v = (torch.randn((sum(new), Hkv, d), device="cuda") for _ in range(2))
        dy.kv_append(k, v, dy.Batch.from_sizes(new, context), dy.PagedCache(k_pages, v_pages, table))
        assert torch.equal(k_pages.flatten(0, 1)[slots], k) and torch.equal(v_pages.flatten(0, 1)[slots], v)


@pytest.mark.parametrize("big", [False, True])
def test_replays_go_on_where_the_pool_stands(dy, big):
    """A recorded call takes the lengths and the pool as they are at each replay, eager calls between."""
    n_seq, page, pages, columns = 64, 16, 9000, 300
    plain = Plain(n_seq, columns, page, np.random.default_rng(1).permutation(pages).astype(np.int32), pages)
    pool, table, _ = on_device(dy, plain)
    s = torch.cuda.Stream()
    held, wanted, granted = (torch.zeros(n_seq, dtype=torch.int32, device="cuda") for _ in range(3))
    slots = torch.full((20000 if big else 64,), -5, dtype=torch.int64, device="cuda")
    slots_want = np.full(slots.numel(), -5, np.int64)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    call = dy.page_plan_call(pool, table, held, wanted, slots=slots, granted=granted, stream=s)
    dy.init()
    with torch.cuda.graph(graph, stream=s):
        call()
    rng = np.random.default_rng(2)
    now = np.zeros(n_seq, np.int32)
    for rep in range(6):
        then = np.minimum(now + rng.integers(0, 400 if big else 2, n_seq), columns * page).astype(np.int32)
        if rep % 3 == 2:
            then[::2] = 0
        held.copy_(torch.from_numpy(now))
        wanted.copy_(torch.from_numpy(then))
        torch.cuda.synchronize()
        if rep % 2:
            got = dy.page_plan(pool, table, held, wanted, slots=slots)
        else:
            graph.replay()
            got = granted
        torch.cuda.synchronize()
        want = plain.plan(now.tolist(), then.tolist(), slots_want)
        check(plain, pool, table, got, want, slots, slots_want)
        now = want


def test_pools_beside_each_other(dy):
    """Calls on several streams, each with a pool of its own."""
    streams = [torch.cuda.Stream() for _ in range(3)]
    plains = [Plain(9, 50, 16, np.arange(400, dtype=np.int32), 400, head=7 * i) for i in range(3)]
    sets = [on_device(dy, p) for p in plains]
    held = [np.zeros(9, np.int32)] * 3
    torch.cuda.synchronize()
    for step in range(10):
        out = []
        for i, st in enumerate(streams):
            wanted = ((held[i] * 7 + 31 * step + 50 * i + np.arange(9)) % 700).astype(np.int32)
            h, w = torch.from_numpy(held[i]).cuda(), torch.from_numpy(wanted).cuda()
            torch.cuda.synchronize()
            out.append((wanted, dy.page_plan(sets[i][0], sets[i][1], h, w, stream=st)))
        torch.cuda.synchronize()
        for i, (wanted, granted) in enumerate(out):
            want = plains[i].plan(held[i].tolist(), wanted.tolist(), [])
            check(plains[i], sets[i][0], sets[i][1], granted, want, torch.zeros(0, dtype=torch.int64), np.zeros(0, np.int64))
            held[i] = want


@pytest.mark.parametrize("n_seq,page,columns,n_slots", [(1, 16, 20, 300), (7, 32, 200, 3000), (64, 16, 300, 20000)])
def test_slots_from_any_number(dy, n_seq, page, columns, n_slots):
    """slots_from at, just above and far above wanted, up to the largest number: no slot for such a sequence, and nothing beside the slots is
    touched.  (Sums of such numbers and a thread's own do not fit 32 bits.)"""
    rng = np.random.default_rng(n_seq)
    far = [1 << 30, (1 << 30) + 1, 2**31 - 2049, 2**31 - 2048, 2**31 - 1024, 2**31 - 257, 2**31 - 256, 2**31 - 2, 2**31 - 1, -2**31]
    plain = Plain(n_seq, columns, page, rng.permutation(n_seq * columns).astype(np.int32), n_seq * columns)
    pool, table, whole = on_device(dy, plain, 3)
    held = np.zeros(n_seq, np.int32)
    for step in range(len(far) + 3):
        wanted = rng.integers(0, columns * page + 1, n_seq).astype(np.int32)
        near = wanted.astype(np.int64) + rng.integers(-3, 3, n_seq)
        since = np.where((np.arange(n_seq) + step) % 3 == 0, near, far[step] if step < len(far) else wanted.astype(np.int64) + step - len(far)).astype(np.int32)
        room = torch.full((n_slots + 64,), -5, dtype=torch.int64, device="cuda")
        slots, slots_want = room[32:32 + n_slots], np.full(n_slots, -5, np.int64)
        granted = dy.page_plan(pool, table, torch.from_numpy(held).cuda(), torch.from_numpy(wanted).cuda(), slots=slots, slots_from=torch.from_numpy(since).cuda())
        want = plain.plan(held.tolist(), wanted.tolist(), slots_want, since.tolist())
        check(plain, pool, table, granted, want, slots, slots_want)
        assert bool((room[:32] == -5).all()) and bool((room[32 + n_slots:] == -5).all())
        held = want
    assert bool((whole[-1] == 99).all()) and bool((whole[:, columns:] == 99).all())
