"""Pages that sequences share: forks, permutations and dropped sequences, pages taken, given back and copied on a write, against a plain
Python account of the pool."""
import pytest
import torch

pytestmark = pytest.mark.gpu
PAGE = 16


@pytest.fixture(scope="module")
def R():
    from paper_2508_09072_amd import binding
    binding.load()
    return binding


def pages_of(n):
    return (n + PAGE - 1) // PAGE


class Pool:
    """Tables, lengths and counts as lists, and what the calls do to them."""

    def __init__(self, seed, lens, max_pages, num_pages, spare_entries=0):
        gen = torch.Generator().manual_seed(seed)
        order = torch.randperm(num_pages, generator=gen).tolist()
        self.max_pages, self.num_pages, self.lens = max_pages, num_pages, list(lens)
        self.table, self.refs = [], [0] * num_pages
        for n in lens:
            held = min(pages_of(n) + spare_entries, max_pages)
            row = [order.pop() for _ in range(held)]
            for p in row:
                self.refs[p] += 1
            self.table.append(row + [-1] * (max_pages - held))

    def reorder(self, sources):
        old, lens = [list(r) for r in self.table], list(self.lens)
        for row in old:
            for p in row:
                if p >= 0:
                    self.refs[p] -= 1
        for b, s in enumerate(sources):
            self.lens[b] = 0 if s < 0 else lens[s]
            held = pages_of(self.lens[b])
            self.table[b] = [] if s < 0 else old[s][:held]
            self.table[b] += [-1] * (self.max_pages - held)
            for p in self.table[b]:
                if p >= 0:
                    self.refs[p] += 1

    def reserve(self, new):
        """Copies (from, to) of the call, or None if the pool is short."""
        B, refs, table = len(new), list(self.refs), [list(r) for r in self.table]
        writers = {}
        for b in range(B):
            if self.lens[b] % PAGE and new[b] > self.lens[b]:
                writers.setdefault(table[b][self.lens[b] // PAGE], []).append(b)
        wants, copies = [], []
        for b in range(B):
            if new[b] < self.lens[b] or pages_of(new[b]) > self.max_pages:
                continue
            used, want = pages_of(self.lens[b]), pages_of(new[b])
            part = table[b][self.lens[b] // PAGE] if self.lens[b] % PAGE and new[b] > self.lens[b] else -1
            if part >= 0 and self.refs[part] > 1 and not (writers[part][-1] == b and len(writers[part]) == self.refs[part]):
                wants.append((b, self.lens[b] // PAGE))
                copies.append((b, part))
            for j in range(used, self.max_pages):
                p = table[b][j]
                if p >= 0 and (j >= want or self.refs[p] > 1):
                    refs[p] -= 1
                    table[b][j] = p = -1
                if p < 0 and j < want:
                    wants.append((b, j))
        free = [p for p in range(self.num_pages) if refs[p] == 0]
        if len(free) < len(wants):
            return None
        taken = {}
        for (b, j), p in zip(wants, free):
            table[b][j] = taken[b, j] = p
            refs[p] = 1
        for _, part in copies:
            refs[part] -= 1
        self.refs, self.table = refs, table
        return [(part, taken[b, self.lens[b] // PAGE]) for b, part in copies]

    def tensors(self):
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        return i32(self.table).reshape(len(self.lens), self.max_pages), i32(self.lens), i32(self.refs)

    def same(self, table, lens, refs):
        assert table.tolist() == self.table
        assert lens.tolist() == self.lens
        assert refs.tolist() == self.refs


def setup(R, pool):
    dims = R.make_dims(len(pool.lens), 1, 1, 1, 64, pool.max_pages, 1, pool.num_pages)
    ws = torch.full((R.reader_pages_workspace_bytes(dims),), 0xff, dtype=torch.uint8, device="cuda")
    return dims, ws, torch.zeros(1, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("lens,sources", [
    ([40], [0]), ([40], [-1]), ([0], [0]), ([40, 16, 0, 33], [0, 1, 2, 3]), ([40, 16, 0, 33], [3, 0, 1, 2]), ([40, 16, 1, 33], [0, 0, 0, 0]),
    ([40, 16, 0, 33], [1, -1, -1, 1]), ([100] * 7, [6, 6, 2, 2, 0, -1, 4]),
])
@pytest.mark.parametrize("spare", [0, 2])
def test_reorder(R, lens, sources, spare):
    pool = Pool(len(lens), lens, 9, 80, spare)
    table, seq, refs = pool.tensors()
    dims, ws, status = setup(R, pool)
    src = torch.tensor(sources, dtype=torch.int32, device="cuda")
    for _ in range(2):                                            # (the second call starts from shared pages)
        R.reader_pages_reorder(dims, src, table, seq, refs, ws, status)
        pool.reorder(sources)
        pool.same(table, seq, refs)
    assert int(status) == 0


def test_reorder_of_a_large_batch(R):
    gen = torch.Generator().manual_seed(1)
    lens = torch.randint(0, 700, (4096,), generator=gen).tolist()
    pool = Pool(2, lens, 50, sum(pages_of(n) for n in lens) + 5)
    table, seq, refs = pool.tensors()
    dims, ws, status = setup(R, pool)
    sources = torch.randint(-1, 4096, (4096,), generator=gen).tolist()
    R.reader_pages_reorder(dims, torch.tensor(sources, dtype=torch.int32, device="cuda"), table, seq, refs, ws, status)
    pool.reorder(sources)
    pool.same(table, seq, refs)
    assert int(status) == 0


def test_sources_lengths_and_entries_out_of_range(R):
    pool = Pool(3, [40, 20, 33], 4, 20)
    table, seq, refs = pool.tensors()
    dims, ws, status = setup(R, pool)
    R.reader_pages_reorder(dims, torch.tensor([3, -2, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), table, seq, refs, ws, status)
    assert int(status) == R.STATUS_BAD_PATH
    pool.same(table, seq, refs)                                   # each is its own source
    status.zero_()
    table[0, 1], table[1, 0] = 20, -3                             # (two pages that are counted, and named no more)
    R.reader_pages_reorder(dims, torch.tensor([1, 0, 2], dtype=torch.int32, device="cuda"), table, seq, refs, ws, status)
    assert int(status) == R.STATUS_BAD_PAGE
    assert table[0, 0] == -3 and table[1, 1] == 20 and seq.tolist() == [20, 40, 33] and refs.tolist() == pool.refs
    status.zero_()
    seq.copy_(torch.tensor([-4, 2 ** 31 - 1, 33], dtype=torch.int32))
    R.reader_pages_reorder(dims, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), table, seq, refs, ws, status)
    assert int(status) == R.STATUS_BAD_LENGTH | R.STATUS_BAD_PAGE
    assert table[0].tolist() == [-1] * 4 and seq.tolist() == [-4, 2 ** 31 - 1, 33]


def reserve(R, pool, new, caches, want_status=0, state=None):
    """The call on the pool's tensors and on caches whose bytes tell pages apart; checks everything and returns the copies."""
    table, seq, refs = state or pool.tensors()
    dims, ws, status = setup(R, pool)
    before = [c.clone() for c in caches if c is not None]
    R.reader_pages_reserve(dims, seq, torch.tensor(new, dtype=torch.int32, device="cuda"), caches[0], caches[1], table, refs, ws, status)
    copies = pool.reserve(new)
    assert int(status) == want_status
    pool.same(table, seq, refs)
    for c, old in zip([c for c in caches if c is not None], before):
        for a, b in copies or []:
            old[:, b] = old[:, a]
        assert torch.equal(c, old)
    return copies


def contents(gen, NL, pages, two=True, shape=(3, 32)):
    return [torch.randint(0, 256, (NL, pages, *shape), generator=gen, dtype=torch.uint8).cuda() if i == 0 or two else None for i in range(2)]


@pytest.mark.parametrize("lens,new", [
    ([40], [41]), ([40], [40]), ([48], [49]), ([0], [1]), ([0], [0]), ([1], [64]), ([40, 16, 0, 33], [60, 16, 33, 34]), ([5] * 70, list(range(5, 75))),
])
@pytest.mark.parametrize("spare", [0, 2])
def test_reserve_without_forks(R, lens, new, spare):
    gen = torch.Generator().manual_seed(4)
    pool = Pool(len(lens), lens, 6, 500, spare)
    assert reserve(R, pool, new, contents(gen, 2, 500)) == []


@pytest.mark.parametrize("lens,sources,new", [
    ([40, 7], [0, 0], [41, 41]),                                  # both write into one page: the last keeps it
    ([40, 7], [0, 0], [40, 41]),                                  # one writes, one does not: a copy
    ([48, 7], [0, 0], [49, 60]),                                  # a full page stays shared
    ([40, 20, 5], [0, 0, 0], [50, 60, 41]),
    ([40, 20, 5], [1, 0, 0], [20, 40, 96]),
    ([33] * 70, [0] * 70, [34 + i % 3 for i in range(70)]),
    ([50, 20, 33, 60] * 20, [i % 7 for i in range(80)], None),
])
@pytest.mark.parametrize("NL,two", [(1, False), (3, True), (0, False)])
def test_reserve_after_forks(R, lens, sources, new, NL, two):
    gen = torch.Generator().manual_seed(5)
    pool = Pool(7, lens, 6, 600)
    pool.reorder(sources)
    new = [n + i % 20 for i, n in enumerate(pool.lens)] if new is None else new
    caches = contents(gen, NL, 600, two) if NL else [None, None]
    assert reserve(R, pool, new, caches) is not None


def test_pages_that_are_reserved_twice_are_not_shared(R):
    """Entries behind a length, without contents, that another sequence holds too are replaced; single ones stay."""
    pool = Pool(8, [20, 20], 6, 30, spare_entries=2)
    for j in (2, 3):                                              # the second sequence names the first one's reserved pages
        pool.refs[pool.table[1][j]] -= 1
        pool.table[1][j] = pool.table[0][j]
        pool.refs[pool.table[0][j]] += 1
    reserve(R, pool, [64, 64], contents(torch.Generator().manual_seed(1), 1, 30))
    assert max(pool.refs) == 1


@pytest.mark.parametrize("lens,new", [
    ([20, 10], [36, 20]), ([20, 16], [21, 90]), ([20, 0], [40, 96]), ([20, 20, 4], [30, 30, 60]), ([20, 20, 4, 4], [30, 30, 60, 60]),
])
def test_a_page_that_is_copied_from_is_not_taken_where_its_other_holders_give_it_back(R, lens, new):
    """Forks of which some have been taken back to fewer positions: a page that one of them is in the middle of lies behind another."""
    for seed in range(4):
        pool = Pool(12 + seed, [20] * len(lens), 6, 30)
        pool.reorder([0] * len(lens))
        pool.lens = list(lens)
        assert len(reserve(R, pool, new, contents(torch.Generator().manual_seed(seed), 3, 30))) > 0
        for p in range(30):
            assert pool.refs[p] == sum(row.count(p) for row in pool.table)


def test_a_pool_that_is_short_changes_nothing(R):
    gen = torch.Generator().manual_seed(6)
    pool = Pool(9, [40, 40, 30], 6, 12, spare_entries=1)
    pool.reorder([0, 0, 2])                                       # five pages held, seven free
    caches = contents(gen, 2, 12)
    before = ([list(r) for r in pool.table], list(pool.refs))
    assert reserve(R, pool, [96, 96, 96], caches, R.STATUS_NO_PAGES) is None             # 1 + 3 + 3 + 4 wanted
    assert before == (pool.table, pool.refs)
    # two entries are held behind the third sequence, and would be given back: 1 + 3 + 3 wanted, 5 + 2 free; one less, and it is short
    for j, p in zip((2, 3, 4), [p for p in range(12) if pool.refs[p] == 0]):
        if j < 4:
            pool.table[2][j] = p
        pool.refs[p] = 1
    before = ([list(r) for r in pool.table], list(pool.refs))
    assert reserve(R, pool, [96, 96, 30], caches, R.STATUS_NO_PAGES) is None
    assert before == (pool.table, pool.refs)
    assert len(reserve(R, pool, [96, 80, 30], caches)) == 1


def test_every_page_of_a_pool_can_be_taken(R):
    pool = Pool(10, [0] * 4, 25, 100)
    reserve(R, pool, [400] * 4, contents(torch.Generator().manual_seed(1), 1, 100))
    assert pool.refs == [1] * 100
    reserve(R, pool, [0, 400, 1, 399], contents(torch.Generator().manual_seed(1), 1, 100))


@pytest.mark.parametrize("num_pages", [4095, 4096, 4097, 70001])
def test_large_pools(R, num_pages):
    gen = torch.Generator().manual_seed(num_pages)
    B = 60
    pool = Pool(11, torch.randint(0, 60 * 16, (B,), generator=gen).tolist(), 70, num_pages)
    pool.reorder([int(x) for x in torch.randint(0, B, (B,), generator=gen)])
    # (free pages at the end only: everything in front is held elsewhere)
    for p in range(num_pages - 900):
        pool.refs[p] += 1
    reserve(R, pool, [n + int(x) for n, x in zip(pool.lens, torch.randint(0, 100, (B,), generator=gen))], [None, None])


def test_lengths_and_entries_out_of_range_of_reserve(R):
    pool = Pool(12, [40, 40, 40, 40], 4, 40)
    table, seq, refs = pool.tensors()
    dims, ws, status = setup(R, pool)
    cache = contents(torch.Generator().manual_seed(1), 1, 40, False)[0]
    R.reader_pages_reserve(dims, seq, torch.tensor([39, 65, -1, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), cache, None, table, refs, ws, status)
    assert int(status) == R.STATUS_BAD_LENGTH
    pool.same(table, seq, refs)
    status.zero_()
    table[0, 2], table[1, 3], table[2, 3] = 40, -9, 1000
    R.reader_pages_reserve(dims, seq, torch.tensor([41, 60, 40, 40], dtype=torch.int32, device="cuda"), cache, None, table, refs, ws, status)
    assert int(status) == R.STATUS_BAD_PAGE
    free = [p for p in range(40) if pool.refs[p] == 0]
    assert table[0, 2] == 40 and table[1, 3] == free[0] and table[2, 3] == -1
    seq.copy_(torch.tensor([-1, 5, 5, 5], dtype=torch.int32))
    status.zero_()
    R.reader_pages_reserve(dims, seq, torch.tensor([5, 5, 5, 5], dtype=torch.int32, device="cuda"), None, None, table, refs, ws, status)
    assert int(status) == R.STATUS_BAD_LENGTH


def test_the_largest_batch(R):
    gen = torch.Generator().manual_seed(13)
    lens = torch.randint(0, 200, (4096,), generator=gen).tolist()
    pool = Pool(14, lens, 16, 90000)
    pool.reorder(torch.randint(0, 300, (4096,), generator=gen).tolist())
    reserve(R, pool, [n + 17 for n in pool.lens], [None, None])


@pytest.mark.parametrize("kind", ["bf16", "4-bit"])
def test_beams_write_without_disturbing_each_other(R, kind):
    """Forks of one sequence append to their own pages: what each of them holds is the common prefix and its own rows."""
    D, Hkv, NL, B = 64, 1, 2, 5
    gen = torch.Generator().manual_seed(15)
    pool = Pool(16, [37, 0, 0, 0, 0], 5, 40)
    table, seq, refs = pool.tensors()
    dims = R.make_dims(B, 1, Hkv, Hkv, D, 5, 1, 40)
    ws, status = torch.empty(R.reader_pages_workspace_bytes(dims), dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    shape = (NL, 40, Hkv, 17 * D) if kind == "4-bit" else (NL, 40, Hkv, PAGE, D)
    k = torch.randint(0, 256, shape, generator=gen, dtype=torch.uint8).cuda()
    v = None if kind == "4-bit" else k.clone()

    def rows(b, c, n):
        """The bytes of the first n positions."""
        import kvq_helpers as K
        t = table[b].tolist()
        at = (lambda s: K.row_bytes(D, s)) if kind == "4-bit" else None
        return torch.stack([c[:, t[j // PAGE]][..., at(j % PAGE)] if at else c[:, t[j // PAGE], :, j % PAGE] for j in range(n)]).cpu()

    R.reader_pages_reorder(dims, torch.zeros(B, dtype=torch.int32, device="cuda"), table, seq, refs, ws, status)
    prefix = rows(0, k, 37)
    R.reader_pages_reserve(dims, seq, seq + 20, k, v, table, refs, ws, status)
    for b in range(B):
        for j in range(37, 57):
            page = int(table[b, j // PAGE])
            if kind == "4-bit":
                import kvq_helpers as K
                block = k[:, page]
                block[..., K.row_bytes(D, j % PAGE).cuda()] = 10 * b + j % 10
            else:
                k[:, page, :, j % PAGE] = 10 * b + j % 10
    for b in range(B):
        got = rows(b, k, 57)
        assert torch.equal(got[:37], prefix)
        for j in range(37, 57):
            assert bool((got[j] == 10 * b + j % 10).all())
    assert int(status) == 0 and int((refs > 1).sum()) == 2        # the two full pages of the prefix


def test_replays_of_a_captured_reorder_and_reserve(R):
    """Captured once; replayed on other selections and lengths, with eager work between, next to a graph that shares the workspace."""
    for B, max_pages, num_pages in ((5, 9, 60), (70, 80, 6000)):  # one workgroup, and a workgroup a sequence
        gen = torch.Generator().manual_seed(B)
        lens = torch.randint(1, 16 * max_pages - 20, (B,), generator=gen).tolist()
        pool = Pool(B, lens, max_pages, num_pages)
        dims, ws, status = setup(R, pool)
        table, seq, refs = pool.tensors()
        caches = contents(gen, 2, num_pages)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        sources, new = i32(list(range(B))), i32(lens)

        def step():
            R.reader_pages_reorder(dims, sources, table, seq, refs, ws, status)
            R.reader_pages_reserve(dims, seq, new, caches[0], caches[1], table, refs, ws, status)

        graphs = []
        step()
        for _ in range(2):
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
                step()
            graphs.append(graph)
        for turn in range(6):
            chosen = torch.randint(0, B, (B,), generator=gen).tolist()
            pool.reorder(chosen)
            wanted = [min(n + turn, 16 * max_pages) for n in pool.lens]
            before = [c.clone() for c in caches]
            copies = pool.reserve(wanted)
            sources.copy_(i32(chosen))
            new.copy_(i32(wanted))
            ws.fill_(0xff)
            torch.cuda.synchronize()
            graphs[turn % 2].replay()
            torch.cuda.synchronize()
            assert int(status) == 0
            pool.same(table, seq, refs)
            for c, old in zip(caches, before):
                for a, b in copies:
                    old[:, b] = old[:, a]
                assert torch.equal(c, old)
            pool.lens = wanted                                    # (the rows that were made room for)
            seq.copy_(new)


def test_two_pools_on_two_streams(R):
    pools = [Pool(40 + i, [30 + i] * 40, 60, 4000) for i in range(2)]
    sources = [torch.randint(-1, 40, (40,), generator=torch.Generator().manual_seed(i)).tolist() for i in range(2)]
    jobs = [(*setup(R, p), *p.tensors(), torch.tensor(s, dtype=torch.int32, device="cuda")) for p, s in zip(pools, sources)]
    new = torch.full((40,), 100, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    for stream, (dims, ws, status, table, seq, refs, src) in zip([torch.cuda.Stream() for _ in pools], jobs):
        with torch.cuda.stream(stream):
            for _ in range(3):
                R.reader_pages_reorder(dims, src, table, seq, refs, ws, status)
                R.reader_pages_reserve(dims, seq, new, None, None, table, refs, ws, status)
    torch.cuda.synchronize()
    for pool, source, (dims, ws, status, table, seq, refs, src) in zip(pools, sources, jobs):
        for _ in range(3):
            pool.reorder(source)
            pool.reserve([100] * 40)
        assert int(status) == 0
        pool.same(table, seq, refs)
