"""The cache in 4 bits on the GPU: rows stored, packed and moved bit by bit, and the attention over it against its 64-bit form."""
import math

import pytest
import torch

import kvq_helpers as K
import prompt_helpers as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    from paper_2508_09072_amd import binding
    binding.load()
    return binding


@pytest.fixture(params=[0, 16, 17, 18, 33, 65, 128, 256])
def rows(R, request):
    """Every kernel takes every problem: query rows a workgroup; 0: as they are chosen."""
    R.reader_tuning_override(R.TUNE_PROMPT_ROWS, request.param or -1)
    yield request.param
    R.reader_tuning_override(R.TUNE_PROMPT_ROWS, -1)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def status_word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def odd_rows(gen, *shape):
    """Rows with sizes far apart, zeros of both signs, ties, subnormals and the largest numbers."""
    x = (torch.randn(shape, generator=gen) * torch.randn((*shape[:-1], 1), generator=gen).mul(12).exp2()).bfloat16()
    flat = x.view(-1, shape[-1])
    flat[0] = 0.0
    flat[1 % len(flat), ::2] = -0.0
    flat[2 % len(flat)] = torch.arange(shape[-1]).remainder(61).sub(30).mul(0.25).bfloat16()
    flat[3 % len(flat)] = torch.tensor(1e-40).bfloat16()
    flat[4 % len(flat)] = torch.linspace(-1, 1, shape[-1]).mul(3.38e38).bfloat16()
    flat[5 % len(flat), 5] = 2.0 ** -126
    return x


# ------------------------------------------------------------------ rows into the cache

@pytest.mark.parametrize("Hkv,D", [(1, 64), (2, 128), (3, 128), (9, 64), (5, 128)])
@pytest.mark.parametrize("new,L", [([1], [0]), ([5, 0, 40, 1], [15, 3, 16, 100]), ([33, 17], [0, 31])])
def test_packed_rows_are_stored(R, Hkv, D, new, L):
    gen = torch.Generator().manual_seed(Hkv + D)
    B, N, pad = len(new), sum(new), 3
    cache = K.Cache(gen, [a + b for a, b in zip(L, new)], Hkv, D)
    k, v = odd_rows(gen, N + pad, Hkv, D), odd_rows(gen, N + pad, Hkv, D)
    k[N:] = math.nan                                              # (padding is not looked at)
    want, cu = cache.data.clone(), [sum(new[:b]) for b in range(B + 1)]
    for b in range(B):
        place = cache.place(b, L[b] + new[b], L[b])
        K.put(want, place, k[cu[b]:cu[b + 1]], False)
        K.put(want, place, v[cu[b]:cu[b + 1]], True)
    got, status = cache.data.cuda(), status_word()
    dims = R.make_dims(B, 1, Hkv, Hkv, D, cache.max_pages, 1, cache.num_pages)
    R.reader_kvq_store(dims, k.cuda(), v.cuda(), i32(cu), i32(L), got, cache.table.cuda(), status)
    assert int(status) == 0 and torch.equal(got.cpu(), want)


@pytest.mark.parametrize("T,L", [(1, [0, 15, 16]), (37, [3, 0, 500]), (128, [1])])
@pytest.mark.parametrize("Hkv,D", [(2, 64), (4, 128)])
def test_rows_of_trees_are_stored(R, T, L, Hkv, D):
    gen = torch.Generator().manual_seed(T)
    B = len(L)
    cache = K.Cache(gen, [a + T for a in L], Hkv, D)
    k, v = odd_rows(gen, B, T, Hkv, D), odd_rows(gen, B, T, Hkv, D)
    want = cache.data.clone()
    for b in range(B):
        K.put(want, cache.place(b, L[b] + T, L[b]), k[b], False)
        K.put(want, cache.place(b, L[b] + T, L[b]), v[b], True)
    got, status = cache.data.cuda(), status_word()
    dims = R.make_dims(B, T, Hkv, Hkv, D, cache.max_pages, 1, cache.num_pages)
    R.reader_kvq_store(dims, k.cuda(), v.cuda(), None, i32(L), got, cache.table.cuda(), status)
    assert int(status) == 0 and torch.equal(got.cpu(), want)


def test_every_bf16_number_is_rounded_as_the_definition_says(R):
    """Each of the 65536 bit patterns below a largest value of its own size, one above and a much smaller one."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = bits[:, None, None].repeat(1, 3, 64)
    size = bits.double().abs().nan_to_num(posinf=1.0, nan=1.0)
    for h, f in enumerate((1.0, 5.0, 300.0)):
        x[:, h, 40] = (size * f).clamp(max=3.38e38).bfloat16()
    N = 65536
    cache = K.Cache(torch.Generator().manual_seed(0), [N], 3, 64)
    status, got = status_word(), cache.data.cuda()
    dims = R.make_dims(1, 1, 3, 3, 64, cache.max_pages, 1, cache.num_pages)
    R.reader_kvq_store(dims, x.cuda(), x.flip(0).contiguous().cuda(), i32([0, N]), i32([0]), got, cache.table.cuda(), status)
    assert int(status) == R.STATUS_BAD_VALUE
    codes, scales, _ = K.quantise(x)
    cache.data = got.cpu()
    pages = cache.table[0].long()
    for value, c, e in ((False, codes, scales), (True, codes.flip(0), scales.flip(0))):
        for s in range(16):
            at, shift = K.code_bytes(64, s, value)
            assert torch.equal((cache.data[pages][:, :, at].long() >> shift) & 15, c[s::16]), (value, s)
            assert torch.equal(cache.data[pages][:, :, K.scale_bytes(64, s, value)].long(), e[s::16].long()), (value, s)


def test_values_that_are_no_numbers_become_zeros(R):
    gen = torch.Generator().manual_seed(5)
    cache = K.Cache(gen, [20], 2, 128)
    for bad in (math.nan, math.inf, -math.inf):
        k, v = torch.randn((20, 2, 128), generator=gen).bfloat16(), torch.randn((20, 2, 128), generator=gen).bfloat16()
        k[3, 1, 70] = bad
        want = cache.data.clone()
        K.put(want, cache.place(0, 20), k, False)
        K.put(want, cache.place(0, 20), v, True)
        got, status = cache.data.cuda(), status_word()
        R.reader_kvq_store(R.make_dims(1, 1, 2, 2, 128, cache.max_pages, 1, cache.num_pages), k.cuda(), v.cuda(), i32([0, 20]), i32([0]), got,
                           cache.table.cuda(), status)
        assert int(status) == R.STATUS_BAD_VALUE and torch.equal(got.cpu(), want)


def test_rows_without_a_place_are_left_out(R):
    gen = torch.Generator().manual_seed(6)
    cache = K.Cache(gen, [40, 40, 40], 2, 64)
    k = torch.randn((30, 2, 64), generator=gen).bfloat16()
    cache.table[0, 1], cache.table[1, 1] = -7, cache.num_pages
    want = cache.data.clone()
    for at, (b, start) in enumerate(((0, 10), (1, 10), (2, 40))):
        place = cache.place(b, min(start + 10, 48), start)
        for i, (page, slot) in enumerate(place):
            if 0 <= page < cache.num_pages:
                K.put(want, [(page, slot)], k[at * 10 + i:at * 10 + i + 1], False)
                K.put(want, [(page, slot)], k[at * 10 + i:at * 10 + i + 1], True)
    got, status = cache.data.cuda(), status_word()
    dims = R.make_dims(3, 1, 2, 2, 64, cache.max_pages, 1, cache.num_pages)
    R.reader_kvq_store(dims, k.cuda(), k.cuda(), i32([0, 10, 20, 30]), i32([10, 10, 40]), got, cache.table.cuda(), status)
    assert int(status) == R.STATUS_BAD_PAGE | R.STATUS_BAD_LENGTH and torch.equal(got.cpu(), want)
    for cu in ([0, 25, 10, 30], [-3, 10, 20, 400], [30, 20, 10, 0]):
        R.reader_kvq_store(dims, k.cuda(), k.cuda(), i32(cu), i32([1, 2, 3]), got, cache.table.cuda(), status)
    R.reader_kvq_store(dims, k.cuda(), k.cuda(), i32([0, 10, 20, 30]), i32([-1, -2 ** 31, 2 ** 31 - 1]), got, cache.table.cuda(), status)
    torch.cuda.synchronize()


@pytest.mark.parametrize("NL,Hkv,D", [(1, 2, 64), (3, 1, 128), (2, 5, 128)])
@pytest.mark.parametrize("L,starts", [([1], None), ([40, 0, 100], None), ([33, 64, 7], [5, 64, 6]), ([300], [17])])
def test_pages_are_packed(R, NL, Hkv, D, L, starts):
    gen = torch.Generator().manual_seed(NL + D)
    B = len(L)
    src, dst = P.Cache(gen, L, Hkv, D, lead=(NL,), spare=9), K.Cache(gen, L, Hkv, D, lead=(NL,))
    for b in range(B):
        src.fill(gen, b, L[b])
    want = dst.data.clone()
    for b in range(B):
        lo = starts[b] if starts else 0
        page, slot = src.place(b, L[b])
        place = dst.place(b, L[b], lo)
        if L[b] > lo:
            for layer in range(NL):
                K.put(want[layer], place, src.k[layer, page, :, slot][lo:], False)
                K.put(want[layer], place, src.v[layer, page, :, slot][lo:], True)
    got, status = dst.data.cuda(), status_word()
    dims = R.make_dims(B, 1, Hkv, Hkv, D, dst.max_pages, 1, dst.num_pages)
    R.reader_kvq_pack(dims, src.k.cuda(), src.v.cuda(), src.table.cuda(), None if starts is None else i32(starts), i32(L), max(L), got,
                      dst.table.cuda(), status)
    assert int(status) == 0 and torch.equal(got.cpu(), want)


def test_pages_that_cannot_be_packed_are_left_out(R):
    gen = torch.Generator().manual_seed(8)
    L = [40, 40, 40, 40, 40]
    src, dst = P.Cache(gen, L, 2, 64, lead=(2,)), K.Cache(gen, L, 2, 64, lead=(2,))
    for b in range(5):
        src.fill(gen, b, 40)
    src.table[0, 0], dst.table[1, 2] = -1, 1 << 30
    ends, starts = [40, 40, 41, -5, 20], [0, 0, 0, 0, 21]
    want = dst.data.clone()
    for b, lo, hi in ((0, 16, 40), (1, 0, 32)):
        page, slot = src.place(b, 40)
        for layer in range(2):
            K.put(want[layer], dst.place(b, hi, lo), src.k[layer, page, :, slot][lo:hi], False)
            K.put(want[layer], dst.place(b, hi, lo), src.v[layer, page, :, slot][lo:hi], True)
    got, status = dst.data.cuda(), status_word()
    dims = R.make_dims(5, 1, 2, 2, 64, dst.max_pages, 1, dst.num_pages)
    R.reader_kvq_pack(dims, src.k.cuda(), src.v.cuda(), src.table.cuda(), i32(starts), i32(ends), 40, got, dst.table.cuda(), status)
    assert int(status) == R.STATUS_BAD_PAGE | R.STATUS_BAD_LENGTH and torch.equal(got.cpu(), want)


@pytest.mark.parametrize("NL,Hkv,D", [(1, 2, 64), (1, 8, 128), (3, 1, 128), (4, 3, 64)])
@pytest.mark.parametrize("paths", [[[0]], [[0, 1, 2]], [[0, 3, 4, 9, 30], [0], [0, 2, 5]], [list(range(40)), [0, 39]], [[0] + list(range(1, 40, 2))]])
def test_the_accepted_path_moves(R, NL, Hkv, D, paths):
    gen = torch.Generator().manual_seed(len(paths))
    B, T, most = len(paths), 40, max(len(p) for p in paths)
    L = [int(x) for x in torch.randint(0, 70, (B,), generator=gen)]
    cache = K.Cache(gen, [n + T for n in L], Hkv, D, lead=(NL,))
    cache.fill_all(gen, [n + T for n in L])
    want = cache.data.clone()
    for b, path in enumerate(paths):
        for j, node in enumerate(path):
            (p0, s0), (p1, s1) = cache.place(b, L[b] + node + 1, L[b] + node)[0], cache.place(b, L[b] + j + 1, L[b] + j)[0]
            want[:, p1][..., K.row_bytes(D, s1)] = cache.data[:, p0][..., K.row_bytes(D, s0)]
    table = torch.tensor([p + [-1] * (most - len(p)) for p in paths], dtype=torch.int32, device="cuda")
    got, status, lens = cache.data.cuda(), status_word(), i32(L)
    dims = R.make_dims(B, T, Hkv, Hkv, D, cache.max_pages, most, cache.num_pages)
    R.reader_kvq_compact_layers(dims, table, i32([len(p) - 1 for p in paths]), got, cache.table.cuda(), lens, status)
    assert int(status) == 0 and torch.equal(got.cpu(), want)
    assert lens.tolist() == [n + len(p) for n, p in zip(L, paths)]


def test_paths_that_are_wrong_leave_the_cache_as_it_is(R):
    gen = torch.Generator().manual_seed(3)
    paths, n = [[0, 2, 1], [1, 2, 3], [0, 1, 10], [0, 5, 6], [0, 1, 2], [0, 3, 4], [0, 3, 4]], [2, 2, 2, 3, -1, 2, 2]
    L = [20] * 7
    cache = K.Cache(gen, [30] * 7, 1, 64, lead=(2,))
    cache.fill_all(gen, [30] * 7)
    cache.table[5, 1] = cache.num_pages
    lens, status, got = i32(L), status_word(), cache.data.cuda()
    dims = R.make_dims(7, 10, 1, 1, 64, cache.max_pages, 3, cache.num_pages)
    R.reader_kvq_compact_layers(dims, i32(paths), i32(n), got, cache.table.cuda(), lens, status)
    assert int(status) == R.STATUS_BAD_PATH | R.STATUS_BAD_PAGE
    assert lens.tolist() == [20] * 6 + [23]
    mine = cache.table[6, 1]
    changed = (got.cpu() != cache.data).flatten(2).any(-1).any(0)
    assert changed.nonzero().flatten().tolist() == [int(mine)]
    # no layers: the lengths alone
    R.reader_kvq_compact_layers(dims, i32(paths), i32(n), torch.empty((0, cache.num_pages, 1, 17 * 64), dtype=torch.uint8, device="cuda"),
                                cache.table.cuda(), lens, status)
    assert lens.tolist() == [20] * 6 + [26]


# ------------------------------------------------------------------ attention

class Problem:
    """Causal rows (parents None) or draft trees over a cache of random codes."""

    def __init__(self, new, L, Hq, Hkv, D, seed=0, parents=None, pad=2, scale_hi=127, spare=3):
        self.gen = gen = torch.Generator().manual_seed(seed)
        self.new, self.L, self.Hq, self.Hkv, self.D, self.parents = new, L, Hq, Hkv, D, parents
        self.B, self.N = len(new), sum(new) + (pad if parents is None else 0)
        self.cache = K.Cache(gen, [l + n for l, n in zip(L, new)], Hkv, D, spare=spare)
        self.cache.fill_all(gen, [l + n for l, n in zip(L, new)], scale_hi=scale_hi)
        self.cu = [sum(new[:b]) for b in range(self.B + 1)]
        self.q = torch.randn((self.N, Hq, D), generator=gen).bfloat16()
        self.sm_scale = 0.0

    def run(self, R, bound=None, status_want=0, stream=None, lse=True):
        tree = self.parents is not None
        T = self.new[0] if tree else 1
        dims = R.make_dims(self.B, T, self.Hq, self.Hkv, self.D, self.cache.max_pages, 1, self.cache.num_pages, sm_scale=self.sm_scale)
        bound = max(l + (0 if tree else n) for l, n in zip(self.L, self.new)) if bound is None else bound
        ws = torch.empty(R.reader_kvq_workspace_bytes(dims, self.N, bound), dtype=torch.uint8, device="cuda")
        ws.fill_(0xff)
        status, data, table = status_word(), self.cache.data.cuda(), self.cache.table.cuda()
        if tree:
            q = self.q.view(self.B, T, self.Hq, self.D).cuda()
            out = torch.full_like(q, 7.0)
            ls = torch.full((self.B, self.Hq, T), 7.0, device="cuda") if lse else None
            R.reader_kvq_tree_attn(dims, q, data, table, i32(self.L), i32(self.parents), out, ls, bound, ws, status)
            out = out.view(self.N, self.Hq, self.D)
            ls = ls.transpose(1, 2).reshape(self.N, self.Hq) if lse else None
        else:
            out = torch.full((self.N, self.Hq, self.D), 7.0, dtype=torch.bfloat16, device="cuda")
            ls = torch.full((self.N, self.Hq), 7.0, device="cuda") if lse else None
            R.reader_kvq_prompt_attn(dims, self.q.cuda(), data, table, i32(self.cu), i32(self.L), out, ls, bound, ws, status)
            end = sum(self.new)
            assert bool((out[end:] == 7.0).all()) and (not lse or bool((ls[end:] == 7.0).all()))
        assert int(status) == status_want
        return out.cpu(), ls.cpu() if lse else None

    def sees(self, b):
        n, L = self.new[b], self.L[b]
        s = torch.ones((n, L + n), dtype=torch.bool).tril(L)
        if self.parents is not None:
            s[:, L:] = K.ancestors(self.parents[b])
        return s

    def check(self, out, lse, only=None, sees=None):
        for b in range(self.B) if only is None else only:
            n, S = self.new[b], self.L[b] + self.new[b]
            if n == 0:
                continue
            lo = self.cu[b]
            o, s, bo, bs = K.attention(self.q[lo:lo + n], self.cache.rows(b, S, False), self.cache.rows(b, S, True),
                                       self.sees(b) if sees is None else sees, self.sm_scale or None)
            P.check(out[lo:lo + n], o, bo, "out of sequence %d" % b)
            if lse is not None:
                P.check(lse[lo:lo + n], s, bs, "lse of sequence %d" % b)


def bushy(gen, B, T):
    return [[-1] + [int(torch.randint(max(0, i // 4 - 2), i, (1,), generator=gen)) for i in range(1, T)] for _ in range(B)]


HEADS = [(4, 1, 128), (3, 1, 64), (8, 2, 64), (2, 2, 128), (16, 1, 128), (6, 2, 128), (7, 1, 64)]
LENGTHS = [
    ([1], [0]), ([1], [31]), ([1], [32]), ([3, 0, 1, 70], [0, 5, 200, 3]), ([65], [0]), ([200, 129], [0, 0]), ([0, 0], [4, 0]),
    ([1] * 9, [0, 1, 15, 16, 17, 100, 511, 512, 777]), ([40, 1, 333], [1000, 2000, 5]),
]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("new,L", LENGTHS)
def test_prompts(R, rows, Hq, Hkv, D, new, L):
    p = Problem(new, L, Hq, Hkv, D, seed=Hq + D + len(new))
    p.check(*p.run(R))


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("T,L", [(1, [0]), (1, [47, 700, 3]), (16, [512]), (33, [0, 1, 31, 250]), (64, [1000, 64]), (128, [5, 300])])
def test_trees(R, rows, Hq, Hkv, D, T, L):
    p = Problem([T] * len(L), L, Hq, Hkv, D, seed=T + D, parents=bushy(torch.Generator().manual_seed(T), len(L), T))
    p.check(*p.run(R))


@pytest.mark.parametrize("parents", [[-1] + list(range(39)), [-1] + [0] * 39, [-1, 0, 0, 2] + [3] * 36])
def test_chains_and_stars(R, rows, parents):
    p = Problem([40], [77], 4, 2, 128, seed=4, parents=[parents])
    p.check(*p.run(R))


def test_wrong_links_make_roots(R, rows):
    gen = torch.Generator().manual_seed(2)
    parents = bushy(gen, 3, 40)
    parents[0][0], parents[0][7], parents[1][20], parents[1][39], parents[2][1] = 3, 7, -1, 1 << 30, -(1 << 31)
    p = Problem([40] * 3, [100, 3, 0], 4, 2, 64, seed=5, parents=parents)
    p.check(*p.run(R, status_want=R.STATUS_BAD_TREE))


@pytest.mark.parametrize("Hq,Hkv,D,new,L", [(4, 2, 128, [900], [0]), (8, 2, 64, [500, 1, 300], [0, 2500, 300]), (2, 1, 128, [1, 1], [9000, 4000]),
                                             (4, 4, 64, [100], [6000]), (16, 2, 128, [130], [1023])])
def test_long(R, rows, Hq, Hkv, D, new, L):
    p = Problem(new, L, Hq, Hkv, D, seed=3)
    p.check(*p.run(R))


def test_scale_and_no_lse(R, rows):
    p = Problem([50], [20], 4, 2, 128, seed=4)
    p.sm_scale = 0.3
    p.check(*p.run(R, lse=False))
    p = Problem([50], [400], 4, 2, 128, seed=4, parents=bushy(torch.Generator().manual_seed(1), 1, 50))
    p.sm_scale = 0.02
    p.check(*p.run(R))


@pytest.mark.parametrize("new,L", [([300], [0]), ([2, 1], [300, 700]), ([60], [900])])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("up", [True, False])
def test_scores_far_from_the_first_ones(R, rows, new, L, D, up):
    """Keys that grow or shrink along the sequence: later scores are hundreds above or below whatever came first."""
    p = Problem(new, L, 4, 2, D, seed=5)
    for b in range(len(new)):
        S = new[b] + L[b]
        for j, (page, slot) in enumerate(p.cache.place(b, S)):
            p.cache.data[page][:, K.scale_bytes(D, slot, False)] = 118 + (12 * j // S if up else 12 - 12 * j // S)
    p.check(*p.run(R))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_queries_of_many_sizes(R, rows, D, tree):
    """Values that are thousands of times smaller than others of their 32, whole rows that are next to nothing, rows of zeros: a kernel
    may hold a query to 2^-15 of the largest of its 32."""
    parents = bushy(torch.Generator().manual_seed(7), 2, 60) if tree else None
    p = Problem([60, 60], [300, 20], 4, 2, D, seed=26, parents=parents)
    size = torch.randint(-14, 3, p.q.shape, generator=p.gen) + torch.randint(-1, 2, p.q.shape[:2], generator=p.gen)[..., None]
    p.q = (p.q * size.float().exp2()).bfloat16()
    p.q[3] = 0.0
    p.q[5] *= 2.0 ** -120
    p.q[7] *= 2.0 ** -100
    p.q[9, :, 32:] = 0.0
    p.q[11, :, 1:] *= 2.0 ** -20
    p.q[65, :, :32] *= 2.0 ** -60
    out, lse = p.run(R)
    for b in range(2):
        mine, S = slice(60 * b, 60 * b + 60), p.L[b] + 60
        want, s, bo, bs = K.attention(p.q[mine], p.cache.rows(b, S, False), p.cache.rows(b, S, True), p.sees(b), query_step=2.0 ** -15)
        P.check(out[mine], want, bo, "out")
        P.check(lse[mine], s, bs, "lse")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_large_scores(R, rows, D, tree):
    """Queries with one value: the keys with the largest one there share the row, the others are 32 (size 2^12) to millions behind.  The
    products are exact: the weights of a value are equal, rounded to bf16 alike, added up in 32 bits, divided, and the output rounded.  A
    weight at a distance x has a relative error of three roundings of x, which is below 104 where it is not zero in 32 bits, and one
    below the smallest normal number is lost."""
    parents = bushy(torch.Generator().manual_seed(5), 2, 40) if tree else None
    p = Problem([40, 40], [500, 3], 4, 2, D, seed=23, parents=parents)
    for size in (2.0 ** 12, 2.0 ** 20, 2.0 ** 28):
        at = torch.randint(0, D, (p.N, 4, 1), generator=p.gen)
        p.q = torch.zeros_like(p.q).scatter_(-1, at, torch.where(torch.rand((p.N, 4, 1), generator=p.gen) < 0.5, -size, size).bfloat16())
        out, lse = p.run(R)
        for b in range(2):
            k, v = p.cache.rows(b, p.L[b] + 40, False), p.cache.rows(b, p.L[b] + 40, True)
            q = p.q[40 * b:40 * b + 40].double().view(40, 2, 2, D).permute(1, 2, 0, 3)
            x = (q @ k[:, None].transpose(-1, -2)).masked_fill(~p.sees(b), -math.inf)
            w = ((x - x.amax(-1, keepdim=True)) * D ** -0.5).exp()
            n = w.sum(-1)
            want, mass = (w @ v[:, None]) / n[..., None], (w @ v[:, None].abs()) / n[..., None]
            flat = lambda t: t.permute(2, 0, 1, *range(3, t.dim())).reshape(40, 4, *t.shape[3:])  # noqa: E731
            S = k.shape[1]
            bound = P.BF16 * (want.abs() + mass) * (1 + 2 * P.BF16) + (320 + S) * P.F32 * mass + S * 2.0 ** -126 * float(v.abs().max())
            P.check(out[40 * b:40 * b + 40], flat(want), flat(bound), "out")
            top = flat(x.amax(-1) * D ** -0.5 + n.log())
            P.check(lse[40 * b:40 * b + 40], top, 8 * P.F32 * (1 + top.abs()), "lse")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_queries_that_are_no_numbers_stay_to_themselves(R, rows, D, tree):
    """Infinite, huge and undefined queries: the call ends, and the other rows are what they are without them."""
    parents = bushy(torch.Generator().manual_seed(6), 2, 70) if tree else None
    p = Problem([70, 70], [900, 40], 4, 2, D, seed=24, parents=parents)
    usual = p.q.clone()
    for bad in (math.nan, math.inf, -math.inf, 3.3e38, 2.0 ** 100, 2.0 ** 45, 2.0 ** 34):
        odd = torch.rand((p.N, 4), generator=p.gen) < 0.2
        p.q = torch.where(odd[..., None], (torch.randn((p.N, 4, D), generator=p.gen).clamp(-1, 1) * bad).bfloat16(), usual)
        p.q[0, 0] = usual[0, 0]
        p.q[1, 0, 3] = bad
        odd[0, 0], odd[1, 0] = False, True
        out, lse = p.run(R)
        for b in range(2):
            mine = slice(70 * b, 70 * b + 70)
            want, s, bo, bs = K.attention(usual[mine], p.cache.rows(b, p.L[b] + 70, False), p.cache.rows(b, p.L[b] + 70, True), p.sees(b))
            good = ~odd[mine]
            P.check(out[mine][good], want[good], bo[good], "out")
            P.check(lse[mine][good], s[good], bs[good], "lse")


def test_scales_at_both_ends(R, rows):
    """The smallest and the largest scales that rows are stored with: weights of one key, values that are next to nothing."""
    p = Problem([3], [60], 2, 1, 64, seed=6)
    p.cache.data[..., 16 * 64 + 32:] = 2
    out, lse = p.run(R)
    p.check(out, lse)
    p.cache.data[..., 16 * 64 + 32:] = 245
    p.check(*p.run(R))


def test_pages_that_do_not_exist_are_left_out(R, rows):
    for parents in (None, bushy(torch.Generator().manual_seed(1), 2, 80)):
        new = [80, 3] if parents is None else [80, 80]
        L = [70, 40]
        p = Problem(new, L, 4, 2, 64, seed=7, parents=parents)
        table = p.cache.table.clone()
        p.cache.table[0, 2], p.cache.table[0, 6] = 1 << 30, -5
        out, lse = p.run(R, status_want=R.STATUS_BAD_PAGE)
        p.cache.table = table
        sees = p.sees(0)
        sees[:, 32:48] = sees[:, 96:112] = False
        p.check(out, lse, only=[1])
        p.check(out, lse, only=[0], sees=sees)


def test_rows_that_see_nothing(R, rows):
    p = Problem([20, 4], [0, 16], 4, 2, 128, seed=8)
    p.cache.table[:] = -1
    out, lse = p.run(R, status_want=R.STATUS_BAD_PAGE)
    assert bool((out[:24] == 0).all()) and bool((lse[:24] == -math.inf).all())
    p = Problem([5, 3], [0, 0], 4, 2, 64, seed=14)
    out, lse = p.run(R, bound=0, status_want=R.STATUS_BAD_LENGTH)
    assert bool((out[:8] == 0).all()) and bool((lse[:8] == -math.inf).all())


def test_a_sequence_beyond_the_bound_is_cut(R, rows):
    p = Problem([30, 10], [100, 0], 4, 2, 64, seed=9)
    out, lse = p.run(R, bound=110, status_want=R.STATUS_BAD_LENGTH)
    p.check(out, lse, only=[1])
    sees = p.sees(0)
    sees[:, 110:] = False
    p.check(out, lse, only=[0], sees=sees)
    # a tree behind the bound: its rows count as those that are there
    p = Problem([10, 10], [60, 7], 4, 2, 64, seed=9, parents=bushy(torch.Generator().manual_seed(1), 2, 10))
    out, lse = p.run(R, bound=50, status_want=R.STATUS_BAD_LENGTH)
    p.check(out, lse, only=[1])
    p.L[0] = 50
    p.check(out, lse, only=[0])


def test_bounds_out_of_order_stay_inside_the_tensors(R, rows):
    p = Problem([4, 5, 6, 3], [20, 0, 3, 40], 4, 2, 64, seed=10, pad=0)
    dims = R.make_dims(4, 1, 4, 2, 64, p.cache.max_pages, 1, p.cache.num_pages)
    bound = p.cache.max_pages * 16
    ws = torch.empty(R.reader_kvq_workspace_bytes(dims, 18, bound), dtype=torch.uint8, device="cuda")
    for cu, L in (([0, 9, 4, 15, 18], p.L), ([-4, 2, 2, 400, 401], p.L), ([18] * 5, p.L), ([9, 7, 5, 2, -7], p.L),
                  ([0, 4, 9, 15, 18], [-1, -(1 << 31), (1 << 31) - 1, 5])):
        out, status = torch.zeros((18, 4, 64), dtype=torch.bfloat16, device="cuda"), status_word()
        R.reader_kvq_prompt_attn(dims, p.q.cuda(), p.cache.data.cuda(), p.cache.table.cuda(), i32(cu), i32(L), out, None, bound, ws, status)
        torch.cuda.synchronize()
        assert cu == [18] * 5 or int(status) & R.STATUS_BAD_LENGTH


def test_the_same_bits_every_time(R, rows):
    p = Problem([700, 1, 90], [10, 3000, 2000], 8, 2, 128, seed=11)
    a, la = p.run(R)
    for _ in range(3):
        b, lb = p.run(R)
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(la, lb)


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (12, 4, 64)])
def test_many_sequences(R, rows, Hq, Hkv, D):
    gen = torch.Generator().manual_seed(12)
    new = [int(n) * (i % 5 != 3) for i, n in enumerate(torch.randint(0, 7, (150,), generator=gen))]
    L = [int(n) for n in torch.randint(0, 90, (150,), generator=gen)]
    p = Problem(new, L, Hq, Hkv, D, seed=13)
    p.check(*p.run(R))
    p = Problem([5] * 150, L, Hq, Hkv, D, seed=13, parents=bushy(gen, 150, 5))
    p.check(*p.run(R))


def test_the_largest_batch(R, rows):
    gen = torch.Generator().manual_seed(16)
    B = 4096
    new, L = torch.randint(0, 4, (B,), generator=gen).tolist(), torch.randint(0, 40, (B,), generator=gen).tolist()
    p = Problem(new, L, 4, 2, 64, seed=17)
    p.check(*p.run(R), only=list(range(60)) + list(range(60, B - 40, 97)) + list(range(B - 40, B)))


def test_far_pages(R, rows):
    """Pages whose blocks start behind 2^32 bytes of the cache."""
    p = Problem([40, 1], [30, 100], 4, 2, 128, seed=15)
    n = (1 << 32) // (2 * 17 * 128) + 40
    data = torch.empty((n, 2, 17 * 128), dtype=torch.uint8, device="cuda")
    far = n - p.cache.num_pages
    data[far:] = p.cache.data.cuda()
    table = torch.where(p.cache.table >= 0, p.cache.table + far, -1).int().cuda()
    dims = R.make_dims(2, 1, 4, 2, 128, p.cache.max_pages, 1, n)
    ws = torch.empty(R.reader_kvq_workspace_bytes(dims, p.N, 101), dtype=torch.uint8, device="cuda")
    out, lse, status = torch.empty((p.N, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((p.N, 4), device="cuda"), status_word()
    R.reader_kvq_prompt_attn(dims, p.q.cuda(), data, table, i32(p.cu), i32(p.L), out, lse, 101, ws, status)
    assert int(status) == 0
    p.check(out.cpu(), lse.cpu())


# ------------------------------------------------------------------ as they are used

@pytest.mark.parametrize("D", [64, 128])
def test_trees_see_what_plain_decoding_sees(R, D):
    """A prompt worked on in bf16 and packed, then steps of draft trees: stored, attended to, accepted, moved.  A chain's rows give
    what single tokens over the same cache give, and the cache ends as plain decoding leaves it."""
    gen = torch.Generator().manual_seed(D)
    B, Hq, Hkv, T, L = 2, 4, 2, 6, [45, 16]
    src = P.Cache(gen, L, Hkv, D, lead=(1,))
    for b in range(B):
        src.fill(gen, b, L[b])
    caches = [K.Cache(torch.Generator().manual_seed(1), [n + 40 for n in L], Hkv, D, lead=(1,)) for _ in range(2)]
    tree, plain = (c.data.cuda() for c in caches)
    table = caches[0].table.cuda()
    make = lambda t, path=1: R.make_dims(B, t, Hq, Hkv, D, caches[0].max_pages, path, caches[0].num_pages)  # noqa: E731
    status, lens = status_word(), i32(L)
    pack_table = torch.full((B, caches[0].max_pages), -1, dtype=torch.int32)
    pack_table[:, :src.max_pages] = src.table
    for c in (tree, plain):
        R.reader_kvq_pack(make(1), src.k.cuda(), src.v.cuda(), pack_table.cuda(), None, lens, max(L), c, table, status)
    assert torch.equal(tree, plain)
    plain_lens = lens.clone()
    for step in range(3):
        q, k, v = (torch.randn((B, T, h, D), generator=gen).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
        # the main chain is nodes 0, 2, 3; the others are wrong guesses
        parents = i32([[-1, 0, 0, 2, 2, 1]] * B)
        path, n = i32([[0, 2, 3]] * B), i32([2] * B)
        bound = int(lens.max())
        out, ws = torch.empty_like(q), torch.empty(R.reader_kvq_workspace_bytes(make(T), B * T, bound), dtype=torch.uint8, device="cuda")
        R.reader_kvq_store(make(T), k, v, None, lens, tree[0], table, status)
        R.reader_kvq_tree_attn(make(T), q, tree[0], table, lens, parents, out, None, bound, ws, status)
        R.reader_kvq_compact_layers(make(T, 3), path, n, tree, table, lens, status)
        for node in (0, 2, 3):
            one = [t[:, node].contiguous() for t in (q, k, v)]
            single = torch.empty_like(one[0])
            R.reader_kvq_store(make(1), one[1], one[2], i32([0, 1, 2]), plain_lens, plain[0], table, status)
            R.reader_kvq_prompt_attn(make(1), one[0], plain[0], table, i32([0, 1, 2]), plain_lens, single, None, int(plain_lens.max()) + 1, ws, status)
            plain_lens += 1
            # two results of the same weights and values, each within the bound of its own rounding
            b16 = P.BF16 * 2
            assert bool(((single.double() - out[:, node].double()).abs() <= 2 * b16 * single.double().abs() + 2 * b16 * 6.0).all())
        assert lens.tolist() == plain_lens.tolist()
        for b in range(B):
            for c in (tree, plain):
                caches[0].data = c[0].cpu()
                rows_ = [caches[0].rows(b, int(lens[b]), value) for value in (False, True)]
                if c is tree:
                    kept = rows_
            assert all(torch.equal(x, y) for x, y in zip(kept, rows_))
    assert int(status) == 0


def test_replays_of_a_captured_step(R):
    """Store, attention and move captured once and replayed, with eager work between the replays and another graph that shares the workspace."""
    gen = torch.Generator().manual_seed(20)
    L, T = [300, 41, 1000], 24
    cache = K.Cache(gen, [n + T for n in L], 2, 128, lead=(2,))
    cache.fill_all(gen, [n + T for n in L])
    data0 = cache.data.cuda()
    data, lens, status = data0.clone(), i32(L), status_word()
    q = torch.randn((3, T, 8, 128), generator=gen).bfloat16().cuda()
    k, v = (torch.randn((3, T, 2, 128), generator=gen).bfloat16().cuda() for _ in range(2))
    parents, path, n = i32(bushy(gen, 3, T)), i32([[0, 1, 5], [0, 2, -1], [0, -1, -1]]), i32([2, 1, 0])
    table = cache.table.cuda()
    dims = R.make_dims(3, T, 8, 2, 128, cache.max_pages, 3, cache.num_pages)
    ws = torch.empty(R.reader_kvq_workspace_bytes(dims, 3 * T, 1000), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(q) for _ in range(2)]
    lse = torch.zeros((3, 8, T), device="cuda")

    def step():
        for layer in range(2):
            R.reader_kvq_store(dims, k, v, None, lens, data[layer], table, status)
            R.reader_kvq_tree_attn(dims, q, data[layer], table, lens, parents, outs[layer], lse, 1000, ws, status)
        R.reader_kvq_compact_layers(dims, path, n, data, table, lens, status)

    def reset():
        data.copy_(data0)
        lens.copy_(i32(L))
        for t in outs + [lse]:
            t.zero_()

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs + [lse, data, lens]]
    assert int(status) == 0 and lens.tolist() == [303, 43, 1001]
    graphs = []
    for _ in range(2):
        reset()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            step()
        graphs.append(graph)
    for turn in range(6):
        reset()
        ws.fill_(0xff)
        noise = torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        assert float(noise) == float(noise)
        for a, b in zip(outs + [lse, data, lens], want):
            assert torch.equal(a, b), "replay %d" % turn


def test_replays_of_captured_packing(R):
    gen = torch.Generator().manual_seed(25)
    L, NL = [100, 33], 2
    cache, source = K.Cache(gen, L, 2, 64, lead=(NL,)), K.Cache(gen, L, 2, 64)
    k, v = (torch.randn((NL, source.num_pages, 2, 16, 64), generator=gen).bfloat16().cuda() for _ in range(2))
    data0 = cache.data.cuda()
    data, lens, status, from_table, table = data0.clone(), i32(L), status_word(), source.table.cuda(), cache.table.cuda()
    dims = R.make_dims(2, 1, 2, 2, 64, max(cache.max_pages, source.max_pages), 1, cache.num_pages)
    assert cache.max_pages == source.max_pages

    def step():
        R.reader_kvq_pack(dims, k, v, from_table, None, lens, 112, data, table, status)

    graph = torch.cuda.CUDAGraph()
    step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    for turn in range(4):
        k.normal_()
        lens.copy_(i32([100 - 30 * turn, 5 * turn]))
        data.copy_(data0)
        step()
        want = data.clone()
        data.copy_(data0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(data, want) and int(status) == 0


def test_two_streams_at_once(R):
    """Calls with workspaces of their own on two streams."""
    problems = [Problem([200], [3000], 8, 2, 128, seed=s) for s in (1, 2)]
    want = [p.run(R)[0] for p in problems]
    streams, jobs = [torch.cuda.Stream() for _ in problems], []
    for p in problems:
        dims = R.make_dims(1, 1, 8, 2, 128, p.cache.max_pages, 1, p.cache.num_pages)
        ws = torch.empty(R.reader_kvq_workspace_bytes(dims, p.N, 3200), dtype=torch.uint8, device="cuda")
        jobs.append((dims, p.q.cuda(), p.cache.data.cuda(), p.cache.table.cuda(), i32(p.cu), i32(p.L), torch.zeros_like(p.q, device="cuda"), ws))
    torch.cuda.synchronize()
    for _ in range(10):
        for s, (dims, q, data, table, cu, L, out, ws) in zip(streams, jobs):
            with torch.cuda.stream(s):
                R.reader_kvq_prompt_attn(dims, q, data, table, cu, L, out, None, 3200, ws, None)
    torch.cuda.synchronize()
    for p, w, j in zip(problems, want, jobs):
        assert torch.equal(j[6].cpu()[:200].view(torch.int16), w[:200].view(torch.int16))
