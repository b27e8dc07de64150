"""reader_prompt_attn against its 64-bit form: head layouts, lengths from none to thousands, chunks and single tokens, masks that
leave nothing, values that no row may see."""
import math

import pytest
import torch

import prompt_helpers as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    from paper_2508_09072_amd import binding
    binding.load()
    return binding


@pytest.fixture(params=[0, 16, 32, 33, 64, 128, 256])
def rows(R, request):
    """Every kernel takes every problem: query rows a workgroup, 0 the plain kernel."""
    R.reader_tuning_override(R.TUNE_PROMPT_ROWS, request.param or -1)
    yield request.param
    R.reader_tuning_override(R.TUNE_PROMPT_ROWS, -1)


class Problem:
    def __init__(self, new, L, Hq, Hkv, D, seed=0, pad=2, k_scale=1.0, fill=True):
        self.gen = gen = torch.Generator().manual_seed(seed)
        self.new, self.L, self.Hq, self.Hkv, self.D = new, L, Hq, Hkv, D
        self.B, self.N = len(new), sum(new) + pad
        self.cache = P.Cache(gen, [l + n for l, n in zip(L, new)], Hkv, D)
        for b in range(self.B):
            if fill and new[b] + L[b]:
                self.cache.fill(gen, b, new[b] + L[b], k_scale=k_scale)
        self.cu = torch.cat([torch.zeros(1), torch.cumsum(torch.tensor(new), 0)]).int()
        self.q = torch.randn((self.N, Hq, D), generator=gen).bfloat16()

    def run(self, R, rows=None, bound=None, status_want=0, sm_scale=0.0):
        variant = 1 if rows == 0 else 0
        bound = max([l + n for l, n in zip(self.L, self.new)]) if bound is None else bound
        dims = R.make_dims(self.B, 1, self.Hq, self.Hkv, self.D, self.cache.max_pages, 1, self.cache.num_pages, variant=variant, sm_scale=sm_scale)
        ws = torch.empty(max(256, R.reader_prompt_workspace_bytes(dims, self.N, bound)), dtype=torch.uint8, device="cuda")
        assert rows is None or R.reader_prompt_rows(dims, self.N, bound) == rows
        ws.fill_(0xff)                                           # (NaN wherever it is taken for floats)
        out = torch.full((self.N, self.Hq, self.D), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((self.N, self.Hq), 7.0, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        R.reader_prompt_attn(dims, self.q.cuda(), self.cache.k.cuda(), self.cache.v.cuda(), self.cache.table.cuda(), self.cu.cuda(),
                             torch.tensor(self.L, dtype=torch.int32, device="cuda"), out, lse, bound, ws, status)
        assert int(status) == status_want
        assert bool((out[sum(self.new):] == 7.0).all()) and bool((lse[sum(self.new):] == 7.0).all())
        return out.cpu(), lse.cpu()

    def want(self, b, scale=None):
        lo, hi, S = int(self.cu[b]), int(self.cu[b + 1]), self.L[b] + self.new[b]
        return P.attention(self.q[lo:hi], self.cache.rows(self.cache.k, b, S), self.cache.rows(self.cache.v, b, S), self.L[b], scale)

    def check(self, out, lse, only=None, scale=None):
        for b in range(self.B) if only is None else only:
            if not self.new[b]:
                continue
            lo, hi = int(self.cu[b]), int(self.cu[b + 1])
            o, s, bo, bs = self.want(b, scale)
            P.check(out[lo:hi], o, bo, "out of sequence %d" % b)
            P.check(lse[lo:hi], s, bs, "lse of sequence %d" % b)


HEADS = [(4, 1, 128), (3, 1, 64), (8, 2, 64), (2, 2, 128), (16, 1, 128), (6, 2, 128), (7, 1, 64)]
LENGTHS = [
    ([1], [0]), ([1], [63]), ([1], [64]), ([3, 0, 1, 70], [0, 5, 200, 3]), ([65], [0]), ([200, 129], [0, 0]),
    ([0, 0], [4, 0]), ([1] * 9, [0, 1, 15, 16, 17, 100, 511, 512, 777]), ([40, 1, 333], [1000, 2000, 5]),
]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("new,L", LENGTHS)
def test_attention(R, rows, Hq, Hkv, D, new, L):
    p = Problem(new, L, Hq, Hkv, D, seed=Hq + D + len(new))
    p.check(*p.run(R, rows))


@pytest.mark.parametrize("Hq,Hkv,D,new,L", [(4, 2, 128, [1500], [0]), (8, 2, 64, [900, 1, 700], [0, 2500, 300]), (2, 1, 128, [1, 1], [9000, 4000]),
                                             (4, 4, 64, [300], [6000]), (16, 2, 128, [257], [1023])])
def test_long(R, rows, Hq, Hkv, D, new, L):
    p = Problem(new, L, Hq, Hkv, D, seed=3)
    p.check(*p.run(R, rows))


def test_scale(R, rows):
    p = Problem([50], [20], 4, 2, 128, seed=4)
    p.check(*p.run(R, rows, sm_scale=0.3), scale=0.3)


@pytest.mark.parametrize("new,L", [([300], [0]), ([2, 1], [300, 700]), ([60], [900])])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_far_above_the_first_ones(R, rows, new, L, D):
    """Keys that grow along the sequence: later scores are hundreds above and below whatever came first."""
    p = Problem(new, L, 4, 2, D, seed=5)
    for b in range(len(new)):
        S = new[b] + L[b]
        page, slot = p.cache.place(b, S)
        p.cache.k[page, :, slot] *= torch.linspace(0, 60, S)[:, None, None].bfloat16()
    p.check(*p.run(R, rows))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("new,L", [([130], [0]), ([5], [60]), ([70, 3], [100, 40])])
def test_what_a_masked_position_holds_does_not_matter(R, rows, bad, new, L):
    """The last token's key and value are not numbers: every row in front of it is what it was."""
    p = Problem(new, L, 4, 2, 128, seed=6)
    clean, clean_lse = p.run(R, rows)
    p.check(clean, clean_lse)
    last = [int(p.cu[b + 1]) - 1 for b in range(p.B)]
    for b in range(p.B):
        page, slot = p.cache.place(b, 1, new[b] + L[b] - 1)
        p.cache.k[page, :, slot] = bad
        p.cache.v[page, :, slot] = bad
    out, lse = p.run(R, rows)
    front = torch.ones(p.N, dtype=torch.bool)
    front[last] = False
    # (a wavefront that meets them goes another way through the sums: the same to rounding, not to the bit)
    want = clean.double()
    P.check(out[front], want[front], 4 * P.BF16 * want[front].abs() + 0.02, "rows in front")
    P.check(lse[front], clean_lse[front].double(), torch.full_like(clean_lse[front].double(), 1e-4), "their lse")
    assert not bool(out[last].isfinite().any())


def test_pages_that_do_not_exist_are_left_out(R, rows):
    new, L = [80, 3], [70, 40]
    p = Problem(new, L, 4, 2, 64, seed=7)
    p.cache.table[0, 2], p.cache.table[0, 6] = 1 << 30, -5
    out, lse = p.run(R, rows, status_want=R.STATUS_BAD_PAGE)
    p.check(out, lse, only=[1])
    S = 150
    gone = torch.zeros(S, dtype=torch.bool)
    gone[32:48] = gone[96:112] = True
    page = torch.where(gone, 0, p.cache.table[0].long().clamp(0, p.cache.num_pages - 1)[torch.arange(S) // 16])
    k = p.cache.k[page, :, torch.arange(S) % 16].double().transpose(0, 1)
    v = p.cache.v[page, :, torch.arange(S) % 16].double().transpose(0, 1)
    for i in range(80):
        keep = (~gone) & (torch.arange(S) <= 70 + i)
        # a row of its own: what it sees, packed
        o, s, bo, bs = P.attention(p.q[i:i + 1], k[:, keep], v[:, keep], int(keep.sum()) - 1)
        P.check(out[i:i + 1], o, bo, "row %d" % i)
        P.check(lse[i:i + 1], s, bs, "lse of row %d" % i)


def test_rows_that_see_nothing(R, rows):
    p = Problem([20, 4], [0, 16], 4, 2, 128, seed=8)
    p.cache.table[:] = -1
    out, lse = p.run(R, rows, status_want=R.STATUS_BAD_PAGE)
    assert bool((out[:24] == 0).all()) and bool((lse[:24] == -math.inf).all())


def test_a_sequence_beyond_the_bound_is_cut(R, rows):
    p = Problem([30, 10], [100, 0], 4, 2, 64, seed=9)
    out, lse = p.run(R, rows, bound=110, status_want=R.STATUS_BAD_LENGTH)
    p.check(out, lse, only=[1])
    k, v = p.cache.rows(p.cache.k, 0, 110), p.cache.rows(p.cache.v, 0, 110)
    for i in (0, 9, 10, 29):
        S = min(101 + i, 110)
        o, s, bo, bs = P.attention(p.q[i:i + 1], k[:, :S], v[:, :S], S - 1)
        P.check(out[i:i + 1], o, bo, "row %d" % i)
        P.check(lse[i:i + 1], s, bs, "lse of row %d" % i)


def test_bounds_out_of_order_stay_inside_the_tensors(R, rows):
    p = Problem([4, 5, 6, 3], [20, 0, 3, 40], 4, 2, 64, seed=10, pad=0)
    for cu in ([0, 9, 4, 15, 18], [-4, 2, 2, 400, 401], [18] * 5, [9, 7, 5, 2, -7]):
        p.cu = torch.tensor(cu, dtype=torch.int32)
        dims = R.make_dims(4, 1, 4, 2, 64, p.cache.max_pages, 1, p.cache.num_pages, variant=1 if rows == 0 else 0)
        bound = p.cache.max_pages * 16
        ws = torch.empty(max(256, R.reader_prompt_workspace_bytes(dims, 18, bound)), dtype=torch.uint8, device="cuda")
        out, status = torch.zeros((18, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        R.reader_prompt_attn(dims, p.q.cuda(), p.cache.k.cuda(), p.cache.v.cuda(), p.cache.table.cuda(), p.cu.cuda(),
                             torch.tensor(p.L, dtype=torch.int32, device="cuda"), out, None, bound, ws, status)
        torch.cuda.synchronize()


def test_the_same_bits_every_time(R, rows):
    p = Problem([700, 1, 90], [10, 3000, 2000], 8, 2, 128, seed=11)
    a, la = p.run(R, rows)
    for _ in range(3):
        b, lb = p.run(R, rows)
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)) and torch.equal(la, lb)


@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 128), (12, 4, 64)])
def test_many_sequences(R, rows, Hq, Hkv, D):
    """More sequences than a wavefront has lanes, some of them without tokens."""
    gen = torch.Generator().manual_seed(12)
    new = [int(n) * (i % 5 != 3) for i, n in enumerate(torch.randint(0, 7, (150,), generator=gen))]
    L = [int(n) for n in torch.randint(0, 90, (150,), generator=gen)]
    p = Problem(new, L, Hq, Hkv, D, seed=13)
    p.check(*p.run(R, rows))


def test_the_largest_batch(R, rows):
    """More sequences than any table in LDS holds."""
    gen = torch.Generator().manual_seed(16)
    B = 4096
    new, L = torch.randint(0, 4, (B,), generator=gen).tolist(), torch.randint(0, 40, (B,), generator=gen).tolist()
    p = Problem(new, L, 4, 2, 64, seed=17)
    out, lse = p.run(R, rows)
    for b in list(range(0, 60)) + list(range(60, B - 40, 97)) + list(range(B - 40, B)):
        if new[b]:
            lo, hi = int(p.cu[b]), int(p.cu[b + 1])
            S = L[b] + new[b]
            want, want_lse, bound, bound_lse = P.attention(p.q[lo:hi], p.cache.rows(p.cache.k, b, S), p.cache.rows(p.cache.v, b, S), L[b])
            P.check(out[lo:hi], want, bound, "out of sequence %d" % b)
            P.check(lse[lo:hi], want_lse, bound_lse, "lse of sequence %d" % b)


def test_more_blocks_of_a_sequence_in_a_range_than_lanes(R, rows):
    if rows == 0:
        pytest.skip("the plain kernel has no ranges, and is too slow")
    n = 40000
    p = Problem([n], [5], 16, 1, 64, seed=18)
    out, lse = p.run(R, rows)
    k, v = p.cache.rows(p.cache.k, 0, n + 5), p.cache.rows(p.cache.v, 0, n + 5)
    for t in [0, 1, 63, 64, 1000, 7777, 20001, n - 65, n - 2, n - 1]:
        want, want_lse, bound, bound_lse = P.attention(p.q[t:t + 1], k[:, :t + 6], v[:, :t + 6], t + 5)
        P.check(out[t:t + 1], want, bound, "out of token %d" % t)
        P.check(lse[t:t + 1], want_lse, bound_lse, "lse of token %d" % t)


def test_no_positions_at_all(R, rows):
    p = Problem([5, 3], [0, 0], 4, 2, 64, seed=14)
    out, lse = p.run(R, rows, bound=0, status_want=R.STATUS_BAD_LENGTH)
    assert bool((out[:8] == 0).all()) and bool((lse[:8] == -math.inf).all())


def test_far_pages(R, rows):
    """Pages whose rows start behind 2^31 elements and 2^32 bytes of the cache."""
    Hq, Hkv, D, new, L = 4, 2, 128, [40, 1], [30, 100]
    p = Problem(new, L, Hq, Hkv, D, seed=15)
    n = (1 << 31) // (Hkv * 16 * D) + 40
    kc, vc = (torch.empty((n, Hkv, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    far = n - p.cache.num_pages
    kc[far:], vc[far:] = p.cache.k.cuda(), p.cache.v.cuda()
    table = torch.where(p.cache.table >= 0, p.cache.table + far, -1).int().cuda()
    dims = R.make_dims(2, 1, Hq, Hkv, D, p.cache.max_pages, 1, n, variant=1 if rows == 0 else 0)
    ws = torch.empty(max(256, R.reader_prompt_workspace_bytes(dims, p.N, 101)), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty((p.N, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.empty((p.N, Hq), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    R.reader_prompt_attn(dims, p.q.cuda(), kc, vc, table, p.cu.cuda(), torch.tensor(L, dtype=torch.int32, device="cuda"), out, lse, 101, ws, status)
    assert int(status) == 0
    p.check(out.cpu(), lse.cpu())
