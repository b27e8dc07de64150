"""Packed bounds and lengths that are out of order, out of range or start behind row 0: the status, the rows of sequences that
are as they should be, and nothing else written."""
import pytest
import torch

import prompt_helpers as P

pytestmark = pytest.mark.gpu
GUARD = 5                                                         # rows, or pages, in front of and behind every output


@pytest.fixture(scope="module")
def R():
    from paper_2508_09072_amd import binding
    binding.load()
    return binding


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def bits(t):
    return t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32)


class Guarded:
    """An output in the middle of a larger buffer, all of which holds `value`."""

    def __init__(self, shape, dtype, value=7.0, inside=None):
        self.all = torch.full((shape[0] + 2 * GUARD, *shape[1:]), value, dtype=dtype, device="cuda")
        self.t = self.all[GUARD:GUARD + shape[0]]
        if inside is not None:
            self.t.copy_(inside)
        self.was = self.all.clone()

    def unchanged(self, written=()):
        """Nothing but these rows of the output is other than it was."""
        same = torch.ones(self.all.shape[0], dtype=torch.bool)
        same[[GUARD + i for i in written]] = False
        assert torch.equal(bits(self.all)[same.cuda()], bits(self.was)[same.cuda()])


N = 18
# bounds, whether something is wrong with them, and who owns which rows for certain: (sequence, its first row, rows)
TABLES = [
    ([18] * 5, False, []),
    ([3, 3, 9, 9, 14], False, [(1, 3, range(3, 9)), (3, 9, range(9, 14))]),
    ([2, 7, 8, 10, 18], False, [(0, 2, range(2, 7)), (1, 7, [7]), (2, 8, [8, 9]), (3, 10, range(10, 18))]),
    ([0, 9, 4, 15, 18], True, [(0, 0, range(0, 4)), (2, 4, range(9, 15)), (3, 15, range(15, 18))]),
    ([-4, 2, 2, 400, 401], True, [(0, 0, [0, 1]), (2, 2, range(2, 18))]),
    ([9, 7, 5, 2, -7], True, []),
]
TOUCHED = {3: range(0, 18)}                                       # (a row that two sequences claim may be either's)


@pytest.mark.parametrize("case", range(len(TABLES)))
@pytest.mark.parametrize("D", [64, 128])
def test_projections(R, case, D):
    cu, wrong, owned = TABLES[case]
    gen = torch.Generator().manual_seed(40 + case)
    Hq, Hkv, L = 4, 2, [20, 0, 3, 40]
    cache = P.Cache(gen, [l + N for l in L], Hkv, D)
    qkv = torch.randn((N, Hq + 2 * Hkv, D), generator=gen).bfloat16()
    a = torch.arange(80, dtype=torch.float64)[:, None] * 500.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)
    cs = torch.cat([a.cos(), a.sin()], 1).float()
    dims = R.make_dims(4, 1, Hq, Hkv, D, cache.max_pages, 1, cache.num_pages)
    q, status = Guarded((N, Hq, D), torch.bfloat16), i32([0])
    kc, vc = Guarded(cache.k.shape, torch.bfloat16, inside=cache.k), Guarded(cache.v.shape, torch.bfloat16, inside=cache.v)
    R.reader_prompt_qkv(dims, qkv.cuda(), i32(cu), i32(L), None, None, None, 0.0, cs.cuda(), False, q.t, kc.t, vc.t, cache.table.cuda(), status)
    assert int(status) == (R.STATUS_BAD_LENGTH if wrong else 0)
    q.unchanged(TOUCHED.get(case, [t for _, _, r in owned for t in r]))
    k, v = kc.t.cpu(), vc.t.cpu()
    for b, first, mine in owned:
        for t in mine:
            pos = torch.tensor([L[b] + t - first])
            wq, bq = P.norm_rotate(qkv[t:t + 1, :Hq], None, 0.0, cs, pos, False)
            P.check(q.t[t:t + 1], wq, bq, "q of row %d" % t)
            wk, bk = P.norm_rotate(qkv[t:t + 1, Hq:Hq + Hkv], None, 0.0, cs, pos, False)
            page, slot = cache.place(b, 1, L[b] + t - first)
            P.check(k[page, :, slot], wk, bk, "k of row %d" % t)
            assert torch.equal(v[page, :, slot].double(), qkv[t:t + 1, Hq + Hkv:].double())
            k[page, :, slot], v[page, :, slot] = cache.k[page, :, slot], cache.v[page, :, slot]
    if case in TOUCHED:                                           # rows 4..8 of sequence 0, or rows 0..4 of sequence 2
        for b, start in ((0, L[0] + 4), (2, L[2])):
            page, slot = cache.place(b, 5, start)
            k[page, :, slot], v[page, :, slot] = cache.k[page, :, slot], cache.v[page, :, slot]
    # nothing else in any page
    assert torch.equal(bits(k), bits(cache.k)) and torch.equal(bits(v), bits(cache.v))
    pages = range(cache.num_pages)
    kc.unchanged(pages)
    vc.unchanged(pages)


@pytest.mark.parametrize("B", [3, 100])
def test_projections_of_lengths_that_are_none(R, B):
    """A negative length of a sequence without tokens, and many sequences with one bound that goes back."""
    gen = torch.Generator().manual_seed(50)
    qkv = torch.randn((B, 3, 64), generator=gen).bfloat16().cuda()
    cu, lens = torch.arange(B + 1), torch.zeros(B, dtype=torch.int64)
    if B == 3:
        cu, lens[1] = torch.tensor([0, 2, 2, 3]), -1
    else:
        cu[60] = 2
    kc, vc = (Guarded((B, 1, 16, 64), torch.bfloat16) for _ in range(2))
    q, status = Guarded((B, 1, 64), torch.bfloat16), i32([0])
    R.reader_prompt_qkv(R.make_dims(B, 1, 1, 1, 64, 1, 1, B), qkv, i32(cu), i32(lens), None, None, None, 0.0, None, False, q.t, kc.t, vc.t,
                        torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1), status)
    assert int(status) == R.STATUS_BAD_LENGTH
    q.unchanged(range(B))
    kc.unchanged(range(B))
    vc.unchanged(range(B))
