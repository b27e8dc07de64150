"""Packed bounds and lengths that are out of order, out of range or start behind row 0: the same status whatever kernel runs,
the rows of sequences that are as they should be, and nothing else written."""
import math

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


@pytest.fixture(params=[0, 16, 32, 33, 64, 128, 256])
def rows(R, request):
    R.reader_tuning_override(R.TUNE_PROMPT_ROWS, request.param or -1)
    yield request.param
    R.reader_tuning_override(R.TUNE_PROMPT_ROWS, -1)


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
def test_attention(R, rows, case, D):
    cu, wrong, owned = TABLES[case]
    gen = torch.Generator().manual_seed(20 + case)
    Hq, Hkv, L = 4, 2, [20, 0, 3, 40]
    cache = P.Cache(gen, [l + N for l in L], Hkv, D)
    for b in range(4):
        cache.fill(gen, b, L[b] + N)
    q = torch.randn((N, Hq, D), generator=gen).bfloat16()
    dims = R.make_dims(4, 1, Hq, Hkv, D, cache.max_pages, 1, cache.num_pages, variant=1 if rows == 0 else 0)
    bound = cache.max_pages * 16
    ws = torch.full((max(256, R.reader_prompt_workspace_bytes(dims, N, bound)),), 0xff, dtype=torch.uint8, device="cuda")
    out, lse, status = Guarded((N, Hq, D), torch.bfloat16), Guarded((N, Hq), torch.float32), i32([0])
    R.reader_prompt_attn(dims, q.cuda(), cache.k.cuda(), cache.v.cuda(), cache.table.cuda(), i32(cu), i32(L), out.t, lse.t, bound, ws, status)
    assert int(status) == (R.STATUS_BAD_LENGTH if wrong else 0)
    touched = TOUCHED.get(case, [t for _, _, r in owned for t in r])
    out.unchanged(touched)
    lse.unchanged(touched)
    for b, first, mine in owned:
        end = max(mine) + 1
        S = L[b] + end - first
        o, s, bo, bs = P.attention(q[first:end], cache.rows(cache.k, b, S), cache.rows(cache.v, b, S), L[b])
        for t in mine:
            P.check(out.t[t], o[t - first], bo[t - first], "row %d" % t)
            P.check(lse.t[t], s[t - first], bs[t - first], "lse of row %d" % t)


@pytest.mark.parametrize("lens,bound", [([5, -3, 9, 2], 100), ([5, 101, 9, 2], 100), ([5, -2 ** 31, 9, 2 ** 31 - 1], 100)])
def test_lengths_of_sequences_without_tokens(R, rows, lens, bound):
    """Nobody reads their keys, but the table is wrong all the same."""
    gen = torch.Generator().manual_seed(30)
    Hq, Hkv, D, new = 4, 2, 64, [6, 0, 7, 0]
    cache = P.Cache(gen, [112] * 4, Hkv, D)
    for b in (0, 2):
        cache.fill(gen, b, lens[b] + new[b])
    q = torch.randn((13, Hq, D), generator=gen).bfloat16()
    dims = R.make_dims(4, 1, Hq, Hkv, D, cache.max_pages, 1, cache.num_pages, variant=1 if rows == 0 else 0)
    ws = torch.full((max(256, R.reader_prompt_workspace_bytes(dims, 13, bound)),), 0xff, dtype=torch.uint8, device="cuda")
    out, status = torch.zeros((13, Hq, D), dtype=torch.bfloat16, device="cuda"), i32([0])
    R.reader_prompt_attn(dims, q.cuda(), cache.k.cuda(), cache.v.cuda(), cache.table.cuda(), i32([0, 6, 6, 13, 13]), i32(lens), out, None, bound,
                         ws, status)
    assert int(status) == R.STATUS_BAD_LENGTH
    for b, lo, hi in ((0, 0, 6), (2, 6, 13)):
        S = lens[b] + hi - lo
        o, _, bo, _ = P.attention(q[lo:hi], cache.rows(cache.k, b, S), cache.rows(cache.v, b, S), lens[b])
        P.check(out[lo:hi], o, bo, "sequence %d" % b)


@pytest.mark.parametrize("B", [100, 300, 4096])
def test_one_bad_bound_among_many(R, rows, B):
    gen = torch.Generator().manual_seed(B)
    Hq, Hkv, D, n = 2, 1, 64, B + 20
    cu = torch.arange(B + 1)
    cu[B // 2] = 1                                                # goes back
    cache = P.Cache(gen, [16] * B, Hkv, D)
    q = torch.randn((n, Hq, D), generator=gen).bfloat16()
    cache.k.zero_(), cache.v.zero_()
    dims = R.make_dims(B, 1, Hq, Hkv, D, 1, 1, cache.num_pages, variant=1 if rows == 0 else 0)
    ws = torch.full((max(256, R.reader_prompt_workspace_bytes(dims, n, 16)),), 0xff, dtype=torch.uint8, device="cuda")
    out, status = Guarded((n, Hq, D), torch.bfloat16), i32([0])
    # (the sequence behind the bad bound runs to its own end over all rows in front: its keys then pass the bound on lengths)
    R.reader_prompt_attn(dims, q.cuda(), cache.k.cuda(), cache.v.cuda(), cache.table.cuda(), i32(cu), i32([0] * B), out.t, None, 16, ws, status)
    assert int(status) == R.STATUS_BAD_LENGTH
    out.unchanged(range(B))


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


@pytest.mark.parametrize("case", range(len(TABLES)))
@pytest.mark.parametrize("decay", [0.0, 0.5])
def test_key_weights(R, case, decay):
    cu, wrong, _ = TABLES[case]
    gen = torch.Generator().manual_seed(60 + case)
    Hq, Hkv, D, L, window = 4, 2, 64, [20, 0, 3, 40], 7
    cache = P.Cache(gen, [l + N for l in L], Hkv, D)
    for b in range(4):
        cache.fill(gen, b, L[b] + N)
    q, lse = torch.randn((N, Hq, D), generator=gen).bfloat16(), 3 + torch.randn((N, Hq), generator=gen)
    W = cache.max_pages * 16
    old = torch.rand((4, Hkv, W), generator=gen)
    w, status = Guarded((4, Hkv, W), torch.float32, inside=old), i32([0])
    dims = R.make_dims(4, 1, Hq, Hkv, D, cache.max_pages, 1, cache.num_pages)
    R.reader_prompt_key_weights(dims, q.cuda(), lse.cuda(), i32(cu), window, cache.k.cuda(), cache.table.cuda(), i32(L), decay, w.t, W, status)
    assert int(status) == (R.STATUS_BAD_LENGTH if wrong else 0)
    good = [b for b in range(4) if 0 <= cu[b] <= cu[b + 1] <= N]
    w.unchanged(good)
    for b in good:
        n, S, end = min(window, cu[b + 1] - cu[b]), L[b] + cu[b + 1] - cu[b], cu[b + 1]
        want = old[b].double() if decay else torch.zeros(Hkv, W, dtype=torch.float64)
        want[:, :S] *= decay
        error = torch.zeros_like(want)
        if n:
            x, bx = P.key_weights(q[end - n:end], lse[end - n:end], cache.rows(cache.k, b, S), S - n)
            want[:, :S] += x
            error[:, :S] = bx
        error[:, :S] += 3 * P.F32 * want[:, :S]
        P.check(w.t[b], want, error, "weights of sequence %d" % b)


def test_key_weights_without_any_position(R):
    """No position is allowed: lengths that have some do not fit, and are said to."""
    gen = torch.Generator().manual_seed(70)
    cache = P.Cache(gen, [20], 1, 64)
    cache.fill(gen, 0, 20)
    q, lse = torch.randn((2, 2, 64), generator=gen).bfloat16().cuda(), torch.zeros((2, 2), device="cuda")
    dims = R.make_dims(1, 1, 2, 1, 64, cache.max_pages, 1, cache.num_pages)
    for decay in (0.0, 1.0):
        w, status = torch.full((1, 1, 32), 2.0, device="cuda"), i32([0])
        R.reader_prompt_key_weights(dims, q, lse, i32([0, 2]), 2, cache.k.cuda(), cache.table.cuda(), i32([5]), decay, w, 0, status)
        assert int(status) == R.STATUS_BAD_LENGTH and bool((w == 2.0).all())
        status.zero_()
        R.reader_prompt_key_weights(dims, q, lse, i32([0, 0]), 2, cache.k.cuda(), cache.table.cuda(), i32([0]), decay, w, 0, status)
        assert int(status) == 0 and bool((w == (2.0 if decay else 0.0)).all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,L", [(1, 40000), (9, 20000), (130, 9000)])
def test_nothing_behind_the_workspace(R, rows, D, n, L):
    """Every range of a launch leaves records, and the workspace is no larger than it has to be."""
    gen = torch.Generator().manual_seed(80)
    Hq, Hkv = 16, 8
    cache = P.Cache(gen, [L + n], Hkv, D)
    cache.fill(gen, 0, L + n)
    q = torch.randn((n, Hq, D), generator=gen).bfloat16()
    dims = R.make_dims(1, 1, Hq, Hkv, D, cache.max_pages, 1, cache.num_pages, variant=1 if rows == 0 else 0)
    need = R.reader_prompt_workspace_bytes(dims, n, L + n)
    ws = torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda")
    out, status = torch.zeros((n, Hq, D), dtype=torch.bfloat16, device="cuda"), i32([0])
    R.reader_prompt_attn(dims, q.cuda(), cache.k.cuda(), cache.v.cuda(), cache.table.cuda(), i32([0, n]), i32([L]), out, None, L + n,
                         ws[256:256 + need], status)
    assert int(status) == 0
    assert bool((ws[:256] == 0xff).all()) and bool((ws[256 + need:] == 0xff).all())
    k, v = cache.rows(cache.k, 0, L + n), cache.rows(cache.v, 0, L + n)
    for t in {0, n - 1}:
        o, _, bo, _ = P.attention(q[t:t + 1], k[:, :L + t + 1], v[:, :L + t + 1], L + t)
        P.check(out[t:t + 1], o, bo, "row %d" % t)
