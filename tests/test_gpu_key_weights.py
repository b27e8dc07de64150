"""reader_key_weights and reader_prompt_key_weights against their 64-bit form."""
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


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


HEADS = [(4, 1, 128), (3, 1, 64), (8, 2, 64), (2, 2, 128), (16, 1, 128), (6, 2, 128)]


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("decay", [0.0, 1.0, 0.75])
def test_step(R, Hq, Hkv, D, decay):
    gen = torch.Generator().manual_seed(D + Hq)
    T, accepted, L = 20, [1, 4, 9, 2, 1], [1, 0, 300, 63, 1000]     # (L: lengths in front of the step)
    B, mp = len(L), 9
    cache = P.Cache(gen, [l + n for l, n in zip(L, accepted)], Hkv, D)
    path = torch.full((B, mp), -1, dtype=torch.int32)
    for b in range(B):
        cache.fill(gen, b, L[b] + accepted[b])
        path[b, :accepted[b]] = torch.cat([torch.zeros(1), 1 + torch.randperm(T - 1, generator=gen)[:accepted[b] - 1].sort().values]).int()
    q = torch.randn((B, T, Hq, D), generator=gen).bfloat16()
    lse = 5 + torch.randn((B, Hq, T), generator=gen)
    W = cache.max_pages * 16 + 5
    old = torch.rand((B, Hkv, W), generator=gen)
    got = old.cuda() if decay else torch.full_like(old, math.nan).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dims = R.make_dims(B, T, Hq, Hkv, D, cache.max_pages, mp, cache.num_pages)
    lens = i32([l + n for l, n in zip(L, accepted)])
    R.reader_key_weights(dims, q.cuda(), lse.cuda(), path.cuda(), i32([n - 1 for n in accepted]), cache.k.cuda(), cache.table.cuda(), lens,
                         decay, got, 1009, status)
    assert int(status) == 0
    for b in range(B):
        n, S = accepted[b], L[b] + accepted[b]
        nodes = path[b, :n].long()
        w, bound = P.key_weights(q[b, nodes], lse[b][:, nodes].t(), cache.rows(cache.k, b, S), L[b])
        want = torch.zeros(Hkv, W, dtype=torch.float64) if decay == 0 else old[b].double().clone()
        want[:, :S] = (decay * old[b, :, :S].double() if decay else 0) + w
        full = torch.zeros(Hkv, W, dtype=torch.float64)
        full[:, :S] = bound + 3 * P.F32 * want[:, :S]
        P.check(got[b], want, full, "weights of sequence %d" % b)


@pytest.mark.parametrize("Hq,Hkv,D", HEADS)
@pytest.mark.parametrize("window", [0, 1, 7, 40, 1000])
def test_prompt(R, Hq, Hkv, D, window):
    gen = torch.Generator().manual_seed(D + window)
    new, L = [0, 1, 50, 130, 17], [5, 0, 0, 700, 47]
    B, N = len(new), sum(new) + 2
    cache = P.Cache(gen, [l + n for l, n in zip(L, new)], Hkv, D)
    for b in range(B):
        cache.fill(gen, b, L[b] + new[b])
    cu = torch.cat([torch.zeros(1), torch.cumsum(torch.tensor(new), 0)]).int()
    q = torch.randn((N, Hq, D), generator=gen).bfloat16()
    lse = 5 + torch.randn((N, Hq), generator=gen)
    W = cache.max_pages * 16
    got = torch.full((B, Hkv, W), math.nan, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dims = R.make_dims(B, 1, Hq, Hkv, D, cache.max_pages, 1, cache.num_pages)
    R.reader_prompt_key_weights(dims, q.cuda(), lse.cuda(), cu.cuda(), window, cache.k.cuda(), cache.table.cuda(), i32(L), 0.0, got, 830, status)
    assert int(status) == 0
    for b in range(B):
        S, n, end = L[b] + new[b], min(window, new[b]), int(cu[b + 1])
        want, full = torch.zeros(Hkv, W, dtype=torch.float64), torch.zeros(Hkv, W, dtype=torch.float64)
        if n:
            w, bound = P.key_weights(q[end - n:end], lse[end - n:end], cache.rows(cache.k, b, S), S - n)
            want[:, :S], full[:, :S] = w, bound
        P.check(got[b], want, full, "weights of sequence %d" % b)


def test_weights_of_one_row_add_up_to_one(R):
    """Against the attention's own log-sum-exp: the weights that a committed token spends are one per query head."""
    gen = torch.Generator().manual_seed(3)
    Hq, Hkv, D, new, L = 8, 2, 128, [33, 5], [400, 90]
    cache = P.Cache(gen, [l + n for l, n in zip(L, new)], Hkv, D)
    for b in range(2):
        cache.fill(gen, b, L[b] + new[b])
    N = sum(new)
    q = torch.randn((N, Hq, D), generator=gen).bfloat16().cuda()
    cu, lens = i32([0, 33, 38]), i32(L)
    dims = R.make_dims(2, 1, Hq, Hkv, D, cache.max_pages, 1, cache.num_pages)
    out, lse = torch.empty_like(q), torch.empty((N, Hq), device="cuda")
    ws = torch.empty(max(256, R.reader_prompt_workspace_bytes(dims, N, 433)), dtype=torch.uint8, device="cuda")
    kc, vc, table = cache.k.cuda(), cache.v.cuda(), cache.table.cuda()
    R.reader_prompt_attn(dims, q, kc, vc, table, cu, lens, out, lse, 433, ws)
    w = torch.empty((2, Hkv, cache.max_pages * 16), device="cuda")
    R.reader_prompt_key_weights(dims, q, lse, cu, 1000, kc, table, lens, 0.0, w, 433)
    total = w.double().sum(-1).cpu()
    want = torch.tensor(new, dtype=torch.float64)[:, None] * (Hq // Hkv)
    # every weight is off by a few score roundings (magnitudes of D = 128 products: sums below 16) on both sides
    assert bool(((total - want).abs() <= want * 2 * (132 * 16 + 64) * P.F32).all())


def test_sequences_that_do_not_fit_are_left_as_they_are(R):
    gen = torch.Generator().manual_seed(4)
    B, T, Hq, Hkv, D, mp = 6, 6, 2, 1, 64, 4
    cache = P.Cache(gen, [40] * B, Hkv, D)
    for b in range(B):
        cache.fill(gen, b, 40)
    q, lse = torch.randn((B, T, Hq, D), generator=gen).bfloat16().cuda(), torch.zeros((B, Hq, T), device="cuda")
    path = torch.tensor([[0, 1, 2, 3], [0, 6, -1, -1], [0, -2, 3, 3], [0, 1, -1, -1], [0, -1, -1, -1], [0, 1, 2, 4]], dtype=torch.int32)
    accept = [4, 1, 1, 1, 0, 3]                                # 4: more than max_path - 1
    lens = [40, 40, 40, 41, 49, 3]                             # 49: no pages for it; 3: shorter than its path
    status, w = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((B, Hkv, 48), 2.0, device="cuda")
    dims = R.make_dims(B, T, Hq, Hkv, D, cache.max_pages, mp, cache.num_pages)
    R.reader_key_weights(dims, q, lse, path.cuda(), i32(accept), cache.k.cuda(), cache.table.cuda(), i32(lens), 0.0, w, 40, status)
    assert int(status) == R.STATUS_BAD_PATH | R.STATUS_BAD_LENGTH
    assert bool((w == 2.0).all())


@pytest.mark.parametrize("decay", [0.0, 1.0])
def test_lengths_at_the_end_of_their_type(R, decay):
    """A length that new tokens, or a path, carry past 2^31 is one that does not fit."""
    gen = torch.Generator().manual_seed(14)
    cache = P.Cache(gen, [40, 40], 1, 64)
    q, lse = torch.randn((8, 2, 64), generator=gen).bfloat16().cuda(), torch.zeros((8, 2), device="cuda")
    lens = i32([2 ** 31 - 1, 2 ** 31 - 3])
    status, w = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((2, 1, 48), 2.0, device="cuda")
    dims = R.make_dims(2, 4, 2, 1, 64, cache.max_pages, 4, cache.num_pages)
    R.reader_prompt_key_weights(dims, q, lse, i32([0, 3, 8]), 2, cache.k.cuda(), cache.table.cuda(), lens, decay, w, 40, status)
    assert int(status) == R.STATUS_BAD_LENGTH
    status.zero_()
    for bad in (lens, i32([-2 ** 31, -1])):
        R.reader_key_weights(dims, q.view(2, 4, 2, 64), lse.view(2, 2, 4), i32([[0, 1, 2, 3]] * 2), i32([3, 0]), cache.k.cuda(), cache.table.cuda(),
                             bad, decay, w, 40, status)
    assert int(status) == R.STATUS_BAD_LENGTH | R.STATUS_BAD_PATH
    assert bool((w == 2.0).all())


def test_keys_behind_a_missing_page_draw_nothing(R):
    gen = torch.Generator().manual_seed(5)
    cache = P.Cache(gen, [100], 1, 64)
    cache.fill(gen, 0, 100)
    rows = cache.rows(cache.k, 0, 100)
    cache.table[0, 3] = cache.num_pages
    q, lse = torch.randn((1, 2, 64), generator=gen).bfloat16(), torch.full((1, 2), 4.0)
    w, status = torch.ones((1, 1, 112), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    dims = R.make_dims(1, 1, 2, 1, 64, cache.max_pages, 1, cache.num_pages)
    R.reader_prompt_key_weights(dims, q.cuda(), lse.cuda(), i32([0, 1]), 4, cache.k.cuda(), cache.table.cuda(), i32([99]), 0.5, w, 100, status)
    assert int(status) == R.STATUS_BAD_PAGE
    want, bound = P.key_weights(q, lse, rows, 99)
    want[:, 48:64], bound[:, 48:64] = 0, 0
    P.check(w[0, :, :100], want + 0.5, bound + 4 * P.F32 * (want + 0.5), "weights")
    assert bool((w[0, 0, 100:] == 1).all())


def test_rows_that_saw_nothing_give_nothing(R):
    gen = torch.Generator().manual_seed(6)
    cache = P.Cache(gen, [20], 1, 128)
    cache.fill(gen, 0, 20)
    q = torch.randn((3, 1, 128), generator=gen).bfloat16()
    lse = torch.tensor([[3.0], [-math.inf], [2.0]])
    w = torch.zeros((1, 1, 32), device="cuda")
    dims = R.make_dims(1, 1, 1, 1, 128, cache.max_pages, 1, cache.num_pages)
    R.reader_prompt_key_weights(dims, q.cuda(), lse.cuda(), i32([0, 3]), 3, cache.k.cuda(), cache.table.cuda(), i32([17]), 1.0, w, 20)
    a, ba = P.key_weights(q[:1], lse[:1], cache.rows(cache.k, 0, 20), 17)
    c, bc = P.key_weights(q[2:], lse[2:], cache.rows(cache.k, 0, 20), 19)
    P.check(w[0, :, :20], a + c, ba + bc + 3 * P.F32 * (a + c), "weights")


# rows of a sequence up to 16, 128, 256, 512, more; one to four sequences a lane, and more than are shared out; few and many
# keys: all that a workgroup's share depends on
@pytest.mark.parametrize("Hq,Hkv,D,B,longest,bound,window", [
    (2, 2, 64, 9, 8000, 8000, 5), (4, 1, 128, 3, 5000, 60000, 32), (8, 2, 64, 4, 3000, 20000, 40), (16, 2, 64, 5, 4000, 9000, 31),
    (16, 1, 64, 3, 5000, 11000, 37), (8, 1, 64, 2, 9000, 9000, 100), (16, 1, 128, 2, 2000, 17000, 66), (1, 1, 64, 70, 300, 3000, 4),
    (2, 1, 64, 130, 120, 2000, 8), (6, 3, 128, 250, 60, 300, 6), (2, 1, 64, 300, 90, 1500, 20)])
@pytest.mark.parametrize("decay", [0.0, 0.5])
def test_keys_shared_out(R, Hq, Hkv, D, B, longest, bound, window, decay):
    gen = torch.Generator().manual_seed(B + window)
    total = torch.randint(0, longest + 1, (B,), generator=gen).tolist()
    total[0], total[-1] = longest, 0
    new = [min(t, int(torch.randint(0, 2 * window, (1,), generator=gen))) for t in total]
    new[0] = min(longest, 2 * window)
    L, N = [t - n for t, n in zip(total, new)], sum(new)
    cache = P.Cache(gen, total, Hkv, D)
    for b in range(B):
        cache.fill(gen, b, total[b])
    W = bound + 3
    table = torch.full((B, (bound + 15) // 16), -1, dtype=torch.int32)
    table[:, :cache.max_pages] = cache.table
    cu = torch.cat([torch.zeros(1), torch.cumsum(torch.tensor(new), 0)]).int()
    q, lse = torch.randn((N, Hq, D), generator=gen).bfloat16(), 5 + torch.randn((N, Hq), generator=gen)
    old = torch.rand((B, Hkv, W), generator=gen)
    bad = B - 2                                              # one sequence with a length that does not fit: left as it is
    lens = L[:bad] + [bound + 1] + L[bad + 1:]
    dims = R.make_dims(B, 1, Hq, Hkv, D, table.shape[1], 1, cache.num_pages)
    args = (q.cuda(), lse.cuda(), cu.cuda(), window, cache.k.cuda(), table.cuda(), i32(lens), decay)
    got, status = old.cuda() if decay else torch.full_like(old, math.nan).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    was = got.clone()
    R.reader_prompt_key_weights(dims, *args, got, bound, status)
    again = was.clone()
    R.reader_prompt_key_weights(dims, *args, again, bound, status)
    assert int(status) == R.STATUS_BAD_LENGTH
    assert torch.equal(got.view(torch.int32), again.view(torch.int32))
    assert torch.equal(got[bad].view(torch.int32), was[bad].view(torch.int32))
    for b in range(B):
        if b == bad:
            continue
        S, n, end = total[b], min(window, new[b]), int(cu[b + 1])
        want, full = torch.zeros(Hkv, W, dtype=torch.float64), torch.zeros(Hkv, W, dtype=torch.float64)
        if decay:
            want = old[b].double()
            want[:, :S] *= decay
            full[:, :S] = 3 * P.F32 * want[:, :S]
        if n:
            w, error = P.key_weights(q[end - n:end], lse[end - n:end], cache.rows(cache.k, b, S), S - n)
            want[:, :S] += w
            full[:, :S] += error + 3 * P.F32 * w
        P.check(got[b], want, full, "weights of sequence %d" % b)
