"""reader_tree_qkv and reader_prompt_qkv against their 64-bit form: both rotations, partial ones, norms, both places for K/V."""
import math

import pytest
import torch

import prompt_helpers as P

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def R():
    from paper_2508_09072_amd import binding
    binding.load()
    return binding


def table(n, rot):
    if not rot:
        return None
    a = torch.arange(n, dtype=torch.float64)[:, None] * 500.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([a.cos(), a.sin()], 1).float()


def weights(gen, D, norm):
    return [(1 + 0.3 * torch.randn(D, generator=gen)).bfloat16() if norm else None for _ in range(2)]


def dev(t):
    return None if t is None else t.cuda()


def expected(qkv, Hq, Hkv, qn, kn, cs, pos, interleaved):
    q = P.norm_rotate(qkv[:, :Hq], qn, EPS, cs, pos, interleaved)
    k = P.norm_rotate(qkv[:, Hq:Hq + Hkv], kn, EPS, cs, pos, interleaved)
    return q, k, qkv[:, Hq + Hkv:].double()


SHAPES = [(8, 8, 64, 64), (6, 2, 128, 128), (16, 1, 128, 64), (5, 5, 64, 16), (12, 4, 128, 48), (4, 2, 128, 0)]


@pytest.mark.parametrize("Hq,Hkv,D,rot", SHAPES)
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("in_cache", [False, True])
def test_tree(R, Hq, Hkv, D, rot, norm, interleaved, in_cache):
    gen = torch.Generator().manual_seed(Hq * D + rot)
    B, T, L = 3, 19, torch.tensor([0, 37, 500], dtype=torch.int32)
    parents = torch.tensor([[-1] + [int(torch.randint(0, i, (1,), generator=gen)) for i in range(1, T)] for _ in range(B)], dtype=torch.int32)
    parents[1] = torch.arange(-1, T - 1)                       # a chain
    qkv = torch.randn((B, T, Hq + 2 * Hkv, D), generator=gen).bfloat16()
    qn, kn = weights(gen, D, norm)
    cs = table(600, rot)
    cache = P.Cache(gen, [int(x) + T for x in L], Hkv, D)
    base = torch.tensor([11, 37, 540], dtype=torch.int32)
    dims = R.make_dims(B, T, Hq, Hkv, D, cache.max_pages, T, cache.num_pages)
    q = torch.full((B, T, Hq, D), math.nan, dtype=torch.bfloat16, device="cuda")
    kt, vt = (None, None) if in_cache else (torch.full((B, T, Hkv, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    kc, vc, status = cache.k.cuda(), cache.v.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    R.reader_tree_qkv(dims, qkv.cuda(), parents.cuda(), L.cuda(), base.cuda(), dev(qn), dev(kn), EPS, dev(cs), interleaved, q, kt, vt,
                      kc, vc, cache.table.cuda(), status)
    assert int(status) == 0
    for b in range(B):
        pos = int(base[b]) + torch.tensor(P.depths(parents[b].tolist()))
        (wq, bq), (wk, bk), wv = expected(qkv[b], Hq, Hkv, qn, kn, cs, pos, interleaved)
        P.check(q[b], wq, bq, "q")
        if in_cache:
            page, slot = cache.place(b, T, int(L[b]))
            gk, gv = kc.cpu()[page, :, slot], vc.cpu()[page, :, slot]
            cache.k[page, :, slot], cache.v[page, :, slot] = gk, gv
        else:
            gk, gv = kt[b], vt[b]
        P.check(gk, wk, bk, "k")
        assert torch.equal(gv.double().cpu(), wv)
    # nothing but those rows has been written
    assert torch.equal(kc.cpu().view(torch.int16), cache.k.view(torch.int16)) and torch.equal(vc.cpu().view(torch.int16), cache.v.view(torch.int16))


@pytest.mark.parametrize("Hq,Hkv,D,rot", SHAPES)
@pytest.mark.parametrize("new", [[5], [0, 1, 33, 0, 16], [1] * 70, [0, 0], [2] + [0] * 200 + [3]])
def test_prompt(R, Hq, Hkv, D, rot, new):
    gen = torch.Generator().manual_seed(sum(new) + D)
    B, N = len(new), sum(new) + 3                                # three rows of padding
    L = [(7 * b) % 50 for b in range(B)]
    cu = torch.cat([torch.zeros(1), torch.cumsum(torch.tensor(new), 0)]).int()
    qkv = torch.randn((N, Hq + 2 * Hkv, D), generator=gen).bfloat16()
    qn, kn = weights(gen, D, True)
    cs = table(128, rot)
    cache = P.Cache(gen, [l + n for l, n in zip(L, new)], Hkv, D)
    dims = R.make_dims(B, 1, Hq, Hkv, D, cache.max_pages, 1, cache.num_pages)
    q = torch.full((N, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    kc, vc, status = cache.k.cuda(), cache.v.cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    R.reader_prompt_qkv(dims, qkv.cuda(), cu.cuda(), torch.tensor(L, dtype=torch.int32, device="cuda"), None, qn.cuda(), kn.cuda(), EPS,
                        dev(cs), False, q, kc, vc, cache.table.cuda(), status)
    assert int(status) == 0
    for b in range(B):
        lo, hi = int(cu[b]), int(cu[b + 1])
        if lo == hi:
            continue
        (wq, bq), (wk, bk), wv = expected(qkv[lo:hi], Hq, Hkv, qn, kn, cs, L[b] + torch.arange(hi - lo), False)
        P.check(q[lo:hi], wq, bq, "q")
        page, slot = cache.place(b, hi - lo, L[b])
        gk, gv = kc.cpu()[page, :, slot], vc.cpu()[page, :, slot]
        P.check(gk, wk, bk, "k")
        assert torch.equal(gv.double(), wv)
        cache.k[page, :, slot], cache.v[page, :, slot] = gk, gv
    assert torch.equal(kc.cpu().view(torch.int16), cache.k.view(torch.int16)) and torch.equal(vc.cpu().view(torch.int16), cache.v.view(torch.int16))
    assert bool((q[sum(new):] == 7.0).all())


def test_heads_that_nothing_is_done_to_keep_their_bits(R):
    gen = torch.Generator().manual_seed(1)
    B, T, Hq, Hkv, D = 1, 2, 2, 1, 128
    bits = torch.randint(-32768, 32768, (B, T, Hq + 2 * Hkv, D), generator=gen, dtype=torch.int32).to(torch.int16)
    dims = R.make_dims(B, T, Hq, Hkv, D, 1, 1, 1)
    q = torch.zeros((B, T, Hq, D), dtype=torch.bfloat16, device="cuda")
    kt, vt = (torch.zeros((B, T, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    R.reader_tree_qkv(dims, bits.view(torch.bfloat16).cuda(), torch.tensor([[-1, 0]], dtype=torch.int32, device="cuda"),
                      torch.zeros(1, dtype=torch.int32, device="cuda"), None, None, None, EPS, None, False, q, kt, vt, None, None, None)
    got = torch.cat([t.cpu().view(torch.int16) for t in (q, kt, vt)], 2)
    assert torch.equal(got, bits)


def test_what_the_tables_do_not_hold_is_left_out(R):
    gen = torch.Generator().manual_seed(5)
    B, T, Hq, Hkv, D = 3, 4, 2, 1, 64
    qkv = torch.randn((B, T, Hq + 2 * Hkv, D), generator=gen).bfloat16().cuda()
    parents = torch.tensor([[-1, 0, 1, 2], [-1, 0, 5, 0], [-1, 0, 0, 0]], dtype=torch.int32, device="cuda")
    L = torch.tensor([30, 3, 14], dtype=torch.int32, device="cuda")
    page_table = torch.tensor([[0, 1], [2, -1], [3, 9]], dtype=torch.int32, device="cuda")
    cs = table(33, 64).cuda()

    def run(lens, status_want):
        kc, vc = (torch.full((4, Hkv, 16, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        q = torch.full((B, T, Hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        R.reader_tree_qkv(R.make_dims(B, T, Hq, Hkv, D, 2, 1, 4), qkv, parents, lens, None, None, None, EPS, cs, False, q, None, None, kc, vc,
                          page_table, status)
        assert int(status) == status_want
        return q.cpu(), kc.cpu()
    q, kc = run(L, R.STATUS_BAD_LENGTH | R.STATUS_BAD_TREE | R.STATUS_BAD_PAGE)
    assert bool((q[0, 3] == 7.0).all()) and not bool((q[0, 2] == 7.0).any())       # position 33 is not in the rotation table
    assert bool(kc[0, 0, :14].isnan().all()) and not bool(kc[1, 0, 14:16].isnan().any())   # positions 30, 31; 32 has no page
    assert not bool(kc[3, 0, 14:16].isnan().any())                                  # sequence 2: 14, 15; the page behind them does not exist
    q, kc = run(torch.tensor([-1, 3, 0], dtype=torch.int32, device="cuda"), R.STATUS_BAD_LENGTH | R.STATUS_BAD_TREE)
    assert bool((q[0, 0] == 7.0).all()) and bool(kc[:2].isnan().all())


def test_bounds_out_of_order_stay_inside_the_tensors(R):
    gen = torch.Generator().manual_seed(6)
    B, N, Hq, Hkv, D = 4, 9, 2, 1, 64
    qkv = torch.randn((N, Hq + 2 * Hkv, D), generator=gen).bfloat16().cuda()
    for cu in ([0, 5, 3, 7, 9], [-4, 2, 2, 40, 41], [9, 9, 9, 9, 9], [3, 2, 1, 0, -7]):
        kc, vc = (torch.full((8, Hkv, 16, D), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        q, status = torch.zeros((N, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        R.reader_prompt_qkv(R.make_dims(B, 1, Hq, Hkv, D, 2, 1, 8), qkv, torch.tensor(cu, dtype=torch.int32, device="cuda"),
                            torch.zeros(B, dtype=torch.int32, device="cuda"), None, None, None, EPS, None, False, q, kc, vc,
                            torch.arange(8, dtype=torch.int32, device="cuda").view(4, 2), status)
        torch.cuda.synchronize()
