"""reader_kv_evict: which rows stay, where they go, what is left alone; to the bit."""
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


def bits(t):
    return t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32)


def run(R, cache, L, w, keep, recent, status_want=0):
    NL, B, Hkv = w.shape[:3]
    dims = R.make_dims(B, 1, Hkv, Hkv, cache.D, cache.max_pages, 1, cache.num_pages)
    ws = torch.full((max(4, R.reader_kv_evict_workspace_bytes(dims, NL, keep)),), 0xff, dtype=torch.uint8, device="cuda")
    k, v, lens, gw = cache.k.cuda(), cache.v.cuda(), torch.tensor(L, dtype=torch.int32, device="cuda"), w.cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    R.reader_kv_evict(dims, keep, recent, k, v, cache.table.cuda(), lens, gw, ws, status)
    assert int(status) == status_want
    return k.cpu(), v.cpu(), lens.cpu().tolist(), gw.cpu()


def expect(cache, L, w, keep, recent, skip=()):
    k, v, gw, lens = cache.k.clone(), cache.v.clone(), w.clone(), list(L)
    for b, n in enumerate(L):
        if n <= keep or b in skip:
            continue
        lens[b] = keep
        page, slot = cache.place(b, n)
        for layer in range(w.shape[0]):
            for h in range(w.shape[2]):
                src = torch.tensor(P.evict(w[layer, b, h, :n], keep, recent), dtype=torch.long)
                for c, o in ((k, cache.k), (v, cache.v)):
                    c[layer, page[:keep], h, slot[:keep]] = o[layer, page[src], h, slot[src]]
                gw[layer, b, h, :n] = 0
                gw[layer, b, h, :keep] = w[layer, b, h, src]
    return k, v, lens, gw


def make(gen, NL, L, Hkv, D, kind="normal"):
    cache = P.Cache(gen, L, Hkv, D, lead=(NL,))
    for b, n in enumerate(L):
        if n:
            cache.fill(gen, b, n)
    w = torch.rand((NL, len(L), Hkv, cache.max_pages * 16 + 3), generator=gen)
    if kind == "ties":
        w = (w * 4).floor()
    elif kind == "equal":
        w = torch.ones_like(w)
    elif kind == "wild":
        w = torch.randn(w.shape, generator=gen) * 10.0 ** torch.randint(-38, 38, w.shape, generator=gen).float()
        w[torch.rand(w.shape, generator=gen) < 0.1] = math.nan
        w[torch.rand(w.shape, generator=gen) < 0.1] = -0.0
        w[torch.rand(w.shape, generator=gen) < 0.1] = 0.0
        w[torch.rand(w.shape, generator=gen) < 0.05] = math.inf
        w[torch.rand(w.shape, generator=gen) < 0.05] = -math.inf
    return cache, w


def same(got, want):
    for g, x in zip((got[0], got[1], got[3]), (want[0], want[1], want[3])):
        assert torch.equal(bits(g), bits(x))
    assert got[2] == want[2]


@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "wild"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("NL,L,Hkv,keep,recent", [
    (1, [50], 1, 20, 5), (2, [3, 0, 700, 64, 65], 2, 64, 10), (3, [130, 17], 2, 16, 16), (1, [100, 1], 1, 1, 0), (1, [33], 1, 0, 0),
    (1, [1500], 2, 1499, 0), (1, [1100, 2000], 1, 1024, 1000),
])
def test_evict(R, kind, D, NL, L, Hkv, keep, recent):
    gen = torch.Generator().manual_seed(keep + D)
    cache, w = make(gen, NL, L, Hkv, D, kind)
    same(run(R, cache, L, w, keep, recent), expect(cache, L, w, keep, recent))


def test_more_positions_than_a_workgroup_holds(R):
    gen = torch.Generator().manual_seed(1)
    L, keep = [40000], 9000
    cache, w = make(gen, 1, L, 1, 64, "ties")
    same(run(R, cache, L, w, keep, 100), expect(cache, L, w, keep, 100))


def test_sequences_that_do_not_fit_are_left_as_they_are(R):
    gen = torch.Generator().manual_seed(2)
    L, keep = [60, 60, 60, 60], 32
    cache, w = make(gen, 2, L, 2, 64)
    bad = list(L)
    bad[0], bad[3] = cache.max_pages * 16 + 1, -4
    good = cache.table.clone()
    cache.table[1, 2] = cache.num_pages
    got = run(R, cache, bad, w, keep, 4, R.STATUS_BAD_LENGTH | R.STATUS_BAD_PAGE)
    cache.table = good
    want = expect(cache, L, w, keep, 4, skip=(0, 1, 3))
    assert got[2] == [bad[0], 60, keep, -4]
    for g, x in zip((got[0], got[1], got[3]), (want[0], want[1], want[3])):
        assert torch.equal(bits(g), bits(x))


@pytest.mark.parametrize("kind", ["normal", "ties"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("NL,L,Hkv,keep,recent", [
    (4, [700, 90], 4, 333, 20), (3, [300, 20, 150], 4, 100, 0), (11, [40], 3, 17, 17), (5, [1500, 900, 1200], 4, 1100, 90),
    (17, [129, 64], 1, 64, 1), (9, [600, 1, 0, 599], 1, 513, 100),
])
def test_many_layers_and_heads(R, kind, D, NL, L, Hkv, keep, recent):
    """32 (layer, sequence, kv head) triples and more, whose rows move in wider slices; several passes of 512 rows, not whole ones."""
    gen = torch.Generator().manual_seed(keep + D + NL)
    cache, w = make(gen, NL, L, Hkv, D, kind)
    same(run(R, cache, L, w, keep, recent), expect(cache, L, w, keep, recent))
