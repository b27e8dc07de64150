"""Where rows of the cache in 4 bits and pages end up: bounds and lengths that are none, places behind 2^32 bytes; and a batch in which
single tokens stand beside a chunk of hundreds."""
import pytest
import torch

import kvq_helpers as K
import prompt_helpers as P
from test_gpu_kvq import Problem, R, i32, rows, status_word  # noqa: F401

pytestmark = pytest.mark.gpu
BAD = [
    # bounds, lengths, and which rows of which sequence go to which positions: for certain, and maybe besides
    ([-3, 10, 20, 400], [1, 2, 3], [(0, 0, 10, 1), (1, 10, 20, 2), (2, 20, 30, 3)], []),
    ([0, 25, 10, 30], [1, 2, 3], [(0, 0, 10, 1), (2, 25, 30, 18)], [(0, 10, 25, 11), (2, 10, 25, 3)]),
    ([30, 20, 10, 0], [1, 2, 3], [], []),
    ([0, 10, 20, 30], [-1, -2 ** 31, 2 ** 31 - 1], [], []),
    ([0, 10, 20, 30], [4, -1, 0], [(0, 0, 10, 4), (2, 20, 30, 0)], []),
]


@pytest.mark.parametrize("cu,L,certain,maybe", BAD)
@pytest.mark.parametrize("D", [64, 128])
def test_rows_are_stored_where_they_belong_or_nowhere(R, cu, L, certain, maybe, D):  # noqa: F811
    gen = torch.Generator().manual_seed(6)
    cache = K.Cache(gen, [48] * 3, 2, D)
    k, v = (torch.randn((30, 2, D), generator=gen).bfloat16() for _ in range(2))
    want, free = cache.data.clone(), torch.zeros_like(cache.data, dtype=torch.bool)
    for b, lo, hi, at in certain:
        K.put(want, cache.place(b, at + hi - lo, at), k[lo:hi], False)
        K.put(want, cache.place(b, at + hi - lo, at), v[lo:hi], True)
    for b, lo, hi, at in maybe:
        for page, slot in cache.place(b, at + hi - lo, at):
            free[page][:, K.row_bytes(D, slot)] = True
    got, status = cache.data.cuda(), status_word()
    dims = R.make_dims(3, 1, 2, 2, D, cache.max_pages, 1, cache.num_pages)
    R.reader_kvq_store(dims, k.cuda(), v.cuda(), i32(cu), i32(L), got, cache.table.cuda(), status)
    assert int(status) == R.STATUS_BAD_LENGTH
    assert torch.equal(got.cpu()[~free], want[~free])


def far_cache(cache, lead=()):
    """The cache's pages as the last ones of more than 2^32 bytes, in front of which all is 7; and its table."""
    n = (1 << 32) // (cache.Hkv * 17 * cache.D) + 40
    data = torch.full((*lead, n, cache.Hkv, 17 * cache.D), 7, dtype=torch.uint8, device="cuda")
    far = n - cache.num_pages
    data[..., far:, :, :] = cache.data.cuda()
    return n, far, data, torch.where(cache.table >= 0, cache.table + far, -1).int().cuda()


def the_same(data, far, want):
    assert torch.equal(data[..., far:, :, :].cpu(), want) and bool((data[..., :far, :, :] == 7).all())


def test_rows_stored_in_far_pages(R):  # noqa: F811
    gen = torch.Generator().manual_seed(31)
    cache = K.Cache(gen, [60, 70], 2, 128)
    n, far, data, table = far_cache(cache)
    k, v = (torch.randn((2, 33, 2, 128), generator=gen).bfloat16() for _ in range(2))
    want, status = cache.data.clone(), status_word()
    for b, at in ((0, 20), (1, 37)):
        K.put(want, cache.place(b, at + 33, at), k[b], False)
        K.put(want, cache.place(b, at + 33, at), v[b], True)
    R.reader_kvq_store(R.make_dims(2, 33, 2, 2, 128, cache.max_pages, 1, n), k.cuda(), v.cuda(), None, i32([20, 37]), data, table, status)
    assert int(status) == 0
    the_same(data, far, want)


def test_far_pages_are_packed_into_far_pages(R):  # noqa: F811
    """Of two layers: the second begins behind 2^32 bytes of the cache in 4 bits, and 2^32 values of the other."""
    gen = torch.Generator().manual_seed(32)
    L = [50, 33]
    src, dst = P.Cache(gen, L, 2, 128, lead=(2,)), K.Cache(gen, L, 2, 128, lead=(2,))
    for b in range(2):
        src.fill(gen, b, L[b])
    want, status = dst.data.clone(), status_word()
    for b in range(2):
        page, slot = src.place(b, L[b])
        for layer in range(2):
            K.put(want[layer], dst.place(b, L[b]), src.k[layer, page, :, slot], False)
            K.put(want[layer], dst.place(b, L[b]), src.v[layer, page, :, slot], True)
    n, far, data, table = far_cache(dst, (2,))
    m = (1 << 32) // (2 * 16 * 128) + 20
    k, v = (torch.empty((2, m, 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[:, m - src.num_pages:], v[:, m - src.num_pages:] = src.k.cuda(), src.v.cuda()
    from_table = torch.where(src.table >= 0, src.table + m - src.num_pages, -1).int().cuda()
    R.reader_kvq_pack(R.make_dims(2, 1, 2, 2, 128, dst.max_pages, 1, n), k, v, from_table, None, i32(L), max(L), data, table, status)
    assert int(status) == 0
    the_same(data, far, want)


def test_the_accepted_path_moves_in_far_pages(R):  # noqa: F811
    gen = torch.Generator().manual_seed(33)
    L, T, path = [20, 45], 24, [0, 3, 5, 20]
    cache = K.Cache(gen, [x + T for x in L], 2, 128, lead=(2,))
    cache.fill_all(gen, [x + T for x in L])
    want, status = cache.data.clone(), status_word()
    for b in range(2):
        for j, node in enumerate(path):
            (p0, s0), (p1, s1) = cache.place(b, L[b] + node + 1, L[b] + node)[0], cache.place(b, L[b] + j + 1, L[b] + j)[0]
            want[:, p1][..., K.row_bytes(128, s1)] = cache.data[:, p0][..., K.row_bytes(128, s0)]
    n, far, data, table = far_cache(cache, (2,))
    lens = i32(L)
    R.reader_kvq_compact_layers(R.make_dims(2, T, 2, 2, 128, cache.max_pages, 4, n), i32([path, path]), i32([3, 3]), data, table, lens, status)
    assert int(status) == 0 and lens.tolist() == [24, 49]
    the_same(data, far, want)


def test_far_pages_are_copied_on_a_write(R):  # noqa: F811
    """Two sequences that share a partly filled page behind 2^32 bytes; the page that the copy takes lies there too."""
    n, page_bytes = (1 << 32) // 4096 + 9, 4096
    cache = torch.randint(0, 256, (2, n, page_bytes), dtype=torch.uint8, device="cuda")
    refs = torch.ones((n,), dtype=torch.int32, device="cuda")
    table = i32([[n - 3, -1], [n - 3, -1]])
    refs[n - 3], refs[n - 2], refs[n - 5] = 2, 0, 0
    dims, status = R.make_dims(2, 1, 1, 1, 64, 2, 1, n), status_word()
    ws = torch.empty((R.reader_pages_workspace_bytes(dims),), dtype=torch.uint8, device="cuda")
    was = cache[:, n - 20:].clone()
    R.reader_pages_reserve(dims, i32([5, 5]), i32([6, 20]), cache, None, table, refs, ws, status)
    assert int(status) == 0 and table.tolist() == [[n - 5, -1], [n - 3, n - 2]]
    assert refs[n - 3] == 1 and refs[n - 5] == 1 and refs[n - 2] == 1
    want = was.clone()
    want[:, 15] = was[:, 17]
    assert torch.equal(cache[:, n - 20:], want)


@pytest.mark.parametrize("D", [64, 128])
def test_single_tokens_beside_a_chunk(R, rows, D):  # noqa: F811
    p = Problem([1, 300, 1, 1, 40, 1], [3000, 1000, 17, 2000, 0, 1], 8, 2, D, seed=28)
    p.check(*p.run(R))
