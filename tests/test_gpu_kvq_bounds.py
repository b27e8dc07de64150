"""Packed bounds that are out of order, out of range or start behind row 0, over the cache in 4 bits: the same status whatever kernel
runs, the rows of sequences that are as they should be, and nothing else written."""
import functools

import pytest
import torch

import kvq_helpers as K
import prompt_helpers as P
from test_gpu_kvq import R, i32, rows  # noqa: F401
from test_gpu_prompt_bounds import TABLES, TOUCHED, Guarded, N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", range(len(TABLES)))
@pytest.mark.parametrize("D", [64, 128])
def test_attention(R, rows, case, D):  # noqa: F811
    cu, wrong, owned = TABLES[case]
    gen = torch.Generator().manual_seed(20 + case)
    Hq, Hkv, L = 4, 2, [20, 0, 3, 40]
    cache = K.Cache(gen, [n + N for n in L], Hkv, D)
    cache.fill_all(gen, [n + N for n in L])
    q = torch.randn((N, Hq, D), generator=gen).bfloat16()
    dims = R.make_dims(4, 1, Hq, Hkv, D, cache.max_pages, 1, cache.num_pages)
    bound = cache.max_pages * 16
    ws = torch.full((R.reader_kvq_workspace_bytes(dims, N, bound),), 0xff, dtype=torch.uint8, device="cuda")
    out, lse, status = Guarded((N, Hq, D), torch.bfloat16), Guarded((N, Hq), torch.float32), i32([0])
    R.reader_kvq_prompt_attn(dims, q.cuda(), cache.data.cuda(), cache.table.cuda(), i32(cu), i32(L), out.t, lse.t, bound, ws, status)
    assert int(status) == (R.STATUS_BAD_LENGTH if wrong else 0)
    touched = TOUCHED.get(case, [t for _, _, r in owned for t in r])
    out.unchanged(touched)
    lse.unchanged(touched)
    for b, first, mine in owned:
        n = max(mine) + 1 - first
        sees = torch.ones((n, L[b] + n), dtype=torch.bool).tril(L[b])
        o, s, bo, bs = K.attention(q[first:first + n], cache.rows(b, L[b] + n, False), cache.rows(b, L[b] + n, True), sees)
        for t in mine:
            P.check(out.t[t], o[t - first], bo[t - first], "row %d" % t)
            P.check(lse.t[t], s[t - first], bs[t - first], "lse of row %d" % t)


@functools.lru_cache(maxsize=None)
def one_token_each(B, Hq):
    """A batch and, of the rows that nobody else claims if the middle one's bound goes back to row 1, what some come to (once for all kernels)."""
    gen = torch.Generator().manual_seed(B)
    cache = K.Cache(gen, [16] * B, 1, 64)
    cache.fill_all(gen, [16] * B)
    q = torch.randn((B + 20, Hq, 64), generator=gen).bfloat16()
    want = {}
    for b in [0] + list(range(B // 2 + 1, B, 1 + B // 100)) + [B - 3, B - 2, B - 1]:
        o, _, bo, _ = K.attention(q[b:b + 1], cache.rows(b, 4, False), cache.rows(b, 4, True), torch.ones((1, 4), dtype=torch.bool))
        want[b] = o, bo
    return cache, q, want


@pytest.mark.parametrize("B,Hq", [(100, 16), (4096, 2)])
def test_one_bad_bound_among_many(R, rows, B, Hq):  # noqa: F811
    """One sequence goes back to row 1 and has half of the batch's rows: those behind it are the others' as ever."""
    cache, q, want = one_token_each(B, Hq)
    cu = torch.arange(B + 1)
    cu[B // 2] = 1
    dims = R.make_dims(B, 1, Hq, 1, 64, 1, 1, cache.num_pages)
    ws = torch.full((R.reader_kvq_workspace_bytes(dims, B + 20, 16),), 0xff, dtype=torch.uint8, device="cuda")
    out, status = Guarded((B + 20, Hq, 64), torch.bfloat16), i32([0])
    R.reader_kvq_prompt_attn(dims, q.cuda(), cache.data.cuda(), cache.table.cuda(), cu.int().cuda(), i32([3] * B), out.t, None, 16, ws, status)
    assert int(status) == R.STATUS_BAD_LENGTH
    out.unchanged(range(B))
    got = out.t.cpu()
    for b, (o, bo) in want.items():
        P.check(got[b:b + 1], o, bo, "row %d" % b)
