"""reader_prompt_attn where a row's softmax reference, its maximum over the first keys that a wavefront sees, says little about its
later keys: scores up to 2^127 times as heavy, scores of minus infinity by their own value."""
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
    R.reader_tuning_override(R.TUNE_PROMPT_ROWS, request.param or -1)
    yield request.param
    R.reader_tuning_override(R.TUNE_PROMPT_ROWS, -1)


def run(R, rows, cache, q, L):
    n, Hq, D = q.shape
    dims = R.make_dims(1, 1, Hq, cache.Hkv, D, cache.max_pages, 1, cache.num_pages, variant=1 if rows == 0 else 0)
    assert R.reader_prompt_rows(dims, n, L + n) == rows
    ws = torch.full((max(256, R.reader_prompt_workspace_bytes(dims, n, L + n)),), 0xff, dtype=torch.uint8, device="cuda")
    out, lse, status = torch.empty_like(q, device="cuda"), torch.empty((n, Hq), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    R.reader_prompt_attn(dims, q.cuda(), cache.k.cuda(), cache.v.cuda(), cache.table.cuda(), torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                         torch.tensor([L], dtype=torch.int32, device="cuda"), out, lse, L + n, ws, status)
    assert int(status) == 0
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("height", [99.0, 118.0, 122.0, 124.5, 127.0])
@pytest.mark.parametrize("n,L", [(1, 9000), (5, 3000), (150, 2300)])
@pytest.mark.parametrize("period,at,each", [(7, 3, 1), (7, 3, 32), (8, 5, 1), (8, 5, 32)])
def test_heavy_keys_in_every_range(R, rows, D, height, n, L, period, at, each):
    """Every seventh or eighth step of 32 keys holds keys that weigh 2^height times what the others do: wavefronts and ranges that start
    in front of one carry sums of about that much against a low reference (with every eighth, many ranges in a row), those that start
    at one carry a high reference."""
    gen = torch.Generator().manual_seed(int(height))
    cache = P.Cache(gen, [L + n], 1, D)
    cache.fill(gen, 0, L + n, k_scale=0.01)
    q = torch.ones((n, 2, D), dtype=torch.bfloat16)
    j = torch.arange(L + n)
    heavy = ((j // 32) % period == at) & (j % 32 < each)
    page, slot = cache.place(0, L + n)
    # <q, k> / sqrt(D) = height ln 2, to the half step of bf16
    cache.k[page[heavy], 0, slot[heavy]] = height * math.log(2.0) / math.sqrt(D)
    out, lse = run(R, rows, cache, q, L)
    want, want_lse, bound, bound_lse = P.attention(q, cache.rows(cache.k, 0, L + n), cache.rows(cache.v, 0, L + n), L)
    P.check(out, want, bound, "out")
    P.check(lse, want_lse, bound_lse, "lse")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [-math.inf, -3e38])
@pytest.mark.parametrize("n,L", [(1, 9000), (5, 3000), (150, 2300), (700, 0)])
@pytest.mark.parametrize("period,part", [(3, 1), (12, 9)])
def test_scores_of_minus_infinity(R, rows, D, value, n, L, period, part):
    """Of every `period` tiles of 64 keys the first `part` score minus infinity (by an infinite key, or by a sum that overflows): they
    weigh nothing, also where they are all that the first tile of a range holds."""
    gen = torch.Generator().manual_seed(n)
    cache = P.Cache(gen, [L + n], 1, D)
    cache.fill(gen, 0, L + n)
    q = (torch.randn((n, 2, D), generator=gen).abs() + 0.1).bfloat16()
    none = (torch.arange(L + n) // 64) % period < part
    if L:
        none[L - 5:] = False                                      # (the rows' own keys, and a few in front, are as ever)
    page, slot = cache.place(0, L + n)
    cache.k[page[none], 0, slot[none]] = value
    out, lse = run(R, rows, cache, q, L)
    k, v = cache.rows(cache.k, 0, L + n), cache.rows(cache.v, 0, L + n)
    for i in sorted({0, n // 2, n - 1, 64, 100}):
        keep = ~none & (torch.arange(L + n) <= L + i)
        if i >= n or not bool(keep.any()):                        # (a row that sees nothing else is not looked at)
            continue
        o, s, bo, bs = P.attention(q[i:i + 1], k[:, keep], v[:, keep], int(keep.sum()) - 1)
        P.check(out[i:i + 1], o, bo, "row %d" % i)
        P.check(lse[i:i + 1], s, bs, "lse of row %d" % i)
