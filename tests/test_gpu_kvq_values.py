"""Attention over the cache in 4 bits at the ends of what it holds: values of V whose weighted sums pass the largest number of 32 bits
where their mean does not, keys with the largest scales under queries that are next to nothing."""
import functools

import pytest
import torch

import kvq_helpers as K
import prompt_helpers as P
from test_gpu_kvq import Problem, R, bushy, rows  # noqa: F401

pytestmark = pytest.mark.gpu
LOWEST, HIGHEST = 2, 252                                          # scale bytes


def shapes(n, L, tree, D):
    parents = bushy(torch.Generator().manual_seed(3), len(L), n[0]) if tree else None
    return Problem(n, L, 4, 2, D, seed=27, parents=parents)


SHAPES = {"short": ([3], [60], False), "single tokens": ([1, 1], [9000, 40], False), "long": ([200, 2], [900, 3000], False), "trees": ([40, 40], [700, 3], True)}


@functools.lru_cache(maxsize=None)
def largest(D, where, shape):
    """The problem and, for each sequence, what it comes to (once for all kernels).  To the bounds of K.attention comes what numbers below
    the smallest normal one lose: bf16's are 2^-133 apart, so that the rounding of an output is off by 2^-134 whatever its size, and each
    of the S products and sums of 32 bits by 2^-150, the weights' sum being at least one of them of weight one."""
    new, L, tree = SHAPES[shape]
    p = shapes(new, L, tree, D)
    pages = p.cache.data
    at = torch.cat([K.scale_bytes(D, s, True) for s in range(16)])
    if where == "some columns":
        for s in range(16):
            pages[..., K.scale_bytes(D, s, True)] = torch.tensor([LOWEST] * (D // 32 - 1) + [HIGHEST], dtype=torch.uint8)
    elif where == "some keys":
        size = torch.tensor([LOWEST, 60, 127, 200, HIGHEST], dtype=torch.uint8)
        pages[..., at] = size[torch.randint(0, 5, (*pages.shape[:-1], len(at)), generator=p.gen)]
    else:
        pages[..., at] = HIGHEST
    if where == "behind a low reference":                         # scores grow by a dozen of nats and more along the sequence
        for b in range(len(new)):
            S = new[b] + L[b]
            for j, (page, slot) in enumerate(p.cache.place(b, S)):
                pages[page][:, K.scale_bytes(D, slot, False)] = 122 + 5 * j // S
    want = []
    for b in range(p.B):
        S, mine = p.L[b] + p.new[b], slice(p.cu[b], p.cu[b] + p.new[b])
        o, lse, bo, bs = K.attention(p.q[mine], p.cache.rows(b, S, False), p.cache.rows(b, S, True), p.sees(b))
        want.append((mine, o, bo + 2.0 ** -134 + 2 * S * 2.0 ** -150, lse, bs))
    return p, want


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("where,shape", [("everywhere", "short"), ("everywhere", "single tokens"), ("everywhere", "long"), ("everywhere", "trees"),
                                         ("some columns", "single tokens"), ("some columns", "trees"), ("some keys", "long"), ("some keys", "trees"),
                                         ("behind a low reference", "long"), ("behind a low reference", "trees")])
def test_the_largest_values(R, rows, D, where, shape):  # noqa: F811
    """No mean of values is larger than all of them; a sum of them is infinite from the second on."""
    p, want = largest(D, where, shape)
    out, lse = p.run(R)
    for b, (mine, o, bo, s, bs) in enumerate(want):
        P.check(out[mine], o, bo, "out of sequence %d" % b)
        P.check(lse[mine], s, bs, "lse of sequence %d" % b)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,L", [([3], [60]), ([200, 2], [900, 3000])])
def test_the_largest_values_under_large_scores(R, rows, D, new, L):  # noqa: F811
    """Queries of one value, 2^20 and more: the keys that are largest there share the row in equal parts."""
    p = shapes(new, L, False, D)
    p.cache.data[..., torch.cat([K.scale_bytes(D, s, True) for s in range(16)])] = HIGHEST
    for size in (2.0 ** 20, 2.0 ** 27):
        at = torch.randint(0, D, (p.N, 4, 1), generator=p.gen)
        p.q = torch.zeros_like(p.q).scatter_(-1, at, torch.where(torch.rand((p.N, 4, 1), generator=p.gen) < 0.5, -size, size).bfloat16())
        out, lse = p.run(R)
        for b in range(len(new)):
            S = L[b] + new[b]
            k, v = p.cache.rows(b, S, False), p.cache.rows(b, S, True)
            mine = slice(p.cu[b], p.cu[b] + new[b])
            x = (p.q[mine].double().view(new[b], 2, 2, D).permute(1, 2, 0, 3) @ k[:, None].transpose(-1, -2)).masked_fill(~p.sees(b), -torch.inf)
            # (the products are exact; a key that is not among the largest is thousands behind)
            w = (x == x.amax(-1, keepdim=True)).double()
            n = w.sum(-1, keepdim=True)
            want, mass = (w @ v[:, None]) / n, (w @ v[:, None].abs()) / n
            bound = P.BF16 * (want.abs() + mass) * (1 + 2 * P.BF16) + (8 + S) * P.F32 * mass
            flat = lambda t: t.permute(2, 0, 1, 3).reshape(new[b], 4, D)  # noqa: E731
            P.check(out[mine], flat(want), flat(bound), "out")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("tree", [False, True])
def test_small_queries_on_the_largest_keys(R, rows, D, tree):  # noqa: F811
    """Queries down to the smallest numbers, under keys so large that their scores matter.  Where a kernel holds queries in pieces, a value is
    off by 2^-15 of the largest of its 32, or by 2^-130.  (The bounds are of first order in the error x of a weight, twice a score's, which is
    below 0.3 in them: exp(x) - 1 < 1.2 x.)"""
    p = shapes([60, 60], [300, 20], tree, D)
    usual = p.q.clone()
    pieces = rows in (0, 128, 256)
    step, floor = (2.0 ** -15, 2.0 ** -130) if pieces else (0.0, 0.0)
    for key, size in ((240, -113), (247, -120), (249, -121), (249, -125)) if pieces else ((240, -113), (249, -121), (HIGHEST, -124), (HIGHEST, -127)):
        p.cache.data[..., torch.cat([K.scale_bytes(D, s, False) for s in range(16)])] = key
        p.q = (usual.double() * 2.0 ** size).bfloat16()
        out, lse = p.run(R)
        for b in range(2):
            mine, S = slice(60 * b, 60 * b + 60), p.L[b] + 60
            o, s, bo, bs = K.attention(p.q[mine], p.cache.rows(b, S, False), p.cache.rows(b, S, True), p.sees(b), query_step=step, query_floor=floor)
            P.check(out[mine], o, 1.2 * bo, "out of sequence %d, queries of 2^%d" % (b, size))
            P.check(lse[mine], s, 1.2 * bs, "lse of sequence %d, queries of 2^%d" % (b, size))
