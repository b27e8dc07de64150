"""The cache in 4 bits in plain words: where a row's bytes are, what they stand for, what a row becomes (torch on the CPU, 64 bits;
nothing here calls the library)."""
import math

import torch

from prompt_helpers import BF16, F32, PAGE

SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
CODES = torch.tensor(SIZES + tuple(-x for x in SIZES), dtype=torch.float64)


def code_bytes(D, s, value):
    """Byte and shift of every value of row s: K's (value False) or V's."""
    d = torch.arange(D)
    if not value:
        return d // (D // 4) * 2 * D + s * (D // 8) + d % (D // 4) // 2, 4 * (d % 2)
    return 8 * D + s // 4 * 2 * D + d // (D // 16) * (D // 8) + s % 4 * (D // 32) + d % (D // 16) // 2, 4 * (d % 2)


def scale_bytes(D, s, value):
    g = torch.arange(D // 32)
    return 16 * D + D // 2 + s // 4 * (D // 8) + 4 * g + s % 4 if value else 16 * D + 16 * g + s


def quantise(x):
    """x [..., D] bf16: (codes [..., D], scale bytes [..., D / 32], whether each group was kept); nearest, ties to the even code."""
    g = x.double().unflatten(-1, (-1, 32))
    kept = g.isfinite().all(-1, keepdim=True)
    g = torch.where(kept, g, torch.zeros_like(g))
    top = g.abs().amax(-1, keepdim=True)
    floor = torch.where(top > 0, torch.frexp(top)[1] - 1, -1000)
    e = floor - 2
    e = (e + (top > 7 * torch.exp2(e.double())).int()).clamp(-125, 125)
    t = g.abs() / torch.exp2(e.double())
    codes = torch.zeros_like(t, dtype=torch.int64)
    for c in range(1, 8):                                    # the border below code c belongs to the even one of its neighbours
        border = (SIZES[c - 1] + SIZES[c]) / 2
        codes += (t >= border) if c % 2 == 0 else (t > border)
    codes += 8 * (torch.signbit(g) & kept)
    return codes.flatten(-2), (e + 127).flatten(-2), kept.flatten(-2)


def put(cache, place, rows, value):
    """Writes rows [n, *lead, Hkv, D] to (page, slot) pairs of a cache [*lead, pages, Hkv, 17 D]."""
    codes, scales, _ = quantise(rows)
    D = rows.shape[-1]
    for i, (page, slot) in enumerate(place):
        at, shift = code_bytes(D, slot, value)
        block = cache[..., page, :, :]
        both = (codes[i][..., 0::2] | codes[i][..., 1::2] << 4)
        block[..., at[0::2]] = both.to(torch.uint8)
        block[..., scale_bytes(D, slot, value)] = scales[i].to(torch.uint8)


def take(cache, place, value):
    """Rows [n, *lead, Hkv, D] in 64 bits."""
    D = cache.shape[-1] // 17
    out = []
    for page, slot in place:
        at, shift = code_bytes(D, slot, value)
        block = cache[..., page, :, :]
        x = CODES[(block[..., at].to(torch.int64) >> shift) & 15].unflatten(-1, (-1, 32))
        out.append((x * torch.exp2(block[..., scale_bytes(D, slot, value)].double() - 127)[..., None]).flatten(-2))
    return torch.stack(out) if out else torch.zeros((0, *cache.shape[:-3], cache.shape[-2], D), dtype=torch.float64)


def row_bytes(D, s):
    """All bytes of row s of a block."""
    return torch.cat([code_bytes(D, s, False)[0][0::2], code_bytes(D, s, True)[0][0::2], scale_bytes(D, s, False), scale_bytes(D, s, True)])


class Cache:
    """A cache in 4 bits for sequences of the given capacities: shuffled pages, 0xff (scales of no value) in all that is not written."""

    def __init__(self, gen, caps, Hkv, D, lead=(), spare=3):
        need = [(c + PAGE - 1) // PAGE for c in caps]
        self.num_pages, self.max_pages = sum(need) + spare, max(1, max(need))
        perm = torch.randperm(self.num_pages, generator=gen)
        self.table = torch.full((len(caps), self.max_pages), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n].int()
            at += n
        self.data = torch.full((*lead, self.num_pages, Hkv, 17 * D), 0xff, dtype=torch.uint8)
        self.Hkv, self.D = Hkv, D

    def place(self, b, end, start=0):
        """Page and slot of positions start .. end - 1."""
        return [(int(self.table[b, j // PAGE]), j % PAGE) for j in range(start, end)]

    def fill_all(self, gen, caps, scale_lo=124, scale_hi=127):
        """Random codes and scales in every row of every sequence."""
        for b, n in enumerate(caps):
            for j0 in range(0, n, PAGE):
                page, rows = int(self.table[b, j0 // PAGE]), min(PAGE, n - j0)
                shape = self.data[..., page, :, :].shape
                block = torch.randint(0, 256, shape, generator=gen, dtype=torch.uint8)
                block[..., 16 * self.D:] = torch.randint(scale_lo, scale_hi, (*shape[:-1], self.D), generator=gen, dtype=torch.uint8)
                at = torch.cat([row_bytes(self.D, s) for s in range(rows)])
                self.data[..., page, :, at] = block[..., at]

    def rows(self, b, n, value):
        """[Hkv, n, D] in 64 bits."""
        pages = self.table[b, :(n + PAGE - 1) // PAGE].long()
        D = self.D
        at = torch.stack([code_bytes(D, s, value)[0] for s in range(PAGE)])              # [16, D]
        shift = code_bytes(D, 0, value)[1]
        g = torch.stack([scale_bytes(D, s, value) for s in range(PAGE)])
        block = self.data[pages]                                                         # [pages, Hkv, 17 D]
        x = CODES[(block[:, :, at].to(torch.int64) >> shift) & 15].unflatten(-1, (-1, 32))
        x = (x * torch.exp2(block[:, :, g].double() - 127)[..., None]).flatten(-2)       # [pages, Hkv, 16, D]
        return x.transpose(0, 1).reshape(self.Hkv, -1, D)[:, :n]


def ancestors(parents):
    """[T, T]: node j is node i or in front of it on its path; a wrong link makes a root."""
    T = len(parents)
    sees = torch.eye(T, dtype=torch.bool)
    for i, p in enumerate(parents):
        if i > 0 and 0 <= p < i:
            sees[i] |= sees[p]
    return sees


def attention(q, k, v, sees, scale=None, query_step=0.0, query_floor=0.0):
    """q [n, Hq, D], k and v [Hkv, S, D] in 64 bits, sees [n, S]: (out, lse, bound on |out error|, bound on |lse error|).  A score is off
    by D roundings of its products' magnitudes and a few of its own, a weight by that much of itself and by its rounding to bf16,
    the output by one more.  query_step: what a query's values may be off by, of the largest of each 32; query_floor: by whatever it is."""
    n, Hq, D = q.shape
    Hkv, S = k.shape[:2]
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    q = q.double().view(n, Hkv, G, D).permute(1, 2, 0, 3)
    x = (q @ k[:, None].transpose(-1, -2)) * scale
    size = (q.abs() @ k[:, None].abs().transpose(-1, -2)) * scale
    x = x.masked_fill(~sees, -math.inf)
    lse = torch.logsumexp(x, -1)
    p = (x - lse[..., None]).exp().masked_fill(~sees, 0.0)
    out, mass = p @ v[:, None], p @ v[:, None].abs()
    score = ((D + 4) * F32 * size.masked_fill(~sees, 0.0) + 8 * F32 * x.masked_fill(~sees, 0.0).abs()).amax(-1)
    if query_step:
        most, sums = q.abs().unflatten(-1, (-1, 32)).amax(-1), k.abs().unflatten(-1, (-1, 32)).sum(-1)
        score = score + query_step * scale * (most @ sums[:, None].transpose(-1, -2)).masked_fill(~sees, 0.0).amax(-1)
    if query_floor:
        score = score + query_floor * scale * k.abs().sum(-1)[:, None, None].expand_as(x).masked_fill(~sees, 0.0).amax(-1)
    rel = 2 * score + 16 * F32 * (1 + lse.abs()) + S * F32
    bound = BF16 * (out.abs() + mass) * (1 + 2 * BF16) + rel[..., None] * mass
    flat = lambda t: t.permute(2, 0, 1, 3).reshape(n, Hq, D)  # noqa: E731
    return flat(out), lse.permute(2, 0, 1).reshape(n, Hq), flat(bound), rel.permute(2, 0, 1).reshape(n, Hq)
