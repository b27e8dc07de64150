"""Plain 64-bit forms of the operators around the verification step, and bounds on what rounding may do to them
(torch on the CPU; nothing here calls the library).

A rounding to bf16 is off by at most 2^-8 of the value, an fp32 sum of n products by at most n 2^-24 times the sum of
their magnitudes.
"""
import math

import torch

PAGE = 16
BF16 = 2.0 ** -8
F32 = 2.0 ** -24


class Cache:
    """A paged cache for sequences of the given capacities: shuffled pages, NaN in everything that is not written."""

    def __init__(self, gen, caps, Hkv, D, lead=(), spare=3):
        need = [(c + PAGE - 1) // PAGE for c in caps]
        self.num_pages, self.max_pages = sum(need) + spare, max(1, max(need))
        perm = torch.randperm(self.num_pages, generator=gen)
        self.table = torch.full((len(caps), self.max_pages), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = perm[at:at + n].int()
            at += n
        self.k = torch.full((*lead, self.num_pages, Hkv, PAGE, D), math.nan, dtype=torch.bfloat16)
        self.v = self.k.clone()
        self.Hkv, self.D = Hkv, D

    def place(self, b, n, start=0):
        j = torch.arange(start, start + n)
        return self.table[b].long()[j // PAGE], j % PAGE

    def fill(self, gen, b, n, start=0, k_scale=1.0):
        page, slot = self.place(b, n, start)
        for c, s in ((self.k, k_scale), (self.v, 1.0)):
            rows = torch.randn((n, *c.shape[:-4], self.Hkv, self.D), generator=gen) * s
            if c.dim() == 5:
                for layer in range(c.shape[0]):
                    c[layer, page, :, slot] = rows[:, layer].bfloat16()
            else:
                c[page, :, slot] = rows.bfloat16()

    def rows(self, c, b, n):
        """[Hkv, n, D] in 64 bits."""
        page, slot = self.place(b, n)
        return c[page, :, slot].double().transpose(0, 1)


def depths(parents):
    d = []
    for i, p in enumerate(parents):
        d.append(0 if i == 0 or p < 0 else d[p] + 1)
    return d


def norm_rotate(x, w, eps, cos_sin, pos, interleaved):
    """x [n, heads, D] bf16, pos [n]: (value, bound on |error|) in 64 bits."""
    D = x.shape[-1]
    x = x.double()
    mag = x.abs()
    if w is not None:
        f = w.double() / (x.square().sum(-1, keepdim=True) / D + eps).sqrt()
        # the sum of D squares, its root, the quotient and two products: D / 2 + 4 roundings at most
        x, mag = x * f, (x * f).abs() * (1 + (D / 2 + 4) * F32)
    slack = (D / 2 + 8) * F32 * mag
    rot = cos_sin.shape[1] if cos_sin is not None else 0
    y = x.clone()
    if rot:
        c, s = cos_sin.double()[pos][:, None, :rot // 2], cos_sin.double()[pos][:, None, rot // 2:]
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
            y[..., a] = x[..., a] * c[..., i] - x[..., b] * s[..., i]
            y[..., b] = x[..., b] * c[..., i] + x[..., a] * s[..., i]
            both = (D / 2 + 12) * F32 * (mag[..., a] + mag[..., b])
            slack[..., a] = both
            slack[..., b] = both
    bound = BF16 * y.abs() * (1 + BF16) + slack if w is not None or rot else torch.zeros_like(y)
    if w is None and rot < D:
        bound[..., rot:] = 0.0                               # values that nothing is done to
    return y, bound


def attention(q, k, v, L, scale=None):
    """q [n, Hq, D], k and v [Hkv, L + n, D] in 64 bits: (out, lse, bound on |out error|, bound on |lse error|)."""
    n, Hq, D = q.shape
    Hkv = k.shape[0]
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    q = q.double().view(n, Hkv, G, D).permute(1, 2, 0, 3)                      # [Hkv, G, n, D]
    x = (q @ k[:, None].transpose(-1, -2)) * scale                            # [Hkv, G, n, S]
    size = (q.abs() @ k[:, None].abs().transpose(-1, -2)) * scale             # sums of magnitudes
    hide = torch.arange(L + n)[None, :] > L + torch.arange(n)[:, None]
    x = x.masked_fill(hide, -math.inf)
    lse = torch.logsumexp(x, -1)
    p = (x - lse[..., None]).exp()
    out = p @ v[:, None]
    mass = p @ v[:, None].abs()
    # a score is off by D roundings of its products' magnitudes and a few of its own, a weight by that much of itself
    score = ((D + 4) * F32 * size.masked_fill(hide, 0.0) + 8 * F32 * x.masked_fill(hide, 0.0).abs()).amax(-1)
    rel = 2 * score + 16 * F32 * (1 + lse.abs())
    bound = BF16 * (out.abs() + mass) * (1 + 2 * BF16) + (rel + (L + n) * F32)[..., None] * mass
    flat = lambda t: t.permute(2, 0, 1, 3).reshape(n, Hq, D)  # noqa: E731
    return flat(out), lse.permute(2, 0, 1).reshape(n, Hq), flat(bound), (rel + (L + n) * F32).permute(2, 0, 1).reshape(n, Hq)


def key_weights(q, lse, k, first, scale=None):
    """q [n, Hq, D], lse [n, Hq], k [Hkv, S, D]: weight drawn by every key [Hkv, S], and a bound on its error; row i sees keys
    up to first + i."""
    n, Hq, D = q.shape
    Hkv, S = k.shape[0], k.shape[1]
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    x = q.double().view(n, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, n * G, D) @ k.transpose(1, 2) * scale
    size = q.double().abs().view(n, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, n * G, D) @ k.abs().transpose(1, 2) * scale
    ref = lse.double().view(n, Hkv, G).permute(1, 0, 2).reshape(Hkv, n * G, 1)
    hide = torch.arange(S)[None, :] > (first + torch.arange(n).repeat_interleave(G))[:, None]
    p = (x - ref).exp().masked_fill(hide, 0.0)
    rel = (D + 4) * F32 * size + 8 * F32 * (x.abs() + ref.abs() + 1) + n * G * F32
    return p.sum(1), (p * rel).sum(1)


def evict(w, keep, recent):
    """Positions that stay, w [n] on the host: the newest `recent` and the heaviest others, lowest position first among equals."""
    n = w.numel()
    order = sorted(range(n - recent), key=lambda j: (0 if w[j] == w[j] else 1, -w[j] if w[j] == w[j] else 0.0, j))
    return sorted(order[:keep - recent] + list(range(n - recent, n)))


def check(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    over = ~(err <= bound)
    if bool(over.any()):
        i = int((err - bound).nan_to_num(nan=math.inf).flatten().argmax())
        raise AssertionError("%s: %d of %d values out of bounds, worst at %d: got %r, want %r, bound %r" % (
            what, int(over.sum()), over.numel(), i, float(got.flatten()[i]), float(want.flatten()[i]), float(bound.flatten()[i])))
