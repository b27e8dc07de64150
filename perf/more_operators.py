"""What a serving program asks of a cache held in 4 bits and of the pages of a cache, as a list of timed cases.

  store    K/V rows become 4-bit rows of the paged cache: of a step's draft trees (reader_kvq_store), or of a prompt that was
           worked on in a bf16 cache (reader_kvq_pack, all layers in one call)
  attn     attention over that cache: of draft trees (reader_kvq_tree_attn), of packed prompts, chunks and single tokens
           (reader_kvq_prompt_attn)
  compact  the accepted path's rows move to where they stay, all layers (reader_kvq_compact_layers)
  reorder  sequences are forked, permuted and dropped by their page tables (reader_pages_reorder)
  reserve  pages for the positions that the next step writes: taken, given back, copied where others hold them too
           (reader_pages_reserve)

The cache: uint8 [pages, kv heads, 17 D], a block of 17 D bytes for the 16 rows of a page.  A row's values stand in groups of 32
with a power of two for each (a byte, the exponent + 127) and 4 bits a value: a sign and 0, 1/2, 1, 3/2, 2, 3, 4 or 6.  The codes
of K, then of V, then the scales of K and of V; `_places` says where a row's bytes are.  A row of bf16 has one form in 4 bits, so
what writes the cache returns its bytes: all of them have to be equal, the zeros' signs too, which is more than equal values.

A case is a dict of sizes and options.  `listed()` names the ones a serving program meets most, `draw()` gives more of the same
ranges, `prepare()` makes what the program has in hand before the call (from the seed alone), `run()` is one pass, `work()` what
the pass cannot do without, `exact()` its result in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False             # True: run() calls the library; False: it computes the same with elementary torch operations

DEVICE = "cuda:0"
PAGE = 16               # tokens per cache page
LOWEST, HIGHEST = -125, 125                # exponents of a group's scale
MOST_SCORES = 5 << 29                      # scores that a drawn attention's padded form may hold


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # one layer's rows of a verification step's draft trees: latency counts, it runs in every layer
        dict(name="store_tree_step", kind="store", form="tree", B=16, Hkv=8, D=128, T=32, L_lo=1024, L_hi=4096),
        # prompts that were worked on in bf16 pages, all layers of a small model: a large one-off
        dict(name="pack_prompts", kind="store", form="pages", NL=8, B=8, Hkv=8, D=128, L_lo=2000, L_hi=8192),
        # the smallest call of a decoding loop: one draft tree of a small model
        dict(name="attn_tree_tiny", kind="attn", form="tree", B=1, Hq=8, Hkv=8, D=64, T=16, L_lo=512, L_hi=512, lse=False),
        # a decoding step of a large model with many users: the largest call
        dict(name="attn_tree_large_batch", kind="attn", form="tree", B=64, Hq=64, Hkv=8, D=128, T=64, L_lo=2048, L_hi=8192,
             lse=False),
        # plain decoding of a batch: one new token per sequence, log-sum-exp asked for
        dict(name="attn_single_tokens", kind="attn", form="prompt", B=16, Hq=32, Hkv=8, D=128, n_lo=1, n_hi=1, L_lo=1024,
             L_hi=16384, lse=True),
        # the next chunk of two long documents, of a large model
        dict(name="attn_chunk_of_long", kind="attn", form="prompt", B=2, Hq=64, Hkv=8, D=128, n_lo=512, n_hi=512, L_lo=20000,
             L_hi=28000, lse=False),
        # behind a verification step: the accepted path of one user, one layer
        dict(name="compact_one_user", kind="compact", NL=1, B=1, Hkv=8, D=64, T=16, L_lo=512, L_hi=512, path=6),
        # ... of many users, all layers of a large model
        dict(name="compact_all_layers", kind="compact", NL=32, B=64, Hkv=8, D=128, T=64, L_lo=512, L_hi=2048, path=8),
        # beams of one prompt after a selection: a few are dropped, a few forked
        dict(name="reorder_beams", kind="reorder", B=8, L_lo=4096, L_hi=4096, pages=300),
        # a large batch of long sequences, one in four forked from another
        dict(name="reorder_large_batch", kind="reorder", B=512, L_lo=1024, L_hi=16384, pages=1100),
        # before a decoding step of a batch: a few more positions each
        dict(name="reserve_step", kind="reserve", form="bf16", NL=2, B=16, Hkv=8, D=128, more=33, L_lo=1024, L_hi=4096,
             forks=0.0),
        # beams that have just been forked: every partly filled page is copied in all layers of the 4-bit cache
        dict(name="reserve_forked", kind="reserve", form="4-bit", NL=32, B=256, Hkv=8, D=128, more=17, L_lo=500, L_hi=2000,
             forks=0.75),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _most(kind):
    w = [work(c) for c in listed() if c["kind"] == kind]
    return max(x["bytes"] for x in w), max(x["flops"] for x in w)


def _low(rng, hi):
    return int(hi * rng.choice((0.1, 0.5, 1.0)))


def draw(rng):
    kind = rng.choice(("store", "store", "attn", "attn", "attn", "attn", "attn", "compact", "reorder", "reserve"))
    nbytes, flops = _most(kind)
    while True:
        Hkv, D, B = rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 128)), _log(rng, 1, 64)
        if kind == "store":
            c = dict(kind=kind, form=rng.choice(("tree", "pages", "rows")), B=B, Hkv=Hkv, D=D)
            L_hi = _log(rng, 1, 16384)
            if c["form"] == "pages":
                c.update(NL=_log(rng, 1, 32))
            elif c["form"] == "tree":
                c.update(T=_log(rng, 1, 128))
            else:
                n_hi = _log(rng, 1, 4096)
                c.update(n_lo=_low(rng, n_hi), n_hi=n_hi)
            c.update(L_lo=_low(rng, L_hi), L_hi=L_hi)
            rows = B * (L_hi + c.get("T", 0) + c.get("n_hi", 0)) * c.get("NL", 1)
            if rows * Hkv * D > 8 * 8 * 8192 * 8 * 128:
                continue
        elif kind == "attn":
            form = rng.choice(("tree", "prompt"))
            c = dict(kind=kind, form=form, B=B, Hq=Hkv * rng.choice((1, 3, 4, 8, 16)), Hkv=Hkv, D=D)
            L_hi = rng.choice((0, _log(rng, 1, 32768), _log(rng, 256, 16384), _log(rng, 256, 16384)))
            if form == "tree":
                c.update(T=_log(rng, 1, 128))
            else:
                n_hi = rng.choice((1, _log(rng, 1, 64), _log(rng, 1, 2048)))
                c.update(n_lo=max(1, _low(rng, n_hi)), n_hi=n_hi)
            c.update(L_lo=_low(rng, L_hi), L_hi=L_hi, lse=rng.random() < 0.5)
            n = c.get("T", c.get("n_hi"))
            if B * n * c["Hq"] * (L_hi + n) > MOST_SCORES or B * (L_hi + n) * Hkv * D > 5 << 27:
                continue
        elif kind == "compact":
            T, L_hi = _log(rng, 4, 128), _log(rng, 16, 16384)
            c = dict(kind=kind, NL=_log(rng, 1, 32), B=B, Hkv=Hkv, D=D, T=T, L_lo=_low(rng, L_hi), L_hi=L_hi,
                     path=rng.randint(1, min(T // 2, 12)))
            if c["NL"] * B * (L_hi + T) * Hkv * D > 32 * 64 * 8 * 2100 * 128:
                continue
        elif kind == "reorder":
            L_hi = _log(rng, 1, 16384)
            c = dict(kind=kind, B=_log(rng, 1, 512), L_lo=_low(rng, L_hi), L_hi=L_hi, pages=(L_hi + 15) // 16 + rng.randint(1, 100))
        else:
            L_hi = _log(rng, 1, 16384)
            c = dict(kind=kind, form=rng.choice(("bf16", "4-bit")), NL=_log(rng, 1, 32), B=_log(rng, 1, 256), Hkv=Hkv, D=D,
                     more=rng.choice((1, rng.randint(1, 140))), L_lo=_low(rng, L_hi), L_hi=L_hi, forks=rng.choice((0.0, 0.25, 0.75)))
            if c["NL"] * c["B"] * (L_hi + c["more"]) * Hkv * D > 32 * 64 * 8 * 2100 * 128:
                continue
        w = work(c)
        if w["bytes"] <= nbytes and w["flops"] <= flops:
            return c


# ------------------------------------------------------------------------------------------------ inputs

def _spread(lo, hi, n, turn=0.6180339887498949):
    """n whole numbers between lo and hi, part of the case: the golden-ratio sequence spreads them evenly."""
    return (lo + ((hi - lo + 1) * ((np.arange(1, n + 1) * turn) % 1.0)).astype(np.int64)).clip(lo, hi)


def _lengths(case):
    """Cached positions of each sequence; of forks, their origin's."""
    L = _spread(case["L_lo"], case["L_hi"], case["B"])
    return L[_origins(case)] if case["kind"] == "reserve" else L


def _origins(case):
    """Which sequence each one was forked from: itself, or one of the first (1 - forks) of them."""
    b = np.arange(case["B"])
    first = max(1, int(round(case["B"] * (1 - case["forks"]))))
    return np.where(b < first, b, b % first)


def _new(case):
    """New tokens of each sequence."""
    if "n_hi" in case:
        return _spread(case["n_lo"], case["n_hi"], case["B"], 0.7548776662466927)
    return np.full((case["B"],), case.get("T", 0), dtype=np.int64)


def _accepted(case):
    """Nodes of the accepted path (the root among them) of each sequence."""
    return _spread(1, case["path"], case["B"], 0.7548776662466927)


def _sources(case):
    """Which sequence every row of the tables becomes: most stay, one in four is a fork of another, a few become empty."""
    b = np.arange(case["B"])
    turn = (b * 0.7548776662466927) % 1.0
    return np.where(turn < 0.25, (b * 7 + 3) % case["B"], np.where(turn > 0.97, -1, b))


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEVICE)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.bfloat16)


def _held(gen, *shape, D):
    """A cache in 4 bits [..., 17 D] as a model's rows leave it: any codes, scales from 1/8 to 1/2."""
    c = torch.randint(0, 256, (*shape, 17 * D), generator=gen, device=DEVICE, dtype=torch.uint8)
    c[..., 16 * D:] = c[..., 16 * D:] % 3 + 124
    return c


class _State:
    """A program's buffers."""

    def __init__(self, case):
        self.case = case
        self.call = None          # the library's arguments, made at the first pass


def _table(rng, lengths, num_pages, max_pages):
    """A page table for these lengths: physical order is a random permutation."""
    need = (np.asarray(lengths, dtype=np.int64) + PAGE - 1) // PAGE
    table = np.full((len(lengths), max_pages), -1, dtype=np.int32)
    table[np.arange(max_pages)[None, :] < need[:, None]] = rng.permutation(num_pages)[: int(need.sum())]
    return table


def _count(lengths):
    return int(((np.asarray(lengths) + PAGE - 1) // PAGE).sum())


def prepare(case, seed):
    rng = np.random.Generator(np.random.PCG64(seed))
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    s = _State(case)
    B, kind, D, Hkv = case["B"], case["kind"], case.get("D"), case.get("Hkv")
    L, new = _lengths(case), _new(case)
    s.seq_lens0 = _i32(L)
    s.seq_lens = s.seq_lens0.clone()
    s.status = torch.zeros((1,), dtype=torch.int32, device=DEVICE)
    if kind == "reorder":
        s.max_pages, s.num_pages = case["pages"], _count(L) + 7
        s.page_table0 = _i32(_table(rng, L, s.num_pages, s.max_pages))
        s.page_refs0 = torch.zeros((s.num_pages,), dtype=torch.int32, device=DEVICE)
        s.page_refs0[s.page_table0[s.page_table0 >= 0].long()] = 1
        s.page_table, s.page_refs = s.page_table0.clone(), s.page_refs0.clone()
        s.sources = _i32(_sources(case))
        return s
    if kind == "reserve":
        origin = _origins(case)
        first = int(origin.max()) + 1
        s.max_pages = int((L.max() + case["more"] + PAGE - 1) // PAGE) + 3
        s.num_pages = _count(L[:first]) + _count(L + case["more"] + PAGE) - _count(L) + B + 5
        s.page_table0 = _i32(_table(rng, L[:first], s.num_pages, s.max_pages)[origin])
        held = s.page_table0[s.page_table0 >= 0].long()
        s.page_refs0 = torch.bincount(held, minlength=s.num_pages).int()
        s.page_table, s.page_refs = s.page_table0.clone(), s.page_refs0.clone()
        s.new_lens = _i32(L + case["more"])
        if case["form"] == "bf16":
            s.k_cache = _normal(gen, case["NL"], s.num_pages, Hkv, PAGE, D)
            s.v_cache = _normal(gen, case["NL"], s.num_pages, Hkv, PAGE, D)
        else:
            s.k_cache, s.v_cache = _held(gen, case["NL"], s.num_pages, Hkv, D=D), None
        return s
    s.max_pages, s.num_pages = max(1, int((L + new + PAGE - 1).max() // PAGE)), _count(L + new) + 3
    s.page_table = _i32(_table(rng, L + new, s.num_pages, s.max_pages))
    s.max_seq_len = int((L + new).max())
    N = int(new.sum())
    s.cu_tokens = _i32(np.concatenate([[0], np.cumsum(new)]))
    if kind == "store":
        NL = case.get("NL", 1)
        s.kvq = torch.zeros((NL, s.num_pages, Hkv, 17 * D), dtype=torch.uint8, device=DEVICE)
        if case["form"] == "pages":
            s.from_table = _i32(_table(rng, L, s.num_pages, s.max_pages))
            s.k, s.v = (_normal(gen, NL, s.num_pages, Hkv, PAGE, D) for _ in range(2))
            s.k.mul_(torch.randn((Hkv, 1, D), generator=gen, device=DEVICE).exp_())      # channels of their own size
        else:
            s.kvq = s.kvq[0]
            shape = (B, case["T"]) if case["form"] == "tree" else (N,)
            s.k, s.v = (_normal(gen, *shape, Hkv, D) for _ in range(2))
            s.k.mul_(torch.randn((Hkv, D), generator=gen, device=DEVICE).exp_())
        return s
    if kind == "compact":
        s.kvq = _held(gen, case["NL"], s.num_pages, Hkv, D=D)
        n = _accepted(case)
        path = np.full((B, case["path"]), -1, dtype=np.int32)
        path[:, 0] = 0
        # (nodes behind all destinations, so that a second pass over the same state moves the same rows)
        pick = np.sort(rng.random((B, case["T"] - case["path"])).argsort(axis=1)[:, : case["path"] - 1], axis=1) + case["path"]
        path[:, 1:] = np.where(np.arange(1, case["path"])[None, :] < n[:, None], pick, -1)
        s.path, s.accept_len = _i32(path), _i32(n - 1)
        return s
    s.kvq = _held(gen, s.num_pages, Hkv, D=D)
    s.parents = None
    if case["form"] == "tree":
        i = np.arange(case["T"])
        low = np.maximum(0, i // 4 - 2)                                                  # bushy trees a few levels deep
        parents = low + (rng.random((B, case["T"])) * (i - low)).astype(np.int64)
        parents[:, 0] = -1
        s.parents = _i32(parents)
        s.max_seq_len = int(L.max())
    s.q = _normal(gen, *((B, case["T"]) if case["form"] == "tree" else (N,)), case["Hq"], D)
    s.out = torch.zeros_like(s.q)
    s.lse = None
    if case["lse"]:
        s.lse = torch.zeros((B, case["Hq"], case["T"]) if case["form"] == "tree" else (N, case["Hq"]), device=DEVICE)
    return s


# ------------------------------------------------------------------------------------------------ a pass: the plain forms

def _places(slot, D):
    """Where the bytes of a page's row `slot` (a tensor) are in its block, [..., D + D / 16]: K's, V's, K's scales, V's."""
    slot = slot[..., None]
    d, g = torch.arange(0, D, 2, device=DEVICE), torch.arange(D // 32, device=DEVICE)
    q, c = D // 4, D // 16                                     # values of a row that stand together in K, in V
    k = (d // q) * (8 * q) + slot * (q // 2) + d % q // 2
    v = 8 * D + (slot // 4) * (2 * D) + (d // c) * (2 * c) + (slot % 4) * (c // 2) + d % c // 2
    ks = 16 * D + g * 16 + slot
    vs = 16 * D + D // 2 + (slot // 4) * (D // 8) + g * 4 + slot % 4
    return torch.cat([k, v, ks, vs], dim=-1)


def _quantised(x):
    """Rows [..., D] as bytes of codes [..., D / 2] and of scales [..., D / 32], and whether a value is no finite number."""
    x = x.double().unflatten(-1, (-1, 32))
    bad = ~x.isfinite().all(-1, keepdim=True)
    x = torch.where(bad, 0.0, x)
    top = x.abs().amax(-1, keepdim=True)
    part, e = torch.frexp(top)                                 # top = part 2^e, part in [1/2, 1)
    e = torch.where(top > 0, (e - 3 + (part > 0.875)).clamp(LOWEST, HIGHEST), LOWEST)
    t = x.abs() * torch.exp2(-e.double())
    code = (t > 0.25).byte() + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5) + (t >= 3.5) + (t > 5.0)
    code = (code + 8 * torch.signbit(x)).byte().flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).byte().flatten(-2), bad.any()


def _dequantised(codes, scales):
    """Values [..., D] in 32 bits of bytes of codes [..., D / 2] and of scales [..., D / 32]."""
    steps = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=DEVICE)
    x = steps[torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).int()].unflatten(-1, (-1, 32))
    return (x * torch.exp2(scales.float() - 127)[..., None]).flatten(-2)


def _rows(first, count):
    """Sequence and position of `count` positions behind `first`, of all sequences."""
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=DEVICE), count)
    return seq, first[seq] + torch.arange(seq.numel(), device=DEVICE) - (count.cumsum(0) - count)[seq]


def _plain_store(s):
    case, D = s.case, s.case["D"]
    kvq = s.kvq if s.kvq.dim() == 4 else s.kvq[None]
    if case["form"] == "pages":
        seq, at = _rows(torch.zeros_like(s.seq_lens).long(), s.seq_lens.long())
        page, slot = s.from_table.long()[seq, at // PAGE], at % PAGE
        k, v = s.k[:, page, :, slot], s.v[:, page, :, slot]                              # [N, NL, Hkv, D]
    else:
        seq, at = _rows(s.seq_lens.long(), s.cu_tokens.long().diff())
        k, v = s.k.reshape(-1, 1, case["Hkv"], D), s.v.reshape(-1, 1, case["Hkv"], D)
    kc, ks, kbad = _quantised(k)
    vc, vs, vbad = _quantised(v)
    page, place = s.page_table.long()[seq, at // PAGE], _places(at % PAGE, D)
    layer, head = torch.arange(kvq.shape[0], device=DEVICE), torch.arange(case["Hkv"], device=DEVICE)
    kvq[layer[:, None, None], page[:, None, None, None], head[:, None], place[:, None, None, :]] = torch.cat([kc, vc, ks, vs], dim=-1)
    s.status |= 16 * (kbad | vbad)
    return {"kvq": s.kvq, "status": s.status}


def _ancestors(parents):
    """[B, T, T]: whether node j is node i itself or in front of it on its path, by doubling the links."""
    T = parents.shape[1]
    up = torch.cat([torch.zeros_like(parents[:, :1]), parents + 1], dim=1).long()         # entry 0: above the root
    near = torch.eye(T + 1, dtype=torch.bool, device=DEVICE).repeat(parents.shape[0], 1, 1)
    for _ in range(T.bit_length()):
        near = near | near.gather(1, up[:, :, None].expand_as(near))
        up = up.gather(1, up)
    return near[:, 1:, 1:]


def _plain_attn(s):
    case = s.case
    B, Hq, Hkv, D = case["B"], case["Hq"], case["Hkv"], case["D"]
    G, new, L = Hq // Hkv, s.cu_tokens.long().diff(), s.seq_lens.long()
    pages = int((_lengths(case) + _new(case)).max() + PAGE - 1) // PAGE
    n, S = int(_new(case).max()), pages * PAGE
    # the keys of all sequences, [B, Hkv, S, D], zeros behind the last one
    block = s.kvq[s.page_table[:, :pages].clamp(min=0).long()]                            # [B, pages, Hkv, 17 D]
    rows = block[..., _places(torch.arange(PAGE, device=DEVICE), D)].permute(0, 2, 1, 3, 4).reshape(B, Hkv, S, -1)
    there = torch.arange(S, device=DEVICE) < (L + new)[:, None]
    k = _dequantised(rows[..., : D // 2], rows[..., D:D + D // 32]) * there[:, None, :, None]
    v = _dequantised(rows[..., D // 2:D], rows[..., D + D // 32:]) * there[:, None, :, None]
    # the queries, [B, Hkv, n G, D], and which keys they see
    seq, row = _rows(torch.zeros_like(new), new)
    q = torch.zeros((B, n, Hkv, G, D), device=DEVICE)
    q[seq, row] = s.q.float().view(-1, Hkv, G, D)
    behind = torch.arange(S, device=DEVICE) - L[:, None]                                  # number of the new token at a key
    sees = behind[:, None, :] <= torch.arange(n, device=DEVICE)[:, None]
    if s.parents is not None:
        tree = _ancestors(s.parents).gather(2, behind.clamp(0, n - 1)[:, None, :].expand(B, n, S))
        sees = sees & (tree | (behind < 0)[:, None, :])
    x = q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D) @ k.transpose(2, 3)
    x = x.view(B, Hkv, n, G, S).mul_(D ** -0.5).masked_fill_(~sees[:, None, :, None, :], -math.inf).view(B, Hkv, n * G, S)
    m = x.amax(-1, keepdim=True)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x @ v).div_(total).view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    s.out.view(-1, Hq, D).copy_(o[seq, row].to(torch.bfloat16))
    if s.lse is not None:
        lse = (m + total.log()).view(B, Hkv, n, G).permute(0, 2, 1, 3).reshape(B, n, Hq)
        s.lse.copy_(lse.transpose(1, 2) if s.parents is not None else lse[seq, row])
    return {"out": s.out, "lse": s.lse, "status": s.status}


def _plain_compact(s):
    case = s.case
    heads = torch.arange(case["Hkv"], device=DEVICE)[:, None]
    seq, j = _rows(torch.ones_like(s.accept_len).long(), s.accept_len.long())
    L, node = s.seq_lens.long()[seq], s.path.long()[seq, j]
    table = s.page_table.long()
    page = lambda at: table[seq, at // PAGE][:, None, None]                               # noqa: E731
    place = lambda at: _places(at % PAGE, case["D"])[:, None, :]                          # noqa: E731
    s.kvq[:, page(L + j), heads, place(L + j)] = s.kvq[:, page(L + node), heads, place(L + node)]
    s.seq_lens += s.accept_len + 1
    return {"kvq": s.kvq, "seq_lens": s.seq_lens, "status": s.status}


def _changed(refs, table, by):
    """Adds `by` to the count of every page that a table names."""
    held = table[table >= 0].long()
    refs.index_add_(0, held, torch.full_like(held, by, dtype=torch.int32))


def _plain_reorder(s):
    src = s.sources.long()
    L = torch.where(src >= 0, s.seq_lens[src.clamp(min=0)], 0)
    holds = torch.arange(s.max_pages, device=DEVICE) < ((L + PAGE - 1) // PAGE)[:, None]
    table = torch.where(holds, s.page_table[src.clamp(min=0)], -1)
    _changed(s.page_refs, s.page_table, -1)
    _changed(s.page_refs, table, 1)
    s.page_table.copy_(table)
    s.seq_lens.copy_(L)
    return {"page_table": s.page_table, "seq_lens": s.seq_lens, "page_refs": s.page_refs, "status": s.status}


def _plain_reserve(s):
    L, new, table, refs = s.seq_lens.long(), s.new_lens.long(), s.page_table.long(), s.page_refs
    B, at = L.numel(), torch.arange(s.max_pages, device=DEVICE)
    used, want = ((L + PAGE - 1) // PAGE)[:, None], ((new + PAGE - 1) // PAGE)[:, None]
    many = (refs[table.clamp(min=0)] > 1) & (table >= 0)
    # entries that are given back: behind what is wanted, or without contents and held by others too
    drop = (table >= 0) & (at >= used) & ((at >= want) | many)
    # partly filled pages that others hold too: the last of the writers keeps one that nobody else holds
    writes = (L % PAGE > 0) & (new > L)
    part = torch.where(writes, table.gather(1, (L // PAGE).clamp(max=s.max_pages - 1)[:, None])[:, 0], -1)
    same = (part[:, None] == part[None, :]) & (part >= 0)[:, None]
    last = torch.where(same, torch.arange(B, device=DEVICE), -1).amax(1) == torch.arange(B, device=DEVICE)
    shared = refs[part.clamp(min=0)]
    copies = (part >= 0) & (shared > 1) & ~(last & (same.sum(1) == shared))
    move = copies[:, None] & (at == (L // PAGE)[:, None])
    _changed(refs, torch.where(drop | move, table, -1), -1)
    table = torch.where(drop, -1, table)
    need = ((table < 0) & (at >= used) & (at < want)) | move
    free = torch.nonzero(refs == 0)[:, 0]
    taken = table.clone()
    taken[need] = free[: int(need.sum())]
    _changed(refs, torch.where(need, taken, -1), 1)
    from_page, to_page = table[move], taken[move]
    s.k_cache[:, to_page] = s.k_cache[:, from_page]
    if s.v_cache is not None:
        s.v_cache[:, to_page] = s.v_cache[:, from_page]
    s.page_table.copy_(taken)
    return _reserve_outputs(s)


def _reserve_outputs(s):
    # (pages are copied bit by bit: their words are compared, not the values)
    k, v = (c.view(torch.int16) if c is not None and c.dtype == torch.bfloat16 else c for c in (s.k_cache, s.v_cache))
    return {"page_table": s.page_table, "page_refs": s.page_refs, "k": k, "v": v, "status": s.status}


# ------------------------------------------------------------------------------------------------ a pass: the library's

def _library(s):
    """The library's call for this state, with the dimensions and the workspace that a program makes once."""
    from paper_2508_09072_amd import binding as R
    case = s.case
    kind, tree = case["kind"], case.get("form") == "tree"
    Hkv, D = case.get("Hkv", 1), case.get("D", 128)
    dims = R.make_dims(case["B"], case.get("T", 1), case.get("Hq", Hkv), Hkv, D, s.max_pages, case.get("path", 1), s.num_pages)
    room = lambda nbytes: torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=DEVICE)     # noqa: E731
    if kind == "store":
        if case["form"] == "pages":
            return lambda: R.reader_kvq_pack(dims, s.k, s.v, s.from_table, None, s.seq_lens, s.max_seq_len, s.kvq, s.page_table, s.status)
        return lambda: R.reader_kvq_store(dims, s.k, s.v, None if tree else s.cu_tokens, s.seq_lens, s.kvq, s.page_table, s.status)
    if kind == "attn":
        N = s.q.numel() // (case["Hq"] * D)
        ws = room(R.reader_kvq_workspace_bytes(dims, N, s.max_seq_len))
        if tree:
            return lambda: R.reader_kvq_tree_attn(dims, s.q, s.kvq, s.page_table, s.seq_lens, s.parents, s.out, s.lse, s.max_seq_len,
                                                  ws, s.status)
        return lambda: R.reader_kvq_prompt_attn(dims, s.q, s.kvq, s.page_table, s.cu_tokens, s.seq_lens, s.out, s.lse, s.max_seq_len,
                                                ws, s.status)
    if kind == "compact":
        return lambda: R.reader_kvq_compact_layers(dims, s.path, s.accept_len, s.kvq, s.page_table, s.seq_lens, s.status)
    ws = room(R.reader_pages_workspace_bytes(dims))
    if kind == "reorder":
        return lambda: R.reader_pages_reorder(dims, s.sources, s.page_table, s.seq_lens, s.page_refs, ws, s.status)
    return lambda: R.reader_pages_reserve(dims, s.seq_lens, s.new_lens, s.k_cache, s.v_cache, s.page_table, s.page_refs, ws, s.status)


def run(s):
    kind = s.case["kind"]
    if kind in ("compact", "reorder"):   # the steps in between have moved the lengths and the tables on
        s.seq_lens.copy_(s.seq_lens0)
    if kind in ("reorder", "reserve"):
        s.page_table.copy_(s.page_table0)
        s.page_refs.copy_(s.page_refs0)
    if not own:
        return {"store": _plain_store, "attn": _plain_attn, "compact": _plain_compact, "reorder": _plain_reorder,
                "reserve": _plain_reserve}[kind](s)
    if s.call is None:
        s.call = _library(s)
    s.call()
    if kind == "store":
        return {"kvq": s.kvq, "status": s.status}
    if kind == "attn":
        return {"out": s.out, "lse": s.lse, "status": s.status}
    if kind == "compact":
        return {"kvq": s.kvq, "seq_lens": s.seq_lens, "status": s.status}
    if kind == "reorder":
        return {"page_table": s.page_table, "seq_lens": s.seq_lens, "page_refs": s.page_refs, "status": s.status}
    return _reserve_outputs(s)


# ------------------------------------------------------------------------------------------------ what it comes to

def work(case):
    B, kind = case["B"], case["kind"]
    L, new = _lengths(case), _new(case)
    if kind == "reorder":
        src = _sources(case)
        held = _count(np.where(src >= 0, L[src.clip(0)], 0))
        return {"bytes": 4 * (_count(L) + held) + 4 * B * case["pages"] + 8 * (_count(L) + 7), "flops": 0}
    Hkv, D = case["Hkv"], case["D"]
    row4 = Hkv * (D + D // 16)                                     # bytes of a position in 4 bits, K and V
    if kind == "reserve":
        origin = _origins(case)
        part = np.unique(origin[L % PAGE > 0], return_counts=True)[1]
        copied = int((part - 1).sum())                             # the last one keeps the page
        page = PAGE * (row4 if case["form"] == "4-bit" else 4 * Hkv * D)
        return {"bytes": 2 * case["NL"] * copied * page + 8 * _count(L + case["more"]) + 8 * B, "flops": 0}
    if kind == "store":
        rows = int((L if case["form"] == "pages" else new).sum()) * case.get("NL", 1)
        return {"bytes": max(1, rows * (4 * Hkv * D + row4)), "flops": 4 * rows * Hkv * D}
    if kind == "compact":
        moved = int((_accepted(case) - 1).sum()) * case["NL"]
        return {"bytes": 2 * moved * row4 + 4 * B * (case["path"] + 3), "flops": 0}
    N, Hq = int(new.sum()), case["Hq"]
    # (row, key) pairs of one head that the program cannot skip: the cached ones, and up to each new token
    seen = int((new * L + new * (new + 1) // 2).sum())
    return {"bytes": 4 * N * Hq * D + int((L + new).sum()) * row4 + (4 * N * Hq if case["lse"] else 0), "flops": 4 * Hq * D * seen}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    """Of the attention alone: everything else is whole numbers."""
    if case["kind"] != "attn":
        return None
    s = prepare(case, seed)
    B, Hq, Hkv, D = case["B"], case["Hq"], case["Hkv"], case["D"]
    G, L, new = Hq // Hkv, _lengths(case).tolist(), _new(case).tolist()
    table = s.page_table.cpu().numpy()
    tree = case["form"] == "tree"
    q = s.q.double().view(-1, Hq, D)
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device=DEVICE)
    # byte and half byte of value d of row r of a page, from the layout's definition; magnitude of a code from its bits
    r, d = np.arange(PAGE)[:, None], np.arange(D)[None, :]
    quarter, sixteenth = D // 4, D // 16
    k_at = d // quarter * 8 * quarter + r * quarter // 2 + d % quarter // 2
    v_at = 8 * D + r // 4 * 2 * D + d // sixteenth * 2 * sixteenth + r % 4 * sixteenth // 2 + d % sixteenth // 2
    ks_at = 16 * D + d // 32 * 16 + r
    vs_at = 16 * D + D // 2 + r // 4 * (D // 8) + d // 32 * 4 + r % 4
    high = np.broadcast_to(d % 2 * 4, (PAGE, D))
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEVICE)                  # noqa: E731

    def values(block, at, scale_at):
        code = block[:, dev(at)].to(torch.int64) >> dev(high).to(torch.int64) & 15
        e, m = code >> 1 & 3, code & 1
        size = torch.where(e > 0, (1 + 0.5 * m.double()) * torch.exp2(e.double() - 1), 0.5 * m.double())
        x = torch.where(code > 7, -size, size) * torch.exp2(block[:, dev(scale_at)].double() - 127)
        return x.reshape(-1, D)

    first = 0
    for b in range(B):
        n, S = new[b], L[b] + new[b]
        page = dev(table[b, : (S + PAGE - 1) // PAGE].astype(np.int64))
        sees = torch.ones((n, S), dtype=torch.bool, device=DEVICE).tril(L[b])
        if tree:
            parents, mine = s.parents[b].tolist(), np.zeros((n, n), dtype=bool)
            for i in range(n):
                if i > 0:
                    mine[i] = mine[parents[i]]
                mine[i, i] = True
            sees[:, L[b]:] = dev(mine)
        for h in range(Hkv):
            block = s.kvq[page, h]
            k, v = values(block, k_at, ks_at)[:S], values(block, v_at, vs_at)[:S]
            x = q[first:first + n, h * G:(h + 1) * G].transpose(0, 1) @ k.t() / math.sqrt(D)     # [G, n, S]
            x = x.masked_fill(~sees, -math.inf)
            lse[first:first + n, h * G:(h + 1) * G] = torch.logsumexp(x, -1).t()
            out[first:first + n, h * G:(h + 1) * G] = (torch.softmax(x, -1) @ v).transpose(0, 1)
        first += n
    if tree:
        lse = lse.view(B, case["T"], Hq).transpose(1, 2)
    return {"out": out.view(s.out.shape), "lse": lse if case["lse"] else None, "status": None}
