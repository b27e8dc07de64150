"""What a serving program asks of the operators around the verification step, as a list of timed cases.

A program fills the paged cache from a prompt, decodes over it, and keeps it within a budget:

  qkv      the projections' output becomes normalised and rotated queries and keys: of a packed batch of prompt tokens
           (reader_prompt_qkv, K/V go into the paged cache) or of draft trees (reader_tree_qkv)
  attn     causal attention of the new tokens of every sequence over its cache (reader_prompt_attn): whole prompts, the
           next chunk of long ones, single tokens
  weights  the attention weight that every cached key has drawn (reader_key_weights: the accepted path of a step;
           reader_prompt_key_weights: the last tokens of a prompt)
  evict    the cache back to its budget: the newest and the heaviest keys of every kv head stay (reader_kv_evict)

A case is a dict of sizes and options.  `listed()` names the ones a serving program meets most, `draw()` gives more of
the same ranges, `prepare()` makes what the program has in hand before the call (from the seed alone), `run()` is one
pass, `work()` what the pass cannot do without, `exact()` its result in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False             # True: run() calls the library; False: it computes the same with elementary torch operations

DEVICE = "cuda:0"
PAGE = 16               # tokens per cache page
EPS = 1e-6
MOST_SCORES = 1 << 29   # scores the plain form holds at a time


# ------------------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # the smallest call of a decoding loop: one draft tree of a small model, no norms; launch and host time
        dict(name="qkv_tree_tiny", kind="qkv", form="tree", B=1, Hq=8, Hkv=8, D=64, T=16, L_lo=512, L_hi=512, norm=False,
             rot=64, interleaved=False, in_cache=False),
        # a decoding step of a large model with many users, tree rows behind each sequence in the cache
        dict(name="qkv_tree_large_batch", kind="qkv", form="tree", B=64, Hq=64, Hkv=8, D=128, T=64, L_lo=2048, L_hi=8192,
             norm=True, rot=128, interleaved=False, in_cache=True),
        # the prompts of a batch that has just arrived
        dict(name="qkv_prompts_packed", kind="qkv", form="prompt", B=16, Hq=32, Hkv=8, D=128, n_lo=301, n_hi=2500, L_lo=0,
             L_hi=0, norm=True, rot=128, interleaved=False),
        # one ordinary prompt of odd length
        dict(name="attn_one_prompt", kind="attn", B=1, Hq=32, Hkv=8, D=128, n_lo=777, n_hi=777, L_lo=0, L_hi=0, lse=False),
        # a long document: the largest call
        dict(name="attn_long_prompt", kind="attn", B=1, Hq=32, Hkv=8, D=128, n_lo=16384, n_hi=16384, L_lo=0, L_hi=0, lse=False),
        # a batch of ragged prompts, head dimension 64, log-sum-exp asked for (the eviction below needs it)
        dict(name="attn_packed_head64", kind="attn", B=12, Hq=32, Hkv=4, D=64, n_lo=100, n_hi=3001, L_lo=0, L_hi=0, lse=True),
        # the next chunk of two long documents, of a large model
        dict(name="attn_chunk_of_long", kind="attn", B=2, Hq=64, Hkv=8, D=128, n_lo=512, n_hi=512, L_lo=20000, L_hi=28000,
             lse=False),
        # plain decoding of a batch: one new token per sequence
        dict(name="attn_single_tokens", kind="attn", B=16, Hq=32, Hkv=8, D=128, n_lo=1, n_hi=1, L_lo=1024, L_hi=16384, lse=True),
        # behind every verification step of a batch: the accepted path's queries
        dict(name="weights_step", kind="weights", form="tree", B=16, Hq=32, Hkv=8, D=128, T=32, L_lo=1024, L_hi=4096, path=6,
             decay=1.0),
        # behind the prompts of four long documents: their last 32 tokens decide what stays
        dict(name="weights_prompt_window", kind="weights", form="prompt", B=4, Hq=32, Hkv=8, D=128, n_lo=100, n_hi=512,
             L_lo=20000, L_hi=32000, window=32, decay=0.0),
        # one layer of one user, a few hundred tokens over its budget
        dict(name="evict_one_layer", kind="evict", NL=1, B=1, Hkv=8, D=128, L_lo=4500, L_hi=4500, keep=4096, recent=256),
        # all layers of a small model after a batch of prompts
        dict(name="evict_all_layers", kind="evict", NL=16, B=8, Hkv=8, D=128, L_lo=3000, L_hi=8192, keep=2048, recent=128),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread evenly over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    Hkv = rng.choice((1, 2, 4, 8))
    return dict(Hq=Hkv * rng.choice((1, 3, 4, 8, 16)), Hkv=Hkv, D=rng.choice((64, 128, 128)))


def _most(kind):
    w = [work(c) for c in listed() if c["kind"] == kind]
    return max(x["bytes"] for x in w), max(x["flops"] for x in w)


def draw(rng):
    kind = rng.choice(("qkv", "qkv", "attn", "attn", "attn", "attn", "weights", "weights", "evict", "evict"))
    nbytes, flops = _most(kind)
    while True:
        if kind == "evict":
            L_hi = _log(rng, 40, 32768)
            keep = max(2, int(L_hi * rng.uniform(0.2, 0.95)))
            c = dict(kind=kind, NL=_log(rng, 1, 32), B=_log(rng, 1, 32), Hkv=rng.choice((1, 2, 4, 8)), D=rng.choice((64, 128, 128)),
                     L_lo=max(1, int(L_hi * rng.choice((0.1, 0.5, 1.0)))), L_hi=L_hi, keep=keep, recent=rng.randint(0, keep // 2))
            if c["NL"] * c["B"] * c["Hkv"] * L_hi * c["D"] > 16 * 8 * 8 * 8192 * 128:
                continue
        else:
            form = rng.choice(("tree", "prompt"))
            c = dict(kind=kind, B=_log(rng, 1, 64), **_heads(rng))
            if kind == "attn" or form == "prompt":
                n_hi = rng.choice((1, _log(rng, 1, 128), _log(rng, 1, 16384), _log(rng, 128, 8192)))
                c.update(n_lo=max(1, int(n_hi * rng.choice((0.05, 0.25, 1.0)))), n_hi=n_hi)
                L_hi = rng.choice((0, _log(rng, 1, 32768), _log(rng, 256, 16384)))
            else:
                c.update(T=_log(rng, 1, 128))
                L_hi = _log(rng, 64, 32768)
            c.update(L_lo=int(L_hi * rng.choice((0.1, 0.5, 1.0))), L_hi=L_hi)
            if kind == "qkv":
                c.update(form=form, norm=rng.random() < 0.6, rot=rng.choice((c["D"], c["D"], c["D"] // 2, c["D"] // 4)),
                         interleaved=rng.random() < 0.4)
                if form == "tree":
                    c["in_cache"] = rng.random() < 0.5
            elif kind == "attn":
                c["lse"] = rng.random() < 0.5
            else:
                c.update(form=form, decay=rng.choice((0.0, 1.0, 0.9)))
                c["path" if form == "tree" else "window"] = rng.randint(1, min(c["T"], 16)) if form == "tree" else _log(rng, 1, 128)
            pages = c["B"] * (c["L_hi"] + c.get("n_hi", c.get("T", 0)))
            if pages * c["Hkv"] * c["D"] > 4 << 28:
                continue
        w = work(c)
        if w["bytes"] <= nbytes and w["flops"] <= flops:
            return c


# ------------------------------------------------------------------------------------------------ inputs

def _spread(lo, hi, n, turn=0.6180339887498949):
    """n whole numbers between lo and hi, part of the case: the golden-ratio sequence spreads them evenly."""
    return np.asarray([lo + int((hi - lo + 1) * (((i + 1) * turn) % 1.0)) if hi > lo else lo for i in range(n)], dtype=np.int64)


def _lengths(case):
    return _spread(case["L_lo"], case["L_hi"], case["B"])


def _new(case):
    """New tokens of each sequence."""
    if case["kind"] != "evict" and "n_hi" in case:
        return _spread(case["n_lo"], case["n_hi"], case["B"], 0.7548776662466927)
    return np.full((case["B"],), case.get("T", 0), dtype=np.int64)


def _accepted(case):
    """Nodes of the accepted path (the root among them) of each sequence, part of the case."""
    return _spread(1, case["path"], case["B"], 0.7548776662466927)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEVICE)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.bfloat16)


def _cos_sin(n, rot):
    """The rotation table of a model: cosines, then sines, of position * 10000^(-2 i / rot), made in 64 bits."""
    freq = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEVICE) / rot)
    angle = torch.arange(n, dtype=torch.float64, device=DEVICE)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().contiguous()


class _State:
    """A program's buffers."""

    def __init__(self, case):
        self.case = case
        self.call = None          # the library's arguments, made at the first pass


def _pages(s, rng, lengths):
    """A page table for these lengths: physical order is a random permutation, a few pages are spare."""
    need = (np.asarray(lengths, dtype=np.int64) + PAGE - 1) // PAGE
    s.max_pages, s.num_pages = max(1, int(need.max())), int(need.sum()) + 3
    table = np.full((len(lengths), s.max_pages), -1, dtype=np.int32)
    table[np.arange(s.max_pages)[None, :] < need[:, None]] = rng.permutation(s.num_pages)[: int(need.sum())]
    s.page_table = _i32(table)


def prepare(case, seed):
    rng = np.random.Generator(np.random.PCG64(seed))
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    s = _State(case)
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    kind, L, new = case["kind"], _lengths(case), _new(case)
    s.seq_lens0 = _i32(L)
    s.seq_lens = s.seq_lens0.clone()
    s.status = torch.zeros((1,), dtype=torch.int32, device=DEVICE)
    if kind == "evict":
        NL = case["NL"]
        _pages(s, rng, L)
        s.k_cache = _normal(gen, NL, s.num_pages, Hkv, PAGE, D)
        s.v_cache = _normal(gen, NL, s.num_pages, Hkv, PAGE, D)
        # accumulated weights: a few heavy keys, a long tail, and many light ones that are equal
        s.max_positions = s.max_pages * PAGE
        w = torch.randn((NL, B, Hkv, s.max_positions), generator=gen, device=DEVICE).mul_(2).exp_()
        w = torch.where(w < 0.3, torch.full_like(w, 0.25), w)
        w.mul_(torch.arange(s.max_positions, device=DEVICE) < s.seq_lens0[:, None, None])
        s.weights0, s.weights = w, w.clone()
        return s
    Hq = case["Hq"]
    _pages(s, rng, L + new)
    tree = case.get("form") == "tree"
    N = int(new.sum())
    s.cu_tokens = _i32(np.concatenate([[0], np.cumsum(new)]))
    s.max_seq_len = int((L + new).max())
    if kind == "qkv":
        s.qkv = _normal(gen, *((B, case["T"]) if tree else (N,)), Hq + 2 * Hkv, D)
        s.q_norm = s.k_norm = None
        if case["norm"]:
            s.q_norm = (1 + 0.2 * torch.randn((D,), generator=gen, device=DEVICE)).to(torch.bfloat16)
            s.k_norm = (1 + 0.2 * torch.randn((D,), generator=gen, device=DEVICE)).to(torch.bfloat16)
        s.cos_sin = _cos_sin(s.max_seq_len, case["rot"])
        s.q = torch.zeros((*s.qkv.shape[:-2], Hq, D), dtype=torch.bfloat16, device=DEVICE)
        s.k_tree = s.v_tree = s.k_cache = s.v_cache = None
        if tree:
            parents = np.full((B, case["T"]), -1, dtype=np.int32)
            for i in range(1, case["T"]):                      # bushy trees a few levels deep
                parents[:, i] = rng.integers(max(0, i // 4 - 2), i, size=B)
            s.parents = _i32(parents)
        if tree and not case["in_cache"]:
            s.k_tree = torch.zeros((B, case["T"], Hkv, D), dtype=torch.bfloat16, device=DEVICE)
            s.v_tree = torch.zeros_like(s.k_tree)
        else:
            s.k_cache = torch.zeros((s.num_pages, Hkv, PAGE, D), dtype=torch.bfloat16, device=DEVICE)
            s.v_cache = torch.zeros_like(s.k_cache)
        return s
    s.k_cache = _normal(gen, s.num_pages, Hkv, PAGE, D)
    if kind == "attn":
        s.v_cache = _normal(gen, s.num_pages, Hkv, PAGE, D)
        if case["L_hi"] >= 16384:                              # long contexts: one key in twenty stands out
            hot = torch.rand((s.num_pages, 1, PAGE, 1), generator=gen, device=DEVICE) < 0.05
            s.k_cache.mul_(1 + 3 * hot)
        s.q = _normal(gen, N, Hq, D)
        s.out = torch.zeros_like(s.q)
        s.lse = torch.zeros((N, Hq), dtype=torch.float32, device=DEVICE) if case["lse"] else None
        return s
    # weights: query rows and the log-sum-exp that the attention gave for them (of normal scores: log of the keys + 1/2)
    seen = torch.from_numpy(L + new).to(DEVICE).float().clamp_(min=1).log() + 0.5
    if tree:
        n = _accepted(case)
        s.q = _normal(gen, B, case["T"], Hq, D)
        s.lse = seen[:, None, None] + 0.3 * torch.randn((B, Hq, case["T"]), generator=gen, device=DEVICE)
        path = np.full((B, case["path"]), -1, dtype=np.int32)
        for b in range(B):
            path[b, : n[b]] = np.concatenate([[0], 1 + np.sort(rng.permutation(case["T"] - 1)[: n[b] - 1])])
        s.path, s.accept_len = _i32(path), _i32(n - 1)
        s.seq_lens = _i32(L + n)                               # the step has appended the path
    else:
        s.q = _normal(gen, N, Hq, D)
        s.lse = torch.repeat_interleave(seen, torch.from_numpy(new).to(DEVICE))[:, None] + \
            0.3 * torch.randn((N, Hq), generator=gen, device=DEVICE)
    s.max_positions = s.max_pages * PAGE
    s.weights = torch.rand((B, Hkv, s.max_positions), generator=gen, device=DEVICE)
    s.weights.mul_(torch.arange(s.max_positions, device=DEVICE) < s.seq_lens0[:, None, None])
    return s


# ------------------------------------------------------------------------------------------------ a pass: the plain forms

def _slots(s, lo, hi, b):
    """Rows of the flattened [pages * page] axis that positions lo .. hi - 1 of sequence b live in."""
    at = torch.arange(lo, hi, device=DEVICE)
    return s.page_table[b].long()[at // PAGE] * PAGE + at % PAGE


def _keys(cache, s, b, n):
    """The first n rows of sequence b, [Hkv, n, D] in 32 bits."""
    at = torch.arange(n, device=DEVICE)
    return cache[s.page_table[b].long()[at // PAGE], :, at % PAGE].float().transpose(0, 1)


def _norm_rotate(x, w, cos, sin, rot, interleaved):
    """x [..., heads, D] in 32 bits, cos and sin [..., 1, rot / 2]."""
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., : rot // 2], r[..., rot // 2:])
    c, d = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([c, d], dim=-1).flatten(-2) if interleaved else torch.cat([c, d], dim=-1)
    return torch.cat([r, x[..., rot:]], dim=-1).to(torch.bfloat16)


def _depths(parents):
    """Depth of every tree node, by doubling the links."""
    T = parents.shape[1]
    up = torch.cat([parents.long() + 1, torch.zeros_like(parents[:, :1]).long()], dim=1).roll(1, 1)   # entry 0: above the root
    d = torch.ones_like(up)
    d[:, 0] = 0
    for _ in range(max(1, T.bit_length())):
        d, up = d + d.gather(1, up), up.gather(1, up)
    return d[:, 1:] - 1


def _plain_qkv(s):
    case = s.case
    Hq, Hkv, tree = case["Hq"], case["Hkv"], case["form"] == "tree"
    new = s.cu_tokens.long().diff()
    seq = torch.repeat_interleave(torch.arange(case["B"], device=DEVICE), new)
    row = torch.arange(seq.numel(), device=DEVICE) - s.cu_tokens.long()[seq]
    x = s.qkv.float()
    at = s.seq_lens.long()[seq] + row                          # where a token's rows live in the cache
    pos = s.seq_lens.long()[:, None] + _depths(s.parents) if tree else at
    half = case["rot"] // 2
    cos, sin = s.cos_sin[pos][..., None, :half], s.cos_sin[pos][..., None, half:]
    s.q.copy_(_norm_rotate(x[..., :Hq, :], s.q_norm, cos, sin, case["rot"], case["interleaved"]))
    k = _norm_rotate(x[..., Hq:Hq + Hkv, :], s.k_norm, cos, sin, case["rot"], case["interleaved"])
    v = s.qkv[..., Hq + Hkv:, :]
    if tree and not case["in_cache"]:
        s.k_tree.copy_(k)
        s.v_tree.copy_(v)
    else:
        page = s.page_table.long()[seq, at // PAGE]
        s.k_cache[page, :, at % PAGE] = k.reshape(-1, Hkv, case["D"])
        s.v_cache[page, :, at % PAGE] = v.reshape(-1, Hkv, case["D"])
    return _qkv_outputs(s)


def _qkv_outputs(s):
    if s.k_tree is not None:
        return {"q": s.q, "k": s.k_tree, "v": s.v_tree, "status": s.status}
    return {"q": s.q, "k": s.k_cache, "v": s.v_cache, "status": s.status}


def _plain_attn(s):
    case = s.case
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    G, L, new = Hq // Hkv, _lengths(case), _new(case)
    first = 0
    for b in range(case["B"]):
        n, S = int(new[b]), int(L[b] + new[b])
        k, v = _keys(s.k_cache, s, b, S), _keys(s.v_cache, s, b, S)
        q = s.q[first:first + n].float().view(n, Hkv, G, D)
        step = max(1, MOST_SCORES // (Hq * S))
        for lo in range(0, n, step):
            rows = min(step, n - lo)
            x = q[lo:lo + rows].permute(1, 0, 2, 3).reshape(Hkv, rows * G, D) @ k.transpose(1, 2) * D ** -0.5
            last = int(L[b]) + lo + torch.arange(rows, device=DEVICE).repeat_interleave(G)
            x.masked_fill_(torch.arange(S, device=DEVICE)[None, :] > last[:, None], -math.inf)
            m = x.amax(-1, keepdim=True)
            x = x.sub_(m).exp_()
            total = x.sum(-1, keepdim=True)
            o = (x @ v / total).view(Hkv, rows, G, D).permute(1, 0, 2, 3).reshape(rows, Hq, D)
            s.out[first + lo:first + lo + rows] = o.to(torch.bfloat16)
            if s.lse is not None:
                s.lse[first + lo:first + lo + rows] = (m + total.log()).view(Hkv, rows, G).permute(1, 0, 2).reshape(rows, Hq)
        first += n
    return {"out": s.out, "lse": s.lse, "status": s.status}


def _weight_rows(s, b):
    """Queries and log-sum-exp of the rows that count for sequence b, and the position of the first of them."""
    case = s.case
    if case["form"] == "tree":
        n = int(_accepted(case)[b])
        nodes = s.path[b, :n].long()
        return s.q[b, nodes], s.lse[b][:, nodes].t(), int(_lengths(case)[b])
    new = _new(case)
    n, end = min(case["window"], int(new[b])), int(new[: b + 1].sum())
    return s.q[end - n:end], s.lse[end - n:end], int(_lengths(case)[b] + new[b]) - n


def _plain_weights(s):
    case = s.case
    Hkv, D = case["Hkv"], case["D"]
    G = case["Hq"] // Hkv
    for b in range(case["B"]):
        q, lse, first = _weight_rows(s, b)
        n = q.shape[0]
        S = first + n
        x = q.float().view(n, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, n * G, D) @ _keys(s.k_cache, s, b, S).transpose(1, 2)
        x = (x * D ** -0.5 - lse.reshape(n, Hkv, G).permute(1, 0, 2).reshape(Hkv, n * G, 1)).exp()
        last = first + torch.arange(n, device=DEVICE).repeat_interleave(G)
        x.masked_fill_(torch.arange(S, device=DEVICE)[None, :] > last[:, None], 0.0)
        old = s.weights[b, :, :S] * case["decay"] if case["decay"] else 0.0
        s.weights[b, :, :S] = old + x.sum(1)
        if not case["decay"]:
            s.weights[b, :, S:] = 0.0
    return {"weights": s.weights, "status": s.status}


def _plain_evict(s):
    case = s.case
    keep, recent, L = case["keep"], case["recent"], _lengths(case)
    for b in range(case["B"]):
        n = int(L[b])
        if n <= keep:
            continue
        w = s.weights[:, b, :, :n]
        heavy = w[..., : n - recent].sort(dim=-1, descending=True, stable=True).indices[..., : keep - recent]
        newest = torch.arange(n - recent, n, device=DEVICE).expand(*w.shape[:2], recent)
        src = torch.cat([heavy, newest], dim=-1).sort(dim=-1).values                    # [NL, Hkv, keep]
        at = _slots(s, 0, n, b)
        for cache in (s.k_cache, s.v_cache):
            rows = cache.permute(0, 2, 1, 3, 4)                                          # [NL, Hkv, pages, page, D]
            layer = torch.arange(case["NL"], device=DEVICE)[:, None, None]
            head = torch.arange(case["Hkv"], device=DEVICE)[None, :, None]
            rows[layer, head, at[:keep] // PAGE, at[:keep] % PAGE] = rows[layer, head, at[src] // PAGE, at[src] % PAGE]
        kept = w.gather(-1, src)
        w.zero_()
        w[..., :keep] = kept
        s.seq_lens[b] = keep
    return _evict_outputs(s)


def _evict_outputs(s):
    return {"k_cache": s.k_cache, "v_cache": s.v_cache, "weights": s.weights, "seq_lens": s.seq_lens, "status": s.status}


# ------------------------------------------------------------------------------------------------ a pass: the library's

def _library(s):
    """The library's call for this state, with the dimensions and the workspace that a program makes once."""
    from paper_2508_09072_amd import binding as R
    case = s.case
    kind, tree = case["kind"], case.get("form") == "tree"
    dims = R.make_dims(case["B"], case.get("T", 1), case.get("Hq", case["Hkv"]), case["Hkv"], case["D"], s.max_pages,
                       case.get("path", 1), s.num_pages)
    if kind == "qkv":
        if tree:
            return lambda: R.reader_tree_qkv(dims, s.qkv, s.parents, s.seq_lens, None, s.q_norm, s.k_norm, EPS, s.cos_sin,
                                             case["interleaved"], s.q, s.k_tree, s.v_tree, s.k_cache, s.v_cache,
                                             s.page_table, s.status)
        return lambda: R.reader_prompt_qkv(dims, s.qkv, s.cu_tokens, s.seq_lens, None, s.q_norm, s.k_norm, EPS, s.cos_sin,
                                           case["interleaved"], s.q, s.k_cache, s.v_cache, s.page_table, s.status)
    if kind == "attn":
        nbytes = R.reader_prompt_workspace_bytes(dims, s.q.shape[0], s.max_seq_len)
        ws = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=DEVICE)
        return lambda: R.reader_prompt_attn(dims, s.q, s.k_cache, s.v_cache, s.page_table, s.cu_tokens, s.seq_lens, s.out,
                                            s.lse, s.max_seq_len, ws, s.status)
    if kind == "weights":
        if tree:
            return lambda: R.reader_key_weights(dims, s.q, s.lse, s.path, s.accept_len, s.k_cache, s.page_table, s.seq_lens,
                                                case["decay"], s.weights, s.max_seq_len, s.status)
        return lambda: R.reader_prompt_key_weights(dims, s.q, s.lse, s.cu_tokens, case["window"], s.k_cache, s.page_table,
                                                   s.seq_lens, case["decay"], s.weights, s.max_seq_len, s.status)
    nbytes = R.reader_kv_evict_workspace_bytes(dims, case["NL"], case["keep"])
    ws = torch.empty((max(nbytes, 256),), dtype=torch.uint8, device=DEVICE)
    return lambda: R.reader_kv_evict(dims, case["keep"], case["recent"], s.k_cache, s.v_cache, s.page_table, s.seq_lens,
                                     s.weights, ws, s.status)


def run(s):
    kind = s.case["kind"]
    if kind == "evict":                  # the steps in between have filled the cache and the weights again
        s.seq_lens.copy_(s.seq_lens0)
        s.weights.copy_(s.weights0)
    if not own:
        return {"qkv": _plain_qkv, "attn": _plain_attn, "weights": _plain_weights, "evict": _plain_evict}[kind](s)
    if s.call is None:
        s.call = _library(s)
    s.call()
    if kind == "qkv":
        return _qkv_outputs(s)
    if kind == "attn":
        return {"out": s.out, "lse": s.lse, "status": s.status}
    if kind == "weights":
        return {"weights": s.weights, "status": s.status}
    return _evict_outputs(s)


# ------------------------------------------------------------------------------------------------ what it comes to

def work(case):
    B, Hkv, D, kind = case["B"], case["Hkv"], case["D"], case["kind"]
    L, new = _lengths(case), _new(case)
    N = int(new.sum())
    if kind == "qkv":
        values = N * (case["Hq"] + 2 * Hkv) * D
        positions = int((L + new).max()) if B else 0
        return {"bytes": 4 * values + 4 * case["rot"] * min(N, positions), "flops": 8 * N * (case["Hq"] + Hkv) * D}
    if kind == "attn":
        keys = int((L + new).sum())
        seen = int((new * L + new * (new + 1) // 2).sum())             # (row, key) pairs of one head
        return {"bytes": 4 * N * case["Hq"] * D + 4 * keys * Hkv * D + (4 * N * case["Hq"] if case["lse"] else 0),
                "flops": 4 * case["Hq"] * D * seen}
    if kind == "weights":
        n = _accepted(case) if case["form"] == "tree" else np.minimum(new, case["window"])
        S = L + (n if case["form"] == "tree" else new)
        seen = int((n * (S - n) + n * (n + 1) // 2).sum())
        weights = (8 if case["decay"] else 4) * Hkv * int(S.sum())
        return {"bytes": 2 * Hkv * D * int(S.sum()) + 2 * case["Hq"] * D * int(n.sum()) + weights, "flops": 2 * case["Hq"] * D * seen}
    over = L[L > case["keep"]]
    heads = case["NL"] * Hkv
    rows = case["keep"] * over.size * heads
    return {"bytes": max(1, 8 * rows * D + 8 * heads * int(over.sum())), "flops": 0}


# ------------------------------------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    B, Hkv, D, kind = case["B"], case["Hkv"], case["D"], case["kind"]
    L, new = _lengths(case).tolist(), _new(case).tolist()
    table = s.page_table.cpu().numpy()

    def rows(b, n):
        """Page and slot of every position of sequence b."""
        j = np.arange(n)
        return torch.from_numpy(table[b, j // PAGE].astype(np.int64)).to(DEVICE), torch.from_numpy(j % PAGE).to(DEVICE)

    if kind == "evict":
        k, v, w = s.k_cache.double(), s.v_cache.double(), s.weights0.double()
        for b in range(B):
            n, keep, recent = L[b], case["keep"], case["recent"]
            if n <= keep:
                continue
            page, slot = rows(b, n)
            mass = s.weights0[:, b, :, :n].double().cpu().numpy().reshape(-1, n)
            for i, m in enumerate(mass):
                layer, head = divmod(i, Hkv)
                order = np.lexsort((np.arange(n - recent), -m[: n - recent]))           # heaviest first, then lowest position
                src = torch.from_numpy(np.sort(np.concatenate([order[: keep - recent], np.arange(n - recent, n)]))).to(DEVICE)
                for c in (k, v):
                    c[layer, page[:keep], head, slot[:keep]] = c[layer, page[src], head, slot[src]]
                row = w[layer, b, head]
                kept = row[src]
                row[:n] = 0
                row[:keep] = kept
        return {"k_cache": k, "v_cache": v, "weights": w, "seq_lens": None, "status": None}
    Hq = case["Hq"]
    G = Hq // Hkv
    if kind == "qkv":
        tree, rot = case["form"] == "tree", case["rot"]
        x = s.qkv.double().reshape(-1, Hq + 2 * Hkv, D)
        where = []                                             # (sequence, position in the cache, rotary position) of every token
        for b in range(B):
            depth = []
            for i in range(new[b]):
                depth.append(i if not tree else 0 if i == 0 else depth[int(s_parent(s, b, i))] + 1)
                where.append((b, L[b] + i, L[b] + depth[i]))
        where = torch.tensor(where, device=DEVICE)
        table64 = s.cos_sin.double()[where[:, 2]]
        turn = torch.complex(table64[:, : rot // 2], table64[:, rot // 2:])[:, None]
        heads = []
        for part, w in ((x[:, :Hq], s.q_norm), (x[:, Hq:Hq + Hkv], s.k_norm)):
            if w is not None:
                part = part / (part.square().sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
            pairs = part[..., :rot].unflatten(-1, (rot // 2, 2) if case["interleaved"] else (2, rot // 2))
            z = torch.complex(*(pairs.unbind(-1) if case["interleaved"] else pairs.unbind(-2))) * turn
            z = torch.view_as_real(z)
            heads.append(torch.cat([(z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2), part[..., rot:]], -1))
        q, k, v = heads[0].reshape(s.q.shape), heads[1], x[:, Hq + Hkv:]
        if s.k_tree is not None:
            return {"q": q, "k": k.reshape(s.k_tree.shape), "v": v.reshape(s.k_tree.shape), "status": None}
        kc, vc = s.k_cache.double(), s.v_cache.double()
        page = s.page_table.long()[where[:, 0], where[:, 1] // PAGE]
        kc[page, :, where[:, 1] % PAGE] = k
        vc[page, :, where[:, 1] % PAGE] = v
        return {"q": q, "k": kc, "v": vc, "status": None}
    if kind == "attn":
        if work(case)["flops"] > 3e12:
            return None
        out = torch.zeros(s.q.shape, dtype=torch.float64, device=DEVICE)
        lse = torch.zeros(s.q.shape[:2], dtype=torch.float64, device=DEVICE)
        first = 0
        for b in range(B):
            page, slot = rows(b, L[b] + new[b])
            for h in range(Hq):
                k, v = s.k_cache[page, h // G, slot].double(), s.v_cache[page, h // G, slot].double()
                for lo in range(0, new[b], 2048):
                    hi = min(new[b], lo + 2048)
                    S = L[b] + hi
                    x = s.q[first + lo:first + hi, h].double() @ k[:S].t() / math.sqrt(D)
                    hide = torch.ones((hi - lo, S), dtype=torch.bool, device=DEVICE).triu(L[b] + lo + 1)
                    x = x.masked_fill(hide, -math.inf)
                    lse[first + lo:first + hi, h] = torch.logsumexp(x, -1)
                    out[first + lo:first + hi, h] = torch.softmax(x, -1) @ v[:S]
            first += new[b]
        return {"out": out, "lse": lse if case["lse"] else None, "status": None}
    weights = s.weights.double() * case["decay"]
    for b in range(B):
        if case["form"] == "tree":
            take = [(b, int(t)) for t in s.path[b].tolist() if t >= 0]
            start = L[b]
        else:
            end = sum(new[: b + 1])
            take = list(range(end - min(case["window"], new[b]), end))
            start = L[b] + new[b] - len(take)
        page, slot = rows(b, start + len(take))
        for i, t in enumerate(take):
            qt, lt = (s.q[t], s.lse[t[0], :, t[1]]) if case["form"] == "tree" else (s.q[t], s.lse[t])
            S = start + i + 1
            kk = s.k_cache[page[:S], :, slot[:S]].double()                            # [S, Hkv, D]
            x = (kk.transpose(0, 1) @ qt.double().view(Hkv, G, D).transpose(1, 2)) / math.sqrt(D)
            weights[b, :, :S] += torch.exp(x - lt.double().view(Hkv, 1, G)).sum(-1)
    return {"weights": weights, "status": None}


def s_parent(s, b, i):
    """Parent of node i of sequence b's tree (on the host)."""
    if not hasattr(s, "parents_host"):
        s.parents_host = s.parents.cpu().numpy()
    return s.parents_host[b, i]
