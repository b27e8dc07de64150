"""The operators around the verification step together, as a program runs them: prompts in two chunks, eviction, a
verification step over what is left, its weights, another eviction.  Every stage is held against its 64-bit form on what
the stage before left on the card.  Then the same chain captured, on other streams, and in caches larger than 32 bits
count."""
import math

import pytest
import torch

import prompt_helpers as P

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def R():
    from paper_2508_09072_amd import binding
    binding.load()
    return binding


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def rotation(n, rot):
    a = torch.arange(n, dtype=torch.float64)[:, None] * 500.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([a.cos(), a.sin()], 1).float()


class Model:
    """Projections, weights and a cache of a few layers; `run` is a program's calls and records what they leave."""

    def __init__(self, R, Hq, Hkv, D, in_cache, seed, chunks=((40, 17, 0), (25, 0, 90)), keep=32, recent=9, window=20, accepted=(3, 1, 5)):
        gen = torch.Generator().manual_seed(seed)
        self.R, self.Hq, self.Hkv, self.D, self.in_cache, self.keep, self.recent, self.window = R, Hq, Hkv, D, in_cache, keep, recent, window
        self.NL, self.B, self.T, self.mp, self.chunks, self.accepted = 2, len(chunks[0]), 14, 6, chunks, accepted
        total = [sum(c[b] for c in chunks) for b in range(self.B)]
        self.total = total
        self.cache = P.Cache(gen, [t + self.T for t in total], Hkv, D, lead=(self.NL,))
        self.k, self.v, self.table = self.cache.k.cuda(), self.cache.v.cuda(), self.cache.table.cuda()
        self.bound, self.cached, W = max(total) + self.T, max(total), max(total) + self.T + 3
        self.w = torch.full((self.NL, self.B, Hkv, W), math.nan, device="cuda")
        rand = lambda *s: torch.randn(s, generator=gen).bfloat16().cuda()  # noqa: E731
        heads = Hq + 2 * Hkv
        self.x = [[rand(sum(c), heads, D) for c in chunks] for _ in range(self.NL)]
        self.tree_x = [rand(self.B, self.T, heads, D) for _ in range(self.NL)]
        self.qn, self.kn = [(1 + 0.3 * torch.randn(D, generator=gen)).bfloat16().cuda() for _ in range(2)]
        self.cs = rotation(max(total) + self.T + 1, D // 2).cuda()
        self.cu = [i32([0] + list(torch.cumsum(torch.tensor(c), 0))) for c in chunks]
        # trees: a chain of accepted nodes among others (node 0 is the root), draft tokens and the model's answers
        parents = torch.tensor([[-1] + [int(torch.randint(0, i, (1,), generator=gen)) for i in range(1, self.T)] for _ in range(self.B)])
        draft = torch.arange(self.T).repeat(self.B, 1) + 100       # (all different)
        target = torch.zeros_like(draft)
        self.paths = []
        for b, n in enumerate(accepted):
            path = sorted(torch.randperm(self.T - 1, generator=gen)[:n].add(1).tolist())
            parents[b, path] = torch.tensor([0] + path[:-1])
            for a, c in zip([0] + path[:-1], path):
                target[b, a] = draft[b, c]
            self.paths.append([0] + path)
        self.parents_host = parents
        self.parents, self.draft, self.target = i32(parents), i32(draft), i32(target)
        self.status, self.lens, self.text = i32([0]), i32([0] * self.B), i32([0] * self.B)
        self.dims = R.make_dims(self.B, self.T, Hq, Hkv, D, self.cache.max_pages, self.mp, self.cache.num_pages)
        dev = dict(device="cuda")
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.q = [[torch.zeros((sum(c), Hq, D), **bf) for c in chunks] for _ in range(self.NL)]
        self.out = [[torch.zeros_like(t) for t in layer] for layer in self.q]
        self.lse = [[torch.zeros(t.shape[:2], **dev) for t in layer] for layer in self.q]
        self.tq = [torch.zeros((self.B, self.T, Hq, D), **bf) for _ in range(self.NL)]
        self.kt = [None if in_cache else torch.zeros((self.B, self.T, Hkv, D), **bf) for _ in range(self.NL)]
        self.vt = [None if in_cache else torch.zeros((self.B, self.T, Hkv, D), **bf) for _ in range(self.NL)]
        self.tout, self.tlse = [torch.zeros_like(t) for t in self.tq], [torch.zeros((self.B, Hq, self.T), **dev) for _ in range(self.NL)]
        self.accept, self.path, self.bonus = i32([0] * self.B), torch.zeros((self.B, self.mp), dtype=torch.int32, device="cuda"), i32([0] * self.B)
        self.layer_lens = [i32([0] * self.B) for _ in range(self.NL)]
        need = max([R.reader_prompt_workspace_bytes(self.dims, sum(c), self.bound) for c in chunks]
                   + [R.reader_workspace_bytes(self.dims, self.cached), R.reader_kv_evict_workspace_bytes(self.dims, self.NL, keep), 256])
        self.ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
        self.start = [t.clone() for t in (self.k, self.v, self.w, self.lens, self.text)]
        self.empty = torch.zeros_like(self.w)

    def reset(self):
        for t, s in zip((self.k, self.v, self.w, self.lens, self.text), self.start):
            t.copy_(s)
        self.status.zero_()
        for group in (self.q, self.out, self.lse):
            for layer in group:
                for t in layer:
                    t.zero_()
        for group in (self.tq, self.tout, self.tlse):
            for t in group:
                t.zero_()

    def left(self):
        flat = [t for group in (self.q, self.out, self.lse) for layer in group for t in layer] + self.tq + self.tout + self.tlse
        return flat + [self.k, self.v, self.w, self.lens, self.text, self.accept, self.path, self.bonus, self.status]

    def chunk(self, c):
        R, d, N = self.R, self.dims, sum(self.chunks[c])
        for l in range(self.NL):
            R.reader_prompt_qkv(d, self.x[l][c], self.cu[c], self.lens, self.text, self.qn, self.kn, EPS, self.cs, False, self.q[l][c],
                                self.k[l], self.v[l], self.table, self.status)
            R.reader_prompt_attn(d, self.q[l][c], self.k[l], self.v[l], self.table, self.cu[c], self.lens, self.out[l][c], self.lse[l][c],
                                 self.bound, self.ws, self.status)
            R.reader_prompt_key_weights(d, self.q[l][c], self.lse[l][c], self.cu[c], self.window, self.k[l], self.table, self.lens,
                                        0.0 if c == 0 else 0.5, self.w[l], self.bound, self.status)
        new = self.cu[c][1:] - self.cu[c][:-1]
        self.lens += new
        self.text += new

    def evict(self):
        self.R.reader_kv_evict(self.dims, self.keep, self.recent, self.k, self.v, self.table, self.lens, self.w, self.ws, self.status)

    def nodes(self, l):
        self.R.reader_tree_qkv(self.dims, self.tree_x[l], self.parents, self.lens, self.text, self.qn, self.kn, EPS, self.cs, False,
                               self.tq[l], self.kt[l], self.vt[l], self.k[l], self.v[l], self.table, self.status)

    def step(self, l):
        R, d = self.R, self.dims
        lens = self.layer_lens[l].copy_(self.lens)
        self.nodes(l)
        R.reader_verify_step(d, self.tq[l], self.kt[l], self.vt[l], self.k[l], self.v[l], self.table, lens, self.parents, self.draft,
                             self.target, self.tout[l], self.tlse[l], self.accept, self.path, self.bonus, self.cached, self.ws, self.status)
        R.reader_key_weights(d, self.tq[l], self.tlse[l], self.path, self.accept, self.k[l], self.table, lens, 1.0, self.w[l],
                             self.bound, self.status)

    def steps(self):
        for l in range(self.NL):
            self.step(l)
        self.text += self.layer_lens[0] - self.lens
        self.lens.copy_(self.layer_lens[0])

    def run(self):
        for c in range(len(self.chunks)):
            self.chunk(c)
        self.evict()
        self.steps()
        self.evict()

    def run_to_the_step(self):
        for c in range(len(self.chunks)):
            self.chunk(c)
        self.evict()
        for l in range(self.NL):
            self.nodes(l)


def rows(model, l, b, n):
    c = model.cache
    page, slot = c.place(b, n)
    return [t[l].cpu()[page, :, slot].double().transpose(0, 1) for t in (model.k, model.v)]


def bits(t):
    return t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32)


@pytest.mark.parametrize("Hq,Hkv,D", [(8, 2, 128), (6, 2, 64), (4, 4, 64)])
@pytest.mark.parametrize("in_cache", [False, True])
def test_together(R, Hq, Hkv, D, in_cache):
    m = Model(R, Hq, Hkv, D, in_cache, seed=Hq * D)
    NL, B = m.NL, m.B
    qn, kn, cs = m.qn.cpu(), m.kn.cpu(), m.cs.cpu()
    for c in range(2):
        L, old = m.lens.cpu().tolist(), m.w.cpu()
        m.chunk(c)
        assert int(m.status) == 0
        cu = m.cu[c].cpu().tolist()
        for l in range(NL):
            for b in range(B):
                lo, hi = cu[b], cu[b + 1]
                n = hi - lo
                x, pos = m.x[l][c][lo:hi].cpu(), L[b] + torch.arange(n)
                k, v = rows(m, l, b, L[b] + n)
                if n:
                    wq, bq = P.norm_rotate(x[:, :Hq], qn, EPS, cs, pos, False)
                    wk, bk = P.norm_rotate(x[:, Hq:Hq + Hkv], kn, EPS, cs, pos, False)
                    P.check(m.q[l][c][lo:hi], wq, bq, "q")
                    P.check(k[:, L[b]:].transpose(0, 1), wk, bk, "k")
                    assert torch.equal(v[:, L[b]:].transpose(0, 1), x[:, Hq + Hkv:].double())
                    q = m.q[l][c][lo:hi].cpu()
                    out, lse, b_out, b_lse = P.attention(q, k, v, L[b])
                    P.check(m.out[l][c][lo:hi], out, b_out, "out")
                    P.check(m.lse[l][c][lo:hi], lse, b_lse, "lse")
                S, last = L[b] + n, min(n, m.window)
                want, full = torch.zeros(Hkv, m.w.shape[-1], dtype=torch.float64), torch.zeros(Hkv, m.w.shape[-1], dtype=torch.float64)
                if c:
                    want = old[l, b].double()
                    want[:, :S] *= 0.5
                if last:
                    w, error = P.key_weights(q[n - last:], m.lse[l][c][hi - last:hi].cpu(), k, S - last)
                    want[:, :S] += w
                    full[:, :S] = error + 3 * P.F32 * want[:, :S]
                P.check(m.w[l, b], want, full, "weights")

    def evicted():
        L, w = m.lens.cpu().tolist(), m.w.cpu()
        was = [[rows(m, l, b, L[b]) for b in range(B)] for l in range(NL)]
        m.evict()
        assert int(m.status) == 0 and m.lens.cpu().tolist() == [min(n, m.keep) for n in L]
        for l in range(NL):
            for b in range(B):
                now = rows(m, l, b, min(L[b], m.keep))
                for h in range(Hkv):
                    src = P.evict(w[l, b, h, :L[b]], m.keep, m.recent) if L[b] > m.keep else list(range(L[b]))
                    assert torch.equal(now[0][h], was[l][b][0][h, src]) and torch.equal(now[1][h], was[l][b][1][h, src])
                    assert torch.equal(m.w[l, b, h, :len(src)].cpu(), w[l, b, h, src]) and not bool(m.w[l, b, h, len(src):].any())

    evicted()
    text = m.text.cpu().tolist()
    assert text == m.total
    L, old = m.lens.cpu().tolist(), m.w.cpu()
    before = [[rows(m, l, b, L[b]) for b in range(B)] for l in range(NL)]
    m.steps()
    assert int(m.status) == 0 and m.accept.cpu().tolist() == list(m.accepted)
    for l in range(NL):
        for b in range(B):
            par, x = m.parents_host[b].tolist(), m.tree_x[l][b].cpu()
            pos = text[b] + torch.tensor(P.depths(par))
            wq, bq = P.norm_rotate(x[:, :Hq], qn, EPS, cs, pos, False)
            P.check(m.tq[l][b], wq, bq, "tree q")
            # the nodes' own keys: exact, from where they were left or from the appended rows, else within their bound
            wk, bk = P.norm_rotate(x[:, Hq:Hq + Hkv], kn, EPS, cs, pos, False)
            path, n = m.paths[b], len(m.paths[b])
            assert m.path[b, :n].cpu().tolist() == path
            k, v = rows(m, l, b, L[b] + n)
            assert torch.equal(k[:, :L[b]], before[l][b][0]) and torch.equal(v[:, :L[b]], before[l][b][1])
            P.check(k[:, L[b]:].transpose(0, 1), wk[path], bk[path], "appended k")
            assert torch.equal(v[:, L[b]:].transpose(0, 1), x[path, Hq + Hkv:].double())
            q, lse = m.tq[l][b].cpu(), m.tlse[l][b].cpu().t()
            # a row of the accepted path saw what is in front of its own appended row
            out, want_lse, b_out, b_lse = P.attention(q[path], k, v, L[b])
            P.check(m.tout[l][b][path], out, b_out, "tree out")
            P.check(lse[path], want_lse, b_lse, "tree lse")
            w, error = P.key_weights(q[path], lse[path], k, L[b])
            want, full = old[l, b].double(), torch.zeros_like(old[l, b]).double()
            want[:, :L[b] + n] += w
            full[:, :L[b] + n] = error + 3 * P.F32 * want[:, :L[b] + n]
            P.check(m.w[l, b], want, full, "weights of the step")
    evicted()


@pytest.mark.parametrize("Hq,Hkv,D,in_cache", [(8, 2, 128, False), (6, 2, 64, True)])
@pytest.mark.parametrize("rows_of_a_workgroup", [-1, 16, 256])
def test_replays_equal_eager(R, Hq, Hkv, D, in_cache, rows_of_a_workgroup):
    """Two programs, each captured, that share one workspace and are replayed in turn, with eager work between."""
    R.reader_tuning_override(R.TUNE_PROMPT_ROWS, rows_of_a_workgroup)
    try:
        a = Model(R, Hq, Hkv, D, in_cache, seed=1)
        b = Model(R, Hq, Hkv, D, in_cache, seed=2, chunks=((100, 3, 1), (1, 1, 60)), keep=20, recent=20, accepted=(1, 2, 3))
        both = max(a.ws.numel(), b.ws.numel())
        a.ws = b.ws = torch.full((both,), 0xff, dtype=torch.uint8, device="cuda")
        want, graphs = [], []
        for m in (a, b):
            m.reset()
            m.run()
            torch.cuda.synchronize()
            assert int(m.status) == 0
            want.append([bits(t).clone() for t in m.left()])
        for m in (a, b):
            m.reset()
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=torch.cuda.Stream()):
                m.run()
            graphs.append(g)
        for replay in range(4):
            for m, g, w in zip((a, b), graphs, want):
                m.reset()
                scratch = torch.randn(1 << 20, device="cuda").sum()
                if replay % 2:
                    torch.cuda.synchronize()
                g.replay()
                if replay == 2:
                    continue                                  # the other program follows at once
                torch.cuda.synchronize()
                assert float(scratch) == float(scratch)
                for i, (t, x) in enumerate(zip(m.left(), w)):
                    assert torch.equal(bits(t), x), "replay %d: tensor %d" % (replay, i)
            torch.cuda.synchronize()
            for m, w in zip((a, b), want):
                assert all(torch.equal(bits(t), x) for t, x in zip(m.left(), w)), "replay %d" % replay
    finally:
        R.reader_tuning_override(R.TUNE_PROMPT_ROWS, -1)


def test_two_streams_at_once(R):
    """Two programs with a workspace each, on two streams other than the tensors' own, at the same time
    (a verification step wants to be ordered with others)."""
    ms = [Model(R, 8, 2, 128, False, seed=3), Model(R, 8, 2, 128, True, seed=4, chunks=((300, 200, 150), (40, 1, 0)), keep=100)]
    want = []
    for m in ms:
        m.reset()
        m.run_to_the_step()
        torch.cuda.synchronize()
        want.append([bits(t).clone() for t in m.left()])
    streams = [torch.cuda.Stream() for _ in ms]
    for _ in range(3):
        for m in ms:
            m.reset()
        torch.cuda.synchronize()
        for m, s in zip(ms, streams):
            with torch.cuda.stream(s):
                m.run_to_the_step()
        torch.cuda.synchronize()
        for m, w in zip(ms, want):
            assert int(m.status) == 0
            for i, (t, x) in enumerate(zip(m.left(), w)):
                assert torch.equal(bits(t), x), "tensor %d" % i


def test_far_pages(R):
    """Pages whose rows start behind 2^31 elements of the cache: written, weighed and moved there, and nothing in front."""
    Hq, Hkv, D, n, keep = 8, 2, 128, 70, 40
    gen = torch.Generator().manual_seed(9)
    page = Hkv * 16 * D
    pages = (1 << 31) // page + 40
    cache = P.Cache(gen, [n], Hkv, D)
    far = pages - cache.num_pages
    table = (cache.table + far).int().cuda()
    # (one layer of the cache is all there is room to look at)
    kc, vc = (torch.zeros((1, pages, Hkv, 16, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x = torch.randn((n, Hq + 2 * Hkv, D), generator=gen).bfloat16().cuda()
    q, out = torch.zeros((n, Hq, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, Hq, D), dtype=torch.bfloat16, device="cuda")
    lse, w = torch.zeros((n, Hq), device="cuda"), torch.full((1, 1, Hkv, 80), math.nan, device="cuda")
    cu, lens, status = i32([0, n]), i32([0]), i32([0])
    dims = R.make_dims(1, 1, Hq, Hkv, D, cache.max_pages, 1, pages)
    ws = torch.empty(max(256, R.reader_prompt_workspace_bytes(dims, n, n), R.reader_kv_evict_workspace_bytes(dims, 1, keep)),
                     dtype=torch.uint8, device="cuda")
    R.reader_prompt_qkv(dims, x, cu, lens, None, None, None, 0.0, None, False, q, kc[0], vc[0], table, status)
    R.reader_prompt_attn(dims, q, kc[0], vc[0], table, cu, lens, out, lse, n, ws, status)
    R.reader_prompt_key_weights(dims, q, lse, cu, n, kc[0], table, lens, 0.0, w[0], n, status)
    lens += n
    k, v = x[:, Hq:Hq + Hkv].cpu().double().transpose(0, 1), x[:, Hq + Hkv:].cpu().double().transpose(0, 1)
    want, bound = P.key_weights(q.cpu(), lse.cpu(), k, 0)
    P.check(w[0, 0, :, :n], want, bound + 3 * P.F32 * want, "weights")
    old = w.cpu()
    R.reader_kv_evict(dims, keep, 7, kc, vc, table, lens, w, ws, status)
    assert int(status) == 0 and int(lens) == keep
    at, slot = cache.place(0, keep)
    at = (at + far).cuda()
    for h in range(Hkv):
        src = P.evict(old[0, 0, h, :n], keep, 7)
        assert torch.equal(kc[0][at, h, slot.cuda()].cpu().double(), k[h, src]) and torch.equal(vc[0][at, h, slot.cuda()].cpu().double(), v[h, src])
    assert not bool(kc[0, :far].any()) and not bool(vc[0, :far].any())
