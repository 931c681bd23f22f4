"""The attention entry points as a server uses them together: prompts, forked sequences, pages that are copied before they are
written, decoding, compaction, between the delta linears of a block; on streams of their own, in captured graphs, with padded
batches.  The reference keeps every sequence's keys and values in plain lists (oracle/attn_oracle.py has the tolerances)."""
import random

import pytest
import torch

import paper_2406_09041_amd as mes
from inputs import synth
from oracle import attn_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _check(got, want, tol, what=""):
    got = got.double().cpu()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {((got - want).abs() / tol.clamp_min(1e-30)).max():.3g} times the tolerance"


class Server:
    """One layer's cache, its page pool, and the same tokens in plain lists."""

    def __init__(self, heads, kvh, dim, page, n_pages, max_seqs, width, e4m3=False, seed=0):
        self.g = torch.Generator().manual_seed(seed)
        self.heads, self.kvh, self.dim, self.page, self.width = heads, kvh, dim, page, width
        scales = [0.01 + 0.02 * torch.rand(1, kvh, generator=self.g) for _ in range(2)] if e4m3 else [None, None]
        self.scales = scales
        self.cache = mes.KvCache(1, n_pages, page, kvh, dim, mes.KV_E4M3 if e4m3 else mes.KV_BF16, *[None if s is None else s.to(DEV) for s in scales])
        self.pool = mes.PagePool(n_pages, page, max_seqs, width)
        self.rotary = mes.rotary_table(width * page, dim)
        self.k, self.v = [[[] for _ in range(max_seqs)] for _ in range(2)]
        self.decode = mes.AttnDecode(self.cache, heads, max_seqs)

    def rows(self, n, heads, std=1.0):
        return (torch.randn(n, heads, self.dim, generator=self.g) * std).to(torch.bfloat16)

    def keep(self, which, x, scale):
        if scale is None:
            return x.to(torch.bfloat16).double()
        return (x / scale[0][:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).double() * scale[0][:, None].double()

    def batch(self, seqs, offsets=None):
        table, length = self.pool.table(seqs, self.width)
        return mes.SeqBatch(length.to(DEV), table.to(DEV), offsets)

    def append(self, seqs, news, qkv=None):
        """Grows the sequences, copies what their writes must not touch, appends; returns the turned queries and the batch."""
        src, dst = self.pool.grow(seqs, news)
        mes.mes_kv_copy_pages(self.cache, src, dst)
        T = sum(news)
        q, k, v = qkv or (self.rows(T, self.heads, 2.0).to(DEV), self.rows(T, self.kvh).to(DEV), self.rows(T, self.kvh).to(DEV))
        off = [0]
        for n in news:
            off.append(off[-1] + n)
        batch = self.batch(seqs, None if set(news) == {1} else _ints(off))
        q_out = mes.mes_kv_append(self.cache, 0, batch, q, k, v, self.rotary)
        pos = torch.tensor([len(self.k[s]) + i for s, n in zip(seqs, news) for i in range(n)])
        kr = O.rotate(k.cpu(), self.rotary.cpu(), pos)
        kk, vv = self.keep("k", kr, self.scales[0]), self.keep("v", v.cpu().float(), self.scales[1])
        for s, a, b in zip(seqs, off, off[1:]):
            self.k[s] += list(kk[a:b])
            self.v[s] += list(vv[a:b])
        want_q = O.rotate(q.cpu(), self.rotary.cpu(), pos).to(torch.bfloat16)
        assert torch.equal(q_out.cpu().view(torch.int16), want_q.view(torch.int16))
        return q_out, batch, off

    def check(self, out, q, seqs, off, what):
        for s, a, b in zip(seqs, off, off[1:]):
            n = len(self.k[s])
            if b > a:
                want, tol = O.attend(q[a:b], torch.stack(self.k[s]), torch.stack(self.v[s]), range(n - (b - a), n), self.dim ** -0.5)
                _check(out[a:b], want, tol, f"{what}, sequence {s}")

    def fork(self, parent, child, n):
        self.pool.fork(parent, child, n)
        self.k[child], self.v[child] = self.k[parent][:n], self.v[parent][:n]

    def free(self, s):
        self.pool.free(s)
        self.k[s], self.v[s] = [], []

    def compact(self):
        src, dst = self.pool.compact()
        mes.mes_kv_copy_pages(self.cache, src, dst)
        return len(src)


@pytest.mark.parametrize("heads,kvh,dim,page,e4m3", [(4, 2, 64, 16, False), (8, 2, 128, 16, False), (4, 4, 64, 32, True), (6, 2, 128, 64, True)])
def test_system_prompts_forks_decoding_and_compaction(heads, kvh, dim, page, e4m3):
    s = Server(heads, kvh, dim, page, n_pages=120, max_seqs=16, width=24, e4m3=e4m3, seed=page)
    # two experts' system prompts, in sequences 14 and 15; both prompts in one call over fresh keys and values
    news = [83, 130]
    q, k, v = s.rows(213, heads, 2.0).to(DEV), s.rows(213, kvh).to(DEV), s.rows(213, kvh).to(DEV)
    q_out, batch, off = s.append([14, 15], news, (q, k, v))
    s.check(mes.mes_attn_extend(s.cache, 0, batch, q_out), q_out, [14, 15], off, "system prompts")
    # users: forks of a system prompt with a question of their own; expert 0 has 3, expert 1 has 2 and one that shares less
    users = [0, 1, 2, 3, 4, 5]
    for u, parent, n in ((0, 14, 83), (1, 14, 83), (2, 14, 83), (3, 15, 130), (4, 15, 130), (5, 15, 70)):
        s.fork(parent, u, n)
    q_out, batch, off = s.append(users, [5, 40, 1, 17, 90, 2])
    s.check(mes.mes_attn_extend(s.cache, 0, batch, q_out), q_out, users, off, "questions")
    rng = random.Random(1)
    for step in range(6):
        if step == 3:
            s.free(1)                                            # an answer ends; its row stays in the batch as padding
            users = [0, 1, 2, 3, 4, 5]
            assert s.compact() > 0
        live = [u for u in users if s.k[u]]
        q_out, _, off = s.append(live, [1] * len(live))
        q_all = torch.zeros(len(users), heads, dim, dtype=torch.bfloat16, device=DEV)
        q_all[[users.index(u) for u in live]] = q_out
        q_all[[i for i, u in enumerate(users) if u not in live]] = float("nan")
        out = s.decode(0, s.batch(users), q_all, [0, 3, 6], [83, 130 if rng.random() < 0.5 else 70])
        for i, u in enumerate(users):
            if u in live:
                s.check(out[i:i + 1], q_all[i:i + 1], [u], [0, 1], f"step {step}")
            else:
                assert not out[i].any()
    for u in users + [14, 15]:
        s.free(u)
    assert s.pool.unused() == 120


def test_a_block_of_delta_linears_around_the_attention():
    """q/k/v -> rotary, cache, attention -> o, for two prompts of two experts and then two decoded tokens: every link checked on what the
    link before gave."""
    d, heads, kvh, dim = 256, 4, 2, 64
    layers = []
    for d_out, seed in ((heads * dim, 1), (kvh * dim, 2), (kvh * dim, 3), (d, 4)):
        wl = synth.small_case(d if d_out != d or seed != 4 else heads * dim, d_out, [0, 40, 71], 8, 2, seed=seed)
        layers.append((mes.mes_pack_base(wl.w_base.to(DEV)), [mes.mes_pack_delta(e.delta.to(DEV), e.salient_idx, 2) for e in wl.experts]))
    qkv, o = mes.DeltaLinearMulti(layers[:3], 71), mes.DeltaLinear(*layers[3], max_tokens=71)
    s = Server(heads, kvh, dim, 16, n_pages=20, max_seqs=2, width=8, seed=7)
    for news in ([40, 31], [1, 1], [1, 1]):
        T = sum(news)
        x = (torch.randn(T, d, generator=s.g)).to(torch.bfloat16).to(DEV)
        seg = [0, news[0], T]
        q, k, v = qkv(x, seg)
        q_out, batch, off = s.append([0, 1], news, (q.view(T, heads, dim), k.view(T, kvh, dim), v.view(T, kvh, dim)))
        if T > 2:
            out = mes.mes_attn_extend(s.cache, 0, batch, q_out)
            kk = torch.stack([x_ for seq in (0, 1) for x_ in s.k[seq]]).to(torch.bfloat16).to(DEV)
            fresh = mes.mes_attn_prompt(q_out, kk, v.view(T, kvh, dim), _ints(off))
            s.check(fresh, q_out, [0, 1], off, "fresh keys")
        else:
            out = s.decode(0, batch, q_out, seg, [0, 0])
        s.check(out, q_out, [0, 1], off, f"{T} rows")
        y = o(out.view(T, heads * dim), seg)
        assert torch.isfinite(y).all() and y.shape == (T, d)


def test_streams_and_captured_graphs():
    """A decode step captured once and replayed while sequences grow, eager work in between; two graphs share a workspace; everything on
    a stream that is not the default one."""
    heads, kvh, dim, n = 8, 2, 64, 5
    s = Server(heads, kvh, dim, 16, n_pages=140, max_seqs=6, width=24, seed=3)
    s.append([5], [130])
    for u in range(n):
        s.fork(5, u, 130)
    side = torch.cuda.Stream()
    seg, prefix = [0, n], [130]
    q, k, v = (torch.zeros(n, h, dim, dtype=torch.bfloat16, device=DEV) for h in (heads, kvh, kvh))
    q_turned, out_a, out_b = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    table, length = (t.to(DEV) for t in s.pool.table(range(n), s.width))
    batch = mes.SeqBatch(length, table)

    def step():
        mes.mes_kv_append(s.cache, 0, batch, q, k, v, s.rotary, q_turned)
        s.decode(0, batch, q_turned, seg, prefix, out_a)
    graphs = []
    with torch.cuda.stream(side):
        # a first write to a forked page copies it: the captured steps then only write to pages of their own
        src, dst = s.pool.grow(range(n), [1] * n)
        mes.mes_kv_copy_pages(s.cache, src, dst)
        t, l = s.pool.table(range(n), s.width)
        table.copy_(t)
        length.copy_(l)
        step()
        for fn in (step, lambda: s.decode(0, batch, q_turned, None, None, out_b)):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                fn()
            graphs.append(g)
    torch.cuda.synchronize()
    eager = mes.AttnDecode(s.cache, heads, n)
    for it in range(5):
        if it:
            assert s.pool.grow(range(n), [1] * n) == ([], [])
        fresh = [s.rows(n, h, 2.0 if h == heads else 1.0) for h in (heads, kvh, kvh)]
        t, l = s.pool.table(range(n), s.width)
        with torch.cuda.stream(side):
            for dst_, src_ in zip((q, k, v, table, length), (*fresh, t, l)):
                dst_.copy_(src_)
            graphs[0].replay()
            graphs[1].replay()                                   # the same sums, nothing shared
        torch.cuda.synchronize()
        pos = torch.full((n,), 130 + it)
        for u in range(n):
            s.k[u].append(O.rotate(fresh[1], s.rotary.cpu(), pos)[u].to(torch.bfloat16).double())
            s.v[u].append(fresh[2][u].double())
        s.check(out_a, q_turned, range(n), range(n + 1), f"replay {it}")
        s.check(out_b, q_turned, range(n), range(n + 1), f"replay {it}, nothing shared")
        again = eager(0, batch, q_turned, seg, prefix)
        assert torch.equal(again.view(torch.int16), out_a.view(torch.int16))
        torch.randn(1000, 1000, device=DEV).sum().item()         # eager work of the program between the replays


def test_prompts_in_a_graph_that_shares_its_workspace():
    heads, kvh, dim, T = 2, 1, 128, 1900                         # long enough to be cut
    g = torch.Generator().manual_seed(8)
    q, k, v = ((torch.randn(T, h, dim, generator=g)).to(torch.bfloat16).to(DEV) for h in (heads, kvh, kvh))
    off = _ints([0, T])
    ws = mes.binding.prompt_workspace(T, 1, heads, kvh, dim, DEV)
    outs = [torch.zeros_like(q) for _ in range(2)]
    mes.mes_attn_prompt(q, k, v, off, outs[0], workspace=ws)
    torch.cuda.synchronize()
    graphs = []
    for o in outs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            mes.mes_attn_prompt(q, k, v, off, o, workspace=ws)
        graphs.append(gr)
    for it in range(3):
        q.copy_(torch.randn(T, heads, dim, generator=g).to(torch.bfloat16))
        off.copy_(_ints([0, T - 300 * it]))                      # lengths are read when the graph runs
        for gr in graphs:
            gr.replay()
        want = mes.mes_attn_prompt(q, k, v, off)
        torch.cuda.synchronize()
        n = T - 300 * it
        assert torch.equal(outs[0][:n].view(torch.int16), want[:n].view(torch.int16)) and torch.equal(outs[1][:n].view(torch.int16), want[:n].view(torch.int16))
        rows = [0, 1, 700, n - 1]
        ref, tol = O.attend(q[rows], k[:n], v[:n], rows, dim ** -0.5)
        _check(outs[0][rows], ref, tol, f"replay {it}")


def test_the_binding_refuses_what_the_library_cannot_see():
    s = Server(4, 2, 64, 16, n_pages=8, max_seqs=2, width=4)
    s.append([0, 1], [3, 2])
    batch = s.batch([0, 1])
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device=DEV)
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device=DEV)
    off = _ints([0, 2])
    for bad in (q.cpu(), q.float(), q.transpose(1, 2), q[:, :, ::2], torch.zeros(2, 8, 64, dtype=torch.bfloat16, device=DEV)[:, ::2]):
        with pytest.raises((AssertionError, mes.MesError)):
            s.decode(0, batch, bad)
        with pytest.raises((AssertionError, mes.MesError)):
            mes.mes_attn_prompt(bad, k, k, off)
    for call in (lambda: mes.mes_attn_prompt(q, k, k[:1], off), lambda: mes.mes_attn_prompt(q, k, k, off.long()), lambda: mes.mes_attn_prompt(q, k, k, off.cpu()),
                 lambda: s.decode(0, batch, q[:1]), lambda: s.decode(0, batch, q, [0, 2], [1, 1]), lambda: mes.mes_kv_append(s.cache, 0, batch, q, k[:, :1], k[:, :1], s.rotary),
                 lambda: mes.mes_kv_append(s.cache, 0, batch, q, k, k, s.rotary[:16]), lambda: mes.mes_attn_extend(s.cache, 1, s.batch([0, 1], off.new_tensor([0, 1, 2])), q),
                 lambda: mes.mes_kv_copy_pages(s.cache, [0], [1, 2]), lambda: mes.SeqBatch(off, off), lambda: mes.KvCache.over(q, q)):
        with pytest.raises((AssertionError, mes.MesError)):
            call()
    with torch.cuda.stream(torch.cuda.Stream()):                 # empty calls
        assert mes.mes_attn_prompt(q[:0], k[:0], k[:0], off[:1]).shape == (0, 4, 64)
        mes.mes_kv_copy_pages(s.cache, [], [])


@pytest.mark.parametrize("n,long,heads,kvh,groups", [(2048, {0: 700}, 8, 8, False), (2048, {}, 4, 2, False), (1500, {7: 1, 900: 600}, 8, 8, True), (900, {}, 4, 1, True)])
def test_decode_of_a_batch_that_is_mostly_padding(n, long, heads, kvh, groups):
    """Few or no tokens among many sequences: every row is written, from a workspace full of bytes that are no numbers of pieces."""
    dim, page, n_pages = 64, 16, 60
    g = torch.Generator().manual_seed(n)
    cache = mes.KvCache(1, n_pages, page, kvh, dim)
    for t in (cache.k, cache.v):
        t.copy_(torch.randn(t.shape, generator=g).to(torch.bfloat16))
    length = torch.zeros(n, dtype=torch.int32)
    for s, tokens in long.items():
        length[s] = tokens
    table = torch.randint(0, n_pages, (n, 44), generator=g, dtype=torch.int32)
    q = torch.randn(n, heads, dim, generator=g).to(torch.bfloat16).to(DEV)
    decode = mes.AttnDecode(cache, heads, n)
    decode.ws.fill_(0x5a)
    out = torch.full_like(q, 3.0)
    decode(0, mes.SeqBatch(length.to(DEV), table.to(DEV)), q, [0, n // 2, n] if groups else None, [20, 30] if groups else None, out)
    rows = [s for s in range(n) if s not in long]
    assert not out[rows].any()
    for s, tokens in long.items():
        k, v = ([t[0, table[s, j // page].item(), :, j % page] for j in range(tokens)] for t in (cache.k.cpu(), cache.v.cpu()))
        want, tol = O.attend(q[s:s + 1], torch.stack(k), torch.stack(v), [tokens - 1], dim ** -0.5)
        _check(out[s:s + 1], want, tol, f"sequence {s}")


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_cache_whose_offsets_pass_32_bits(e4m3):
    """Two layers of 2.7e9 values each: pages at both ends, written, copied and read."""
    heads, kvh, dim, page, n_pages = 16, 8, 128, 256, 10400
    one = torch.ones(2, kvh, device=DEV) * 0.02 if e4m3 else None
    cache = mes.KvCache(2, n_pages, page, kvh, dim, mes.KV_E4M3 if e4m3 else mes.KV_BF16, one, one)
    assert cache.k[0].numel() > 2 ** 31
    g = torch.Generator().manual_seed(9)
    lens, T = [300, 513], 813
    table = _ints([[n_pages - 1, 3, 0], [n_pages - 2, 8300, n_pages - 3]])
    q, k, v = (torch.randn(T, h, dim, generator=g).to(torch.bfloat16).to(DEV) for h in (heads, kvh, kvh))
    batch = mes.SeqBatch(_ints(lens), table, _ints([0, 300, 813]))
    mes.mes_kv_append(cache, 1, batch, None, k, v, None)
    assert not cache.k[0, -1].view(torch.uint8).any() and not cache.k[0, :4].view(torch.uint8).any()      # the other layer
    stored = [x.cpu().double() for x in (k, v)]
    if e4m3:
        scale = one[0, 0].cpu()
        stored = [(x.cpu().float() / scale).clamp(-448, 448).to(torch.float8_e4m3fn).double() * scale.double() for x in (k, v)]
    for move in (False, True):
        if move:
            mes.mes_kv_copy_pages(cache, [n_pages - 1, 8300], [8200, n_pages - 4])
            table.copy_(_ints([[8200, 3, 0], [n_pages - 2, n_pages - 4, n_pages - 3]]))
            for pg in (n_pages - 1, 8300):
                cache.k[1, pg].view(torch.uint8).zero_()
        out = mes.mes_attn_extend(cache, 1, batch, q)
        last = q[[299, 812]].contiguous()
        one_each = mes.AttnDecode(cache, heads, 2)(1, batch, last)
        for s, (a, b) in enumerate(((0, 300), (300, 813))):
            rows = [0, 1, (b - a) // 2, b - a - 1]
            want, tol = O.attend(q[[a + r for r in rows]], stored[0][a:b], stored[1][a:b], rows, dim ** -0.5)
            _check(out[[a + r for r in rows]], want, tol, f"sequence {s}, move {move}")
            _check(one_each[s:s + 1], want[-1:], tol[-1:], f"decoded, sequence {s}, move {move}")


@pytest.mark.parametrize("n_seqs", [2, 70])
def test_extend_with_the_largest_lengths(n_seqs):
    """A length far past the table's room: every row sees all tokens of the table; the lowest one: none."""
    heads, kvh, dim, page = 4, 2, 64, 16
    g = torch.Generator().manual_seed(n_seqs)
    cache = mes.KvCache(1, 50, page, kvh, dim)
    for t in (cache.k, cache.v):
        t.copy_(torch.randn(t.shape, generator=g).to(torch.bfloat16))
    table = torch.randint(0, 50, (n_seqs, 20), generator=g, dtype=torch.int32)
    length = torch.full((n_seqs,), 2 ** 31 - 1, dtype=torch.int32)
    length[-1] = -2 ** 31
    q = torch.randn(3 * n_seqs, heads, dim, generator=g).to(torch.bfloat16).to(DEV)
    off = _ints([3 * s for s in range(n_seqs + 1)])
    batch = mes.SeqBatch(length.to(DEV), table.to(DEV), off)
    before = cache.k.clone()
    mes.mes_kv_append(cache, 0, batch, None, q[:, :kvh], q[:, kvh:], None)        # no row has a place
    assert torch.equal(cache.k.view(torch.int16), before.view(torch.int16))
    for ws in (None, mes.binding.prompt_workspace(3 * n_seqs, n_seqs, heads, kvh, dim, DEV)):
        out = mes.mes_attn_extend(cache, 0, batch, q, workspace=ws)
        assert not out[-3:].any()
        for s in (0, n_seqs - 2):
            k, v = (torch.cat([x[0, p].transpose(0, 1) for p in table[s].tolist()]) for x in (cache.k.cpu(), cache.v.cpu()))
            want, tol = O.attend(q[3 * s:3 * s + 3], k, v, [319] * 3, dim ** -0.5)
            _check(out[3 * s:3 * s + 3], want, tol, f"sequence {s}")
