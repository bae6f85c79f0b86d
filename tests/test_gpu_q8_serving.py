"""The 8-bit paged cache as a server uses it, from a layer's projections on: contexts normed, turned, compressed and admitted, tokens projected, appended (one or several, turned before
or on the way) and attended to; captured steps, other streams, requests that come and go, too few pages, and what is refused before anything changes."""
import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200.pipeline import Compressor, PagedCache
import q8_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


class _Server:
    """The cache, beside it the rows that every place should hold."""

    def __init__(self, batch, heads, g, d, dtype, rope, ret_pages, apx_pages, seed=0, ret_rows=2000):
        kind = vec.VECTOR_BF16 if dtype == BF else vec.VECTOR_F32
        self.shape, self.one = (vec.Shape(b, 1, heads * g, heads, d, kind, 16, 7, 0.0, int(rope), 10000.0) for b in (batch, 1))
        self.dtype, self.rope, self.LH = dtype, rope, heads
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.W = self.rand(heads, d, d) / d ** 0.5
        self.weights = self.rand(1, d).abs() + 0.5, self.rand(1, d).abs() + 0.5
        self.paged = PagedCache(self.shape, ret_pages, apx_pages, ret_rows, 2000, bits=8)
        self.rows = {}
        self.q = None

    def rand(self, *s):
        return torch.randn(*s, generator=self.gen, device=DEV).to(self.dtype)

    def projections(self, batch, n):
        """Parts of a fused projection, queries, keys and values."""
        sh = self.shape
        return self.rand(batch, n, (sh.n_q_heads + 2 * sh.n_kv_heads) * sh.head_dim).split([sh.n_q_heads * sh.head_dim] + [sh.n_kv_heads * sh.head_dim] * 2, dim=-1)

    def admit(self, place, N, percent):
        budget = vec.vector_plan_budget(N, N * percent // 100, -1, 16)
        comp = Compressor(self.one, budget)
        Q, K, V = comp.project(*self.projections(1, N), *self.weights)
        assert Q.shape == (self.LH, self.one.group, 16, self.one.head_dim)
        comp.score(Q, K)
        comp.route(K, V, self.W)
        there = self.paged.admit(place, comp, K, V)
        k, v, r, a = (t.double().cpu().numpy() for t in (K, V, comp.ret_idx, comp.apx_idx))
        r, a = r.astype(int), a.astype(int)
        if bool(there):
            self.rows[place] = [(plain.Held().append(k[u, r[u]]), plain.Held().append(v[u, r[u]]), plain.rounded(k[u, a[u]]), r[u].tolist()) for u in range(self.LH)]
        return bool(there)

    def keep(self, k, v, pos, n=1):
        """n rows [batch][n][LH][d] of every place that is taken."""
        for place, units in self.rows.items():
            for u, (hk, hv, _, p) in enumerate(units):
                hk.append(k[place, :n, u].double().cpu().numpy())
                hv.append(v[place, :n, u].double().cpu().numpy())
                p += pos[place, :n].tolist()

    def step(self, pos):
        B, d = self.shape.batch, self.shape.head_dim
        at = torch.full((B, 1), pos, dtype=torch.int32, device=DEV)
        self.q, k, v = self.paged.project(*self.projections(B, 1), *self.weights, at)
        self.paged.append(k, v, at)
        self.keep(k.view(B, 1, self.LH, d), v.view(B, 1, self.LH, d), at.cpu().numpy())

    def check(self, out):
        c, d = self.paged.cache, self.shape.head_dim
        assert vec.vector_device_fault() == 0
        most = int(c.ret_len.max()) + 1
        new = lambda n: torch.empty(self.shape.units, n, d, dtype=self.dtype, device=DEV)  # noqa: E731
        k, v, a = new(most), new(most), new(int(c.apx_len.max()) + 1)
        vec.vector_read_q8(self.shape, c, k, v, a)
        k, v, a, table, rpos = (t.cpu().numpy() if t.dtype == torch.int32 else t.double().cpu().numpy() for t in (k, v, a, c.ret_table, c.ret_pos))
        for b in range(self.shape.batch):
            for u in range(self.LH):
                at = b * self.LH + u
                if b not in self.rows:
                    assert not k[at].any() and not a[at].any() and not out[at].any()
                    continue
                hk, hv, ak, p = self.rows[b][u]
                n = len(hk.rows)
                assert int(c.ret_len[b]) == n and np.array_equal(k[at, :n], hk.values(d)) and np.array_equal(v[at, :n], hv.values(d)) and np.array_equal(a[at, :len(ak)], ak)
                r = np.arange(n)
                assert rpos[table[b][r // 32], u, r % 32].tolist() == p
                plain.check_decode(self.shape, self.q, c, self.W, out, self.rope, [at])


@pytest.mark.parametrize("dtype,d,g,rope", [(BF, 128, 4, True), (F32, 64, 2, False), (BF, 64, 3, True), (F32, 128, 1, True)])
def test_requests_come_grow_and_go(dtype, d, g, rope):
    s = _Server(4, 2, g, d, dtype, rope, 60, 80)
    out = torch.empty(s.shape.units, g, d, dtype=F32, device=DEV)

    def steps(pos, n=1):
        for i in range(n):
            s.step(pos + i)
            s.paged.decode(s.q, s.W, out)
            s.check(out)

    assert s.admit(2, 700, 30) and s.admit(0, 333, 40)
    steps(700, 3)
    assert s.admit(3, 1200, 20)
    steps(1200, 2)
    s.paged.end(2)
    del s.rows[2]
    steps(1300)
    assert s.admit(1, 900, 25) and s.admit(2, 450, 30)
    steps(1400, 40)                                                # blocks' ends are crossed
    s.paged.end(0, 1, 2, 3)
    assert s.paged.free_pages() == (60, 80)


def test_several_tokens_at_once():
    """Drafted tokens and a prompt's piece, turned before; then keys turned on the way, which give the same values as turned in advance but for what the rows between are rounded to."""
    s = _Server(3, 2, 4, 128, BF, True, 60, 30)
    s.admit(0, 400, 40), s.admit(2, 300, 50)
    out = torch.empty(6, 4, 128, dtype=BF, device=DEV)
    for n in (5, 1, 70):
        pos = torch.randint(0, 5000, (3, n), dtype=torch.int32, device=DEV)
        q, k, v = s.projections(3, n)
        rows = [torch.empty(6, n, 128, dtype=BF, device=DEV) for _ in range(2)]
        vec.vector_norm_rope(s.shape, n, k=k, v=v, k_out=rows[0], v_out=rows[1], pos=pos)
        k_rows, v_rows = (t.view(3, 2, n, 128).transpose(1, 2).contiguous() for t in rows)
        s.paged.append(k_rows, v_rows, pos)
        s.keep(k_rows, v_rows, pos.cpu().numpy(), n)
        s.q = s.rand(6, 4, 128)
        s.paged.decode(s.q, s.W, out)
        s.check(out)
    n, before = 9, s.paged.cache.ret_len.clone()
    pos = torch.randint(0, 5000, (3, n), dtype=torch.int32, device=DEV)
    _, k, v = s.projections(3, n)
    s.paged.append(k, v, pos, rotate=True)
    assert (s.paged.cache.ret_len - before).tolist() == [n, 0, n]
    got = torch.empty(6, int(s.paged.cache.ret_len.max()), 128, dtype=BF, device=DEV)
    vec.vector_read_q8(s.shape, s.paged.cache, got, torch.empty_like(got))
    for b in (0, 2):
        x = plain.turned(k[b].view(n, 2, 128).double().cpu().numpy(), pos[b].cpu().numpy()[:, None])
        for u in range(2):
            r = got[b * 2 + u, int(before[b]):int(before[b]) + n].double().cpu().numpy()
            assert np.all(np.abs(r - x[:, u]) <= 2.0 ** -4 * np.abs(x[:, u]) + 2.0 ** -4)          # a rounding; scales are 2^-4 at the most
    s.paged.decode(s.q, s.W, out)
    plain.check_decode(s.shape, s.q, s.paged.cache, s.W, out, True, [0, 1, 4, 5])


def test_a_captured_step_follows_the_requests():
    """One graph of projection, append and attention, replayed while requests cross pages' ends, come and go, beside eager calls and another graph on the same cache."""
    s = _Server(3, 2, 4, 128, BF, True, 50, 60, 1)
    sh = s.shape
    qkv, at = s.projections(3, 1), torch.zeros(3, 1, dtype=torch.int32, device=DEV)
    out, k, v = torch.empty(6, 4, 128, dtype=F32, device=DEV), torch.empty(6, 1, 128, dtype=BF, device=DEV), torch.empty(6, 1, 128, dtype=BF, device=DEV)
    q = torch.empty(6, 4, 1, 128, dtype=BF, device=DEV)
    s.admit(0, 500, 50)
    s.q = q[:, :, 0]

    def step():
        vec.vector_norm_rope(sh, 1, *qkv, q, k, v, *s.weights, at)
        s.paged.append(k, v, at)
        s.paged.decode(s.q, s.W, out)
    step()
    s.keep(k.view(3, 1, 2, 128), v.view(3, 1, 2, 128), at.cpu().numpy())
    s.check(out)
    kept = s.paged.cache.ret_len.clone()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    assert torch.equal(s.paged.cache.ret_len, kept)               # capturing runs nothing
    for i in range(70):
        if i == 20:
            s.admit(2, 260, 60)
        if i == 50:
            s.paged.end(0)
            del s.rows[0]
        for t in qkv:
            t.copy_(s.rand(*t.shape))
        at.fill_(500 + i)
        if i % 3 == 2:
            step()
        else:
            graph.replay()
        s.keep(k.view(3, 1, 2, 128), v.view(3, 1, 2, 128), at.cpu().numpy())
        if i % 9 == 0 or i == 69:
            s.check(out)


def test_too_few_pages():
    """An admission that does not fit takes nothing; tokens that find too few pages are cut off behind the pages' end; the other request does not notice."""
    s = _Server(2, 1, 2, 64, BF, False, 5, 20, 2)
    assert s.admit(0, 200, 40)                                    # 40 retained rows of 200 tokens: two pages
    left = s.paged.free_pages()
    assert not s.admit(1, 600, 50) and s.paged.free_pages() == left and s.paged.cache.ret_len.tolist()[1] == 0
    s.paged.end(1)
    n0 = int(s.paged.cache.ret_len[0])
    room = 32 * 5 - n0
    x, pos = s.rand(2, room + 50, 1, 64), torch.arange(2 * (room + 50), dtype=torch.int32, device=DEV).view(2, -1)
    s.paged.append(x, x, pos)
    s.keep(x, x, pos.cpu().numpy(), room)
    out = torch.empty(2, 2, 64, dtype=F32, device=DEV)
    s.q = s.rand(2, 2, 64)
    s.paged.decode(s.q, s.W, out)
    s.check(out)
    assert s.paged.free_pages()[0] == 0 and int(s.paged.cache.ret_len[0]) == 160
    s.step(3)                                                     # no page at all: nothing is written
    del s.rows[0][0][0].rows[-1], s.rows[0][0][1].rows[-1], s.rows[0][0][3][-1]
    s.paged.decode(s.q, s.W, out)
    s.check(out)


def test_refused_before_anything_changes():
    s = _Server(2, 2, 2, 128, BF, True, 20, 20, 3)
    s.admit(0, 300, 40)
    p, before = s.paged, s.paged.cache.ret_len.clone()
    x, pos = s.rand(2, 3, 2, 128), torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    for k, v, at in ((x.float(), x, pos), (x, x[:, :2], pos), (x, x, None), (x, x, pos[:, :2]), (x, x, pos.long()), (x.transpose(1, 2), x, pos), (x.flatten()[:-1], x, pos),
                     (torch.empty(x.numel() + 1, dtype=BF, device=DEV)[1:].view_as(x), x, pos)):
        with pytest.raises(ValueError):
            p.append(k, v, at)
    still = _Server(1, 1, 1, 64, BF, False, 4, 4).paged
    with pytest.raises(ValueError, match="turned"):
        still.append(torch.zeros(1, 64, dtype=BF, device=DEV), torch.zeros(1, 64, dtype=BF, device=DEV), pos[:1, :1], rotate=True)
    four = PagedCache(s.shape, 4, 4, 100, 100)
    with pytest.raises(ValueError, match="turned"):
        four.append(x[:, 0], x[:, 0], pos[:, 0], rotate=True)
    with pytest.raises(ValueError, match="bits"):
        PagedCache(s.shape, 4, 4, 100, 100, bits=6)
    assert torch.equal(p.cache.ret_len, before) and p.free_pages()[0] == 20 - -(-int(before[0]) // 32)


def test_two_streams_at_once():
    """Two servers of one process, each on a stream of its own."""
    servers = [_Server(2, 2, 4, 128, BF, True, 60, 60, 4 + i) for i in range(2)]
    for s in servers:
        s.admit(0, 900, 40), s.admit(1, 500, 30)
    streams = [torch.cuda.Stream() for _ in servers]
    outs = [torch.empty(4, 4, 128, dtype=BF, device=DEV) for _ in servers]
    torch.cuda.synchronize()
    ends = [torch.cuda.Event() for _ in servers]
    for i in range(12):
        for s, st, out in zip(servers, streams, outs):
            with torch.cuda.stream(st):
                s.step(1000 + i)
                s.paged.decode(s.q, s.W, out)
    for st, e in zip(streams, ends):
        e.record(st)
    torch.cuda.synchronize()
    for s, out in zip(servers, outs):
        s.check(out)
