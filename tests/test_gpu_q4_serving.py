"""The paged cache as a server uses it: requests admitted from a Compressor, growing, ending and making room for others; captured steps, other
streams, places that nobody has taken."""
import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200.pipeline import Compressor, PagedCache
import q4_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"


class _Server:
    """The rows that every place should hold, beside the cache."""

    def __init__(self, batch, layers, heads, g, d, dtype, rope, ret_pages, apx_pages, seed=0):
        self.dt = vec.VECTOR_BF16 if dtype == torch.bfloat16 else vec.VECTOR_F32
        self.shape = vec.Shape(batch, layers, heads * g, heads, d, self.dt, 16, 7, 0.0, int(rope), 10000.0)
        self.one = vec.Shape(1, layers, heads * g, heads, d, self.dt, 16, 7, 0.0, int(rope), 10000.0)
        self.dtype, self.rope, self.LH = dtype, rope, layers * heads
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.W = self.rand(self.LH, d, d) / d ** 0.5
        self.paged = PagedCache(self.shape, ret_pages, apx_pages, 2000, 2000)
        self.rows = {}

    def rand(self, *s):
        return torch.randn(*s, generator=self.gen, device=DEV).to(self.dtype)

    def admit(self, place, N, percent):
        sh, d = self.one, self.one.head_dim
        budget = vec.vector_plan_budget(N, N * percent // 100, -1, 16)
        comp = Compressor(sh, budget)
        K, V = self.rand(self.LH, N, d), self.rand(self.LH, N, d)
        comp.score(self.rand(self.LH, sh.group, 16, d), K)
        comp.route(K, V, self.W)
        self.paged.admit(place, comp, K, V)
        torch.cuda.synchronize()
        k, v, r, a = (t.double().cpu().numpy() for t in (K, V, comp.ret_idx, comp.apx_idx))
        r, a = r.astype(int), a.astype(int)
        self.rows[place] = [[plain.rounded(k[u, r[u]]), plain.rounded(v[u, r[u]]), plain.rounded(k[u, a[u]]), a[u]] for u in range(self.LH)]

    def append_rows(self, k, v):
        for place, units in self.rows.items():
            for u, rows in enumerate(units):
                for i, x in ((0, k), (1, v)):
                    rows[i] = np.concatenate([rows[i], plain.rounded(x[place * self.LH + u][None].double().cpu().numpy())])

    def check(self, q, out):
        for place in range(self.shape.batch):
            for u in range(self.LH):
                got = out[place * self.LH + u].double().cpu().numpy()
                if place not in self.rows:
                    assert not got.any()
                    continue
                rk, rv, ak, pos = self.rows[place][u]
                o, *sizes = plain.attend(q[place * self.LH + u].double().cpu().numpy(), rk, rv, ak, self.W[u].double().cpu().numpy(), self.shape.head_dim ** -0.5,
                                         pos if self.rope else None)
                assert np.all(np.abs(got - o) <= plain.tolerance(o, *sizes, self.dtype, out.dtype, self.rope)), (place, u)


@pytest.mark.parametrize("dtype,d,g,rope", [(torch.bfloat16, 128, 4, False), (torch.float32, 64, 2, False), (torch.bfloat16, 64, 3, True)])
def test_requests_come_grow_and_go(dtype, d, g, rope):
    s = _Server(4, 2, 2, g, d, dtype, rope, 24, 30)
    U, B = s.shape.units, 4
    out = torch.empty(U, g, d, dtype=torch.float32, device=DEV)

    def step(pos):
        k, v, q = s.rand(U, d), s.rand(U, d), s.rand(U, g, d)
        s.paged.append(k, v, torch.full((B,), pos, dtype=torch.int32, device=DEV))
        s.paged.decode(q, s.W, out)
        torch.cuda.synchronize()
        assert vec.vector_device_fault() == 0
        s.append_rows(k, v)
        s.check(q, out)

    s.paged.decode(s.rand(U, g, d), s.W, out)                    # nobody there
    torch.cuda.synchronize()
    assert not out.any()
    s.admit(2, 700, 30)
    s.admit(0, 333, 40)
    for i in range(3):
        step(700 + i)
    s.admit(3, 1200, 20)
    for i in range(2):
        step(1200 + i)
    s.paged.end(2)
    del s.rows[2]
    step(1300)
    s.admit(1, 900, 25)
    s.admit(2, 450, 30)
    for i in range(2):
        step(1400 + i)
    s.paged.end(0, 1, 2, 3)
    assert s.paged.free_pages() == (24, 30)


def test_a_captured_step_follows_the_requests():
    """One graph of append and attention, replayed while requests cross pages' ends, come and go; the launches are the same."""
    s = _Server(3, 1, 2, 4, 128, torch.bfloat16, False, 20, 20, 1)
    U, B = s.shape.units, 3
    k, v, q, pos = s.rand(U, 128), s.rand(U, 128), s.rand(U, 4, 128), torch.zeros(B, dtype=torch.int32, device=DEV)
    out = torch.empty(U, 4, 128, dtype=torch.float32, device=DEV)
    s.admit(0, 500, 50)
    s.paged.decode(q, s.W, out)                                  # first calls set kernels up
    keep = s.paged.cache.ret_len.clone()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        s.paged.append(k, v, pos)
        s.paged.decode(q, s.W, out)
    torch.cuda.synchronize()
    assert torch.equal(s.paged.cache.ret_len, keep)              # capturing runs nothing
    for i in range(70):
        if i == 20:
            s.admit(2, 260, 60)
        if i == 50:
            s.paged.end(0)
            del s.rows[0]
        for t in (k, v, q):
            t.copy_(s.rand(*t.shape))
        graph.replay()
        torch.cuda.synchronize()
        s.append_rows(k, v)
        if i % 9 == 0 or i in (20, 50, 69):
            s.check(q, out)


def test_pages_run_out():
    """A request that finds no page keeps its length, and its answers; the others grow on."""
    s = _Server(2, 1, 1, 2, 64, torch.bfloat16, False, 3, 8, 2)
    s.admit(0, 180, 50)                                          # 45 retained rows
    s.admit(1, 250, 50)                                          # 63: the last row of a page is free, and one page is left
    n0 = [int(x) for x in s.paged.cache.ret_len]
    out = torch.empty(2, 2, 64, dtype=torch.float32, device=DEV)
    for i in range(90):
        k, v, q = s.rand(2, 64), s.rand(2, 64), s.rand(2, 2, 64)
        before = s.paged.cache.ret_len.tolist()
        s.paged.append(k, v, torch.zeros(2, dtype=torch.int32, device=DEV))
        s.paged.decode(q, s.W, out)
        torch.cuda.synchronize()
        after = s.paged.cache.ret_len.tolist()
        for p in (0, 1):
            if after[p] > before[p]:
                for j, x in ((0, k), (1, v)):
                    s.rows[p][0][j] = np.concatenate([s.rows[p][0][j], plain.rounded(x[p][None].double().cpu().numpy())])
        if i % 10 == 0:
            s.check(q, out)
    assert s.paged.free_pages()[0] == 0 and sorted(s.paged.cache.ret_len.tolist()) == [64, 128] and n0 == [45, 63]


def test_other_streams_and_shared_workspace():
    """Calls on a stream of their own, and two captured graphs that share a workspace, one after the other."""
    a = plain.problem(2, 1, 2, 4, 128, torch.bfloat16, [(300, 700), (90, 0)], 21)
    b = plain.problem(2, 1, 2, 4, 128, torch.bfloat16, [(10, 20), (900, 1100)], 22)
    want = [plain.decode(*p, torch.bfloat16) for p in (a, b)]
    ws = torch.empty(max(vec.vector_decode_q4_workspace_bytes(p[0]) for p in (a, b)), dtype=torch.uint8, device=DEV)
    outs = [torch.empty_like(w) for w in want]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        vec.vector_decode_attn_q4(a[0], a[1], a[2], a[3], outs[0], ws)
    vec.vector_decode_attn_q4(b[0], b[1], b[2], b[3], outs[1], torch.empty_like(ws), stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, want))
    graphs = []
    for p, o in zip((a, b), outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            vec.vector_decode_attn_q4(p[0], p[1], p[2], p[3], o, ws)
    for _ in range(3):
        for o in outs:
            o.zero_()
        for gr in graphs + graphs[::-1]:
            gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want))


def test_both_routes_of_the_binding():
    """The extension module's calls and ctypes' (by an explicit stream) give the same; what does not fit is refused before anything is launched."""
    sh, q, c, W = plain.problem(2, 1, 2, 2, 64, torch.bfloat16, [(100, 80), (70, 10)], 5)
    outs = [torch.empty(4, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ws = torch.empty(vec.vector_decode_q4_workspace_bytes(sh), dtype=torch.uint8, device=DEV)
    st = torch.cuda.current_stream()
    for o, stream in zip(outs, (None, st)):
        vec.vector_decode_attn_q4(sh, q, c, W, o, ws, stream)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
    from paper_2605_23258_b200 import binding
    m = binding._marshal()
    assert m.decode_attn_q4(sh, q, c, W, outs[0], ws, None) == 0 and m.decode_attn_q4(sh, q, c, W, outs[0], ws[:64], None) == -5
    short = vec.Q4Cache(c.ret_pages[:, :, :-8].contiguous(), *[getattr(c, n) for n in ("apx_pages", "ret_table", "apx_table", "ret_len", "apx_len")])
    for args in ((sh, q[:2], c, W, outs[0]), (sh, q, c, W[:1], outs[0]), (sh, q, short, W, outs[0]), (sh, q, c, W, outs[0][:3]), (sh, q.float(), c, W, outs[0])):
        assert m.decode_attn_q4(*args, ws, None) is None
        with pytest.raises(ValueError):
            vec.vector_decode_attn_q4(*args, ws)
    with pytest.raises(vec.VectorError) as e:
        vec.vector_decode_attn_q4(sh, q, c, W, outs[0], None)
    assert e.value.status == -5
    ints = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    with pytest.raises(ValueError):
        vec.vector_block_tables(ints(2), ints(2), 64, c.ret_table, ints(4), ints(1), ints(1), ints(1), ints(2), ints(3))
    slots = torch.tensor([[3, 9], [64, 70]], dtype=torch.int32, device=DEV)
    rows = [[torch.empty(4, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(3)] for _ in range(2)]
    for r, stream in zip(rows, (None, st)):
        vec.vector_read_q4(sh, c, slots, r[0], r[1], slots, r[2], stream)
    torch.cuda.synchronize()
    assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip(*rows))
