"""Writers and reader of the 4-bit paged cache against the plain form, bit for bit, and nothing but the named rows changed."""
import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
import q4_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _shape(batch, layers, heads, d, dtype):
    return vec.Shape(batch, layers, heads, heads, d, vec.VECTOR_BF16 if dtype == torch.bfloat16 else vec.VECTOR_F32, 16)


def _cache(sh, ret_pages, apx_pages, rng):
    c = vec.alloc_q4_cache(sh, ret_pages, apx_pages, 1, 1)
    for t in (c.ret_pages, c.apx_pages):
        t.copy_(torch.from_numpy(rng.integers(0, 256, tuple(t.shape), dtype=np.uint8)))
    for t in (c.ret_pos, c.apx_pos):
        t.fill_(-7)
    return c


def _hard_rows(n, d, rng, dtype):
    """Rows of many sizes; some groups on the borders between codes, of one number, of zeros, beyond the range, with NaN and infinities."""
    x = rng.standard_normal((n, d)) * np.exp(rng.uniform(-10, 8, (n, 1)))
    s = plain.SCALES[rng.integers(1, 227, (n, d // 16))]
    t = rng.choice([0, 0.25, 0.5, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6], (n, d)) * rng.choice([-1, 1], (n, d))
    on_border = rng.random((n, d // 16)) < 0.4
    x = np.where(np.repeat(on_border, 16, 1), t * np.repeat(s, 16, 1), x)
    x = torch.from_numpy(x).to(dtype)
    if dtype == torch.float32:                       # next to the borders too
        u = torch.from_numpy(rng.integers(-1, 2, (n, d)).astype(np.int32))
        x = torch.where(x != 0, (x.view(torch.int32) + u).view(torch.float32), x)
    if n > 8:
        x[1, :16] = 0
        x[2, 3] = float("nan")
        x[3, 20] = float("inf")
        x[4, 5] = -float("inf")
        x[5] = -0.0
        x[6] = 1e30
        x[7] = 2.0 ** -17 if dtype == torch.bfloat16 else 1e-40
    return x


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch,layers,heads,N,percent,n_a", [(1, 1, 1, 40, 50, -1), (2, 2, 3, 333, 30, -1), (1, 1, 2, 300, 20, 0), (1, 2, 1, 300, 40, 120), (3, 1, 1, 1500, 25, -1)])
def test_compact_and_read(dtype, d, batch, layers, heads, N, percent, n_a):
    rng = np.random.default_rng(N + d)
    sh = _shape(batch, layers, heads, d, dtype)
    LH, U = layers * heads, sh.units
    b = vec.vector_plan_budget(N, N * percent // 100, n_a, 16)
    K, V = (torch.stack([_hard_rows(N, d, rng, dtype) for _ in range(U)]) for _ in range(2))
    idx = np.stack([rng.permutation(N)[:b.n_pool] for _ in range(U)]).astype(np.int32)
    ri, ai = np.sort(idx[:, :b.n_ret], 1), np.sort(idx[:, b.n_ret:], 1)
    pages = [(batch * n + 63) // 64 + 2 for n in (b.n_ret, b.n_apx)]
    cache = _cache(sh, *pages, rng)
    rs, as_ = (rng.permutation(p * 64)[:batch * n].reshape(batch, n).astype(np.int32) for p, n in zip(pages, (b.n_ret, b.n_apx)))
    want = [t.cpu().numpy().copy() for t in (cache.ret_pages, cache.apx_pages, cache.ret_pos, cache.apx_pos)]
    vals = {}
    for u in range(U):
        s, lh = u // LH, u % LH
        rk, rv, ak = (x[u].double().numpy()[i[u]] for x, i in ((K, ri), (V, ri), (K, ai)))
        plain.put_rows(want[0], rs[s], lh, 0, rk)
        plain.put_rows(want[0], rs[s], lh, 1, rv)
        plain.put_rows(want[1], as_[s], lh, 0, ak)
        want[2][rs[s] // 64, lh, rs[s] % 64] = ri[u]
        want[3][as_[s] // 64, lh, as_[s] % 64] = ai[u]
        vals[u] = [plain.rounded(x) if len(x) else x for x in (rk, rv, ak)]
    on = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
    vec.vector_compact_q4(sh, b, K.to(DEV), V.to(DEV), on(ri), on(ai), cache, on(rs), on(as_))
    out = [torch.full((U, n, d), 3.0, dtype=dtype, device=DEV) for n in (b.n_ret, b.n_ret, b.n_apx)]
    vec.vector_read_q4(sh, cache, on(rs), out[0], out[1], on(as_), out[2])
    torch.cuda.synchronize()
    # codes of groups that are not numbers, and the sign of zero, may be anything: pages are compared as values, the rest of them as bytes
    for got, w, slots, parts in ((cache.ret_pages, want[0], rs, 2), (cache.apx_pages, want[1], as_, 1)):
        got = got.cpu().numpy()
        for lh in range(LH):
            for which in range(parts):
                allv = np.arange(got.shape[0] * 64)
                assert np.array_equal(plain.row_values(got, allv, lh, which, d), plain.row_values(w, allv, lh, which, d), equal_nan=True)
        cut = 64 * d // 2
        scales = lambda t: t.reshape(t.shape[0], LH, parts, -1)[..., cut:]  # noqa: E731
        assert np.array_equal(scales(got), scales(w))
    assert np.array_equal(cache.ret_pos.cpu().numpy(), want[2]) and np.array_equal(cache.apx_pos.cpu().numpy(), want[3])
    for u in range(U):
        for got, w in zip(out, vals[u]):
            assert np.array_equal(got[u].double().cpu().numpy(), w, equal_nan=True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_skipped(dtype, d):
    """Token indices outside the context and slots outside the pool leave everything as it is; reading such a slot gives zeros."""
    rng = np.random.default_rng(5)
    sh = _shape(1, 1, 2, d, dtype)
    b = vec.vector_plan_budget(200, 60, 10, 16)
    K, V = (torch.from_numpy(rng.standard_normal((2, 200, d))).to(dtype).to(DEV) for _ in range(2))
    cache = _cache(sh, 2, 1, rng)
    before = [t.clone() for t in (cache.ret_pages, cache.apx_pages, cache.ret_pos, cache.apx_pos)]
    ri = torch.full((2, b.n_ret), 5, dtype=torch.int32)
    ri[0, ::2], ri[1, ::2] = -1, 200
    ri[:, 1::2] = 2 ** 31 - 1
    ai = torch.arange(b.n_apx, dtype=torch.int32).repeat(2, 1)
    rs = torch.arange(b.n_ret, dtype=torch.int32).reshape(1, -1)
    as_ = torch.full((1, b.n_apx), -1, dtype=torch.int32)
    as_[0, 1::2], as_[0, 2] = 64, -2 ** 31
    vec.vector_compact_q4(sh, b, K, V, ri.to(DEV), ai.to(DEV), cache, rs.to(DEV), as_.to(DEV))
    vec.vector_append_q4(sh, cache, K[:, 0].contiguous(), V[:, 0].contiguous(), None, torch.tensor([128], dtype=torch.int32, device=DEV), torch.tensor([1], dtype=torch.int32, device=DEV))
    start = torch.tensor([0, 0], dtype=torch.int32, device=DEV)
    vec.vector_append_q4(sh, cache, K[:, 0].contiguous(), V[:, 0].contiguous(), start, torch.tensor([3], dtype=torch.int32, device=DEV), torch.tensor([1], dtype=torch.int32, device=DEV))
    start = torch.tensor([1, 2], dtype=torch.int32, device=DEV)          # beyond the slots that were written
    vec.vector_append_q4(sh, cache, K[:, 0].contiguous(), V[:, 0].contiguous(), start, torch.tensor([3], dtype=torch.int32, device=DEV), torch.tensor([1], dtype=torch.int32, device=DEV))
    out = torch.full((2, b.n_apx, d), 3.0, dtype=dtype, device=DEV)
    vec.vector_read_q4(sh, cache, None, None, None, as_.to(DEV), out)
    torch.cuda.synchronize()
    for t, w in zip((cache.ret_pages, cache.apx_pages, cache.ret_pos, cache.apx_pos), before):
        assert torch.equal(t, w)
    assert not out.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("batch,layers,heads", [(1, 1, 1), (5, 2, 3), (64, 1, 8)])
def test_append(dtype, d, batch, layers, heads):
    rng = np.random.default_rng(batch)
    sh = _shape(batch, layers, heads, d, dtype)
    LH, U = layers * heads, sh.units
    cache = _cache(sh, 4, 0, rng)
    k, v = (_hard_rows(U, d, rng, dtype) for _ in range(2))
    grows = rng.random(batch) < 0.7 if batch > 1 else np.array([True])
    start = np.concatenate([[0], np.cumsum(grows)]).astype(np.int32)
    slots = np.full(batch, -1, np.int32)
    slots[:grows.sum()] = rng.permutation(256)[:grows.sum()]
    pos = rng.integers(0, 1 << 30, batch).astype(np.int32)
    want, wpos = cache.ret_pages.cpu().numpy().copy(), cache.ret_pos.cpu().numpy().copy()
    for s in np.flatnonzero(grows):
        for lh in range(LH):
            at = slots[start[s]:start[s] + 1]
            plain.put_rows(want, at, lh, 0, k[s * LH + lh][None].double().numpy())
            plain.put_rows(want, at, lh, 1, v[s * LH + lh][None].double().numpy())
            wpos[at // 64, lh, at % 64] = pos[s]
    on = lambda x: (x if torch.is_tensor(x) else torch.from_numpy(x)).to(DEV)  # noqa: E731
    vec.vector_append_q4(sh, cache, on(k), on(v), on(start), on(slots), on(pos))
    direct = _cache(sh, 4, 0, np.random.default_rng(batch))
    own = np.array([slots[start[s]] if grows[s] else -1 for s in range(batch)], np.int32)
    vec.vector_append_q4(sh, direct, on(k), on(v), None, on(own), on(pos))
    torch.cuda.synchronize()
    got = cache.ret_pages.cpu().numpy()
    assert torch.equal(cache.ret_pages, direct.ret_pages) and np.array_equal(cache.ret_pos.cpu().numpy(), wpos)
    for lh in range(LH):
        for which in range(2):
            assert np.array_equal(plain.row_values(got, np.arange(256), lh, which, d), plain.row_values(want, np.arange(256), lh, which, d), equal_nan=True)
