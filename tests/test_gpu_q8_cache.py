"""Writing and reading the 8-bit paged cache against its definition in 64 bits: compaction, new rows by ones and by thousands, scales that grow, keys turned on the way, rows
of wider rows, lengths and pages that are none."""
import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200 import binding
import q8_plain as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda"


def _shape(batch, layers, heads, d, dtype, rope=0):
    return vec.Shape(batch, layers, heads, heads, d, vec.VECTOR_BF16 if dtype == BF else vec.VECTOR_F32, 16, 7, 0.0, rope, 10000.0)


def _ints(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _cache(sh, ret_rows, apx_rows, seed, positions=True):
    """Pages with whatever was in memory, tables with room for so many rows a sequence in no order, one page in none of them."""
    rng = np.random.default_rng(seed)
    LH, tile, B = sh.n_layers * sh.n_kv_heads, plain.tile_bytes(sh.head_dim), sh.batch
    got = []
    for rows, parts in ((ret_rows, 2), (apx_rows, 1)):
        width = max(-(-rows // 32), 1)
        pages = B * width + 1
        got += [torch.from_numpy(rng.integers(0, 256, (pages, LH, parts * tile), dtype=np.uint8)).to(DEV), _ints(rng.permutation(pages)[:B * width].reshape(B, width)),
                _ints(np.full((pages, LH, 32), -7))]
    rp, rt, rpos, ap, at, apos = got
    return vec.Q8Cache(rp, ap, rt, at, _ints([ret_rows] * B), _ints([apx_rows] * B), rpos if positions else None, apos if positions else None)


def _read(sh, c, n_ret, n_apx=0):
    new = lambda n: torch.full((sh.units, n, sh.head_dim), 5.0, dtype=sh.torch_dtype, device=DEV)  # noqa: E731
    k, v, a = new(n_ret), new(n_ret), new(n_apx)
    vec.vector_read_q8(sh, c, k, v, a if n_apx else None)
    return tuple(t.double().cpu().numpy() for t in (k, v, a))


def _values(rng, dtype, *size):
    x = rng.standard_normal(size) * np.exp(rng.uniform(-4, 3, size[:-1] + (1,)))
    x[..., 3] *= 20.0                                                          # a channel that is larger than the others
    return torch.from_numpy(x).to(dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,batch,layers,heads,N,pairs,n_a", [(128, 1, 1, 8, 900, 400, 200), (64, 3, 2, 3, 333, 97, 20), (128, 2, 1, 2, 100, 33, 1), (64, 1, 1, 1, 40, 32, 0),
                                                              (128, 1, 1, 1, 64, 32, 32), (64, 2, 1, 1, 17, 16, 0)])
def test_compaction_and_back(dtype, d, batch, layers, heads, N, pairs, n_a):
    rng = np.random.default_rng(d + N)
    sh, b = _shape(batch, layers, heads, d, dtype), vec.vector_plan_budget(N, pairs, n_a, 16)
    U, LH = sh.units, layers * heads
    K, V = _values(rng, dtype, U, N, d), _values(rng, dtype, U, N, d)
    if N == 900:                                                               # a block of zeros, a NaN, infinities, the ends of the range
        K[0, :, :5], V[0, 40] = 0, float("nan")
        K[1, 7, 9], K[1, 300, 2], V[2, 11, 1] = float("nan"), float("inf"), float("-inf")
        K[3] *= 1e30 if dtype == F32 else 2.0 ** 40
        V[3] *= 2.0 ** -45
    pick = np.stack([rng.permutation(N)[:b.n_pool] for _ in range(U)]).astype(np.int32)
    ret, apx = np.sort(pick[:, :b.n_ret]), np.sort(pick[:, b.n_ret:])
    c = _cache(sh, b.n_ret + 5, b.n_apx + 40, N)
    c.ret_len[:], c.apx_len[:] = b.n_ret, b.n_apx
    before = [t.clone() for t in (c.ret_pages, c.apx_pages, c.ret_pos)]
    vec.vector_compact_q8(sh, b, K.to(DEV), V.to(DEV), _ints(ret), _ints(apx), c)
    got = _read(sh, c, b.n_ret + 3, b.n_apx + 3)
    k, v = K.double().numpy(), V.double().numpy()
    for u in range(U):
        for x, rows, n in ((got[0], k[u, ret[u]], b.n_ret), (got[1], v[u, ret[u]], b.n_ret), (got[2], k[u, apx[u]], b.n_apx)):
            assert np.array_equal(x[u, :n], plain.rounded(rows), equal_nan=True) and not x[u, n:].any(), u
        table, lh = c.ret_table[u // LH].cpu().numpy(), u % LH
        at = np.arange(b.n_ret)
        assert np.array_equal(c.ret_pos.cpu().numpy()[table[at // 32], lh, at % 32], ret[u])
        if b.n_apx:
            at = np.arange(b.n_apx)
            assert np.array_equal(c.apx_pos.cpu().numpy()[c.apx_table[u // LH].cpu().numpy()[at // 32], lh, at % 32], apx[u])
    # rows behind the last, and pages in no table, are as they were
    for now, was, n, table, parts in ((c.ret_pages, before[0], b.n_ret, c.ret_table, 2), (c.apx_pages, before[1], b.n_apx, c.apx_table, 1)):
        now, was, tile = now.cpu().numpy().copy(), was.cpu().numpy().copy(), plain.tile_bytes(d)
        for t in table.cpu().numpy():
            for part in range(parts):
                for block in range(-(-n // 32)):
                    for x in (now, was):
                        x[t[block], :, part * tile:part * tile + min(n - 32 * block, 32) * d] = 0
                        x[t[block], :, part * tile + 32 * d] = 0
        assert np.array_equal(now, was)
    assert int((c.ret_pos != before[2]).sum()) <= U * b.n_ret


def test_compaction_of_what_is_not_there():
    """Lengths shorter than the budget's, a page outside the pool, tokens outside the context, a negative length."""
    rng = np.random.default_rng(3)
    sh, b = _shape(4, 1, 2, 128, BF), vec.vector_plan_budget(200, 110, 10, 16)                     # 100 retained, 20 key-only
    K, V = _values(rng, BF, 8, 200, 128), _values(rng, BF, 8, 200, 128)
    ret, apx = np.tile(np.arange(0, 200, 2), (8, 1)), np.tile(np.arange(1, 41, 2), (8, 1))
    ret[2, 5], ret[3, 40], apx[0, 0] = -1, 200, 2**31 - 1
    c = _cache(sh, 128, 32, 1)
    c.ret_len[:], c.apx_len[:] = _ints([0, 100, 70, -3]), _ints([20, 20, 20, 20])
    c.ret_table[1, 1], c.ret_table[2, 0] = -1, c.ret_pages.shape[0]
    before = c.ret_pages.clone()
    vec.vector_compact_q8(sh, b, K.to(DEV), V.to(DEV), _ints(ret), _ints(apx), c)
    k, v, a = _read(sh, c, 100, 20)
    for u in range(8):
        rows = K[u].double().numpy()[np.clip(ret[u], 0, 199)]
        rows[(ret[u] < 0) | (ret[u] >= 200)] = 0
        keys = K[u].double().numpy()[np.clip(apx[u], 0, 199)]
        keys[apx[u] >= 200] = 0
        assert np.array_equal(a[u], plain.rounded(keys))
        n = [0, 100, 70, 0][u // 2]
        want = plain.rounded(rows[:n])
        want[[r for r in range(n) if (u // 2 == 1 and r // 32 == 1) or (u // 2 == 2 and r // 32 == 0)]] = 0
        assert np.array_equal(k[u, :n], want) and not k[u, n:].any() and not v[u, n:].any()
    for b_ in (0, 3):
        assert torch.equal(c.ret_pages[c.ret_table[b_].long()], before[c.ret_table[b_].long()])


@pytest.mark.parametrize("dtype,d,layers,heads", [(BF, 128, 1, 3), (F32, 128, 2, 1), (BF, 64, 1, 2), (F32, 64, 1, 1)])
def test_rows_come_by_ones_and_by_hundreds(dtype, d, layers, heads):
    """Every call's rows against the definition, bit by bit: beginnings within a block, blocks crossed, scales that grow, sequences without new rows."""
    rng = np.random.default_rng(d + layers)
    B, LH = 4, layers * heads
    sh = _shape(B, layers, heads, d, dtype)
    c = _cache(sh, 700, 0, 5)
    held = [[plain.Held() for _ in range(LH * 2)] for _ in range(B)]
    length, pos_of = np.zeros(B, int), [[] for _ in range(B)]
    for n, each in ((1, [1, 1, 0, 1]), (1, [1, 0, 1, 1]), (5, [5, 3, 0, 1]), (40, [40, 27, 25, 0]), (33, [33, 33, 33, 1]), (1, [1, 1, 1, 1]), (300, [300, 1, 299, 32]), (64, [0, 64, 64, 31])):
        k, v = (_values(rng, dtype, B, n, LH, d) * float(2 ** rng.integers(0, 6)) for _ in range(2))
        pos = rng.integers(-5, 1 << 20, (B, n))
        first, length = length, length + each
        c.ret_len[:] = _ints(length)
        vec.vector_append_q8(sh, c, k.to(DEV), v.to(DEV), _ints(first), _ints(pos))
        most = int(length.max()) + 2
        rk, rv, _ = _read(sh, c, most)
        rpos = c.ret_pos.cpu().numpy()
        for b in range(B):
            pos_of[b] += pos[b, :each[b]].tolist()
            at = np.arange(length[b])
            for u in range(LH):
                for is_v, (x, got) in enumerate(((k, rk), (v, rv))):
                    want = held[b][2 * u + is_v].append(x[b, :each[b], u].double().numpy()).values(d)
                    assert np.array_equal(got[b * LH + u, :length[b]], want) and not got[b * LH + u, length[b]:].any(), (n, b, u, is_v)
                assert rpos[c.ret_table[b].cpu().numpy()[at // 32], u, at % 32].tolist() == pos_of[b]


def test_rows_that_are_not_given_or_have_no_place():
    rng = np.random.default_rng(4)
    sh = _shape(5, 1, 1, 64, BF)
    c = _cache(sh, 96, 0, 2, positions=False)
    x = _values(rng, BF, 5, 8, 1, 64)
    before = c.ret_pages.clone()
    # more rows counted than given; length below the first row; beyond the table; a page outside the pool; a negative first row
    c.ret_len[:], first = _ints([50, 10, 2**31 - 1, 40, 4]), _ints([10, 20, 92, 30, -3])
    c.ret_table[3, 1] = -9
    vec.vector_append_q8(sh, c, x.to(DEV), x.to(DEV), first)
    c.ret_len[:] = _ints([96] * 5)
    k, _, _ = _read(sh, c, 96)
    t = c.ret_table.cpu().numpy()
    was = lambda b, block: before.cpu().numpy()[t[b, block]]  # noqa: E731
    now = lambda b, block: c.ret_pages.cpu().numpy()[t[b, block]]  # noqa: E731
    codes = lambda page, r: page[0, plain._PLACES[64][r]]  # noqa: E731
    for r in range(18, 32):
        assert np.array_equal(codes(now(0, 0), r), codes(was(0, 0), r))            # only eight rows were given
    assert np.array_equal(now(0, 1), was(0, 1)) and all(np.array_equal(now(1, i), was(1, i)) for i in range(3))
    assert np.array_equal(now(2, 0), was(2, 0)) and not np.array_equal(now(2, 2), was(2, 2))
    new = k[3, 30:32]
    step = 2.0 ** -3 * np.abs(x[3, :2, 0].double().numpy()) + 2.0 ** -9 * 2.0 ** (float(now(3, 0)[0, 32 * 64]) - 32)
    assert np.all(np.abs(new - x[3, :2, 0].double().numpy()) <= step)
    assert np.array_equal(k[4, :4], plain.rounded(x[4, :4, 0].double().numpy()))     # counted from row 0


@pytest.mark.parametrize("LH", [2, 3])                       # heads that share a thread block by two, and alone
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
def test_keys_are_turned_on_the_way(dtype, d, LH):
    """Within half a step of the turned key in 64 bits, and what fp32 makes of it: sine and cosine (2^-24 and 2e-9 of angle and series), two products and a sum."""
    rng = np.random.default_rng(d)
    B, n = 3, 45
    sh = _shape(B, 1, LH, d, dtype, 1)
    c = _cache(sh, 70, 0, 3)
    c.ret_len[:], first = _ints([45, 60, 64]), np.array([0, 20, 31])
    k, v = _values(rng, dtype, B, n, LH, d), _values(rng, dtype, B, n, LH, d)
    pos = rng.integers(0, 1 << 20, (B, n))
    pos[1] = np.arange(n) - 7
    pos[0, :3] = 0
    for b in range(B):                                                              # rows before, of a scale that is smaller than the new ones'
        vec.vector_append_q8(_shape(1, 1, LH, d, dtype), vec.Q8Cache(c.ret_pages, c.apx_pages, c.ret_table[b:b + 1], c.apx_table[b:b + 1], _ints([first[b]]), c.apx_len[b:b + 1]),
                             torch.ones(1, 32, LH, d, dtype=dtype, device=DEV) / 64, torch.ones(1, 32, LH, d, dtype=dtype, device=DEV), _ints([0]))
    vec.vector_append_q8(sh, c, k.to(DEV), v.to(DEV), _ints(first), _ints(pos), rotate=True)
    rk, rv, _ = _read(sh, c, 64)
    for b in range(B):
        rows = min(int(c.ret_len[b]) - first[b], n)
        for u in range(LH):
            x = k[b, :rows, u].double().numpy()
            want, got = plain.turned(x, pos[b, :rows]), rk[b * LH + u, first[b]:first[b] + rows]
            size = np.tile(np.abs(x[:, :d // 2]) + np.abs(x[:, d // 2:]), (1, 2))
            scale = np.repeat([2.0 ** plain.exponent(want[max(32 * i - first[b], 0):32 * (i + 1) - first[b]]) for i in range(first[b] // 32, (first[b] + rows - 1) // 32 + 1)], 32)
            scale = scale[first[b] % 32:][:rows, None]
            big = np.maximum(np.abs(want), np.abs(got))
            unit = np.exp2(np.maximum(np.floor(np.log2(np.maximum(big, 1e-300) / scale)), -6) - 3) * scale
            assert np.all(np.abs(got - want) <= unit / 2 + 6 * 2.0 ** -24 * size), (b, u)
            if pos[b, 0] == 0:
                assert np.array_equal(got[:3], plain.number(plain.encode(x[:3], int(np.log2(scale[0, 0])))) * scale[:3])
            h = plain.Held().append(np.ones((first[b], d))).append(v[b, :rows, u].double().numpy()) if first[b] else plain.Held().append(v[b, :rows, u].double().numpy())
            assert np.array_equal(rv[b * LH + u, first[b]:first[b] + rows], h.values(d)[first[b]:])


def test_a_nan_and_infinities_among_new_rows():
    sh = _shape(1, 1, 1, 128, BF)
    c = _cache(sh, 32, 0, 8, positions=False)
    x = torch.ones(1, 4, 1, 128, dtype=BF)
    x[0, 1, 0, 5], x[0, 2, 0, 7] = float("nan"), float("inf")
    c.ret_len[0] = 2
    vec.vector_append_q8(sh, c, x[:, :2].contiguous().to(DEV), x[:, :2].contiguous().to(DEV), _ints([0]))
    k, _, _ = _read(sh, c, 2)
    assert np.isnan(k[0, 1, 5]) and np.isnan(k).sum() == 1 and (k[0, 0] == 1).all()
    c.ret_len[0] = 4
    vec.vector_append_q8(sh, c, x[:, 2:].contiguous().to(DEV), x[:, 2:].contiguous().to(DEV), _ints([2]))
    k, _, _ = _read(sh, c, 4)
    assert np.isnan(k[0, 1, 5]) and k[0, 2, 7] == 448 * 2.0 ** 31 and (np.delete(k[0].ravel(), [128 + 5, 256 + 7]) == 0).all()


def test_rows_of_wider_rows_and_both_ways_of_marshalling(monkeypatch):
    rng = np.random.default_rng(6)
    B, LH, d, n = 3, 2, 128, 7
    sh = _shape(B, 1, LH, d, BF)
    wide = _values(rng, BF, B, n, (2 * LH + 1) * d).to(DEV)
    k, v = wide[..., d:d + LH * d], wide[..., d + LH * d:]
    got = []
    for way in ("module", "module", "ctypes", "ctypes"):
        if way == "ctypes":
            monkeypatch.setattr(binding, "_marshal_module", binding._CtypesOnly())
        c = _cache(sh, 64, 0, 9)
        c.ret_len[:] = _ints([7, 3, 20])
        strided = len(got) % 2 == 0
        pos = _ints(np.arange(B * n).reshape(B, n))
        vec.vector_append_q8(sh, c, k if strided else k.contiguous(), v.unflatten(-1, (LH, d)) if strided else v.contiguous(), _ints([0, 0, 13]), pos)
        got.append((c.ret_pages, c.ret_pos, *_read(sh, c, 33)))
    for other in got[1:]:
        assert torch.equal(got[0][0], other[0]) and torch.equal(got[0][1], other[1]) and np.array_equal(got[0][2], other[2], equal_nan=True) and np.array_equal(got[0][3], other[3], equal_nan=True)      # rows before sequence 2's first are what was in memory
    assert np.array_equal(got[0][2][0, :7], plain.rounded(k[0, :, :d].double().cpu().numpy()))
    b = vec.vector_plan_budget(64, 40, 8, 16)
    K, idx = _values(rng, BF, B * LH, 64, d).to(DEV), _ints(np.tile(np.arange(48), (B * LH, 1)))
    pages = []
    for module in (None, binding._CtypesOnly()):
        monkeypatch.setattr(binding, "_marshal_module", module)
        c = _cache(sh, 32, 16, 9)
        vec.vector_compact_q8(sh, b, K, K, idx[:, :32].contiguous(), idx[:, 32:].contiguous(), c)
        pages.append((c.ret_pages, c.apx_pages))
    assert torch.equal(pages[0][0], pages[1][0]) and torch.equal(pages[0][1], pages[1][1])


def test_refusals_of_the_binding():
    sh = _shape(2, 1, 2, 128, BF)
    c = _cache(sh, 64, 32, 1)
    x = torch.zeros(2, 3, 2, 128, dtype=BF, device=DEV)
    for bad in (dict(k=x.float()), dict(v=x[:, :2]), dict(first=_ints([0])), dict(pos=_ints([0, 1])), dict(pos=_ints([[0] * 4] * 2)), dict(k=x.transpose(1, 2))):
        with pytest.raises(ValueError):
            vec.vector_append_q8(sh, c, bad.get("k", x), bad.get("v", x), bad.get("first", _ints([0, 0])), bad.get("pos", _ints([[0] * 3] * 2)))
    with pytest.raises(vec.VectorError, match="null"):
        vec.vector_append_q8(sh, c, x, x, _ints([0, 0]))
    with pytest.raises(vec.VectorError, match="shape"):
        vec.vector_append_q8(sh, c, x, x, _ints([0, 0]), _ints([[0] * 3] * 2), rotate=True)
    out = torch.zeros(4, 3, 128, dtype=BF, device=DEV)
    for k, v in ((out, None), (None, out), (out, out[:, :2].contiguous()), (out.flatten()[:-1], out.flatten()[:-1]), (out.float(), out.float()), (out.cpu(), out.cpu())):
        with pytest.raises(ValueError):
            vec.vector_read_q8(sh, c, k, v)
    four = vec.alloc_q4_cache(sh, 4, 4, 2, 2)
    with pytest.raises(ValueError, match="pages"):
        vec.vector_read_q8(sh, four, torch.zeros(4, 3, 128, dtype=BF, device=DEV), torch.zeros(4, 3, 128, dtype=BF, device=DEV))
    with pytest.raises(ValueError, match="pages"):
        vec.vector_decode_attn_q4(sh, torch.zeros(4, 1, 128, dtype=BF, device=DEV), c, torch.zeros(2, 128, 128, dtype=BF, device=DEV), torch.zeros(4, 1, 128, dtype=BF, device=DEV))
