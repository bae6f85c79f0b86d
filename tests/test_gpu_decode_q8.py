"""Attention over the 8-bit paged cache against 64 bits on the same stored rows: every type, head size and group, lengths around a page's end, blocks of very different
scales, sequences without rows, rotary keys, entries of tables that name no page, numbers that are none."""
import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200 import binding
import q4_plain
import q8_plain as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("d,g", [(128, 4), (64, 4), (128, 1), (128, 8), (64, 3), (64, 7), (128, 5)])
def test_lengths_around_a_page(dtype, out_dtype, d, g, rope):
    lengths = [(1, 0), (0, 1), (31, 32), (32, 33), (0, 0), (33, 0), (130, 257), (0, 500), (17, 16)]
    p = plain.problem(len(lengths), 1, 1, g, d, dtype, lengths, d + g, rope)
    out = plain.decode(*p, out_dtype)
    plain.check_decode(*p, out, rope)
    assert not out[4].any()


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype,d,g,batch,layers,heads,lengths", [
    (BF, 128, 4, 1, 1, 8, [(700, 1500)]),
    (BF, 128, 2, 3, 2, 2, [(20, 10), (900, 0), (333, 700)]),
    (BF, 64, 4, 2, 3, 4, [(511, 513), (0, 2000)]),
    (F32, 128, 3, 2, 1, 2, [(100, 1000), (1000, 100)]),
    (F32, 64, 8, 2, 1, 2, [(129, 1), (5, 640)]),
    (BF, 128, 1, 40, 1, 1, [(i * 7 % 300, i * 11 % 200) for i in range(40)]),
])
def test_batches(dtype, d, g, batch, layers, heads, lengths, rope):
    p = plain.problem(batch, layers, heads, g, d, dtype, lengths, 3, rope)
    for out_dtype in (F32, BF):
        plain.check_decode(*p, plain.decode(*p, out_dtype), rope)


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("out_dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_blocks_of_very_different_scales(d, out_dtype, rope):
    """Scales up and down by 2^30 from block to block: the sums change their unit and come back."""
    p = plain.problem(2, 1, 2, 3, d, BF, [(300, 300), (0, 400)], d, rope, spread=15.0)
    plain.check_decode(*p, plain.decode(*p, out_dtype), rope)


@pytest.mark.parametrize("which", ["largest", "smallest", "both"])
def test_scales_at_the_ends_of_their_range(which):
    """Values of 2^39 and of 2^-41, in one sequence too; keys that small make all weights alike."""
    sh, q, c, W = plain.problem(1, 1, 1, 4, 128, BF, [(96, 64)], 3)
    tile, t = plain.tile_bytes(128), c.ret_table[0].long()
    c.ret_pages[:, :, 32 * 128] = 0                                                   # keys: 2^-32
    c.apx_pages[:, :, 32 * 128] = 0
    for i in range(3):
        c.ret_pages[t[i], 0, tile + 32 * 128] = {"largest": 63, "smallest": 0, "both": 63 * (i % 2)}[which]
    plain.check_decode(sh, q, c, W, plain.decode(sh, q, c, W, F32), False)


def test_a_page_that_nobody_wrote_is_read_within_bounds():
    """A scale that is no code counts as the largest."""
    sh, q, c, W = plain.problem(1, 1, 1, 2, 128, BF, [(20, 0)], 5)
    c.ret_pages[c.ret_table[0, 0].long(), 0, plain.tile_bytes(128) + 32 * 128] = 255
    got = plain.decode(sh, q, c, W, F32)
    c.ret_pages[c.ret_table[0, 0].long(), 0, plain.tile_bytes(128) + 32 * 128] = 63
    assert torch.equal(got, plain.decode(sh, q, c, W, F32)) and torch.isfinite(got).all()


def test_many_units():
    """More units than there are workers, every length short."""
    lengths = [(3 * i % 130, 5 * i % 70) for i in range(33)]
    p = plain.problem(33, 4, 16, 2, 64, BF, lengths, 9)
    out = plain.decode(*p, F32)
    plain.check_decode(*p, out, False, range(0, p[0].units, 13))


def test_a_long_sequence():
    p = plain.problem(1, 1, 2, 4, 128, BF, [(9000, 17000)], 4)
    for out_dtype in (F32, BF):
        plain.check_decode(*p, plain.decode(*p, out_dtype), False)


def test_no_tier_at_all():
    sh, q, c, W = plain.problem(2, 1, 2, 2, 128, BF, [(100, 0), (40, 0)], 6)
    empty = torch.empty(0, 2, 4128, dtype=torch.uint8, device="cuda")
    none = vec.Q8Cache(c.ret_pages, empty, c.ret_table, torch.empty(2, 0, dtype=torch.int32, device="cuda"), c.ret_len, c.apx_len)
    plain.check_decode(sh, q, c, W, plain.decode(sh, q, none, W, F32), False)


def test_pages_that_are_none():
    """An entry outside the pool: its rows are not there; so are rows of a length beyond the table, and a negative length has none."""
    sh, q, c, W = plain.problem(3, 1, 1, 4, 128, BF, [(200, 300), (100, 100), (70, 10)], 8)
    c.ret_table[0, 1], c.ret_table[1, 0], c.apx_table[0, 4] = -1, c.ret_pages.shape[0], 2**31 - 1
    c.ret_len[2], c.apx_len[2] = -5, 1000
    c.apx_table[2, :] = -3
    c.apx_table[2, 1] = 0
    out = plain.decode(sh, q, c, W, F32)
    ret = [[r for r in range(200) if r // 32 != 1], list(range(32, 100)), []]
    apx = [[r for r in range(300) if r // 32 != 4], range(100), range(32, 64)]
    written = c.apx_pages[0, 0, 32 * 128].item() <= 63                               # sequence 2 attends to page 0 as it is
    for b in range(3):
        if b == 2 and not (written and bool((c.apx_pages[0, 0, :32 * 128] & 127 != 127).all())):
            continue
        plain.check_decode(sh, q, c, W, out, False, [b], ret_rows=ret[b], apx_rows=apx[b])


def test_numbers_that_are_none():
    """A NaN in a stored value shows in its own channel, one in a key in all of its unit, one in a query in its head; other sequences do not notice."""
    sh, q, c, W = plain.problem(4, 1, 1, 2, 128, BF, [(70, 70)] * 4, 10)
    t, tile = c.ret_table.long(), plain.tile_bytes(128)
    c.ret_pages[t[0, 1], 0, tile + plain.place(5, 9, 128)] = 127                       # value row 37 of sequence 0, channel 9
    c.ret_pages[t[1, 0], 0, plain.place(6, 100, 128)] = 255                           # key row 6 of sequence 1
    q[2, 1, 17] = float("nan")
    for out_dtype in (F32, BF):
        out = plain.decode(sh, q, c, W, out_dtype)
        nan = torch.isnan(out)
        assert nan[0, :, 9].all() and nan[0].sum() == 2 and nan[1].all() and nan[2, 1].all() and not nan[2, 0].any()
        plain.check_decode(sh, q, c, W, out, False, [3])


def test_rows_behind_the_last_may_be_anything():
    sh, q, c, W = plain.problem(2, 1, 2, 4, 64, BF, [(45, 70), (3, 1)], 11)
    first = [plain.decode(sh, q, c, W, t) for t in (F32, BF)]
    pool, keep = (c.ret_pages, c.apx_pages), []
    for pages, table, lengths, parts in ((pool[0], c.ret_table, c.ret_len, 2), (pool[1], c.apx_table, c.apx_len, 1)):
        x = pages.cpu().numpy()
        used = np.zeros(x.shape, bool)
        for b in range(2):
            for r in range(int(lengths[b])):
                for part in range(parts):
                    used[int(table[b, r // 32]), :, part * 2080 + np.append(plain._PLACES[64][r % 32], 32 * 64)] = True
        x = np.where(used, x, 127)                                                     # NaN, and scales that are none
        keep.append(torch.from_numpy(x).cuda())
    c.ret_pages, c.apx_pages = keep
    for was, t in zip(first, (F32, BF)):
        assert torch.equal(plain.decode(sh, q, c, W, t), was)


def test_sm_scale_and_repeated_calls(monkeypatch):
    sh, q, c, W = plain.problem(2, 1, 2, 4, 128, BF, [(300, 500), (10, 2000)], 11)
    first = plain.decode(sh, q, c, W, F32)
    for _ in range(3):
        assert torch.equal(plain.decode(sh, q, c, W, F32), first)
    sh.sm_scale = 128 ** -0.5
    assert torch.equal(plain.decode(sh, q, c, W, F32), first)
    monkeypatch.setattr(binding, "_marshal_module", binding._CtypesOnly())
    assert torch.equal(plain.decode(sh, q, c, W, F32), first)
    sh.sm_scale = 1e-6                                                               # all weights alike
    assert not torch.equal(plain.decode(sh, q, c, W, F32), first)


def test_logits_of_any_size():
    """Queries far outside fp16's range: logits of 1e9 pick one key; a logit scale at the end of fp32's range: all weights are alike."""
    sh, q, c, W = plain.problem(1, 1, 1, 2, 128, BF, [(80, 0)], 12)
    keys, rows = (plain.row_values(c.ret_pages.cpu().numpy(), c.ret_table[0].cpu().numpy(), range(80), 0, w, 128) for w in (0, 1))
    q.mul_(1e6)
    out = plain.decode(sh, q, c, W, F32)
    best = (q[0].double().cpu().numpy() @ keys.T).argmax(-1)
    assert abs(out[0].double().cpu().numpy() - rows[best]).max() <= 2.0 ** -20 * abs(rows).max()
    sh.sm_scale = 1e-38
    q.div_(1e6)
    out = plain.decode(sh, q, c, W, F32)
    assert abs(out[0].double().cpu().numpy() - rows.mean(0)).max() <= 2.0 ** -20 * np.abs(rows).mean(0).max()


def test_the_largest_batch():
    """1024 sequences, a few rows each, most places empty; one more is refused."""
    lengths = [(i % 7, (i * 5) % 11) if i % 3 == 0 else (0, 0) for i in range(1024)]
    lengths[1023] = (200, 129)
    p = plain.problem(1024, 1, 1, 2, 64, BF, lengths, 13)
    out = plain.decode(*p, F32)
    plain.check_decode(*p, out, False, [0, 3, 999, 1020, 1022, 1023])
    assert not out[1::3].any() and not out[2::3].any()


def test_offsets_beyond_32_bits():
    """Pages beyond 4 GB of both pools, written, appended to, read back and attended to."""
    sh = vec.Shape(1, 1, 4, 1, 128, vec.VECTOR_BF16, 16)
    pages = (1 << 32) // 4128 + 20
    c = vec.alloc_q8_cache(sh, pages, pages, 3, 2, positions=False)
    rng = np.random.default_rng(2)
    budget = vec.vector_plan_budget(200, 80, 30, 16)                             # 50 retained, 60 key-only
    K, V = (torch.from_numpy(rng.standard_normal((1, 200, 128))).to(BF).cuda() for _ in range(2))
    idx = torch.from_numpy(rng.permutation(200)[:110].astype(np.int32)).cuda()
    ret, apx = idx[:50].sort().values[None].contiguous(), idx[50:].sort().values[None].contiguous()
    c.ret_table[0] = torch.tensor([pages - 1, 0, pages - 2])
    c.apx_table[0] = torch.tensor([pages - 2, pages - 1])
    c.ret_len[0], c.apx_len[0] = 50, 60
    vec.vector_compact_q8(sh, budget, K, V, ret, apx, c)
    new = torch.from_numpy(rng.standard_normal((1, 20, 128))).to(BF).cuda()
    c.ret_len[0] = 70
    vec.vector_append_q8(sh, c, new, new, torch.tensor([50], dtype=torch.int32, device="cuda"))
    got = [torch.empty(1, n, 128, dtype=BF, device="cuda") for n in (70, 70, 60)]
    vec.vector_read_q8(sh, c, *got)
    torch.cuda.synchronize()
    rows = [x[0].double().cpu().numpy()[i[0].long().cpu().numpy()] for x, i in ((K, ret), (V, ret), (K, apx))]
    more = new[0].double().cpu().numpy()
    want = [plain.Held().append(rows[0]).append(more).values(128), plain.Held().append(rows[1]).append(more).values(128), plain.rounded(rows[2])]
    for x, w in zip(got, want):
        assert np.array_equal(x[0].double().cpu().numpy(), w)
    q, W = torch.randn(1, 4, 128, device="cuda").to(BF), (torch.randn(1, 128, 128, device="cuda") / 11).to(BF)
    out = plain.decode(sh, q, c, W, F32)
    o, *sizes = q4_plain.attend(q[0].double().cpu().numpy(), *want, W[0].double().cpu().numpy(), 128 ** -0.5)
    assert np.all(np.abs(out[0].double().cpu().numpy() - o) <= q4_plain.tolerance(o, *sizes, BF, F32, False))


def _shared(batch, g, d, dtype, rk, rv, q, sm_scale):
    """`batch` sequences that share the pages of rows rk, rv, which are held exactly."""
    n = len(rk)
    shape = vec.Shape(batch, 1, g, 1, d, vec.VECTOR_BF16 if dtype == BF else vec.VECTOR_F32, 16, 7, sm_scale, 0, 10000.0)
    pages = -(-n // 32)
    pool = np.zeros((pages, 1, 2 * plain.tile_bytes(d)), np.uint8)
    for which, x in ((0, rk), (1, rv)):
        plain.put_rows(pool, np.arange(pages), 0, which, x)
        assert np.array_equal(plain.row_values(pool, np.arange(pages), range(n), 0, which, d), x)
    ints = lambda x: torch.as_tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    c = vec.Q8Cache(torch.from_numpy(pool).cuda(), torch.empty(0, 1, plain.tile_bytes(d), dtype=torch.uint8, device="cuda"), ints(np.tile(np.arange(pages), (batch, 1))),
                    torch.empty(batch, 0, dtype=torch.int32, device="cuda"), ints(np.full(batch, n)), ints(np.zeros(batch)))
    return shape, torch.from_numpy(q).to(dtype).cuda().expand(batch, g, d).contiguous(), c, torch.zeros(1, d, d, dtype=dtype, device="cuda")


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("d,g", [(128, 4), (64, 4), (128, 8), (64, 1)])
@pytest.mark.parametrize("gap", [8, 14, 18])
def test_a_sink_without_a_value(dtype, out_dtype, d, g, gap):
    """A key that takes all the weight and has a value of zero, before thousands whose weights are e^-gap of it and make the output, with values whose blocks' scales go up and down.  Tolerance as over
    the 4-bit pages: logits are exact but for the factor (2^-23 twice of gap, twice), exponentials 2^-21 twice, weights 2^-11 twice in one fp16 part and 2^-21 twice in two, sums of 16 rows 2^-20 and
    n / 16 of these 2^-24 each, twice (2^-23 where they are cut off), and the result's own rounding."""
    n = 3500
    rng = np.random.default_rng(gap)
    rk, rv = np.zeros((n, d)), rng.choice([0.5, 1.0, 1.5, 2.0, 3.0], (n, d)) * np.repeat(2.0 ** rng.integers(-6, 7, -(-n // 32)), 32)[:n, None]
    rk[1:, 5], rk[:, 4] = -2.0, 3.0
    rv[0] = 0
    q = np.zeros((g, d))
    q[:, 5] = 1.0
    sh, qt, c, W = _shared(1000, g, d, dtype, rk, rv, q, gap / 2.0)
    out = plain.decode(sh, qt, c, W, out_dtype).double().cpu().numpy()
    p = np.exp(-float(gap))
    o = (p * rv[1:].sum(0) / (1 + (n - 1) * p))[None, None]
    exact = F32 in (dtype, out_dtype)
    steps = -(-n // 16) * (2.0 ** -24 if exact else 2.0 ** -23)
    tol = (gap * 2.0 ** -23 * 2 + 2.0 ** -20 + (2.0 ** -20 if exact else 2.0 ** -10) + 2.0 ** -20 + 2 * steps + (2.0 ** -24 if out_dtype == F32 else 2.0 ** -8)) * o
    err = np.abs(out - o)
    assert np.all(err <= tol), float((err / tol).max())


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("d,g,top", [(128, 4, 1 << 20), (64, 3, 1 << 30), (128, 2, 1 << 30), (64, 8, 1 << 30)])
def test_far_positions(dtype, out_dtype, d, g, top):
    """Positions up to 2^30: the tolerance is that of near ones."""
    sh, q, c, W = plain.problem(2, 1, 1, g, d, dtype, [(0, 200), (90, 65)], 32, rope=True)
    c.apx_pos.copy_(torch.randint(top // 2, top, c.apx_pos.shape, generator=torch.Generator().manual_seed(1), dtype=torch.int32))
    plain.check_decode(sh, q, c, W, plain.decode(sh, q, c, W, out_dtype), True)


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("d", [64, 128])
def test_the_largest_stored_keys_turned(dtype, out_dtype, d):
    """Keys of 448 2^31 in every channel, whose pairs turn to 634 2^31: the even heads attend to one alone, for the odd ones its weight is zero.  No logit term in the tolerance of the even
    heads, as the weights are one and zero."""
    at, g = 37, 4
    sh, q, c, W = plain.problem(1, 1, 1, g, d, dtype, [(70, 130)], 31, rope=True)
    t, page = c.apx_table.cpu().numpy()[0], int(c.apx_table[0, at // 32])
    pool = c.apx_pages.cpu().numpy()
    x = np.zeros((32, d))
    x[at % 32] = 448 * 2.0 ** 31
    plain.put_rows(pool, [page], 0, 0, x)
    c.apx_pages.copy_(torch.from_numpy(pool))
    c.apx_pos[page, 0, at % 32] = 7854
    q[0] = q[0].abs()
    q[0, 1::2] *= -1
    out = plain.decode(sh, q, c, W, out_dtype)
    rows = np.arange(130)
    ak, pos = plain.row_values(pool, t, rows, 0, 0, d), c.apx_pos.cpu().numpy()[t[rows // 32], 0, rows % 32]
    rk, rv = (plain.row_values(c.ret_pages.cpu().numpy(), c.ret_table[0].cpu().numpy(), range(70), 0, w, d) for w in (0, 1))
    none = np.zeros((0, d))
    for heads, pick in ((slice(0, None, 2), rows == at), (slice(1, None, 2), rows != at)):
        even = heads.start == 0
        o, spread, logit, turned = q4_plain.attend(q[0, heads].double().cpu().numpy(), none if even else rk, none if even else rv, ak[pick], W[0].double().cpu().numpy(), d ** -0.5, pos[pick])
        tol = q4_plain.tolerance(o, spread, logit * heads.start, turned, dtype, out_dtype, True)
        err = np.abs(out[0, heads].double().cpu().numpy() - o)
        assert np.all(np.isfinite(err)) and np.all(err <= tol), (heads.start, float((err / tol).max()))
