"""Attention over the 4-bit paged cache against 64 bits on the same stored rows: every type, head size and group, lengths around a page's
end, sequences without rows, rotary keys, entries of tables that name no page."""
import pytest
import torch

import paper_2605_23258_b200 as vec
import q4_plain as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)])
@pytest.mark.parametrize("d,g", [(128, 4), (64, 4), (128, 1), (128, 8), (64, 3), (64, 7), (128, 5)])
def test_lengths_around_a_page(dtype, out_dtype, d, g, rope):
    lengths = [(1, 0), (0, 1), (63, 64), (64, 65), (0, 0), (65, 0), (130, 257), (0, 500)]
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
    empty = torch.empty(0, 2, 4608, dtype=torch.uint8, device="cuda")
    none = vec.Q4Cache(c.ret_pages, empty, c.ret_table, torch.empty(2, 0, dtype=torch.int32, device="cuda"), c.ret_len, c.apx_len)
    out = plain.decode(sh, q, none, W, F32)
    plain.check_decode(sh, q, c, W, out, False)


def test_pages_that_are_none():
    """An entry outside the pool: its rows are not there; so are rows of a length beyond the table, and a negative length has none."""
    sh, q, c, W = plain.problem(3, 1, 1, 4, 128, BF, [(200, 300), (100, 100), (70, 10)], 8)
    n = c.ret_pages.shape[0]
    c.ret_table[0, 1], c.ret_table[1, 0], c.apx_table[0, 4] = -1, n, 2**31 - 1
    c.ret_len[2], c.apx_len[2] = -5, 1000
    c.apx_table[2, :] = -3
    c.apx_table[2, 1] = 0
    out = plain.decode(sh, q, c, W, F32)
    keep = [[r for r in range(200) if r // 64 != 1], list(range(64, 100))]
    import numpy as np
    rp, ap = c.ret_pages.cpu().numpy(), c.apx_pages.cpu().numpy()
    for b in range(3):
        rows = keep[b] if b < 2 else []
        apx = [r for r in range(300) if r // 64 != 4] if b == 0 else range(100) if b == 1 else range(64, 128)
        rt, at = c.ret_table[b].cpu().numpy(), c.apx_table[b].cpu().numpy()
        rs = np.array([rt[r // 64] * 64 + r % 64 for r in rows], np.int64)
        as_ = np.array([at[r // 64] * 64 + r % 64 for r in apx], np.int64)
        rk, rv = (plain.row_values(rp, rs, 0, w, 128) if len(rs) else np.zeros((0, 128)) for w in (0, 1))
        o, *sizes = plain.attend(q[b].double().cpu().numpy(), rk, rv, plain.row_values(ap, as_, 0, 0, 128), W[0].double().cpu().numpy(), 128 ** -0.5)
        err = np.abs(out[b].double().cpu().numpy() - o)
        assert np.all(err <= plain.tolerance(o, *sizes, BF, F32, False)), b


def test_rows_of_numbers_that_are_none():
    """A stored row that holds a NaN shows in its own sequence's outputs alone."""
    sh, q, c, W = plain.problem(2, 1, 1, 2, 128, BF, [(70, 70), (70, 70)], 10)
    page = int(c.ret_table[0, 0])
    c.ret_pages[page, 0, 4608 + 4096 + 8 * 5:4608 + 4096 + 8 * 6] = 255             # value row 5 of sequence 0
    out = plain.decode(sh, q, c, W, F32)
    assert torch.isnan(out[0]).all()
    plain.check_decode(sh, q, c, W, out, False, [1])


def test_sm_scale_and_repeated_calls():
    sh, q, c, W = plain.problem(2, 1, 2, 4, 128, BF, [(300, 500), (10, 2000)], 11)
    first = plain.decode(sh, q, c, W, F32)
    for _ in range(3):
        assert torch.equal(plain.decode(sh, q, c, W, F32), first)
    sh.sm_scale = 128 ** -0.5
    assert torch.equal(plain.decode(sh, q, c, W, F32), first)
    sh.sm_scale = 1e-6                                                               # all weights alike
    assert not torch.equal(plain.decode(sh, q, c, W, F32), first)


def test_large_queries_and_keys():
    """Queries far outside fp16's range, keys at its end: logits of 1e9 pick one key."""
    sh, q, c, W = plain.problem(1, 1, 1, 2, 128, BF, [(80, 0)], 12)
    q.mul_(1e6)
    out = plain.decode(sh, q, c, W, F32)
    rows = plain.row_values(c.ret_pages.cpu().numpy(), plain.slots_of(c.ret_table[0].cpu().numpy(), 80), 0, 1, 128)
    keys = plain.row_values(c.ret_pages.cpu().numpy(), plain.slots_of(c.ret_table[0].cpu().numpy(), 80), 0, 0, 128)
    best = (q[0].double().cpu().numpy() @ keys.T).argmax(-1)
    assert abs(out[0].double().cpu().numpy() - rows[best]).max() <= 2.0 ** -20 * abs(rows).max()


def test_the_largest_batch():
    """1024 sequences, a few rows each, most places empty; one more is refused."""
    lengths = [(i % 7, (i * 5) % 11) if i % 3 == 0 else (0, 0) for i in range(1024)]
    lengths[1023] = (200, 129)
    p = plain.problem(1024, 1, 1, 2, 64, BF, lengths, 13)
    out = plain.decode(*p, F32)
    plain.check_decode(*p, out, False, [0, 3, 999, 1020, 1022, 1023])
    assert not out[1::3].any() and not out[2::3].any()


def test_offsets_beyond_32_bits():
    """Pages beyond 4 GB of both pools, written, read back and attended to."""
    import numpy as np
    sh = vec.Shape(1, 1, 4, 1, 128, vec.VECTOR_BF16, 16)
    pages = (1 << 32) // 4608 + 20
    c = vec.alloc_q4_cache(sh, pages, pages, 2, 2, positions=False)
    rng = np.random.default_rng(2)
    budget = vec.vector_plan_budget(200, 100, 30, 16)                            # 70 retained, 60 key-only
    K, V = (torch.from_numpy(rng.standard_normal((1, 200, 128))).to(BF).cuda() for _ in range(2))
    idx = torch.from_numpy(rng.permutation(200)[:130].astype(np.int32)).cuda()
    ret, apx = idx[:70].sort().values[None].contiguous(), idx[70:].sort().values[None].contiguous()
    c.ret_table[0] = torch.tensor([pages - 1, 0])
    c.apx_table[0] = torch.tensor([pages - 2, pages - 1])
    c.ret_len[0], c.apx_len[0] = 70, 60
    rs, as_ = (torch.from_numpy(plain.slots_of(t[0].cpu().numpy(), n)[None].astype(np.int32)).cuda() for t, n in ((c.ret_table, 70), (c.apx_table, 60)))
    vec.vector_compact_q4(sh, budget, K, V, ret, apx, c, rs, as_)
    got = [torch.empty(1, n, 128, dtype=BF, device="cuda") for n in (70, 70, 60)]
    vec.vector_read_q4(sh, c, rs, got[0], got[1], as_, got[2])
    torch.cuda.synchronize()
    want = [plain.rounded(x[0].double().cpu().numpy()[i[0].long().cpu().numpy()]) for x, i in ((K, ret), (V, ret), (K, apx))]
    for x, w in zip(got, want):
        assert np.array_equal(x[0].double().cpu().numpy(), w)
    q, W = torch.randn(1, 4, 128, device="cuda").to(BF), (torch.randn(1, 128, 128, device="cuda") / 11).to(BF)
    out = plain.decode(sh, q, c, W, F32)
    o, *sizes = plain.attend(q[0].double().cpu().numpy(), *want, W[0].double().cpu().numpy(), 128 ** -0.5)
    assert np.all(np.abs(out[0].double().cpu().numpy() - o) <= plain.tolerance(o, *sizes, BF, F32, False))


def test_scales_of_logits_near_nothing():
    """A logit scale at the end of fp32's range: all weights are alike, and rows that are not there still have none."""
    sh, q, c, W = plain.problem(1, 1, 1, 2, 128, BF, [(70, 0)], 14)
    sh.sm_scale = 1e-38
    out = plain.decode(sh, q, c, W, F32)
    import numpy as np
    rows = plain.row_values(c.ret_pages.cpu().numpy(), plain.slots_of(c.ret_table[0].cpu().numpy(), 70), 0, 1, 128)
    assert abs(out[0].double().cpu().numpy() - rows.mean(0)).max() <= 2.0 ** -20 * np.abs(rows).mean(0).max()
