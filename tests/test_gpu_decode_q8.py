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
