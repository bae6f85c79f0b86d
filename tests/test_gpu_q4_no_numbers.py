"""Queries, keys and values that are no numbers, in attention over the 4-bit paged cache: what they reach is NaN, wherever the rows of a sequence
are cut into workers' pieces, and nothing else is."""
import numpy as np
import pytest
import torch

import q4_plain as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
TYPES = [(BF, BF), (BF, F32), (F32, F32)]


def _spoil(c, tier, d, b, row, which=0):
    """Scales of 255 for a stored row: each of its channels reads as NaN."""
    table, pages = (c.ret_table, c.ret_pages) if tier == "ret" else (c.apx_table, c.apx_pages)
    at = which * plain.tile_bytes(d) + plain.ROWS * d // 2 + row % plain.ROWS * (d // 16)
    pages[int(table[b, row // plain.ROWS]), :, at:at + d // 16] = 255


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("d,g,value", [(128, 3, float("nan")), (64, 2, float("nan")), (128, 8, float("nan")), (128, 3, float("inf")), (64, 5, float("-inf"))])
def test_a_query_that_is_none(dtype, out_dtype, d, g, value, rope):
    sh, q, c, W = plain.problem(3, 1, 1, g, d, dtype, [(70, 130), (3, 0), (0, 65)], 41, rope)
    q[:, 1, d // 2 + 3] = value
    out = plain.decode(sh, q, c, W, out_dtype)
    assert torch.isnan(out[:, 1]).all()
    rest = [h for h in range(g) if h != 1]
    for u in range(3):
        with np.errstate(invalid="ignore"):
            o, *sizes = plain.expected(sh, q, c, W, u, 0, rope)
            tol = plain.tolerance(o, *sizes, dtype, out_dtype, rope)
        assert np.all(np.abs(out[u].double().cpu().numpy() - o)[rest] <= tol[rest]), u


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("tier,lengths,row", [("ret", (1, 0), 0), ("apx", (0, 1), 0), ("ret", (65, 0), 64), ("ret", (129, 200), 128), ("apx", (10, 65), 64), ("apx", (300, 64), 63),
                                              ("ret", (64, 64), 0), ("apx", (0, 1281), 1280)])
def test_a_key_that_is_none(dtype, out_dtype, tier, lengths, row, rope):
    """Alone in its sequence, alone in the last page, or among others."""
    sh, q, c, W = plain.problem(2, 1, 1, 4, 128, dtype, [lengths, (70, 70)], 42, rope)
    _spoil(c, tier, 128, 0, row)
    out = plain.decode(sh, q, c, W, out_dtype)
    assert torch.isnan(out[0]).all()
    plain.check_decode(sh, q, c, W, out, rope, [1])


@pytest.mark.parametrize("dtype,out_dtype", TYPES)
@pytest.mark.parametrize("page", [0, 1, 4])
def test_a_value_that_is_none_and_weighs_nothing(dtype, out_dtype, page):
    """Its page's logits lie thousands below the others': the product is NaN all the same, whether or not the page is a worker's only one."""
    d, n = 128, 5 * 64
    sh, q, c, W = plain.problem(1, 1, 1, 2, d, dtype, [(n, 0)], 43)
    q[0, 1] = q[0, 0]
    pool = c.ret_pages.cpu().numpy()
    slots = plain.slots_of(c.ret_table[0].cpu().numpy(), n)
    u = q[0, 0].double().cpu().numpy()
    plain.put_rows(pool, slots[64 * page:64 * page + 64], 0, 0, np.tile(-4000 * u, (64, 1)))
    c.ret_pages.copy_(torch.from_numpy(pool))
    assert torch.isfinite(plain.decode(sh, q, c, W, out_dtype)).all()
    _spoil(c, "ret", d, 0, 64 * page + 7, 1)
    assert torch.isnan(plain.decode(sh, q, c, W, out_dtype)).all()


def test_rows_that_are_not_there_stay_zeros():
    """A sequence of no rows, and one whose table names no page, beside one with a NaN."""
    sh, q, c, W = plain.problem(3, 1, 2, 3, 64, BF, [(0, 0), (100, 70), (64, 1)], 44)
    c.ret_table[1], c.apx_table[1] = -1, 1 << 20
    _spoil(c, "apx", 64, 2, 0)
    out = plain.decode(sh, q, c, W, BF)
    assert not out[:4].any() and torch.isnan(out[4:]).all()
