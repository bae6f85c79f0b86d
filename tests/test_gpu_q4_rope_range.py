"""Rotary keys of the 4-bit paged cache at the ends of what is stored and of the positions: channels of 61440, whose pairs turn to 86889, and far tokens."""
import numpy as np
import pytest
import torch

import q4_plain as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("d,g", [(128, 2), (64, 2), (128, 8), (64, 5)])
def test_the_largest_stored_keys(dtype, out_dtype, d, g):
    """A key of 61440 in every channel: the even heads attend to it alone, for the odd ones its weight is zero, and whatever it turns to has no part
    in their sums.  No logit term in the tolerance of the even heads: the weights are one and zero, 1e5 apart."""
    at = 37
    sh, q, c, W = plain.problem(2, 1, 1, g, d, dtype, [(70, 130), (10, 90)], 31, rope=True)
    pool, table = c.apx_pages.cpu().numpy(), c.apx_table.cpu().numpy()
    plain.put_rows(pool, plain.slots_of(table[0], 130)[at:at + 1], 0, 0, np.full((1, d), 61440.0))
    c.apx_pages.copy_(torch.from_numpy(pool))
    c.apx_pos[int(table[0, 0]), 0, at] = 7854                                      # slow channels: an eighth of a turn
    q[0] = q[0].abs()
    q[0, 1::2] *= -1
    out = plain.decode(sh, q, c, W, out_dtype)
    plain.check_decode(sh, q, c, W, out, True, [1])
    n, m = 70, 130
    rs, as_ = plain.slots_of(c.ret_table[0].cpu().numpy(), n), plain.slots_of(table[0], m)
    rk, rv = (plain.row_values(c.ret_pages.cpu().numpy(), rs, 0, w, d) for w in (0, 1))
    ak, pos = plain.row_values(pool, as_, 0, 0, d), c.apx_pos.cpu().numpy()[as_ // 64, 0, as_ % 64]
    rest = np.arange(m) != at
    for heads, rows in ((slice(0, None, 2), slice(at, at + 1)), (slice(1, None, 2), rest)):
        none = np.zeros((0, d))
        o, spread, logit, turned = plain.attend(q[0, heads].double().cpu().numpy(), none if heads.start == 0 else rk, none if heads.start == 0 else rv, ak[rows],
                                                W[0].double().cpu().numpy(), d ** -0.5, pos[rows])
        tol = plain.tolerance(o, spread, logit * heads.start, turned, dtype, out_dtype, True)
        err = np.abs(out[0, heads].double().cpu().numpy() - o)
        assert np.all(np.isfinite(err)) and np.all(err <= tol), (heads.start, float((err / tol).max()))


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("d,g,top", [(128, 4, 1 << 20), (64, 3, 1 << 30), (128, 2, 1 << 30)])
def test_far_positions(dtype, out_dtype, d, g, top):
    """Positions up to 2^30: the tolerance is that of near ones."""
    sh, q, c, W = plain.problem(2, 1, 1, g, d, dtype, [(0, 200), (90, 65)], 32, rope=True)
    c.apx_pos.copy_(torch.randint(top // 2, top, c.apx_pos.shape, generator=torch.Generator().manual_seed(1), dtype=torch.int32))
    plain.check_decode(sh, q, c, W, plain.decode(sh, q, c, W, out_dtype), True)


@pytest.mark.parametrize("dtype,out_dtype", [(BF, F32), (F32, F32)])
@pytest.mark.parametrize("d,g,size", [(128, 4, 2.0 ** -7), (64, 4, 2.0 ** -12), (128, 8, 2.0 ** -12), (64, 6, 2.0 ** -7)])
def test_small_keys_keep_their_parts(dtype, out_dtype, d, g, size):
    """Keys far below one under fp32 results: a turned one has 22 bits (the tolerance is relative to its size)."""
    sh, q, c, W = plain.problem(2, 1, 1, g, d, dtype, [(0, 150), (0, 65)], 33, rope=True)
    pool, table = c.apx_pages.cpu().numpy(), c.apx_table.cpu().numpy()
    rng = np.random.default_rng(5)
    for b, n in ((0, 150), (1, 65)):
        plain.put_rows(pool, plain.slots_of(table[b], n), 0, 0, rng.standard_normal((n, d)) * size)
    c.apx_pages.copy_(torch.from_numpy(pool))
    plain.check_decode(sh, q, c, W, plain.decode(sh, q, c, W, out_dtype), True)
