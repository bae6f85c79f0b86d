"""Logits far beyond fp32's last whole number, in attention over the 4-bit paged cache: the reference is rounded, and a weight against it may be any power of two."""
import numpy as np
import pytest
import torch

import q4_plain as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("d,g", [(128, 4), (64, 7)])
def test_one_key_is_picked_at_every_size(dtype, out_dtype, d, g, rope):
    """Retained keys, logits of 2^20 to 2^40: the largest is ahead by far more than fp32's resolution there, so that the output is its value row (a weight is one or zero;
    the result's own rounding and 2^-20 of sums)."""
    n = 4 * 64 + 9
    sh, q, c, W = plain.problem(1, 1, 1, g, d, dtype, [(n, 0)], 51, rope)
    slots = plain.slots_of(c.ret_table[0].cpu().numpy(), n)
    keys, rows = (plain.row_values(c.ret_pages.cpu().numpy(), slots, 0, w, d) for w in (0, 1))
    own, compared = 2.0 ** -24 if out_dtype == F32 else 2.0 ** -8, 0
    for e in range(20, 41):
        for step in (1.0, 1.3, 1.7):
            scaled = (q * (step * 2.0 ** e / 8)).to(dtype)
            s = scaled[0].double().cpu().numpy() @ keys.T
            two = np.sort(s, -1)[:, -2:]
            ahead = two[:, 1] - two[:, 0] > 1e-4 * np.abs(s).max()              # a thousand times 2^-23
            best = rows[s.argmax(-1)]
            out = plain.decode(sh, scaled, c, W, out_dtype).double().cpu().numpy()[0]
            err = np.abs(out - best)[ahead]
            assert np.all(err <= (own + 2.0 ** -20) * np.abs(best[ahead])), (e, step, err.max())
            assert np.all(np.isfinite(out)), (e, step)
            compared += int(ahead.sum())
    assert compared > 21 * 3 * g // 2


@pytest.mark.parametrize("out_dtype", [BF, F32])
def test_logits_beyond_fp32_are_no_numbers(out_dtype):
    """Finite queries whose largest logit is infinite in fp32: NaN, as infinity less infinity is, in the piece of the sequence that has it and so in the whole."""
    sh, q, c, W = plain.problem(1, 1, 1, 2, 128, BF, [(64 * 40, 0)], 52)
    pool = c.ret_pages.cpu().numpy()
    slots = plain.slots_of(c.ret_table[0].cpu().numpy(), 64 * 40)
    for row in (5, 700):
        plain.put_rows(pool, slots[row:row + 1], 0, 0, np.full((1, 128), 61440.0))
    c.ret_pages.copy_(torch.from_numpy(pool))
    q[0, 0] = 1e38
    out = plain.decode(sh, q, c, W, out_dtype)
    assert torch.isnan(out[0, 0]).all() and torch.isfinite(out[0, 1]).all()
