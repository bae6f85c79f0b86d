"""Small weights and small query channels in attention over the 4-bit paged cache: a key that takes all the weight and has a value of zero, before
thousands whose weights are e^-8 to e^-18 of it and make the output; a query channel 2^-26 of the largest whose keys make the logits."""
import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
import q4_plain as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _shared(batch, g, d, dtype, rk, rv, q, sm_scale):
    """`batch` sequences that share the pages of rows rk, rv."""
    n = len(rk)
    shape = vec.Shape(batch, 1, g, 1, d, vec.VECTOR_BF16 if dtype == BF else vec.VECTOR_F32, 16, 7, sm_scale, 0, 10000.0)
    pages = -(-n // plain.ROWS)
    pool = np.zeros((pages, 1, 2 * plain.tile_bytes(d)), np.uint8)
    for which, x in ((0, rk), (1, rv)):
        plain.put_rows(pool, np.arange(n), 0, which, x)
        assert np.array_equal(plain.row_values(pool, np.arange(n), 0, which, d), x)          # held exactly
    ints = lambda x: torch.as_tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = ints(np.tile(np.arange(pages), (batch, 1)))
    c = vec.Q4Cache(torch.from_numpy(pool).cuda(), torch.empty(0, 1, plain.tile_bytes(d), dtype=torch.uint8, device="cuda"), table, torch.empty(batch, 0, dtype=torch.int32, device="cuda"),
                    ints(np.full(batch, n)), ints(np.zeros(batch)))
    W = torch.zeros(1, d, d, dtype=dtype, device="cuda")
    return shape, torch.from_numpy(q).to(dtype).cuda().expand(batch, g, d).contiguous(), c, W


def _steps(n, exact):
    """What adding up the sums of 16 rows each loses of n rows' sum."""
    return -(-n // 16) * (2.0 ** -24 if exact else 2.0 ** -23)


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("d,g", [(128, 4), (64, 4), (128, 8), (64, 1)])
@pytest.mark.parametrize("gap", [8, 14, 16, 18])
def test_a_sink_without_a_value(dtype, out_dtype, d, g, gap):
    """Logits come from one channel each and are exact; the factor that makes them exponents of two has two roundings (2^-23 in all), and their difference from the
    reference one: gap 2^-23 each of a weight.  Exponentials 2^-21 twice, weights as vector.h has them (one fp16 part 2^-11, twice; two parts 2^-21, twice), sums of 16 rows 2^-20, of
    n / 16 of these 2^-24 each, twice (2^-23 where they are cut off), and the result's own rounding.  The sink's value is zero, so all of this counts against the tail's sum."""
    n = 3500
    rng = np.random.default_rng(gap)
    rk, rv = np.zeros((n, d)), rng.choice([0.5, 1.0, 1.5, 2.0, 3.0], (n, d))
    rk[1:, 5], rk[:, 4] = -2.0, 3.0                                # a scale of 1/2
    rv[:, ::16] = 3.0                                              # a scale of 1/2 for every group
    rv[0] = 0
    q = np.zeros((g, d))
    q[:, 5] = 1.0
    batch = 1000                                                   # more units than workers would share: most pieces of a sequence are long
    sh, q, c, W = _shared(batch, g, d, dtype, rk, rv, q, gap / 2.0)
    out = plain.decode(sh, q, c, W, out_dtype).double().cpu().numpy()
    p = np.exp(-float(gap))
    o = (p * rv[1:].sum(0) / (1 + (n - 1) * p))[None, None]
    exact = F32 in (dtype, out_dtype)
    tol = (gap * 2.0 ** -23 * 2 + 2.0 ** -20 + (2.0 ** -20 if exact else 2.0 ** -10) + 2.0 ** -20 + 2 * _steps(n, exact) + (2.0 ** -24 if out_dtype == F32 else 2.0 ** -8)) * o
    err = np.abs(out - o)
    assert np.all(err <= tol), float((err / tol).max())


@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("d,g", [(128, 4), (64, 3)])
def test_a_small_query_channel(dtype, out_dtype, d, g):
    """Channel 0 of a query is 2^26 times channel 1, and its keys are zero there: the logits come from channel 1, whose parts keep their bits (fp32: 22, bf16: all 8)."""
    n = 130
    rng = np.random.default_rng(3)
    rk, rv = np.zeros((n, d)), rng.choice([0.5, 1.0, 1.5, 2.0, 3.0], (n, d))
    rk[:, 1], rk[:, 2] = rng.choice([-6.0, -4.0, -3.0, -1.0, 1.0, 2.0, 4.0, 6.0], n) * 8192.0, 6 * 8192.0
    rv[:, ::16] = 3.0
    q = np.zeros((g, d))
    q[:, 0] = 1.25
    small = (1 + rng.integers(0, 1 << 23, g) / 2.0 ** 23) * 2.0 ** -26
    q[:, 1] = torch.from_numpy(small).to(dtype).double().numpy()
    scale = float(np.float32(8.0 / (6 * 8192 * 2.0 ** -26)))        # logits of 8 to 16
    sh, qt, c, W = _shared(2, g, d, dtype, rk, rv, q, scale)
    out = plain.decode(sh, qt, c, W, out_dtype).double().cpu().numpy()
    s = q[:, 1:2] * rk[:, 1][None] * scale
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    o, size = p @ rv, np.abs(s).max(-1, keepdims=True)
    exact = F32 in (dtype, out_dtype)
    # a logit's relative error: 2^-21 where a query is in two parts, 2^-22 from the factor and the product; it counts twice
    tol = (2 * size * 2.0 ** -20 + 2.0 ** -20 + (2.0 ** -20 if exact else 2.0 ** -10) + 2.0 ** -20 + 2 * _steps(n, exact) + (2.0 ** -24 if out_dtype == F32 else 2.0 ** -8)) * o
    err = np.abs(out - o)
    assert np.all(err <= tol), float((err / tol).max())
