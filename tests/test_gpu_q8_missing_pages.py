"""A sequence of the 8-bit cache with a negative retained length, and a key-only length beyond its table whose entries name no page but one: attention is over that page's rows alone."""
import pytest
import torch

import paper_2605_23258_b200 as vec
import q8_plain as plain

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("dtype,out_dtype", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block", [1, 4, 10])                                         # of the table, its last one too
def test_one_page_of_a_length_beyond_the_table(d, dtype, out_dtype, rope, block):
    sh, q, c, W = plain.problem(3, 1, 2, 4, d, dtype, [(200, 300), (100, 100), (70, 10)], 8, rope)
    assert c.apx_table.shape[1] == 11
    full, other = c.apx_table[0, 0].item(), c.apx_table[1, 2].item()                  # 32 rows of each are written
    c.ret_len[2], c.apx_len[2] = -5, 1000
    c.apx_table[2, :] = torch.tensor([-3, c.apx_pages.shape[0], 2**31 - 1] * 4, dtype=torch.int32)[:11]
    c.apx_table[2, block] = full
    out = plain.decode(sh, q, c, W, out_dtype)
    plain.check_decode(sh, q, c, W, out, rope, [4, 5], ret_rows=[], apx_rows=range(32 * block, 32 * block + 32))
    plain.check_decode(sh, q, c, W, out, rope, [0, 1, 2, 3])                          # the others do not notice
    c.apx_table[2, 0 if block else 1] = other                                         # and of two
    out = plain.decode(sh, q, c, W, out_dtype)
    plain.check_decode(sh, q, c, W, out, rope, [4, 5], ret_rows=[], apx_rows=[*range(32), *range(32 * block, 32 * block + 32)])
    assert vec.vector_device_fault() == 0
