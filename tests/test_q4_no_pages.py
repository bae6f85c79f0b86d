"""A stack that never has a free page: no memory is its memory, as an empty tensor's is."""
import pytest
import torch

import paper_2605_23258_b200 as vec


def test_no_stack_is_no_null_pointer():
    """Told from a missing one by its capacity; the refusal that is left is the batch's."""
    def call(free, cap):
        P = 4096
        return vec.load_library().vector_block_tables(0, P, P, 64, P, 4, free, cap, P, P, P, P, P, P, 4, None)
    assert call(None, 0) == -2 and call(None, 1) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [3, 1500])
def test_requests_get_no_rows(batch):
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    lengths, added, table, left, first, start, slots = ints(batch), ints(batch) + 2, ints(batch, 2) - 1, ints(1), ints(batch), ints(batch + 1), ints(2 * batch)
    lengths[0], added[0], table[0, 0] = 3, -3, 7                                     # a page that comes back finds no place either
    lengths[1], table[1, 0] = 62, 9                                                  # and rows that need no new page are there
    vec.vector_block_tables(lengths, added, 64, table, ints(0), left, lengths, left, first, start, slots)
    torch.cuda.synchronize()
    assert lengths[:3].tolist() == [0, 64, 0] and not lengths[2:].any() and left.item() == 0 and start[:3].tolist() == [0, 0, 2]
    assert slots[:4].tolist() == [9 * 64 + 62, 9 * 64 + 63, -1, -1] and (slots[2:] == -1).all()
