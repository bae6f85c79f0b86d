"""Page tables, lengths and slots against the plain form, request by request."""
import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
import q4_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _run(lengths, added, page, table, stack, n_free, n_slots, in_place=False, offset=0):
    ints = lambda n: torch.full((n,), -99, dtype=torch.int32, device=DEV)  # noqa: E731
    on = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)  # noqa: E731
    B = len(lengths)
    L, T, F, n = on(lengths), on(table), on(stack), on([n_free])
    new, left = (L, n) if in_place else (ints(B), ints(1))
    first, start, slots = ints(B), ints(B + 1), ints(n_slots + offset)[offset:]
    vec.vector_block_tables(L, on(added), page, T, F, n, new, left, first, start, slots if n_slots else None)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in (new, first, T, F, left, start, slots)]


def _check(lengths, added, page, table, stack, n_free, n_slots, **kw):
    want = plain.tables(lengths, added, page, table, stack, n_free)
    new, first, T, F, left, start, slots = _run(lengths, added, page, table, stack, n_free, n_slots, **kw)
    assert new.tolist() == want[0] and first.tolist() == want[1] and T.tolist() == want[2] and F.tolist() == want[3]
    assert left.tolist() == [want[4]] and start.tolist() == want[5]
    assert slots.tolist() == (want[6] + [-1] * n_slots)[:n_slots]


def _case(B, most, page, seed, free):
    rng = np.random.default_rng(seed)
    lengths = np.where(rng.random(B) < 0.3, 0, rng.integers(0, most + 1, B))
    what = rng.random(B)
    added = np.where(what < 0.3, 1, np.where(what < 0.5, rng.integers(0, most + 1, B), np.where(what < 0.7, -rng.integers(0, most + 1, B), 0)))
    width = -(-most // page) + 1
    order = rng.permutation(B * width + 5)
    table, at = np.full((B, width), -1), 0
    for b in range(B):
        n = -(-int(lengths[b]) // page)
        table[b, :n] = order[at:at + n]
        at += n
    stack = np.full(B * width + 5, -1)
    n_free = min(free, len(order) - at)
    stack[:n_free] = order[at:at + n_free]
    return lengths, added, page, table, stack, n_free


@pytest.mark.parametrize("B,most,page,free", [(1, 1, 1, 5), (1, 1000, 64, 99), (7, 300, 16, 10**6), (64, 700, 64, 10**6), (64, 700, 64, 40), (300, 40, 7, 10**6), (1024, 100, 64, 10**6),
                                              (1025, 30, 16, 10**6), (3000, 20, 64, 500), (33, 5000, 3, 10**6), (40, 3, 64, 0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_tables(B, most, page, free, in_place):
    for seed in range(2):
        c = _case(B, most, page, seed, free)
        rows = int(np.maximum(c[1], 0).sum())
        for n_slots in {0, rows, rows + 130, max(rows // 2, 1)}:
            _check(*c, n_slots, in_place=in_place)


def test_slots_off_a_16_byte_boundary_and_many_idle_requests():
    c = _case(2000, 4, 64, 3, 10**6)
    added = c[1].copy()
    added[5:1990] = 0
    added[-1] = 5000                                     # more than its table's row holds
    _check(c[0], added, *c[2:], int(np.maximum(added, 0).sum()) + 3, offset=1)


def test_lengths_out_of_range():
    """A negative length counts as none, one beyond the table as a full table; shrinking by more than there is ends a request."""
    table = np.arange(12).reshape(4, 3)
    _check([-5, 100, 20, 7], [3, 4, -2**31, 10**6], 8, table, np.r_[np.arange(20, 25), np.full(20, -1)], 5, 40)


def test_a_captured_step_follows_its_lengths():
    B, page, steps = 5, 4, 11
    lengths = torch.tensor([0, 3, 4, 5, 9], dtype=torch.int32, device=DEV)
    added = torch.tensor([1, 1, 0, 1, -1], dtype=torch.int32, device=DEV)
    table = torch.full((B, 8), -1, dtype=torch.int32, device=DEV)
    host = table.cpu().numpy()
    at = 0
    for b, n in enumerate([0, 3, 4, 5, 9]):
        for i in range(-(-n // page)):
            host[b, i], at = at, at + 1
    table.copy_(torch.from_numpy(host))
    stack = torch.arange(100, 140, dtype=torch.int32, device=DEV)
    n_free = torch.tensor([30], dtype=torch.int32, device=DEV)
    first, start, slots = (torch.empty(n, dtype=torch.int32, device=DEV) for n in (B, B + 1, B))
    state = [lengths.tolist(), table.tolist(), stack.tolist(), 30]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        vec.vector_block_tables(lengths, added, page, table, stack, n_free, lengths, n_free, first, start, slots)
    for _ in range(steps):
        graph.replay()
        torch.cuda.synchronize()
        new, old, t, s, h, st, sl = plain.tables(state[0], added.tolist(), page, state[1], state[2], state[3])
        assert (lengths.tolist(), first.tolist(), table.tolist(), stack.tolist(), n_free.item(), start.tolist(), slots.tolist()) == (new, old, t, s, h, st, (sl + [-1] * B)[:B])
        state = [new, t, s, h]


@pytest.mark.parametrize("B", [6, 1500])
def test_changes_whose_sum_is_beyond_31_bits(B):
    """Requests that ask for all there could be: pages go as far as they go, sums stop at 2^31 - 1."""
    lengths, added = np.zeros(B, int), np.full(B, 2**31 - 1)
    table, stack = np.full((B, 3), -1), np.arange(10)
    new, first, T, F, left, start, slots = _run(lengths, added, 4, table, stack, 10, 40)
    assert new.tolist() == [12, 12, 12, 4] + [0] * (B - 4) and left.tolist() == [0]
    assert T[:4].tolist() == [[9, 8, 7], [6, 5, 4], [3, 2, 1], [0, -1, -1]] and start[:3].tolist() == [0, 2**31 - 1, 2**31 - 1]
    assert slots.tolist() == [p * 4 + r for p in (9, 8, 7) for r in range(4)] + [-1] * 28
