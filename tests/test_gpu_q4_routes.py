"""The five calls of the 4-bit paged cache through ctypes: the same kernels, results and refusals as through the extension module."""
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200 import binding as B
import q4_plain as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"


class _Nothing:
    """Leaves every call to ctypes."""

    def __getattr__(self, name):
        return lambda *args: None



def _step(d, dtype, rope, stream):
    """Tables, compaction, append, reading back and attention of two sequences; everything that they write."""
    gen = torch.Generator(device=DEV).manual_seed(7)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(dtype)  # noqa: E731
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    sh = vec.Shape(2, 1, 4, 2, d, vec.VECTOR_BF16 if dtype == torch.bfloat16 else vec.VECTOR_F32, 16, 7, 0.0, int(rope), 10000.0)
    budget = vec.vector_plan_budget(300, 120, -1, 16)
    c = vec.alloc_q4_cache(sh, 8, 9, 4, 4)
    for t in (c.ret_pages, c.apx_pages, c.ret_pos, c.apx_pos):
        t.zero_()
    K, V, W, q, k, v = rand(4, 300, d), rand(4, 300, d), rand(2, d, d), rand(4, 2, d), rand(4, d), rand(4, d)
    idx = torch.argsort(torch.rand(4, 300, generator=gen, device=DEV), 1).int()
    ret, apx = (x.sort(1).values.contiguous() for x in (idx[:, :budget.n_ret], idx[:, budget.n_ret:budget.n_ret + budget.n_apx]))
    got = [c.ret_pages, c.apx_pages, c.ret_pos, c.apx_pos]
    slots = {}
    for tier, n, pages, table, length in (("ret", budget.n_ret, 8, c.ret_table, c.ret_len), ("apx", budget.n_apx, 9, c.apx_table, c.apx_len)):
        slots[tier] = ints(2, n)
        free, left, first, start = torch.arange(pages, dtype=torch.int32, device=DEV), ints(1) + pages, ints(2), ints(3)
        vec.vector_block_tables(length, ints(2) + n, 64, table, free, left, length, left, first, start, slots[tier], stream)
        got += [table, length, left, first, start, slots[tier]]
    vec.vector_compact_q4(sh, budget, K, V, ret, apx, c, slots["ret"], slots["apx"], stream)
    at = torch.tensor([5 * 64 + 3, 1], dtype=torch.int32, device=DEV)
    vec.vector_append_q4(sh, c, k, v, None, at, ints(2) + 300, stream)
    rows = [torch.empty(4, n, d, dtype=dtype, device=DEV) for n in (budget.n_ret, budget.n_ret, budget.n_apx)]
    vec.vector_read_q4(sh, c, slots["ret"], rows[0], rows[1], slots["apx"], rows[2], stream)
    out = torch.empty(4, 2, d, dtype=torch.float32, device=DEV)
    vec.vector_decode_attn_q4(sh, q, c, W, out, torch.empty(vec.vector_decode_q4_workspace_bytes(sh), dtype=torch.uint8, device=DEV), stream)
    torch.cuda.synchronize()
    return got + rows + [out]


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("d,dtype,rope", [(128, torch.bfloat16, False), (64, torch.float32, False), (64, torch.bfloat16, True)])
def test_a_step_by_either_route(monkeypatch, d, dtype, rope, given):
    stream = torch.cuda.current_stream() if given else None
    with monkeypatch.context() as m:
        m.setattr(B, "_marshal_module", _Nothing())
        before = vec.vector_kernel_launches()
        want = _step(d, dtype, rope, stream)
        launches = vec.vector_kernel_launches() - before
    before = vec.vector_kernel_launches()
    got = _step(d, dtype, rope, stream)
    assert vec.vector_kernel_launches() - before == launches
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    if B.marshal_path() and type(B._marshal()).__name__ == "module":
        module = B._marshal()
        taken = {name: 0 for name in ("block_tables", "compact_q4", "append_q4", "read_q4", "decode_attn_q4")}

        class Counting:
            def __getattr__(self, name):
                def call(*args):
                    rc = getattr(module, name)(*args)
                    taken[name] += rc is not None
                    return rc
                return call
        with monkeypatch.context() as m:
            m.setattr(B, "_marshal_module", Counting())
            _step(d, dtype, rope, stream)
        assert taken == {"block_tables": 2, "compact_q4": 1, "append_q4": 1, "read_q4": 1, "decode_attn_q4": 1}


def test_ctypes_refuses_the_same(monkeypatch):
    sh, q, c, W = plain.problem(2, 1, 2, 2, 64, torch.bfloat16, [(100, 80), (70, 10)], 5)
    out, ws = torch.empty(4, 2, 64, dtype=torch.bfloat16, device=DEV), torch.empty(vec.vector_decode_q4_workspace_bytes(sh), dtype=torch.uint8, device=DEV)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)  # noqa: E731
    monkeypatch.setattr(B, "_marshal_module", _Nothing())
    short = vec.Q4Cache(c.ret_pages[:, :, :-8].contiguous(), *[getattr(c, n) for n in ("apx_pages", "ret_table", "apx_table", "ret_len", "apx_len")])
    for args in ((sh, q[:2], c, W, out), (sh, q, c, W[:1], out), (sh, q, short, W, out), (sh, q, c, W, out[:3]), (sh, q.float(), c, W, out)):
        with pytest.raises(ValueError):
            vec.vector_decode_attn_q4(*args, ws)
    for w in (None, ws[:64]):
        with pytest.raises(vec.VectorError) as e:
            vec.vector_decode_attn_q4(sh, q, c, W, out, w)
        assert e.value.status == -5
    with pytest.raises(ValueError):
        vec.vector_block_tables(ints(2), ints(2), 64, c.ret_table, ints(4), ints(1), ints(1), ints(1), ints(2), ints(3))
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        vec.vector_append_q4(sh, c, x[:3], x, None, ints(2), ints(2))
    with pytest.raises(vec.VectorError):
        vec.vector_append_q4(sh, c, x, x, None, ints(1), ints(2))
    with pytest.raises(ValueError):
        vec.vector_read_q4(sh, c, ints(2, 3), torch.empty(4, 2, 64, dtype=torch.bfloat16, device=DEV), torch.empty(4, 3, 64, dtype=torch.bfloat16, device=DEV))
