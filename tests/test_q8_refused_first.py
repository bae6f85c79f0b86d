"""What an 8-bit paged cache refuses, it refuses before its tables change: lengths that had grown would count rows that nobody wrote."""
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200 import binding
from paper_2605_23258_b200.pipeline import Compressor, PagedCache

BF = torch.bfloat16


class _OnGpu(torch.Tensor):
    """A tensor that says it is on a GPU: for what the host alone looks at."""
    is_cuda = True

    def get_device(self):
        return getattr(self, "at", 0)


def _on(t, device=0):
    t = t.as_subclass(_OnGpu)
    t.at = device
    return t


@pytest.fixture
def changes(monkeypatch):
    """The calls that would have changed the tables; nothing runs on a GPU."""
    calls = []
    monkeypatch.setattr(binding, "vector_block_tables", lambda *a, **k: calls.append(a))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return calls


def _paged(batch=2, rope=0):
    return PagedCache(vec.Shape(batch, 1, 4, 2, 128, vec.VECTOR_BF16, 16, 7, 0.0, rope), 8, 8, 100, 100, device="cpu", bits=8)


@pytest.mark.parametrize("which", ["k_new", "v_new", "pos"])
def test_new_rows_of_another_device(changes, which):
    given = dict(k_new=torch.zeros(2, 3, 256, dtype=BF), v_new=torch.zeros(2, 3, 256, dtype=BF), pos=torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError, match="device"):
        _paged().append(**{name: _on(t, int(name == which)) for name, t in given.items()})
    assert not changes


@pytest.mark.parametrize("rows", [lambda: torch.zeros(256, dtype=BF).expand(1, 3, 256), lambda: torch.zeros(1024, dtype=BF).as_strided((1, 3, 256), (768, 128, 1))])
def test_new_rows_that_overlap(changes, rows):
    x, pos = _on(rows()), _on(torch.zeros(1, 3, dtype=torch.int32))
    for k, v in ((x, _on(torch.zeros(1, 3, 256, dtype=BF))), (_on(torch.zeros(1, 3, 256, dtype=BF)), x)):
        with pytest.raises(ValueError, match="apart"):
            _paged(1).append(k, v, pos)
    assert not changes


@pytest.mark.parametrize("which", ["K", "V", "ret_idx", "apx_idx"])
def test_a_context_of_another_device(changes, which):
    paged, one = _paged(), vec.Shape(1, 1, 4, 2, 128, vec.VECTOR_BF16, 16)
    comp = Compressor(one, vec.vector_plan_budget(150, 60, -1, 16), device="cpu")
    at = lambda name, t: _on(t, int(name == which))  # noqa: E731
    K, V = (at(name, torch.zeros(2, 150, 128, dtype=BF)) for name in ("K", "V"))
    comp.ret_idx, comp.apx_idx = at("ret_idx", comp.ret_idx), at("apx_idx", comp.apx_idx)
    with pytest.raises(ValueError, match="device"):
        paged.admit(0, comp, K, V)
    assert not changes and not paged._taken


@pytest.mark.gpu
def test_lengths_and_pages_are_as_they_were():
    """Broadcast and overlapping rows of one sequence and of two."""
    for batch in (1, 2):
        paged = PagedCache(vec.Shape(batch, 1, 4, 2, 128, vec.VECTOR_BF16, 16), 8, 8, 100, 100, bits=8)
        paged.active.fill_(1)
        dense, pos = torch.zeros(batch, 3, 256, dtype=BF, device="cuda"), torch.zeros(batch, 3, dtype=torch.int32, device="cuda")
        for bad in (dense[:, :1].expand(batch, 3, 256), dense[:1, :1].expand(batch, 3, 256), torch.zeros(4096, dtype=BF, device="cuda").as_strided((batch, 3, 256), (384, 128, 1))):
            for k, v in ((bad, dense), (dense, bad)):
                with pytest.raises(ValueError):
                    paged.append(k, v, pos)
        assert not paged.cache.ret_len.any() and paged.free_pages() == (8, 8)
        paged.append(dense, dense, pos)
        assert paged.cache.ret_len.tolist() == [3] * batch and paged.free_pages() == (8 - batch, 8)


def test_a_cache_of_another_device(changes):
    """The current device is another one than the cache's, whose tensors were made together."""
    paged = _paged()
    paged.cache.ret_pages = _on(paged.cache.ret_pages, 1)
    x, pos = _on(torch.zeros(2, 3, 256, dtype=BF)), _on(torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError, match="device"):
        paged.append(x, x, pos)
    comp = Compressor(vec.Shape(1, 1, 4, 2, 128, vec.VECTOR_BF16, 16), vec.vector_plan_budget(150, 60, -1, 16), device="cpu")
    with pytest.raises(ValueError, match="device"):
        paged.admit(0, comp, *(_on(torch.zeros(2, 150, 128, dtype=BF)) for _ in range(2)))
    assert not changes
