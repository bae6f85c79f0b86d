"""A token's own index is no position of a generated token: PagedCache.project needs positions where keys are turned by them."""
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200 import binding
from paper_2605_23258_b200.pipeline import PagedCache


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rope", [0, 1])
def test_positions_of_generated_tokens(monkeypatch, rope, bits):
    calls = []
    monkeypatch.setattr(binding, "vector_norm_rope", lambda *a: calls.append(a))
    paged = PagedCache(vec.Shape(3, 1, 4, 2, 64, vec.VECTOR_F32, 16, 7, 0.0, rope), 8, 8, 100, 100, device="cpu", bits=bits)
    q, k, v, w = torch.zeros(3, 1, 256), torch.zeros(3, 1, 128), torch.zeros(3, 1, 128), torch.ones(1, 64)
    if rope:
        for weights in ((), (w, w)):
            with pytest.raises(ValueError, match="pos"):
                paged.project(q, k, v, *weights)
        assert not calls
    else:
        paged.project(q, k, v, w, w)                            # no positions, none needed
    got = paged.project(q, k, v, w, w, torch.zeros(3, 1, dtype=torch.int32))
    assert len(calls) == 2 - rope and [tuple(t.shape) for t in got] == [(6, 2, 64), (6, 64), (6, 64)]
