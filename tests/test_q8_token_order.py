"""Several new tokens of the 8-bit cache are [batch][n] rows: the same numbers in the order of a context, [units][n][d], are refused, and the order that is wanted comes from projections directly."""
import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200 import binding
from paper_2605_23258_b200.pipeline import PagedCache

BF = torch.bfloat16


class _OnGpu(torch.Tensor):
    """A tensor that says it is on a GPU: for what the host alone looks at."""
    is_cuda = True

    def get_device(self):
        return 0


def _on(t):
    return t.as_subclass(_OnGpu)


# sequences, layers * heads, tokens: the numbers alike where they can be
SIZES = [(2, 2, 3), (1, 4, 4), (2, 2, 2), (3, 2, 6), (1, 2, 70)]


def _wrong(B, LH, n, device="cpu"):
    x = torch.zeros(B * LH, n, 128, dtype=BF, device=device)
    yield x
    yield x.view(B, LH, n, 128) if LH != n else x
    yield x.view(-1)
    yield torch.zeros(n, B, LH, 128, dtype=BF, device=device) if n != B else x


def _right(B, LH, n, device="cpu"):
    x = torch.zeros(B, n, LH, 128, dtype=BF, device=device)
    return [x, x.flatten(2), x.flatten(0, 1).flatten(1), torch.zeros(B, n, LH * 128 + 8, dtype=BF, device=device)[..., 8:]]


@pytest.mark.parametrize("B,LH,n", SIZES)
def test_the_order_of_a_context_is_refused(monkeypatch, B, LH, n):
    calls = []
    monkeypatch.setattr(binding, "vector_block_tables", lambda *a, **k: calls.append(a))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    paged = PagedCache(vec.Shape(B, 1, LH, LH, 128, vec.VECTOR_BF16, 16), 8, 8, 100, 100, device="cpu", bits=8)
    pos, good = _on(torch.zeros(B, n, dtype=torch.int32)), _on(_right(B, LH, n)[0])
    first = _on(torch.zeros(B, dtype=torch.int32))
    for bad in _wrong(B, LH, n):
        for k, v in ((_on(bad), good), (good, _on(bad))):
            with pytest.raises(ValueError, match=r"must be \["):
                paged.append(k, v, pos)
            with pytest.raises(ValueError, match=r"must be \["):
                vec.vector_append_q8(paged.shape, paged.cache, k, v, first, pos)
    assert not calls
    for x in _right(B, LH, n):
        assert binding._new_rows(paged.shape, n, _on(x), "k_new")[1] == (LH * 128 + 8 if x.stride(-2) % 128 else LH * 128)
    assert binding._new_rows(paged.shape, 1, _on(torch.zeros(B * LH, 128, dtype=BF)), "k_new")[1] == LH * 128                 # one token: both orders are the same


@pytest.mark.gpu
@pytest.mark.parametrize("B,LH,n", SIZES)
def test_the_module_refuses_it_too(B, LH, n):
    c = vec.alloc_q8_cache(vec.Shape(B, 1, LH, LH, 128, vec.VECTOR_BF16, 16), B * 4, 4, 4, 2)
    c.ret_table.copy_(torch.arange(B * 4, dtype=torch.int32).view(B, 4))
    sh, pos, first = vec.Shape(B, 1, LH, LH, 128, vec.VECTOR_BF16, 16), torch.zeros(B, n, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    m, good = binding._marshal(), _right(B, LH, n, "cuda")
    for x in good:
        assert m.append_q8(sh, c, x, good[0], first, pos, False, None) == 0 == m.append_q8(sh, c, good[0], x, first, pos, False, None)
    for x in _wrong(B, LH, n, "cuda"):
        assert m.append_q8(sh, c, x, good[0], first, pos, False, None) is None is m.append_q8(sh, c, good[0], x, first, pos, False, None)
        with pytest.raises(ValueError, match=r"must be \["):
            vec.vector_append_q8(sh, c, x, good[0], first, pos)


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,n", [(3, 2, 5), (2, 4, 4), (1, 2, 40)])
def test_normed_tokens_from_projections(B, H, n):
    """A shape of a sequence a token: the rows that the tokens of longer sequences are, in the order that new rows have."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    shape = lambda batch: vec.Shape(batch, 1, 2 * H, H, 128, vec.VECTOR_BF16, 16, 7, 0.0, 1, 10000.0)  # noqa: E731
    k, v = torch.randn(B, n, 2 * H * 128, generator=gen, device="cuda").to(BF).split(H * 128, dim=-1)
    w, pos = torch.rand(1, 128, generator=gen, device="cuda").to(BF) + 0.5, torch.randint(0, 5000, (B, n), generator=gen, device="cuda", dtype=torch.int32)
    context, tokens = ([torch.empty(*size, 128, dtype=BF, device="cuda") for _ in range(2)] for size in ((B * H, n), (B * n * H, 1)))
    vec.vector_norm_rope(shape(B), n, k=k, v=v, k_out=context[0], v_out=context[1], k_weight=w, pos=pos)
    vec.vector_norm_rope(shape(B * n), 1, k=k, v=v, k_out=tokens[0], v_out=tokens[1], k_weight=w, pos=pos)
    paged = PagedCache(shape(B), 8, 8, 100, 100, bits=8)
    paged.active.fill_(1)
    paged.append(*(t.view(B, n, H * 128) for t in tokens), pos)
    got = [torch.empty(B * H, n, 128, dtype=BF, device="cuda") for _ in range(2)]
    vec.vector_read_q8(shape(B), paged.cache, *got)
    for t, c, g in zip(tokens, context, got):
        c = c.view(B, H, n, 128).transpose(1, 2)
        assert torch.equal(t.view(B, n, H, 128), c)
        c, g = c.double().cpu().numpy(), g.view(B, H, n, 128).transpose(1, 2).double().cpu().numpy()
        assert np.all(np.abs(g - c) <= 2.0 ** -4 * np.abs(c) + 2.0 ** -10 * np.abs(c).max())           # half a step of e4m3; below 2^-6 of a scale of at most max / 224, half of 2^-9 of it
