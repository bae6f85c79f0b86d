"""What PagedCache.admit refuses, and an admission that does not fit: nothing is taken, and the other requests do not notice."""
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200.pipeline import Compressor, PagedCache

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = 64


def _shape(batch, **kw):
    return vec.Shape(**{**dict(batch=batch, n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=D, dtype=vec.VECTOR_BF16, window=16), **kw})


def _context(N, pairs, n_a=-1, seed=0, **kw):
    """A routed context: its Compressor, keys and values."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV).bfloat16()  # noqa: E731
    sh = _shape(1, **kw)
    comp = Compressor(sh, vec.vector_plan_budget(N, pairs, n_a, 16))
    K, V = rand(2, N, sh.head_dim), rand(2, N, sh.head_dim)
    comp.score(rand(2, sh.group, 16, sh.head_dim), K)
    comp.route(K, V, rand(2, sh.head_dim, sh.head_dim) / 8)
    return comp, K, V


def _state(p):
    """Everything that tells who holds what."""
    c = p.cache
    return [t.cpu().clone() for t in (c.ret_len, c.apx_len, p.n_ret_free, p.n_apx_free, p.active)]


def _held(p):
    """The pages that the tables name for their sequences, tier by tier."""
    out = []
    for table, length in ((p.cache.ret_table, p.cache.ret_len), (p.cache.apx_table, p.cache.apx_len)):
        out.append([int(x) for b in range(len(length)) for x in table[b, :-(-int(length[b]) // 64)]])
    return out


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("ret_pages,apx_pages", [(3, 9), (9, 5)])
def test_too_few_pages_are_left(ret_pages, apx_pages):
    """Two pages of retained and four of key-only rows a request: in either pool there is room for one only."""
    p = PagedCache(_shape(3), ret_pages, apx_pages, 512, 512)
    first, second = (_context(400, 200, seed=i) for i in (1, 2))
    assert first[0].budget.n_ret == 100 and first[0].budget.n_apx == 200
    assert bool(p.admit(0, *first)) is True
    q, W, out = torch.randn(6, 2, D, device=DEV).bfloat16(), torch.randn(2, D, D, device=DEV).bfloat16(), torch.empty(6, 2, D, device=DEV)
    before, alone = _state(p), p.decode(q, W, out).clone()
    assert bool(p.admit(2, *second)) is False
    assert _same(_state(p), before) and torch.equal(p.decode(q, W, out), alone) and not out[4:].any()
    p.append(torch.randn(6, D, device=DEV).bfloat16(), torch.randn(6, D, device=DEV).bfloat16(), torch.zeros(3, dtype=torch.int32, device=DEV))
    assert p.cache.ret_len.tolist() == [101, 0, 0]
    p.end(2)
    p.end(0)
    assert p.free_pages() == (ret_pages, apx_pages)
    assert bool(p.admit(2, *second)) is True
    assert p.cache.ret_len.tolist() == [0, 0, 100] and p.cache.apx_len.tolist() == [0, 0, 200]
    assert p.active.tolist() == [0, 0, 1] and p.decode(q, W, out)[4:].any()
    for pages, n in zip(_held(p), (2, 4)):
        assert len(set(pages)) == len(pages) == n


def test_what_the_host_knows_is_refused():
    """Before anything changes: contexts longer than a place or a pool, a taken place, none, other models' compressors, rows that compaction refuses."""
    p = PagedCache(_shape(2), 4, 8, 200, 300)
    comp, K, V = _context(400, 200)
    p.admit(0, comp, K, V)
    before = _state(p)
    wide, far = _context(700, 300, 20), _context(900, 400, 170)           # 280 retained rows; 230, and 340 key-only ones
    assert wide[0].budget.n_ret == 280 and far[0].budget.n_ret == 230 and far[0].budget.n_apx == 340
    for args, what in (((1, *wide), "retained"), ((1, *far), "key-only"), ((0, comp, K, V), "place"), ((1, *_context(400, 200, n_q_heads=8)), "layers and heads"),
                       ((1, *_context(400, 200, rope_enabled=1)), "rotary"), ((1, comp, K[:1], V), "K"), ((1, comp, K, V.float()), "V"), ((1, comp, K.cpu(), V), "K"),
                       ((1, comp, K.transpose(0, 1), V), "K"), ((1, comp, torch.empty(K.numel() + 1, dtype=K.dtype, device=DEV)[1:].view(K.shape), V), "K"),
                       ((1, _context(500, 240, 160 // 2 + 1)[0], K, V), "K")):
        with pytest.raises(ValueError, match=what):
            p.admit(*args)
        assert _same(_state(p), before), what
    for place in (2, -3):
        with pytest.raises(IndexError):
            p.admit(place, comp, K, V)
        with pytest.raises(IndexError):
            p.end(place)
        assert _same(_state(p), before)
    small = PagedCache(_shape(2), 1, 8, 200, 300)
    with pytest.raises(ValueError, match="pool"):
        small.admit(0, comp, K, V)
    assert bool(p.admit(-1, comp, K, V)) and p.cache.ret_len.tolist() == [100, 100]
    p.end(-1, 0)
    assert p.free_pages() == (4, 8) and not p.active.any()
    assert bool(p.admit(1, comp, K, V))


def test_rotary_bases_and_positions():
    p = PagedCache(_shape(2, rope_enabled=1, rope_theta=5e5), 4, 8, 200, 300)
    with pytest.raises(ValueError, match="rotary"):
        p.admit(0, *_context(400, 200, rope_enabled=1, rope_theta=1e4))
    assert bool(p.admit(0, *_context(400, 200, rope_enabled=1, rope_theta=5e5)))
    with pytest.raises(ValueError, match="positions"):
        PagedCache(_shape(2, rope_enabled=1), 4, 8, 200, 300, positions=False)


@pytest.mark.parametrize("rope", [0, 1])
def test_no_key_only_rows_and_no_pages_for_them(rope):
    """A budget that approximates nothing, over a cache without key-only pages."""
    p = PagedCache(_shape(2, rope_enabled=rope), 6, 0, 300, 0)
    comp, K, V = _context(400, 130, 0, rope_enabled=rope)
    assert comp.budget.n_apx == 0
    assert bool(p.admit(1, comp, K, V))
    q, W = torch.randn(4, 2, D, device=DEV).bfloat16(), torch.randn(2, D, D, device=DEV).bfloat16()
    out = p.decode(q, W, torch.empty(4, 2, D, device=DEV))
    assert torch.isfinite(out).all() and out[2:].any() and not out[:2].any()
    with pytest.raises(ValueError, match="key-only|pool"):
        p.admit(0, *_context(400, 200, rope_enabled=rope))
    assert p.free_pages() == (3, 0)
    p.end(0, 1)
    assert p.free_pages() == (6, 0)
