"""CPU checks of the 4-bit paged cache: the plain form that the GPU tests compare with, sizes, and what the entry points refuse."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
import q4_plain as plain

BF, F32 = vec.VECTOR_BF16, vec.VECTOR_F32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2605_23258_b200.build import build
    build()


def test_plain_rounding_is_the_nearest_code():
    x = np.array([[0, 0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, -0.25, -0.75, -2.5, -5, -5.0001, 0.1]])
    codes, scales = plain.encode(x)
    assert scales[0, 0] == 15 << 3                                                            # 6 = 6 s: s = 1
    assert plain.values(codes, scales)[0].tolist() == [0, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, 0, -1, -2, -4, -6, 0]
    for most, s in ((6.0001, 1.125), (1e-9, 2.0 ** -17), (7e4, 10240.0), (np.inf, 10240.0), (2.0 ** -17 * 6, 2.0 ** -17)):
        assert plain.scale_value(plain.encode(np.array([[most] + [0] * 15]))[1])[0, 0] == s
    assert np.isnan(plain.rounded(np.array([[np.nan] + [6] * 31]))[0, :16]).all() and (plain.rounded(np.array([[np.nan] + [6] * 31]))[0, 16:] == 6).all()
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 64)) * np.exp(rng.uniform(-8, 6, (200, 1)))
    got = plain.rounded(x).reshape(-1, 16)
    s = plain.scale_value(plain.encode(x)[1]).reshape(-1, 1)
    size = np.abs(x.reshape(-1, 16))
    step = np.where(size <= 2 * s, 0.5, np.where(size <= 4 * s, 1, 2)) * s            # between the codes on either side of x
    assert np.all(np.abs(got - x.reshape(-1, 16)) <= step / 2 * (1 + 1e-12))


@pytest.mark.parametrize("d", [64, 128])
def test_plain_layout_is_a_permutation(d):
    byte, shift, scale = plain.places(d)
    assert sorted(zip(byte.tolist(), shift.tolist())) == [(i // 2, 4 * (i % 2)) for i in range(d)] and sorted(scale.tolist()) == list(range(d // 16))
    pages = np.zeros((3, 2, 2 * plain.tile_bytes(d)), np.uint8)
    x = np.random.default_rng(1).standard_normal((5, d))
    plain.put_rows(pages, [0, 63, 64, 100, 191], 1, 1, x)
    assert np.array_equal(plain.row_values(pages, [0, 63, 64, 100, 191], 1, 1, d), plain.rounded(x)) and not pages[:, 0].any()


def test_tile_bytes():
    for d, n in ((64, 2304), (128, 4608)):
        sh = vec.Shape(1, 1, 1, 1, d, BF, 16)
        assert vec.vector_q4_tile_bytes(sh) == n == plain.tile_bytes(d) and vec.vector_decode_q4_workspace_bytes(sh) > 0
    assert vec.vector_q4_tile_bytes(vec.Shape(1, 1, 1, 1, 96, BF, 16)) == 0 == vec.vector_decode_q4_workspace_bytes(vec.Shape(1, 1, 1, 1, 96, BF, 16))


P = 4096                                                     # a pointer that no refused call follows


def _cache(**kw):
    base = dict(ret_pages=P, apx_pages=P, ret_table=P, apx_table=P, ret_len=P, apx_len=P, ret_pos=0, apx_pos=P, n_ret_pages=4, n_apx_pages=4, ret_width=2, apx_width=2)
    base.update(kw)
    from paper_2605_23258_b200 import binding
    return binding._pack_q4_cache(*base.values())


def _shape(**kw):
    base = dict(batch=2, n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=F32, window=16)
    base.update(kw)
    return vec.Shape(**base)


def _decode(shape=None, q=P, cache=None, W=P, out=P, out_dtype=0, ws=P, ws_bytes=1 << 40):
    return vec.load_library().vector_decode_attn_q4((shape or _shape())._p(), q, cache if cache is not None else _cache(), W, out, out_dtype, ws, ws_bytes, None)


def test_decode_refusals():
    OK_TO_REFUSE = {"null": -1, "shape": -2, "dtype": -3, "workspace": -5}
    for kw, why in ((dict(q=None), "null"), (dict(W=None), "null"), (dict(out=None), "null"), (dict(out_dtype=2), "dtype"), (dict(shape=_shape(head_dim=96)), "shape"),
                    (dict(shape=_shape(batch=1025)), "shape"), (dict(ws=None), "workspace"), (dict(ws=P + 16), "workspace"), (dict(ws_bytes=0), "workspace"),
                    (dict(q=P + 4), "shape"), (dict(W=P + 8), "shape"), (dict(out=P + 2), "shape"), (dict(shape=_shape(dtype=7)), "dtype"),
                    (dict(cache=_cache(ret_pages=0)), "null"), (dict(cache=_cache(ret_pages=P + 8)), "shape"), (dict(cache=_cache(n_ret_pages=-1)), "shape"),
                    (dict(cache=_cache(n_apx_pages=1 << 25)), "shape"), (dict(cache=_cache(ret_table=0)), "null"), (dict(cache=_cache(apx_len=0)), "null"),
                    (dict(cache=_cache(ret_width=-1)), "shape"), (dict(cache=_cache(apx_width=(1 << 24) + 1)), "shape"),
                    (dict(shape=_shape(rope_enabled=1), cache=_cache(apx_pos=0)), "null")):
        assert _decode(**kw) == OK_TO_REFUSE[why], kw
    assert vec.load_library().vector_decode_attn_q4(_shape()._p(), P, None, P, P, 0, P, 1 << 40, None) == -1


def test_writers_and_reader_refuse():
    lib, b = vec.load_library(), vec.vector_plan_budget(100, 40, -1, 16)
    sh = _shape()._p()

    def compact(shape=sh, budget=b._p(), K=P, V=P, ri=P, ai=P, c=None, rs=P, as_=P):
        return lib.vector_compact_q4(shape, budget, K, V, ri, ai, c if c is not None else _cache(), rs, as_, None)
    for kw, rc in ((dict(K=None), -1), (dict(V=None), -1), (dict(ri=None), -1), (dict(ai=None), -1), (dict(rs=None), -1), (dict(as_=None), -1), (dict(K=P + 8), -2),
                   (dict(c=_cache(apx_pages=0, n_apx_pages=0)), -1), (dict(c=_cache(apx_pages=P + 1)), -2), (dict(budget=vec.Budget(100, 40, 20, 61, 40, 20, 39)._p()), -4)):
        assert compact(**kw) == rc, kw

    def append(c=None, k=P, v=P, start=None, slots=P, n=2, pos=None):
        return lib.vector_append_q4(sh, c if c is not None else _cache(), k, v, start, slots, n, pos, None)
    for kw, rc in ((dict(k=None), -1), (dict(v=None), -1), (dict(slots=None), -1), (dict(n=1), -2), (dict(start=P, n=-1), -2), (dict(v=P + 4), -2), (dict(c=_cache(ret_pos=P)), -1)):
        assert append(**kw) == rc, kw

    def read(rs=P, n=3, k=P, v=P, as_=P, m=3, a=P, c=None):
        return lib.vector_read_q4(sh, c if c is not None else _cache(), rs, n, k, v, as_, m, a, None)
    for kw, rc in ((dict(rs=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(as_=None), -1), (dict(a=None), -1), (dict(n=-1), -2), (dict(m=1 << 30), -2), (dict(k=P + 4), -2)):
        assert read(**kw) == rc, kw
    assert read(n=0, m=0) == 0                                # nothing to do


def test_block_tables_refusals():
    lib = vec.load_library()

    def call(batch=2, lengths=P, added=P, page=64, table=P, width=4, free=P, cap=8, n_free=P, new=P, new_free=P, first=P, start=P, slots=P, n=4):
        return lib.vector_block_tables(batch, lengths, added, page, table, width, free, cap, n_free, new, new_free, first, start, slots, n, None)
    for name in ("lengths", "added", "table", "free", "n_free", "new", "new_free", "first", "start", "slots"):
        assert call(**{name: None}) == -1, name
    for kw in (dict(batch=0), dict(batch=65536), dict(page=0), dict(width=0), dict(cap=-1), dict(n=-1), dict(n=1 << 31), dict(page=1 << 20, width=1 << 11)):
        assert call(**kw) == -2, kw


def test_binding_checks_tensors():
    sh = _shape()
    tile = vec.vector_q4_tile_bytes(sh)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    c = vec.Q4Cache(torch.zeros(2, 2, 2 * tile, dtype=torch.uint8), torch.zeros(2, 2, tile, dtype=torch.uint8), ints(2, 2), ints(2, 2), ints(2), ints(2))
    assert len(c._p()) == 8 * ctypes.sizeof(ctypes.c_void_p) + 24
    with pytest.raises(ValueError, match="CUDA"):
        vec.vector_decode_attn_q4(sh, torch.zeros(4, 2, 64), c, torch.zeros(2, 64, 64), torch.zeros(4, 2, 64))
    with pytest.raises(ValueError, match="CUDA"):
        vec.vector_block_tables(ints(2), ints(2), 64, ints(2, 2), ints(4), ints(1), ints(2), ints(1), ints(2), ints(3))


def test_plain_tables_worked_by_hand():
    # pages of 4; request 0 ends, 1 grows over a page's end, 2 is admitted, 3 drops a page's worth, 4 finds the stack empty
    new, old, table, stack, height, start, slots = plain.tables([5, 3, 0, 9, 4], [-5, 2, 6, -4, 5], 4, [[7, 8, -1], [1, -1, -1], [-1, -1, -1], [2, 3, 4], [5, -1, -1]], [9, 0, 0, 0, 0, 0], 1)
    assert new == [0, 5, 6, 5, 8] and old == [5, 3, 0, 9, 4] and height == 0 and start == [0, 0, 2, 8, 8, 13]
    assert stack[:4] == [9, 7, 8, 4] and table == [[7, 8, -1], [1, 4, -1], [8, 7, -1], [2, 3, 4], [5, 9, -1]]
    assert slots == [7, 16, 32, 33, 34, 35, 28, 29, 36, 37, 38, 39, -1]
