"""CPU checks of the 8-bit paged cache and of the way from projections: the plain form that the GPU tests compare with, sizes, what the entry points refuse, and
rows that lie within wider ones."""
import glob
import os
import re

import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
import q8_plain as plain
from paper_2605_23258_b200 import binding
from paper_2605_23258_b200.build import CSRC

BF, F32 = vec.VECTOR_BF16, vec.VECTOR_F32
P = 4096                                                     # a pointer that no refused call follows


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2605_23258_b200.build import build
    build()


def test_plain_rounding_is_the_nearest_code():
    assert plain.NUMBERS[-1] == 448 and plain.NUMBERS[1] == 2.0 ** -9 and len(plain.NUMBERS) == 127 and np.all(np.diff(plain.NUMBERS) > 0)
    x = torch.randn(4000, dtype=torch.float64) * torch.exp(torch.empty(4000).uniform_(-8, 6))
    x = x.clamp(-448, 448).float()
    got = plain.number(plain.encode(x.double().numpy(), 0))
    assert np.array_equal(got, x.to(torch.float8_e4m3fn).double().numpy())
    mid = (plain.NUMBERS[1:] + plain.NUMBERS[:-1]) / 2                                       # ties
    assert np.array_equal(plain.number(plain.encode(mid, 0)), torch.from_numpy(mid).float().to(torch.float8_e4m3fn).double().numpy())
    for most, e in ((448, 0), (448.0001, 1), (224, -1), (0, -32), (1e-30, -32), (np.inf, 31), (448 * 2.0 ** 31, 31), (1e12, 31), (1.0, -8), (1.75, -8), (1.76, -7)):
        assert plain.exponent([[most, 0], [0, -most / 2 if most < 1e30 else 0]]) == e, most
    assert plain.exponent([[np.nan, 3.0]]) == plain.exponent([[3.0]]) and np.isnan(plain.rounded(np.array([[np.nan, 3.0]]))[0, 0])
    assert plain.rounded(np.array([[np.inf, -np.inf]])).tolist() == [[448 * 2.0 ** 31, -448 * 2.0 ** 31]]


@pytest.mark.parametrize("d", [64, 128])
def test_plain_layout_is_a_permutation(d):
    assert sorted(plain._PLACES[d].flatten().tolist()) == list(range(32 * d))
    pages = np.zeros((4, 2, 2 * plain.tile_bytes(d)), np.uint8)
    x = np.random.default_rng(1).standard_normal((70, d))
    plain.put_rows(pages, [3, 0, 2], 1, 1, x)
    assert np.array_equal(plain.row_values(pages, [3, 0, 2], range(70), 1, 1, d), plain.rounded(x)) and not pages[:, 0].any() and not pages[1].any()
    h = plain.Held().append(x[:40]).append(x[40:])
    assert np.abs(h.values(d) - plain.rounded(x)).max() <= np.abs(x).max() / 8


def test_tile_bytes():
    for d, n in ((64, 2080), (128, 4128)):
        sh = vec.Shape(1, 1, 1, 1, d, BF, 16)
        assert vec.vector_q8_tile_bytes(sh) == n == plain.tile_bytes(d) and vec.vector_decode_q8_workspace_bytes(sh) > 0
    assert vec.vector_q8_tile_bytes(vec.Shape(1, 1, 1, 1, 96, BF, 16)) == 0 == vec.vector_decode_q8_workspace_bytes(vec.Shape(1, 1, 1, 1, 96, BF, 16))


def _cache(**kw):
    base = dict(ret_pages=P, apx_pages=P, ret_table=P, apx_table=P, ret_len=P, apx_len=P, ret_pos=0, apx_pos=P, n_ret_pages=4, n_apx_pages=4, ret_width=2, apx_width=2)
    base.update(kw)
    return binding._pack_q4_cache(*base.values())


def _shape(**kw):
    base = dict(batch=2, n_layers=1, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype=F32, window=16)
    base.update(kw)
    return vec.Shape(**base)


NULL, SHAPE, DTYPE, BUDGET, WORKSPACE = -1, -2, -3, -4, -5
BAD_POOLS = ((dict(ret_pages=0), NULL), (dict(ret_pages=P + 8), SHAPE), (dict(n_ret_pages=-1), SHAPE), (dict(n_apx_pages=1 << 26), SHAPE), (dict(ret_width=-1), SHAPE),
             (dict(apx_width=(1 << 25) + 1), SHAPE), (dict(apx_pos=P + 4), SHAPE))


def test_decode_refusals():
    def decode(shape=None, q=P, cache=None, W=P, out=P, out_dtype=0, ws=P, ws_bytes=1 << 40):
        return vec.load_library().vector_decode_attn_q8((shape or _shape())._p(), q, cache if cache is not None else _cache(), W, out, out_dtype, ws, ws_bytes, None)
    for kw, rc in ((dict(q=None), NULL), (dict(W=None), NULL), (dict(out=None), NULL), (dict(out_dtype=2), DTYPE), (dict(shape=_shape(head_dim=96)), SHAPE),
                   (dict(shape=_shape(batch=1025)), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws=P + 16), WORKSPACE), (dict(ws_bytes=0), WORKSPACE),
                   (dict(q=P + 4), SHAPE), (dict(W=P + 8), SHAPE), (dict(out=P + 2), SHAPE), (dict(shape=_shape(dtype=7)), DTYPE), (dict(cache=_cache(ret_table=0)), NULL),
                   (dict(cache=_cache(apx_len=0)), NULL), (dict(shape=_shape(rope_enabled=1), cache=_cache(apx_pos=0)), NULL), *((dict(cache=_cache(**c)), rc) for c, rc in BAD_POOLS)):
        assert decode(**kw) == rc, kw
    assert vec.load_library().vector_decode_attn_q8(_shape()._p(), P, None, P, P, 0, P, 1 << 40, None) == NULL


def test_writers_and_reader_refuse():
    lib, b = vec.load_library(), vec.vector_plan_budget(100, 40, -1, 16)
    sh = _shape()._p()

    def compact(budget=b._p(), K=P, V=P, ri=P, ai=P, c=None):
        return lib.vector_compact_q8(sh, budget, K, V, ri, ai, c if c is not None else _cache(), None)
    for kw, rc in ((dict(K=None), NULL), (dict(V=None), NULL), (dict(ri=None), NULL), (dict(ai=None), NULL), (dict(K=P + 8), SHAPE), (dict(c=_cache(ret_len=0)), NULL),
                   (dict(c=_cache(apx_table=0)), NULL), (dict(c=_cache(apx_pages=0, n_apx_pages=0)), NULL), (dict(budget=vec.Budget(100, 40, 20, 61, 40, 20, 39)._p()), BUDGET),
                   *((dict(c=_cache(**c)), rc) for c, rc in BAD_POOLS)):
        assert compact(**kw) == rc, kw

    def append(shape=sh, c=None, k=P, ks=128, v=P, vs=128, n=3, first=P, pos=None, rotate=0):
        return lib.vector_append_q8(shape, c if c is not None else _cache(), k, ks, v, vs, n, first, pos, rotate, None)
    turns = _shape(rope_enabled=1)._p()
    for kw, rc in ((dict(k=None), NULL), (dict(v=None), NULL), (dict(first=None), NULL), (dict(n=-1), SHAPE), (dict(n=(1 << 30) + 1), SHAPE), (dict(ks=127), SHAPE), (dict(vs=0), SHAPE),
                   (dict(ks=130), SHAPE), (dict(v=P + 4), SHAPE), (dict(c=_cache(ret_pos=P)), NULL), (dict(rotate=1), SHAPE), (dict(shape=turns, rotate=1), NULL),
                   (dict(c=_cache(ret_table=0)), NULL), (dict(c=_cache(ret_pages=0, n_ret_pages=0)), NULL), (dict(vs=1 << 41), SHAPE), *((dict(c=_cache(**c)), rc) for c, rc in BAD_POOLS)):
        assert append(**kw) == rc, kw
    assert append(n=0, k=None) == 0                           # nothing to do

    def read(n=3, k=P, v=P, m=3, a=P, c=None):
        return lib.vector_read_q8(sh, c if c is not None else _cache(), n, k, v, m, a, None)
    for kw, rc in ((dict(k=None), NULL), (dict(v=None), NULL), (dict(a=None), NULL), (dict(n=-1), SHAPE), (dict(m=1 << 30), SHAPE), (dict(k=P + 4), SHAPE), (dict(c=_cache(ret_len=0)), NULL),
                   *((dict(c=_cache(**c)), rc) for c, rc in BAD_POOLS)):
        assert read(**kw) == rc, kw
    assert read(n=0, m=0) == 0


def test_norm_rope_refusals():
    lib = vec.load_library()

    def call(shape=None, N=10, q=P, qs=256, qw=P, first=0, qo=P, k=P, ks=128, kw=P, ko=P, v=P, vs=128, vo=P, pos=None, eps=1e-6):
        return lib.vector_norm_rope((shape or _shape())._p(), N, q, qs, qw, first, qo, k, ks, kw, ko, v, vs, vo, pos, eps, None)
    for kw, rc in ((dict(N=-1), SHAPE), (dict(N=(1 << 30) + 1), SHAPE), (dict(first=-1), SHAPE), (dict(first=11), SHAPE), (dict(eps=-1e-6), SHAPE), (dict(eps=float("nan")), SHAPE),
                   (dict(qo=None), NULL), (dict(ko=None), NULL), (dict(vo=None), NULL), (dict(qs=255), SHAPE), (dict(ks=127), SHAPE), (dict(vs=64), SHAPE), (dict(qs=257), SHAPE),
                   (dict(q=P + 4), SHAPE), (dict(ko=P + 8), SHAPE), (dict(kw=P + 4), SHAPE), (dict(shape=_shape(head_dim=96)), SHAPE), (dict(shape=_shape(dtype=3)), DTYPE),
                   (dict(shape=_shape(batch=30000), N=1 << 30), SHAPE)):
        assert call(**kw) == rc, kw
    assert call(N=0) == 0 and call(q=None, k=None, v=None) == 0 and call(first=10, k=None, v=None) == 0


class _OnGpu(torch.Tensor):
    """A tensor that says it is on a GPU: for what looks at shapes and strides alone."""
    is_cuda = True


def test_rows_within_wider_rows():
    def rows(t, count, width):
        p, stride = binding._rows(t.as_subclass(_OnGpu), torch.float32, count, width, "t")
        assert p == t.data_ptr()
        return stride
    x = torch.zeros(3, 5, 4, 8)
    assert rows(x, 15, 32) == 32 and rows(x.flatten(), 15, 32) == 32 and rows(x, 60, 8) == 8
    wide = torch.zeros(3, 5, 100)
    assert rows(wide[..., 8:40], 15, 32) == 100 and rows(wide[..., 8:40].unflatten(-1, (4, 8)), 15, 32) == 100 and rows(wide[:, :1, 8:40], 3, 32) == 500 and rows(wide[:1, :1, 8:40], 1, 32) == 32
    assert rows(torch.zeros(0, 5, 32), 0, 32) == 32
    for t, count, width in ((x.transpose(1, 2), 15, 32), (wide[..., :64:2], 15, 32), (wide[:, 1:3, :32], 6, 32), (wide.transpose(0, 1)[..., :32], 15, 32)):
        with pytest.raises(ValueError, match="row"):
            rows(t, count, width)
    with pytest.raises(ValueError, match="15 rows of 32"):
        rows(torch.zeros(3, 5, 31), 15, 32)
    with pytest.raises(ValueError, match="dtype"):
        binding._rows(x.double().as_subclass(_OnGpu), torch.float32, 15, 32, "t")
    with pytest.raises(ValueError, match="CUDA"):
        binding._rows(x, torch.float32, 15, 32, "t")


def test_binding_checks_tensors():
    sh = _shape()
    tile = vec.vector_q8_tile_bytes(sh)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    c = vec.Q8Cache(torch.zeros(2, 2, 2 * tile, dtype=torch.uint8), torch.zeros(2, 2, tile, dtype=torch.uint8), ints(2, 2), ints(2, 2), ints(2), ints(2))
    x = torch.zeros(2, 1, 2, 64)
    for call in (lambda: vec.vector_decode_attn_q8(sh, torch.zeros(4, 2, 64), c, torch.zeros(2, 64, 64), torch.zeros(4, 2, 64)), lambda: vec.vector_append_q8(sh, c, x, x, ints(2)),
                 lambda: vec.vector_read_q8(sh, c, torch.zeros(4, 3, 64), torch.zeros(4, 3, 64)), lambda: vec.vector_norm_rope(sh, 1, k=x, k_out=torch.zeros(4, 1, 64))):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="q_first"):
        vec.vector_norm_rope(sh, 4, q_first=5)


def test_no_two_sources_define_the_same_struct():
    """The linker keeps one of two functions of the same name, a template's in two sources among them: what their members launch would be the other's kernels."""
    seen = {}
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        scope = []
        for line in open(path).read().splitlines():
            m = re.match(r"namespace (\w+) \{", line)
            if m:
                scope.append(m.group(1))
            elif line.startswith("}  // namespace"):
                scope.pop()
            m = re.match(r"(?:template <.*> )?struct (\w+)(?! *<)[^;]*\{", line)
            if m:
                name = "::".join([*scope, m.group(1)])
                assert seen.setdefault(name, path) == path, name
    assert len(seen) >= 15
