"""Rows within wider rows, as both ways of marshalling find them: what is taken lies where the kernels will read it, and broadcast or overlapping rows are refused."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200 import binding
from paper_2605_23258_b200.build import CSRC


class _OnGpu(torch.Tensor):
    """A tensor that says it is on a GPU: for what looks at shapes and strides alone."""
    is_cuda = True


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    """The two rules: a view's distance between rows of `width` elements, or None where it is refused."""
    at = tmp_path_factory.mktemp("rows")
    (at / "rows.cpp").write_text('#include "rows.h"\nextern "C" int rows(const int64_t* n, const int64_t* s, int d, int64_t w, int64_t* to) { return vec::row_distance(n, s, d, w, to); }\n')
    subprocess.check_call([os.environ.get("CXX", "g++"), "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(at / "rows.cpp"), "-o", str(at / "rows.so")])
    lib = ctypes.CDLL(str(at / "rows.so"))

    def module(t, width):
        if t.is_contiguous():
            return width
        many, to = ctypes.c_int64 * max(t.dim(), 1), ctypes.c_int64()
        return to.value if lib.rows(many(*t.shape), many(*t.stride()), t.dim(), ctypes.c_int64(width), ctypes.byref(to)) else None

    def ctypes_way(t, width):
        try:
            return binding._rows(t.as_subclass(_OnGpu), t.dtype, t.numel() // width, width, "t")[1]
        except ValueError:
            return None
    return module, ctypes_way


def _broadcasts(W):
    one, two, wide = torch.arange(W), torch.arange(2 * W).view(2, 1, W), torch.arange(12 * W).view(2, 2, 3 * W)
    return [one.expand(5, W), one.expand(1, 5, W), one.expand(2, 5, W), two.expand(2, 5, W), two.view(2, W).expand(5, 2, W), two.unflatten(-1, (4, W // 4)).expand(2, 5, 4, W // 4),
            two[:, :, None].expand(2, 3, 4, W), wide[:, :1, W:2 * W].expand(2, 5, W), one.as_strided((3, W // 2), (1, 1)), torch.arange(4 * W).as_strided((3, W), (W // 2, 1))]


def test_broadcast_rows_are_refused(rules):
    for t in _broadcasts(32):
        width = t.shape[-1] * (t.shape[-2] if t.dim() == 4 and t.shape[-1] == 8 else 1)
        for rule in rules:
            assert rule(t, width) is None, (tuple(t.shape), t.stride())


def test_what_is_taken_lies_where_it_is_read(rules):
    """Views of any sizes and strides: both rules say the same, and an element of a row is where its pointer and distance put it."""
    rng, taken = random.Random(1), 0
    store = torch.arange(20000)
    for _ in range(30000):
        dims = rng.randint(1, 4)
        sizes = [rng.choice([1, 1, 2, 3, 4, 8]) for _ in range(dims)]
        strides, step = [], 1
        for n in reversed(sizes):
            strides.insert(0, rng.choice([step, step, step, step * 2, step + 8, 0, 1, rng.randint(0, 40)]))
            step = max(strides[0], 1) * n
        if sum((n - 1) * s for n, s in zip(sizes, strides)) >= store.numel():
            continue
        t = store.as_strided(sizes, strides)
        for width in {w for w in (1, 2, 4, 8, 16, 32, 24, t.numel()) if t.numel() % w == 0}:
            module, other = (rule(t, width) for rule in rules)
            assert module == other, (sizes, strides, width)
            if module is not None:
                taken += 1
                n = t.numel() // width
                assert n == 1 or module >= width
                assert torch.equal(t.reshape(n, width), torch.arange(n)[:, None] * module + torch.arange(width)), (sizes, strides, width)
    assert taken > 10000


@pytest.mark.gpu
@pytest.mark.parametrize("way", ["module", "ctypes"])
def test_calls_refuse_broadcast_rows(way, monkeypatch):
    if way == "ctypes":
        monkeypatch.setattr(binding, "_marshal_module", binding._CtypesOnly())
    sh = vec.Shape(2, 1, 2, 2, 64, vec.VECTOR_F32, 16)
    c = vec.alloc_q8_cache(sh, 4, 4, 2, 2)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    x, dense = torch.zeros(2, 1, 128, device="cuda").expand(2, 5, 128), torch.zeros(2, 5, 128, device="cuda")
    for k, v in ((x, dense), (dense, x), (x[:1].expand(2, 5, 128), dense)):
        with pytest.raises(ValueError, match="rows must lie"):
            vec.vector_append_q8(sh, c, k, v, ints(2), ints(2, 5))
        with pytest.raises(ValueError, match="rows must lie"):
            vec.vector_norm_rope(sh, 5, k=k, v=v, k_out=torch.zeros(4, 5, 64, device="cuda"), v_out=torch.zeros(4, 5, 64, device="cuda"))
