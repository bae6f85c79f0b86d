"""Projections to rows, norms and positions, against 64 bits (80 for the angles): types, head sizes, tokens from one to thousands, the window's queries alone, rows of wider rows,
far and negative positions, and both ways of marshalling."""
import numpy as np
import pytest
import torch

import paper_2605_23258_b200 as vec
from paper_2605_23258_b200 import binding

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda"


def _shape(batch, layers, q_heads, heads, d, dtype, rope=1, theta=10000.0, window=1):
    return vec.Shape(batch, layers, q_heads, heads, d, vec.VECTOR_BF16 if dtype == BF else vec.VECTOR_F32, window, 7, 0.0, rope, theta)


def _expected(x, w, pos, eps, theta):
    """x [..., d] (64 bits), w [d] or None, pos [...] or None: rows, and the size of what is summed up for each channel."""
    d = x.shape[-1]
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    if pos is None:
        return x, np.abs(x)
    half = d // 2
    ang = pos[..., None].astype(np.longdouble) * np.longdouble(theta) ** (-np.arange(half).astype(np.longdouble) / half)
    cs, sn = np.cos(ang).astype(np.float64), np.sin(ang).astype(np.float64)
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * cs - b * sn, b * cs + a * sn], -1), np.concatenate([np.abs(a) + np.abs(b)] * 2, -1)


def _close(got, want, size, dtype):
    """fp32 arithmetic: the mean of squares (a chain of eight and five sums, halved by the root: 7), the root's reciprocal (4), weight times sine or cosine (1, and 2 for these
    themselves), two products, a sum and the factor (4), in units of 2^-24 of the size: 18 and less than 2^-19.  An angle is right to 2^-32 of a turn, the series to 2e-9.  Then the result's own rounding."""
    own = 2.0 ** -8 if dtype == BF else 2.0 ** -24
    err = np.abs(got.double().cpu().numpy() - want)
    tol = 2.0 ** -19 * size + own * np.abs(want) + 1e-37
    assert np.all(err <= tol), float((err / tol).max())


def _run(sh, N, qkv, first, weights, pos, eps=1e-6, want=("q", "k", "v")):
    U, g, d = sh.units, sh.group, sh.head_dim
    new = lambda *s: torch.full((*s, d), float("nan"), dtype=sh.torch_dtype, device=DEV)  # noqa: E731
    out = {"q": new(U, g, N - first), "k": new(U, N), "v": new(U, N)}
    pick = lambda n, x: x if n in want else None  # noqa: E731
    vec.vector_norm_rope(sh, N, pick("q", qkv[0]), pick("k", qkv[1]), pick("v", qkv[2]), pick("q", out["q"]), pick("k", out["k"]), pick("v", out["v"]), weights[0], weights[1], pos, first, eps)
    return out


def _check(sh, N, qkv, first, weights, pos, out, eps=1e-6, want=("q", "k", "v"), theta=10000.0):
    B, L, d = sh.batch, sh.n_layers, sh.head_dim
    at = np.broadcast_to(np.arange(N), (B, N)) if pos is None else pos.cpu().numpy().reshape(B, N)
    for name, x, w, heads, f in (("q", qkv[0], weights[0], sh.n_q_heads, first), ("k", qkv[1], weights[1], sh.n_kv_heads, 0), ("v", qkv[2], None, sh.n_kv_heads, 0)):
        if name not in want:
            assert torch.isnan(out[name]).all()
            continue
        x = x.reshape(B, L, N, heads, d).double().cpu().numpy()[:, :, f:]
        for l in range(L):
            wl = None if w is None else w[l].double().cpu().numpy()
            p = None if name == "v" or not sh.rope_enabled else np.broadcast_to(at[:, f:, None], x.shape[:1] + x.shape[2:4])
            e, size = _expected(x[:, l], wl, p, eps, theta)
            got = out[name].reshape(B, L, heads, N - f, d)[:, l]
            if name == "v":
                assert np.array_equal(got.double().cpu().numpy(), e.transpose(0, 2, 1, 3))
            else:
                _close(got, e.transpose(0, 2, 1, 3), size.transpose(0, 2, 1, 3), BF if sh.dtype == vec.VECTOR_BF16 else F32)


def _problem(seed, sh, N, spread=2.0):
    rng = np.random.default_rng(seed)
    d, heads = sh.head_dim, sh.n_q_heads + 2 * sh.n_kv_heads
    x = rng.standard_normal((sh.batch, sh.n_layers, N, heads * d)) * np.exp(rng.uniform(-spread, spread, (sh.batch, sh.n_layers, N, 1)))
    x = torch.from_numpy(x).to(sh.torch_dtype).to(DEV)
    w = [torch.from_numpy(rng.uniform(0.3, 2, (sh.n_layers, d))).to(sh.torch_dtype).to(DEV) for _ in range(2)]
    return x.split([sh.n_q_heads * d, sh.n_kv_heads * d, sh.n_kv_heads * d], dim=-1), w, rng


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rope,norm", [(1, True), (1, False), (0, True), (0, False)])
@pytest.mark.parametrize("d,batch,layers,q_heads,heads,N,first", [(128, 1, 1, 32, 8, 1, 0), (128, 5, 1, 6, 2, 1, 0), (64, 2, 3, 8, 8, 37, 30), (128, 1, 1, 3, 1, 1001, 0), (64, 1, 2, 5, 5, 64, 64),
                                                                  (128, 2, 1, 4, 4, 17, 16), (64, 3, 1, 7, 1, 700, 0)])
def test_sizes_and_types(dtype, rope, norm, d, batch, layers, q_heads, heads, N, first):
    sh = _shape(batch, layers, q_heads, heads, d, dtype, rope)
    qkv, w, rng = _problem(d + N, sh, N)
    pos = torch.from_numpy(rng.integers(0, 1 << 20, (batch, N)).astype(np.int32)).to(DEV)
    w = w if norm else [None, None]
    out = _run(sh, N, qkv, first, w, pos)
    _check(sh, N, qkv, first, w, pos, out)


def test_parts_alone_and_positions_of_their_own():
    sh = _shape(2, 1, 4, 2, 128, BF)
    qkv, w, _ = _problem(1, sh, 50)
    for want, weights in ((("q",), [w[0], None]), (("k",), [None, w[1]]), (("v",), w), (("q", "v"), [None, None]), (("k", "v"), [None, w[1]])):
        out = _run(sh, 50, qkv, 7, weights, None, want=want)
        _check(sh, 50, qkv, 7, weights, None, out, want=want)


@pytest.mark.parametrize("theta", [10000.0, 500000.0, 1e6])
def test_far_and_negative_positions(theta):
    sh = _shape(1, 1, 2, 1, 128, F32, theta=theta)
    pos = torch.tensor([[0, 1, -1, 131071, 131072, 2**30 + 12345, 2**31 - 1, -2**31, 77777777]], dtype=torch.int32, device=DEV)
    qkv, w, _ = _problem(2, sh, 9)
    out = _run(sh, 9, qkv, 0, w, pos)
    _check(sh, 9, qkv, 0, w, pos, out, theta=theta)


def test_rows_of_any_size():
    """A row of zeros stays one, large and small rows have the same norm, a NaN and an infinity stay in their head."""
    sh = _shape(1, 1, 2, 2, 64, F32, 0)
    x = torch.randn(1, 1, 6, 128, device=DEV)
    x[0, 0, 0, :64], x[0, 0, 1, :64], x[0, 0, 2] = 0, x[0, 0, 1, 64:] * 2.0 ** 50, x[0, 0, 2] * 2.0 ** -30
    x[0, 0, 3, 5], x[0, 0, 4, 70] = float("nan"), float("inf")
    w = [None, torch.ones(1, 64, device=DEV)]
    out = _run(sh, 6, (x, x, x), 0, w, None, eps=1e-30, want=("k",))["k"]
    assert not out[0, 0].any() and (out[0, 1] - out[1, 1]).abs().max() <= 2.0 ** -20
    e = torch.nn.functional.rms_norm(x[0, 0, 2].double().view(2, 64), (64,), eps=1e-30)
    assert (out[:, 2].double() - e).abs().max() <= 2.0 ** -18
    assert torch.isnan(out[0, 3]).all() and torch.isfinite(out[1, 3]).all() and torch.isnan(out[1, 4, 6]) and not out[1, 4, :6].any() and torch.isfinite(out[0, 4]).all()


def test_both_ways_of_marshalling_and_streams(monkeypatch):
    sh = _shape(3, 1, 4, 2, 128, BF)
    qkv, w, rng = _problem(5, sh, 21)
    pos = torch.from_numpy(rng.integers(0, 5000, (3, 21)).astype(np.int32)).to(DEV)
    first = _run(sh, 21, qkv, 4, w, pos)
    dense = _run(sh, 21, [t.contiguous() for t in qkv], 4, w, pos)
    heads = _run(sh, 21, [t.unflatten(-1, (-1, 128)) for t in qkv], 4, w, pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = _run(sh, 21, qkv, 4, w, pos)
    torch.cuda.synchronize()
    monkeypatch.setattr(binding, "_marshal_module", binding._CtypesOnly())
    plain = _run(sh, 21, qkv, 4, w, pos)
    for x in (dense, heads, other, plain):
        assert all(torch.equal(first[n], x[n]) for n in first)
    for bad in (dict(q=qkv[0][..., :-128]), dict(k_weight=w[1].float()), dict(pos=pos[:2]), dict(pos=torch.cat([pos, pos], 1)), dict(q_out=first["q"][:2]), dict(v=qkv[2].transpose(0, 2)), dict(q_first=22)):
        kw = dict(q=qkv[0], k=qkv[1], v=qkv[2], q_out=first["q"], k_out=first["k"], v_out=first["v"], q_weight=w[0], k_weight=w[1], pos=pos, q_first=4)
        kw.update(bad)
        with pytest.raises(ValueError):
            vec.vector_norm_rope(sh, 21, **kw)


def test_many_heads_and_long_contexts():
    """More heads than a launch has rows of blocks for, and more than 2^31 numbers of a projection."""
    sh = _shape(1, 1, 65535, 65535, 64, BF, 1)
    x = torch.randn(1, 1, 1, 65535 * 64, device=DEV, dtype=BF)
    out = _run(sh, 1, (x, x, x), 0, [None, None], torch.tensor([[3]], dtype=torch.int32, device=DEV))
    assert torch.equal(out["q"][:, 0, 0], out["k"][:, 0]) and torch.equal(out["v"].flatten(), x.flatten())
    small = _shape(1, 1, 8, 8, 64, BF, 1)
    y = x[..., -512:].contiguous()
    part = _run(small, 1, (y, y, y), 0, [None, None], torch.tensor([[3]], dtype=torch.int32, device=DEV))
    assert torch.equal(part["k"], out["k"][-8:])
    del out, part
    sh, N = _shape(1, 1, 8, 8, 128, BF, 1), 2_200_000
    k = torch.randn(1, 1, N, 1024, device=DEV, dtype=BF)
    out = torch.empty(8, N, 128, device=DEV, dtype=BF)
    vec.vector_norm_rope(sh, N, k=k, k_out=out)
    at = torch.tensor([[0, 1, N // 2, N - 2, N - 1]], dtype=torch.int32, device=DEV)
    few = torch.empty(8, 5, 128, device=DEV, dtype=BF)
    vec.vector_norm_rope(sh, 5, k=k[:, :, at[0].long()].contiguous(), k_out=few, pos=at)
    assert torch.equal(out[:, at[0].long()], few)
