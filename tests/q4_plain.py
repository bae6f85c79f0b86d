"""The 4-bit paged cache in plain numpy and 64 bits, from its definition: rounding to codes and scales, the place of every code in a
page, attention over the rows, and tables and slots request by request."""
import numpy as np
import torch

import paper_2605_23258_b200 as vec

ROWS = 64
NUMBERS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)


def scale_value(code):
    e, m = np.asarray(code).astype(np.int64) >> 3, np.asarray(code).astype(np.int64) & 7
    v = np.where(e > 0, (1 + m / 8.0) * np.exp2(e - 15.0), m / 8.0 * 2.0 ** -14)
    return np.where(e == 31, np.nan, v)


SCALES = scale_value(np.arange(227))


def encode(x):
    """x [n][d] -> codes [n][d], scale codes [n][d / 16]."""
    x = np.asarray(x, np.float64)
    x = x.reshape(len(x), x.shape[1] // 16, 16)
    with np.errstate(invalid="ignore", divide="ignore"):
        most = np.abs(x).max(-1)
        bad = np.isnan(most)
        sc = np.minimum(np.searchsorted(6 * SCALES, np.where(bad, 0, most), side="left"), 226)
        s = SCALES[sc][..., None]
        t = np.where(s > 0, np.abs(x) / s, 0.0)
        t = np.minimum(np.where(np.isnan(t), 0, t), 7.0)            # beyond 6 all are as near
        dist = np.abs(t[..., None] - NUMBERS)
        near = dist.argmin(-1)                      # the lower code of two equally near ones; it is the even one or its neighbour is
        up = np.minimum(near + 1, 7)
        tie = np.take_along_axis(dist, near[..., None], -1)[..., 0] == np.take_along_axis(dist, up[..., None], -1)[..., 0]
        code = np.where(tie & (near % 2 == 1) & (near < 7), up, near)
    return (code + 8 * (x < 0)).reshape(len(x), -1 if len(x) else 16 * x.shape[1]), np.where(bad, 255, sc)


def values(codes, scales):
    v = np.where(codes & 8, -1.0, 1.0) * NUMBERS[codes & 7]
    return (v.reshape(len(codes), codes.shape[1] // 16, 16) * scale_value(scales)[..., None]).reshape(codes.shape)


def rounded(x):
    return values(*encode(x))


def tile_bytes(d):
    return ROWS * (d // 2 + d // 16)


def places(d):
    """Byte and shift of every channel's code in a row, and place of every group's scale."""
    byte, shift, scale = [], [], []
    for c in range(d):
        low, up = c % (d // 2), c // (d // 2)
        e = low // (d // 8) * (d // 4) + up * (d // 8) + low % (d // 8)
        byte.append(e // 2), shift.append(4 * (e % 2))
    for g in range(d // 16):
        scale.append(2 * (g % (d // 32)) + g // (d // 32))
    return np.array(byte), np.array(shift), np.array(scale)


def row_values(pages, slots, lh, which, d):
    """Rows [n][d] of the slots of one (layer, KV head); pages: numpy [P][LH][parts * tile]."""
    byte, shift, scale = places(d)
    t = pages[:, lh, which * tile_bytes(d):(which + 1) * tile_bytes(d)]
    slots = np.asarray(slots, np.int64)
    page, row = slots // ROWS, slots % ROWS
    codes = t[page[:, None], row[:, None] * (d // 2) + byte[None, :]] >> shift & 15
    return values(codes.astype(np.int64), t[page[:, None], ROWS * d // 2 + row[:, None] * (d // 16) + scale[None, :]])


def put_rows(pages, slots, lh, which, x):
    """The same in the other direction, into numpy pages."""
    d = x.shape[1]
    byte, shift, scale = places(d)
    codes, sc = encode(x)
    t = pages[:, lh, which * tile_bytes(d):(which + 1) * tile_bytes(d)]
    packed = np.zeros((len(x), d // 2), np.uint8)
    np.bitwise_or.at(packed, (slice(None), byte), (codes << shift).astype(np.uint8))
    stored = np.zeros((len(x), d // 16), np.uint8)
    stored[:, scale] = sc
    for i, s in enumerate(np.asarray(slots, np.int64)):
        r = s % ROWS
        t[s // ROWS, r * (d // 2):(r + 1) * (d // 2)] = packed[i]
        t[s // ROWS, ROWS * d // 2 + r * (d // 16):ROWS * d // 2 + (r + 1) * (d // 16)] = stored[i]


def slots_of(table, n):
    i = np.arange(n)
    return table[i // ROWS].astype(np.int64) * ROWS + i % ROWS


def tables(lengths, added, page, table, stack, n_free):
    """One request after another; returns new lengths, table, stack, its height, row starts and slots."""
    lengths, table, stack = list(map(int, lengths)), [list(map(int, r)) for r in table], list(map(int, stack))
    pages = lambda n: -(-n // page)  # noqa: E731
    old = [min(max(n, 0), len(table[0]) * page) for n in lengths]
    new = [max(n + int(a), 0) for n, a in zip(old, added)]
    height = int(n_free)
    for b, a in enumerate(added):
        for i in range(pages(new[b]), pages(old[b])):
            stack[height] = table[b][i]
            height += 1
    start, slots = [0], []
    for b, a in enumerate(added):
        a = int(a)
        if a > 0:
            have = pages(old[b])
            while have < min(pages(new[b]), len(table[b])) and height > 0:
                height -= 1
                table[b][have] = stack[height]
                have += 1
            new[b] = min(new[b], have * page)
            for i in range(old[b], old[b] + a):
                slots.append(table[b][i // page] * page + i % page if i < new[b] else -1)
        start.append(start[-1] + max(a, 0))
    return new, old, table, stack, height, start, slots


def attend(q, rk, rv, ak, W, scale, pos=None, theta=10000.0):
    """q [g][d] over retained rows rk, rv and key-only rows ak, 64 bits: the output, and what a relative error of the logits (per head), of
    the weights and of a turned key can make of it: (o, spread, logit_size, turned_size)."""
    q, rk, rv, ak, W = (np.asarray(x, np.float64) for x in (q, rk, rv, ak, W))
    k = np.concatenate([rk, ak])
    if not len(k):
        z = np.zeros_like(q)
        return z, z, np.zeros((len(q), 1)), z
    s = q @ k.T * scale
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    kt, size = ak, np.abs(ak)
    if pos is not None:
        half = ak.shape[1] // 2
        ang = np.asarray(pos, np.float64)[:, None] * theta ** (-np.arange(half) / half)
        x, y, cs, sn = ak[:, :half], ak[:, half:], np.cos(ang), np.sin(ang)
        kt = np.concatenate([x * cs + y * sn, y * cs - x * sn], 1)
        size = np.concatenate([np.abs(x) + np.abs(y)] * 2, 1)
    n = len(rk)
    o = p[:, :n] @ rv + p[:, n:] @ kt @ W.T
    spread = p[:, :n] @ np.abs(rv) + p[:, n:] @ np.abs(kt) @ np.abs(W).T
    return o, spread, (np.abs(q) @ np.abs(k).T).max(-1, keepdims=True) * scale, p[:, n:] @ size @ np.abs(W).T


def tolerance(o, spread, logit_size, turned_size, dtype, out_dtype, rope):
    """What an output may be off by, elementwise.  A logit sums head_dim exact products in fp32, in at most sixteen sums that are cut off or
    rounded (2^-23 each of the sum of magnitudes); that is the relative error of a weight, which comes in twice, with the sum of weights.  An
    exponential: 2^-21.  The weights' parts: 2^-11 twice where one fp16 part carries them (bf16 in and out), else 2^-21.  Sums of weights
    times rows and the map's product: 2^-20.  A key turned back: sine, cosine, two products and the sum in fp16, 2^-11 each of |x| + |y|, and its angle, whose
    phase is held to 2^-32 of a turn a position: 2 pi 131072 2^-33 = 1e-4; in parts of 22 bits with an accurate angle, 2^-19 in all.
    The result's own rounding."""
    exact = dtype == torch.float32 or out_dtype == torch.float32
    weight = 2.0 ** -20 if exact else 2.0 ** -10
    turn = (2.0 ** -19 if exact else 4 * 2.0 ** -11 + 1.2e-4) if rope else 0.0
    own = 2.0 ** -24 if out_dtype == torch.float32 else 2.0 ** -8
    return (2 * 16 * 2.0 ** -23 * logit_size + 2.0 ** -20 + weight + 2.0 ** -20) * spread + turn * turned_size + own * np.abs(o) + 1e-30


def problem(batch, layers, heads, g, d, dtype, lengths, seed, rope=False, spare=2, device="cuda"):
    """A paged cache of sequences with `lengths` = [(n_ret, n_apx)], in pages that held something else before, with the queries and maps.
    Keys at page borders lean towards the queries, so that each carries a visible share of its output."""
    rng = np.random.default_rng(seed)
    LH = layers * heads
    shape = vec.Shape(batch, layers, heads * g, heads, d, vec.VECTOR_BF16 if dtype == torch.bfloat16 else vec.VECTOR_F32, 16, 7, 0.0, int(rope), 10000.0)
    q = torch.from_numpy(rng.standard_normal((batch * LH, g, d))).to(dtype)
    W = torch.from_numpy(rng.standard_normal((LH, d, d)) / np.sqrt(d)).to(dtype)
    pools = {}
    for tier, parts in (("ret", 2), ("apx", 1)):
        rows = [n[parts == 1] for n in lengths]
        pages = [-(-n // ROWS) for n in rows]
        total = sum(pages) + spare
        order = rng.permutation(total).astype(np.int32)
        table = np.full((batch, max(pages + [1]) + 1), -1, np.int32)
        at = 0
        for b, n in enumerate(pages):
            table[b, :n] = order[at:at + n]
            at += n
        pool = rng.integers(0, 256, (total, LH, parts * tile_bytes(d)), dtype=np.uint8)
        pos = rng.integers(0, 131072, (total, LH, ROWS)).astype(np.int32)
        for b, n in enumerate(rows):
            for lh in range(LH):
                k = rng.standard_normal((n, d)) * 1.5
                u = q[b * LH + lh, 0].double().numpy()
                edge = [r for r in range(n) if r % ROWS in (0, ROWS - 1) or r == n - 1]
                k[edge] += 3.0 * u / np.linalg.norm(u)
                put_rows(pool, slots_of(table[b], n), lh, 0, k)
                if parts == 2:
                    put_rows(pool, slots_of(table[b], n), lh, 1, rng.standard_normal((n, d)) * np.exp(rng.uniform(-3, 1, (n, 1))))
        pools[tier] = (pool, table, np.array(rows, np.int32), pos)
    on = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(device)  # noqa: E731
    (rp, rt, rl, rpos), (ap, at_, al, apos) = pools["ret"], pools["apx"]
    cache = vec.Q4Cache(on(rp), on(ap), on(rt), on(at_), on(rl), on(al), on(rpos), on(apos))
    return shape, q.to(device), cache, W.to(device)


def expected(shape, q, cache, W, b, lh, rope):
    """attend()'s answer for one unit of a cache on any device."""
    d, LH = shape.head_dim, shape.n_layers * shape.n_kv_heads
    n, m = int(cache.ret_len[b]), int(cache.apx_len[b])
    rp, ap = cache.ret_pages.cpu().numpy(), cache.apx_pages.cpu().numpy()
    rs, as_ = slots_of(cache.ret_table[b].cpu().numpy(), n), slots_of(cache.apx_table[b].cpu().numpy(), m)
    empty = np.zeros((0, d))
    rk, rv = (row_values(rp, rs, lh, w, d) if n else empty for w in (0, 1))
    ak = row_values(ap, as_, lh, 0, d) if m else empty
    pos = cache.apx_pos.cpu().numpy()[as_ // ROWS, lh, as_ % ROWS] if rope and m else (np.zeros(0) if rope else None)
    return attend(q[b * LH + lh].double().cpu().numpy(), rk, rv, ak, W[lh].double().cpu().numpy(), 1 / np.sqrt(d), pos)


def decode(shape, q, cache, W, out_dtype):
    out = torch.full(q.shape, float("nan"), dtype=out_dtype, device=q.device)
    ws = torch.empty(vec.vector_decode_q4_workspace_bytes(shape), dtype=torch.uint8, device=q.device)
    vec.vector_decode_attn_q4(shape, q, cache, W, out, ws)
    torch.cuda.synchronize()
    assert vec.vector_device_fault() == 0
    return out


def check_decode(shape, q, cache, W, out, rope, units=None):
    LH = shape.n_layers * shape.n_kv_heads
    worst = 0.0
    for u in units if units is not None else range(shape.units):
        o, *sizes = expected(shape, q, cache, W, u // LH, u % LH, rope)
        tol = tolerance(o, *sizes, q.dtype, out.dtype, rope)
        err = np.abs(out[u].double().cpu().numpy() - o)
        assert np.all(np.isfinite(err)), u
        assert np.all(err <= tol), (u, float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
        worst = max(worst, float((err / tol).max()))
    return worst
