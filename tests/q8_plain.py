"""The 8-bit paged cache in plain numpy and 64 bits, from its definition: rounding of blocks, the place of every channel in a page, new rows under a scale that
grows; attention and its tolerance are those of the 4-bit cache's plain form, over these rows."""
import numpy as np
import torch

import paper_2605_23258_b200 as vec
import q4_plain

ROWS, LOW, HIGH = 32, -32, 31


def number(code):
    """What codes stand for, without a scale, from their bits."""
    c = np.asarray(code).astype(np.int64)
    e, m = c >> 3 & 15, (c & 7) / 8.0
    v = np.where(e > 0, np.ldexp(1 + m, e - 7), np.ldexp(m, -6))
    v = np.where(c & 127 == 127, np.nan, v)
    return np.where(c & 128, -v, v)


NUMBERS = number(np.arange(127))


def exponent(x):
    """Of the scale of a block: the smallest in range with 448 2^e >= the largest magnitude, NaN aside."""
    x = np.abs(np.asarray(x, np.float64))
    most = min(np.max(x[~np.isnan(x)], initial=0.0), 448 * 2.0 ** HIGH)
    e = LOW
    while 448 * 2.0 ** e < most:
        e += 1
    return e


def encode(x, e):
    """Codes of x under a scale: the nearest number, ties to the even code."""
    x = np.asarray(x, np.float64)
    bad = np.isnan(x)
    size = np.minimum(np.abs(np.where(bad, 0, x)) * 2.0 ** -e, 448.0)
    up = np.minimum(np.searchsorted(NUMBERS, size, side="left"), 126)           # NUMBERS[up] >= size
    down = np.maximum(up - 1, 0)
    a, b = size - NUMBERS[down], NUMBERS[up] - size
    code = np.where((b < a) | ((b == a) & (up % 2 == 0)), up, down)
    return (np.where(bad, 127, code) | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def rounded(x, e=None):
    """Rows of a sequence, [n][d], as they are held when they are written at once."""
    x = np.asarray(x, np.float64)
    got = np.empty_like(x)
    for r in range(0, len(x), ROWS):
        e_r = exponent(x[r:r + ROWS])
        got[r:r + ROWS] = number(encode(x[r:r + ROWS], e_r)) * 2.0 ** e_r
    return got


class Held:
    """One unit's rows of a tier, keys or values, growing."""

    def __init__(self):
        self.rows, self.scales = [], []

    def append(self, x):
        """New rows [n][d] in one call."""
        x = np.asarray(x, np.float64)
        at = 0
        while at < len(x):
            first = len(self.rows) % ROWS
            part = x[at:at + ROWS - first]
            e = exponent(part)
            if first == 0:
                self.scales.append(e)
            elif e > self.scales[-1]:
                self.rows[-first:] = [number(encode(r, e)) * 2.0 ** e for r in self.rows[-first:]]
                self.scales[-1] = e
            e = self.scales[-1]
            self.rows += [number(encode(r, e)) * 2.0 ** e for r in part]
            at += len(part)
        return self

    def values(self, d):
        return np.array(self.rows).reshape(-1, d)


def turned(k, pos, theta=10000.0):
    """Rows [n][d] turned by their positions."""
    k = np.asarray(k, np.float64)
    half = k.shape[-1] // 2
    ang = np.asarray(pos, np.float64)[..., None] * theta ** (-np.arange(half) / half)
    x, y, cs, sn = k[..., :half], k[..., half:], np.cos(ang), np.sin(ang)
    return np.concatenate([x * cs - y * sn, y * cs + x * sn], -1)


def tile_bytes(d):
    return ROWS * d + 32


def place(row, c, d):
    """Byte of channel c of a page's row."""
    if d == 128:
        return row * d + (c // 64 ^ row & 1) * 64 + c % 64
    return row * d + c % 32 // 8 * 16 + c // 32 * 8 + c % 8


def _places(d):
    return np.array([[place(r, c, d) for c in range(d)] for r in range(ROWS)])


_PLACES = {d: _places(d) for d in (64, 128)}


def put_rows(pages, table, lh, which, x):
    """Rows [n][d] of a sequence, written at once, into numpy pages [P][LH][parts * tile]."""
    d = x.shape[1]
    t = pages[:, lh, which * tile_bytes(d):(which + 1) * tile_bytes(d)]
    for r in range(0, len(x), ROWS):
        part = x[r:r + ROWS]
        e = exponent(part)
        t[table[r // ROWS], _PLACES[d][:len(part)]] = encode(part, e)
        t[table[r // ROWS], ROWS * d] = e - LOW


def row_values(pages, table, rows, lh, which, d):
    """The rows (numbers of them) of a sequence, [n][d]."""
    rows = np.asarray(rows, np.int64)
    t = pages[:, lh, which * tile_bytes(d):(which + 1) * tile_bytes(d)]
    page = np.asarray(table, np.int64)[rows // ROWS]
    return number(t[page[:, None], _PLACES[d][rows % ROWS]]) * 2.0 ** (t[page, ROWS * d].astype(np.float64) + LOW)[:, None]


def problem(batch, layers, heads, g, d, dtype, lengths, seed, rope=False, spare=2, device="cuda", spread=2.0):
    """A paged cache of sequences with `lengths` = [(n_ret, n_apx)], in pages that held something else before, with the queries and maps.  Blocks' scales differ by `spread` and
    keys at page borders lean towards the queries, so that each carries a visible share of its output."""
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
                k = rng.standard_normal((n, d)) * np.repeat(np.exp2(rng.uniform(-spread, spread / 4, -(-n // ROWS))), ROWS)[:n, None]
                u = q[b * LH + lh, 0].double().numpy()
                edge = [r for r in range(n) if r % ROWS in (0, ROWS - 1) or r == n - 1]
                k[edge] += 3.0 * u / np.linalg.norm(u)
                put_rows(pool, table[b], lh, 0, k)
                if parts == 2:
                    put_rows(pool, table[b], lh, 1, rng.standard_normal((n, d)) * np.exp(rng.uniform(-3, 1, (n, 1))))
        pools[tier] = (pool, table, np.array(rows, np.int32), pos)
    on = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(device)  # noqa: E731
    (rp, rt, rl, rpos), (ap, at_, al, apos) = pools["ret"], pools["apx"]
    cache = vec.Q8Cache(on(rp), on(ap), on(rt), on(at_), on(rl), on(al), on(rpos), on(apos))
    return shape, q.to(device), cache, W.to(device)


def expected(shape, q, cache, W, b, lh, rope, ret_rows=None, apx_rows=None):
    """q4_plain.attend()'s answer for one unit of a cache on any device."""
    d, LH = shape.head_dim, shape.n_layers * shape.n_kv_heads
    ret_rows, apx_rows = range(int(cache.ret_len[b])) if ret_rows is None else ret_rows, range(int(cache.apx_len[b])) if apx_rows is None else apx_rows
    rp, ap = cache.ret_pages.cpu().numpy(), cache.apx_pages.cpu().numpy()
    rt, at = cache.ret_table[b].cpu().numpy(), cache.apx_table[b].cpu().numpy()
    empty = np.zeros((0, d))
    rk, rv = (row_values(rp, rt, ret_rows, lh, w, d) if len(ret_rows) else empty for w in (0, 1))
    ak = row_values(ap, at, apx_rows, lh, 0, d) if len(apx_rows) else empty
    a = np.asarray(apx_rows, np.int64)
    pos = cache.apx_pos.cpu().numpy()[at[a // ROWS], lh, a % ROWS] if rope and len(a) else (np.zeros(0) if rope else None)
    return q4_plain.attend(q[b * LH + lh].double().cpu().numpy(), rk, rv, ak, W[lh].double().cpu().numpy(), 1 / np.sqrt(d), pos)


def decode(shape, q, cache, W, out_dtype):
    out = torch.full(q.shape, float("nan"), dtype=out_dtype, device=q.device)
    ws = torch.empty(vec.vector_decode_q8_workspace_bytes(shape), dtype=torch.uint8, device=q.device)
    vec.vector_decode_attn_q8(shape, q, cache, W, out, ws)
    torch.cuda.synchronize()
    assert vec.vector_device_fault() == 0
    return out


def check_decode(shape, q, cache, W, out, rope, units=None, **rows):
    """The tolerance is q4_plain's: the arithmetic is the same, and the powers of two that are factors here cost no rounding."""
    LH = shape.n_layers * shape.n_kv_heads
    for u in units if units is not None else range(shape.units):
        o, *sizes = expected(shape, q, cache, W, u // LH, u % LH, rope, **rows)
        tol = q4_plain.tolerance(o, *sizes, q.dtype, out.dtype, rope)
        err = np.abs(out[u].double().cpu().numpy() - o)
        assert np.all(np.isfinite(err)), u
        assert np.all(err <= tol), (u, float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))
