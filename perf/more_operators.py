"""The 8-bit paged cache and the way from a model's projections to it: what serving over a compressed cache calls, and what each call has to compute.

Rows of the mixed cache (retained tokens: key and value; key-only tokens: key) are held as e4m3 numbers (sign, four exponent bits, three mantissa bits,
largest 448) times a power of two, one for each block of 32 tokens, head, and keys or values: 2^e with the smallest e in [-32, 31] for which 448 2^e is not
below the largest magnitude of the block; a channel is the nearest such number, ties to the even one.  A page is a block.  An operation ("op") of a case is

  rows     vector_norm_rope: queries, keys and values of a layer's projections into rows of heads, norms and positions applied
  store    vector_compact_q8 of a compressed context into its pages, and vector_read_q8 of the rows
  chunk    several new tokens of every sequence: vector_append_q8, keys turned by their positions on the way, and vector_read_q8 of all rows
  step     one generated token: vector_block_tables, vector_append_q8, vector_decode_attn_q8
  decode   vector_decode_attn_q8 over the pages
"""
import math

import torch

own = False
_DEVICE = "cuda"
_ROWS = 32                                   # rows of a page, and of a block that shares a scale
_LOW, _HIGH = -32, 31                        # exponents of a block's scale
_THETA = 10000.0


# ---- cases -----------------------------------------------------------------------------------------------------------------------
def _rows_case(batch, tokens, q_heads, kv_heads, head_dim, dtype, norm, rope, first, with_v=True, far=0):
    """first: the first token whose queries are wanted; far: positions begin there."""
    return {"op": "rows", "batch": batch, "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "norm": norm,
            "rope": rope, "first": first, "with_v": with_v, "far": far}


def _model(op, batch, layers, q_heads, kv_heads, head_dim, dtype, N, percent, ragged=False, rope=False, out="bf16", empty=0, new=1):
    return {"op": op, "batch": batch, "layers": layers, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype,
            "N": N, "percent": percent, "ragged": ragged, "rope": rope, "out": out, "empty": empty, "new": new}


def listed():
    cases = {
        # queries and keys of one generated token of 64 requests, one layer of an 8B model's geometry: latency
        "rows_step_batch64": _rows_case(64, 1, 32, 8, 128, "bf16", True, True, 0, with_v=False, far=8192),
        # a layer's prompt on its way to compression: window queries, keys and values out of the fused projection
        "rows_prompt": _rows_case(1, 32768, 32, 8, 128, "bf16", True, True, 32704),
        # all queries too, in fp32, 64-channel heads, a length that is no multiple of anything
        "rows_fp32_head64": _rows_case(3, 5003, 8, 4, 64, "fp32", True, True, 0),
        # one layer's rows to 8 bits as its prefill ends, an 8B model's attention geometry, and back
        "store_one_layer": _model("store", 1, 1, 32, 8, 128, "bf16", 8192, 20),
        # the whole compressed cache of a 32-layer model
        "store_32_layers": _model("store", 1, 32, 32, 8, 128, "bf16", 32768, 20),
        # five drafted tokens of each of 32 requests, behind rows that fill their blocks in part
        "chunk_drafts": _model("chunk", 32, 1, 32, 8, 128, "bf16", 700, 40, ragged=True, rope=True, new=5),
        # a piece of four prompts that are kept in full
        "chunk_prompt": _model("chunk", 4, 1, 32, 8, 128, "bf16", 1000, 30, ragged=True, rope=True, new=2048),
        # one layer's step of a single request: the latency of a generated token is this, times the layers
        "step_one_layer": _model("step", 1, 1, 32, 8, 128, "bf16", 8192, 20),
        # one layer's step of a batch of requests of all lengths, some places of the batch not taken, rotary keys
        "step_batch64_ragged": _model("step", 64, 1, 32, 8, 128, "bf16", 8192, 20, ragged=True, rope=True, empty=5),
        # a 70B model's geometry at its longest context: the largest call
        "decode_80_layers": _model("decode", 1, 80, 64, 8, 128, "bf16", 131072, 5),
        # all 32 layers of eight requests in one call
        "decode_batch8_32_layers": _model("decode", 8, 32, 32, 8, 128, "bf16", 16384, 10, ragged=True),
        # 64-channel heads, results in fp32
        "decode_head64": _model("decode", 4, 16, 32, 8, 64, "bf16", 16384, 20, ragged=True, out="fp32"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["rows", "rows", "rows", "store", "store", "chunk", "chunk", "step", "step", "decode", "decode", "decode"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    kv_heads, g, head_dim = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 3, 4, 4, 8]), rng.choice([64, 128, 128])
    if op == "rows":
        batch, tokens = _log_int(rng, 1, 64), _log_int(rng, 1, 65536)
        row = kv_heads * (g + 2) * head_dim * (2 if dtype == "bf16" else 4)
        while batch * tokens > max(4e8 / row, 1):
            if tokens > batch:
                tokens = (tokens + 1) // 2
            else:
                batch = (batch + 1) // 2
        return _rows_case(batch, tokens, kv_heads * g, kv_heads, head_dim, dtype, rng.random() < 0.7, rng.random() < 0.8, rng.choice([0, 0, max(0, tokens - 64)]),
                          with_v=rng.random() < 0.6, far=rng.choice([0, 1000, 100000]))
    N, percent = _log_int(rng, 300, 131072), rng.choice([5, 10, 15, 20, 25, 30, 40])
    batch, layers = _log_int(rng, 1, 64), _log_int(rng, 1, 80)
    new = 1
    if op == "store":
        batch = min(batch, 4)
    if op == "chunk":
        N, layers, new = min(N, 4000), min(layers, 4), _log_int(rng, 1, 4096)
    # cut until the keys of the longest sequences take at most 0.5 GB in 8 bits, the keys of a stored context 0.8 GB and of a chunk 0.4 GB
    es = 2.0 if dtype == "bf16" else 4.0
    rows = {"store": N, "chunk": N + new}.get(op, N * percent / 100.0 + 64)
    most = {"store": 0.8e9 / es, "chunk": 0.4e9 / es}.get(op, 0.5e9) / (head_dim * kv_heads * rows)
    if dtype == "fp32" and op in ("step", "decode"):
        most = min(most, 1e6 / (kv_heads * rows))
    while batch * layers > max(most, 1):
        if layers >= batch:
            layers = (layers + 1) // 2
        else:
            batch = (batch + 1) // 2
    # keys are turned by sums of fp32 products before they are rounded: in fp32, where a number next to a border may go either way, they come turned
    rope = dtype == "bf16" and op in ("chunk", "step", "decode") and rng.random() < 0.4
    return _model(op, batch, layers, kv_heads * g, kv_heads, head_dim, dtype, N, percent, ragged=op != "store" and rng.random() < 0.6, rope=rope,
                  out="fp32" if dtype == "fp32" else "bf16" if op == "step" else rng.choice(["bf16", "bf16", "fp32"]),
                  empty=rng.choice([0, 0, 1]) if op in ("step", "decode") and batch > 2 else 0, new=new)


def _tiers(N, percent):
    """Rows of the two tiers of a context of N tokens: n_a = min((N - Bp) / 2, Bp / 2), Bp - n_a retained, 2 n_a key-only."""
    pairs = max(N * percent // 100, 16)
    n_a = min((N - pairs) // 2, pairs // 2)
    return pairs - n_a, 2 * n_a


def _context_lengths(c):
    """Tokens of each sequence of the batch; a place that nobody has taken has none."""
    r = torch.Generator().manual_seed(c["batch"] * 131 + c["N"])
    N = [c["N"]] * c["batch"]
    if c["ragged"]:
        share = torch.rand(c["batch"], generator=r).tolist()
        N = [max(64, round(c["N"] * (0.1 + 0.9 * s))) for s in share]
        N[-1] = c["N"]
    for i in range(c["empty"]):
        N[i * 2] = 0
    return N


def _lengths(c):
    """Rows of the two tiers of each sequence before the call; some tokens were generated since the context was compressed."""
    got = []
    for i, N in enumerate(_context_lengths(c)):
        ret, apx = _tiers(N, c["percent"]) if N else (0, 0)
        got.append((ret + (i * 37 + c["N"]) % 150 if N else 0, apx))
    return got


def _held_bytes(rows, d):
    return rows * d + math.ceil(rows / _ROWS)


def work(c):
    d, es = c["head_dim"], 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "rows":
        rows = c["batch"] * ((c["tokens"] - c["first"]) * c["q_heads"] + c["tokens"] * c["kv_heads"] * (2 if c["with_v"] else 1))
        return {"bytes": float(2 * rows * d * es + 4 * c["batch"] * c["tokens"]), "flops": 0.0}
    LH = c["layers"] * c["kv_heads"]
    if c["op"] == "store":
        ret, apx = _tiers(c["N"], c["percent"])
        units = c["batch"] * LH
        return {"bytes": float(units * ((2 * ret + apx) * 2 * d * es + 2 * _held_bytes(ret, d) + _held_bytes(apx, d) + 4 * (ret + apx))), "flops": 0.0}
    lengths = _lengths(c)
    if c["op"] == "chunk":
        rows = sum(r + c["new"] for r, _ in lengths)
        new = c["batch"] * c["new"]
        # new rows in; rows that were there read, all rows out; positions
        return {"bytes": float(2 * LH * (new * d * es + _held_bytes(rows, d) + rows * d * es) + 4 * new), "flops": 0.0}
    extra = 1 if c["op"] == "step" else 0
    ret, apx = sum(r + (extra if r else 0) for r, _ in lengths), sum(a for _, a in lengths)
    g = c["q_heads"] // c["kv_heads"]
    heads = c["batch"] * LH * g
    out = 2 if c["out"] == "bf16" else 4
    turned = 4 * apx * LH if c["rope"] else 0
    return {"bytes": float(LH * (2 * _held_bytes(ret, d) + _held_bytes(apx, d)) + LH * d * d * es + heads * d * (es + out) + turned + extra * c["batch"] * LH * 2 * d * es),
            "flops": float(2 * g * d * LH * (2 * ret + 2 * apx) + 2 * heads * d * d)}


# ---- what a program has in hand --------------------------------------------------------------------------------------------------
def _rand(gen, *shape):
    return torch.rand(*shape, generator=gen, device=_DEVICE)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=_DEVICE)


def _spread(gen, shape, lo, hi):
    return torch.exp(math.log(lo) + _rand(gen, *shape) * math.log(hi / lo))


def _law(c, gen):
    """Channel scales of keys and queries spread over a factor of eight per (layer, KV head), one key channel in a hundred twenty times
    larger; values of a token are as large as its own factor says."""
    LH, d = c["layers"] * c["kv_heads"], c["head_dim"]
    sigma_k, sigma_q = _spread(gen, (LH, 1, d), 0.5, 4.0), _spread(gen, (LH, 1, d), 0.5, 4.0)
    big = torch.argsort(_rand(gen, LH, 1, d), dim=2)[..., :max(1, d // 100)]
    sigma_k.scatter_(2, big, sigma_k.gather(2, big) * 20.0)
    return sigma_k, sigma_q


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _prepare_rows(c, seed):
    gen = torch.Generator(device=_DEVICE).manual_seed(seed * 7919 + 11)
    B, N, d, dtype = c["batch"], c["tokens"], c["head_dim"], _type(c["dtype"])
    heads = c["q_heads"] + 2 * c["kv_heads"]
    x = torch.empty(B, N, heads * d, dtype=dtype, device=_DEVICE)              # a layer's fused projection: queries, keys, values
    sigma = _spread(gen, (heads * d,), 0.2, 3.0)
    for b in range(B):
        x[b] = (_randn(gen, N, heads * d) * sigma).to(dtype)
    q, k, v = x.split([c["q_heads"] * d, c["kv_heads"] * d, c["kv_heads"] * d], dim=-1)
    s = {"q": q, "k": k, "v": v, "q_weight": None, "k_weight": None}
    if c["norm"]:
        s["q_weight"], s["k_weight"] = (_spread(gen, (1, d), 0.5, 2.0).to(dtype) for _ in range(2))
    start = torch.randint(0, 512, (B, 1), generator=gen, device=_DEVICE) + c["far"]
    s["pos"] = (start + torch.arange(N, device=_DEVICE)[None, :]).int().contiguous()
    return s


def _prepare_store(c, seed):
    gen = torch.Generator(device=_DEVICE).manual_seed(seed * 7919 + 5)
    B, LH, d, N, dtype = c["batch"], c["layers"] * c["kv_heads"], c["head_dim"], c["N"], _type(c["dtype"])
    ret, apx = _tiers(N, c["percent"])
    sigma_k, _ = _law(c, gen)
    K = torch.empty(B * LH, N, d, dtype=dtype, device=_DEVICE)
    V = torch.empty_like(K)
    for u in range(0, B * LH, c["kv_heads"]):
        at = u % LH
        K[u:u + c["kv_heads"]] = (_randn(gen, c["kv_heads"], N, d) * sigma_k[at:at + c["kv_heads"]]).to(dtype)
        V[u:u + c["kv_heads"]] = (_randn(gen, c["kv_heads"], N, d) * _spread(gen, (c["kv_heads"], N, 1), 0.02, 2.0)).to(dtype)
    kept = torch.argsort(_rand(gen, B * LH, N), dim=1)[:, :ret + apx].int()
    s = {"K": K, "V": V, "ret": ret, "apx": apx,
         "ret_idx": kept[:, :ret].sort(dim=1).values.contiguous(), "apx_idx": kept[:, ret:].sort(dim=1).values.contiguous()}
    s.update(_pools(c, gen, [(ret, apx)] * B, 0))
    s["ret_len"], s["apx_len"] = (torch.full((B,), n, dtype=torch.int32, device=_DEVICE) for n in (ret, apx))
    return s


def _tile(d):
    return _ROWS * d + 32


def _pools(c, gen, lengths, more):
    """Pages of both tiers with whatever was in memory, and tables that take them in no order; the last page is in no table."""
    LH, tile = c["layers"] * c["kv_heads"], _tile(c["head_dim"])
    s = {}
    for tier, parts, rows in (("ret", 2, [r + more for r, _ in lengths]), ("apx", 1, [a for _, a in lengths])):
        have = [(n + _ROWS - 1) // _ROWS for n in rows]
        width, pages = max(max(have), 1), sum(have) + 3
        order = torch.randperm(pages - 1, generator=gen, device=_DEVICE).int()
        table = torch.full((c["batch"], width), -1, dtype=torch.int32, device=_DEVICE)
        at = 0
        for b, h in enumerate(have):
            table[b, :h] = order[at:at + h]
            at += h
        s[tier + "_table"] = table
        s[tier + "_pages"] = torch.randint(0, 256, (pages, LH, parts * tile), generator=gen, device=_DEVICE, dtype=torch.uint8)
    return s


def _prepare_cache(c, seed):
    gen = torch.Generator(device=_DEVICE).manual_seed(seed * 7919 + 7)
    B, H, d, dtype = c["batch"], c["kv_heads"], c["head_dim"], _type(c["dtype"])
    LH, g, more = c["layers"] * H, c["q_heads"] // H, 0 if c["op"] == "decode" else c["new"]
    lengths = _lengths(c)
    sigma_k, sigma_q = _law(c, gen)
    s = _pools(c, gen, lengths, more)
    for i, tier in ((0, "ret"), (1, "apx")):
        s[tier + "_len"] = torch.tensor([n[i] for n in lengths], dtype=torch.int32, device=_DEVICE)
    s["apx_pos"] = torch.randint(0, c["N"], (s["apx_pages"].shape[0], LH, _ROWS), generator=gen, device=_DEVICE, dtype=torch.int32)
    for b, (ret, apx) in enumerate(lengths):
        for at in range(0, LH, H):
            part = slice(at, at + H)
            for n, tier, is_v in ((ret, "ret", 0), (ret, "ret", 1), (apx, "apx", 0)):
                if n and not (c["op"] == "chunk" and tier == "apx"):
                    blocks = (n + _ROWS - 1) // _ROWS
                    x = torch.zeros(H, blocks * _ROWS, d, device=_DEVICE)
                    x[:, :n] = _randn(gen, H, n, d) * (_spread(gen, (H, n, 1), 0.02, 2.0) if is_v else sigma_k[part])
                    x = x.unflatten(1, (blocks, _ROWS))
                    _put(s[tier + "_pages"], s[tier + "_table"][b, :blocks], part, is_v, x, _exponent(x))
    s["q"] = (_randn(gen, B, LH, g, d) * sigma_q[None]).to(dtype).flatten(0, 1)
    s["W"] = (_randn(gen, LH, d, d) / math.sqrt(d)).to(dtype)
    if more:
        # rows of all heads of a token behind one another, as a projection leaves them
        s["k_new"] = (_randn(gen, B, more, LH, d) * sigma_k[None, None, :, 0]).to(dtype)
        s["v_new"] = (_randn(gen, B, more, LH, d) * _spread(gen, (B, more, LH, 1), 0.02, 2.0)).to(dtype)
        s["pos"] = (c["N"] + torch.arange(more, device=_DEVICE, dtype=torch.int32)[None, :]).expand(B, -1).contiguous()
    if c["op"] == "chunk":
        s["first_row"] = s["ret_len"]
        s["ret_len"] = s["ret_len"] + c["new"]
    if c["op"] == "step":
        s["added"] = (s["ret_len"] > 0).int()
        # the pages behind a request's rows are not in its table yet: they lie on the stack of free pages
        have = (s["ret_len"].long() + _ROWS - 1) // _ROWS
        full = (s["ret_len"].long() + s["added"] + _ROWS - 1) // _ROWS
        i = torch.arange(s["ret_table"].shape[1], device=_DEVICE)[None, :]
        free = s["ret_table"][(i >= have[:, None]) & (i < full[:, None])]
        s["ret_table"][(i >= have[:, None])] = -1
        s["free"] = torch.full((s["ret_pages"].shape[0],), -1, dtype=torch.int32, device=_DEVICE)
        s["free"][:free.numel()] = free
        s["n_free"] = torch.tensor([free.numel()], dtype=torch.int32, device=_DEVICE)
    return s


def prepare(case, seed):
    s = {"rows": _prepare_rows, "store": _prepare_store}.get(case["op"], _prepare_cache)(case, seed)
    s["case"] = case
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------------------
_constants = {}


def _constant(name, make):
    if name not in _constants:
        _constants[name] = make().to(_DEVICE)
    return _constants[name]


def _byte_of(d):
    """Where the channels of a block's 32 rows lie in its bytes, [32 * d].  128 channels: as they are, the halves of an odd row changed; 64 channels:
    eight low ones, then those half a head above them."""
    r, c = torch.arange(_ROWS)[:, None], torch.arange(d)[None, :]
    place = ((c // 64) ^ (r & 1)) * 64 + c % 64 if d == 128 else (c % 32) // 8 * 16 + c // 32 * 8 + c % 8 + 0 * r
    return (r * d + place).flatten()


def _exponent(x):
    """The exponents of the scales of blocks x [..., 32, d]."""
    most = torch.nan_to_num(x.float().abs(), nan=0.0, posinf=3.4e38).amax((-1, -2)).clamp(max=448.0 * 2.0 ** _HIGH)
    m, k = torch.frexp(most)
    return torch.where(most > 0, k - 9 + (m > 0.875), _LOW).clamp(_LOW, _HIGH)


def _power(e):
    """2^e, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _put(pages, to, part, is_v, x, e):
    """Blocks x [heads][n][32][d] with their scales' exponents e [heads][n] into the pages `to` [n] of the heads `part`."""
    d = x.shape[-1]
    tile = _tile(d)
    size = (x.float() * _power(-e)[..., None, None]).clamp(-448.0, 448.0)
    codes = size.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    stored = torch.empty_like(codes)
    stored[..., _constant(("bytes", d), lambda: _byte_of(d))] = codes
    t = pages.unflatten(-1, (pages.shape[-1] // tile, tile))[:, part, is_v]
    at = to.long()
    t[:, :, :_ROWS * d][at] = stored.transpose(0, 1)
    t[:, :, _ROWS * d][at] = (e - _LOW).to(torch.uint8).transpose(0, 1)


def _blocks(pages, which, at, d):
    """The blocks of pages `at` as values [*at][LH][32][d], and their exponents [*at][LH]."""
    tile = _tile(d)
    t = pages.unflatten(-1, (pages.shape[-1] // tile, tile))[:, :, which]
    e = t[..., _ROWS * d][at].int().clamp(max=_HIGH - _LOW) + _LOW
    x = t[..., :_ROWS * d][at].index_select(-1, _constant(("bytes", d), lambda: _byte_of(d))).view(torch.float8_e4m3fn).float()
    return (x * _power(e)[..., None]).unflatten(-1, (_ROWS, d)), e


def _held(pages, table, lengths, d, which):
    """Rows of every sequence, [batch][LH][width * 32][d], with zeros behind a sequence's last row, and which are its rows."""
    x, _ = _blocks(pages, which, table.long().clamp(0, pages.shape[0] - 1), d)
    x = x.transpose(1, 2).flatten(2, 3)
    there = torch.arange(x.shape[2], device=_DEVICE)[None, :] < lengths[:, None]
    return torch.where(there[:, None, :, None], x, 0.0), there


def _cos_sin(pos, half):
    inv = _THETA ** (-torch.arange(half, device=_DEVICE, dtype=torch.float64) / half)
    angle = (pos.double()[..., None] * inv).remainder(2 * math.pi)
    return torch.cos(angle).float(), torch.sin(angle).float()


def _turned(x, pos, back=False):
    half = x.shape[-1] // 2
    cs, sn = _cos_sin(pos, half)
    if back:
        sn = -sn
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cs - b * sn, b * cs + a * sn], dim=-1)


def _plain_rows(s):
    c = s["case"]
    d, dtype = c["head_dim"], _type(c["dtype"])

    def heads(x, weight, pos, rope):
        x = x.float().unflatten(-1, (-1, d))                                       # [B][N][heads][d]
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float()
        if rope:
            x = _turned(x, pos[..., None])
        return x.transpose(1, 2).contiguous().to(dtype)
    got = {"q": heads(s["q"][:, c["first"]:], s["q_weight"], s["pos"][:, c["first"]:], c["rope"]).unflatten(1, (c["kv_heads"], -1)).flatten(0, 1),
           "k": heads(s["k"], s["k_weight"], s["pos"], c["rope"]).flatten(0, 1)}
    if c["with_v"]:
        got["v"] = heads(s["v"], None, None, False).flatten(0, 1)
    return got


def _plain_append(s, first, length, table):
    """New rows into the blocks that they touch, beside the rows that are there."""
    c = s["case"]
    LH, d, new, pages = c["layers"] * c["kv_heads"], c["head_dim"], c["new"], s["ret_pages"]
    spare = pages.shape[0] - 1
    touched = (new + _ROWS - 2) // _ROWS + 1
    block = first.long()[:, None] // _ROWS + torch.arange(touched, device=_DEVICE)[None, :]                       # [B][touched]
    row = block[..., None] * _ROWS + torch.arange(_ROWS, device=_DEVICE)                                           # [B][touched][32]
    is_old, is_new = row < first[:, None, None], (row >= first[:, None, None]) & (row < length[:, None, None])
    used = is_new.any(-1)
    page = torch.where(used, table.gather(1, block.clamp(max=table.shape[1] - 1)).long(), spare)
    page = torch.where(page < 0, spare, page)
    at = (row - first[:, None, None]).clamp(0, new - 1)                                                            # which new row
    b = torch.arange(c["batch"], device=_DEVICE)[:, None, None]
    for is_v, x in ((0, s["k_new"]), (1, s["v_new"])):
        x = x.float()
        if c["rope"] and not is_v:
            x = _turned(x, s["pos"][..., None])
        x = torch.where(is_new[..., None, None], x[b, at], 0.0).transpose(2, 3)                                    # [B][touched][LH][32][d]
        old, e = _blocks(pages, is_v, page, d)
        e = torch.maximum(_exponent(x), torch.where(is_old.any(-1)[..., None], e, _LOW))
        x = torch.where(is_old[:, :, None, :, None], old, x)
        _put(pages, page.flatten(), slice(0, LH), is_v, x.flatten(0, 1).transpose(0, 1), e.flatten(0, 1).transpose(0, 1))


def _plain_attention(s, ret_len, ret_table):
    c = s["case"]
    B, LH, d = c["batch"], c["layers"] * c["kv_heads"], c["head_dim"]
    q = s["q"].float().unflatten(0, (B, LH)) * (1 / math.sqrt(d))
    rk, there_r = _held(s["ret_pages"], ret_table, ret_len, d, 0)
    ak, there_a = _held(s["apx_pages"], s["apx_table"], s["apx_len"], d, 0)
    logit = torch.cat([q @ rk.transpose(-1, -2), q @ ak.transpose(-1, -2)], dim=-1)
    there = torch.cat([there_r, there_a], dim=-1)[:, None, None, :]
    logit = torch.where(there, logit, -math.inf)
    most = logit.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(logit - most)
    total = p.sum(-1, keepdim=True)
    n = rk.shape[2]
    del rk
    rv, _ = _held(s["ret_pages"], ret_table, ret_len, d, 1)
    o = p[..., :n] @ rv
    del rv
    if c["rope"]:
        at = s["apx_table"].long().clamp(0, s["apx_pages"].shape[0] - 1)
        ak = _turned(ak, s["apx_pos"][at].transpose(1, 2).flatten(2, 3), back=True)
    o = o + (p[..., n:] @ ak) @ s["W"].float().transpose(-1, -2)
    o = torch.where(total > 0, o / total.clamp(min=1e-30), 0.0)
    return o.flatten(0, 1).to(_type(c["out"]))


def _plain_tables(lengths, added, table, free, n_free, page, n_slots):
    """New lengths, table, stack of free pages and its height, first new rows, row starts and slots, of requests that grow or stay."""
    old, width = lengths.long(), table.shape[1]
    have, new = (old + page - 1) // page, old + added.long()
    need = ((new + page - 1) // page).clamp(max=width) - have
    before = torch.cumsum(need, 0) - need
    got = torch.minimum(need, (n_free.long() - before).clamp(min=0))
    i = torch.arange(width, device=_DEVICE)[None, :]
    fresh = (i >= have[:, None]) & (i < (have + got)[:, None])
    table = torch.where(fresh, free[(n_free.long() - 1 - before[:, None] - (i - have[:, None])).clamp(0, free.numel() - 1)], table)
    held = torch.minimum(new, (have + got) * page)
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=_DEVICE), torch.cumsum(added.long(), 0)])
    k = torch.arange(n_slots, device=_DEVICE)
    b = torch.searchsorted(start, k, right=True) - 1
    there = b < lengths.numel()
    b = b.clamp(max=lengths.numel() - 1)
    row = old[b] + k - start[b]
    slots = torch.where(there & (row < held[b]), table[b, (row // page).clamp(max=width - 1)] * page + row % page, -1)
    return held.int(), table, old.int(), slots.int()


def _run_plain(s):
    c = s["case"]
    if c["op"] == "rows":
        return _plain_rows(s)
    B, LH, d = c["batch"], c["layers"] * c["kv_heads"], c["head_dim"]
    dtype = _type(c["dtype"])
    if c["op"] == "store":
        def keep(X, tier, is_v):
            idx, n, table = s[tier + "_idx"], s[tier], s[tier + "_table"]
            if not n:
                return
            blocks = (n + _ROWS - 1) // _ROWS
            x = X.gather(1, idx.long()[..., None].expand(-1, -1, d))
            x = torch.nn.functional.pad(x, (0, 0, 0, blocks * _ROWS - n)).unflatten(1, (blocks, _ROWS)).unflatten(0, (B, LH)).transpose(0, 1).flatten(1, 2)   # [LH][B * blocks][32][d]
            _put(s[tier + "_pages"], table[:, :blocks].flatten(), slice(0, LH), is_v, x, _exponent(x))
        keep(s["K"], "ret", 0)
        keep(s["V"], "ret", 1)
        keep(s["K"], "apx", 0)
        back = lambda tier, which: _held(s[tier + "_pages"], s[tier + "_table"], s[tier + "_len"], d, which)[0][:, :, :s[tier]].flatten(0, 1).to(dtype).contiguous()  # noqa: E731
        return {"ret_k": back("ret", 0), "ret_v": back("ret", 1), "apx_k": back("apx", 0)}
    if c["op"] == "chunk":
        _plain_append(s, s["first_row"], s["ret_len"], s["ret_table"])
        most = max(r for r, _ in _lengths(c)) + c["new"]
        back = lambda which: _held(s["ret_pages"], s["ret_table"], s["ret_len"], d, which)[0][:, :, :most].flatten(0, 1).to(dtype).contiguous()  # noqa: E731
        return {"ret_k": back(0), "ret_v": back(1)}
    if c["op"] == "decode":
        return _plain_attention(s, s["ret_len"], s["ret_table"])
    held, table, first, slots = _plain_tables(s["ret_len"], s["added"], s["ret_table"], s["free"], s["n_free"], _ROWS, B)
    _plain_append(s, first, held, table)
    return {"out": _plain_attention(s, held, table), "lengths": held, "table": table, "slots": slots}


# ---- the framework's calls -------------------------------------------------------------------------------------------------------
def _handle(s):
    """What a program keeps: shape, cache, buffers of outputs, workspace."""
    import paper_2605_23258_b200 as vec
    c = s["case"]
    B, d, dtype = c["batch"], c["head_dim"], _type(c["dtype"])
    kind = vec.VECTOR_BF16 if c["dtype"] == "bf16" else vec.VECTOR_F32
    new = lambda *size, t=dtype: torch.empty(*size, dtype=t, device=_DEVICE)  # noqa: E731
    if c["op"] == "rows":
        shape = vec.Shape(B, 1, c["q_heads"], c["kv_heads"], d, kind, 16, 7, 0.0, int(c["rope"]), _THETA)
        U, N = B * c["kv_heads"], c["tokens"]
        return {"vec": vec, "shape": shape, "q": new(U, c["q_heads"] // c["kv_heads"], N - c["first"], d), "k": new(U, N, d), "v": new(U, N, d) if c["with_v"] else None}
    LH = c["layers"] * c["kv_heads"]
    shape = vec.Shape(B, c["layers"], c["q_heads"], c["kv_heads"], d, kind, 16, 7, 0.0, int(c["rope"]), _THETA)
    cache = vec.Q8Cache(s["ret_pages"], s["apx_pages"], s["ret_table"], s["apx_table"], s["ret_len"], s["apx_len"], None, s.get("apx_pos"))
    h = {"vec": vec, "shape": shape, "cache": cache}
    if c["op"] == "store":
        h["budget"] = vec.vector_plan_budget(c["N"], max(c["N"] * c["percent"] // 100, 16), -1, 16)
        h["ret_k"], h["ret_v"], h["apx_k"] = new(B * LH, s["ret"], d), new(B * LH, s["ret"], d), new(B * LH, s["apx"], d)
        return h
    if c["op"] == "chunk":
        most = max(r for r, _ in _lengths(c)) + c["new"]
        h["ret_k"], h["ret_v"] = new(B * LH, most, d), new(B * LH, most, d)
        return h
    h["out"] = new(*s["q"].shape, t=_type(c["out"]))
    h["ws"] = new(vec.vector_decode_q8_workspace_bytes(shape), t=torch.uint8)
    if c["op"] == "step":
        ints = lambda n: new(n, t=torch.int32)  # noqa: E731
        h["n_free"], h["first_row"], h["row_start"], h["slots"] = ints(1), ints(B), ints(B + 1), ints(B)
        cache.ret_len = ints(B)
    return h


def _run_own(s):
    h = s.get("handle")
    if h is None:
        h = s["handle"] = _handle(s)
    vec, c = h["vec"], s["case"]
    op = c["op"]
    if op == "rows":
        vec.vector_norm_rope(h["shape"], c["tokens"], q=s["q"], q_weight=s["q_weight"], q_first=c["first"], q_out=h["q"], k=s["k"], k_weight=s["k_weight"], k_out=h["k"],
                             v=s["v"] if c["with_v"] else None, v_out=h["v"], pos=s["pos"], eps=1e-6)
        return {"q": h["q"], "k": h["k"], "v": h["v"]} if c["with_v"] else {"q": h["q"], "k": h["k"]}
    if op == "store":
        vec.vector_compact_q8(h["shape"], h["budget"], s["K"], s["V"], s["ret_idx"], s["apx_idx"], h["cache"])
        vec.vector_read_q8(h["shape"], h["cache"], h["ret_k"], h["ret_v"], h["apx_k"])
        return {"ret_k": h["ret_k"], "ret_v": h["ret_v"], "apx_k": h["apx_k"]}
    if op == "chunk":
        vec.vector_append_q8(h["shape"], h["cache"], s["k_new"], s["v_new"], s["first_row"], s["pos"], rotate=c["rope"])
        vec.vector_read_q8(h["shape"], h["cache"], h["ret_k"], h["ret_v"])
        return {"ret_k": h["ret_k"], "ret_v": h["ret_v"]}
    if op == "decode":
        vec.vector_decode_attn_q8(h["shape"], s["q"], h["cache"], s["W"], h["out"], h["ws"])
        return h["out"]
    vec.vector_block_tables(s["ret_len"], s["added"], _ROWS, s["ret_table"], s["free"], s["n_free"], h["cache"].ret_len, h["n_free"], h["first_row"], h["row_start"], h["slots"])
    vec.vector_append_q8(h["shape"], h["cache"], s["k_new"], s["v_new"], h["first_row"], s["pos"], rotate=c["rope"])
    vec.vector_decode_attn_q8(h["shape"], s["q"], h["cache"], s["W"], h["out"], h["ws"])
    return {"out": h["out"], "lengths": h["cache"].ret_len, "table": s["ret_table"], "slots": h["slots"]}


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ---- 64 bits ---------------------------------------------------------------------------------------------------------------------
def _two_to(e):
    """2^e in 64 bits, from its bits (a power function may be off in its last place, which decides ties)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_nearest(x, floor=None):
    """What blocks x [..., 32, d] (64 bits) are held as, by distance, and their scales; floor: scales that they have at the least."""
    most = torch.where(torch.isfinite(x), x.abs(), 0.0).amax((-1, -2), keepdim=True)
    steps = _two_to(torch.arange(_LOW, _HIGH + 1, device=_DEVICE))
    s = steps[torch.bucketize(most / 448, steps).clamp(max=steps.numel() - 1)]
    if floor is not None:
        s = torch.maximum(s, floor)
    t = x.abs() / s
    unit = _two_to(torch.frexp(t.clamp(min=2.0 ** -6)).exponent - 4)      # three mantissa bits
    return torch.sign(x) * torch.round(t / unit) * unit * s, s   # round: ties to even


def _exact_blocks(pages, page, unit, which, d):
    """The values [n][32][d] of blocks of one (layer, KV head), from their bits, and their scales [n][1][1]."""
    tile = _ROWS * d + 32
    flat = pages[page.long(), unit, which * tile:(which + 1) * tile].long()
    r, ch = torch.arange(_ROWS, device=_DEVICE)[:, None], torch.arange(d, device=_DEVICE)[None, :]
    if d == 128:
        place = torch.where(r % 2 == 1, (ch + 64) % 128, ch)
    else:
        place = 16 * (ch % 32 // 8) + 8 * (ch // 32) + ch % 8 + r * 0
    code = flat[:, (r * d + place).flatten()].unflatten(-1, (_ROWS, d))
    e, m = code >> 3 & 15, (code & 7).double()
    v = torch.where(e > 0, _two_to(e - 7) * (1 + m / 8), m * 2.0 ** -9)
    v = torch.where((code & 127) == 127, math.nan, torch.where(code >= 128, -v, v))
    s = _two_to(flat[:, _ROWS * d] - 32)[:, None, None]
    return v * s, s


def _exact_turned(x, pos, way):
    """x [..., d] turned by way * pos, as complex numbers."""
    half = x.shape[-1] // 2
    inv = torch.pow(torch.tensor(_THETA, dtype=torch.float64, device=_DEVICE), -torch.arange(half, device=_DEVICE, dtype=torch.float64) / half)
    angle = way * pos.double()[..., None] * inv
    z = torch.complex(x[..., :half], x[..., half:]) * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], dim=-1)


def _exact_appended(s, b, u, which, n, table):
    """The rows of one (layer, KV head) of sequence b after n new ones, 64 bits."""
    c = s["case"]
    d = c["head_dim"]
    first = _lengths(c)[b][0]
    blocks = (first + n + _ROWS - 1) // _ROWS
    x = torch.zeros(blocks * _ROWS, d, dtype=torch.float64, device=_DEVICE)
    floor = torch.zeros(blocks, 1, 1, dtype=torch.float64, device=_DEVICE)
    have = (first + _ROWS - 1) // _ROWS
    if have:
        old, scales = _exact_blocks(s["ret_pages"], table[:have], u, which, d)
        x[:first] = old.flatten(0, 1)[:first]
        floor[:have] = scales
    new = (s["v_new"] if which else s["k_new"])[b, :n, u].double()
    if c["rope"] and not which:
        new = _exact_turned(new, s["pos"][b, :n], 1)
    x[first:first + n] = new
    return _exact_nearest(x.unflatten(0, (blocks, _ROWS)), floor)[0].flatten(0, 1)[:first + n]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    d = c["head_dim"]
    if c["op"] == "rows":
        if c["batch"] * c["tokens"] * c["q_heads"] * d > 4e8:
            return None

        def heads(x, weight, pos, rope):
            x = x.double().unflatten(-1, (-1, d))
            if weight is not None:
                x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / d + 1e-6) * weight.double()
            return (_exact_turned(x, pos[..., None], 1) if rope else x).transpose(1, 2).flatten(0, 1)
        f = c["first"]
        q = heads(s["q"][:, f:], s["q_weight"], s["pos"][:, f:], c["rope"]).unflatten(0, (-1, c["q_heads"] // c["kv_heads"]))
        got = {"q": q, "k": heads(s["k"], s["k_weight"], s["pos"], c["rope"])}
        return dict(got, v=heads(s["v"], None, None, False)) if c["with_v"] else got
    B, LH = c["batch"], c["layers"] * c["kv_heads"]
    if c["op"] == "store":
        def kept(X, idx):
            got = []
            for u in range(B * LH):
                x = X[u, idx[u].long()].double()
                n = x.shape[0]
                blocks = (n + _ROWS - 1) // _ROWS
                full = torch.zeros(blocks * _ROWS, d, dtype=torch.float64, device=_DEVICE)
                full[:n] = x
                got.append(_exact_nearest(full.unflatten(0, (blocks, _ROWS)))[0].flatten(0, 1)[:n] if n else x)
            return torch.stack(got)
        return {"ret_k": kept(s["K"], s["ret_idx"]), "ret_v": kept(s["V"], s["ret_idx"]), "apx_k": kept(s["K"], s["apx_idx"])}
    if B * LH > 4096:
        return None
    lengths = _lengths(c)
    if c["op"] == "chunk":
        most = max(r for r, _ in lengths) + c["new"]
        got = {"ret_k": torch.zeros(B * LH, most, d, dtype=torch.float64, device=_DEVICE)}
        got["ret_v"] = torch.zeros_like(got["ret_k"])
        for b, (n, _) in enumerate(lengths):
            for u in range(LH):
                for which, name in ((0, "ret_k"), (1, "ret_v")):
                    got[name][b * LH + u, :n + c["new"]] = _exact_appended(s, b, u, which, c["new"], s["ret_table"][b])
        return got
    g = c["q_heads"] // c["kv_heads"]
    out = torch.zeros(B * LH, g, d, dtype=torch.float64, device=_DEVICE)
    for b, (n, m) in enumerate(lengths):
        if n + m == 0:
            continue
        ret, apx = s["ret_table"][b, :(n + _ROWS - 1) // _ROWS], s["apx_table"][b, :(m + _ROWS - 1) // _ROWS]
        for u in range(LH):
            if c["op"] == "step":
                rk, rv = (_exact_appended(s, b, u, which, 1, s["ret_table"][b]) for which in (0, 1))
            else:
                rk, rv = (_exact_blocks(s["ret_pages"], ret, u, which, d)[0].flatten(0, 1)[:n] for which in (0, 1))
            ak = _exact_blocks(s["apx_pages"], apx, u, 0, d)[0].flatten(0, 1)[:m]
            p = torch.softmax(s["q"][b * LH + u].double() @ torch.cat([rk, ak]).T / math.sqrt(d), dim=-1)
            if c["rope"]:
                ak = _exact_turned(ak, s["apx_pos"][apx.long(), u].flatten()[:m], -1)
            k = rk.shape[0]
            out[b * LH + u] = p[:, :k] @ rv + (p[:, k:] @ ak) @ s["W"][u].double().T
    return out if c["op"] == "decode" else {"out": out, "lengths": None, "table": None, "slots": None}
