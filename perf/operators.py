"""The 4-bit paged cache: what serving many requests over a compressed cache calls, and what each call has to compute.

Rows of the mixed cache (retained tokens: key and value; key-only tokens: key) are held in microscaled 4-bit floating point: a group of
16 channels has a scale s of five exponent and three mantissa bits (the smallest with 6 s >= max |x|), each channel the nearest of
{0, 1/2, 1, 3/2, 2, 3, 4, 6} s with its sign, ties to the even code.  Rows live in pages of 64, one list of pages a sequence and tier,
shared by all (layer, KV head).  An operation ("op") of a case is

  tables   vector_block_tables: tables, lengths and slots of all requests after some grew, shrank or ended
  store    vector_compact_q4 of a compressed context into its pages, and vector_read_q4 of the rows
  decode   vector_decode_attn_q4 over the pages
  step     one generated token: vector_block_tables, vector_append_q4, vector_decode_attn_q4
"""
import math

import torch

own = False
_DEVICE = "cuda"
_ROWS = 64                                   # rows of a page
_TOP = 226                                   # code of the largest scale, 10240: 6 s stays within fp16


# ---- cases -----------------------------------------------------------------------------------------------------------------------
def _tables(requests, most, page, kind):
    return {"op": "tables", "requests": requests, "most": most, "page": page, "kind": kind}


def _model(op, batch, layers, q_heads, kv_heads, head_dim, dtype, N, percent, ragged=False, rope=False, out="bf16", empty=0):
    return {"op": op, "batch": batch, "layers": layers, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype,
            "N": N, "percent": percent, "ragged": ragged, "rope": rope, "out": out, "empty": empty}


def listed():
    cases = {
        # a generation step of a batch: every request grows by one row, a page now and then
        "tables_step": _tables(64, 4096, 64, "step"),
        # a scheduler's turn: some requests are admitted with their prompts, some end, the others grow by a row
        "tables_turn": _tables(512, 8192, 64, "turn"),
        # one layer's rows to 4 bits as its prefill ends, an 8B model's attention geometry
        "store_one_layer": _model("store", 1, 1, 32, 8, 128, "bf16", 8192, 20),
        # the whole compressed cache of a 32-layer model
        "store_32_layers": _model("store", 1, 32, 32, 8, 128, "bf16", 32768, 20),
        # fp32 rows of 64 channels, a length that is no multiple of anything
        "store_fp32_head64": _model("store", 2, 4, 8, 4, 64, "fp32", 15013, 25),
        # one layer's step of a single request: the latency of a generated token is this, times the layers
        "step_one_layer": _model("step", 1, 1, 32, 8, 128, "bf16", 8192, 20),
        # one layer's step of a batch of requests of all lengths, some places of the batch not taken
        "step_batch64_ragged": _model("step", 64, 1, 32, 8, 128, "bf16", 8192, 20, ragged=True, empty=5),
        # all 32 layers of eight requests in one call
        "decode_batch8_32_layers": _model("decode", 8, 32, 32, 8, 128, "bf16", 16384, 10, ragged=True),
        # a 70B model's geometry at its longest context: the largest call
        "decode_80_layers": _model("decode", 1, 80, 64, 8, 128, "bf16", 131072, 5),
        # rotary keys, which the map sees turned back
        "decode_rope_batch16": _model("decode", 16, 1, 32, 8, 128, "bf16", 30001, 20, rope=True),
        # 64-channel heads, results in fp32
        "decode_head64": _model("decode", 4, 16, 32, 8, 64, "bf16", 16384, 20, ragged=True, out="fp32"),
        # fp32 queries and map
        "decode_fp32": _model("decode", 2, 2, 8, 2, 128, "fp32", 4001, 25, ragged=True, out="fp32"),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["tables", "store", "store", "decode", "decode", "decode", "decode", "step", "step"])
    if op == "tables":
        return _tables(_log_int(rng, 1, 2048), _log_int(rng, 16, 8192), rng.choice([16, 32, 64, 64, 64, 128, 100]), rng.choice(["step", "turn"]))
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    kv_heads, g, head_dim = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 3, 4, 4, 8]), rng.choice([64, 128, 128])
    N, percent = _log_int(rng, 300, 131072), rng.choice([5, 10, 15, 20, 25, 30, 40])
    batch, layers = _log_int(rng, 1, 64), _log_int(rng, 1, 80)
    if op == "store":
        batch = min(batch, 4)
    # cut until the keys of the longest sequences take at most 1.1 GB in 4 bits, and a stored context at most 4 GB of rows
    bits = {"store": 8.0 if dtype == "bf16" else 16.0}.get(op, 2.0)
    most = (1.6e9 if op != "store" else 2.0e9) / (bits * head_dim * kv_heads * (N if op == "store" else N * percent / 100.0 + 64))
    if dtype == "fp32" and op != "store":
        most = min(most, 1e6 / (kv_heads * (N * percent / 100.0 + 64)))
    while batch * layers > max(most, 1):
        if layers >= batch:
            layers = (layers + 1) // 2
        else:
            batch = (batch + 1) // 2
    return _model(op, batch, layers, kv_heads * g, kv_heads, head_dim, dtype, N, percent, ragged=op != "store" and rng.random() < 0.6,
                  rope=op != "store" and rng.random() < 0.3, out="fp32" if dtype == "fp32" else rng.choice(["bf16", "bf16", "fp32"]),
                  empty=rng.choice([0, 0, 1]) if op != "store" and batch > 2 else 0)


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


def work(c):
    if c["op"] == "tables":
        lengths, added, pages = _requests(c)
        rows = sum(max(a, 0) for a in added)
        return {"bytes": 4.0 * (5 * len(lengths) + rows + pages), "flops": 0.0}
    LH, d, es = c["layers"] * c["kv_heads"], c["head_dim"], 2 if c["dtype"] == "bf16" else 4
    held = d / 2 + d / 16
    if c["op"] == "store":
        ret, apx = _tiers(c["N"], c["percent"])
        rows = c["batch"] * LH * (2 * ret + apx)
        return {"bytes": float(rows * (2 * d * es + held)) + c["batch"] * LH * (ret + apx) * 8, "flops": 0.0}
    lengths = _lengths(c)
    extra = 1 if c["op"] == "step" else 0
    ret, apx = sum(r + (extra if r else 0) for r, _ in lengths), sum(a for _, a in lengths)
    g = c["q_heads"] // c["kv_heads"]
    heads = c["batch"] * LH * g
    out = 2 if c["out"] == "bf16" else 4
    turned = 4 * apx * LH if c["rope"] else 0
    return {"bytes": float(LH * (2 * ret + apx) * held + LH * d * d * es + heads * d * (es + out) + turned + extra * c["batch"] * LH * 2 * d * es),
            "flops": float(2 * g * d * LH * (2 * ret + 2 * apx) + 2 * heads * d * d)}


# ---- what a program has in hand --------------------------------------------------------------------------------------------------
def _requests(c):
    """Lengths, changes and the number of pages involved, of a tables case."""
    r = torch.Generator().manual_seed(c["requests"] * 7 + c["most"])
    n, most, page = c["requests"], c["most"], c["page"]
    lengths = torch.randint(1, most + 1, (n,), generator=r)
    added = torch.ones(n, dtype=torch.int64)
    if c["kind"] == "turn":
        what = torch.rand(n, generator=r)
        prompt = torch.randint(1, most + 1, (n,), generator=r)
        lengths = torch.where(what < 0.3, 0, lengths)
        added = torch.where(what < 0.3, prompt, torch.where(what < 0.45, -lengths, torch.where(what < 0.55, -torch.minimum(lengths, torch.tensor(5)), added)))
    new = lengths + added
    pages = int(((new + page - 1) // page - (lengths + page - 1) // page).abs().sum())
    return lengths.tolist(), added.tolist(), pages


def _prepare_tables(c, seed):
    gen = torch.Generator().manual_seed(seed * 7919 + 3)
    lengths, added, _ = _requests(c)
    mix = torch.randperm(len(lengths), generator=gen)
    lengths, added = torch.tensor(lengths)[mix], torch.tensor(added)[mix]
    page = c["page"]
    have = (lengths + page - 1) // page
    width = (c["most"] + page - 1) // page + 2
    order = torch.randperm(int(have.sum()) + len(lengths) * width // 2 + 64, generator=gen).int()
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    taken = torch.arange(width)[None, :] < have[:, None]
    table[taken] = order[:int(have.sum())]
    free = order[int(have.sum()):]
    stack = torch.full((order.numel(),), -1, dtype=torch.int32)
    stack[:free.numel()] = free
    total = int(added.clamp(min=0).sum())
    on = lambda t: t.to(_DEVICE)  # noqa: E731
    return {"lengths": on(lengths.int()), "added": on(added.int()), "table": on(table), "free": on(stack),
            "n_free": torch.tensor([free.numel()], dtype=torch.int32, device=_DEVICE), "slots": max(total, 1), "page": page}


def _rand(gen, *shape):
    return torch.rand(*shape, generator=gen, device=_DEVICE)


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


def _rows(gen, sigma, n, dtype):
    return (torch.randn(sigma.shape[0], n, sigma.shape[2], generator=gen, device=_DEVICE) * sigma).to(dtype)


def _prepare_store(c, seed):
    gen = torch.Generator(device=_DEVICE).manual_seed(seed * 7919 + 5)
    B, LH, d, N, dtype = c["batch"], c["layers"] * c["kv_heads"], c["head_dim"], c["N"], _type(c["dtype"])
    ret, apx = _tiers(N, c["percent"])
    sigma_k, _ = _law(c, gen)
    K = torch.empty(B * LH, N, d, dtype=dtype, device=_DEVICE)
    V = torch.empty_like(K)
    for u in range(0, B * LH, c["kv_heads"]):
        at = u % LH
        K[u:u + c["kv_heads"]] = _rows(gen, sigma_k[at:at + c["kv_heads"]], N, dtype)
        V[u:u + c["kv_heads"]] = (torch.randn(c["kv_heads"], N, d, generator=gen, device=_DEVICE) * _spread(gen, (c["kv_heads"], N, 1), 0.02, 2.0)).to(dtype)
    kept = torch.argsort(_rand(gen, B * LH, N), dim=1)[:, :ret + apx].int()
    ret_idx, apx_idx = kept[:, :ret].sort(dim=1).values.contiguous(), kept[:, ret:].sort(dim=1).values.contiguous()
    s = {"K": K, "V": V, "ret_idx": ret_idx, "apx_idx": apx_idx, "ret": ret, "apx": apx}
    s.update(_pools(c, gen, [(ret, apx)] * B, 0))
    s["ret_slots"], s["apx_slots"] = (_slots_of(s[t + "_table"], n) for t, n in (("ret", ret), ("apx", apx)))
    return s


def _slots_of(table, n):
    """The slots of the first n rows of every sequence, [batch][n]."""
    i = torch.arange(n, device=_DEVICE)
    return (table[:, i // _ROWS] * _ROWS + (i % _ROWS)[None, :]).int().contiguous()


def _pools(c, gen, lengths, more):
    """Pages of both tiers with whatever was in memory, and tables that take them in no order."""
    LH, tile = c["layers"] * c["kv_heads"], _ROWS * (c["head_dim"] // 2 + c["head_dim"] // 16)
    s = {}
    for tier, parts, rows in (("ret", 2, [r + more for r, _ in lengths]), ("apx", 1, [a for _, a in lengths])):
        have = [(n + _ROWS - 1) // _ROWS for n in rows]
        width, pages = max(max(have), 1), sum(have) + 3
        order = torch.randperm(pages, generator=gen, device=_DEVICE).int()
        table = torch.full((c["batch"], width), -1, dtype=torch.int32, device=_DEVICE)
        at = 0
        for b, h in enumerate(have):
            table[b, :h] = order[at:at + h]
            at += h
        s[tier + "_table"] = table
        s[tier + "_pages"] = torch.randint(0, 256, (pages, LH, parts * tile), generator=gen, device=_DEVICE, dtype=torch.uint8)
    return s


def _prepare_decode(c, seed):
    gen = torch.Generator(device=_DEVICE).manual_seed(seed * 7919 + 7)
    B, L, H, d, dtype = c["batch"], c["layers"], c["kv_heads"], c["head_dim"], _type(c["dtype"])
    LH, g, more = L * H, c["q_heads"] // c["kv_heads"], 1 if c["op"] == "step" else 0
    lengths = _lengths(c)
    sigma_k, sigma_q = _law(c, gen)
    s = _pools(c, gen, lengths, more)
    for i, tier in ((0, "ret"), (1, "apx")):
        s[tier + "_len"] = torch.tensor([n[i] for n in lengths], dtype=torch.int32, device=_DEVICE)
    s["apx_pos"] = torch.randint(0, c["N"], (s["apx_pages"].shape[0], LH, _ROWS), generator=gen, device=_DEVICE, dtype=torch.int32)
    for b, (ret, apx) in enumerate(lengths):
        for at in range(0, LH, H):
            part = slice(at, at + H)
            for n, pages, tier, is_v in ((ret, "ret_pages", "ret", 0), (ret, "ret_pages", "ret", 1), (apx, "apx_pages", "apx", 0)):
                if n:
                    x = torch.randn(H, n, d, generator=gen, device=_DEVICE)
                    x *= _spread(gen, (H, n, 1), 0.02, 2.0) if is_v else sigma_k[part]
                    _put(s[pages], _slots_of(s[tier + "_table"][b:b + 1], n)[0], part, is_v, x)
    s["q"] = torch.empty(B * LH, g, d, dtype=dtype, device=_DEVICE)
    for b in range(B):
        s["q"][b * LH:(b + 1) * LH] = _rows(gen, sigma_q, g, dtype)
    s["W"] = (torch.randn(LH, d, d, generator=gen, device=_DEVICE) / math.sqrt(d)).to(dtype)
    if more:
        s["k_new"], s["v_new"] = (_rows(gen, sigma_k, B, dtype).transpose(0, 1).reshape(B * LH, d).contiguous(),
                                  torch.randn(B * LH, d, generator=gen, device=_DEVICE).to(dtype))
        s["added"] = (s["ret_len"] > 0).int()
        s["pos"] = torch.full((B,), c["N"], dtype=torch.int32, device=_DEVICE)
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
    s = {"tables": _prepare_tables, "store": _prepare_store}.get(case["op"], _prepare_decode)(case, seed)
    s["case"] = case
    return s


# ---- plain forms -----------------------------------------------------------------------------------------------------------------
_constants = {}


def _constant(name, make):
    if name not in _constants:
        _constants[name] = make().to(_DEVICE)
    return _constants[name]


def _scale_values():
    """The values of the 256 scale codes: five exponent bits of bias 15 and three mantissa bits, none of sign; exponent 31 is not a number."""
    code = torch.arange(256)
    e, m = code // 8, (code % 8).float()
    v = torch.where(e > 0, (1 + m / 8) * torch.exp2(e.float() - 15), m / 8 * 2.0 ** -14)
    return torch.where(e == 31, float("nan"), v)


def _code_values():
    v = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    return torch.cat([v, -v])


def _stored_order(d):
    """Where each channel lies in a row: four pieces, each a run of low channels and the run half a head above it."""
    c = torch.arange(d)
    low, half, run = c % (d // 2), c // (d // 2), d // 8
    return low // run * (2 * run) + half * run + low % run


def _group_order(d):
    g, half = torch.arange(d // 16), d // 32
    return 2 * (g % half) + g // half


def _quantise(x):
    """x [..., d] -> codes [..., d] and scale codes [..., d / 16], both in the channels' own order."""
    x = x.float().unflatten(-1, (-1, 16))
    scales = _constant("scales", _scale_values)
    size = x.abs()
    most = size.amax(-1)
    bad = torch.isnan(most)
    sc = torch.searchsorted(6 * scales[:_TOP + 1].contiguous(), torch.where(bad, 0, most)).clamp(max=_TOP)
    s = scales[sc][..., None]
    code = sum((size > b * s) if up else (size >= b * s) & (s > 0) for b, up in ((0.25, 1), (0.75, 0), (1.25, 1), (1.75, 0), (2.5, 1), (3.5, 0), (5.0, 1)))
    code = code + 8 * (x < 0)
    return code.flatten(-2).to(torch.uint8), torch.where(bad, 255, sc).to(torch.uint8)


def _parts(pages, d, parts):
    """Views of the codes [P][LH][parts][64][d / 2] and the scales [P][LH][parts][64][d / 16] of pages."""
    t = pages.unflatten(-1, (parts, -1))
    cut = _ROWS * d // 2
    return t[..., :cut].unflatten(-1, (_ROWS, -1)), t[..., cut:].unflatten(-1, (_ROWS, -1))


def _put(pages, slots, part, is_v, x):
    """Rows x [h][n][d] of the heads `part` into the slots [n]."""
    d = x.shape[-1]
    tile = _ROWS * (d // 2 + d // 16)
    codes, scales = _quantise(x)
    stored = torch.empty_like(codes)
    stored[..., _constant(("order", d), lambda: _stored_order(d))] = codes
    stored = stored[..., 0::2] | stored[..., 1::2] << 4
    sc = torch.empty_like(scales)
    sc[..., _constant(("groups", d), lambda: _group_order(d))] = scales
    to_codes, to_scales = _parts(pages, d, pages.shape[-1] // tile)
    page, row = slots.long() // _ROWS, slots.long() % _ROWS
    to_codes[:, part, is_v][page, :, row] = stored.transpose(0, 1)
    to_scales[:, part, is_v][page, :, row] = sc.transpose(0, 1)


def _values(codes, scales):
    """What rows of stored bytes stand for, fp32."""
    d = codes.shape[-1] * 2
    nibbles = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    v = _constant("codes", _code_values)[nibbles.int()[..., _constant(("order", d), lambda: _stored_order(d))]]
    s = _constant("scales", _scale_values)[scales.int()[..., _constant(("groups", d), lambda: _group_order(d))]]
    return (v.unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)


def _held(pages, table, lengths, d, which, parts):
    """Rows of every sequence, [batch][LH][width * 64][d], with zeros behind a sequence's last row, and which are its rows."""
    codes, scales = _parts(pages, d, parts)
    at = table.long().clamp(0, pages.shape[0] - 1)
    x = _values(codes[:, :, which][at], scales[:, :, which][at])                  # [batch][width][LH][64][d]
    x = x.transpose(1, 2).flatten(2, 3)
    there = torch.arange(x.shape[2], device=_DEVICE)[None, :] < lengths[:, None]
    return torch.where(there[:, None, :, None], x, 0.0), there


def _turned_back(k, pos):
    half = k.shape[-1] // 2
    inv = 10000.0 ** (-torch.arange(half, device=_DEVICE, dtype=torch.float64) / half)
    angle = (pos.double()[..., None] * inv).remainder(2 * math.pi)
    cs, sn = torch.cos(angle).float(), torch.sin(angle).float()
    x, y = k[..., :half], k[..., half:]
    return torch.cat([x * cs + y * sn, y * cs - x * sn], dim=-1)


def _plain_attention(s, ret_len, ret_table):
    c = s["case"]
    B, LH, d = c["batch"], c["layers"] * c["kv_heads"], c["head_dim"]
    q = s["q"].float().unflatten(0, (B, LH)) * (1 / math.sqrt(d))
    rk, there_r = _held(s["ret_pages"], ret_table, ret_len, d, 0, 2)
    ak, there_a = _held(s["apx_pages"], s["apx_table"], s["apx_len"], d, 0, 1)
    logit = torch.cat([q @ rk.transpose(-1, -2), q @ ak.transpose(-1, -2)], dim=-1)
    there = torch.cat([there_r, there_a], dim=-1)[:, None, None, :]
    logit = torch.where(there, logit, -math.inf)
    most = logit.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(logit - most)
    total = p.sum(-1, keepdim=True)
    n = rk.shape[2]
    del rk
    rv, _ = _held(s["ret_pages"], ret_table, ret_len, d, 1, 2)
    o = p[..., :n] @ rv
    del rv
    if c["rope"]:
        at = s["apx_table"].long().clamp(0, s["apx_pages"].shape[0] - 1)
        ak = _turned_back(ak, s["apx_pos"][at].transpose(1, 2).flatten(2, 3))
    o = o + (p[..., n:] @ ak) @ s["W"].float().transpose(-1, -2)
    o = torch.where(total > 0, o / total.clamp(min=1e-30), 0.0)
    return o.flatten(0, 1).to(_type(c["out"]))


def _plain_tables(lengths, added, table, free, n_free, page, n_slots):
    """New lengths, table, stack of free pages and its height, first new rows, row starts and slots."""
    old, grow, width = lengths.long().clamp(min=0), added.long(), table.shape[1]
    have = (old + page - 1) // page
    new = (old + grow).clamp(min=0)
    wanted = ((new + page - 1) // page).clamp(max=width)
    back = (have - wanted).clamp(min=0)
    before_back = torch.cumsum(back, 0) - back
    height = n_free.long() + back.sum()
    i = torch.arange(width, device=_DEVICE)[None, :]
    gone = (i >= wanted[:, None]) & (i < have[:, None]) & (grow < 0)[:, None]
    stack = torch.cat([free, free[:1]])
    to = torch.where(gone, n_free.long() + before_back[:, None] + i - wanted[:, None], free.numel())
    stack.scatter_(0, to.flatten(), table.flatten())
    stack = stack[:-1]
    need = torch.where(grow > 0, (wanted - have).clamp(min=0), 0)
    before = torch.cumsum(need, 0) - need
    got = torch.minimum(need, (height - before).clamp(min=0))
    fresh = (i >= have[:, None]) & (i < (have + got)[:, None])
    table = torch.where(fresh, stack[(height - 1 - before[:, None] - (i - have[:, None])).clamp(0, stack.numel() - 1)], table)
    held = torch.where(grow > 0, torch.minimum(new, (have + got) * page), new)
    rows = grow.clamp(min=0)
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=_DEVICE), torch.cumsum(rows, 0)])
    k = torch.arange(n_slots, device=_DEVICE)
    b = torch.searchsorted(start, k, right=True) - 1
    there = b < lengths.numel()
    b = b.clamp(max=lengths.numel() - 1)
    row = old[b] + k - start[b]
    slots = torch.where(there & (row < held[b]), table[b, (row // page).clamp(max=width - 1)] * page + row % page, -1)
    return held.int(), table, stack, (height - got.sum()).int().reshape(1), old.int(), start.int(), slots.int()


def _run_plain(s):
    c = s["case"]
    if c["op"] == "tables":
        held, table, stack, height, first, start, slots = _plain_tables(s["lengths"], s["added"], s["table"], s["free"], s["n_free"], s["page"], s["slots"])
        return {"lengths": held, "table": table, "free": stack, "n_free": height, "first_row": first, "row_start": start, "slots": slots}
    if c["op"] == "store":
        B, LH, d = c["batch"], c["layers"] * c["kv_heads"], c["head_dim"]
        rows = lambda X, idx: X.gather(1, idx.long()[..., None].expand(-1, -1, d)).unflatten(0, (B, LH)).transpose(0, 1).flatten(1, 2)  # noqa: E731  [LH][batch * n][d]
        heads = slice(0, LH)
        _put(s["ret_pages"], s["ret_slots"].flatten(), heads, 0, rows(s["K"], s["ret_idx"]))
        _put(s["ret_pages"], s["ret_slots"].flatten(), heads, 1, rows(s["V"], s["ret_idx"]))
        _put(s["apx_pages"], s["apx_slots"].flatten(), heads, 0, rows(s["K"], s["apx_idx"]))

        def back(pages, slots, which, parts):
            codes, scales = _parts(pages, d, parts)
            at = slots.long()
            x = _values(codes[:, :, which][at // _ROWS, :, at % _ROWS], scales[:, :, which][at // _ROWS, :, at % _ROWS])    # [batch][n][LH][d]
            return x.transpose(1, 2).flatten(0, 1).to(_type(c["dtype"]))
        return {"ret_k": back(s["ret_pages"], s["ret_slots"], 0, 2), "ret_v": back(s["ret_pages"], s["ret_slots"], 1, 2),
                "apx_k": back(s["apx_pages"], s["apx_slots"], 0, 1)}
    if c["op"] == "decode":
        return _plain_attention(s, s["ret_len"], s["ret_table"])
    B, LH, d = c["batch"], c["layers"] * c["kv_heads"], c["head_dim"]
    held, table, _, _, _, _, slots = _plain_tables(s["ret_len"], s["added"], s["ret_table"], s["free"], s["n_free"], _ROWS, B)
    # the row of a request: slots lie behind one another for the requests that grow; a place that nobody has taken writes what another one writes
    mine = (torch.cumsum(s["added"], 0) - s["added"]).long().clamp(max=B - 1)
    taken = s["added"] > 0
    any_one = torch.argmax(taken.int()).reshape(1)
    who = torch.where(taken, torch.arange(B, device=_DEVICE), any_one)
    at = slots[mine[who]]
    for is_v, new in ((0, s["k_new"]), (1, s["v_new"])):
        _put(s["ret_pages"], at, slice(0, LH), is_v, new.unflatten(0, (B, LH))[who].transpose(0, 1))
    return {"out": _plain_attention(s, held, table), "lengths": held, "table": table, "slots": slots}


# ---- the framework's calls -------------------------------------------------------------------------------------------------------
def _handle(s):
    """What a program keeps: shape, cache, buffers of outputs, workspace."""
    import paper_2605_23258_b200 as vec
    c = s["case"]
    if c["op"] == "tables":
        B = s["lengths"].numel()
        ints = lambda n: torch.empty(n, dtype=torch.int32, device=_DEVICE)  # noqa: E731
        return {"vec": vec, "lengths": ints(B), "n_free": ints(1), "first_row": ints(B), "row_start": ints(B + 1), "slots": ints(s["slots"])}
    B, LH, d, dtype = c["batch"], c["layers"] * c["kv_heads"], c["head_dim"], _type(c["dtype"])
    shape = vec.Shape(B, c["layers"], c["q_heads"], c["kv_heads"], d, vec.VECTOR_BF16 if c["dtype"] == "bf16" else vec.VECTOR_F32, 16, 7, 0.0, int(c["rope"]), 10000.0)
    lengths = [torch.zeros(B, dtype=torch.int32, device=_DEVICE) for _ in range(2)]
    cache = vec.Q4Cache(s["ret_pages"], s["apx_pages"], s["ret_table"], s["apx_table"], s.get("ret_len", lengths[0]), s.get("apx_len", lengths[1]),
                        None, s.get("apx_pos"))
    h = {"vec": vec, "shape": shape, "cache": cache}
    if c["op"] == "store":
        h["budget"] = vec.vector_plan_budget(c["N"], max(c["N"] * c["percent"] // 100, 16), -1, 16)
        h["ret_k"], h["ret_v"] = (torch.empty(B * LH, s["ret"], d, dtype=dtype, device=_DEVICE) for _ in range(2))
        h["apx_k"] = torch.empty(B * LH, s["apx"], d, dtype=dtype, device=_DEVICE)
        return h
    h["out"] = torch.empty(s["q"].shape, dtype=_type(c["out"]), device=_DEVICE)
    h["ws"] = torch.empty(vec.vector_decode_q4_workspace_bytes(shape), dtype=torch.uint8, device=_DEVICE)
    if c["op"] == "step":
        ints = lambda n: torch.empty(n, dtype=torch.int32, device=_DEVICE)  # noqa: E731
        h["n_free"], h["first_row"], h["row_start"], h["slots"] = ints(1), ints(B), ints(B + 1), ints(B)
        cache.ret_len = ints(B)
    return h


def _run_own(s):
    h = s.get("handle")
    if h is None:
        h = s["handle"] = _handle(s)
    vec, op = h["vec"], s["case"]["op"]
    if op == "tables":
        vec.vector_block_tables(s["lengths"], s["added"], s["page"], s["table"], s["free"], s["n_free"], h["lengths"], h["n_free"], h["first_row"], h["row_start"], h["slots"])
        return {"lengths": h["lengths"], "table": s["table"], "free": s["free"], "n_free": h["n_free"], "first_row": h["first_row"],
                "row_start": h["row_start"], "slots": h["slots"]}
    if op == "store":
        vec.vector_compact_q4(h["shape"], h["budget"], s["K"], s["V"], s["ret_idx"], s["apx_idx"], h["cache"], s["ret_slots"], s["apx_slots"])
        vec.vector_read_q4(h["shape"], h["cache"], s["ret_slots"], h["ret_k"], h["ret_v"], s["apx_slots"], h["apx_k"])
        return {"ret_k": h["ret_k"], "ret_v": h["ret_v"], "apx_k": h["apx_k"]}
    if op == "decode":
        vec.vector_decode_attn_q4(h["shape"], s["q"], h["cache"], s["W"], h["out"], h["ws"])
        return h["out"]
    vec.vector_block_tables(s["ret_len"], s["added"], _ROWS, s["ret_table"], s["free"], s["n_free"], h["cache"].ret_len, h["n_free"], h["first_row"], h["row_start"], h["slots"])
    vec.vector_append_q4(h["shape"], h["cache"], s["k_new"], s["v_new"], h["row_start"], h["slots"], s["pos"])
    vec.vector_decode_attn_q4(h["shape"], s["q"], h["cache"], s["W"], h["out"], h["ws"])
    return {"out": h["out"], "lengths": h["cache"].ret_len, "table": s["ret_table"], "slots": h["slots"]}


def run(state):
    if own:
        return _run_own(state)
    return _run_plain(state)


# ---- 64 bits ---------------------------------------------------------------------------------------------------------------------
def _exact_scale(code):
    """Value of scale codes, from their bits."""
    code = code.long()
    e, m = code >> 3, (code & 7).double()
    v = torch.ldexp(torch.where(e > 0, m + 8, m), torch.where(e > 0, e, torch.ones_like(e)) - 18)
    return torch.where(e == 31, math.nan, v)


def _exact_number(nibble):
    """Value of codes, from their bits: sign, two exponent bits, one mantissa bit."""
    n = nibble.long()
    e, m = n >> 1 & 3, (n & 1).double()
    v = torch.where(e > 0, torch.ldexp(1 + m / 2, e - 1), m / 2)
    return torch.where(n >= 8, -v, v)


def _exact_rows(pages, slots, unit, which, d):
    """Rows [n][d] of one (layer, KV head), 64 bits, channel by channel from the definition of the layout."""
    tile = _ROWS * (d // 2 + d // 16)
    flat = pages[:, unit, which * tile:(which + 1) * tile]
    page, row = slots.long() // _ROWS, slots.long() % _ROWS
    c = torch.arange(d, device=_DEVICE)
    low, up = c % (d // 2), c // (d // 2)
    place = low // (d // 8) * (d // 4) + up * (d // 8) + low % (d // 8)
    byte = flat[page[:, None], row[:, None] * (d // 2) + place[None, :] // 2].long()
    nibble = byte >> (4 * (place % 2))[None, :] & 15
    group = c // 16
    sc = flat[page[:, None], _ROWS * d // 2 + row[:, None] * (d // 16) + (2 * (group % (d // 32)) + group // (d // 32))[None, :]]
    return _exact_number(nibble) * _exact_scale(sc)


def _exact_nearest(x):
    """What x [n][d] is held as, 64 bits: the nearest multiples of the scale, by distance."""
    x = x.double().reshape(x.shape[0], -1, 16)
    codes = torch.arange(_TOP + 1, device=x.device)
    scales = _exact_scale(codes)
    most = x.abs().amax(-1)
    s = scales[torch.bucketize(most / 6, scales).clamp(max=_TOP)][..., None]
    t = torch.where(s > 0, x.abs() / s, 0.0)
    step = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))
    held = (torch.round(t / step) * step).clamp(max=6.0)        # round: ties to even, which are the even codes
    return (torch.sign(x) * held * s).flatten(1)


def exact(case, seed):
    if case["op"] == "tables":
        return None
    s = prepare(case, seed)
    c = case
    B, LH, d = c["batch"], c["layers"] * c["kv_heads"], c["head_dim"]
    if c["op"] == "store":
        got = {"ret_k": [], "ret_v": [], "apx_k": []}
        for u in range(B * LH):
            got["ret_k"].append(_exact_nearest(s["K"][u, s["ret_idx"][u].long()]))
            got["ret_v"].append(_exact_nearest(s["V"][u, s["ret_idx"][u].long()]))
            got["apx_k"].append(_exact_nearest(s["K"][u, s["apx_idx"][u].long()]))
        return {k: torch.stack(v) for k, v in got.items()}
    if B * LH > 4096:
        return None
    g, lengths = c["q_heads"] // c["kv_heads"], _lengths(c)
    out = torch.zeros(B * LH, g, d, dtype=torch.float64, device=_DEVICE)
    half = d // 2
    inv = torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=_DEVICE), -torch.arange(half, device=_DEVICE, dtype=torch.float64) / half)
    for b, (n, m) in enumerate(lengths):
        if n + m == 0:
            continue
        ret, apx = _slots_of(s["ret_table"][b:b + 1], n)[0], _slots_of(s["apx_table"][b:b + 1], m)[0]
        for u in range(LH):
            at = b * LH + u
            rk, rv, ak = _exact_rows(s["ret_pages"], ret, u, 0, d), _exact_rows(s["ret_pages"], ret, u, 1, d), _exact_rows(s["apx_pages"], apx, u, 0, d)
            if c["op"] == "step":
                rk, rv = torch.cat([rk, _exact_nearest(s["k_new"][at:at + 1])]), torch.cat([rv, _exact_nearest(s["v_new"][at:at + 1])])
            p = torch.softmax(s["q"][at].double() @ torch.cat([rk, ak]).T / math.sqrt(d), dim=-1)
            if c["rope"]:
                angle = s["apx_pos"][apx.long() // _ROWS, u, apx.long() % _ROWS].double()[:, None] * inv
                z = torch.complex(ak[:, :half], ak[:, half:]) * torch.polar(torch.ones_like(angle), -angle)
                ak = torch.cat([z.real, z.imag], dim=1)
            k = rk.shape[0]
            out[at] = p[:, :k] @ rv + (p[:, k:] @ ak) @ s["W"][u].double().T
    return out if c["op"] == "decode" else {"out": out, "lengths": None, "table": None, "slots": None}
