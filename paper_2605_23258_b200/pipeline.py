"""Buffer ownership and call order around the C-ABI: no arithmetic of the method here.

``Compressor`` allocates (through PyTorch) every buffer the device calls need
once, then ``compress`` issues vector_score -> vector_route -> vector_compact on
the current stream and ``decode`` issues vector_decode_attn.  ``calibrate_maps``
fans vector_calibrate (host least squares) out over host threads.
"""
from __future__ import annotations

from concurrent.futures import ThreadPoolExecutor
import os

import torch

from . import binding as B


def calibrate_maps(kv_pairs, lam: float, threads: int | None = None, want_r2: bool = False):
    """kv_pairs: iterable of (K [n][d], V [n][d]) host tensors, one per (layer, KV head).
    Returns W fp32 [LH][d][d] (y = W x), and the list of R^2 when asked."""
    pairs = list(kv_pairs)
    threads = threads or min(len(pairs), os.cpu_count() or 1)
    with ThreadPoolExecutor(max_workers=max(threads, 1)) as ex:
        res = list(ex.map(lambda kv: B.vector_calibrate(kv[0], kv[1], lam, want_r2), pairs))
    if want_r2:
        return torch.stack([r[0] for r in res]), [r[1] for r in res]
    return torch.stack(res)


def project(shape: B.Shape, n_tokens: int, q, k, v, q_weight=None, k_weight=None, pos=None, eps: float = 1e-6, q_first: int = 0):
    """A layer's projections, rows of a token's heads or parts of wider rows, as the rows that the calls take: q [U][g][n_tokens - q_first][d], k and v [U][n_tokens][d],
    queries and keys normed where they have a weight and turned by their positions where the shape has rotary ones."""
    rows = lambda *size: torch.empty(*size, shape.head_dim, dtype=shape.torch_dtype, device=k.device)  # noqa: E731
    got = rows(shape.units, shape.group, n_tokens - q_first), rows(shape.units, n_tokens), rows(shape.units, n_tokens)
    B.vector_norm_rope(shape, n_tokens, q, k, v, *got, q_weight, k_weight, pos, q_first, eps)
    return got


class Compressor:
    """Owns the device buffers of one (shape, budget) and issues the hot-path calls."""

    def __init__(self, shape: B.Shape, budget: B.Budget, extra_rows: int = 0, device="cuda",
                 keep_eps: bool = False):
        self.shape, self.budget, self.device = shape, budget, device
        U, N = shape.units, budget.n_tokens
        self.scores = torch.empty(U, N, dtype=torch.float32, device=device)
        self.tier = torch.empty(U, N, dtype=torch.uint8, device=device)
        self.ret_idx = torch.empty(U, max(budget.n_ret, 1), dtype=torch.int32, device=device)[:, :budget.n_ret]
        self.apx_idx = torch.empty(U, max(budget.n_apx, 1), dtype=torch.int32, device=device)[:, :budget.n_apx]
        self.ret_idx = self.ret_idx.contiguous()
        self.apx_idx = self.apx_idx.contiguous()
        self.eps = torch.empty(U, budget.n_pool, dtype=torch.float32, device=device) if keep_eps else None
        self.pool_idx = torch.empty(U, budget.n_pool, dtype=torch.int32, device=device) if keep_eps else None
        self.cache = B.alloc_cache(shape, budget, extra_rows, device)
        self.ws = B.alloc_workspace(shape, budget, device)

    def project(self, q, k, v, q_weight=None, k_weight=None, pos=None, eps: float = 1e-6):
        """The layers' projections of a whole context, [B][L][N] rows, as (Q_obs, K, V) of compress."""
        N = self.budget.n_tokens
        return project(self.shape, N, q, k, v, q_weight, k_weight, pos, eps, q_first=N - self.shape.window)

    def score(self, Q_obs, K):
        B.vector_score(self.shape, Q_obs, K, self.budget.n_tokens, self.scores, None, self.ws)

    def route(self, K, V, W):
        B.vector_route(self.shape, self.budget, self.scores, K, V, W, self.tier, self.ret_idx, self.apx_idx,
                       self.eps, self.pool_idx, self.ws)

    def compact(self, K, V):
        self.cache.n_ret, self.cache.n_apx = self.budget.n_ret, self.budget.n_apx
        B.vector_compact(self.shape, self.budget, K, V, self.ret_idx, self.apx_idx, self.cache)

    def compress(self, Q_obs, K, V, W):
        """Prefill-time compression of all units: score, route, compact (asynchronous)."""
        self.score(Q_obs, K)
        self.route(K, V, W)
        self.compact(K, V)
        return self.cache

    def append(self, k_new, v_new, pos: int):
        """Keeps a generated token in full: writes its row behind the retained pool."""
        c, sh = self.cache, self.shape
        # One kernel copies plain rows on the current device; the rest of what can be assigned to the rows is assigned: other types,
        # strided rows, rows off a 16-byte boundary.
        if B.append_rows(sh, c, k_new, v_new, pos):
            c.n_ret += 1
            return
        rk, rv = c.ret_k, c.ret_v
        U, cap, d = rk.shape
        if c.n_ret >= cap:
            raise ValueError("retained pool is full")
        # A shape or a cache of a class that packs in its own way: the entry point itself says what it refuses.
        if (type(pos) is int and -2**31 <= pos < 2**31 and type(k_new) is type(v_new) is torch.Tensor
                and k_new.shape == v_new.shape == (U, d) and U == sh.units and d == sh.head_dim
                and k_new.get_device() == v_new.get_device() == rv.get_device() == rk.get_device() >= 0 and rk.get_device() == torch.cuda.current_device()
                and k_new.dtype == v_new.dtype == sh.torch_dtype and k_new.is_contiguous() and v_new.is_contiguous()
                and rv.nbytes == rk.nbytes and rk.is_contiguous() and rv.is_contiguous() and c.ret_pos.numel() == U * cap
                and not (k_new.requires_grad or v_new.requires_grad)):
            try:
                B.vector_append(sh, c, k_new, v_new, pos)
                c.n_ret += 1
                return
            except B.VectorError as e:
                if e.status != -2:
                    raise
        c.ret_k[:, c.n_ret] = k_new
        c.ret_v[:, c.n_ret] = v_new
        c.ret_pos[:, c.n_ret] = pos
        c.n_ret += 1

    def decode(self, q, W, out, mode: int = 0):
        B.vector_decode_attn(self.shape, q, self.cache, W, out, mode, self.ws)
        return out


class PagedCache:
    """The compressed caches of many requests in 4 bits, or 8, and pages, one place of a batch each: requests are admitted with a compressed context,
    grow by a generated token a step (8 bits: or by several, and their keys may be turned on the way), and end, each with a length of its own.

    shape.batch is the number of places; all device work is asynchronous on the current stream, and `append` and `decode` read nothing back, so
    that a captured step follows the requests' lengths.  Pages are counted on the device: whether an admission found enough of them is an answer on the
    device, too.  A place is taken from `admit` on, whatever that answered, until `end`.  A step covers all layers of the shape; a model
    whose layers follow one another keeps a PagedCache a layer.
    """

    def __init__(self, shape: B.Shape, ret_pages: int, apx_pages: int, ret_rows: int, apx_rows: int, positions: bool = True, device="cuda", bits: int = 4):
        """Pools of so many pages (of 64 rows in 4 bits, of 32 in 8); places for at most ret_rows retained and apx_rows key-only rows of a request."""
        if bits not in (4, 8):
            raise ValueError(f"rows are held in 4 bits or in 8, not in {bits}")
        self.bits, self.page_rows = bits, B.VECTOR_PAGE_ROWS if bits == 4 else B.VECTOR_Q8_PAGE_ROWS
        if shape.rope_enabled and not positions:
            raise ValueError("keys with rotary positions are turned back by their positions: positions must be kept")
        self.shape, self.device = shape, device
        pages = lambda rows: max(self._pages(rows), 1)  # noqa: E731
        self.cache = (B.alloc_q4_cache if bits == 4 else B.alloc_q8_cache)(shape, ret_pages, apx_pages, pages(ret_rows), pages(apx_rows), positions, device)
        n = shape.batch
        ints = lambda *size: torch.zeros(*size, dtype=torch.int32, device=device)  # noqa: E731
        # stacks of free pages, the first page on top
        self.ret_free, self.apx_free = (torch.arange(p - 1, -1, -1, dtype=torch.int32, device=device) for p in (ret_pages, apx_pages))
        self.n_ret_free, self.n_apx_free = ints(1).fill_(ret_pages), ints(1).fill_(apx_pages)
        self.active, self.first_row, self.row_start, self.slots = ints(n), ints(n), ints(n + 1), ints(n)
        self.ws = torch.empty((B.vector_decode_q4_workspace_bytes if bits == 4 else B.vector_decode_q8_workspace_bytes)(shape), dtype=torch.uint8, device=device)
        self._taken = set()

    def _pages(self, rows: int) -> int:
        return -(-rows // self.page_rows)

    def _place(self, place: int) -> int:
        return range(self.shape.batch)[place]

    def _change(self, tier: str, added, slots=None):
        c = self.cache
        table, length, stack, left = ((c.ret_table, c.ret_len, self.ret_free, self.n_ret_free) if tier == "ret"
                                      else (c.apx_table, c.apx_len, self.apx_free, self.n_apx_free))
        B.vector_block_tables(length, added, self.page_rows, table, stack, left, length, left, self.first_row, self.row_start, slots)

    def _check_admission(self, place: int, comp: Compressor, K, V):
        sh, b, mine, c = comp.shape, comp.budget, self.shape, self.cache
        if sh.batch != 1 or any(getattr(sh, f) != getattr(mine, f) for f in ("n_layers", "n_kv_heads", "n_q_heads", "head_dim", "dtype")):
            raise ValueError("the compressor is for one sequence of the same layers and heads")
        if bool(sh.rope_enabled) != bool(mine.rope_enabled) or (mine.rope_enabled and sh.rope_theta != mine.rope_theta):
            raise ValueError("the compressor's rotary positions are not the cache's")
        if place in self._taken:
            raise ValueError(f"place {place} is taken")
        for n, table, pages, kind in ((b.n_ret, c.ret_table, c.ret_pages, "retained"), (b.n_apx, c.apx_table, c.apx_pages, "key-only")):
            if self._pages(n) > table.shape[1]:
                raise ValueError(f"{n} {kind} rows, and a place is for {table.shape[1] * self.page_rows}")
            if self._pages(n) > pages.shape[0]:
                raise ValueError(f"{n} {kind} rows, and the pool of pages holds {pages.shape[0] * self.page_rows}")
        for t, name in ((K, "K"), (V, "V")):
            if B._sized(t, sh.torch_dtype, sh.units * b.n_tokens * sh.head_dim, name) % 16:
                raise ValueError(f"{name} must lie at a multiple of 16 bytes")
        if self.bits == 8:
            B._on_current_device(K, V, comp.ret_idx, comp.apx_idx, *B._of_cache(c))

    def admit(self, place: int, comp: Compressor, K, V) -> torch.Tensor:
        """Takes the routed context of a Compressor of one sequence (its score and route have been called) to a place that is not taken.  Returns whether
        it is there, one bool on the device: where either pool has too few free pages left, nothing is taken, and the place stays without rows.  What the host knows is refused
        before anything changes: a taken place, a context longer than a place or a pool, another model's."""
        place = self._place(place)
        self._check_admission(place, comp, K, V)
        b = comp.budget
        there = ((self.n_ret_free >= self._pages(b.n_ret)) & (self.n_apx_free >= self._pages(b.n_apx)))[0]
        slots, added = {}, {}
        for tier, n in (("ret", b.n_ret), ("apx", b.n_apx)):
            slots[tier] = torch.empty(n, dtype=torch.int32, device=self.device) if self.bits == 4 else None
            added[tier] = torch.zeros(self.shape.batch, dtype=torch.int32, device=self.device)
            added[tier][place] = there * n
        for tier in ("ret", "apx"):
            self._change(tier, added[tier], slots[tier])
        if self.bits == 4:
            B.vector_compact_q4(comp.shape, b, K, V, comp.ret_idx, comp.apx_idx, self.cache, slots["ret"], slots["apx"])
        else:                                               # rows go where the place's table and lengths say: nowhere, where it got no pages
            c, at = self.cache, slice(place, place + 1)
            mine = B.Q8Cache(c.ret_pages, c.apx_pages, c.ret_table[at], c.apx_table[at], c.ret_len[at], c.apx_len[at], c.ret_pos, c.apx_pos)
            B.vector_compact_q8(comp.shape, b, K, V, comp.ret_idx, comp.apx_idx, mine)
        self.active[place] = there
        self._taken.add(place)
        return there

    def end(self, *places: int):
        """Gives the pages of these places back."""
        at = [self._place(p) for p in places]
        gone = torch.zeros(self.shape.batch, dtype=torch.int32, device=self.device)
        gone[at] = -2**31
        for tier in ("ret", "apx"):
            self._change(tier, gone)
        self.active[at] = 0
        self._taken.difference_update(at)

    def project(self, q, k, v, q_weight=None, k_weight=None, pos=None, eps: float = 1e-6):
        """The layers' projections of one token of every place, [B][L] rows, as the rows of append and decode: q [U][g][d], k and v [U][d].  pos [batch], the tokens' positions, is needed where
        the shape has rotary ones: queries and keys come turned by it, so that append takes them without rotate."""
        if self.shape.rope_enabled and pos is None:
            raise ValueError("pos is missing: queries and keys are turned by the tokens' positions")
        q, k, v = project(self.shape, 1, q, k, v, q_weight, k_weight, pos, eps)
        return q[:, :, 0], k[:, 0], v[:, 0]

    def append(self, k_new, v_new, pos, rotate: bool = False):
        """A generated token of every active place: k_new, v_new [U][d], pos [batch] int32.  A request that finds no page left keeps its length.
        8 bits: or n tokens, [batch][n] rows of all layers' and heads' channels with pos [batch][n] (vector_append_q8 says how they come from projections), of which a request that finds too few
        pages keeps the first ones; rotate: the keys are still to be turned by their positions."""
        if self.bits == 8:
            sh = self.shape                                 # what is refused is refused before the tables change
            n = k_new.numel() // (sh.units * sh.head_dim)
            if rotate and not sh.rope_enabled:
                raise ValueError("keys are turned where the shape has rotary positions")
            for t, name in ((k_new, "k_new"), (v_new, "v_new")):
                at, stride = B._new_rows(sh, n, t, name)
                if at % 16 or stride * t.element_size() % 16:
                    raise ValueError(f"{name}: rows must lie at multiples of 16 bytes")
            if pos is None and (rotate or self.cache.ret_pos is not None):
                raise ValueError("pos is missing")
            B._positions(pos, sh.batch * n)
            B._on_current_device(k_new, v_new, pos, self.cache.ret_pages)      # the cache's tensors were made on one device; asking each of them took 2 us
            self._change("ret", self.active if n == 1 else self.active * n)
            B.vector_append_q8(self.shape, self.cache, k_new, v_new, self.first_row, pos, rotate)
            return
        if rotate:
            raise ValueError("the 4-bit cache takes keys that have been turned")
        self._change("ret", self.active, self.slots)
        B.vector_append_q4(self.shape, self.cache, k_new, v_new, self.row_start, self.slots, pos)

    def decode(self, q, W, out):
        (B.vector_decode_attn_q4 if self.bits == 4 else B.vector_decode_attn_q8)(self.shape, q, self.cache, W, out, self.ws)
        return out

    def free_pages(self) -> tuple[int, int]:
        """Pages left in the two pools (waits for the device)."""
        return int(self.n_ret_free), int(self.n_apx_free)
