// The kernels of attention over the 4-bit paged cache (decode_q4.cu).
//
// Streaming kernel.  A tile is a page of one unit: 64 keys and their values, or 64 key-only keys.  The sequence of all units' tiles, each
// weighted by what it costs, is cut into equal contiguous ranges, one per warp: a warp is a worker of its own, which copies its tiles into
// its own ring of slots (cp.async.bulk, one mbarrier a slot) and never waits for another warp.  It keeps one running state for a
// unit's tier and writes it as a partial record when it leaves that.  The lengths lie on the device, so every block sums up the
// sequences' costs itself.
//
// A worker takes 32 keys at a time.  A stored row's piece t is what lane t of a quad holds of a 16 x 16 fragment whose rows are keys: one 16-byte load (8 for
// 64 channels) of codes and two scales a row, one conversion and one product for two channels, and no exchange between lanes:
//   S^T = K Q^T    m16n8k16, keys down, the query heads across: no padding to sixteen rows of queries
//   softmax        in fp32, against a reference that follows the maximum only when that has moved by more than SLACK (powers of two); the weights go to fp16
//   O^T += V^T P^T channels down, heads across; both operands are the registers at hand after an 8 x 8 transpose (movmatrix), and so are the key sums
//                  A^T += K^T P^T of key-only keys, from the very registers that gave the logits
// The sum of the weights is one more row of that product, a row of ones, so that a weight's rounding to fp16 is in numerator and denominator alike.
// Stored rows are exact in fp16, so the products are.  Queries are scaled by a power of two a head to fp16's range; fp32 queries take two fp16 parts.
// EXACT (fp32 queries or fp32 output): weights, and keys turned back, in two fp16 parts, and sums of 32 keys added up outside the tensor cores,
// which cut their sums off instead of rounding them.
//
// Merge kernel.  A block per unit combines its records, applies the map to the key sums on the tensor cores (in three bf16 parts: 24 bits) and normalises.
#ifndef VECTOR_DECODE_Q4_CUH_
#define VECTOR_DECODE_Q4_CUH_

#include "common.cuh"
#include "internal.h"
#include "q4.cuh"
#include "rope.cuh"
#include "tcgen05.cuh"
#include "tma.cuh"

namespace vec {
namespace dq4 {

constexpr int WARPS = 12, SLOTS = 2;                 // slots of a warp's ring
constexpr int MAX_BATCH = VECTOR_Q4_MAX_BATCH;
constexpr int COST_RET = 2, COST_APX = 1, COST_MOST = 2;      // of a tile
constexpr float SLACK = 8.f;

struct Cache {
    const unsigned char *ret, *apx;
    const int32_t *ret_table, *apx_table, *ret_len, *apx_len, *apx_pos;
    int64_t n_ret_pages, n_apx_pages;
    int32_t ret_width, apx_width, LH, batch;
};
// Rows of a sequence in a tier: what its table can hold at the most.
__device__ __forceinline__ int rows_of(const int32_t* len, int b, int width) { return width ? min(max(len[b], 0), width * q4::ROWS) : 0; }
__device__ __forceinline__ int tiles_of(int rows) { return (rows + q4::ROWS - 1) / q4::ROWS; }

// ---- workspace: prefix sums of the costs [batch + 1], then the records
__host__ __device__ inline size_t prefix_bytes(int batch) { return (((size_t)batch + 1) * 8 + 255) & ~(size_t)255; }
// A record: for each tier [heads, rounded up to even][m, l] and the sums, in the order of the fragments.
__host__ __device__ inline int even_heads(int g) { return (g + 1) & ~1; }
__host__ __device__ inline int tier_floats(int g, int d) { return even_heads(g) * (d + 2); }

// How the cost X of all tiles is dealt to workers.  Every range is as long as a tile's cost at the least, so each begins a tile.
struct Deal {
    int64_t X;
    int workers;
    __device__ __forceinline__ Deal(int64_t x, int most) : X(x), workers((int)max(min((int64_t)most, x / COST_MOST), (int64_t)1)) {}
    __device__ __forceinline__ int64_t begin(int w) const { return X * w / workers; }
    __device__ __forceinline__ int owner(int64_t x) const { return (int)(((x + 1) * workers - 1) / X); }
};
// First tile of a unit that begins at r or later, r counted from the unit's beginning.
__device__ __forceinline__ int tile_from(int64_t r, int nr) {
    return r <= (int64_t)COST_RET * nr ? (int)((r + COST_RET - 1) / COST_RET) : nr + (int)((r - (int64_t)COST_RET * nr + COST_APX - 1) / COST_APX);
}

template <typename T, int D, bool ROPE, bool EXACT> struct Cfg {
    static constexpr int THREADS = 32 * WARPS;
    static constexpr int SLOT_BYTES = 2 * q4::Row<D>::TILE;
    static constexpr int POS_AT = q4::Row<D>::TILE;                    // of a key-only tile's positions, within a slot
    static constexpr int SMEM_BYTES = WARPS * SLOTS * SLOT_BYTES;      // and behind them the prefix sums
    static constexpr int Q_PARTS = sizeof(T) == 4 ? 2 : 1;
    static constexpr int PAIRS = D / 8;                                // channel pairs of a lane in a row
    static constexpr int O_TILES = D / 16;
};

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose(uint32_t a) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;\n" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma_h2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;\n" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 unpack_h2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// Where a worker is in the sequence of tiles.
struct Walk {
    int b, lh, t, n_ret, n_apx;                 // sequence, (layer, KV head), tile of the unit, rows
    __device__ __forceinline__ void enter(const Cache& c) {
        n_ret = rows_of(c.ret_len, b, c.ret_width);
        n_apx = rows_of(c.apx_len, b, c.apx_width);
    }
    __device__ __forceinline__ int tiles() const { return tiles_of(n_ret) + tiles_of(n_apx); }
    __device__ __forceinline__ void settle(const Cache& c, const int64_t* prefix) {       // t may be behind the unit's last tile
        if (t < tiles()) return;
        t = 0;
        if (++lh < c.LH) return;
        lh = 0;
        do ++b; while (b < c.batch && prefix[b + 1] == prefix[b]);
        if (b < c.batch) enter(c);
    }
    // The first tile that begins at cost x or later.
    __device__ __forceinline__ void find(const Cache& c, const int64_t* prefix, int64_t x) {
        int lo = 0, hi = c.batch + 1;           // the last b with prefix[b] <= x
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (prefix[mid] <= x) lo = mid;
            else hi = mid;
        }
        b = lo; lh = 0; t = 0; n_ret = 0; n_apx = 0;
        if (b >= c.batch) return;
        enter(c);
        const int64_t r = x - prefix[b], unit = (prefix[b + 1] - prefix[b]) / c.LH;
        lh = (int)(r / unit);
        t = tile_from(r - lh * unit, tiles_of(n_ret));
        settle(c, prefix);
    }
};

// What a slot holds, for its consumer: unit, rows that are there, tier, whether it is the unit's first tile.
struct Tile { int unit, rows, apx, first; };

template <typename T, int D, bool ROPE, bool EXACT>
__global__ void __launch_bounds__(Cfg<T, D, ROPE, EXACT>::THREADS, 1)
decode_q4_stream(const T* q, Cache c, int g, float scale_log2e, unsigned char* ws, int* fault, RopePhases phases) {
    using C = Cfg<T, D, ROPE, EXACT>;
    using R = q4::Row<D>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t full[WARPS][SLOTS];
    __shared__ Tile tiles[WARPS][SLOTS];
    __shared__ int64_t sums[WARPS];
    __shared__ uint32_t phase32[ROPE ? D / 2 : 1];
    __shared__ RopePhase phase64[ROPE && EXACT ? D / 2 : 1];
    int64_t* prefix = reinterpret_cast<int64_t*>(smem + C::SMEM_BYTES);
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) tma::mbar_init(&full[wid][s], 1);
        tma::mbar_fence_init();
    }
    if constexpr (ROPE) {
        if (threadIdx.x < D / 2) {
            phase32[threadIdx.x] = (uint32_t)((phases.phase[threadIdx.x] + 0x80000000ull) >> 32);
            if constexpr (EXACT) phase64[threadIdx.x] = rope_phase_words(phases.phase[threadIdx.x]);
        }
    }
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    // ---- costs of the sequences, summed up
    int64_t carry = 0;
    for (int b0 = 0; b0 < c.batch; b0 += C::THREADS) {
        const int b = b0 + threadIdx.x;
        int64_t x = 0;
        if (b < c.batch)
            x = (int64_t)c.LH * (COST_RET * tiles_of(rows_of(c.ret_len, b, c.ret_width)) + COST_APX * tiles_of(rows_of(c.apx_len, b, c.apx_width)));
        int64_t s = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        if (lane == 31) sums[wid] = s;
        __syncthreads();
        int64_t before = carry, all = carry;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { all += sums[w]; if (w < wid) before += sums[w]; }
        if (b < c.batch) prefix[b] = before + s - x;
        carry = all;
        __syncthreads();
    }
    if (threadIdx.x == 0) prefix[c.batch] = carry;
    __syncthreads();
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b <= c.batch; b += C::THREADS) reinterpret_cast<int64_t*>(ws)[b] = prefix[b];
    const Deal deal(carry, gridDim.x * WARPS);
    const int worker = wid * gridDim.x + blockIdx.x;        // neighbours in the sequence on different multiprocessors
    if (carry == 0 || worker >= deal.workers) return;

    float* records = reinterpret_cast<float*>(ws + prefix_bytes(c.batch));
    const int rec = 2 * tier_floats(g, D), heads = even_heads(g), units = c.batch * c.LH;
    unsigned char* ring = smem + wid * SLOTS * C::SLOT_BYTES;
    const uint64_t policy = tma::policy_evict_first();

    // ---- the producing side: `next` walks SLOTS tiles ahead
    Walk next, end;
    end.find(c, prefix, deal.begin(worker + 1));
    next.find(c, prefix, deal.begin(worker));
    auto more = [&] { return next.b != end.b || next.lh != end.lh || next.t != end.t; };
    auto issue = [&](int s) {
        const int nr = tiles_of(next.n_ret);
        const bool apx = next.t >= nr;
        const int p = apx ? next.t - nr : next.t;
        const int64_t page = apx ? c.apx_table[(size_t)next.b * c.apx_width + p] : c.ret_table[(size_t)next.b * c.ret_width + p];
        const bool there = page >= 0 && page < (apx ? c.n_apx_pages : c.n_ret_pages);
        if (lane == 0) {
            tiles[wid][s] = Tile{next.b * c.LH + next.lh, there ? min((apx ? next.n_apx : next.n_ret) - p * q4::ROWS, (int)q4::ROWS) : 0, apx, next.t == 0};
            const size_t at = (size_t)page * c.LH + next.lh;
            if (!there) {
                tma::mbar_arrive(&full[wid][s]);
            } else if (apx) {
                tma::mbar_expect_tx(&full[wid][s], R::TILE + (ROPE ? 4 * q4::ROWS : 0));
                tma::load_bulk_hint(ring + s * C::SLOT_BYTES, c.apx + at * R::TILE, R::TILE, &full[wid][s], policy);
                if (ROPE) tma::load_bulk_hint(ring + s * C::SLOT_BYTES + C::POS_AT, c.apx_pos + at * q4::ROWS, 4 * q4::ROWS, &full[wid][s], policy);
            } else {
                tma::mbar_expect_tx(&full[wid][s], 2 * R::TILE);
                tma::load_bulk_hint(ring + s * C::SLOT_BYTES, c.ret + at * 2 * R::TILE, 2 * R::TILE, &full[wid][s], policy);
            }
        }
        ++next.t;
        next.settle(c, prefix);
    };
    int ahead = 0;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s)
        if (more()) { issue(s); ++ahead; }
    __syncwarp();

    // ---- the consuming side
    uint32_t qb[C::Q_PARTS][C::O_TILES][2];
    float fac[2] = {0.f, 0.f}, m[2] = {-INFINITY, -INFINITY}, O[C::O_TILES][4], L[4];
    auto clear = [&] {
        m[0] = m[1] = -INFINITY;
#pragma unroll
        for (int t = 0; t < C::O_TILES; ++t) O[t][0] = O[t][1] = O[t][2] = O[t][3] = 0.f;
        L[0] = L[1] = L[2] = L[3] = 0.f;
    };
    clear();
    // The queries of a unit as B fragments: head gid, the channels of piece tig.  Scaled so that the largest lies in [2^7, 2^8).
    auto load_queries = [&](int unit) {
        const T* row = q + ((size_t)unit * g + min(gid, g - 1)) * D;
        float x[2 * C::PAIRS];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < C::PAIRS; ++i) x[h * C::PAIRS + i] = gid < g ? to_f32(row[h * (D / 2) + tig * (D / 8) + i]) : 0.f;
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * C::PAIRS; ++i) most = fmaxf(most, fabsf(x[i]));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int e = min(max((int)(__float_as_uint(most) >> 23) - 127, -100), 127);
        const float up = __uint_as_float((uint32_t)(127 + 7 - e) << 23);
        const float down = scale_log2e * __uint_as_float((uint32_t)(max(127 - 7 + e, 1)) << 23);
        fac[0] = __shfl_sync(0xffffffffu, down, (2 * tig) * 4);
        fac[1] = __shfl_sync(0xffffffffu, down, (2 * tig + 1) * 4);
#pragma unroll
        for (int i = 0; i < C::PAIRS; ++i) {
            const float a = x[2 * i] * up, b = x[2 * i + 1] * up;
            const uint32_t hi = pack_h2(a, b);
            qb[0][i / 2][i % 2] = hi;
            if constexpr (C::Q_PARTS == 2) {
                const float2 f = unpack_h2(hi);
                qb[1][i / 2][i % 2] = pack_h2(a - f.x, b - f.y);
            }
        }
    };
    // Rows 16 i + gid and 16 i + gid + 8 of a tile's 32 rows at `row0`, as A fragments; rows from `rows` on are zero.
    auto load_rows = [&](const unsigned char* tile, int row0, int rows, uint32_t (&x)[2][2][C::PAIRS]) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 16 * i + 8 * h + gid, row = row0 + r;
                uint32_t w[4];
                if constexpr (D == 128) {
                    const uint4 v = *reinterpret_cast<const uint4*>(tile + row * R::CODES + tig * 16);
                    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
                } else {
                    const uint2 v = *reinterpret_cast<const uint2*>(tile + row * R::CODES + tig * 8);
                    w[0] = v.x; w[1] = v.y;
                }
                uint32_t s = *reinterpret_cast<const uint16_t*>(tile + R::SCALES_AT + row * R::GROUPS + 2 * (D == 128 ? tig : tig >> 1));
                if (r >= rows) s = 0;                                  // what lies there may be no number
                const uint32_t s2[2] = {(s & 0xffu) * 0x00800080u, (s >> 8) * 0x00800080u};
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    uint32_t p[4];
                    q4::decode_word(w[j], p);
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[i][h][4 * j + k] = mul_h2(p[k], s2[j / (D / 64)]);
                }
            }
    };

    int unit = -1, apx = 0, wrote = 0, slot_rec = 0;
    // The state of a tier to its record; an empty one's sums are not read.
    auto put_tier = [&](int tier, bool empty) {
        float* p = records + (size_t)slot_rec * rec + tier * tier_floats(g, D);
        if (2 * tig >= heads) return;
        if (gid == 0) *reinterpret_cast<float4*>(p + 4 * tig) = empty ? make_float4(-INFINITY, 0.f, -INFINITY, 0.f) : make_float4(m[0], L[0], m[1], L[1]);
        if (empty) return;
        float4* o = reinterpret_cast<float4*>(p + 2 * heads);
#pragma unroll
        for (int t = 0; t < C::O_TILES; ++t) o[(t * (heads / 2) + tig) * 8 + gid] = make_float4(O[t][0], O[t][1], O[t][2], O[t][3]);
    };
    auto leave_unit = [&] {
        if (unit < 0) return;
        put_tier(apx, false);
        wrote |= 1 << apx;
        if (!(wrote & 1)) put_tier(0, true);
        if (!(wrote & 2)) put_tier(1, true);
    };

    for (int i = 0; ahead > 0; ++i) {
        const int s = i % SLOTS;
        if (!tma::mbar_wait_warp(&full[wid][s], (i / SLOTS) & 1, fault, 21)) {
            for (int k = i; k < i + ahead; ++k) tma::mbar_wait_warp(&full[wid][k % SLOTS], (k / SLOTS) & 1, fault, 21);     // copies in flight
            return;
        }
        const Tile tile = tiles[wid][s];
        if (tile.unit != unit) {
            leave_unit();
            unit = tile.unit; apx = tile.apx; wrote = 0;
            slot_rec = tile.first ? unit : units + worker;
            clear();
            load_queries(unit);
        } else if (tile.apx != apx) {
            put_tier(apx, false);
            wrote |= 1 << apx;
            apx = tile.apx;
            clear();
        }
        const unsigned char* at = ring + s * C::SLOT_BYTES;
#pragma unroll 1
        for (int row0 = 0; row0 < tile.rows; row0 += 32) {
            const int rows = tile.rows - row0;
            uint32_t x[2][2][C::PAIRS];
            load_rows(at, row0, rows, x);
            float S[2][4];
#pragma unroll
            for (int k = 0; k < 2; ++k) S[k][0] = S[k][1] = S[k][2] = S[k][3] = 0.f;
#pragma unroll
            for (int p = 0; p < C::Q_PARTS; ++p)
#pragma unroll
                for (int t = 0; t < C::O_TILES; ++t)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        mma(S[k], x[k][0][2 * t], x[k][1][2 * t], x[k][0][2 * t + 1], x[k][1][2 * t + 1], qb[p][t][0], qb[p][t][1]);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) S[k][e] *= fac[e & 1];
            if (rows < 32) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (16 * k + 8 * (e >> 1) + gid >= rows) S[k][e] = -INFINITY;
            }
            // ---- softmax against the reference m
            float top[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) top[h] = fmaxf(fmaxf(S[0][h], S[0][2 + h]), fmaxf(S[1][h], S[1][2 + h]));
            if (__any_sync(0xffffffffu, top[0] > m[0] + SLACK || top[1] > m[1] + SLACK)) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], o));
                    const float now = fmaxf(m[h], top[h]), f = m[h] == now ? 1.f : tc::ex2(m[h] - now);
                    m[h] = now;
#pragma unroll
                    for (int t = 0; t < C::O_TILES; ++t) { O[t][h] *= f; O[t][2 + h] *= f; }
                    L[h] *= f; L[2 + h] *= f;
                }
            }
            uint32_t ph[2][2], pl[2][2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float a = tc::ex2(S[k][2 * h] - m[0]), b = tc::ex2(S[k][2 * h + 1] - m[1]);
                    const uint32_t hi = pack_h2(a, b);
                    ph[k][h] = transpose(hi);
                    if constexpr (EXACT) {
                        const float2 f = unpack_h2(hi);
                        pl[k][h] = transpose(pack_h2(a - f.x, b - f.y));
                    }
                }
            if (!tile.apx) load_rows(at + R::TILE, row0, rows, x);
            uint32_t lo[2][2][ROPE && EXACT ? C::PAIRS : 1];           // second parts of keys turned back
            if constexpr (ROPE) {
                if (tile.apx) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int r = 16 * k + 8 * h + gid;
                            const uint32_t pos = r < rows ? (uint32_t)reinterpret_cast<const int32_t*>(at + C::POS_AT)[row0 + r] : 0u;
#pragma unroll
                            for (int j = 0; j < C::PAIRS / 2; ++j) {
                                const int ch = tig * (D / 8) + 2 * j;
                                uint32_t &u = x[k][h][j], &v = x[k][h][C::PAIRS / 2 + j];
                                if constexpr (EXACT) {
                                    uint64_t cs, sn;
                                    rope_cos_sin2(rope_angle((int32_t)pos, phase64[ch]), rope_angle((int32_t)pos, phase64[ch + 1]), cs, sn);
                                    const float2 uf = unpack_h2(u), vf = unpack_h2(v);
                                    const uint64_t u2 = tc::pack2(uf.x, uf.y), v2 = tc::pack2(vf.x, vf.y);
                                    auto parts = [](uint64_t z, uint32_t& hi, uint32_t& low) {
                                        float a, b;
                                        tc::unpack2(z, a, b);
                                        hi = pack_h2(a, b);
                                        const float2 f = unpack_h2(hi);
                                        low = pack_h2(a - f.x, b - f.y);
                                    };
                                    const uint64_t neg = tc::pack2(-1.f, -1.f);
                                    parts(tc::fma2(u2, cs, tc::mul2(v2, sn)), u, lo[k][h][j]);
                                    parts(tc::fma2(u2, tc::mul2(sn, neg), tc::mul2(v2, cs)), v, lo[k][h][C::PAIRS / 2 + j]);
                                } else {
                                    float c0, s0, c1, s1;
                                    rope_phase32_cos_sin(pos, phase32[ch], c0, s0);
                                    rope_phase32_cos_sin(pos, phase32[ch + 1], c1, s1);
                                    const uint32_t cs = pack_h2(c0, c1), sn = pack_h2(s0, s1), a = u, b = v;
                                    u = fma_h2(a, cs, mul_h2(b, sn));
                                    v = fma_h2(b, cs, mul_h2(a ^ 0x80008000u, sn));
                                }
                            }
                        }
                }
            }
            const bool two = ROPE && EXACT && tile.apx;
#pragma unroll
            for (int t = 0; t < C::O_TILES; ++t) {
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t a0 = transpose(x[k][0][2 * t]), a1 = transpose(x[k][0][2 * t + 1]), a2 = transpose(x[k][1][2 * t]),
                                   a3 = transpose(x[k][1][2 * t + 1]);
                    if constexpr (EXACT) {
                        mma(sum, a0, a1, a2, a3, pl[k][0], pl[k][1]);
                        if constexpr (ROPE)
                            if (two)
                                mma(sum, transpose(lo[k][0][2 * t]), transpose(lo[k][0][2 * t + 1]), transpose(lo[k][1][2 * t]), transpose(lo[k][1][2 * t + 1]),
                                    ph[k][0], ph[k][1]);
                        mma(sum, a0, a1, a2, a3, ph[k][0], ph[k][1]);
                    } else {
                        mma(O[t], a0, a1, a2, a3, ph[k][0], ph[k][1]);
                    }
                }
                if constexpr (EXACT) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) O[t][e] += sum[e];
                }
            }
            constexpr uint32_t ONE = 0x3c003c00u;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if constexpr (EXACT) mma(sum, ONE, ONE, ONE, ONE, pl[k][0], pl[k][1]);
                mma(sum, ONE, ONE, ONE, ONE, ph[k][0], ph[k][1]);
            }
            L[0] += sum[0]; L[1] += sum[1];
        }
        __syncwarp();                                                  // every lane has read the slot
        --ahead;
        if (more()) { issue(s); ++ahead; __syncwarp(); }
    }
    leave_unit();
}

constexpr int MERGE_THREADS = 256;

// The records of a unit into its outputs.
template <typename T, int D, typename TO>
__global__ void __launch_bounds__(MERGE_THREADS)
decode_q4_merge(const unsigned char* ws, Cache c, int g, int most_workers, const T* W, TO* __restrict__ out) {
    constexpr int NW = MERGE_THREADS / 32, ROWS_W = 16;
    constexpr bool TENSOR = sizeof(T) == 2;
    __shared__ __align__(16) float val[8][D + 4], keys[8][D + 4];
    __shared__ float ref[8], inv[8];
    const int u = blockIdx.x, b = u / c.LH, lh = u - b * c.LH;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    // the map's rows of this warp, requested ahead of the wait: rows 16 wid + gid (+ 8), channels of lane tig
    uint4 w[2][TENSOR ? D / 32 : 1];
    if constexpr (TENSOR) {
        if (wid < D / ROWS_W) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < D / 32; ++i)
                    w[h][i] = *reinterpret_cast<const uint4*>(W + ((size_t)lh * D + ROWS_W * wid + 8 * h + gid) * D + 32 * i + 8 * tig);
        }
    }
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    const int64_t* prefix = reinterpret_cast<const int64_t*>(ws);
    const float* records = reinterpret_cast<const float*>(ws + prefix_bytes(c.batch));
    const int heads = even_heads(g), tier = tier_floats(g, D), units = c.batch * c.LH;
    const int64_t p0 = prefix[b], p1 = prefix[b + 1], X = prefix[c.batch];
    TO* o = out + (size_t)u * g * D;
    if (p0 == p1) {                                                   // nothing to attend to
        for (int e = threadIdx.x; e < g * D; e += MERGE_THREADS) store_out(o + e, 0.f);
        return;
    }
    const int64_t cost = (p1 - p0) / c.LH, from = p0 + lh * cost;
    const Deal deal(X, most_workers);
    const int nr = tiles_of(rows_of(c.ret_len, b, c.ret_width)), na = tiles_of(rows_of(c.apx_len, b, c.apx_width));
    const int w0 = deal.owner(from);
    int last = deal.owner(from + cost - 1);
    if (last > w0 && tile_from(deal.begin(last) - from, nr) >= nr + na) --last;       // its range begins within the unit's last tile
    const int pieces = last - w0 + 1;                                 // the unit's own record, then those of workers w0 + 1 ..
    auto piece = [&](int i) { return records + (size_t)(i == 0 ? u : units + w0 + i) * 2 * tier; };
    // ---- a warp a head: the largest reference, the sum of the weights
    for (int h = wid; h < g; h += NW) {
        float M = -INFINITY;
        for (int i = lane; i < 2 * pieces; i += 32) M = fmaxf(M, piece(i >> 1)[(i & 1) * tier + 2 * h]);
        M = warp_max(M);
        float Lsum = 0.f;
        for (int i = lane; i < 2 * pieces; i += 32) {
            const float2 ml = *reinterpret_cast<const float2*>(piece(i >> 1) + (i & 1) * tier + 2 * h);
            if (!(ml.x == -INFINITY)) Lsum = fmaf(exp2f(ml.x - M), ml.y, Lsum);
        }
        Lsum = warp_sum(Lsum);
        if (lane == 0) { ref[h] = M; inv[h] = Lsum == 0.f ? 0.f : 1.f / Lsum; }
    }
    if (threadIdx.x < 8 && threadIdx.x >= g) { ref[threadIdx.x] = 0.f; inv[threadIdx.x] = 0.f; }
    __syncthreads();
    // ---- sums of values and of keys, four numbers (two rows of two heads) a thread
    const int quads = D / 16 * (heads / 2) * 8;
    for (int e = threadIdx.x; e < 2 * quads; e += MERGE_THREADS) {
        const int which = e >= quads, i = e - which * quads, row = i & 7, hp = (i >> 3) % (heads / 2), t = (i >> 3) / (heads / 2);
        const float M0 = ref[2 * hp], M1 = ref[2 * hp + 1];
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < pieces; ++k) {
            const float* p = piece(k) + which * tier;
            const float4 ml = *reinterpret_cast<const float4*>(p + 4 * hp);
            if (ml.x == -INFINITY && ml.z == -INFINITY) continue;
            const float4 v = *reinterpret_cast<const float4*>(p + 2 * heads + 4 * i);
            const float f0 = exp2f(ml.x - M0), f1 = exp2f(ml.z - M1);
            a.x = fmaf(f0, v.x, a.x); a.y = fmaf(f1, v.y, a.y); a.z = fmaf(f0, v.z, a.z); a.w = fmaf(f1, v.w, a.w);
        }
        // rows `row` and `row` + 8 of O tile t: channel pairs 2 t and 2 t + 1 of piece row / 2
        float (*to)[D + 4] = which ? keys : val;
        const int c0 = q4::Row<D>::channel_of(row / 2 * (D / 4) + 4 * t + row % 2), c1 = q4::Row<D>::channel_of(row / 2 * (D / 4) + 4 * t + 2 + row % 2);
        to[2 * hp][c0] = a.x; to[2 * hp + 1][c0] = a.y; to[2 * hp][c1] = a.z; to[2 * hp + 1][c1] = a.w;
    }
    __syncthreads();
    // ---- the map
    if constexpr (TENSOR) {
        if (wid < D / ROWS_W) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
            const int head = min(gid, heads - 1);
            if (na > 0) {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const uint32_t r0[4] = {w[0][i].x, w[0][i].y, w[0][i].z, w[0][i].w}, r1[4] = {w[1][i].x, w[1][i].y, w[1][i].z, w[1][i].w};
                    const float4 k0 = *reinterpret_cast<const float4*>(&keys[head][32 * i + 8 * tig]), k1 = *reinterpret_cast<const float4*>(&keys[head][32 * i + 8 * tig + 4]);
                    uint32_t part[4][3];
                    split_bf16<3>(k0.x, k0.y, part[0]); split_bf16<3>(k0.z, k0.w, part[1]);
                    split_bf16<3>(k1.x, k1.y, part[2]); split_bf16<3>(k1.z, k1.w, part[3]);
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int p = 2; p >= 0; --p)
                            asm volatile(
                                "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                                : "+f"(acc[0]), "+f"(acc[1]), "+f"(acc[2]), "+f"(acc[3])
                                : "r"(r0[2 * s]), "r"(r1[2 * s]), "r"(r0[2 * s + 1]), "r"(r1[2 * s + 1]), "r"(part[2 * s][p]), "r"(part[2 * s + 1][p]));
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int h = 2 * tig + (e & 1), ch = ROWS_W * wid + 8 * (e >> 1) + gid;
                if (h < g) store_out(o + h * D + ch, (val[h][ch] + acc[e]) * inv[h]);
            }
        }
    } else {
        for (int r = wid; r < D; r += NW) {
            float wr[D / 32];
#pragma unroll
            for (int j = 0; j < D / 32; ++j) wr[j] = to_f32(W[((size_t)lh * D + r) * D + 32 * j + lane]);
            for (int h = 0; h < g; ++h) {
                float x = 0.f;
#pragma unroll
                for (int j = 0; j < D / 32; ++j) x = fmaf(wr[j], keys[h][32 * j + lane], x);
                x = warp_sum(x);
                if (lane == 0) store_out(o + h * D + r, (val[h][r] + x) * inv[h]);
            }
        }
    }
}

}  // namespace dq4
}  // namespace vec
#endif
