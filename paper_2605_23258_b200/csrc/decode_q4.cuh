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

#include <type_traits>

#include "common.cuh"
#include "internal.h"
#include "q4.cuh"
#include "rope.cuh"
#include "tcgen05.cuh"
#include "tma.cuh"

namespace vec {
namespace dq4 {

constexpr int MAX_BATCH = VECTOR_Q4_MAX_BATCH;
// What a tile of either tier costs a worker, in small numbers.
struct Costs {
    int ret, apx;
    __host__ __device__ int most() const { return ret > apx ? ret : apx; }
};
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
    __device__ __forceinline__ Deal(int64_t x, int workers_at_most, Costs cost)
        : X(x), workers((int)max(min((int64_t)workers_at_most, x / cost.most()), (int64_t)1)) {}
    __device__ __forceinline__ int64_t begin(int w) const { return X * w / workers; }
    __device__ __forceinline__ int owner(int64_t x) const { return (int)(((x + 1) * workers - 1) / X); }
};
// First tile of a unit that begins at r or later, r counted from the unit's beginning.
__device__ __forceinline__ int tile_from(int64_t r, int nr, Costs cost) {
    const int64_t ret = (int64_t)cost.ret * nr;
    return r <= ret ? (int)((r + cost.ret - 1) / cost.ret) : nr + (int)((r - ret + cost.apx - 1) / cost.apx);
}

template <typename T, int D, bool ROPE, bool EXACT> struct Cfg {
    static constexpr int WARPS = EXACT && D == 128 ? 8 : 12;
    static constexpr int ENTRIES = WARPS == 12 ? 3 : 4;                // of a warp's ring, a tile each
    static constexpr int THREADS = 32 * WARPS;
    static constexpr int POS_AT = q4::Row<D>::TILE;                    // of a key-only tile's positions, within an entry
    static constexpr int ENTRY_BYTES = q4::Row<D>::TILE + (ROPE ? 4 * q4::ROWS : 0);
    static constexpr int SMEM_BYTES = WARPS * ENTRIES * ENTRY_BYTES;   // and behind them the prefix sums
    static constexpr int Q_PARTS = sizeof(T) == 4 ? 2 : 1;
    static constexpr int PAIRS = D / 8;                                // channel pairs of a lane in a row
    static constexpr int O_TILES = D / 16;
    static constexpr int N_APX = ROPE ? 1 : 2;                         // key-only rows of a step, in sixteens
    static constexpr Costs COST = ROPE ? Costs{2, 3} : Costs{4, 3};
};

// Not volatile, like the transposes: the compiler may move them past one another, so that one's operands are on their way during the next.
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose(uint32_t a) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(a));
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
__device__ __forceinline__ uint32_t neg_h2(uint32_t a) {
    uint32_t r;
    asm("neg.f16x2 %0, %1;\n" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 unpack_h2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// A worker's way through the sequence of tiles, as runs: tiles of one tier of one unit.
struct Runs {
    Costs cost;
    int64_t left;                               // cost up to the end of the worker's range
    int b, lh, n_ret, n_apx;                    // sequence, (layer, KV head), rows
    int apx, p, count;                          // the run: tier, first tile of it, tiles
    __device__ __forceinline__ void enter(const Cache& c) {
        n_ret = rows_of(c.ret_len, b, c.ret_width);
        n_apx = rows_of(c.apx_len, b, c.apx_width);
    }
    // The run that begins with tile t of the present unit, or of the next one if there is none; no tiles at the end of the range.
    __device__ __forceinline__ void run(const Cache& c, const int64_t* prefix, int t) {
        int nr = tiles_of(n_ret);
        if (t >= nr + tiles_of(n_apx)) {
            t = 0;
            if (++lh == c.LH) {
                lh = 0;
                do ++b; while (b < c.batch && prefix[b + 1] == prefix[b]);
                if (b < c.batch) { enter(c); nr = tiles_of(n_ret); }
            }
        }
        apx = t >= nr;
        p = apx ? t - nr : t;
        const int each = apx ? cost.apx : cost.ret;
        const int64_t in_range = (left + each - 1) / each;
        count = b < c.batch ? (int)max(min((int64_t)((apx ? tiles_of(n_apx) : nr) - p), in_range), (int64_t)0) : 0;
        left -= (int64_t)count * each;
    }
    __device__ __forceinline__ void next(const Cache& c, const int64_t* prefix) { run(c, prefix, p + count + (apx ? tiles_of(n_ret) : 0)); }
    // The first run of the costs [x, end).
    __device__ __forceinline__ void find(const Cache& c, const int64_t* prefix, int64_t x, int64_t end) {
        int lo = 0, hi = c.batch;               // the last b with prefix[b] <= x
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (prefix[mid] <= x) lo = mid;
            else hi = mid;
        }
        b = lo;
        enter(c);
        const int64_t unit = (prefix[b + 1] - prefix[b]) / c.LH;
        lh = (int)((x - prefix[b]) / unit);
        const int64_t r = x - prefix[b] - lh * unit;
        const int nr = tiles_of(n_ret), t = tile_from(r, nr, cost);
        left = end - x - ((int64_t)cost.ret * min(t, nr) + (int64_t)cost.apx * max(t - nr, 0) - r);
        run(c, prefix, t);
    }
};

// What an entry of a ring holds, for its consumer: unit, rows that are there, whether it is the unit's first tile.
enum Kind { KEYS, VALUES, KEY_ONLY };
struct Entry { int unit, rows, kind, first; };

// Sine and cosine of an angle in 2^-32 turns, by its upper 23 bits (8e-7): they become a number in [1, 2) and that a multiple of 2 pi
// about zero, without a conversion from integers, which would wait for the unit that the sine and the cosine keep busy.
__device__ __forceinline__ void turn_cos_sin(uint32_t angle, float& cs, float& sn) {
    const float turns = __uint_as_float((angle >> 9) ^ 0x3fc00000u);         // 1 + (angle + half a turn) modulo a turn
    __sincosf(fmaf(turns, 6.283185307179586f, -9.42477796076938f), &sn, &cs);
}
// N neighbouring numbers at a multiple of 16 bytes.
template <int N> __device__ __forceinline__ void load_run(const float* p, float* x) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const float4 v = reinterpret_cast<const float4*>(p)[i];
        x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
    }
}
template <int N> __device__ __forceinline__ void load_run(const __nv_bfloat16* p, float* x) {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
        const uint4 v = reinterpret_cast<const uint4*>(p)[i];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) { x[8 * i + 2 * j] = __uint_as_float(w[j] << 16); x[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
    }
}

template <typename T, int D, bool ROPE, bool EXACT>
__global__ void __launch_bounds__(Cfg<T, D, ROPE, EXACT>::THREADS, 1)
decode_q4_stream(const T* q, Cache c, int g, Costs cost, float scale_log2e, unsigned char* ws, int* fault, RopePhases phases) {
    using C = Cfg<T, D, ROPE, EXACT>;
    using R = q4::Row<D>;
    constexpr int WARPS = C::WARPS, ENTRIES = C::ENTRIES;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t full[WARPS][ENTRIES];
    __shared__ Entry entries[WARPS][ENTRIES];
    __shared__ int64_t sums[WARPS];
    __shared__ __align__(8) uint32_t phase32[ROPE ? D / 2 : 1];
    __shared__ RopePhase phase64[ROPE && EXACT ? D / 2 : 1];
    int64_t* prefix = reinterpret_cast<int64_t*>(smem + C::SMEM_BYTES);
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < ENTRIES; ++s) tma::mbar_init(&full[wid][s], 1);
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
            x = (int64_t)c.LH * ((int64_t)cost.ret * tiles_of(rows_of(c.ret_len, b, c.ret_width)) + (int64_t)cost.apx * tiles_of(rows_of(c.apx_len, b, c.apx_width)));
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
    const Deal deal(carry, gridDim.x * WARPS, cost);
    const int worker = wid * gridDim.x + blockIdx.x;        // neighbours in the sequence on different multiprocessors
    if (carry == 0 || worker >= deal.workers) return;

    float* records = reinterpret_cast<float*>(ws + prefix_bytes(c.batch));
    const int rec = 2 * tier_floats(g, D), heads = even_heads(g), units = c.batch * c.LH;
    unsigned char* ring = smem + wid * ENTRIES * C::ENTRY_BYTES;
    const uint64_t policy = tma::policy_evict_first();

    // ---- the producing side, ENTRIES ahead: `run` is where it is, `k` tiles of it are on their way, and lane l has the page of tile l of 32
    Runs run;
    run.cost = cost;
    run.find(c, prefix, deal.begin(worker), deal.begin(worker + 1));
    int k = 0, page = -1, values = 0;
    auto issue = [&](int s) {
        if ((k & 31) == 0 && k + lane < run.count && !values)
            page = run.apx ? c.apx_table[(size_t)run.b * c.apx_width + run.p + k + lane] : c.ret_table[(size_t)run.b * c.ret_width + run.p + k + lane];
        const int at = __shfl_sync(0xffffffffu, page, k & 31);
        if (lane == 0) {
            const bool there = at >= 0 && at < (run.apx ? c.n_apx_pages : c.n_ret_pages);
            const int p = run.p + k;
            const size_t tile = (size_t)at * c.LH + run.lh;
            entries[wid][s] = Entry{run.b * c.LH + run.lh, there ? min((run.apx ? run.n_apx : run.n_ret) - p * q4::ROWS, (int)q4::ROWS) : 0,
                                    run.apx ? KEY_ONLY : values ? VALUES : KEYS, p == 0 && (!run.apx || run.n_ret == 0)};
            uint64_t* bar = &full[wid][s];
            unsigned char* to = ring + s * C::ENTRY_BYTES;
            if (!there) {
                tma::mbar_arrive(bar);
            } else {
                tma::mbar_expect_tx(bar, R::TILE + (ROPE && run.apx ? 4 * q4::ROWS : 0));
                tma::load_bulk_hint(to, run.apx ? c.apx + tile * R::TILE : c.ret + (2 * tile + values) * R::TILE, R::TILE, bar, policy);
                if (ROPE && run.apx) tma::load_bulk_hint(to + C::POS_AT, c.apx_pos + tile * q4::ROWS, 4 * q4::ROWS, bar, policy);
            }
        }
        if (!run.apx) values ^= 1;
        if (!values && ++k == run.count) {
            run.next(c, prefix);
            k = 0;
        }
    };
    int ahead = 0;                             // entries on their way or not yet done with
#pragma unroll
    for (int s = 0; s < ENTRIES; ++s)
        if (run.count > 0) { issue(s); ++ahead; }
    __syncwarp();

    // ---- the consuming side
    uint32_t qb[C::Q_PARTS][C::O_TILES][2];
    float fac[2] = {0.f, 0.f}, m[2] = {-INFINITY, -INFINITY}, O[C::O_TILES][4], L[2];
    auto clear = [&] {
        m[0] = m[1] = -INFINITY;
#pragma unroll
        for (int t = 0; t < C::O_TILES; ++t) O[t][0] = O[t][1] = O[t][2] = O[t][3] = 0.f;
        L[0] = L[1] = 0.f;
    };
    clear();
    // The queries of a unit as B fragments: head gid, the channels of piece tig.  Scaled so that the largest lies in [2^7, 2^8).
    auto load_queries = [&](int unit) {
        const T* row = q + ((size_t)unit * g + min(gid, g - 1)) * D + tig * (D / 8);
        float x[2 * C::PAIRS];
#pragma unroll
        for (int h = 0; h < 2; ++h) load_run<C::PAIRS>(row + h * (D / 2), &x[h * C::PAIRS]);
        if (gid >= g) {
#pragma unroll
            for (int i = 0; i < 2 * C::PAIRS; ++i) x[i] = 0.f;
        }
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
    // Rows row0 + gid and row0 + gid + 8 of a tile as A fragments.
    auto load_rows = [&](const unsigned char* tile, int row0, uint32_t (&x)[2][C::PAIRS]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = row0 + 8 * h + gid;
            uint32_t w[4];
            if constexpr (D == 128) {
                const uint4 v = *reinterpret_cast<const uint4*>(tile + row * R::CODES + tig * 16);
                w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            } else {
                const uint2 v = *reinterpret_cast<const uint2*>(tile + row * R::CODES + tig * 8);
                w[0] = v.x; w[1] = v.y;
            }
            const uint32_t s = *reinterpret_cast<const uint16_t*>(tile + R::SCALES_AT + row * R::GROUPS + 2 * (D == 128 ? tig : tig >> 1));
            const uint32_t s2[2] = {(s & 0xffu) * 0x00800080u, (s >> 8) * 0x00800080u};
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                uint32_t p[4];
                q4::decode_word(w[j], p);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[h][4 * j + i] = mul_h2(p[i], s2[j / (D / 64)]);
            }
        }
    };
    // Logits of 16 keys, in chains of two products (EXACT) or of half of them.
    auto logits = [&](const uint32_t (&x)[2][C::PAIRS], float (&S)[4]) {
        S[0] = S[1] = S[2] = S[3] = 0.f;
        constexpr int CHAIN = EXACT ? 2 : C::O_TILES / 2;
#pragma unroll
        for (int p = C::Q_PARTS - 1; p >= 0; --p)
#pragma unroll
            for (int t0 = 0; t0 < C::O_TILES; t0 += CHAIN) {
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = t0; t < t0 + CHAIN; ++t) mma(sum, x[0][2 * t], x[1][2 * t], x[0][2 * t + 1], x[1][2 * t + 1], qb[p][t][0], qb[p][t][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) S[e] += sum[e];
            }
    };
    // Weights of N x 16 keys, of which `rows` are there, from their logits, against the reference m (fac > 0); as B fragments.
    auto weigh = [&](auto& S, int rows, auto& ph, auto& pl) {
        constexpr int N = sizeof(S) / sizeof(S[0]);
        if (rows < 16 * N) {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (16 * i + 8 * (e >> 1) + gid >= rows) S[i][e] = -INFINITY;
        }
        float top[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            top[h] = fmaxf(S[0][h], S[0][2 + h]);
#pragma unroll
            for (int i = 1; i < N; ++i) top[h] = fmaxf(top[h], fmaxf(S[i][h], S[i][2 + h]));
            top[h] *= fac[h];
        }
        if (__any_sync(0xffffffffu, top[0] > m[0] + SLACK || top[1] > m[1] + SLACK)) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], o));
                const float now = fmaxf(m[h], top[h]), f = m[h] == now ? 1.f : tc::ex2(m[h] - now);
                m[h] = now;
#pragma unroll
                for (int t = 0; t < C::O_TILES; ++t) { O[t][h] *= f; O[t][2 + h] *= f; }
                L[h] *= f;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float a = tc::ex2(fmaf(S[i][2 * h], fac[0], -m[0])), b = tc::ex2(fmaf(S[i][2 * h + 1], fac[1], -m[1]));
                const uint32_t hi = pack_h2(a, b);
                ph[i][h] = transpose(hi);
                if constexpr (EXACT) {
                    const float2 f = unpack_h2(hi);
                    pl[i][h] = transpose(pack_h2(a - f.x, b - f.y));
                }
            }
    };
    // Sums of 16 rows x, times their weights; lo: second parts of the rows, where there are any.
    auto add_rows = [&](const uint32_t (&x)[2][C::PAIRS], const uint32_t (&ph)[2], const uint32_t (&pl)[2], const auto& lo, auto with_lo) {
#pragma unroll
        for (int t = 0; t < C::O_TILES; ++t) {
            const uint32_t a0 = transpose(x[0][2 * t]), a1 = transpose(x[0][2 * t + 1]), a2 = transpose(x[1][2 * t]), a3 = transpose(x[1][2 * t + 1]);
            if constexpr (EXACT) {
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
                mma(sum, a0, a1, a2, a3, pl[0], pl[1]);
                if constexpr (with_lo.value) mma(sum, transpose(lo[0][2 * t]), transpose(lo[0][2 * t + 1]), transpose(lo[1][2 * t]), transpose(lo[1][2 * t + 1]), ph[0], ph[1]);
                mma(sum, a0, a1, a2, a3, ph[0], ph[1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) O[t][e] += sum[e];
            } else {
                mma(O[t], a0, a1, a2, a3, ph[0], ph[1]);
            }
        }
        constexpr uint32_t ONE = 0x3c003c00u;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        if constexpr (EXACT) mma(sum, ONE, ONE, ONE, ONE, pl[0], pl[1]);
        mma(sum, ONE, ONE, ONE, ONE, ph[0], ph[1]);
        L[0] += sum[0]; L[1] += sum[1];
    };

    // The 16 rows at row0 turned back by their positions; lo: second parts.
    auto turn_back = [&](const unsigned char* tile, int row0, uint32_t (&x)[2][C::PAIRS], auto& lo) {
        int32_t pos[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) pos[h] = reinterpret_cast<const int32_t*>(tile + C::POS_AT)[row0 + 8 * h + gid];
#pragma unroll
        for (int j = 0; j < C::PAIRS / 2; ++j) {
            const int ch = tig * (D / 8) + 2 * j;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t &u = x[h][j], &v = x[h][C::PAIRS / 2 + j];
                if constexpr (EXACT) {
                    uint64_t cs, sn;
                    rope_cos_sin2(rope_angle(pos[h], phase64[ch]), rope_angle(pos[h], phase64[ch + 1]), cs, sn);
                    const float2 uf = unpack_h2(u), vf = unpack_h2(v);
                    const uint64_t u2 = tc::pack2(uf.x, uf.y), v2 = tc::pack2(vf.x, vf.y);
                    auto parts = [](uint64_t z, uint32_t& hi, uint32_t& low) {
                        float a, b;
                        tc::unpack2(z, a, b);
                        hi = pack_h2(a, b);
                        const float2 f = unpack_h2(hi);
                        low = pack_h2(a - f.x, b - f.y);
                    };
                    parts(tc::fma2(u2, cs, tc::mul2(v2, sn)), u, lo[h][j]);
                    parts(tc::fma2(u2, tc::mul2(sn, tc::pack2(-1.f, -1.f)), tc::mul2(v2, cs)), v, lo[h][C::PAIRS / 2 + j]);
                } else {
                    const uint2 ph2 = *reinterpret_cast<const uint2*>(&phase32[ch]);
                    float c0, s0, c1, s1;
                    turn_cos_sin((uint32_t)pos[h] * ph2.x, c0, s0);
                    turn_cos_sin((uint32_t)pos[h] * ph2.y, c1, s1);
                    const uint32_t cs = pack_h2(c0, c1), sn = pack_h2(s0, s1), a = u, b = v;
                    u = fma_h2(a, cs, mul_h2(b, sn));
                    v = fma_h2(neg_h2(a), sn, mul_h2(b, cs));
                }
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

    int at = 0, phase = 0;                                              // the entry at hand, and its barrier's phase
    auto wait = [&] {
        if (tma::mbar_wait_warp(&full[wid][at], phase, fault, 21)) return true;
        for (; ahead > 0; --ahead) {                                   // copies in flight still land in this block's memory
            tma::mbar_wait_warp(&full[wid][at], phase, fault, 21);
            if (++at == ENTRIES) { at = 0; phase ^= 1; }
        }
        return false;
    };
    auto release = [&](int s) {
        __syncwarp();                                                  // every lane has read the entry
        --ahead;
        if (run.count > 0) { issue(s); ++ahead; __syncwarp(); }
    };
    // What lies behind the last row may be no number: scales of zero there.
    auto blank = [&](unsigned char* tile, int rows) {
        for (int i = rows * R::GROUPS + lane; i < q4::ROWS * R::GROUPS; i += 32) tile[R::SCALES_AT + i] = 0;
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
    };
    while (ahead > 0) {
        if (!wait()) return;
        const Entry entry = entries[wid][at];
        const int tier = entry.kind == KEY_ONLY;
        if (entry.unit != unit) {
            leave_unit();
            unit = entry.unit; apx = tier; wrote = 0;
            slot_rec = entry.first ? unit : units + worker;
            clear();
            load_queries(unit);
        } else if (tier != apx) {
            put_tier(apx, false);
            wrote |= 1 << apx;
            apx = tier;
            clear();
        }
        unsigned char* tile = ring + at * C::ENTRY_BYTES;
        if (!tier) {
            const unsigned char* keys = tile;
            const int of_keys = at;
            if (++at == ENTRIES) { at = 0; phase ^= 1; }
            if (!wait()) return;
            tile = ring + at * C::ENTRY_BYTES;
            if (entry.rows < q4::ROWS) blank(tile, entry.rows);
#pragma unroll 1
            for (int row0 = 0; row0 < entry.rows; row0 += 32) {
                uint32_t x[2][C::PAIRS], ph[2][2], pl[2][2];
                float S[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    load_rows(keys, row0 + 16 * i, x);
                    logits(x, S[i]);
                }
                weigh(S, entry.rows - row0, ph, pl);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    load_rows(tile, row0 + 16 * i, x);
                    add_rows(x, ph[i], pl[i], x, std::false_type());
                }
            }
            release(of_keys);
        } else {
            constexpr int N = C::N_APX;
            if (entry.rows < q4::ROWS) blank(tile, entry.rows);
#pragma unroll 1
            for (int row0 = 0; row0 < entry.rows; row0 += 16 * N) {
                uint32_t x[N][2][C::PAIRS], ph[N][2], pl[N][2], lo[ROPE && EXACT ? N : 1][ROPE && EXACT ? 2 : 1][ROPE && EXACT ? C::PAIRS : 1];
                float S[N][4];
#pragma unroll
                for (int i = 0; i < N; ++i) load_rows(tile, row0 + 16 * i, x[i]);
#pragma unroll
                for (int i = 0; i < N; ++i) logits(x[i], S[i]);
                weigh(S, entry.rows - row0, ph, pl);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if constexpr (ROPE) turn_back(tile, row0 + 16 * i, x[i], lo[EXACT ? i : 0]);
                    add_rows(x[i], ph[i], pl[i], lo[ROPE && EXACT ? i : 0], std::bool_constant<ROPE && EXACT>());
                }
            }
        }
        release(at);
        if (++at == ENTRIES) { at = 0; phase ^= 1; }
    }
    leave_unit();
}

constexpr int MERGE_THREADS = 256;
constexpr int FEW_PIECES = 4;        // records of a unit that every thread weighs for itself
constexpr int MERGE_CHUNK = 64;      // records weighed at a time where there are more

// The map's rows 16 w + gid and 16 w + gid + 8 as a thread holds them: channels 32 i + 8 tig .. + 7 of each.
template <typename T, int D> struct MapRows;
template <int D> struct MapRows<__nv_bfloat16, D> {
    static constexpr int PARTS = 1;
    uint4 w[2][D / 32];
    __device__ __forceinline__ void load(const __nv_bfloat16* W, int tig) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) w[h][i] = *reinterpret_cast<const uint4*>(W + h * 8 * D + 32 * i + 8 * tig);
    }
    __device__ __forceinline__ void pairs(int h, int i, uint32_t (&p)[4][1]) const { p[0][0] = w[h][i].x; p[1][0] = w[h][i].y; p[2][0] = w[h][i].z; p[3][0] = w[h][i].w; }
};
template <int D> struct MapRows<float, D> {
    static constexpr int PARTS = 3;
    float4 w[2][D / 16];
    __device__ __forceinline__ void load(const float* W, int tig) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < D / 16; ++i) w[h][i] = *reinterpret_cast<const float4*>(W + h * 8 * D + 32 * (i / 2) + 8 * tig + 4 * (i % 2));
    }
    __device__ __forceinline__ void pairs(int h, int i, uint32_t (&p)[4][3]) const {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float4 v = w[h][2 * i + j];
            split_bf16<3>(v.x, v.y, p[2 * j]);
            split_bf16<3>(v.z, v.w, p[2 * j + 1]);
        }
    }
};

// The records of a unit into its outputs.
template <typename T, int D, typename TO>
__global__ void __launch_bounds__(MERGE_THREADS)
decode_q4_merge(const unsigned char* ws, Cache c, int g, Costs cost, int most_workers, const T* W, TO* __restrict__ out) {
    constexpr int NW = MERGE_THREADS / 32, ROWS_W = 16;
    __shared__ __align__(16) float val[8][D + 4], keys[8][D + 4];
    __shared__ float ref[8], inv[8], fac[2][8][MERGE_CHUNK];
    const int u = blockIdx.x, b = u / c.LH, lh = u - b * c.LH;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    MapRows<T, D> map;                   // requested ahead of the wait: the streaming kernel does not write it
    if (wid < D / ROWS_W) map.load(W + ((size_t)lh * D + ROWS_W * wid + gid) * D, tig);
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    const int64_t* prefix = reinterpret_cast<const int64_t*>(ws);
    const float* records = reinterpret_cast<const float*>(ws + prefix_bytes(c.batch));
    const int heads = even_heads(g), tier = tier_floats(g, D), units = c.batch * c.LH;
    const int64_t p0 = prefix[b], p1 = prefix[b + 1], X = prefix[c.batch];
    const int nr = tiles_of(rows_of(c.ret_len, b, c.ret_width)), na = tiles_of(rows_of(c.apx_len, b, c.apx_width));
    TO* o = out + (size_t)u * g * D;
    if (p0 == p1) {                                                   // nothing to attend to
        for (int e = threadIdx.x; e < g * D; e += MERGE_THREADS) store_out(o + e, 0.f);
        return;
    }
    const int64_t unit_cost = (int64_t)cost.ret * nr + (int64_t)cost.apx * na, from = p0 + lh * unit_cost;
    const Deal deal(X, most_workers, cost);
    const int w0 = deal.owner(from);
    int last = deal.owner(from + unit_cost - 1);
    if (last > w0 && tile_from(deal.begin(last) - from, nr, cost) >= nr + na) --last;       // its range begins within the unit's last tile
    const int pieces = last - w0 + 1;                                 // the unit's own record, then those of workers w0 + 1 ..
    const float *own = records + (size_t)u * 2 * tier, *others = records + (size_t)(units + w0) * 2 * tier;
    auto piece = [&](int i) { return i == 0 ? own : others + (size_t)i * 2 * tier; };
    // Four numbers of a tier's sums are a thread's: rows `row` and `row` + 8 of O tile t, heads 2 hp and 2 hp + 1.
    const int quads = D / 16 * (heads / 2) * 8;
    auto put = [&](int which, int i, float4 a) {
        const int row = i & 7, hp = (i >> 3) % (heads / 2), t = (i >> 3) / (heads / 2);
        float (*to)[D + 4] = which ? keys : val;                      // channel pairs 2 t and 2 t + 1 of piece row / 2
        const int c0 = q4::Row<D>::channel_of(row / 2 * (D / 4) + 4 * t + row % 2), c1 = q4::Row<D>::channel_of(row / 2 * (D / 4) + 4 * t + 2 + row % 2);
        to[2 * hp][c0] = a.x; to[2 * hp + 1][c0] = a.y; to[2 * hp][c1] = a.z; to[2 * hp + 1][c1] = a.w;
    };
    auto add = [](float4& a, float f0, float f1, const float4& v) {
        a.x = fmaf(f0, v.x, a.x); a.y = fmaf(f1, v.y, a.y); a.z = fmaf(f0, v.z, a.z); a.w = fmaf(f1, v.w, a.w);
    };
    if (pieces <= FEW_PIECES) {
        // everything a thread needs is requested at once: the heads' references and sums of all records, and its numbers
        for (int e = threadIdx.x; e < 2 * quads; e += MERGE_THREADS) {
            const int which = e >= quads, i = e - which * quads, hp = (i >> 3) % (heads / 2);
            float4 ml[FEW_PIECES][2], v[FEW_PIECES];
#pragma unroll
            for (int k = 0; k < FEW_PIECES; ++k) {
                ml[k][0] = ml[k][1] = make_float4(-INFINITY, 0.f, -INFINITY, 0.f);
                v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k < pieces) {
                    ml[k][0] = *reinterpret_cast<const float4*>(piece(k) + 4 * hp);
                    ml[k][1] = *reinterpret_cast<const float4*>(piece(k) + tier + 4 * hp);
                    v[k] = *reinterpret_cast<const float4*>(piece(k) + which * tier + 2 * heads + 4 * i);
                }
            }
            float M0 = -INFINITY, M1 = -INFINITY;
#pragma unroll
            for (int k = 0; k < FEW_PIECES; ++k)
#pragma unroll
                for (int r = 0; r < 2; ++r) { M0 = fmaxf(M0, ml[k][r].x); M1 = fmaxf(M1, ml[k][r].z); }
            float L0 = 0.f, L1 = 0.f;
            float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < FEW_PIECES; ++k)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    if (ml[k][r].x == -INFINITY && ml[k][r].z == -INFINITY) continue;      // no such record, or an empty one: its numbers are not any
                    const float f0 = exp2f(ml[k][r].x - M0), f1 = exp2f(ml[k][r].z - M1);
                    L0 = fmaf(f0, ml[k][r].y, L0); L1 = fmaf(f1, ml[k][r].w, L1);
                    if (r == which) add(a, f0, f1, v[k]);
                }
            put(which, i, a);
            if (which == 0 && i < 8 * (heads / 2) && (i & 7) == 0) { inv[2 * hp] = L0 == 0.f ? 0.f : 1.f / L0; inv[2 * hp + 1] = L1 == 0.f ? 0.f : 1.f / L1; }
        }
    } else {
        // a warp a head: the largest reference, the sum of the weights
        for (int h = wid; h < heads; h += NW) {
            float M = -INFINITY;
            for (int i = lane; i < 2 * pieces; i += 32) M = fmaxf(M, piece(i >> 1)[(i & 1) * tier + 2 * h]);
            M = warp_max(M);
            float sum = 0.f;
            for (int i = lane; i < 2 * pieces; i += 32) {
                const float2 ml = *reinterpret_cast<const float2*>(piece(i >> 1) + (i & 1) * tier + 2 * h);
                if (!(ml.x == -INFINITY)) sum = fmaf(exp2f(ml.x - M), ml.y, sum);
            }
            sum = warp_sum(sum);
            if (lane == 0) { ref[h] = M; inv[h] = sum == 0.f ? 0.f : 1.f / sum; }
        }
        float4 a[D / 64] = {};                                        // at most D / 64 rounds of numbers, with eight heads
        for (int k0 = 0; k0 < pieces; k0 += MERGE_CHUNK) {
            const int n = min(pieces - k0, MERGE_CHUNK);
            __syncthreads();
            for (int e = threadIdx.x; e < 2 * heads * n; e += MERGE_THREADS) {
                const int k = e / (2 * heads), r = e - k * 2 * heads, h = r >> 1, which = r & 1;
                const float m = piece(k0 + k)[which * tier + 2 * h];
                fac[which][h][k] = m == -INFINITY ? 0.f : exp2f(m - ref[h]);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                const int e = threadIdx.x + j * MERGE_THREADS;
                if (e >= 2 * quads) break;
                const int which = e >= quads, i = e - which * quads, hp = (i >> 3) % (heads / 2);
                const float *f0 = fac[which][2 * hp], *f1 = fac[which][2 * hp + 1];
                constexpr int UN = 8;
                for (int k = 0; k < n; k += UN) {
                    float4 v[UN];
#pragma unroll
                    for (int z = 0; z < UN; ++z) {
                        v[z] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (k + z < n && (f0[k + z] != 0.f || f1[k + z] != 0.f))
                            v[z] = *reinterpret_cast<const float4*>(piece(k0 + k + z) + which * tier + 2 * heads + 4 * i);
                    }
#pragma unroll
                    for (int z = 0; z < UN; ++z)
                        if (k + z < n) add(a[j], f0[k + z], f1[k + z], v[z]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const int e = threadIdx.x + j * MERGE_THREADS;
            if (e < 2 * quads) put(e >= quads, e >= quads ? e - quads : e, a[j]);
        }
    }
    __syncthreads();
    // ---- the map: its rows down, heads across; the key sums, and an fp32 map, in three bf16 parts, products down to 2^-16 of the largest
    if (wid >= D / ROWS_W) return;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    if (na > 0) {
        const int head = min(gid, heads - 1);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            constexpr int P = MapRows<T, D>::PARTS;
            uint32_t r0[4][P], r1[4][P], part[4][3];
            map.pairs(0, i, r0);
            map.pairs(1, i, r1);
            const float4 k0 = *reinterpret_cast<const float4*>(&keys[head][32 * i + 8 * tig]), k1 = *reinterpret_cast<const float4*>(&keys[head][32 * i + 8 * tig + 4]);
            split_bf16<3>(k0.x, k0.y, part[0]); split_bf16<3>(k0.z, k0.w, part[1]);
            split_bf16<3>(k1.x, k1.y, part[2]); split_bf16<3>(k1.z, k1.w, part[3]);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int p = 2; p >= 0; --p)
#pragma unroll
                    for (int r = P - 1; r >= 0; --r)
                        if (p + r <= 2)
                            asm volatile(
                                "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                                : "+f"(sum[0]), "+f"(sum[1]), "+f"(sum[2]), "+f"(sum[3])
                                : "r"(r0[2 * s][r]), "r"(r1[2 * s][r]), "r"(r0[2 * s + 1][r]), "r"(r1[2 * s + 1][r]), "r"(part[2 * s][p]), "r"(part[2 * s + 1][p]));
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += sum[e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int h = 2 * tig + (e & 1), ch = ROWS_W * wid + 8 * (e >> 1) + gid;
        if (h < g) store_out(o + h * D + ch, (val[h][ch] + acc[e]) * inv[h]);
    }
}

}  // namespace dq4
}  // namespace vec
#endif
