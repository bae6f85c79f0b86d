// The kernels of attention over the 4-bit paged cache (decode_q4.cu).
//
// Streaming kernel.  A tile is a page of one unit: 64 keys and their values, or 64 key-only keys.  The sequence of all units' tiles, each
// weighted by what it costs, is cut into equal contiguous ranges, one per warp: a warp is a worker of its own, which copies its tiles into
// its own ring of slots (cp.async.bulk, one mbarrier a slot) and never waits for another warp.  It keeps one running state for a
// unit's tier and writes it as a partial record when it leaves that.  The lengths lie on the device, so every block sums up the
// sequences' costs itself.
//
// A worker takes 16 or 32 keys at a time.  A stored row's piece t is what lane t of a quad holds of a 16 x 16 fragment whose rows are keys: one 16-byte load (8 for
// 64 channels) of codes and two scales a row, one conversion and one product for two channels, and no exchange between lanes:
//   S^T = K Q^T    m16n8k16, keys down, the query heads across: no padding to sixteen rows of queries
//   softmax        in fp32, against a reference that follows the maximum only when that has moved by more than SLACK (powers of two); the weights go to fp16, LEAD above one
//   O^T += V^T P^T channels down, heads across; both operands are the registers at hand after an 8 x 8 transpose (movmatrix), and so are the key sums
//                  A^T += K^T P^T of key-only keys, from the very registers that gave the logits
// The sum of the weights is one more row of that product, a row of ones, so that a weight's rounding to fp16 is in numerator and denominator alike.
// Stored rows are exact in fp16, so the products are; halves of them too.  Queries are scaled by a power of two a head to fp16's range; fp32 queries take two fp16 parts.
// EXACT (fp32 queries or fp32 output): weights, and keys turned back, in two fp16 parts, and sums of 16 keys added up outside the tensor cores,
// which cut their sums off instead of rounding them.
//
// Merge kernel.  A block combines the records of a unit, or of several sequences' units of one (layer, KV head), applies the map to the key sums on the
// tensor cores (in three bf16 parts: 24 bits) and normalises.
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
template <int RET, int APX> struct Costs { static constexpr int ret = RET, apx = APX, most = RET > APX ? RET : APX; };
// A weight is 2^(logit - reference), and the reference is the largest logit so far less LEAD, or up to SLACK below that: weights reach 2^15 of fp16's range.  They have eleven bits
// down to 2^-14, 2^-27 of the largest, and end at 2^-25, so that thousands of small weights count behind one key that takes nearly all.
// 640 units 183.3 us, 2048 units 127.5; LEAD 7 and SLACK 8, which moves the reference less often, 182.3 and 125.6.
constexpr float LEAD = 13.f, SLACK = 2.f;
static_assert(LEAD + SLACK <= 15.f, "weights are below 65504");
// What second parts are multiplied by, which their products' sums give back: they keep eleven bits where they would be subnormal.
constexpr float PART = 2048.f;

struct Cache {
    const unsigned char *ret, *apx;
    const int32_t *ret_table, *apx_table, *ret_len, *apx_len, *apx_pos;
    int64_t n_ret_pages, n_apx_pages;
    int32_t ret_width, apx_width, LH, batch;
};
// Rows of a sequence in a tier: what its table can hold at the most.
__device__ __forceinline__ int rows_of(const int32_t* len, int b, int width) { return width ? min(max(len[b], 0), width * q4::ROWS) : 0; }
__device__ __forceinline__ int tiles_of(int rows) { return (rows + q4::ROWS - 1) / q4::ROWS; }

// ---- workspace: the first and the last worker of every unit that has tiles, then the records
__host__ __device__ inline size_t ends_bytes(int units) { return ((size_t)units * 8 + 255) & ~(size_t)255; }
// Whether a unit's ends are what workers wrote.  They are not where a streaming warp's wait gave up before it got there: then they are whatever the workspace
// held, and no record's address may come from them.
__host__ __device__ constexpr bool ends_are_workers(int first, int last, int workers) { return first >= 0 && first <= last && last < workers; }
// A record: for each tier [heads, rounded up to even][m, l] and the sums, in the order of the fragments.
__host__ __device__ inline int even_heads(int g) { return (g + 1) & ~1; }
__host__ __device__ inline int tier_floats(int g, int d) { return even_heads(g) * (d + 2); }

// How the cost X of all tiles is dealt to workers.  Every range is as long as a tile at the least, so each begins one.  Where there is work for all workers the
// bounds are the multiples of one fp64 number, the same for all who ask, and a range of more than a tile; where there is not, whole numbers.
struct Deal {
    int64_t X;
    int workers;
    double step;                    // 0: few tiles
    __device__ __forceinline__ Deal(int64_t x, int workers_at_most, int most_cost) : X(x), workers(workers_at_most), step(0.) {
        if (x > (int64_t)workers_at_most * (most_cost + 1)) step = (double)x / workers_at_most;
        else workers = max(min((int)x / most_cost, workers_at_most), 1);
    }
    __device__ __forceinline__ int64_t begin(int w) const {
        if (w == workers) return X;
        return step > 0. ? (int64_t)(step * w) : (int64_t)((uint32_t)X * (uint32_t)w / (uint32_t)workers);      // under 2^32: X is a few times the workers there
    }
};
// a / b, in 32 bits where they do.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// First tile of a unit that begins at r or later, r counted from the unit's beginning.
template <typename Cost> __device__ __forceinline__ int tile_from(int64_t r, int nr) {
    const int64_t ret = (int64_t)Cost::ret * nr;
    return r <= ret ? (int)((r + Cost::ret - 1) / Cost::ret) : nr + (int)((r - ret + Cost::apx - 1) / Cost::apx);
}

// FOLD: EXACT with at most four heads, whose first and second parts of weights are eight columns of one product.
template <typename T, int D, bool ROPE, bool EXACT, bool FOLD> struct Cfg {
    static_assert(EXACT || !FOLD, "one part needs no folding");
    static constexpr int WARPS = EXACT && D == 128 && (!FOLD || ROPE || sizeof(T) == 4) ? 8 : 12;
    static constexpr int ENTRIES = WARPS == 12 ? 3 : 4;                // of a warp's ring, a tile each
    static constexpr int THREADS = 32 * WARPS;
    static constexpr int POS_AT = q4::Row<D>::TILE;                    // of a key-only tile's positions, within an entry
    static constexpr int ENTRY_BYTES = q4::Row<D>::TILE + (ROPE ? 4 * q4::ROWS : 0);
    static constexpr int SMEM_BYTES = WARPS * ENTRIES * ENTRY_BYTES;   // and behind them the prefix sums
    static constexpr int Q_PARTS = sizeof(T) == 4 ? 2 : 1;
    // Rows that may be turned are taken halved: a pair of stored channels, 61440 each, turns to 86889 at the most, and half of that is within fp16's 65504.
    static constexpr float ROW_UNIT = ROPE ? .5f : 1.f;
    static constexpr int PAIRS = D / 8;                                // channel pairs of a lane in a row
    static constexpr int O_TILES = D / 16;
    // Rows of a softmax step, in sixteens.  us by (retained, key-only), 128 units of 3000 and 6000 rows, four heads: 128 channels (2, 1) 44.4, (1, 1) 45.1, (2, 2) 46.1, fp32 results 47.4,
    // 47.9, 49.8, rotary keys 70.8, 70.6, 80, with fp32 results, by the costs (2, 3), 150, 148, 207; 64 channels (2, 2) 32.8, (2, 1) 33.9, (1, 1) 34.1, fp32 results 34.8, 35.9, 36.7, rotary keys, which take
    // (2, 1): 47.1 either way, 48.7.
    static constexpr int N_RET = 2, N_APX = D == 64 && !ROPE ? 2 : 1;
    // What tiles of the tiers cost, (retained, key-only).  us for 128 units of 3000 and 6000 rows, four heads, 128 channels and 64: (4, 3) 44 and 33, (1, 1) 47 and 35, (2, 1) 48 and
    // 34, (2, 3) 52 and 40; fp32 results 47 and 35, 50 and 37, 51 and 37, 55 and 42.  Rotary keys: (2, 3) 70.8 and 47.0, (1, 2) 70.3 and 52.6, (1, 1) 78 and 48, (4, 3) 81 and 49; fp32 results,
    // turned in two parts: (1, 2) 140 and 76, (2, 3) 150 and 80, (1, 1) 171 and 88, (4, 3) 189 and 91.  fp32 queries and eight heads order them alike.
    using Cost = std::conditional_t<!ROPE, Costs<4, 3>, std::conditional_t<EXACT, Costs<1, 2>, Costs<2, 3>>>;
};

// Not volatile, like the transposes: the compiler may move them past one another, so that one's operands are on their way during the next.
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same product on its own: nothing to add it to, and no registers to clear for that.
__device__ __forceinline__ void mma_alone(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
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
// Infinities stay: an infinite query's logits are none.
__device__ __forceinline__ uint32_t pack_h2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Weights, cut off at 65504, which they pass only where logits are 2^23 and more and their last places, by which the reference is lower, are ones.  NaN stays.
__device__ __forceinline__ uint32_t pack_weights(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;\n" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// The reference for a largest logit, which is rounded: under LEAD below it by one or two of its last places, so that the logit itself, before its rounding, is never the lower
// one.  From 2^28 on it could be by 16 and more, and no weight would be left.  An infinite one stays, and gives NaN.
__device__ __forceinline__ float reference(float top) { return top * (top > 0.f ? 1.f - 0x1p-23f : 1.f + 0x1p-23f) - LEAD; }
__device__ __forceinline__ float2 unpack_h2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// A worker's way through the sequence of tiles, as runs: tiles of one tier of one unit.
template <typename Cost> struct Runs {
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
        const int each = apx ? Cost::apx : Cost::ret;
        const int64_t in_range = apx ? (left + Cost::apx - 1) / Cost::apx : (left + Cost::ret - 1) / Cost::ret;
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
        const int nr = tiles_of(n_ret);
        const int64_t unit = (int64_t)Cost::ret * nr + (int64_t)Cost::apx * tiles_of(n_apx);
        lh = (int)divide(x - prefix[b], unit);
        const int64_t r = x - prefix[b] - lh * unit;
        const int t = tile_from<Cost>(r, nr);
        left = end - x - ((int64_t)Cost::ret * min(t, nr) + (int64_t)Cost::apx * max(t - nr, 0) - r);
        run(c, prefix, t);
    }
};

// What an entry of a ring holds, for its consumer: unit, rows that are there, whether it is the unit's first (1) or last (2) tile.
enum Kind { KEYS, VALUES, KEY_ONLY };
struct Entry { int unit, rows, kind, edge; };

// Phases of two neighbouring channel pairs, turns a position: multiples of 2^-32, and what these leave, in radians.
struct __align__(16) TwoPhases { uint32_t turns[2]; float rest[2]; };
__device__ __forceinline__ void put_phase(TwoPhases& to, int which, unsigned long long phase) {
    to.turns[which] = (uint32_t)((phase + 0x80000000ull) >> 32);
    to.rest[which] = (float)(int32_t)(uint32_t)phase * 3.4061215800865545e-19f;      // 2 pi / 2^64
}
// Where the pair of channels 2 j, 2 j + 1 of piece tig's lies: what the four lanes of a quad read together is 64 bytes in a row (in the channels' order they met in one bank:
// 128 units 70.9 us in place of 70.3).
__device__ __forceinline__ constexpr int phase_place(int tig, int j) { return 4 * j + tig; }
// Sine and cosine of a position times a phase.  Of the product modulo a turn the upper 23 bits count (8e-7): they become a number in [1, 2) and that a multiple of 2 pi
// about zero, without a conversion from integers, which would wait for the unit that the sine and the cosine keep busy.  The phase's rest, under 2^-33 of a turn a position,
// comes on top: 1e-4 at position 131072, 0.8 at 2^30 (16 sequences of 3000 and 6000 rows in 8 heads: 70.4 us, without it 67; by an integer product in its place 72.6).
__device__ __forceinline__ void turn_cos_sin(uint32_t pos, float pos_f, uint32_t phase, float rest, float& cs, float& sn) {
    const float turns = __uint_as_float(((pos * phase) >> 9) ^ 0x3fc00000u);         // 1 + (angle + half a turn) modulo a turn
    __sincosf(fmaf(turns, 6.283185307179586f, fmaf(pos_f, rest, -9.42477796076938f)), &sn, &cs);
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

template <typename T, int D, bool ROPE, bool EXACT, bool FOLD>
__global__ void __launch_bounds__(Cfg<T, D, ROPE, EXACT, FOLD>::THREADS, 1)
decode_q4_stream(const T* q, Cache c, int g, float scale_log2e, unsigned char* ws, int* fault, RopePhases phases) {
    using C = Cfg<T, D, ROPE, EXACT, FOLD>;
    using R = q4::Row<D>;
    constexpr int WARPS = C::WARPS, ENTRIES = C::ENTRIES;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t full[WARPS][ENTRIES];
    __shared__ Entry entries[WARPS][ENTRIES];
    __shared__ int64_t sums[WARPS];
    __shared__ TwoPhases phase32[ROPE && !EXACT ? D / 4 : 1];
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
            if constexpr (EXACT) phase64[threadIdx.x] = rope_phase_words(phases.phase[threadIdx.x]);
            else put_phase(phase32[phase_place(threadIdx.x / (D / 8), threadIdx.x % (D / 8) / 2)], threadIdx.x % 2, phases.phase[threadIdx.x]);
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
            x = (int64_t)c.LH * ((int64_t)C::Cost::ret * tiles_of(rows_of(c.ret_len, b, c.ret_width)) + (int64_t)C::Cost::apx * tiles_of(rows_of(c.apx_len, b, c.apx_width)));
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
    const Deal deal(carry, gridDim.x * WARPS, C::Cost::most);
    const int worker = wid * gridDim.x + blockIdx.x;        // neighbours in the sequence on different multiprocessors
    if (carry == 0 || worker >= deal.workers) return;

    const int rec = 2 * tier_floats(g, D), heads = even_heads(g), units = c.batch * c.LH;
    int2* ends = reinterpret_cast<int2*>(ws);
    float* records = reinterpret_cast<float*>(ws + ends_bytes(units));
    unsigned char* ring = smem + wid * ENTRIES * C::ENTRY_BYTES;
    const uint64_t policy = tma::policy_evict_first();

    // ---- the producing side, ENTRIES ahead: `run` is where it is, `k` tiles of it are on their way, and lane l has the page of tile l of 32
    Runs<typename C::Cost> run;
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
                                    run.apx ? KEY_ONLY : values ? VALUES : KEYS,
                                    (p == 0 && (!run.apx || run.n_ret == 0) ? 1 : 0) | (run.apx ? (p + 1) * q4::ROWS >= run.n_apx : run.n_apx == 0 && (p + 1) * q4::ROWS >= run.n_ret ? 1 : 0) << 1};
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
    float fac[2] = {0.f, 0.f}, m[2] = {-INFINITY, -INFINITY}, O[C::O_TILES][4], L[4];
    auto clear = [&] {
        m[0] = m[1] = -INFINITY;
#pragma unroll
        for (int t = 0; t < C::O_TILES; ++t) O[t][0] = O[t][1] = O[t][2] = O[t][3] = 0.f;
        L[0] = L[1] = L[2] = L[3] = 0.f;                               // L: the same sums in all rows, of which two numbers are used
    };
    clear();
    // The queries of a unit as B fragments: head gid, the channels of piece tig.  Scaled so that the largest lies in [2^14, 2^15): channels of 2^-28
    // of it still have eleven bits.
    auto load_queries = [&](int unit) {
        const int head = FOLD ? gid & 3 : gid;
        const T* row = q + ((size_t)unit * g + min(head, g - 1)) * D + tig * (D / 8);
        float x[2 * C::PAIRS];
#pragma unroll
        for (int h = 0; h < 2; ++h) load_run<C::PAIRS>(row + h * (D / 2), &x[h * C::PAIRS]);
        if (head >= g) {
#pragma unroll
            for (int i = 0; i < 2 * C::PAIRS; ++i) x[i] = 0.f;
        }
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < 2 * C::PAIRS; ++i) most = fmaxf(most, fabsf(x[i]));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const int e = min(max((int)(__float_as_uint(most) >> 23) - 127, -100), 127);
        const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
        const float down = fmaxf(scale_log2e / C::ROW_UNIT * __uint_as_float((uint32_t)(127 - 14 + e) << 23), 1.2e-38f);      // above zero: a masked logit stays -inf
        fac[0] = __shfl_sync(0xffffffffu, down, (2 * tig) * 4);
        fac[1] = __shfl_sync(0xffffffffu, down, (2 * tig + 1) * 4);
#pragma unroll
        for (int i = 0; i < C::PAIRS; ++i) {
            const float a = x[2 * i] * up, b = x[2 * i + 1] * up;
            const uint32_t hi = pack_h2(a, b);
            qb[0][i / 2][i % 2] = hi;
            if constexpr (C::Q_PARTS == 2) {
                const float2 f = unpack_h2(hi);
                qb[1][i / 2][i % 2] = pack_h2((a - f.x) * PART, (b - f.y) * PART);
            }
        }
    };
    // Rows row0 + gid and row0 + gid + 8 of a tile as A fragments, times ROW_UNIT (exact: nothing stored is below 2^-18).
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
            const unsigned char* s = tile + R::SCALES_AT + row * R::GROUPS + 2 * (D == 128 ? tig : tig >> 1);
            uint32_t s2[2] = {s[0] * 0x00800080u, s[1] * 0x00800080u};
            if constexpr (ROPE)
#pragma unroll
                for (int i = 0; i < 2; ++i) s2[i] = mul_h2(s2[i], 0x38003800u);
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                uint32_t p[4];
                q4::decode_word(w[j], p);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[h][4 * j + i] = mul_h2(p[i], s2[j / (D / 64)]);
            }
        }
    };
    // Logits of 16 keys, in chains of two products (EXACT) or of half of them. 640 units at D = 128: chains of four 184 us, of two 187, of one 196, of eight
    // 190: shorter ones pay for more sums, longer ones wait for the product before.
    auto logits = [&](const uint32_t (&x)[2][C::PAIRS], float (&S)[4]) {
        constexpr int CHAIN = EXACT ? 2 : C::O_TILES / 2;
#pragma unroll
        for (int p = C::Q_PARTS - 1; p >= 0; --p)
#pragma unroll
            for (int t0 = 0; t0 < C::O_TILES; t0 += CHAIN) {
                float sum[4];
#pragma unroll
                for (int t = t0; t < t0 + CHAIN; ++t) {
                    const uint32_t a0 = x[0][2 * t], a1 = x[1][2 * t], a2 = x[0][2 * t + 1], a3 = x[1][2 * t + 1];
                    if (t == t0) mma_alone(sum, a0, a1, a2, a3, qb[p][t][0], qb[p][t][1]);
                    else mma(sum, a0, a1, a2, a3, qb[p][t][0], qb[p][t][1]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) S[e] = p == C::Q_PARTS - 1 && t0 == 0 ? sum[e] : p == 0 && t0 == 0 ? fmaf(S[e], 1.f / PART, sum[e]) : S[e] + sum[e];
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
        if (__any_sync(0xffffffffu, top[0] > m[0] + (LEAD + SLACK) || top[1] > m[1] + (LEAD + SLACK))) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], o));
                const float now = fmaxf(m[h], reference(top[h])), f = m[h] == now ? 1.f : tc::ex2(m[h] - now);
                m[h] = now;
#pragma unroll
                for (int t = 0; t < C::O_TILES; ++t) { O[t][h] *= f; O[t][2 + h] *= f; }
                L[h] *= f; L[2 + h] *= f;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float a = tc::ex2(fmaf(S[i][2 * h], fac[0], -m[0])), b = tc::ex2(fmaf(S[i][2 * h + 1], fac[1], -m[1]));
                const uint32_t hi = pack_weights(a, b);
                if constexpr (EXACT) {
                    const float2 f = unpack_h2(hi);
                    const uint32_t low = pack_weights((a - f.x) * PART, (b - f.y) * PART);
                    ph[i][h] = transpose(FOLD && tig >= 2 ? low : hi);
                    if constexpr (!FOLD) pl[i][h] = transpose(low);
                } else {
                    ph[i][h] = transpose(hi);
                }
            }
    };
    // Sums of 16 rows x, times their weights; lo: second parts of the rows, where there are any, PART times as large.
    auto add_rows = [&](const uint32_t (&x)[2][C::PAIRS], const uint32_t (&ph)[2], const uint32_t (&pl)[2], const auto& lo, auto with_lo) {
#pragma unroll
        for (int t = 0; t < C::O_TILES; ++t) {
            const uint32_t a0 = transpose(x[0][2 * t]), a1 = transpose(x[0][2 * t + 1]), a2 = transpose(x[1][2 * t]), a3 = transpose(x[1][2 * t + 1]);
            if constexpr (EXACT) {
                float sum[4];
                mma_alone(sum, a0, a1, a2, a3, ph[0], ph[1]);
                if constexpr (!FOLD || with_lo.value) {
                    float second[4];
                    if constexpr (!FOLD) mma_alone(second, a0, a1, a2, a3, pl[0], pl[1]);
                    if constexpr (with_lo.value) {
                        const uint32_t l0 = transpose(lo[0][2 * t]), l1 = transpose(lo[0][2 * t + 1]), l2 = transpose(lo[1][2 * t]), l3 = transpose(lo[1][2 * t + 1]);
                        if constexpr (FOLD) mma_alone(second, l0, l1, l2, l3, ph[0], ph[1]);
                        else mma(second, l0, l1, l2, l3, ph[0], ph[1]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] = fmaf(second[e], 1.f / PART, sum[e]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) O[t][e] += sum[e];
            } else {
                mma(O[t], a0, a1, a2, a3, ph[0], ph[1]);
            }
        }
        constexpr uint32_t ONE = 0x3c003c00u;
        if constexpr (EXACT) {
            float sum[4];
            mma_alone(sum, ONE, ONE, ONE, ONE, ph[0], ph[1]);
            if constexpr (!FOLD) {
                float second[4];
                mma_alone(second, ONE, ONE, ONE, ONE, pl[0], pl[1]);
                sum[0] = fmaf(second[0], 1.f / PART, sum[0]); sum[1] = fmaf(second[1], 1.f / PART, sum[1]);
            }
            L[0] += sum[0]; L[1] += sum[1];
        } else {
            mma(L, ONE, ONE, ONE, ONE, ph[0], ph[1]);
        }
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
                        low = pack_h2((a - f.x) * PART, (b - f.y) * PART);
                    };
                    parts(tc::fma2(u2, cs, tc::mul2(v2, sn)), u, lo[h][j]);
                    parts(tc::fma2(u2, tc::mul2(sn, tc::pack2(-1.f, -1.f)), tc::mul2(v2, cs)), v, lo[h][C::PAIRS / 2 + j]);
                } else {
                    const TwoPhases two = phase32[phase_place(tig, j)];
                    const float at = (float)pos[h];
                    float c0, s0, c1, s1;
                    turn_cos_sin((uint32_t)pos[h], at, two.turns[0], two.rest[0], c0, s0);
                    turn_cos_sin((uint32_t)pos[h], at, two.turns[1], two.rest[1], c1, s1);
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
        if constexpr (FOLD)
            if (!empty) {                                              // columns of first and second parts become one
#pragma unroll
                for (int t = 0; t < C::O_TILES; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) O[t][e] = fmaf(__shfl_xor_sync(0xffffffffu, O[t][e], 2), 1.f / PART, O[t][e]);      // the lower lanes', which hold the first parts
#pragma unroll
                for (int h = 0; h < 2; ++h) L[h] = fmaf(__shfl_xor_sync(0xffffffffu, L[h], 2), 1.f / PART, L[h]);
            }
        if (2 * tig >= heads) return;
        if (gid == 0) *reinterpret_cast<float4*>(p + 4 * tig) = empty ? make_float4(-INFINITY, 0.f, -INFINITY, 0.f) : make_float4(m[0], L[0], m[1], L[1]);
        if (empty) return;
        float4* o = reinterpret_cast<float4*>(p + 2 * heads);
#pragma unroll
        for (int t = 0; t < C::O_TILES; ++t) {
            constexpr float back = 1.f / C::ROW_UNIT;
            o[(t * (heads / 2) + tig) * 8 + gid] = make_float4(O[t][0] * back, O[t][1] * back, O[t][2] * back, O[t][3] * back);
        }
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
    bool fresh = false;                                                // whether a unit's queries are still to be fetched
    if (ahead > 0) load_queries(entries[wid][0].unit);                 // while the first tile is on its way
    while (ahead > 0) {
        if (!wait()) return;
        const Entry entry = entries[wid][at];
        const int tier = entry.kind == KEY_ONLY;
        if (entry.unit != unit) {
            leave_unit();
            unit = entry.unit; apx = tier; wrote = 0;
            slot_rec = entry.edge & 1 ? unit : units + worker;
            clear();
            if (fresh) load_queries(unit);
            fresh = true;
        } else if (tier != apx) {
            put_tier(apx, false);
            wrote |= 1 << apx;
            apx = tier;
            clear();
        }
        if (lane == 0) {
            if (entry.edge & 1) ends[unit].x = worker;
            if (entry.edge & 2) ends[unit].y = worker;
        }
        unsigned char* tile = ring + at * C::ENTRY_BYTES;
        if (!tier) {
            const unsigned char* keys = tile;
            const int of_keys = at;
            if (++at == ENTRIES) { at = 0; phase ^= 1; }
            if (!wait()) return;
            tile = ring + at * C::ENTRY_BYTES;
            constexpr int N = C::N_RET;
            if (entry.rows < q4::ROWS) blank(tile, entry.rows);
#pragma unroll 1
            for (int row0 = 0; row0 < entry.rows; row0 += 16 * N) {
                uint32_t x[2][C::PAIRS], ph[N][2], pl[N][2];
                float S[N][4];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    load_rows(keys, row0 + 16 * i, x);
                    logits(x, S[i]);
                }
                weigh(S, entry.rows - row0, ph, pl);
#pragma unroll
                for (int i = 0; i < N; ++i) {
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

// Threads of a merge block, which takes the records of a unit in groups of MERGE_THREADS, each a part of the records.
constexpr int MERGE_THREADS = 256, MERGE_MOST = 1024;
constexpr int MERGE_CHUNK = 64;      // records of a unit that are weighed at a time
constexpr float EMPTY = -1.f;        // in place of the factor of a record without rows

// The map in shared memory, its 16-byte pieces so that a fragment's rows do not meet in a bank: pieces of odd rows change places.
template <typename T, int D> struct MapTile {
    static constexpr int PIECES = D * sizeof(T) / 16, BYTES = D * PIECES * 16, FLIP = sizeof(T) == 2 ? 4 : 1, PARTS = sizeof(T) == 2 ? 1 : 3;
    __device__ __forceinline__ static int at(int row, int piece) { return (row * PIECES + (piece ^ ((row & 1) * FLIP))) * 16; }
    template <int THREADS> __device__ __forceinline__ static void request(unsigned char* to, const T* W) {
        for (int i = threadIdx.x; i < D * PIECES; i += THREADS)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(tma::smem_u32(to + at(i / PIECES, i % PIECES))), "l"(reinterpret_cast<const uint4*>(W) + i) : "memory");
        asm volatile("cp.async.commit_group;\n" ::: "memory");
    }
    // Channels 32 i + 8 tig .. + 7 of a row, as four pairs in PARTS bf16 parts.
    __device__ __forceinline__ static void pairs(const unsigned char* from, int row, int i, int tig, uint32_t (&p)[4][PARTS]) {
        if constexpr (PARTS == 1) {
            const uint4 v = *reinterpret_cast<const uint4*>(from + at(row, 4 * i + tig));
            p[0][0] = v.x; p[1][0] = v.y; p[2][0] = v.z; p[3][0] = v.w;
        } else {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 v = *reinterpret_cast<const float4*>(from + at(row, 8 * i + 2 * tig + j));
                split_bf16<3>(v.x, v.y, p[2 * j]);
                split_bf16<3>(v.z, v.w, p[2 * j + 1]);
            }
        }
    }
};

// A merge block's own shared memory beside the map, and how many blocks a multiprocessor holds: by registers four (bf16 maps) or three, by its 228 KB of shared memory, of which
// the system takes one a block, two of fp32 maps of 128 channels (64 KB).
template <int D> constexpr int merge_shared() { return 2 * 8 * (D + 4) * 4 + 3 * 8 * 4 + 2 * 8 * MERGE_CHUNK * 4 + MERGE_CHUNK * 2 * 8 * 8; }
template <typename T, int D, int THREADS> constexpr int merge_blocks() {
    constexpr int by_registers = THREADS == MERGE_MOST ? 1 : sizeof(T) == 2 ? 4 : 3, by_memory = 228 * 1024 / (MapTile<T, D>::BYTES + merge_shared<D>() + 1024);
    return by_memory < by_registers ? by_memory : by_registers;
}

// The records of `seqs` sequences' units of one (layer, KV head) into their outputs: the map is fetched once for all of them.
// HP: pairs of heads; workers: of the streaming kernel.
template <typename T, int D, int HP, int THREADS>
__global__ void __launch_bounds__(THREADS, (merge_blocks<T, D, THREADS>()))
decode_q4_merge(const unsigned char* ws, Cache c, int g, int seqs, int workers, const T* W, void* __restrict__ out, int out_bf16) {
    constexpr int NW = THREADS / 32, GROUPS = THREADS / MERGE_THREADS, ROWS_W = 16, heads = 2 * HP;
    // Four numbers of a tier's sums are a thread's, ROUNDS times at the most: rows `row` and `row` + 8 of O tile t, heads 2 hp and 2 hp + 1.
    constexpr int quads = D / 16 * HP * 8, ROUNDS = (2 * quads + MERGE_THREADS - 1) / MERGE_THREADS;
    using Map = MapTile<T, D>;
    extern __shared__ __align__(16) unsigned char map[];
    __shared__ __align__(16) float val[8][D + 4], keys[8][D + 4];
    __shared__ float ref[8], sum[8], scale[8], fac[2][8][MERGE_CHUNK];
    __shared__ float2 ml[MERGE_CHUNK][2][8];
    const int lh = blockIdx.x % c.LH, b0 = blockIdx.x / c.LH * seqs;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    const int group = threadIdx.x / MERGE_THREADS, t0 = threadIdx.x % MERGE_THREADS;
    Map::template request<THREADS>(map, W + (size_t)lh * D * D);           // ahead of the wait: the streaming kernel does not write it
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    const int units = c.batch * c.LH;
    constexpr int tier = heads * (D + 2);
    auto put_out = [&](size_t at, float x) {
        if (out_bf16) reinterpret_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(x);
        else reinterpret_cast<float*>(out)[at] = x;
    };
    for (int b = b0; b < min(b0 + seqs, c.batch); ++b) {
        const int u = b * c.LH + lh;
        const int n_apx = rows_of(c.apx_len, b, c.apx_width), n_ret = rows_of(c.ret_len, b, c.ret_width);
        const int2 ends = reinterpret_cast<const int2*>(ws)[u];
        const float* records = reinterpret_cast<const float*>(ws + ends_bytes(units));
        const size_t o = (size_t)u * g * D;
        if (n_ret + n_apx == 0) {                                     // nothing to attend to, and no record
            for (int e = threadIdx.x; e < g * D; e += THREADS) put_out(o + e, 0.f);
            continue;
        }
        if (!ends_are_workers(ends.x, ends.y, workers)) {
            for (int e = threadIdx.x; e < g * D; e += THREADS) put_out(o + e, __int_as_float(0x7fffffff));
            continue;
        }
        const int pieces = ends.y - ends.x + 1;                       // the unit's own record, then those of the workers behind its first
        const float *own = records + (size_t)u * 2 * tier, *others = records + (size_t)(units + ends.x) * 2 * tier;
        auto piece = [&](int i) { return i == 0 ? own : others + (size_t)i * 2 * tier; };
        float4 a[ROUNDS] = {};
        for (int k0 = 0; k0 < pieces; k0 += MERGE_CHUNK) {
            const int n = min(pieces - k0, MERGE_CHUNK);
            constexpr int UN = 4;                                     // numbers of so many records are requested at a time
            float4 v[UN];
            auto request = [&](int j, int k) {
                const int e = t0 + j * MERGE_THREADS, which = e >= quads, i = e - which * quads;
                if (e >= 2 * quads) return;
#pragma unroll
                for (int z = 0; z < UN; ++z)
                    if (k + z * GROUPS < n) v[z] = *reinterpret_cast<const float4*>(piece(k0 + k + z * GROUPS) + which * tier + 2 * heads + 4 * i);
            };
            for (int e = threadIdx.x; e < 2 * heads * n; e += THREADS) {
                const int k = e / (2 * heads), r = e - k * 2 * heads, which = r >= heads, h = r - which * heads;
                ml[k][which][h] = *reinterpret_cast<const float2*>(piece(k0 + k) + which * tier + 2 * h);
            }
            request(0, group);
            __syncthreads();
            // a warp a head: the largest reference so far, what the sums so far and every record take against it
            for (int h = wid; h < heads; h += NW) {
                const float before = k0 ? ref[h] : -INFINITY;
                float M = before;
                for (int i = lane; i < 2 * n; i += 32) M = fmaxf(M, ml[i >> 1][i & 1][h].x);
                M = warp_max(M);
                float L = 0.f;
                // An empty record has no sum either, and its numbers are not any.  One of logits that are all NaN has no reference, but a sum, which is NaN: its factor is
                // zero or NaN, its numbers count.  So does one whose factor is zero because its logits are small.
                for (int i = lane; i < 2 * n; i += 32) {
                    const float2 x = ml[i >> 1][i & 1][h];
                    const bool empty = x.x == -INFINITY && x.y == 0.f;
                    const float f = empty ? EMPTY : exp2f(x.x - M);
                    if (!empty) L = fmaf(f, x.y, L);
                    fac[i & 1][h][i >> 1] = f;
                }
                L = warp_sum(L);
                if (lane == 0) {
                    const float f = before == -INFINITY ? 0.f : exp2f(before - M);
                    scale[h] = f;
                    ref[h] = M;
                    sum[h] = k0 ? fmaf(f, sum[h], L) : L;
                }
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < ROUNDS; ++j) {
                const int e = t0 + j * MERGE_THREADS, which = e >= quads, i = e - which * quads, hp = (i >> 3) % HP;
                if (e >= 2 * quads) break;
                const float *f0 = fac[which][2 * hp], *f1 = fac[which][2 * hp + 1];
                if (k0) { const float s0 = scale[2 * hp], s1 = scale[2 * hp + 1]; a[j].x *= s0; a[j].y *= s1; a[j].z *= s0; a[j].w *= s1; }
                if (j) request(j, group);
                for (int k = group; k < n;) {
                    const float4 w[UN] = {v[0], v[1], v[2], v[3]};
                    const int at = k;
                    if ((k += UN * GROUPS) < n) request(j, k);
#pragma unroll
                    for (int z = 0; z < UN; ++z) {
                        if (at + z * GROUPS >= n) break;
                        const float x0 = f0[at + z * GROUPS], x1 = f1[at + z * GROUPS];
                        if (x0 == EMPTY) continue;                     // then so is x1: a tier of a record is empty for all heads
                        a[j].x = fmaf(x0, w[z].x, a[j].x); a[j].y = fmaf(x1, w[z].y, a[j].y); a[j].z = fmaf(x0, w[z].z, a[j].z); a[j].w = fmaf(x1, w[z].w, a[j].w);
                    }
                }
            }
            if (k0 + MERGE_CHUNK < pieces) __syncthreads();
        }
        // the groups' sums, one after another
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) {
            if (group == q) {
#pragma unroll
                for (int j = 0; j < ROUNDS; ++j) {
                    const int e = t0 + j * MERGE_THREADS, which = e >= quads, i = e - which * quads;
                    if (e >= 2 * quads) break;
                    const int row = i & 7, hp = (i >> 3) % HP, t = (i >> 3) / HP;
                    float (*to)[D + 4] = which ? keys : val;          // channel pairs 2 t and 2 t + 1 of piece row / 2
                    const int c0 = q4::Row<D>::channel_of(row / 2 * (D / 4) + 4 * t + row % 2), c1 = q4::Row<D>::channel_of(row / 2 * (D / 4) + 4 * t + 2 + row % 2);
                    if (q) { a[j].x += to[2 * hp][c0]; a[j].y += to[2 * hp + 1][c0]; a[j].z += to[2 * hp][c1]; a[j].w += to[2 * hp + 1][c1]; }
                    to[2 * hp][c0] = a[j].x; to[2 * hp + 1][c0] = a[j].y; to[2 * hp][c1] = a[j].z; to[2 * hp + 1][c1] = a[j].w;
                }
            }
            if (q + 1 < GROUPS) __syncthreads();
        }
        asm volatile("cp.async.wait_group 0;\n" ::: "memory");
        __syncthreads();
        // ---- the map: its rows down, heads across; the key sums, and an fp32 map, in three bf16 parts, products down to 2^-16 of the largest
        if (wid < D / ROWS_W) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
            if (n_apx > 0) {
                const int head = min(gid, heads - 1);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    constexpr int P = Map::PARTS;
                    uint32_t r0[4][P], r1[4][P], part[4][3];
                    Map::pairs(map, ROWS_W * wid + gid, i, tig, r0);
                    Map::pairs(map, ROWS_W * wid + 8 + gid, i, tig, r1);
                    const float4 x0 = *reinterpret_cast<const float4*>(&keys[head][32 * i + 8 * tig]), x1 = *reinterpret_cast<const float4*>(&keys[head][32 * i + 8 * tig + 4]);
                    split_bf16<3>(x0.x, x0.y, part[0]); split_bf16<3>(x0.z, x0.w, part[1]);
                    split_bf16<3>(x1.x, x1.y, part[2]); split_bf16<3>(x1.z, x1.w, part[3]);
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        float once[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int p = 2; p >= 0; --p)
#pragma unroll
                            for (int r = P - 1; r >= 0; --r)
                                if (p + r <= 2)
                                    asm volatile(
                                        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                                        : "+f"(once[0]), "+f"(once[1]), "+f"(once[2]), "+f"(once[3])
                                        : "r"(r0[2 * s][r]), "r"(r1[2 * s][r]), "r"(r0[2 * s + 1][r]), "r"(r1[2 * s + 1][r]), "r"(part[2 * s][p]), "r"(part[2 * s + 1][p]));
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[e] += once[e];
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int h = 2 * tig + (e & 1), ch = ROWS_W * wid + 8 * (e >> 1) + gid;
                if (h < g) put_out(o + h * D + ch, sum[h] == 0.f ? 0.f : (val[h][ch] + acc[e]) / sum[h]);
            }
        }
        __syncthreads();                                              // the sums are free for the next sequence
    }
    asm volatile("cp.async.wait_group 0;\n" ::: "memory");
}

}  // namespace dq4
}  // namespace vec
#endif
