// What writes and reads the 8-bit paged cache (q8.cuh): compaction of a routed context into its pages, new rows of generated or drafted tokens and
// prompts, and rows read back.  A block of threads has a page's tile of one (layer, KV head): its rows' largest magnitude decides their scale.
#include "common.cuh"
#include "internal.h"
#include "q8.cuh"
#include "rope.cuh"

namespace vec {
namespace q8 {

// us, 256 units of 13100 rows, 128 channels of bf16 (197 at the copy rate, either way): compaction 205, with the rows requested behind the table's answer and
// compared as fp32 numbers 290; reading back 198, a run at a time 244.  fp32 (329) 328 and 444; 64 channels of bf16 (99) 128 and 119, of fp32 (164) 187 and 245.
constexpr int THREADS = 128;

// How a tile's rows are dealt to the threads: 16 bytes of a stored row each, E channels.
template <typename T, int D> struct Deal {
    static constexpr int E = 16 / (int)sizeof(T), LANES = D / E, PER = THREADS / LANES, PASSES = ROWS / PER;
    static_assert(PASSES * PER == ROWS && LANES <= 32, "whole rows, a row within a warp");
};
__device__ __forceinline__ void widen(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void widen(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
}
template <int E> __device__ __forceinline__ void put_codes(unsigned char* to, const float (&x)[E], float inv) {
    const uint32_t lo = to_codes(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    if constexpr (E == 8) *reinterpret_cast<uint2*>(to) = make_uint2(lo, to_codes(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
    else *reinterpret_cast<uint32_t*>(to) = lo;
}

struct Pools {
    unsigned char *ret, *apx;
    int32_t *ret_pos, *apx_pos;
    const int32_t *ret_table, *apx_table, *ret_len, *apx_len;
    uint32_t n_ret_pages, n_apx_pages;
    int ret_width, apx_width, LH;
};
// Rows of a sequence: what its table can hold at the most.
__device__ __forceinline__ int rows_of(const int32_t* len, int b, int width) { return width ? min(max(len[b], 0), width * ROWS) : 0; }
// A block of rows of a sequence's tier; which: 0 = keys, 1 = values of a retained page, 2 = keys of a key-only page.
template <int D> struct Place {
    int rows;                    // of the sequence's tier
    unsigned char* tile;         // null: the block has no page in the pool
    int32_t* pos;                // of the tile's rows, or null
    __device__ __forceinline__ Place(const Pools& p, int b, int lh, int which, int block) : tile(nullptr), pos(nullptr) {
        const bool ret = which < 2;
        const int width = ret ? p.ret_width : p.apx_width;
        rows = rows_of(ret ? p.ret_len : p.apx_len, b, width);
        if (block >= width) return;
        const uint32_t page = (uint32_t)(ret ? p.ret_table : p.apx_table)[(size_t)b * width + block];
        if (page >= (ret ? p.n_ret_pages : p.n_apx_pages)) return;
        const size_t at = (size_t)page * p.LH + lh;
        tile = ret ? p.ret + (2 * at + which) * Row<D>::TILE : p.apx + at * Row<D>::TILE;
        int32_t* all = which == 0 ? p.ret_pos : which == 2 ? p.apx_pos : nullptr;
        if (all) pos = all + at * ROWS;
    }
};

// The largest magnitude of a thread's stored numbers, as the bits of an fp32 number; NaN does not count.  Magnitudes order like their bits, NaN above all: where one
// comes out, the slow way is taken.
template <int N> __device__ __forceinline__ uint32_t largest_of(const uint4 (&v)[N], __nv_bfloat16) {
    uint32_t most = 0;
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const uint32_t w[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("max.u16x2 %0, %0, %1;\n" : "+r"(most) : "r"(w[i] & 0x7fff7fffu));
    }
    most = max(most & 0xffff0000u, most << 16);
    if (most > 0x7f800000u) {
        most = 0;
#pragma unroll
        for (int p = 0; p < N; ++p) {
            const uint32_t w[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t size = (i & 1 ? w[i / 2] : w[i / 2] << 16) & 0x7fff0000u;
                most = max(most, size > 0x7f800000u ? 0u : size);
            }
        }
    }
    return most;
}
template <int N> __device__ __forceinline__ uint32_t largest_of(const uint4 (&v)[N], float) {
    uint32_t most = 0;
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const uint32_t w[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t size = w[i] & 0x7fffffffu;
            most = max(most, size > 0x7f800000u ? 0u : size);
        }
    }
    return most;
}
template <int N, int E> __device__ __forceinline__ uint32_t largest_of(const float (&x)[N][E]) {
    uint32_t most = 0;
#pragma unroll
    for (int p = 0; p < N; ++p)
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const uint32_t size = __float_as_uint(x[p][i]) & 0x7fffffffu;
            most = max(most, size > 0x7f800000u ? 0u : size);
        }
    return most;
}
// The largest of all threads' numbers, of N heads.
template <int N> __device__ __forceinline__ void largest(uint32_t (&most)[N], uint32_t (&shared)[N][THREADS / 32]) {
#pragma unroll
    for (int h = 0; h < N; ++h) {
        most[h] = __reduce_max_sync(0xffffffffu, most[h]);
        if (threadIdx.x % 32 == 0) shared[h][threadIdx.x / 32] = most[h];
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < N; ++h)
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) most[h] = max(most[h], shared[h][w]);
}

// Blocks of a unit: [0, br) retained keys, [br, 2 br) values, then key-only rows.  grid: (blocks, LH, batch).  The rows are on their way as soon as their
// indices are there, beside the table and the length.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS)
compact_kernel(const T* K, const T* V, int64_t N, const int32_t* ret_idx, const int32_t* apx_idx, int n_ret, int n_apx, Pools pools) {
    using L = Deal<T, D>;
    __shared__ uint32_t shared[1][THREADS / 32];
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    const int lh = blockIdx.y, b = blockIdx.z, u = b * pools.LH + lh;
    const int br = (n_ret + ROWS - 1) / ROWS, which = (int)blockIdx.x < br ? 0 : (int)blockIdx.x < 2 * br ? 1 : 2;
    const int block = blockIdx.x - which * br, n = which < 2 ? n_ret : n_apx, given = min(n - block * ROWS, ROWS);
    const int32_t* idx = (which < 2 ? ret_idx : apx_idx) + (size_t)u * n + block * ROWS;
    const int lane = threadIdx.x % L::LANES, row0 = threadIdx.x / L::LANES;
    const T* src = (which == 1 ? V : K) + (size_t)u * N * D + lane * L::E;
    int tok[L::PASSES];
    uint4 v[L::PASSES];
#pragma unroll
    for (int p = 0; p < L::PASSES; ++p) tok[p] = row0 + p * L::PER < given ? idx[row0 + p * L::PER] : -1;
    const Place<D> place(pools, b, lh, which, block);
#pragma unroll
    for (int p = 0; p < L::PASSES; ++p) {
        v[p] = make_uint4(0, 0, 0, 0);
        if ((unsigned long long)(long long)tok[p] < (unsigned long long)N) v[p] = *reinterpret_cast<const uint4*>(src + (size_t)tok[p] * D);
    }
    if (!place.tile) return;
    const int rows = min(place.rows - block * ROWS, given);               // rows behind the sequence's last are left as they were
    if (rows <= 0) return;
    if (rows < given) {
#pragma unroll
        for (int p = 0; p < L::PASSES; ++p)
            if (row0 + p * L::PER >= rows) v[p] = make_uint4(0, 0, 0, 0);
    }
    uint32_t most[1] = {largest_of(v, T())};
    largest(most, shared);
    const int e = exponent(most[0]);
    const float inv = power(-e);
#pragma unroll
    for (int p = 0; p < L::PASSES; ++p) {
        const int r = row0 + p * L::PER;
        if (r >= rows) continue;
        float x[L::E];
        widen(v[p], x);
        put_codes(place.tile + r * D + Row<D>::byte_of(r, lane * L::E), x, inv);
        if (lane == 0 && place.pos) place.pos[r] = tok[p];
    }
    if (threadIdx.x == 0) place.tile[Row<D>::SCALE_AT] = (unsigned char)(e - LOW);
}

// Rows [first_row[b], ret_len[b]) of a sequence, n_new at the most, into the blocks that they touch, HEADS neighbouring heads a thread block, whose angles are
// computed once.  grid: (touched blocks x 2, LH / HEADS, batch).
template <typename T, int D, bool ROTATE, int HEADS>
__global__ void __launch_bounds__(THREADS)
append_kernel(const T* k_new, int64_t k_stride, const T* v_new, int64_t v_stride, int n_new, const int32_t* first_row, const int32_t* pos, Pools pools, RopePhases phases) {
    using L = Deal<T, D>;
    __shared__ uint32_t shared[HEADS][THREADS / 32];
    __shared__ RopePhase phase[ROTATE ? D / 2 : 1];                       // a thread's index into a kernel's parameters would be served a lane at a time
    if constexpr (ROTATE) {
        if (threadIdx.x < D / 2) phase[threadIdx.x] = rope_phase_words(phases.phase[threadIdx.x]);
        __syncthreads();
    }
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    const int lh = blockIdx.y * HEADS, b = blockIdx.z, is_v = blockIdx.x & 1;
    const int first = max(first_row[b], 0), block = first / ROWS + (int)(blockIdx.x >> 1);
    const Place<D> place(pools, b, lh, is_v, block);
    if (!place.tile) return;
    // of this block: rows [lo, hi) are new
    const int lo = max(first - block * ROWS, 0), hi = min((int)min((int64_t)place.rows, (int64_t)first + n_new) - block * ROWS, ROWS);
    if (lo >= hi) return;
    const int64_t from = (int64_t)b * n_new + block * ROWS - first;       // the source's row of the block's row 0
    const T* src = is_v ? v_new + from * v_stride : k_new + from * k_stride;
    const int64_t stride = is_v ? v_stride : k_stride;
    const int lane = threadIdx.x % L::LANES, row0 = threadIdx.x / L::LANES;
    constexpr int APART = 2 * Row<D>::TILE;                               // from a head's tile to the next one's
    int had[HEADS];
    uint4 v[HEADS][L::PASSES];
    int32_t at[L::PASSES];
#pragma unroll
    for (int p = 0; p < L::PASSES; ++p) {
        const int r = row0 + p * L::PER;
        const bool there = r >= lo && r < hi;
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            v[h][p] = make_uint4(0, 0, 0, 0);
            if (there) v[h][p] = *reinterpret_cast<const uint4*>(src + r * stride + (lh + h) * D + lane * L::E);
        }
        at[p] = pos && there && !is_v ? pos[from + r] : 0;
    }
#pragma unroll
    for (int h = 0; h < HEADS; ++h) had[h] = lo > 0 ? exponent_of(place.tile + h * APART, Row<D>::SCALE_AT) : LOW;
    float x[HEADS][L::PASSES][L::E];
#pragma unroll
    for (int p = 0; p < L::PASSES; ++p) {
        const int r = row0 + p * L::PER;
        const bool there = r >= lo && r < hi;
#pragma unroll
        for (int h = 0; h < HEADS; ++h) {
            widen(v[h][p], x[h][p]);
            if (there && lane == 0 && place.pos) place.pos[h * ROWS + r] = at[p];
        }
        if constexpr (ROTATE)
            if (!is_v && __any_sync(0xffffffffu, there)) {                // the partner of a channel is half a row away
                const bool upper = lane >= L::LANES / 2;
                // two lanes half a row apart have the same angles: each computes half of them
                const int c = lane % (L::LANES / 2) * L::E + (upper ? L::E / 2 : 0);
                uint64_t cs[L::E / 2], sn[L::E / 2];
#pragma unroll
                for (int i = 0; i < L::E / 4; ++i) {
                    uint64_t mine_c, mine_s;
                    rope_cos_sin2_fine(rope_angle(at[p], phase[c + 2 * i]), rope_angle(at[p], phase[c + 2 * i + 1]), mine_c, mine_s);
                    const uint64_t other_c = __shfl_xor_sync(0xffffffffu, mine_c, L::LANES / 2), other_s = __shfl_xor_sync(0xffffffffu, mine_s, L::LANES / 2);
                    const uint64_t sign = upper ? 0ull : 0x8000000080000000ull;
                    cs[i] = upper ? other_c : mine_c;
                    cs[i + L::E / 4] = upper ? mine_c : other_c;
                    sn[i] = (upper ? other_s : mine_s) ^ sign;
                    sn[i + L::E / 4] = (upper ? mine_s : other_s) ^ sign;
                }
#pragma unroll
                for (int h = 0; h < HEADS; ++h) {
                    float y[L::E];
                    widen(make_uint4(__shfl_xor_sync(0xffffffffu, v[h][p].x, L::LANES / 2), __shfl_xor_sync(0xffffffffu, v[h][p].y, L::LANES / 2),
                                     __shfl_xor_sync(0xffffffffu, v[h][p].z, L::LANES / 2), __shfl_xor_sync(0xffffffffu, v[h][p].w, L::LANES / 2)), y);
#pragma unroll
                    for (int i = 0; i < L::E / 2; ++i)
                        tc::unpack2(tc::fma2(tc::pack2(x[h][p][2 * i], x[h][p][2 * i + 1]), cs[i], tc::mul2(tc::pack2(y[2 * i], y[2 * i + 1]), sn[i])), x[h][p][2 * i], x[h][p][2 * i + 1]);
                }
            }
    }
    uint32_t most[HEADS];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) most[h] = largest_of(x[h]);
    largest(most, shared);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        unsigned char* tile = place.tile + h * APART;
        const int e = max(exponent(most[h]), had[h]);
        if (e > had[h] && lo > 0) {                                       // rows that were there, under the larger scale
            const float down = power(had[h] - e);
            for (int i = threadIdx.x; i < lo * D / 4; i += THREADS) {
                uint32_t* w = reinterpret_cast<uint32_t*>(tile) + i;
                float y[4];
                decode_word(*w, y);
                *w = to_codes(y[0] * down, y[1] * down, y[2] * down, y[3] * down);
            }
        }
        const float inv = power(-e);
#pragma unroll
        for (int p = 0; p < L::PASSES; ++p) {
            const int r = row0 + p * L::PER;
            if (r >= lo && r < hi) put_codes(tile + r * D + Row<D>::byte_of(r, lane * L::E), x[h][p], inv);
        }
        if (threadIdx.x == 0 && (e > had[h] || lo == 0)) tile[Row<D>::SCALE_AT] = (unsigned char)(e - LOW);      // its old value has been read by all threads: a barrier lies between
    }
}

__device__ __forceinline__ void put_run(__nv_bfloat16* to, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void put_run(float* to, const float (&x)[8]) {
    reinterpret_cast<float4*>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(to)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// The first rows of every sequence as the values that they stand for, [U][n][D]; rows that a sequence does not have are zeros.  grid: as compact_kernel's.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS)
read_kernel(int n_ret, int n_apx, Pools pools, T* __restrict__ ret_k, T* __restrict__ ret_v, T* __restrict__ apx_k) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    constexpr int RUNS = D / 8;                                           // of eight channels: a thread's part of a row
    const int lh = blockIdx.y, b = blockIdx.z, u = b * pools.LH + lh;
    const int br = (n_ret + ROWS - 1) / ROWS, which = (int)blockIdx.x < br ? 0 : (int)blockIdx.x < 2 * br ? 1 : 2;
    const int block = blockIdx.x - which * br, n = which < 2 ? n_ret : n_apx;
    const Place<D> place(pools, b, lh, which, block);
    const int wanted = min(n - block * ROWS, ROWS), rows = place.tile ? min(place.rows - block * ROWS, wanted) : 0;
    const float s = rows > 0 ? power(exponent_of(place.tile, Row<D>::SCALE_AT)) : 0.f;
    T* out = (which == 0 ? ret_k : which == 1 ? ret_v : apx_k) + ((size_t)u * n + block * ROWS) * D;
    constexpr int N = ROWS * RUNS / THREADS;                              // all of a thread's loads are on their way before the first store
    uint2 w[N];
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const int r = (p * THREADS + threadIdx.x) / RUNS, run = threadIdx.x % RUNS;
        w[p] = make_uint2(0, 0);
        if (r < rows) w[p] = *reinterpret_cast<const uint2*>(place.tile + r * D + Row<D>::byte_of(r, 8 * run));
    }
#pragma unroll
    for (int p = 0; p < N; ++p) {
        const int r = (p * THREADS + threadIdx.x) / RUNS, run = threadIdx.x % RUNS;
        if (r >= wanted) continue;
        float x[8], y[4];
        decode_word(w[p].x, y);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = y[j] * s;
        decode_word(w[p].y, y);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 + j] = y[j] * s;
        put_run(out + (size_t)r * D + 8 * run, x);
    }
}

static Pools pools_of(const Dims& dm, const vector_q8_cache* c) {
    return {(unsigned char*)c->ret_pages, (unsigned char*)c->apx_pages, c->ret_pos, c->apx_pos, c->ret_table, c->apx_table, c->ret_len, c->apx_len,
            (uint32_t)c->n_ret_pages, (uint32_t)c->n_apx_pages, c->ret_width, c->apx_width, dm.LH};
}
static int blocks_of(int64_t rows) { return (int)((rows + ROWS - 1) / ROWS); }

struct CompactCall {
    const Dims& dm; const vector_budget* b; const void *K, *V; const int32_t *ret_idx, *apx_idx; Pools pools; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        const dim3 grid(2 * blocks_of(b->n_ret) + blocks_of(b->n_apx), dm.LH, dm.U / dm.LH);
        VEC_CUDA_CHECK(launch_maybe_dependent(true, compact_kernel<T, D>, grid, dim3(THREADS), 0, st, (const T*)K, (const T*)V, b->n_tokens, ret_idx, apx_idx,
                                              (int)b->n_ret, (int)b->n_apx, pools));
        return VECTOR_OK;
    }
};
struct AppendCall {
    const Dims& dm; const void* k; int64_t k_stride; const void* v; int64_t v_stride; int64_t n_new; const int32_t *first_row, *pos; bool rotate; Pools pools; cudaStream_t st;
    template <typename T, int D, bool ROTATE, int HEADS> vector_status put() const {
        RopePhases ph = {};
        if (ROTATE) rope_phases(dm.theta, D, &ph);
        // the most blocks that n_new rows touch: all but one of them from a block's last row on
        const dim3 grid(2 * (1 + blocks_of(n_new - 1)), dm.LH / HEADS, dm.U / dm.LH);
        VEC_CUDA_CHECK(launch_maybe_dependent(true, append_kernel<T, D, ROTATE, HEADS>, grid, dim3(THREADS), 0, st, (const T*)k, k_stride, (const T*)v, v_stride, (int)n_new, first_row, pos,
                                              pools, ph));
        return VECTOR_OK;
    }
    // us by one head a thread block and by two, turned, in 8 heads: 2048 rows of four sequences (7.7 at the copy rate; not turned 11.3 and 11.9), 64 rows of 32,
    // 300 of one, 5 rows and one row of 32:
    //   bf16, 128 channels  19.7 17.3, 8.1 7.0, 4.0 3.9, 3.9 3.8, 3.3 3.4     64 channels  11.8 9.1, 5.4 5.4, 3.3 3.2, 3.3 3.2, 3.3 3.2
    //   fp32, 128 channels  23.2 21.0, 9.2 8.4, 4.6 5.1, 4.5 4.8, 4.1 4.0     64 channels  13.5 11.2, 5.7 6.1, 3.3 3.2, 3.3 3.2, 3.3 3.2
    // fp32 not turned 16.0 and 34.6.
    template <typename T, int D> vector_status run() const {
        if (!rotate) return put<T, D, false, 1>();
        return dm.LH % 2 == 0 ? put<T, D, true, 2>() : put<T, D, true, 1>();
    }
};
struct ReadCall {
    const Dims& dm; int64_t n_ret, n_apx; void *ret_k, *ret_v, *apx_k; Pools pools; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        const dim3 grid(2 * blocks_of(n_ret) + blocks_of(n_apx), dm.LH, dm.U / dm.LH);
        VEC_CUDA_CHECK(launch_maybe_dependent(true, read_kernel<T, D>, grid, dim3(THREADS), 0, st, (int)n_ret, (int)n_apx, pools, (T*)ret_k, (T*)ret_v, (T*)apx_k));
        return VECTOR_OK;
    }
};
// The call's kernel for the shape's element type and head size.
template <typename Call> static vector_status by_type(const Dims& dm, const Call& call) {
    using B = __nv_bfloat16;
    if (dm.dtype == VECTOR_F32) return dm.d == 64 ? call.template run<float, 64>() : call.template run<float, 128>();
    return dm.d == 64 ? call.template run<B, 64>() : call.template run<B, 128>();
}
// What a call needs of a tier that it has rows of.
static vector_status check_tier(const void* pages, const int32_t* table, const int32_t* len, int32_t width) { return pages && (width == 0 || (table && len)) ? VECTOR_OK : VECTOR_ERR_NULL; }

}  // namespace q8

vector_status check_q8_cache(const vector_q8_cache* c) {
    if (!c) return VECTOR_ERR_NULL;
    if (c->n_ret_pages < 0 || c->n_apx_pages < 0 || c->n_ret_pages >= q8::MAX_PAGES || c->n_apx_pages >= q8::MAX_PAGES) return VECTOR_ERR_SHAPE;
    constexpr int32_t most_width = (1 << 30) / VECTOR_Q8_PAGE_ROWS;
    if (c->ret_width < 0 || c->apx_width < 0 || c->ret_width > most_width || c->apx_width > most_width) return VECTOR_ERR_SHAPE;
    if ((c->n_ret_pages > 0 && !c->ret_pages) || (c->n_apx_pages > 0 && !c->apx_pages)) return VECTOR_ERR_NULL;
    if (((uintptr_t)c->ret_pages | (uintptr_t)c->apx_pages | (uintptr_t)c->apx_pos) & 15) return VECTOR_ERR_SHAPE;
    return VECTOR_OK;
}

}  // namespace vec

using namespace vec;

extern "C" size_t vector_q8_tile_bytes(const vector_shape* shape) {
    Dims dm;
    if (check_shape(shape, &dm) != VECTOR_OK) return 0;
    return dm.d == 64 ? q8::Row<64>::TILE : q8::Row<128>::TILE;
}

extern "C" vector_status vector_compact_q8(const vector_shape* shape, const vector_budget* budget, const void* K, const void* V, const int32_t* ret_idx,
                                           const int32_t* apx_idx, const vector_q8_cache* cache, void* stream) {
    Dims dm;
    vector_status rc = check_shape(shape, &dm);
    if (rc != VECTOR_OK) return rc;
    if ((rc = check_budget(budget, dm.w)) != VECTOR_OK) return rc;
    if ((rc = check_q8_cache(cache)) != VECTOR_OK) return rc;
    if (!K || !V) return VECTOR_ERR_NULL;
    if (budget->n_ret > 0 && (!ret_idx || (rc = q8::check_tier(cache->ret_pages, cache->ret_table, cache->ret_len, cache->ret_width)) != VECTOR_OK)) return VECTOR_ERR_NULL;
    if (budget->n_apx > 0 && (!apx_idx || (rc = q8::check_tier(cache->apx_pages, cache->apx_table, cache->apx_len, cache->apx_width)) != VECTOR_OK)) return VECTOR_ERR_NULL;
    if (((uintptr_t)K | (uintptr_t)V) & 15) return VECTOR_ERR_SHAPE;
    if (2 * budget->n_ret + budget->n_apx == 0) return VECTOR_OK;
    if (2 * budget->n_ret + budget->n_apx > (int64_t(1) << 30)) return VECTOR_ERR_SHAPE;
    return q8::by_type(dm, q8::CompactCall{dm, budget, K, V, ret_idx, apx_idx, q8::pools_of(dm, cache), (cudaStream_t)stream});
}

extern "C" vector_status vector_append_q8(const vector_shape* shape, const vector_q8_cache* cache, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                                          int64_t n_new, const int32_t* first_row, const int32_t* pos, int32_t rotate, void* stream) {
    Dims dm;
    vector_status rc = check_shape(shape, &dm);
    if (rc != VECTOR_OK) return rc;
    if ((rc = check_q8_cache(cache)) != VECTOR_OK) return rc;
    if (n_new < 0 || n_new > (int64_t(1) << 30)) return VECTOR_ERR_SHAPE;
    const int64_t row = (int64_t)dm.LH * dm.d, most = int64_t(1) << 40;
    if (k_stride < row || v_stride < row || k_stride > most || v_stride > most) return VECTOR_ERR_SHAPE;
    if (rotate && !dm.rope) return VECTOR_ERR_SHAPE;                      // no base to turn by
    if (n_new == 0) return VECTOR_OK;
    if (!k_new || !v_new || !first_row || ((cache->ret_pos || rotate) && !pos)) return VECTOR_ERR_NULL;
    if ((rc = q8::check_tier(cache->ret_pages, cache->ret_table, cache->ret_len, cache->ret_width)) != VECTOR_OK) return rc;
    if (((uintptr_t)k_new | (uintptr_t)v_new | (uintptr_t)(k_stride * dm.esize) | (uintptr_t)(v_stride * dm.esize)) & 15) return VECTOR_ERR_SHAPE;
    return q8::by_type(dm, q8::AppendCall{dm, k_new, k_stride, v_new, v_stride, n_new, first_row, pos, rotate != 0, q8::pools_of(dm, cache), (cudaStream_t)stream});
}

extern "C" vector_status vector_read_q8(const vector_shape* shape, const vector_q8_cache* cache, int64_t n_ret, void* ret_k, void* ret_v, int64_t n_apx, void* apx_k,
                                        void* stream) {
    Dims dm;
    vector_status rc = check_shape(shape, &dm);
    if (rc != VECTOR_OK) return rc;
    if ((rc = check_q8_cache(cache)) != VECTOR_OK) return rc;
    if (n_ret < 0 || n_apx < 0 || n_ret > (int64_t(1) << 30) || n_apx > (int64_t(1) << 30) || 2 * n_ret + n_apx > (int64_t(1) << 30)) return VECTOR_ERR_SHAPE;
    if (n_ret > 0 && (!ret_k || !ret_v || (cache->ret_width > 0 && (!cache->ret_table || !cache->ret_len)))) return VECTOR_ERR_NULL;
    if (n_apx > 0 && (!apx_k || (cache->apx_width > 0 && (!cache->apx_table || !cache->apx_len)))) return VECTOR_ERR_NULL;
    if (((uintptr_t)ret_k | (uintptr_t)ret_v | (uintptr_t)apx_k) & 15) return VECTOR_ERR_SHAPE;
    if (n_ret + n_apx == 0) return VECTOR_OK;
    return q8::by_type(dm, q8::ReadCall{dm, n_ret, n_apx, ret_k, ret_v, apx_k, q8::pools_of(dm, cache), (cudaStream_t)stream});
}
