// What writes and reads the 4-bit paged cache (q4.cuh): compaction of a routed context into its pages, a generated token's rows, and
// rows read back.  A writing thread has two groups of 16 channels of a row, half a head apart: their largest magnitudes, scales and codes need no
// other thread, and the codes are 16 neighbouring bytes of the stored row, the scales two.
#include "common.cuh"
#include "internal.h"
#include "q4.cuh"

namespace vec {
namespace q4 {

constexpr int THREADS = 128;
// Rows that a thread has in flight, of compaction and of reading back.  us for 256 units of 13100 rows, 128 channels of bf16: compaction by one row 194, two 201,
// four 245 (bound by what its threads execute: 0.75 of the issue slots; a thread a group of 16 channels instead of two 262); reading back 227, 220, 232 (a copy of
// its bytes: 168).  fp32, 64 channels: compaction 22, 27, 30; reading back 23.4, 24.5, 26.5.
constexpr int COMPACT_PASSES = 1;
template <typename T> constexpr int READ_PASSES = sizeof(T) == 4 ? 1 : 2;

// 16 channels at p, which is a multiple of 16 bytes.
__device__ __forceinline__ void load_group(const __nv_bfloat16* p, uint4 (&v)[2]) {
    v[0] = reinterpret_cast<const uint4*>(p)[0];
    v[1] = reinterpret_cast<const uint4*>(p)[1];
}
__device__ __forceinline__ void load_group(const float* p, uint4 (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
}
template <typename T> struct Raw { static constexpr int N = sizeof(T) == 2 ? 2 : 4; };

// Pairs of groups of a row; the codes of pair p's groups p and p + PAIRS are its bytes 16 p .. + 15 (64 channels: in four-byte turns), its scales bytes 2 p and 2 p + 1.
template <int D> struct Pair { static constexpr int N = Row<D>::GROUPS / 2, APART = D / 2; };
template <int D>
__device__ __forceinline__ void put_pair(unsigned char* tile, int row, int pair, uint2 low, uint2 high, uint32_t low_scale, uint32_t high_scale) {
    static_assert(Row<D>::byte_of(16) == 16 && Row<D>::scale_of(1) == 2 && Row<D>::scale_of(Pair<D>::N) == 1, "where a pair lies");
    *reinterpret_cast<uint4*>(tile + row * Row<D>::CODES + 16 * pair) = D == 128 ? make_uint4(low.x, low.y, high.x, high.y) : make_uint4(low.x, high.x, low.y, high.y);
    *reinterpret_cast<uint16_t*>(tile + Row<D>::SCALES_AT + row * Row<D>::GROUPS + 2 * pair) = (uint16_t)(low_scale | high_scale << 8);
}

struct Pools {
    unsigned char *ret, *apx;
    int32_t *ret_pos, *apx_pos;
    uint32_t ret_slots, apx_slots;       // rows of a pool: a slot at or beyond it is none
    int LH;
};
// Tile of a page for (layer, KV head) lh; which: 0 = keys, 1 = values of a retained page.
template <int D> __device__ __forceinline__ unsigned char* ret_tile(const Pools& p, uint32_t page, int lh, int which) {
    return p.ret + (((size_t)page * p.LH + lh) * 2 + which) * Row<D>::TILE;
}
template <int D> __device__ __forceinline__ unsigned char* apx_tile(const Pools& p, uint32_t page, int lh) {
    return p.apx + ((size_t)page * p.LH + lh) * Row<D>::TILE;
}

// Logical row r of a unit: [0, n_ret) K -> retained keys, [n_ret, 2 n_ret) V -> retained values, then K -> key-only rows.  Rows are
// dealt to PASSES x THREADS / Pair::N a block, so that a thread has PASSES rows' loads in flight.  grid: (chunks, LH, batch).
template <typename T, int D, int PASSES>
__global__ void __launch_bounds__(THREADS)
compact_kernel(const T* K, const T* V, int64_t N, const int32_t* ret_idx, const int32_t* apx_idx, int n_ret, int n_apx,
               const int32_t* ret_slots, const int32_t* apx_slots, Pools pools) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    constexpr int P = Pair<D>::N, PER = THREADS / P;
    const int lh = blockIdx.y, b = blockIdx.z, u = b * pools.LH + lh;
    const int pair = threadIdx.x % P, r0 = blockIdx.x * PASSES * PER + threadIdx.x / P, rows = 2 * n_ret + n_apx;
    const size_t unit = (size_t)u * N;
    const T* src[PASSES];
    int slot[PASSES], tok[PASSES], what[PASSES];                      // what: 0 retained key, 1 value, 2 key-only
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = r0 + p * PER;
        src[p] = nullptr; slot[p] = 0; tok[p] = 0;
        what[p] = r < n_ret ? 0 : r < 2 * n_ret ? 1 : 2;
        if (r >= rows) continue;
        const int i = r - what[p] * n_ret;
        const bool ret = what[p] < 2;
        tok[p] = ret ? ret_idx[(size_t)u * n_ret + i] : apx_idx[(size_t)u * n_apx + i];
        slot[p] = ret ? ret_slots[(size_t)b * n_ret + i] : apx_slots[(size_t)b * n_apx + i];
        // a token outside the context or a slot outside the pool: the row is skipped
        if ((unsigned long long)(long long)tok[p] < (unsigned long long)N && (uint32_t)slot[p] < (ret ? pools.ret_slots : pools.apx_slots))
            src[p] = (what[p] == 1 ? V : K) + (unit + tok[p]) * D + 16 * pair;
    }
    uint4 v[PASSES][2][Raw<T>::N];
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
        if (src[p]) { load_group(src[p], v[p][0]); load_group(src[p] + Pair<D>::APART, v[p][1]); }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        if (!src[p]) continue;
        uint32_t scale[2];
        const uint2 low = encode_group(v[p][0], scale[0]), high = encode_group(v[p][1], scale[1]);
        const uint32_t page = (uint32_t)slot[p] / ROWS;
        const int row = slot[p] % ROWS;
        put_pair<D>(what[p] < 2 ? ret_tile<D>(pools, page, lh, what[p]) : apx_tile<D>(pools, page, lh), row, pair, low, high, scale[0], scale[1]);
        int32_t* pos = what[p] == 0 ? pools.ret_pos : what[p] == 2 ? pools.apx_pos : nullptr;
        if (pair == 0 && pos) pos[((size_t)page * pools.LH + lh) * ROWS + row] = tok[p];
    }
}

// One generated token's rows: of sequence b to slots[row_start[b]] (where it has a new row), or to slots[b].
template <typename T, int D>
__global__ void __launch_bounds__(THREADS)
append_kernel(const T* k_new, const T* v_new, const int32_t* row_start, const int32_t* slots, int64_t n_slots, const int32_t* pos, Pools pools,
              int U) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    constexpr int P = Pair<D>::N;
    const long long i = (long long)blockIdx.x * THREADS + threadIdx.x;     // (unit, key or value, pair of groups)
    const int pair = (int)(i % P), is_v = (int)(i / P) & 1, u = (int)(i / (2 * P));
    if (u >= U) return;
    const int b = u / pools.LH, lh = u - b * pools.LH;
    int64_t at = b;
    if (row_start) {
        at = row_start[b];
        if (row_start[b + 1] <= at) return;
    }
    if (at < 0 || at >= n_slots) return;
    const uint32_t slot = (uint32_t)slots[at];
    if (slot >= pools.ret_slots) return;
    const T* src = (is_v ? v_new : k_new) + (size_t)u * D + 16 * pair;
    uint4 v[2][Raw<T>::N];
    load_group(src, v[0]);
    load_group(src + Pair<D>::APART, v[1]);
    uint32_t scale[2];
    const uint2 low = encode_group(v[0], scale[0]), high = encode_group(v[1], scale[1]);
    put_pair<D>(ret_tile<D>(pools, slot / ROWS, lh, is_v), slot % ROWS, pair, low, high, scale[0], scale[1]);
    if (pair == 0 && !is_v && pools.ret_pos) pools.ret_pos[((size_t)(slot / ROWS) * pools.LH + lh) * ROWS + slot % ROWS] = pos[b];
}

__device__ __forceinline__ void store_group(__nv_bfloat16* p, const float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(x[8 * i + 2 * j], x[8 * i + 2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t*>(&v);
        }
        reinterpret_cast<uint4*>(p)[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
__device__ __forceinline__ void store_group(float* p, const float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
}

// Rows of slots as the values they stand for, [U][n][D] each; a slot outside its pool gives zeros.  The rows of a unit as in compact_kernel, but a
// thread has one group: what it writes of a row is one sector then (128 channels of bf16, us for 256 units of 13100 rows: 220; two groups 228, eight channels 248).
template <typename T, int D, int PASSES>
__global__ void __launch_bounds__(THREADS)
read_kernel(const int32_t* ret_slots, const int32_t* apx_slots, int n_ret, int n_apx, Pools pools, T* __restrict__ ret_k, T* __restrict__ ret_v,
            T* __restrict__ apx_k) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    constexpr int G = Row<D>::GROUPS, PER = THREADS / G;
    const int lh = blockIdx.y, b = blockIdx.z, u = b * pools.LH + lh;
    const int group = threadIdx.x % G, r0 = blockIdx.x * PASSES * PER + threadIdx.x / G, rows = 2 * n_ret + n_apx;
    const int code_at = Row<D>::byte_of(16 * group), scale_at = Row<D>::SCALES_AT + Row<D>::scale_of(group);
    uint2 codes[PASSES];
    uint32_t scale[PASSES];
    T* dst[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = r0 + p * PER;
        dst[p] = nullptr; codes[p] = make_uint2(0, 0); scale[p] = 0;
        if (r >= rows) continue;
        const int what = r < n_ret ? 0 : r < 2 * n_ret ? 1 : 2, i = r - what * n_ret;
        const uint32_t slot = (uint32_t)(what < 2 ? ret_slots[(size_t)b * n_ret + i] : apx_slots[(size_t)b * n_apx + i]);
        dst[p] = (what == 0 ? ret_k : what == 1 ? ret_v : apx_k) + ((size_t)u * (what < 2 ? n_ret : n_apx) + i) * D + 16 * group;
        if (slot >= (what < 2 ? pools.ret_slots : pools.apx_slots)) continue;
        const unsigned char* tile = what < 2 ? ret_tile<D>(pools, slot / ROWS, lh, what) : apx_tile<D>(pools, slot / ROWS, lh);
        const unsigned char* at = tile + slot % ROWS * Row<D>::CODES + code_at;
        if constexpr (D == 128) codes[p] = *reinterpret_cast<const uint2*>(at);
        else codes[p] = make_uint2(*reinterpret_cast<const uint32_t*>(at), *reinterpret_cast<const uint32_t*>(at + 8));      // in the next piece
        scale[p] = tile[slot % ROWS * G + scale_at];
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        if (!dst[p]) continue;
        const float s = scale_value(scale[p]);
        float x[16];
        const uint32_t w[2] = {codes[p].x, codes[p].y};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t two[4];
            decode_word(w[h], two);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&two[i]));
                x[8 * h + 2 * i] = f.x * s; x[8 * h + 2 * i + 1] = f.y * s;
            }
        }
        store_group(dst[p], x);
    }
}

static Pools pools_of(const Dims& dm, const vector_q4_cache* c) {
    return {(unsigned char*)c->ret_pages, (unsigned char*)c->apx_pages, c->ret_pos, c->apx_pos, (uint32_t)(c->n_ret_pages * ROWS),
            (uint32_t)(c->n_apx_pages * ROWS), dm.LH};
}
// Blocks over `rows` rows of every unit, `per_block` to a block.
static dim3 row_blocks(const Dims& dm, int64_t rows, int per_block) {
    return dim3((unsigned)((rows + per_block - 1) / per_block), (unsigned)dm.LH, (unsigned)(dm.U / dm.LH));
}

struct CompactCall {
    const Dims& dm; const vector_budget* b; const void *K, *V; const int32_t *ret_idx, *apx_idx, *ret_slots, *apx_slots; Pools pools; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        constexpr int PASSES = COMPACT_PASSES;
        const dim3 blocks = row_blocks(dm, 2 * b->n_ret + b->n_apx, PASSES * (THREADS / Pair<D>::N));
        VEC_CUDA_CHECK(launch_maybe_dependent(true, compact_kernel<T, D, PASSES>, blocks, dim3(THREADS), 0, st, (const T*)K, (const T*)V, b->n_tokens,
                                              ret_idx, apx_idx, (int)b->n_ret, (int)b->n_apx, ret_slots, apx_slots, pools));
        return VECTOR_OK;
    }
};
struct AppendCall {
    const Dims& dm; const void *k, *v; const int32_t *row_start, *slots; int64_t n_slots; const int32_t* pos; Pools pools; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        const long long n = (long long)dm.U * 2 * Pair<D>::N;
        VEC_CUDA_CHECK(launch_maybe_dependent(true, append_kernel<T, D>, dim3((unsigned)((n + THREADS - 1) / THREADS)), dim3(THREADS), 0, st, (const T*)k,
                                              (const T*)v, row_start, slots, n_slots, pos, pools, dm.U));
        return VECTOR_OK;
    }
};
struct ReadCall {
    const Dims& dm; const int32_t *ret_slots, *apx_slots; int64_t n_ret, n_apx; void *ret_k, *ret_v, *apx_k; Pools pools; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        constexpr int PASSES = READ_PASSES<T>;
        const dim3 blocks = row_blocks(dm, 2 * n_ret + n_apx, PASSES * (THREADS / Row<D>::GROUPS));
        VEC_CUDA_CHECK(launch_maybe_dependent(true, read_kernel<T, D, PASSES>, blocks, dim3(THREADS), 0, st, ret_slots, apx_slots, (int)n_ret, (int)n_apx,
                                              pools, (T*)ret_k, (T*)ret_v, (T*)apx_k));
        return VECTOR_OK;
    }
};
// The call's kernel for the shape's element type and head size.
template <typename Call> static vector_status by_type(const Dims& dm, const Call& call) {
    using B = __nv_bfloat16;
    if (dm.dtype == VECTOR_F32) return dm.d == 64 ? call.template run<float, 64>() : call.template run<float, 128>();
    return dm.d == 64 ? call.template run<B, 64>() : call.template run<B, 128>();
}

}  // namespace q4

vector_status check_q4_cache(const vector_q4_cache* c) {
    if (!c) return VECTOR_ERR_NULL;
    if (c->n_ret_pages < 0 || c->n_apx_pages < 0 || c->n_ret_pages >= q4::MAX_PAGES || c->n_apx_pages >= q4::MAX_PAGES) return VECTOR_ERR_SHAPE;
    if ((c->n_ret_pages > 0 && !c->ret_pages) || (c->n_apx_pages > 0 && !c->apx_pages)) return VECTOR_ERR_NULL;
    if (((uintptr_t)c->ret_pages | (uintptr_t)c->apx_pages) & 15) return VECTOR_ERR_SHAPE;
    return VECTOR_OK;
}

}  // namespace vec

using namespace vec;

extern "C" size_t vector_q4_tile_bytes(const vector_shape* shape) {
    Dims dm;
    if (check_shape(shape, &dm) != VECTOR_OK) return 0;
    return dm.d == 64 ? q4::Row<64>::TILE : q4::Row<128>::TILE;
}

extern "C" vector_status vector_compact_q4(const vector_shape* shape, const vector_budget* budget, const void* K, const void* V,
                                           const int32_t* ret_idx, const int32_t* apx_idx, const vector_q4_cache* cache,
                                           const int32_t* ret_slots, const int32_t* apx_slots, void* stream) {
    Dims dm;
    vector_status rc = check_shape(shape, &dm);
    if (rc != VECTOR_OK) return rc;
    if ((rc = check_budget(budget, dm.w)) != VECTOR_OK) return rc;
    if ((rc = check_q4_cache(cache)) != VECTOR_OK) return rc;
    if (!K || !V) return VECTOR_ERR_NULL;
    if (budget->n_ret > 0 && (!ret_idx || !ret_slots || !cache->ret_pages)) return VECTOR_ERR_NULL;
    if (budget->n_apx > 0 && (!apx_idx || !apx_slots || !cache->apx_pages)) return VECTOR_ERR_NULL;
    if (((uintptr_t)K | (uintptr_t)V) & 15) return VECTOR_ERR_SHAPE;
    if (2 * budget->n_ret + budget->n_apx == 0) return VECTOR_OK;
    if (2 * budget->n_ret + budget->n_apx > (int64_t(1) << 30)) return VECTOR_ERR_SHAPE;
    return q4::by_type(dm, q4::CompactCall{dm, budget, K, V, ret_idx, apx_idx, ret_slots, apx_slots, q4::pools_of(dm, cache), (cudaStream_t)stream});
}

extern "C" vector_status vector_append_q4(const vector_shape* shape, const vector_q4_cache* cache, const void* k_new, const void* v_new,
                                          const int32_t* row_start, const int32_t* slots, int64_t n_slots, const int32_t* pos, void* stream) {
    Dims dm;
    vector_status rc = check_shape(shape, &dm);
    if (rc != VECTOR_OK) return rc;
    if ((rc = check_q4_cache(cache)) != VECTOR_OK) return rc;
    if (!k_new || !v_new || !slots || !cache->ret_pages || (cache->ret_pos && !pos)) return VECTOR_ERR_NULL;
    if (n_slots < 0 || (!row_start && n_slots < shape->batch)) return VECTOR_ERR_SHAPE;
    if (((uintptr_t)k_new | (uintptr_t)v_new) & 15) return VECTOR_ERR_SHAPE;
    return q4::by_type(dm, q4::AppendCall{dm, k_new, v_new, row_start, slots, n_slots, pos, q4::pools_of(dm, cache), (cudaStream_t)stream});
}

extern "C" vector_status vector_read_q4(const vector_shape* shape, const vector_q4_cache* cache, const int32_t* ret_slots, int64_t n_ret,
                                        void* ret_k, void* ret_v, const int32_t* apx_slots, int64_t n_apx, void* apx_k, void* stream) {
    Dims dm;
    vector_status rc = check_shape(shape, &dm);
    if (rc != VECTOR_OK) return rc;
    if ((rc = check_q4_cache(cache)) != VECTOR_OK) return rc;
    if (n_ret < 0 || n_apx < 0 || n_ret > (int64_t(1) << 30) || n_apx > (int64_t(1) << 30) || 2 * n_ret + n_apx > (int64_t(1) << 30)) return VECTOR_ERR_SHAPE;
    if (n_ret > 0 && (!ret_slots || !ret_k || !ret_v || !cache->ret_pages)) return VECTOR_ERR_NULL;
    if (n_apx > 0 && (!apx_slots || !apx_k || !cache->apx_pages)) return VECTOR_ERR_NULL;
    if (((uintptr_t)ret_k | (uintptr_t)ret_v | (uintptr_t)apx_k) & 15) return VECTOR_ERR_SHAPE;
    if (n_ret + n_apx == 0) return VECTOR_OK;
    return q4::by_type(dm, q4::ReadCall{dm, ret_slots, apx_slots, n_ret, n_apx, ret_k, ret_v, apx_k, q4::pools_of(dm, cache), (cudaStream_t)stream});
}
