// What writes and reads the 4-bit paged cache (q4.cuh): compaction of a routed context into its pages, a generated token's rows, and
// rows read back.  A thread has one group of 16 channels of a row: its largest magnitude, scale and codes need no other thread.
#include "common.cuh"
#include "internal.h"
#include "q4.cuh"

namespace vec {
namespace q4 {

constexpr int THREADS = 128;
// Rows that a thread has in flight.  bf16, 256 units of 13100 rows: compaction by one row a thread 268 us, two 258, four 275, reading back 220, 208, 222.  fp32
// rows are twice as long: 25 and 22 us by one, 28 and 25 by two.
template <typename T> constexpr int PASSES_OF = sizeof(T) == 4 ? 1 : 2;

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

// A group's codes and scale into row `row` of a tile.
template <int D>
__device__ __forceinline__ void put_group(unsigned char* tile, int row, int group, uint2 codes, uint32_t scale) {
    unsigned char* r = tile + row * Row<D>::CODES;
    if constexpr (D == 128) {
        *reinterpret_cast<uint2*>(r + Row<D>::byte_of(16 * group)) = codes;
    } else {                                                          // half a group to each of two pieces
        *reinterpret_cast<uint32_t*>(r + Row<D>::byte_of(16 * group)) = codes.x;
        *reinterpret_cast<uint32_t*>(r + Row<D>::byte_of(16 * group + 8)) = codes.y;
    }
    tile[Row<D>::SCALES_AT + row * Row<D>::GROUPS + Row<D>::scale_of(group)] = (unsigned char)scale;
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
// dealt to PASSES x THREADS / GROUPS a block, so that a thread has PASSES rows' loads in flight.
template <typename T, int D, int PASSES>
__global__ void __launch_bounds__(THREADS)
compact_kernel(const T* K, const T* V, int64_t N, const int32_t* ret_idx, const int32_t* apx_idx, int n_ret, int n_apx,
               const int32_t* ret_slots, const int32_t* apx_slots, Pools pools, int chunks) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    constexpr int G = Row<D>::GROUPS, PER = THREADS / G;
    const int u = blockIdx.x / chunks, chunk = blockIdx.x - u * chunks;
    const int b = u / pools.LH, lh = u - b * pools.LH;
    const int group = threadIdx.x % G, rsub = threadIdx.x / G, rows = 2 * n_ret + n_apx;
    const T* src[PASSES];
    int slot[PASSES], tok[PASSES], what[PASSES];                      // what: 0 retained key, 1 value, 2 key-only
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = (chunk * PASSES + p) * PER + rsub;
        src[p] = nullptr; slot[p] = 0; tok[p] = 0;
        what[p] = r < n_ret ? 0 : r < 2 * n_ret ? 1 : 2;
        if (r >= rows) continue;
        const int i = r - what[p] * n_ret;
        const bool ret = what[p] < 2;
        tok[p] = ret ? ret_idx[(size_t)u * n_ret + i] : apx_idx[(size_t)u * n_apx + i];
        slot[p] = ret ? ret_slots[(size_t)b * n_ret + i] : apx_slots[(size_t)b * n_apx + i];
        // a token outside the context or a slot outside the pool: the row is skipped
        if ((unsigned long long)(long long)tok[p] < (unsigned long long)N && (uint32_t)slot[p] < (ret ? pools.ret_slots : pools.apx_slots))
            src[p] = (what[p] == 1 ? V : K) + ((size_t)u * N + tok[p]) * D + 16 * group;
    }
    uint4 v[PASSES][Raw<T>::N];
#pragma unroll
    for (int p = 0; p < PASSES; ++p)
        if (src[p]) load_group(src[p], v[p]);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        if (!src[p]) continue;
        uint32_t scale;
        const uint2 codes = encode_group(v[p], scale);
        const uint32_t page = (uint32_t)slot[p] / ROWS;
        const int row = slot[p] % ROWS;
        put_group<D>(what[p] < 2 ? ret_tile<D>(pools, page, lh, what[p]) : apx_tile<D>(pools, page, lh), row, group, codes, scale);
        int32_t* pos = what[p] == 0 ? pools.ret_pos : what[p] == 2 ? pools.apx_pos : nullptr;
        if (group == 0 && pos) pos[((size_t)page * pools.LH + lh) * ROWS + row] = tok[p];
    }
}

// One generated token's rows: of sequence b to slots[row_start[b]] (where it has a new row), or to slots[b].
template <typename T, int D>
__global__ void __launch_bounds__(THREADS)
append_kernel(const T* k_new, const T* v_new, const int32_t* row_start, const int32_t* slots, int64_t n_slots, const int32_t* pos, Pools pools,
              int U) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    constexpr int G = Row<D>::GROUPS;
    const long long i = (long long)blockIdx.x * THREADS + threadIdx.x;     // (unit, key or value, group)
    const int group = (int)(i % G), is_v = (int)(i / G) & 1, u = (int)(i / (2 * G));
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
    uint4 v[Raw<T>::N];
    load_group((is_v ? v_new : k_new) + (size_t)u * D + 16 * group, v);
    uint32_t scale;
    const uint2 codes = encode_group(v, scale);
    put_group<D>(ret_tile<D>(pools, slot / ROWS, lh, is_v), slot % ROWS, group, codes, scale);
    if (group == 0 && !is_v && pools.ret_pos) pools.ret_pos[((size_t)(slot / ROWS) * pools.LH + lh) * ROWS + slot % ROWS] = pos[b];
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

// Rows of slots as the values they stand for, [U][n][D] each; a slot outside its pool gives zeros.  The rows of a unit as in compact_kernel.
template <typename T, int D, int PASSES>
__global__ void __launch_bounds__(THREADS)
read_kernel(const int32_t* ret_slots, const int32_t* apx_slots, int n_ret, int n_apx, Pools pools, T* __restrict__ ret_k, T* __restrict__ ret_v,
            T* __restrict__ apx_k, int chunks) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    constexpr int G = Row<D>::GROUPS, PER = THREADS / G;
    const int u = blockIdx.x / chunks, chunk = blockIdx.x - u * chunks;
    const int b = u / pools.LH, lh = u - b * pools.LH;
    const int group = threadIdx.x % G, rsub = threadIdx.x / G, rows = 2 * n_ret + n_apx;
    const unsigned char* tile[PASSES];
    int row[PASSES];
    T* dst[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int r = (chunk * PASSES + p) * PER + rsub;
        tile[p] = nullptr; dst[p] = nullptr; row[p] = 0;
        if (r >= rows) continue;
        const int what = r < n_ret ? 0 : r < 2 * n_ret ? 1 : 2, i = r - what * n_ret;
        const uint32_t slot = (uint32_t)(what < 2 ? ret_slots[(size_t)b * n_ret + i] : apx_slots[(size_t)b * n_apx + i]);
        if (slot < (what < 2 ? pools.ret_slots : pools.apx_slots))
            tile[p] = what < 2 ? ret_tile<D>(pools, slot / ROWS, lh, what) : apx_tile<D>(pools, slot / ROWS, lh);
        row[p] = slot % ROWS;
        dst[p] = (what == 0 ? ret_k : what == 1 ? ret_v : apx_k) + ((size_t)u * (what < 2 ? n_ret : n_apx) + i) * D + 16 * group;
    }
    uint2 codes[PASSES];
    uint32_t scale[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        codes[p] = make_uint2(0, 0); scale[p] = 0;
        if (!tile[p]) continue;
        const unsigned char* r = tile[p] + row[p] * Row<D>::CODES;
        if constexpr (D == 128) {
            codes[p] = *reinterpret_cast<const uint2*>(r + Row<D>::byte_of(16 * group));
        } else {
            codes[p].x = *reinterpret_cast<const uint32_t*>(r + Row<D>::byte_of(16 * group));
            codes[p].y = *reinterpret_cast<const uint32_t*>(r + Row<D>::byte_of(16 * group + 8));
        }
        scale[p] = tile[p][Row<D>::SCALES_AT + row[p] * G + Row<D>::scale_of(group)];
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        if (!dst[p]) continue;
        const float s = scale_value(scale[p]);
        float x[16];
        const uint32_t w[2] = {codes[p].x, codes[p].y};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t pair[4];
            decode_word(w[h], pair);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&pair[i]));
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
// Blocks of a launch over `rows` rows of every unit, `per_block` to a block; 0 where they are too many.
static unsigned row_blocks(const Dims& dm, int64_t rows, int per_block, int* chunks) {
    const int64_t n = (rows + per_block - 1) / per_block, blocks = n * dm.U;
    *chunks = (int)n;
    return blocks > 0x7fffffffLL ? 0u : (unsigned)blocks;
}

struct CompactCall {
    const Dims& dm; const vector_budget* b; const void *K, *V; const int32_t *ret_idx, *apx_idx, *ret_slots, *apx_slots; Pools pools; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        constexpr int PASSES = PASSES_OF<T>;
        int chunks;
        const unsigned blocks = row_blocks(dm, 2 * b->n_ret + b->n_apx, PASSES * (THREADS / Row<D>::GROUPS), &chunks);
        if (!blocks) return VECTOR_ERR_SHAPE;
        VEC_CUDA_CHECK(launch_maybe_dependent(true, compact_kernel<T, D, PASSES>, dim3(blocks), dim3(THREADS), 0, st, (const T*)K, (const T*)V, b->n_tokens,
                                              ret_idx, apx_idx, (int)b->n_ret, (int)b->n_apx, ret_slots, apx_slots, pools, chunks));
        return VECTOR_OK;
    }
};
struct AppendCall {
    const Dims& dm; const void *k, *v; const int32_t *row_start, *slots; int64_t n_slots; const int32_t* pos; Pools pools; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        const long long n = (long long)dm.U * 2 * Row<D>::GROUPS;
        VEC_CUDA_CHECK(launch_maybe_dependent(true, append_kernel<T, D>, dim3((unsigned)((n + THREADS - 1) / THREADS)), dim3(THREADS), 0, st, (const T*)k,
                                              (const T*)v, row_start, slots, n_slots, pos, pools, dm.U));
        return VECTOR_OK;
    }
};
struct ReadCall {
    const Dims& dm; const int32_t *ret_slots, *apx_slots; int64_t n_ret, n_apx; void *ret_k, *ret_v, *apx_k; Pools pools; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        constexpr int PASSES = PASSES_OF<T>;
        int chunks;
        const unsigned blocks = row_blocks(dm, 2 * n_ret + n_apx, PASSES * (THREADS / Row<D>::GROUPS), &chunks);
        if (!blocks) return VECTOR_ERR_SHAPE;
        VEC_CUDA_CHECK(launch_maybe_dependent(true, read_kernel<T, D, PASSES>, dim3(blocks), dim3(THREADS), 0, st, ret_slots, apx_slots, (int)n_ret, (int)n_apx,
                                              pools, (T*)ret_k, (T*)ret_v, (T*)apx_k, chunks));
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
