// Generation-time attention over the 8-bit paged cache (q8.cuh).  The kernels are those of the 4-bit pages, in decode_q4.cuh, with another kind of tile: a
// worker's chain of loads, products and softmax bounds them, not the bytes (640 units of 3277 and 6552 rows, 1.1 GB, 227 us, of which copies alone take 198; at
// the copy rate 171).
#include "decode_q4.cuh"

namespace vec {
namespace dq8 {             // names of its own: the linker keeps one of two functions of the same name
using namespace dq4;

constexpr int MOST_WARPS = 16;          // of a streaming block, over all kernels

static size_t ws_bytes_of(const Dims& dm) {
    return ends_bytes(dm.U) + ((size_t)dm.U + sm_count() * MOST_WARPS) * 2 * tier_floats(dm.g, dm.d) * 4;
}

struct Call {
    const Dims& dm; const void* q; Cache c; const void* W; void* out; int out_dtype; unsigned char* ws; cudaStream_t st;

    template <typename T, int D, bool ROPE, bool EXACT, bool FOLD> vector_status both() const {
        using C = Cfg<T, D, ROPE, EXACT, FOLD, Bits8>;
        static_assert(C::WARPS <= MOST_WARPS && C::SMEM_BYTES + (MAX_BATCH + 1) * 8 + 2048 <= 227 * 1024, "a block's shared memory, its own variables included");
        auto kern = decode_q4_stream<T, D, ROPE, EXACT, FOLD, Bits8>;
        static PerDeviceOnce once;
        if (once.first()) {
            const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM_BYTES + (MAX_BATCH + 1) * 8);
            if (e != cudaSuccess) { once.undo(); VEC_CUDA_CHECK(e); }
        }
        int* fault = kernel_fault_address();
        if (!fault) return VECTOR_ERR_CUDA;
        RopePhases ph = {};
        if (ROPE) rope_phases(dm.theta, D, &ph);
        VEC_CUDA_CHECK(launch_maybe_dependent(true, kern, dim3(sm_count()), dim3(C::THREADS), C::SMEM_BYTES + (size_t)(c.batch + 1) * 8, st, (const T*)q, c, dm.g,
                                              dm.scale * 1.4426950408889634f, ws, fault, ph));
        return merge<T, D>(sm_count() * C::WARPS);
    }
    template <typename T, int D, int HP, int THREADS> vector_status merge_by(int seqs, int workers) const {
        auto kern = decode_q4_merge<T, D, HP, THREADS, Bits8>;
        constexpr int smem = MapTile<T, D>::BYTES;
        static PerDeviceOnce once;
        if (once.first()) {
            const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
            if (e != cudaSuccess) { once.undo(); VEC_CUDA_CHECK(e); }
        }
        VEC_CUDA_CHECK(launch_maybe_dependent(true, kern, dim3((unsigned)(dm.LH * ((c.batch + seqs - 1) / seqs))), dim3(THREADS), smem, st, (const unsigned char*)ws, c,
                                              dm.g, seqs, workers, (const T*)W, out, out_dtype == VECTOR_BF16 ? 1 : 0));
        return VECTOR_OK;
    }
    // As over the 4-bit pages, whose records are the same: no more units than multiprocessors take a large block each, more units small blocks, and as many
    // sequences for a map that is fetched once as leave one round of blocks.
    template <typename T, int D, int HP> vector_status merge_heads(int workers) const {
        if (dm.U <= sm_count()) return merge_by<T, D, HP, MERGE_MOST>(1, workers);
        const int resident = merge_blocks<T, D, MERGE_THREADS>() * sm_count(), rounds = (dm.U + resident - 1) / resident;
        return merge_by<T, D, HP, MERGE_THREADS>(rounds < c.batch ? rounds : c.batch, workers);
    }
    template <typename T, int D> vector_status merge(int workers) const {
        return dm.g <= 2 ? merge_heads<T, D, 1>(workers) : dm.g <= 4 ? merge_heads<T, D, 2>(workers) : dm.g <= 6 ? merge_heads<T, D, 3>(workers) : merge_heads<T, D, 4>(workers);
    }
    template <typename T, int D> vector_status run() const {
        const bool exact = dm.dtype == VECTOR_F32 || out_dtype == VECTOR_F32;
        if constexpr (sizeof(T) == 2)
            if (!exact) return dm.rope ? both<T, D, true, false, false>() : both<T, D, false, false, false>();
        if (dm.g <= 4) return dm.rope ? both<T, D, true, true, true>() : both<T, D, false, true, true>();
        return dm.rope ? both<T, D, true, true, false>() : both<T, D, false, true, false>();
    }
};

}  // namespace dq8
}  // namespace vec

using namespace vec;

extern "C" size_t vector_decode_q8_workspace_bytes(const vector_shape* shape) {
    Dims dm;
    if (check_shape(shape, &dm) != VECTOR_OK) return 0;
    return dq8::ws_bytes_of(dm);
}

extern "C" vector_status vector_decode_attn_q8(const vector_shape* shape, const void* q, const vector_q8_cache* cache, const void* W, void* out,
                                               int32_t out_dtype, void* ws, size_t ws_bytes, void* stream) {
    Dims dm;
    vector_status rc = check_shape(shape, &dm);
    if (rc != VECTOR_OK) return rc;
    if ((rc = check_q8_cache(cache)) != VECTOR_OK) return rc;
    if (!q || !W || !out) return VECTOR_ERR_NULL;
    if (out_dtype != VECTOR_F32 && out_dtype != VECTOR_BF16) return VECTOR_ERR_DTYPE;
    if (shape->batch > VECTOR_Q4_MAX_BATCH) return VECTOR_ERR_SHAPE;
    if (cache->ret_width > 0 && (!cache->ret_table || !cache->ret_len)) return VECTOR_ERR_NULL;
    if (cache->apx_width > 0 && (!cache->apx_table || !cache->apx_len)) return VECTOR_ERR_NULL;
    if (dm.rope && cache->n_apx_pages > 0 && !cache->apx_pos) return VECTOR_ERR_NULL;
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < dq8::ws_bytes_of(dm)) return VECTOR_ERR_WORKSPACE;
    if (((uintptr_t)q | (uintptr_t)W | (uintptr_t)out) & 15) return VECTOR_ERR_SHAPE;
    const dq4::Cache c = {(const unsigned char*)cache->ret_pages, (const unsigned char*)cache->apx_pages, cache->ret_table, cache->apx_table,
                          cache->ret_len, cache->apx_len, cache->apx_pos, cache->n_ret_pages, cache->n_apx_pages, cache->ret_width, cache->apx_width, dm.LH,
                          shape->batch};
    const dq8::Call call = {dm, q, c, W, out, out_dtype, (unsigned char*)ws, (cudaStream_t)stream};
    if (dm.dtype == VECTOR_F32) return dm.d == 64 ? call.run<float, 64>() : call.run<float, 128>();
    return dm.d == 64 ? call.run<__nv_bfloat16, 64>() : call.run<__nv_bfloat16, 128>();
}
