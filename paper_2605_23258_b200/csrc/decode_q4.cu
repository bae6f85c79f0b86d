// Generation-time attention over the 4-bit paged cache (q4.cuh): what vector_decode_attn computes, of rows that lie in pages, with lengths of
// their own for every sequence.
#include "common.cuh"
#include "internal.h"
#include "q4.cuh"

namespace vec {
namespace dq4 {

constexpr int WARPS = 8;

struct Cache {
    const unsigned char *ret, *apx;
    const int32_t *ret_table, *apx_table, *ret_len, *apx_len, *apx_pos;
    int64_t n_ret_pages, n_apx_pages;
    int32_t ret_width, apx_width, LH;
};
// Rows of a sequence in a tier: what its table can hold at the most.
__device__ __forceinline__ int rows_of(const int32_t* len, int b, int width) { return width ? min(max(len[b], 0), width * q4::ROWS) : 0; }

// A block a unit, a row across a warp's lanes: lane l has elements [l D/32, (l+1) D/32) of a row, and its rotary partner is lane l ^ 4.
template <typename T, int D, bool ROPE>
__global__ void __launch_bounds__(32 * WARPS)
decode_q4_rows(const T* q, Cache c, const T* W, int g, float scale, float theta, void* __restrict__ out, int out_bf16) {
    using R = q4::Row<D>;
    constexpr int E = D / 32;
    __shared__ float sum[WARPS][2][D], ml[WARPS][2], key_sum[D], o_val[D];
    __shared__ double inv_freq[ROPE ? D / 2 : 1];
    if (ROPE) { rope_fill_inv_freq(inv_freq, D, theta); __syncthreads(); }
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    const int u = blockIdx.x / g, a = blockIdx.x - u * g, b = u / c.LH, lh = u - b * c.LH;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int n_ret = rows_of(c.ret_len, b, c.ret_width), n_apx = rows_of(c.apx_len, b, c.apx_width);
    float qr[E], acc[2][E] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) qr[e] = to_f32(q[((size_t)u * g + a) * D + R::channel_of(lane * E + e)]) * scale;
    auto load = [&](const unsigned char* tile, int row, float (&x)[E]) {
        const unsigned char* p = tile + row * R::CODES + lane * (E / 2);
        const uint32_t w = E == 4 ? *reinterpret_cast<const uint16_t*>(p) : *p;
        const float s = q4::scale_value(tile[R::SCALES_AT + row * R::GROUPS + R::scale_of(R::channel_of(lane * E) / 16)]);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint32_t n = w >> (4 * e), size = n & 7;
            const float f = size < 2 ? 0.5f * size : __uint_as_float(((126 + (size >> 1)) << 23) | (size & 1) << 22);
            x[e] = (n & 8 ? -f : f) * s;
        }
    };
    for (int i = wid; i < n_ret + n_apx; i += WARPS) {
        const bool ret = i < n_ret;
        const int r = ret ? i : i - n_ret, row = r % q4::ROWS;
        const int64_t page = ret ? c.ret_table[(size_t)b * c.ret_width + r / q4::ROWS] : c.apx_table[(size_t)b * c.apx_width + r / q4::ROWS];
        if (page < 0 || page >= (ret ? c.n_ret_pages : c.n_apx_pages)) continue;
        const unsigned char* tile = ret ? c.ret + ((size_t)page * c.LH + lh) * 2 * R::TILE : c.apx + ((size_t)page * c.LH + lh) * R::TILE;
        float k[E], v[E], s = 0.f;
        load(tile, row, k);
#pragma unroll
        for (int e = 0; e < E; ++e) s = fmaf(qr[e], k[e], s);
        s = warp_sum(s);
        if (ret) {
            load(tile + R::TILE, row, v);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = k[e];
            if (ROPE) {
                const double pos = (double)c.apx_pos[((size_t)page * c.LH + lh) * q4::ROWS + row];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float cs, sn;
                    const int ch = R::channel_of(lane * E + e);
                    rope_cos_sin(pos, inv_freq[ch % (D / 2)], cs, sn);
                    const float other = __shfl_xor_sync(0xffffffffu, k[e], 4);
                    v[e] = ch < D / 2 ? fmaf(k[e], cs, other * sn) : fmaf(k[e], cs, -other * sn);
                }
            }
        }
        const float mn = fmaxf(m, s), corr = __expf(m - mn), p = __expf(s - mn);
        m = mn;
        l = l * corr + p;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            acc[0][e] = fmaf(acc[0][e], corr, ret ? p * v[e] : 0.f);
            acc[1][e] = fmaf(acc[1][e], corr, ret ? 0.f : p * v[e]);
        }
    }
    if (lane == 0) { ml[wid][0] = m; ml[wid][1] = l; }
#pragma unroll
    for (int e = 0; e < E; ++e) { sum[wid][0][R::channel_of(lane * E + e)] = acc[0][e]; sum[wid][1][R::channel_of(lane * E + e)] = acc[1][e]; }
    __syncthreads();
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) M = fmaxf(M, ml[w][0]);
    float f[WARPS];
#pragma unroll
    for (int w = 0; w < WARPS; ++w) { f[w] = ml[w][0] > -INFINITY ? __expf(ml[w][0] - M) : 0.f; L = fmaf(f[w], ml[w][1], L); }
    for (int e = threadIdx.x; e < 2 * D; e += 32 * WARPS) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) x = fmaf(f[w], sum[w][e / D][e % D], x);
        (e < D ? o_val : key_sum)[e % D] = x;
    }
    __syncthreads();
    for (int r = wid; r < D; r += WARPS) {
        float x = 0.f;
        for (int j = lane; j < D; j += 32) x = fmaf(to_f32(W[((size_t)lh * D + r) * D + j]), key_sum[j], x);
        x = warp_sum(x);
        const float o = L > 0.f ? (o_val[r] + x) / L : 0.f;              // nothing to attend to: zeros
        const size_t at = ((size_t)u * g + a) * D + r;
        if (lane == 0) {
            if (out_bf16) reinterpret_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(o);
            else reinterpret_cast<float*>(out)[at] = o;
        }
    }
}

}  // namespace dq4
}  // namespace vec

using namespace vec;

extern "C" size_t vector_decode_q4_workspace_bytes(const vector_shape* shape) {
    Dims dm;
    if (check_shape(shape, &dm) != VECTOR_OK) return 0;
    return 256;
}

extern "C" vector_status vector_decode_attn_q4(const vector_shape* shape, const void* q, const vector_q4_cache* cache, const void* W, void* out,
                                               int32_t out_dtype, void* ws, size_t ws_bytes, void* stream) {
    Dims dm;
    vector_status rc = check_shape(shape, &dm);
    if (rc != VECTOR_OK) return rc;
    if ((rc = check_q4_cache(cache)) != VECTOR_OK) return rc;
    if (!q || !W || !out) return VECTOR_ERR_NULL;
    if (out_dtype != VECTOR_F32 && out_dtype != VECTOR_BF16) return VECTOR_ERR_DTYPE;
    constexpr int32_t most_width = (1 << 30) / VECTOR_PAGE_ROWS;
    if (cache->ret_width < 0 || cache->apx_width < 0 || cache->ret_width > most_width || cache->apx_width > most_width || shape->batch > VECTOR_Q4_MAX_BATCH)
        return VECTOR_ERR_SHAPE;
    if (cache->ret_width > 0 && (!cache->ret_table || !cache->ret_len)) return VECTOR_ERR_NULL;
    if (cache->apx_width > 0 && (!cache->apx_table || !cache->apx_len)) return VECTOR_ERR_NULL;
    if (dm.rope && cache->n_apx_pages > 0 && !cache->apx_pos) return VECTOR_ERR_NULL;
    if (!ws || ((uintptr_t)ws & 255) || ws_bytes < vector_decode_q4_workspace_bytes(shape)) return VECTOR_ERR_WORKSPACE;
    if (((uintptr_t)q | (uintptr_t)W | (uintptr_t)out | (uintptr_t)cache->apx_pos) & 15) return VECTOR_ERR_SHAPE;
    const dq4::Cache c = {(const unsigned char*)cache->ret_pages, (const unsigned char*)cache->apx_pages, cache->ret_table, cache->apx_table,
                          cache->ret_len, cache->apx_len, cache->apx_pos, cache->n_ret_pages, cache->n_apx_pages, cache->ret_width, cache->apx_width, dm.LH};
    auto launch = [&](auto kern, auto t) -> vector_status {
        using T = decltype(t);
        VEC_CUDA_CHECK(launch_maybe_dependent(true, kern, dim3((unsigned)(dm.U * dm.g)), dim3(32 * dq4::WARPS), 0, (cudaStream_t)stream, (const T*)q, c,
                                              (const T*)W, dm.g, dm.scale, dm.theta, out, out_dtype == VECTOR_BF16 ? 1 : 0));
        return VECTOR_OK;
    };
    using B = __nv_bfloat16;
    if (dm.dtype == VECTOR_F32) {
        if (dm.d == 64) return dm.rope ? launch(dq4::decode_q4_rows<float, 64, true>, float()) : launch(dq4::decode_q4_rows<float, 64, false>, float());
        return dm.rope ? launch(dq4::decode_q4_rows<float, 128, true>, float()) : launch(dq4::decode_q4_rows<float, 128, false>, float());
    }
    if (dm.d == 64) return dm.rope ? launch(dq4::decode_q4_rows<B, 64, true>, B()) : launch(dq4::decode_q4_rows<B, 64, false>, B());
    return dm.rope ? launch(dq4::decode_q4_rows<B, 128, true>, B()) : launch(dq4::decode_q4_rows<B, 128, false>, B());
}
