// From a layer's projections to the rows that this library takes: queries, keys and values of every token, heads behind one another, become a row a head, tokens
// behind one another; on the way queries and keys are normed a head at a time and turned by their positions.
//
//   y = x / sqrt(mean(x^2) + eps) * w,   then for each pair of channels (c, c + D/2) and t = pos theta^(-2c/D):   (y_c cos t - y' sin t, y' cos t + y_c sin t)
//
// LANES threads have a row of a head, 16 bytes each, and take one token's heads in turn: the factors of a channel, w cos t and (of the pair's other channel, with its sign) w sin t, are
// computed once for all heads, and a row then takes a sum of squares over its lanes, one exchange of its raw bytes with the lane half a head away, two products and a factor a channel.
// All in fp32, rounded once.  Bound by memory where there are many tokens; a few are bound by the chain load, sum, store.
#include "common.cuh"
#include "internal.h"
#include "rope.cuh"

namespace vec {
namespace rows {

constexpr int THREADS = 256, AHEAD = 4;      // heads that a thread has in flight
template <typename T, int D> struct Lanes { static constexpr int E = 16 / (int)sizeof(T), N = D / E, GROUPS = THREADS / N; };

// One of the three projections.
struct Part {
    const void* in;              // null: not asked for
    int64_t stride;              // elements between tokens
    const void* weight;          // [L][D], or null
    void* out;                   // [B L][heads][tokens - first][D]
    int64_t first;               // tokens before it are left out
    int heads, turned;
};
struct Args { Part part[3]; const int32_t* pos; int64_t n_tokens, total; float eps; int L, per, heads; };

__device__ __forceinline__ void widen(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void widen(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ uint4 narrow(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 narrow(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}

// grid: (groups of tokens of all sequences and layers, runs of `per` heads of the three projections in a row).
template <typename T, int D>
__global__ void __launch_bounds__(THREADS)
norm_rope_kernel(Args a, RopePhases phases) {
    using G = Lanes<T, D>;
    constexpr int E = G::E, N = G::N;
    __shared__ RopePhase phase[D / 2];
    if (threadIdx.x < D / 2) phase[threadIdx.x] = rope_phase_words(phases.phase[threadIdx.x]);
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    __syncthreads();
    const int lane = threadIdx.x % N;
    const int64_t row = (int64_t)blockIdx.x * G::GROUPS + threadIdx.x / N;
    const bool there = row < a.total;                                    // the warp's exchanges need all of its threads
    const int64_t at = there ? row : 0, bl = (at >> 32) == 0 && (a.n_tokens >> 32) == 0 ? (uint32_t)at / (uint32_t)a.n_tokens : at / a.n_tokens, t = at - bl * a.n_tokens;
    const int b = (int)(bl / a.L), l = (int)(bl - (int64_t)b * a.L);
    const int32_t pos = a.pos ? a.pos[(int64_t)b * a.n_tokens + t] : (int32_t)t;
    const bool upper = lane >= N / 2;
    const int pair = lane % (N / 2) * E;
    float cs[E], sn[E];
#pragma unroll
    for (int i = 0; i < E; i += 2) {
        uint64_t cs2, sn2;
        rope_cos_sin2(rope_angle(pos, phase[pair + i]), rope_angle(pos, phase[pair + i + 1]), cs2, sn2);
        tc::unpack2(cs2, cs[i], cs[i + 1]);
        tc::unpack2(sn2, sn[i], sn[i + 1]);
    }
    const int h0 = blockIdx.y * a.per, h1 = min(h0 + a.per, a.heads);
    int base = 0;
#pragma unroll 1
    for (int which = 0; which < 3; ++which) {
        const Part& part = a.part[which];
        const int n = part.in ? part.heads : 0, from = max(h0 - base, 0), to = min(h1 - base, n);
        base += n;
        const bool wanted = there && t >= part.first;
        if (from >= to || !__any_sync(0xffffffffu, wanted)) continue;
        const T* src = reinterpret_cast<const T*>(part.in) + at * part.stride + lane * E;
        const int64_t tokens = a.n_tokens - part.first;
        T* dst = reinterpret_cast<T*>(part.out) + (bl * part.heads * tokens + t - part.first) * D + lane * E;
        // factors of a channel and of its pair's other one
        float mine[E], other[E];
        const bool normed = part.weight != nullptr, turned = part.turned;
        if (normed) {
            const T* w = reinterpret_cast<const T*>(part.weight) + (size_t)l * D;
            widen(*reinterpret_cast<const uint4*>(w + lane * E), mine);
            widen(*reinterpret_cast<const uint4*>(w + (lane ^ (N / 2)) * E), other);
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) mine[i] = other[i] = 1.f;
        }
        if (turned) {
#pragma unroll
            for (int i = 0; i < E; ++i) { mine[i] *= cs[i]; other[i] *= upper ? sn[i] : -sn[i]; }
        }
#pragma unroll 1
        for (int h = from; h < to; h += AHEAD) {
            uint4 v[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                v[j] = make_uint4(0, 0, 0, 0);
                if (wanted && h + j < to) v[j] = *reinterpret_cast<const uint4*>(src + (h + j) * D);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (h + j >= to) break;
                if (normed || turned) {
                    float x[E], y[E], r = 1.f;
                    widen(v[j], x);
                    if (normed) {
                        float sum = 0.f;
#pragma unroll
                        for (int i = 0; i < E; ++i) sum = fmaf(x[i], x[i], sum);
#pragma unroll
                        for (int o = N / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                        r = rsqrtf(fmaf(sum, 1.f / D, a.eps));
                    }
                    if (turned) {
                        uint4 w;
                        w.x = __shfl_xor_sync(0xffffffffu, v[j].x, N / 2); w.y = __shfl_xor_sync(0xffffffffu, v[j].y, N / 2);
                        w.z = __shfl_xor_sync(0xffffffffu, v[j].z, N / 2); w.w = __shfl_xor_sync(0xffffffffu, v[j].w, N / 2);
                        widen(w, y);
#pragma unroll
                        for (int i = 0; i < E; ++i) x[i] = r * fmaf(x[i], mine[i], y[i] * other[i]);
                    } else {
#pragma unroll
                        for (int i = 0; i < E; ++i) x[i] = r * (x[i] * mine[i]);
                    }
                    v[j] = narrow(x);
                }
                if (wanted) *reinterpret_cast<uint4*>(dst + (int64_t)(h + j) * tokens * D) = v[j];
            }
        }
    }
}

struct Call {
    const Dims& dm; Args a; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        using G = Lanes<T, D>;
        Args args = a;
        // A group of lanes takes as many heads of its token as leave the multiprocessors 32 warps each: the angles and factors are computed once for all of them.
        const int64_t wanted = (int64_t)sm_count() * 1024 / G::N, runs = (wanted + a.total - 1) / a.total;
        args.per = (int)(runs >= a.heads ? 1 : (a.heads + runs - 1) / runs);
        if (args.per < (a.heads + 65534) / 65535) args.per = (a.heads + 65534) / 65535;
        RopePhases ph = {};
        if (dm.rope) rope_phases(dm.theta, D, &ph);
        const dim3 grid((unsigned)((a.total + G::GROUPS - 1) / G::GROUPS), (unsigned)((a.heads + args.per - 1) / args.per));
        VEC_CUDA_CHECK(launch_maybe_dependent(true, norm_rope_kernel<T, D>, grid, dim3(THREADS), 0, st, args, ph));
        return VECTOR_OK;
    }
};

}  // namespace rows
}  // namespace vec

using namespace vec;

extern "C" vector_status vector_norm_rope(const vector_shape* shape, int64_t n_tokens, const void* q, int64_t q_stride, const void* q_weight, int64_t q_first, void* q_out,
                                          const void* k, int64_t k_stride, const void* k_weight, void* k_out, const void* v, int64_t v_stride, void* v_out, const int32_t* pos,
                                          float eps, void* stream) {
    Dims dm;
    const vector_status rc = check_shape(shape, &dm);
    if (rc != VECTOR_OK) return rc;
    if (n_tokens < 0 || n_tokens > (int64_t(1) << 30) || q_first < 0 || q_first > n_tokens || !(eps >= 0.f)) return VECTOR_ERR_SHAPE;
    const int H[3] = {shape->n_q_heads, shape->n_kv_heads, shape->n_kv_heads};
    rows::Args a = {{{q, q_stride, q_weight, q_out, q_first, H[0], dm.rope}, {k, k_stride, k_weight, k_out, 0, H[1], dm.rope}, {v, v_stride, nullptr, v_out, 0, H[2], 0}},
                    pos, n_tokens, (int64_t)shape->batch * shape->n_layers * n_tokens, eps, shape->n_layers, 0, 0};
    uintptr_t bits = 0;
    for (int i = 0; i < 3; ++i) {
        rows::Part& p = a.part[i];
        if (p.first == n_tokens) p.in = nullptr;
        if (!p.in) continue;
        if (!p.out) return VECTOR_ERR_NULL;
        if (p.stride < (int64_t)p.heads * dm.d || p.stride > (int64_t(1) << 40)) return VECTOR_ERR_SHAPE;
        bits |= (uintptr_t)p.in | (uintptr_t)p.weight | (uintptr_t)p.out | (uintptr_t)(p.stride * dm.esize);
        a.heads += p.heads;
    }
    if (bits & 15) return VECTOR_ERR_SHAPE;
    if (a.heads == 0) return VECTOR_OK;
    if (a.total > (int64_t(1) << 33)) return VECTOR_ERR_SHAPE;            // blocks of a launch
    const rows::Call call = {dm, a, (cudaStream_t)stream};
    using B = __nv_bfloat16;
    if (dm.dtype == VECTOR_F32) return dm.d == 64 ? call.run<float, 64>() : call.run<float, 128>();
    return dm.d == 64 ? call.run<B, 64>() : call.run<B, 128>();
}
