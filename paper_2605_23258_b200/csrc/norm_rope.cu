// From a layer's projections to the rows that this library takes: queries, keys and values of every token, heads behind one another, become a row a head,
// tokens behind one another; on the way queries and keys are normed a head at a time and turned by their positions.
//
//   y = x / sqrt(mean(x^2) + eps) * w,   then for each pair of channels (c, c + D/2) and t = pos theta^(-2c/D):   (y_c cos t - y' sin t, y' cos t + y_c sin t)
//
// A group of D / E lanes has a token and a run of heads of one projection, 16 bytes of a row a lane, several rows on their way at once: the factors of a
// channel, w cos t and (of the pair's other channel, with its sign) w sin t, are computed once for the run, and a row then takes a sum of squares over its
// lanes, one exchange of its raw bytes with the lane half a head away, two products and a factor a channel, two channels an instruction.  All in fp32, rounded
// once.  Bound by memory where there are many tokens (0.89 to 0.95 of the copy rate; 0.81 where the rows are over in 23 us), by one launch and the chain load,
// sum, store where there are few (64 tokens 3.4 us).
#include "common.cuh"
#include "internal.h"
#include "rope.cuh"

namespace vec {
namespace rows {

// us for a prompt of 32768 tokens in 32 and 8 heads of 128 channels, window queries, keys and values (270 MB, 41.2 at the copy rate), and with all queries (805
// MB, 123.2): 46.4 and 129.2; blocks of 256 threads 50 and 155, four rows of a head on their way 46.1 and 130.7 (fp32, 64 channels: 22.9, eight 24.1), eight
// blocks a multiprocessor, which spill, 50 and 156, six 48 and 134; angles and factors for every eight heads 46.5 and 140; both lanes of a pair computing all
// its angles, and products one at a time, 49 and 150.
constexpr int THREADS = 128;
template <typename T> constexpr int AHEAD_OF = sizeof(T) == 2 ? 8 : 4;       // heads' rows that a lane has on their way
template <typename T, int D> struct Lanes { static constexpr int E = 16 / (int)sizeof(T), N = D / E, GROUPS = THREADS / N; };

// One of the three projections.
struct Part {
    const void* in;              // null: not asked for
    int64_t stride;              // elements between tokens
    const void* weight;          // [L][D], or null
    void* out;                   // [B L][heads][tokens - first][D]
    int64_t first;               // tokens before it are left out
    int heads, turned;
    int64_t rows;                // tokens of all sequences and layers that are not
    unsigned blocks, runs;       // of the launch, and of heads that the blocks take in turn
};
struct Args { Part part[3]; const int32_t* pos; int64_t n_tokens; float eps; int L, per; };

// 16 bytes of a row as pairs of fp32 numbers, and back.
__device__ __forceinline__ void widen(const uint4& v, uint64_t (&x)[4]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = tc::pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ void widen(const uint4& v, uint64_t (&x)[2]) {
    x[0] = tc::pack2(__uint_as_float(v.x), __uint_as_float(v.y));
    x[1] = tc::pack2(__uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ uint4 narrow(const uint64_t (&x)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        tc::unpack2(x[i], a, b);
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 narrow(const uint64_t (&x)[2]) {
    float a, b, c, d;
    tc::unpack2(x[0], a, b);
    tc::unpack2(x[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
}
__device__ __forceinline__ uint64_t swap_lanes(uint64_t x, int mask) { return __shfl_xor_sync(0xffffffffu, x, mask); }

// a / b, in 32 bits where they do.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) { return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b; }

// grid: the projections' blocks in a row; of each, blocks of THREADS / N tokens, whose runs of `per` heads are neighbours: a token's row is read at about one time.
template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 7)
norm_rope_kernel(Args a, RopePhases phases) {
    using G = Lanes<T, D>;
    constexpr int E = G::E, N = G::N, AHEAD = AHEAD_OF<T>;
    __shared__ RopePhase phase[D / 2];                                   // a thread's index into a kernel's parameters would be served a lane at a time
    if (threadIdx.x < D / 2) phase[threadIdx.x] = rope_phase_words(phases.phase[threadIdx.x]);
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    __syncthreads();
    unsigned block = blockIdx.x;
    int which = 0;
    while (which < 2 && block >= a.part[which].blocks) block -= a.part[which++].blocks;
    const Part& part = a.part[which];
    const int from = (int)(block % part.runs) * a.per, to = min(from + a.per, part.heads);
    const int lane = threadIdx.x % N;
    const int64_t row = (int64_t)(block / part.runs) * G::GROUPS + threadIdx.x / N;
    const bool there = row < part.rows;                                  // the warp's exchanges need all of its threads
    const int64_t tokens = a.n_tokens - part.first, at = there ? row : 0, bl = divide(at, tokens), t = at - bl * tokens + part.first;
    const T* src = reinterpret_cast<const T*>(part.in) + (bl * a.n_tokens + t) * part.stride + lane * E;
    T* dst = reinterpret_cast<T*>(part.out) + (bl * part.heads * tokens + t - part.first) * D + lane * E;
    const bool normed = part.weight != nullptr, turned = part.turned;
    uint64_t mine[E / 2], other[E / 2];                                  // factors of a channel and of its pair's other one
#pragma unroll 1
    for (int h = from; h < to; h += AHEAD) {
        uint4 v[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            v[j] = make_uint4(0, 0, 0, 0);
            if (there && h + j < to) v[j] = *reinterpret_cast<const uint4*>(src + (size_t)(h + j) * D);
        }
        if (h == from && (normed || turned)) {                           // while the rows are on their way
            const int b = (int)divide(bl, a.L), l = (int)(bl - (int64_t)b * a.L);
            if (normed) {
                const T* w = reinterpret_cast<const T*>(part.weight) + (size_t)l * D;
                widen(*reinterpret_cast<const uint4*>(w + lane * E), mine);
                widen(*reinterpret_cast<const uint4*>(w + (lane ^ (N / 2)) * E), other);
            } else {
#pragma unroll
                for (int i = 0; i < E / 2; ++i) mine[i] = other[i] = tc::pack2(1.f, 1.f);
            }
            if (turned) {
                const int32_t pos = a.pos ? a.pos[(int64_t)b * a.n_tokens + t] : (int32_t)t;
                const bool upper = lane >= N / 2;
                // two lanes half a row apart have the same angles: each computes half of them
                const int pair = lane % (N / 2) * E + (upper ? E / 2 : 0);
#pragma unroll
                for (int i = 0; i < E / 4; ++i) {
                    uint64_t cs, sn;
                    rope_cos_sin2(rope_angle(pos, phase[pair + 2 * i]), rope_angle(pos, phase[pair + 2 * i + 1]), cs, sn);
                    const uint64_t cs_o = swap_lanes(cs, N / 2), sn_o = swap_lanes(sn, N / 2);
                    const uint64_t sign = upper ? 0ull : 0x8000000080000000ull;
                    mine[i] = tc::mul2(mine[i], upper ? cs_o : cs);
                    mine[i + E / 4] = tc::mul2(mine[i + E / 4], upper ? cs : cs_o);
                    other[i] = tc::mul2(other[i], (upper ? sn_o : sn) ^ sign);
                    other[i + E / 4] = tc::mul2(other[i + E / 4], (upper ? sn : sn_o) ^ sign);
                }
            }
        }
        if (normed || turned) {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (h + j >= to) break;
                uint64_t x[E / 2];
                float r = 1.f;
                widen(v[j], x);
                if (normed) {
                    uint64_t squares = tc::mul2(x[0], x[0]);
#pragma unroll
                    for (int i = 1; i < E / 2; ++i) squares = tc::fma2(x[i], x[i], squares);
                    float sum, rest;
                    tc::unpack2(squares, sum, rest);
                    sum += rest;
#pragma unroll
                    for (int o = N / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    r = rsqrtf(fmaf(sum, 1.f / D, a.eps));
                }
                const uint64_t r2 = tc::pack2(r, r);
                if (turned) {
                    uint4 w;
                    w.x = __shfl_xor_sync(0xffffffffu, v[j].x, N / 2); w.y = __shfl_xor_sync(0xffffffffu, v[j].y, N / 2);
                    w.z = __shfl_xor_sync(0xffffffffu, v[j].z, N / 2); w.w = __shfl_xor_sync(0xffffffffu, v[j].w, N / 2);
                    uint64_t y[E / 2];
                    widen(w, y);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) x[i] = tc::mul2(r2, tc::fma2(x[i], mine[i], tc::mul2(y[i], other[i])));
                } else {
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) x[i] = tc::mul2(r2, tc::mul2(x[i], mine[i]));
                }
                v[j] = narrow(x);
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (there && h + j < to) *reinterpret_cast<uint4*>(dst + (int64_t)(h + j) * tokens * D) = v[j];
    }
}

struct Call {
    const Dims& dm; Args a; cudaStream_t st;
    template <typename T, int D> vector_status run() const {
        using G = Lanes<T, D>;
        Args args = a;
        // Heads of a run: as many as leave the multiprocessors 32 warps each, so that the angles and factors are computed once for all of them.
        int64_t rows = 0, blocks = 0;
        for (const Part& p : a.part) rows += p.rows * p.heads;
        const int64_t per = rows / ((int64_t)sm_count() * 1024 / G::N);
        args.per = (int)(per < 1 ? 1 : per > 1 << 20 ? 1 << 20 : per);
        for (Part& p : args.part) {
            p.runs = (unsigned)((p.heads + args.per - 1) / args.per);
            const int64_t all = (p.rows + G::GROUPS - 1) / G::GROUPS * p.runs;
            blocks += all;
            if (blocks > 0x7fffffffLL) return VECTOR_ERR_SHAPE;
            p.blocks = (unsigned)all;
        }
        if (blocks == 0) return VECTOR_OK;
        RopePhases ph = {};
        if (dm.rope) rope_phases(dm.theta, D, &ph);
        VEC_CUDA_CHECK(launch_maybe_dependent(true, norm_rope_kernel<T, D>, dim3((unsigned)blocks), dim3(THREADS), 0, st, args, ph));
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
                    pos, n_tokens, eps, shape->n_layers, 0};
    uintptr_t bits = 0;
    for (rows::Part& p : a.part) {
        if (!p.in || p.first == n_tokens) continue;                       // no rows
        if (!p.out) return VECTOR_ERR_NULL;
        if (p.stride < (int64_t)p.heads * dm.d || p.stride > (int64_t(1) << 40)) return VECTOR_ERR_SHAPE;
        bits |= (uintptr_t)p.in | (uintptr_t)p.weight | (uintptr_t)p.out | (uintptr_t)(p.stride * dm.esize);
        p.rows = (int64_t)shape->batch * shape->n_layers * (n_tokens - p.first);
    }
    if (bits & 15) return VECTOR_ERR_SHAPE;
    const rows::Call call = {dm, a, (cudaStream_t)stream};
    using B = __nv_bfloat16;
    if (dm.dtype == VECTOR_F32) return dm.d == 64 ? call.run<float, 64>() : call.run<float, 128>();
    return dm.d == 64 ? call.run<B, 64>() : call.run<B, 128>();
}
