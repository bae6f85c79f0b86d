// Attention over the 8-bit paged cache on the tcgen05 tensor cores, for heads of 128 channels without rotary positions: stored rows are operands as they are.
//
// A chunk is up to four neighbouring pages of one unit's tier: 128 keys, the rows of a product.  Per chunk
//   S [keys][heads]     = K Q^T      A: keys as they lie (K contiguous), 16 KB that TMA brings; B: queries in e4m3 parts
//   O^T [channels][heads] = V^T P^T  A: values as they lie, read the other way round (M contiguous); B: weights in e4m3 parts.  Key-only rows: K^T P^T of the rows that gave the logits
// and nothing converts a stored number or moves it between registers: what the kernel of decode_q4.cuh spends most of its time on.  A query is the sum of QP parts, each the nearest e4m3
// number to what the ones before it leave, times 32^i; a weight of PP: parts are columns of one product, whose sums are weighed by 32^-i.  An A operand is fetched from shared memory in 32 cycles
// whatever the columns up to 64, so parts cost no time there.  With three parts a bf16 query is exact down to 2^-14 of its head's largest channel, and right to 2^-28 of that below; weights are right to
// 2^-4PP of themselves and 2^-(5 PP + 11) of the largest.  The scale of a page of keys is a factor of its logits; that of values one of the page's weights, relative to the chunk's largest scale.
// Sums of a chunk are added up outside the tensor cores, in fp32.
//
// One block a multiprocessor, its warps apart: one brings pages (a ring of SLOTS chunks of keys or values), one issues products, one prepares the queries of the next unit, four weigh: a
// thread a key for the logits and weights, a thread a channel for the sums.  Workers, here blocks, and their records are those of decode_q4.cuh.
#ifndef VECTOR_DECODE_Q8_TC_CUH_
#define VECTOR_DECODE_Q8_TC_CUH_

#include "decode_q4.cuh"

namespace vec {
namespace dq8 {
using namespace dq4;

// Largest weights lie in (2^LEAD8, 2^(LEAD8 + SLACK8)], below e4m3's 448.
constexpr float LEAD8 = 6.f, SLACK8 = 2.f, PART8 = 32.f;
constexpr int PAGES = 4, KEYS = PAGES * q8::ROWS, CHANNELS = 128;
using TcCost = Costs<2, 1>;

// G: heads, rounded up to four or eight.
template <typename T, bool EXACT, int G> struct TcCfg {
    static constexpr int QP = sizeof(T) == 2 ? 3 : 5, PP = EXACT ? 5 : 4;
    static constexpr int N1 = (QP * G + 15) / 16 * 16, N2 = (PP * G + 15) / 16 * 16;      // columns of the two products
    static constexpr int SLOTS = 11, SLOT_BYTES = KEYS * CHANNELS, Q_BYTES = N1 * CHANNELS, P_BYTES = N2 * KEYS;
    static constexpr int Q_AT = SLOTS * SLOT_BYTES, P_AT = Q_AT + 2 * Q_BYTES, TRAIL_AT = P_AT + 2 * P_BYTES, PREFIX_AT = TRAIL_AT + SLOTS * PAGES * 32;
    static constexpr int THREADS = 256, WEIGHERS = 128;
    static constexpr uint32_t S_COL = 0, O_COL = 128, TMEM = 256;                          // two buffers each, 64 columns apart
    static constexpr size_t smem(int batch) { return 1024 + PREFIX_AT + (size_t)(batch + 1) * 8; }      // the slots begin at a multiple of 1024 bytes
};

// Channels 0 .. 63 and 64 .. 127 of all tiles of a pool, [tile][row pair][row][64]: the halves of odd rows lie the other way round.
struct TcMaps { CUtensorMap ret[2], apx[2]; };

struct Chunk { int unit, kind, pages, edge, rows[PAGES]; };               // kind: as in Entry, of keys; -1: no more
enum { END = -1 };

template <int N> __device__ __forceinline__ void load_columns(uint32_t at, float (&x)[N]) {
    static_assert(N == 16 || N == 32 || N == 48, "columns of a product");
    if constexpr (N >= 32) {
        uint32_t r[32];
        tc::tmem_ld32(at, r);
        if constexpr (N == 48) {
            uint32_t q[16];
            tc::tmem_ld16(at + 32, q);
            tc::tmem_ld_wait(r);
            tc::tmem_ld_wait16(q);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[32 + i] = __uint_as_float(q[i]);
        } else {
            tc::tmem_ld_wait(r);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
    } else {
        uint32_t r[16];
        tc::tmem_ld16(at, r);
        tc::tmem_ld_wait16(r);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
    }
}
// The sums of head h's parts, which lie G columns apart.
template <int PARTS, int G, int N> __device__ __forceinline__ float joined(const float (&x)[N], int h) {
    float s = x[(PARTS - 1) * G + h];
#pragma unroll
    for (int i = PARTS - 2; i >= 0; --i) s = fmaf(s, 1.f / PART8, x[i * G + h]);
    return s;
}

template <typename T, bool EXACT, int G>
__global__ void __launch_bounds__(TcCfg<T, EXACT, G>::THREADS, 1)
decode_q8_stream_tc(const __grid_constant__ TcMaps maps, const T* q, Cache c, int g, float scale_log2e, unsigned char* ws, int* fault) {
    using C = TcCfg<T, EXACT, G>;
    constexpr int D = CHANNELS, ROWS = q8::ROWS, TILE = q8::Row<D>::TILE, SLOTS = C::SLOTS;
    extern __shared__ unsigned char raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) uint64_t full[SLOTS], empty[SLOTS], s_full[2], p_full[2], o_full[2], q_full[2], q_empty[2], meet;
    __shared__ Chunk chunks[SLOTS];
    __shared__ int64_t sums[C::THREADS / 32];
    __shared__ float fac_of[2][G], most[4][G], total[4][G];
    __shared__ int votes[2][4];
    __shared__ uint32_t tmem_at;
    int64_t* prefix = reinterpret_cast<int64_t*>(smem + C::PREFIX_AT);
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        // a slot is free when its product is done and the four weighing warps have read its scales
        for (int s = 0; s < SLOTS; ++s) { tma::mbar_init(&full[s], 1); tma::mbar_init(&empty[s], 5); }
        for (int i = 0; i < 2; ++i) {
            tma::mbar_init(&s_full[i], 1); tma::mbar_init(&p_full[i], C::WEIGHERS); tma::mbar_init(&o_full[i], 1);
            tma::mbar_init(&q_full[i], 1); tma::mbar_init(&q_empty[i], 5);
        }
        tma::mbar_init(&meet, 4);
        tma::mbar_fence_init();
    }
    for (int i = threadIdx.x; i < 2 * C::Q_BYTES / 16; i += C::THREADS) reinterpret_cast<uint4*>(smem + C::Q_AT)[i] = make_uint4(0, 0, 0, 0);      // rows of no part and no head stay so
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    // ---- costs of the sequences, summed up
    int64_t carry = 0;
    for (int b0 = 0; b0 < c.batch; b0 += C::THREADS) {
        const int b = b0 + threadIdx.x;
        int64_t x = 0;
        if (b < c.batch)
            x = (int64_t)c.LH * ((int64_t)TcCost::ret * tiles_of<Bits8>(rows_of<Bits8>(c.ret_len, b, c.ret_width)) + (int64_t)TcCost::apx * tiles_of<Bits8>(rows_of<Bits8>(c.apx_len, b, c.apx_width)));
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
        for (int w = 0; w < C::THREADS / 32; ++w) { all += sums[w]; if (w < wid) before += sums[w]; }
        if (b < c.batch) prefix[b] = before + s - x;
        carry = all;
        __syncthreads();
    }
    if (threadIdx.x == 0) prefix[c.batch] = carry;
    __syncthreads();
    const Deal deal(carry, gridDim.x, TcCost::most);
    const int worker = blockIdx.x;
    if (carry == 0 || worker >= deal.workers) return;
    if (wid == 0) { tc::tmem_alloc(&tmem_at, C::TMEM); tc::tmem_relinquish(); }
    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");       // the cleared queries
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = tmem_at;
    // The next slot of the ring and how often it has been used: every warp goes through the ring in the same order.
    struct Ring { int s = 0, use = 0; __device__ __forceinline__ void next() { if (++s == SLOTS) { s = 0; ++use; } } };

    if (wid == 4) {
        // ---- pages on their way
        const uint64_t policy = tma::policy_evict_first();
        Runs<Bits8, TcCost> run;
        run.find(c, prefix, deal.begin(worker), deal.begin(worker + 1));
        Ring ring;
        bool ok = true;
        auto take = [&] { return ok = ok && (ring.use == 0 || tma::mbar_wait_warp(&empty[ring.s], (ring.use - 1) & 1, fault, 41)); };
        for (; ok && run.count > 0; run.next(c, prefix)) {
            int page = -1;
            for (int k = 0; ok && k < run.count; k += PAGES) {
                if ((k & 31) == 0 && k + lane < run.count)
                    page = run.apx ? c.apx_table[(size_t)run.b * c.apx_width + run.p + k + lane] : c.ret_table[(size_t)run.b * c.ret_width + run.p + k + lane];
                const int at = __shfl_sync(0xffffffffu, page, (k & 31) + (lane & 3)), n = min(run.count - k, PAGES), p = run.p + k;
                const bool there = lane < n && at >= 0 && at < (run.apx ? c.n_apx_pages : c.n_ret_pages);
                const int bytes = __popc(__ballot_sync(0xffffffffu, there)) * (ROWS * D + 32);
                for (int values = 0; values < (run.apx ? 1 : 2); ++values) {
                    if (!take()) break;
                    const int s = ring.s;
                    if (lane < PAGES) chunks[s].rows[lane] = there ? min((run.apx ? run.n_apx : run.n_ret) - (p + lane) * ROWS, ROWS) : 0;
                    if (lane == 0) {
                        chunks[s].unit = run.b * c.LH + run.lh;
                        chunks[s].kind = run.apx ? KEY_ONLY : dq4::KEYS;
                        chunks[s].pages = n;
                        chunks[s].edge = (p == 0 && (!run.apx || run.n_ret == 0) ? 1 : 0) |
                                         (run.apx ? (p + n) * ROWS >= run.n_apx : run.n_apx == 0 && (p + n) * ROWS >= run.n_ret ? 1 : 0) << 1;
                    }
                    __syncwarp();
                    if (lane == 0) {
                        if (bytes) tma::mbar_expect_tx(&full[s], bytes);
                        else tma::mbar_arrive(&full[s]);
                    }
                    __syncwarp();
                    if (there) {
                        const size_t tile = ((size_t)at * c.LH + run.lh) * (run.apx ? 1 : 2) + values;
                        const CUtensorMap* map = run.apx ? maps.apx : maps.ret;
                        unsigned char* to = smem + s * C::SLOT_BYTES + lane * (ROWS * 64);
                        tma::load_4d_hint(to, &map[0], 0, 0, 0, (int)tile, &full[s], policy);
                        tma::load_4d_hint(to + KEYS * 64, &map[1], 0, 0, 0, (int)tile, &full[s], policy);
                        tma::load_bulk_hint(smem + C::TRAIL_AT + (s * PAGES + lane) * 32, (run.apx ? c.apx : c.ret) + tile * TILE + ROWS * D, 32, &full[s], policy);
                    }
                    ring.next();
                }
            }
        }
        if (take()) {
            if (lane == 0) { chunks[ring.s].kind = END; tma::mbar_arrive(&full[ring.s]); }
        } else {
            // a wait gave up: copies in flight still land in this block's memory
            for (int i = 0; i < SLOTS; ++i) {
                if (ring.s == 0) { if (ring.use == 0) break; ring.s = SLOTS; --ring.use; }
                --ring.s;
                tma::mbar_wait_warp(&full[ring.s], ring.use & 1, fault, 42);
            }
        }
    } else if (wid == 5) {
        // ---- products
        if (lane == 0) {
            constexpr uint32_t to_keys = tc::instr_desc_f8(KEYS, C::N1, false, false), to_channels = tc::instr_desc_f8(D, C::N2, true, true);
            Ring ring;
            int unit = -1, units = 0, prev_slot = -1, prev_use = 0, prev_pages = 0;
            for (int i = 0;; ++i) {
                if (!tma::mbar_wait(&full[ring.s], ring.use & 1, fault, 43)) break;
                const int kind = chunks[ring.s].kind, pages = chunks[ring.s].pages, keys = ring.s;
                int slot = ring.s, use = ring.use;
                if (kind != END) {
                    if (kind == dq4::KEYS) { ring.next(); slot = ring.s; use = ring.use; }
                    ring.next();
                    if (chunks[keys].unit != unit) {
                        if (unit >= 0) tc::mma_commit(&q_empty[(units - 1) & 1]);
                        unit = chunks[keys].unit;
                        if (!tma::mbar_wait(&q_full[units & 1], (units >> 1) & 1, fault, 44)) break;
                        ++units;
                    }
                    const uint32_t a = tma::smem_u32(smem + keys * C::SLOT_BYTES), b = tma::smem_u32(smem + C::Q_AT + ((units - 1) & 1) * C::Q_BYTES);
#pragma unroll
                    for (int st = 0; st < D / 32; ++st)
                        tc::mma_f8(tmem + C::S_COL + 64 * (i & 1), tc::smem_desc(a + st / 2 * (KEYS * 64) + st % 2 * 32, tc::BYTES64, 512), tc::smem_desc(b + 32 * st, tc::BYTES128, 1024), to_keys, st > 0);
                    tc::mma_commit(&s_full[i & 1]);
                    if (slot != keys) tc::mma_commit(&empty[keys]);
                }
                if (prev_slot >= 0) {
                    const int buf = (i - 1) & 1;
                    if (!tma::mbar_wait(&p_full[buf], ((i - 1) >> 1) & 1, fault, 45) || !tma::mbar_wait(&full[prev_slot], prev_use & 1, fault, 46)) break;
                    tc::fence_after_sync();
                    const uint32_t a = tma::smem_u32(smem + prev_slot * C::SLOT_BYTES), b = tma::smem_u32(smem + C::P_AT + buf * C::P_BYTES);
                    for (int p = 0; p < prev_pages; ++p)
                        tc::mma_f8(tmem + C::O_COL + 64 * buf, tc::smem_desc(a + p * (ROWS * 64), tc::BYTES64, 512, KEYS * 64), tc::smem_desc(b + p * (ROWS * 16), tc::NONE, KEYS * 16, 128), to_channels,
                                   p > 0);
                    tc::mma_commit(&o_full[buf]);
                    tc::mma_commit(&empty[prev_slot]);
                }
                if (kind == END) break;
                prev_slot = slot; prev_use = use; prev_pages = pages;
            }
        }
        __syncwarp();
    } else if (wid == 6) {
        // ---- queries of the units to come: a lane has four channels of every head
        Runs<Bits8, TcCost> run;
        run.find(c, prefix, deal.begin(worker), deal.begin(worker + 1));
        int unit = -1, units = 0;
        for (; run.count > 0; run.next(c, prefix)) {
            if (run.b * c.LH + run.lh == unit) continue;
            unit = run.b * c.LH + run.lh;
            const int buf = units & 1;
            float x[G][4];
#pragma unroll
            for (int h = 0; h < G; ++h) {
                const T* row = q + ((size_t)unit * g + min(h, g - 1)) * D + 4 * lane;
                if constexpr (sizeof(T) == 4) {
                    const float4 v = *reinterpret_cast<const float4*>(row);
                    x[h][0] = v.x; x[h][1] = v.y; x[h][2] = v.z; x[h][3] = v.w;
                } else {
                    const uint2 v = *reinterpret_cast<const uint2*>(row);
                    x[h][0] = __uint_as_float(v.x << 16); x[h][1] = __uint_as_float(v.x & 0xffff0000u); x[h][2] = __uint_as_float(v.y << 16); x[h][3] = __uint_as_float(v.y & 0xffff0000u);
                }
            }
            if (units >= 2 && !tma::mbar_wait_warp(&q_empty[buf], ((units >> 1) - 1) & 1, fault, 47)) break;
            ++units;
#pragma unroll
            for (int h = 0; h < G; ++h) {
                if (h >= g) break;
                float top = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (!(fabsf(x[h][i]) <= 3.4028235e38f)) x[h][i] = __int_as_float(0x7fffffff);      // an infinite query's logits are none
                    top = fmaxf(top, fabsf(x[h][i]));
                }
                top = warp_max(top);
                const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -100), 127);             // the largest channel lies in [2^7, 2^8)
                const float up = __uint_as_float((uint32_t)(127 + 7 - e) << 23);
                if (lane == 0) fac_of[buf][h] = fmaxf(scale_log2e * __uint_as_float((uint32_t)(127 - 7 + e) << 23), 1.2e-38f);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[h][i] *= up;
#pragma unroll
                for (int p = 0; p < C::QP; ++p) {
                    const int row = p * G + h;
                    const uint32_t code = q8::to_codes(x[h][0], x[h][1], x[h][2], x[h][3]);
                    *reinterpret_cast<uint32_t*>(smem + C::Q_AT + buf * C::Q_BYTES + row * D + ((lane / 4) ^ (row & 7)) * 16 + lane % 4 * 4) = code;
                    float y[4];
                    q8::decode_word(code, y);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[h][i] = (x[h][i] - y[i]) * PART8;
                }
            }
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            __syncwarp();
            if (lane == 0) tma::mbar_arrive(&q_full[buf]);
        }
    } else if (wid < 4) {
        // ---- weights and sums
        const int rec = 2 * tier_floats(g, D), heads = even_heads(g), n_units = c.batch * c.LH;
        int2* ends = reinterpret_cast<int2*>(ws);
        float* records = reinterpret_cast<float*>(ws + ends_bytes(n_units));
        const uint32_t my_lanes = (uint32_t)wid << 21;                    // of tensor memory: keys or channels 32 wid + lane
        float fac[G], m[G], L[G], O[G];
        auto clear = [&] {
#pragma unroll
            for (int h = 0; h < G; ++h) { m[h] = -INFINITY; L[h] = 0.f; O[h] = 0.f; }
        };
        clear();
#pragma unroll
        for (int h = 0; h < G; ++h) fac[h] = 1.2e-38f;
        int met = 0;
        // The four warps meet; bounded, as every wait here.
        auto meeting = [&] {
            __syncwarp();
            if (lane == 0) tma::mbar_arrive(&meet);
            return tma::mbar_wait_warp(&meet, met++ & 1, fault, 48);
        };
        // The sums of the chunk before, which are on their way: chunk `i`, whose values were weighed relative to 2^held.
        bool pending = false;
        float held = 1.f;
        auto drain = [&](int i) {
            if (!pending) return true;
            pending = false;
            if (!tma::mbar_wait_warp(&o_full[i & 1], (i >> 1) & 1, fault, 49)) return false;
            tc::fence_after_sync();
            float x[C::N2];
            load_columns(tmem + my_lanes + C::O_COL + 64 * (i & 1), x);
#pragma unroll
            for (int h = 0; h < G; ++h) O[h] = fmaf(joined<C::PP, G>(x, h), held, O[h]);
            tc::fence_before_sync();
            return true;
        };
        int unit = -1, apx = 0, wrote = 0, slot_rec = 0, units = 0;
        // The state of a tier to its record, in the order in which the merge reads it; an empty one's sums are not read.
        auto put_tier = [&](int tier, bool none) {
            float* p = records + (size_t)slot_rec * rec + tier * tier_floats(g, D);
            if (!none) {
#pragma unroll
                for (int h = 0; h < G; ++h) {
                    const float s = warp_sum(L[h]);
                    if (lane == 0) total[wid][h] = s;
                }
                if (!meeting()) return false;
            }
            if (threadIdx.x < heads) {
                float ref = -INFINITY, sum = 0.f;
                if (!none) {
#pragma unroll
                    for (int h = 0; h < G; ++h)
                        if (h == (int)threadIdx.x) { ref = m[h]; sum = (total[0][h] + total[1][h]) + (total[2][h] + total[3][h]); }
                }
                *reinterpret_cast<float2*>(p + 2 * threadIdx.x) = make_float2(ref, sum);
            }
            if (none) return true;
            const int ch = threadIdx.x, k = ch / 64 * 16 + ch % 16, row = ch % 64 / 16 * 2 + (k & 1), t = k / 4, pair = k >> 1 & 1;      // as q4::Row<128>::channel_of
#pragma unroll
            for (int hp = 0; hp < G / 2; ++hp)
                if (2 * hp < heads) *reinterpret_cast<float2*>(p + 2 * heads + ((t * (heads / 2) + hp) * 8 + row) * 4 + 2 * pair) = make_float2(O[2 * hp], O[2 * hp + 1]);
            return meeting();                                             // the totals are free again
        };
        auto leave_unit = [&] {
            if (unit < 0) return true;
            if (!put_tier(apx, false)) return false;
            wrote |= 1 << apx;
            return ((wrote & 1) || put_tier(0, true)) && ((wrote & 2) || put_tier(1, true));
        };
        Ring ring;
        for (int i = 0;; ++i) {
            if (!tma::mbar_wait_warp(&full[ring.s], ring.use & 1, fault, 50)) break;
            const Chunk& chunk = chunks[ring.s];
            const int kind = chunk.kind;
            if (kind == END) {
                if (drain(i - 1)) leave_unit();
                break;
            }
            const int tier = kind == KEY_ONLY, chunk_unit = chunk.unit, pages = chunk.pages, edge = chunk.edge, rows = wid < pages ? chunk.rows[wid] : 0, keys = ring.s;
            const unsigned char* trail = smem + C::TRAIL_AT + keys * PAGES * 32;
            const int e_keys = rows > 0 ? q8::exponent_of(trail + wid * 32, 0) : 0;
            int top_e = q8::LOW;                                          // of the pages that are weighed: the chunk's largest
            if (tier) {
#pragma unroll
                for (int p = 0; p < PAGES; ++p)
                    if (p < pages && chunk.rows[p] > 0) top_e = max(top_e, q8::exponent_of(trail + p * 32, 0));
            }
            __syncwarp();
            if (lane == 0) tma::mbar_arrive(&empty[keys]);                // the chunk's entry and scales have been read; the tensor cores hold the slot as long as they need it
            if (chunk_unit != unit || tier != apx) {
                if (!drain(i - 1)) break;
                if (chunk_unit != unit) {
                    if (!leave_unit()) break;
                    unit = chunk_unit; wrote = 0;
                    slot_rec = edge & 1 ? unit : n_units + worker;
                    if (!tma::mbar_wait_warp(&q_full[units & 1], (units >> 1) & 1, fault, 51)) break;
#pragma unroll
                    for (int h = 0; h < G; ++h)
                        if (h < g) fac[h] = fac_of[units & 1][h];
                    __syncwarp();
                    if (lane == 0) tma::mbar_arrive(&q_empty[units & 1]);
                    ++units;
                } else {
                    if (!put_tier(apx, false)) break;
                    wrote |= 1 << apx;
                }
                apx = tier;
                clear();
            }
            if (threadIdx.x == 0) {
                if (edge & 1) ends[unit].x = worker;
                if (edge & 2) ends[unit].y = worker;
            }
            // ---- logits of a key
            if (!tma::mbar_wait_warp(&s_full[i & 1], (i >> 1) & 1, fault, 52)) break;
            tc::fence_after_sync();
            float x[G];
            {
                float s[C::N1];
                load_columns(tmem + my_lanes + C::S_COL + 64 * (i & 1), s);
#pragma unroll
                for (int h = 0; h < G; ++h) x[h] = joined<C::QP, G>(s, h);
            }
            const bool there = lane < rows;
            const float of_page = q8::power(e_keys);
            bool beyond = false;
#pragma unroll
            for (int h = 0; h < G; ++h) {
                x[h] *= fminf(fmaxf(fac[h] * of_page, 1.2e-38f), 3.4e38f);
                beyond |= there && x[h] > m[h] + (LEAD8 + SLACK8);
            }
            const int any = __any_sync(0xffffffffu, beyond);
            if (lane == 0) votes[i & 1][wid] = any;
            if (!meeting()) break;
            if (votes[i & 1][0] | votes[i & 1][1] | votes[i & 1][2] | votes[i & 1][3]) {      // the references follow the largest logits
#pragma unroll
                for (int h = 0; h < G; ++h) {
                    const float t = warp_max(there ? x[h] : -INFINITY);
                    if (lane == 0) most[wid][h] = t;
                }
                if (!drain(i - 1) || !meeting()) break;
#pragma unroll
                for (int h = 0; h < G; ++h) {
                    const float t = fmaxf(fmaxf(most[0][h], most[1][h]), fmaxf(most[2][h], most[3][h]));
                    const float now = fmaxf(m[h], t * (t > 0.f ? 1.f - 0x1p-23f : 1.f + 0x1p-23f) - LEAD8), f = m[h] == now ? 1.f : tc::ex2(m[h] - now);      // see reference()
                    m[h] = now;
                    O[h] *= f; L[h] *= f;
                }
            }
            // ---- weights
            ring.next();
            int slot = keys;
            int e_page = e_keys;
            if (!tier) {
                slot = ring.s;
                if (!tma::mbar_wait_warp(&full[slot], ring.use & 1, fault, 53)) break;
                ring.next();
                const unsigned char* values = smem + C::TRAIL_AT + slot * PAGES * 32;
                e_page = rows > 0 ? q8::exponent_of(values + wid * 32, 0) : 0;
#pragma unroll
                for (int p = 0; p < PAGES; ++p)
                    if (p < pages && chunks[slot].rows[p] > 0) top_e = max(top_e, q8::exponent_of(values + p * 32, 0));
                __syncwarp();
                if (lane == 0) tma::mbar_arrive(&empty[slot]);
            }
            const float relative = q8::power(rows > 0 ? e_page - top_e : 0);
            uint32_t w[C::N2 / 4];
#pragma unroll
            for (int h = 0; h < G; ++h) {
                const float weight = there ? tc::ex2(x[h] - m[h]) : 0.f;
                L[h] += weight;
                x[h] = weight * relative;
            }
#pragma unroll
            for (int p = 0; p < C::N2 / G; ++p)
#pragma unroll
                for (int h = 0; h < G; h += 4) {
                    uint32_t& code = w[(p * G + h) / 4];
                    code = 0;
                    if (p >= C::PP) continue;
                    code = q8::to_codes(x[h], x[h + 1], x[h + 2], x[h + 3]);
                    if (p + 1 == C::PP) continue;
                    float y[4];
                    q8::decode_word(code, y);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[h + j] = (x[h + j] - y[j]) * PART8;
                }
            unsigned char* to = smem + C::P_AT + (i & 1) * C::P_BYTES + threadIdx.x * 16;
#pragma unroll
            for (int j = 0; j < C::N2 / 16; ++j) *reinterpret_cast<uint4*>(to + j * (KEYS * 16)) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
            // what lies behind a page's last row may be no number
            if (wid < pages && rows < ROWS)
                for (int j = rows * 4 + lane; j < ROWS * 4; j += 32)
#pragma unroll
                    for (int half = 0; half < 2; ++half) reinterpret_cast<uint4*>(smem + slot * C::SLOT_BYTES + half * (KEYS * 64) + wid * (ROWS * 64))[j] = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            tc::fence_before_sync();
            tma::mbar_arrive(&p_full[i & 1]);
            if (!drain(i - 1)) break;
            pending = true;
            held = q8::power(top_e);
        }
    }
    tc::fence_before_sync();
    __syncthreads();
    if (wid == 0) tc::tmem_dealloc(tmem, C::TMEM);
}

}  // namespace dq8
}  // namespace vec
#endif
