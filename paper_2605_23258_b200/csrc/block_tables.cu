// Page tables, lengths and slots of a batch of requests after some grew, shrank or ended (vector_block_tables), from nothing but the
// requests' lengths and changes.  Everything is a prefix sum over the requests: pages released (pushed on the stack of free pages in the
// requests' order), pages wanted (popped in that order) and rows added.  So no answer depends on the order in which threads run.
//
// What bounds a step of a batch is latency: one block does all of it, a thread a request.  Where prompts are admitted there are many pages and
// slots to write: blocks on all multiprocessors, each of which sums up the requests for itself and takes a part of the pages and slots; a page that a
// request releases and another one takes in the same call is looked up where it was, so that no block waits for another one.  720000 slots
// and 15000 pages of 512 requests: 12 us, with one block for the pages and a second kernel for the slots 22.  More than 1024 requests: one block moves the pages, a second kernel writes the slots.
#include "common.cuh"
#include "internal.h"

namespace vec {
namespace bt {

constexpr int THREADS = 1024, SLOT_THREADS = 256, SLOTS_PER_WARP = 128;
constexpr int BLOCK_SLOTS = THREADS;            // slots that a block of block_tables_batch is there for, while there are multiprocessors

struct Args {
    const int32_t *lengths, *added;
    int32_t *new_lengths, *table, *stack, *new_n_free, *first_row, *row_start, *slots;
    const int32_t* n_free;
    int64_t n_slots;
    int32_t batch, page_rows, width, cap_free;
};

// A request's change in pages; rows: after the change, if there are pages enough.  width * page_rows is below 2^31.
struct Change { int64_t old_rows, rows; int have, want; };
__device__ __forceinline__ Change change_of(const Args& a, int b) {
    Change c;
    const int64_t most = (int64_t)a.width * a.page_rows;
    c.old_rows = min((int64_t)max(a.lengths[b], 0), most);
    c.rows = max(c.old_rows + a.added[b], (int64_t)0);
    c.have = (int)(((uint32_t)c.old_rows + (uint32_t)a.page_rows - 1) / (uint32_t)a.page_rows);
    c.want = (int)(((uint32_t)min(c.rows, most) + (uint32_t)a.page_rows - 1) / (uint32_t)a.page_rows);
    return c;
}

// Sum of x over the threads before this one; `total` over all.  All threads of the block.
__device__ __forceinline__ int64_t scan(int64_t x, int64_t* warps, int64_t& total) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    int64_t s = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
    }
    __syncthreads();                                             // the sums of the scan before have been read
    if (lane == 31) warps[wid] = s;
    __syncthreads();
    int64_t w = warps[lane];                                     // THREADS / 32 = 32 warps
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
    }
    total = __shfl_sync(0xffffffffu, w, 31);
    const int64_t before = __shfl_sync(0xffffffffu, w, max(wid - 1, 0));
    return s - x + (wid ? before : 0);
}

// A sum as a start: what is beyond 2^31 - 1 stays there, behind every slot and page that there can be.
__device__ __forceinline__ int32_t start_of(int64_t sum) { return (int32_t)min(sum, (int64_t)0x7fffffff); }

// The request that row k of the added rows belongs to: the last b in [lo, hi) with start[b] <= k.
__device__ __forceinline__ int request_of(const int32_t* start, int lo, int hi, int64_t k) {
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= k) lo = mid;
        else hi = mid;
    }
    return lo;
}
// Slot of row `row` in page `page`, -1 where that is none.
__device__ __forceinline__ int32_t slot_of(int64_t page, int64_t row, int32_t page_rows) {
    const int64_t slot = page * page_rows + (int64_t)((uint32_t)row % (uint32_t)page_rows);
    return page < 0 || slot > 0x7fffffffLL ? -1 : (int32_t)slot;
}
__device__ __forceinline__ int32_t slot_of_row(const Args& a, int b, int64_t row, int64_t rows) {
    if (row >= rows) return -1;                                  // no page was left for it
    return slot_of(a.table[(size_t)b * a.width + (uint32_t)row / (uint32_t)a.page_rows], row, a.page_rows);
}

// Moves pages between the tables' rows and the stack, one page a thread and step, MOVES steps' loads in flight: page e of `total`, which is the
// i-th of request b0 + k (starts[k] <= e, i = e - starts[k]), lies at entry first[k] + i of the request's row.  f(entry, e).
template <typename Load, typename Store>
__device__ __forceinline__ void move_pages(const Args& a, int b0, int n, int total, const int32_t* starts, const int32_t* first, Load load, Store store) {
    constexpr int MOVES = 4;
    for (int e0 = threadIdx.x; e0 < total; e0 += MOVES * THREADS) {
        int32_t v[MOVES];
        int32_t* entry[MOVES];
#pragma unroll
        for (int j = 0; j < MOVES; ++j) {
            const int e = e0 + j * THREADS;
            if (e < total) {
                const int k = request_of(starts, 0, n, e);
                entry[j] = a.table + (size_t)(b0 + k) * a.width + first[k] + (e - starts[k]);
                v[j] = load(entry[j], e);
            }
        }
#pragma unroll
        for (int j = 0; j < MOVES; ++j)
            if (e0 + j * THREADS < total) store(entry[j], e0 + j * THREADS, v[j]);
    }
}

__global__ void __launch_bounds__(THREADS)
block_tables_plan(Args a) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    __shared__ int64_t warps[32];
    __shared__ int32_t starts[THREADS], first[THREADS];
    const int t = threadIdx.x;
    int64_t height = min(max((int64_t)a.n_free[0], (int64_t)0), (int64_t)a.cap_free);

    // ---- released pages go on the stack, a request's in the order of its table
    int64_t total = 0;
    for (int b0 = 0; b0 < a.batch; b0 += THREADS) {
        const int b = b0 + t, n = min(a.batch - b0, THREADS);
        Change c = {};
        if (b < a.batch) c = change_of(a, b);
        const int back = max(c.have - c.want, 0);
        if (!__syncthreads_or(back > 0)) continue;
        starts[t] = start_of(scan(back, warps, total));
        first[t] = c.want;
        __syncthreads();
        move_pages(a, b0, n, (int)min(total, (int64_t)a.cap_free - height), starts, first, [&](const int32_t* entry, int) { return *entry; },
                   [&](int32_t*, int e, int32_t v) { a.stack[height + e] = v; });
        height = min(height + total, (int64_t)a.cap_free);
        __syncthreads();
    }
    // ---- wanted pages come off it, as far as they go; lengths and the rows' starts
    int64_t needed = 0, added = 0;
    for (int b0 = 0; b0 < a.batch; b0 += THREADS) {
        const int b = b0 + t, n = min(a.batch - b0, THREADS);
        Change c = {};
        int grow = 0;
        if (b < a.batch) { c = change_of(a, b); grow = a.added[b]; }
        const int need = max(c.want - c.have, 0);
        const int64_t start = added + scan(max(grow, 0), warps, total);
        added += total;
        int64_t before = needed;
        if (__syncthreads_or(need > 0)) {
            const int64_t mine = scan(need, warps, total);
            before += mine;
            starts[t] = start_of(mine);
            first[t] = c.have;
            __syncthreads();
            const int64_t top = height - 1 - needed;
            move_pages(a, b0, n, (int)max(min(total, top + 1), (int64_t)0), starts, first, [&](const int32_t*, int e) { return a.stack[top - e]; },
                       [&](int32_t* entry, int, int32_t v) { *entry = v; });
            needed += total;
            __syncthreads();
        }
        if (b < a.batch) {
            const int got = (int)min((int64_t)need, max(height - before, (int64_t)0));
            const int32_t s = start_of(start), rows = (int32_t)(grow > 0 ? min(c.rows, (int64_t)(c.have + got) * a.page_rows) : c.rows);
            a.first_row[b] = (int32_t)c.old_rows;
            a.row_start[b] = s;
            a.new_lengths[b] = rows;
        }
    }
    if (t == 0) {
        a.row_start[a.batch] = start_of(added);
        a.new_n_free[0] = (int32_t)(height - min(needed, height));
    }
}

// At most THREADS requests, a thread a request in every block.  Blocks take parts of the pages and slots; `small` outputs, one number a request, are
// written by the first block, in a launch of their own (parts = 0) where other blocks may still read what they overwrite.
__global__ void __launch_bounds__(THREADS)
block_tables_batch(Args a, int parts, int small) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    __shared__ int64_t warps[32];
    __shared__ int32_t row_start[THREADS], need_start[THREADS], back_start[THREADS], olds[THREADS], news[THREADS], haves[THREADS], wants[THREADS];
    const int t = threadIdx.x;
    const int64_t n_free = min(max((int64_t)a.n_free[0], (int64_t)0), (int64_t)a.cap_free);
    Change c = {};
    int grow = 0;
    if (t < a.batch) { c = change_of(a, t); grow = a.added[t]; }
    const int back = max(c.have - c.want, 0), need = max(c.want - c.have, 0);
    int64_t total, backs = 0, before_back = 0;
    int64_t rows, needs, start, before;
    if (!__syncthreads_or(grow >= 1 << 21 || need >= 1 << 21)) {      // rows and pages wanted in one sum: THREADS of them stay below 2^31
        const int64_t both = scan(((int64_t)max(grow, 0) << 32) | (uint32_t)need, warps, total);
        rows = total >> 32; needs = (int64_t)(uint32_t)total; start = both >> 32; before = (int64_t)(uint32_t)both;
    } else {
        start = scan(max(grow, 0), warps, rows);
        before = scan(need, warps, needs);
    }
    if (__syncthreads_or(back > 0)) before_back = scan(back, warps, backs);
    const int64_t height = min(n_free + backs, (int64_t)a.cap_free), pops = min(needs, height), pushes = height - n_free;
    const int got = (int)min((int64_t)need, max(height - before, (int64_t)0));
    const int32_t now = (int32_t)(grow > 0 ? min(c.rows, (int64_t)(c.have + got) * a.page_rows) : c.rows);
    if (small && blockIdx.x == 0) {
        if (t < a.batch) {
            a.first_row[t] = (int32_t)c.old_rows;
            a.row_start[t] = start_of(start);
            a.new_lengths[t] = now;
        }
        if (t == 0) {
            a.row_start[a.batch] = start_of(rows);
            a.new_n_free[0] = (int32_t)(height - pops);
        }
    }
    if (!parts) return;
    row_start[t] = start_of(start); need_start[t] = start_of(before); back_start[t] = start_of(before_back);
    olds[t] = (int32_t)c.old_rows; news[t] = now; haves[t] = c.have; wants[t] = c.want;
    __syncthreads();
    auto released = [&](int64_t e) {                             // the e-th released page
        const int k = request_of(back_start, 0, a.batch, e);
        return a.table[(size_t)k * a.width + wants[k] + (e - back_start[k])];
    };
    auto taken = [&](int64_t e) {                                // the e-th page that is taken from the stack
        const int64_t at = height - 1 - e;
        return at >= n_free ? released(at - n_free) : a.stack[at];
    };
    // few pages and few slots are different warps' work
    const int64_t i0 = (int64_t)blockIdx.x * THREADS + t, step = (int64_t)gridDim.x * THREADS, i1 = step - 1 - i0;
    for (int64_t e = i1; e < pops; e += step) {
        const int k = request_of(need_start, 0, a.batch, e);
        a.table[(size_t)k * a.width + haves[k] + (e - need_start[k])] = taken(e);
    }
    for (int64_t e = i1; e < pushes; e += step) a.stack[n_free + e] = released(e);
    if (a.n_slots <= step) {                                     // a slot a thread
        if (i0 >= a.n_slots) return;
        int32_t slot = -1;
        if (i0 < rows) {
            const int b = request_of(row_start, 0, a.batch, i0);
            const int64_t row = olds[b] + (i0 - row_start[b]);
            if (row < news[b]) {                                 // else no page was left for it
                const int64_t j = (uint32_t)row / (uint32_t)a.page_rows;
                slot = slot_of(j < haves[b] ? a.table[(size_t)b * a.width + j] : taken(need_start[b] + (j - haves[b])), row, a.page_rows);
            }
        }
        a.slots[i0] = slot;
        return;
    }
    const bool wide = ((uintptr_t)a.slots & 15) == 0;
    for (int64_t k0 = 4 * i0; k0 < a.n_slots; k0 += 4 * step) {
        int32_t slot[4] = {-1, -1, -1, -1};
        if (k0 < rows) {
            int b = request_of(row_start, 0, a.batch, k0);
            int32_t page = -1;
            int64_t index = -1;                                  // of the page at hand within its request
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t k = k0 + i;
                if (k >= rows) break;
                if (b + 1 < a.batch && row_start[b + 1] <= k) { b = request_of(row_start, b + 1, a.batch, k); index = -1; }
                const int64_t row = olds[b] + (k - row_start[b]);
                if (row >= news[b]) continue;
                const int64_t j = (uint32_t)row / (uint32_t)a.page_rows;
                if (j != index) { page = j < haves[b] ? a.table[(size_t)b * a.width + j] : taken(need_start[b] + (j - haves[b])); index = j; }
                slot[i] = slot_of(page, row, a.page_rows);
            }
        }
        if (wide && k0 + 4 <= a.n_slots) {
            *reinterpret_cast<int4*>(a.slots + k0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k0 + i < a.n_slots) a.slots[k0 + i] = slot[i];
        }
    }
}

// The slots of all added rows, SLOTS_PER_WARP neighbours a warp, four a lane; -1 behind the last.
__global__ void __launch_bounds__(SLOT_THREADS)
block_tables_slots(Args a) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    const int lane = threadIdx.x & 31;
    const int64_t k0 = ((int64_t)blockIdx.x * (SLOT_THREADS / 32) + (threadIdx.x >> 5)) * SLOTS_PER_WARP;
    if (k0 >= a.n_slots) return;
    const int64_t added = a.row_start[a.batch];
    int32_t got[4] = {-1, -1, -1, -1};
    const int64_t k = k0 + 4 * lane;
    if (k0 < added) {
        // the warp looks for the request of its first row: 32 places at a time
        int lo = 0, hi = a.batch;
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, at = lo + lane * step;
            const unsigned under = __ballot_sync(0xffffffffu, at < hi && a.row_start[min(at, a.batch)] <= k0);
            const int last = 31 - __clz(under);                  // lane 0 looks at lo, which is not beyond the row
            hi = min(lo + (last + 1) * step, hi);
            lo += last * step;
        }
        int b = lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (k + i >= added) break;
            if (a.row_start[b + 1] <= k + i) b = request_of(a.row_start, b + 1, a.batch, k + i);
            got[i] = slot_of_row(a, b, a.first_row[b] + (k + i - a.row_start[b]), a.new_lengths[b]);
        }
    }
    if (k + 4 <= a.n_slots && ((uintptr_t)a.slots & 15) == 0) {
        *reinterpret_cast<int4*>(a.slots + k) = make_int4(got[0], got[1], got[2], got[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (k + i < a.n_slots) a.slots[k + i] = got[i];
    }
}

}  // namespace bt
}  // namespace vec

using namespace vec;

extern "C" vector_status vector_block_tables(int32_t batch, const int32_t* lengths, const int32_t* added, int32_t page_rows, int32_t* table,
                                             int32_t width, int32_t* free_pages, int32_t cap_free, const int32_t* n_free, int32_t* new_lengths,
                                             int32_t* new_n_free, int32_t* first_row, int32_t* row_start, int32_t* slots, int64_t n_slots,
                                             void* stream) {
    if (!lengths || !added || !table || (cap_free > 0 && !free_pages) || !n_free || !new_lengths || !new_n_free || !first_row || !row_start) return VECTOR_ERR_NULL;
    if (n_slots > 0 && !slots) return VECTOR_ERR_NULL;
    if (batch < 1 || batch > 65535 || page_rows < 1 || width < 1 || cap_free < 0 || n_slots < 0 || n_slots > 0x7fffffffLL ||
        (int64_t)width * page_rows > 0x7fffffffLL)
        return VECTOR_ERR_SHAPE;
    const bt::Args a = {lengths, added, new_lengths, table, free_pages, new_n_free, first_row, row_start, slots, n_free, n_slots, batch, page_rows, width, cap_free};
    cudaStream_t st = (cudaStream_t)stream;
    if (batch <= bt::THREADS) {
        const int64_t blocks = (n_slots + bt::BLOCK_SLOTS - 1) / bt::BLOCK_SLOTS, most = sm_count();
        const int grid = (int)(blocks < 1 ? 1 : blocks > most ? most : blocks);
        // other blocks read the lengths and the stack's height as they were
        const bool apart = grid > 1 && (new_lengths == lengths || new_n_free == n_free);
        VEC_CUDA_CHECK(launch_maybe_dependent(true, bt::block_tables_batch, dim3(grid), dim3(bt::THREADS), 0, st, a, 1, apart ? 0 : 1));
        if (apart) VEC_CUDA_CHECK(launch_maybe_dependent(true, bt::block_tables_batch, dim3(1), dim3(bt::THREADS), 0, st, a, 0, 1));
        return VECTOR_OK;
    }
    VEC_CUDA_CHECK(launch_maybe_dependent(true, bt::block_tables_plan, dim3(1), dim3(bt::THREADS), 0, st, a));
    if (n_slots == 0) return VECTOR_OK;
    const int64_t per_block = (int64_t)bt::SLOT_THREADS / 32 * bt::SLOTS_PER_WARP;
    VEC_CUDA_CHECK(launch_maybe_dependent(true, bt::block_tables_slots, dim3((unsigned)((n_slots + per_block - 1) / per_block)), dim3(bt::SLOT_THREADS), 0, st, a));
    return VECTOR_OK;
}
