// Page tables, slots and positions from the lengths of the sequences.
//
// Everything follows from two prefix sums over the sequences: of their new rows, and of the pages they take (or give back).
// What there is to write (8 bytes a row) takes a microsecond or two at the largest sizes; the rest is launch latency and the
// chain  lengths -> sums -> which sequence a row belongs to -> page -> slot.  So one launch does all of it: every CTA forms the sums
// of all sequences itself (1,024 at a time, a thread each), instead of waiting for one that does, and then serves its own part of the rows, finding
// a row's sequence by bisection in shared memory.  That needs inputs that nobody writes meanwhile, hence the rule that outputs are
// not inputs.  Both calls of a step of 64 sequences take 4.8 us on the GPU (the host, which needs 3.5 us a call, is the bound there), 700 arrivals with
// room for 1.1M rows 11 us, 8.9 MB of it written in about 4.
#include "internal.h"
#include "ptx.cuh"

namespace pevlm {

constexpr int kMostThreads = 1024;

struct Sums {
    int64_t rows, pages;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) { return {a.rows + b.rows, a.pages + b.pages}; }
__device__ __forceinline__ Sums shifted_up(const Sums& a, int by) {
    return {__shfl_up_sync(0xffffffffu, a.rows, by), __shfl_up_sync(0xffffffffu, a.pages, by)};
}

// Inclusive sums over the CTA's threads; `all`: over all of them.
template <int THREADS>
__device__ __forceinline__ Sums scan(Sums x, Sums& all) {
    constexpr int kWarps = THREADS / 32;
    __shared__ Sums of_warp[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int by = 1; by < 32; by *= 2) {
        const Sums y = shifted_up(x, by);
        if (lane >= by) x = x + y;
    }
    if (lane == 31) of_warp[warp] = x;
    __syncthreads();
    if (kWarps <= 4) {
        Sums before{0, 0};
        all = {0, 0};
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w == warp) before = all;
            all = all + of_warp[w];
        }
        return x + before;
    }
    Sums w = of_warp[lane % kWarps];
#pragma unroll
    for (int by = 1; by < 32; by *= 2) {
        const Sums y = shifted_up(w, by);
        if (lane >= by) w = w + y;
    }
    const Sums before{__shfl_sync(0xffffffffu, w.rows, max(warp - 1, 0)), __shfl_sync(0xffffffffu, w.pages, max(warp - 1, 0))};
    all = {__shfl_sync(0xffffffffu, w.rows, kWarps - 1), __shfl_sync(0xffffffffu, w.pages, kWarps - 1)};
    return warp > 0 ? x + before : x;
}

// Last of the n ascending starts that is <= x (the first one is).
__device__ __forceinline__ int last_at_or_before(const int* starts, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int clamped(int x, int lo, int hi) { return min(max(x, lo), hi); }

// A thread has ROWS neighbouring rows at a time.
template <int THREADS, int ROWS>
__global__ void __launch_bounds__(THREADS) assign_kernel(const __grid_constant__ AssignParams p) {
    __shared__ int s_start[THREADS], s_len[THREADS], s_top[THREADS];  // of the sequences of this turn
    grid_wait();
    grid_launch_dependents();
    const int tid = threadIdx.x, P = 1 << p.page_shift, capacity = p.max_pages << p.page_shift;
    const int64_t count = clamped(*p.free_count, 0, p.num_pages);
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * p.rows_per_cta, row1 = min(row0 + p.rows_per_cta, p.max_rows);
    Sums base{0, 0};
    int64_t taken = 0;  // pages of the sequences that got theirs: what the last of them has as its inclusive sum
    for (int r0 = 0; r0 < p.num_seqs; r0 += THREADS) {
        const int r = r0 + tid, n = min(THREADS, p.num_seqs - r0);
        const bool there = r < p.num_seqs;
        const int len = there ? clamped(p.lens[r], 0, capacity) : 0;
        const int add = there ? max(p.new_lens[r], 0) : 0;
        const int have = (len + P - 1) >> p.page_shift;
        const bool fits = static_cast<int64_t>(len) + add <= capacity;  // its row of the table
        const int need = fits ? ((len + add + P - 1) >> p.page_shift) - have : 0;
        Sums all;
        const Sums to = base + scan<THREADS>(Sums{add, need}, all);
        // Of those that fit their rows, the ones that get pages are all up to some sequence: behind the first that takes the sums past
        // n_rows or past the free list no later one with new rows (with fresh pages) stays within.  So no page is passed over.
        const bool granted = there && fits && to.rows <= p.n_rows && (need == 0 || to.pages <= count);
        if (blockIdx.x == 0) {
            if (there) {
                p.lens_out[r] = granted ? len + add : len;
                if (p.key_lens) p.key_lens[r] = granted ? len + add : add > 0 ? 0 : len;
                p.row_start[r + 1] = static_cast<int>(min(to.rows, static_cast<int64_t>(INT32_MAX)));
            }
            if (granted && need > 0) taken = to.pages;
        }
        const int64_t first = base.rows, last = base.rows + all.rows;  // rows of this turn's sequences
        if (first < row1 && last > row0) {
            // A fresh page's place on the free list: page index i of the sequence at s_top - i.  Sequences turned away have s_len = -1.
            s_start[tid] = there ? static_cast<int>(min(to.rows - add, p.max_rows)) : INT32_MAX;
            s_len[tid] = granted ? len : -1 - len;
            s_top[tid] = static_cast<int>(count - 1 - (to.pages - need) + have);
            __syncthreads();
            // (rows and positions fit 31 bits: at most 2^30 rows, and a position is below the 2^30 of a table's row or that many behind it)
            const int lo = static_cast<int>(max(first, row0)), hi = static_cast<int>(min(last, row1));
            for (int g = lo / ROWS * ROWS + ROWS * tid; g < hi; g += ROWS * THREADS) {
                int q = last_at_or_before(s_start, n, max(g, lo));
                int slot[ROWS], position[ROWS], page = -1, page_q = -1, page_index = -1;  // neighbours mostly share a page
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    const int row = g + i;
                    slot[i] = -1;
                    position[i] = 0;
                    if (row < lo || row >= hi) continue;
                    while (q + 1 < n && s_start[q + 1] <= row) ++q;  // sequences without rows are passed over
                    const int held = s_len[q] < 0 ? -1 - s_len[q] : s_len[q];
                    const int pos = held + (row - s_start[q]);
                    position[i] = pos;
                    if (s_len[q] < 0) continue;
                    const int index = pos >> p.page_shift;
                    if (q != page_q || index != page_index) {
                        int32_t* const entry = p.page_table + static_cast<int64_t>(r0 + q) * p.max_pages + index;
                        const bool fresh = index >= (held + P - 1) >> p.page_shift;
                        page = fresh ? p.free_list[s_top[q] - index] : *entry;
                        page_q = q;
                        page_index = index;
                        if (fresh && (pos & (P - 1)) == 0) *entry = page;
                    }
                    if (page >= 0 && page < p.num_pages) slot[i] = (page << p.page_shift) + (pos & (P - 1));
                }
                if (ROWS % 4 == 0 && g >= lo && g + ROWS <= hi) {
#pragma unroll
                    for (int i = 0; i + 3 < ROWS; i += 4) {
                        *reinterpret_cast<int4*>(p.slots + g + i) = make_int4(slot[i], slot[i + 1], slot[i + 2], slot[i + 3]);
                        *reinterpret_cast<int4*>(p.positions + g + i) = make_int4(position[i], position[i + 1], position[i + 2], position[i + 3]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < ROWS; ++i) {
                        if (g + i < lo || g + i >= hi) continue;
                        p.slots[g + i] = slot[i];
                        p.positions[g + i] = position[i];
                    }
                }
            }
        }
        base = base + all;
        __syncthreads();  // the arrays and the warps' sums are written again
    }
    // rows that no sequence has
    for (int64_t row = max(base.rows, row0) + tid; row < row1; row += THREADS) {
        p.slots[row] = -1;
        p.positions[row] = 0;
    }
    if (blockIdx.x == 0) {
        __shared__ int most;
        if (tid == 0) most = 0;
        __syncthreads();
        if (taken > 0) atomicMax(&most, static_cast<int>(taken));  // at most count
        __syncthreads();
        if (tid == 0) {
            p.row_start[0] = 0;
            *p.free_count_out = static_cast<int>(count) - most;
        }
    }
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) release_kernel(const __grid_constant__ ReleaseParams p) {
    __shared__ int s_start[THREADS];
    grid_wait();
    grid_launch_dependents();
    const int tid = threadIdx.x, P = 1 << p.page_shift, capacity = p.max_pages << p.page_shift;
    const int64_t count = clamped(*p.free_count, 0, p.num_pages);
    Sums base{0, 0};
    for (int r0 = 0; r0 < p.num_seqs; r0 += THREADS) {
        const int r = r0 + tid, n = min(THREADS, p.num_seqs - r0);
        const bool there = r < p.num_seqs;
        const int len = there ? clamped(p.lens[r], 0, capacity) : 0;
        const bool finished = there && p.finished[r] != 0;
        const int given = finished ? (len + P - 1) >> p.page_shift : 0;
        Sums all;
        const Sums to = base + scan<THREADS>(Sums{0, given}, all);
        if (blockIdx.x == 0 && there) p.lens_out[r] = finished ? 0 : len;
        if (all.pages > 0) {
            s_start[tid] = static_cast<int>(min(to.pages - given - base.pages, static_cast<int64_t>(INT32_MAX)));
            __syncthreads();
            const int64_t at = count + base.pages, room = min(all.pages, p.num_pages - at);
            for (int64_t i = static_cast<int64_t>(blockIdx.x) * THREADS + tid; i < room; i += static_cast<int64_t>(gridDim.x) * THREADS) {
                const int q = last_at_or_before(s_start, n, static_cast<int>(i));
                p.free_list[at + i] = p.page_table[static_cast<int64_t>(r0 + q) * p.max_pages + (i - s_start[q])];
            }
        }
        base = base + all;
        __syncthreads();
    }
    if (blockIdx.x == 0 && tid == 0) *p.free_count_out = static_cast<int>(min(count + base.pages, static_cast<int64_t>(p.num_pages)));
}

// Few sequences and rows: CTAs of 128 threads, whose barriers and sums take less.  Both calls on the GPU, 128 against 1,024 threads of four rows: 1 sequence of one row
// 3.3 / 5.1 us, 64 of one 3.9 / 6.6, 128 of one 3.9 / 7.0, 128 of four 6.1 / 6.2, 64 of 32 rows 13.7 / 6.0, 512 of one 9.2 / 7.2, 1,024 of one 15.8 / 7.6.
cudaError_t launch_assign(AssignParams p, cudaStream_t stream) {
    if (p.num_seqs <= 128 && p.max_rows <= 512) {
        p.rows_per_cta = p.max_rows;
        return launch_chained<assign_kernel<128, 1>>(dim3(1), 128, 0, stream, p);
    }
    const int64_t want = (p.max_rows + 4 * kMostThreads - 1) / (4 * kMostThreads);
    const unsigned grid = static_cast<unsigned>(want < 1 ? 1 : want > kNumSms ? kNumSms : want);
    p.rows_per_cta = ((p.max_rows + grid - 1) / grid + 3) & ~3ll;
    return launch_chained<assign_kernel<kMostThreads, 4>>(dim3(grid), kMostThreads, 0, stream, p);
}

cudaError_t launch_release(const ReleaseParams& p, cudaStream_t stream) {
    const int64_t entries = static_cast<int64_t>(p.num_seqs) * p.max_pages;
    if (p.num_seqs <= 128) {
        const int64_t want = entries / 1024;
        return launch_chained<release_kernel<128>>(dim3(static_cast<unsigned>(want < 1 ? 1 : want > 16 ? 16 : want)), 128, 0, stream, p);
    }
    const int64_t want = entries / (8 * kMostThreads);
    return launch_chained<release_kernel<kMostThreads>>(dim3(static_cast<unsigned>(want < 1 ? 1 : want > 32 ? 32 : want)), kMostThreads, 0, stream, p);
}

}  // namespace pevlm
