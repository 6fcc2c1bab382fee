// Attention over the packed cache for many rows per sequence and kv head (question blocks, chunks of a prefill): the tensor cores' tiles.
//
// The same pipeline as attn_kernel.cu on pairs of CTAs (S = Q K^T and O += P V with tcgen05.mma.cta_group::2, M = 256; scores, probabilities and
// accumulator side by side in TMEM; two softmax warpgroups that take the key tiles in turn), with operands that come out of 4 bits:
//   warps 0-3, 4-7  softmax, one thread per row
//   warps 8-11  feeder: turns the CTA's half of every K tile (64 keys) and V tile (D/2 columns) from e2m1 codes and e4m3 scales into fp16 in
//               the swizzled layout the MMAs read, brings Q's rows into it, and between two items writes out the finished one
//   warps 12, 14 (first CTA of the pair) issue the MMAs, warp 12 of the second hands its feeder's work over; warp 13 fetches the packed tiles (cp.async.bulk, 16 tokens of a page each),
//   warp 15     makes the work items
// Everything is fp16 instead of bf16: the cache's values are exact in it and two instructions a pair make them (a conversion and the product
// with the scale; bf16 would take five); rows of Q are scaled by a power of two (RowPower in packed_list.cuh), whose inverse goes into the row's softmax
// scale; probabilities (at most 2^8 above the reference, and raised by kHeadroom) keep 11 bits.
// A row block is 256 rows (token, head of the group), each CTA's 128 against the same keys, so a pair unpacks every tile once for 256 rows; with
// 4.5 bits a value the cache itself is no bandwidth to speak of.  What bounds it is what bounds attn_kernel.cu: the softmax
// beside running MMAs, and the power of the tensor cores: 256 tokens of 28/4 heads against 74K keys take 254 us back to back at the power cap (1,070
// TFLOP/s), 220 in a burst (1,230).  The feeder (one warp a scheduler) is just fast enough: its tile has to take less than the 1,500 to 1,750
// cycles of the softmax's, so it converts four chunks side by side, keeps V two tiles behind K (a V tile's place is free only when the softmax has
// been through the tile four before), and does not tell the other CTA itself (see the hand-over).  Before these steps: 362 us.
// Work is dealt out as in packed_list.cuh, with tiles of 128 keys and pairs of CTAs as workers: a unit that crosses from one pair to the next is left
// as shares for packed_merge_kernel.  Items follow from lengths on the device, and every wait is bounded as in attn_kernel.cu.
#include "packed_list.cuh"

namespace pevlm {

constexpr int kTileThreads = 512;
constexpr int kFeedRing = 4;     // K tiles and V tiles in fp16
constexpr int kFedRing = 8;      // tiles whose masks are kept: the feeder may be four tiles ahead of a softmax warp that has yet to look
constexpr int kRawRing = 3;      // packed tiles in flight
constexpr int kTileItems = 4;    // work items in flight
constexpr int kTileSums = 4;     // items whose row sums may be in flight between softmax and epilogue (a softmax warp that has no tile in an
                                 // item leaves its sums at once: up to three items of one tile ahead of the one that is written out)
constexpr int kTileTurn = 40;    // see kTurn in attn_kernel.cu
constexpr float kTileRescaleLog2 = 8.0f;
constexpr uint32_t kTileTmemP = 2 * kTile, kTileTmemO = 3 * kTile;

enum TileWaitId : int {
    kTwItem = 41, kTwItemFree = 42, kTwRaw = 43, kTwRawFree = 44, kTwKFree = 45, kTwVFree = 46, kTwQ = 47, kTwQFree = 48, kTwK = 49, kTwV = 50, kTwSRead = 51,
    kTwS = 52, kTwFed = 53, kTwP = 54, kTwPV = 55, kTwPFree = 56, kTwOFree = 57, kTwSum = 58, kTwODone = 59
};

template <int D>
struct PackedTileLayout {
    static constexpr int kPanels = D / 64;
    static constexpr int kRows = 2 * kTile;                       // of a unit
    static constexpr int kShareFloats = kRows * (D + 2);
    static constexpr int kQPanelBytes = kTile * 128, kKPanelBytes = kTile / 2 * 128;
    static constexpr int kQBytes = kPanels * kQPanelBytes, kKBytes = kPanels * kKPanelBytes, kVBytes = kTile * D;
    static constexpr int kSubBytes = 18 * D, kRawBytes = 8 * kSubBytes;  // 16 tokens; a tile
    static constexpr int kQ = 0, kK = kQBytes, kV = kK + kFeedRing * kKBytes, kRaw = kV + kFeedRing * kVBytes;
    static constexpr int kTotal = kRaw + kRawRing * kRawBytes;
};

// A piece of a unit: its tiles [t0, t0 + nt), of those that its own rows see.
struct TileItem {
    int nt, t0, ns, skip;
    int len, n, row0, head, chunk;
    int seq;
    int whole, second;  // nothing is left for the merge; the share's place
};

__host__ __device__ constexpr uint32_t make_idesc_f16(int m, int n, bool b_mn_major) {
    return make_idesc_bf16(m, n, b_mn_major) & ~((1u << 7) | (1u << 10));  // A and B format 0: fp16
}
// Arrivals and waits of one CTA for what the other has written to its own shared memory.
__device__ __forceinline__ void mbar_arrive_release_cluster(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait_cluster(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ void mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile WaitState& state, int which) {
    int n = 0;
#pragma unroll 1
    while (!mbar_try_wait_cluster(bar, parity)) {
        if (++n > state.tries) {
            if (state.expired == 0) state.expired = which;
            state.tries = kGraceTries;
            return;
        }
    }
}

template <typename T>
__device__ __forceinline__ T ld_shared(uint32_t addr) {
    T x;
    if constexpr (sizeof(T) == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(addr) : "memory");
    else if constexpr (sizeof(T) == 8) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(addr) : "memory");
    else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(addr) : "memory");
    return x;
}
// The eight codes of a word times a scale (twice in a word), as eight fp16 in shared memory.
__device__ __forceinline__ void st_shared_values(uint32_t addr, uint32_t codes, uint32_t scale2) {
    uint32_t x[4];
    halves_of_word(codes, x);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(mul_f16x2(x[0], scale2)), "r"(mul_f16x2(x[1], scale2)), "r"(mul_f16x2(x[2], scale2)),
                 "r"(mul_f16x2(x[3], scale2)));  // (ordered by the fence behind a tile's stores, and free to mix with one another's conversions)
}

__device__ __forceinline__ int same_in_warp(int x) { return __shfl_sync(0xffffffffu, x, 0); }
// Between the two softmax warps of a scheduler, see attn_kernel.cu; no limit: both go through the same tiles whatever happens.
__device__ __forceinline__ void turn_wait(int what, int wg, int quarter) { asm volatile("bar.sync %0, 64;" ::"r"(what + wg * 4 + quarter) : "memory"); }
__device__ __forceinline__ void turn_pass(int what, int wg, int quarter) { asm volatile("bar.arrive %0, 64;" ::"r"(what + (wg ^ 1) * 4 + quarter) : "memory"); }

// Worker `me` of the list, by one warp: its part.  A lane has four neighbouring sequences at a time.
__device__ __forceinline__ PackedPart part_by_warp(const PackedAttnParams& p, int rows_per_chunk, int me, int workers) {
    const int lane = threadIdx.x & 31;
    auto tiles_of = [&](int r) { return r < p.num_seqs ? seq_tiles<7>(p, packed_seq<7>(p, r, rows_per_chunk)) : 0; };
    int64_t total = 0;
    for (int r0 = 4 * lane; r0 < p.num_seqs; r0 += 128) {
#pragma unroll
        for (int i = 0; i < 4; ++i) total += tiles_of(r0 + i);
    }
#pragma unroll
    for (int by = 16; by > 0; by /= 2) total += __shfl_xor_sync(0xffffffffu, total, by);
    PackedPart part{PackedDeal(total, workers), 0, 0, {}};
    const int64_t lo = part.deal.start(me);
    if (lo >= part.deal.start(me + 1)) return part;
    int64_t base = 0;
    for (int r0 = 0; r0 < p.num_seqs; r0 += 128) {
        const int r = r0 + 4 * lane;
        int64_t mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) mine += tiles_of(r + i);
        const int64_t to = base + warp_inclusive(mine);
        const unsigned past = __ballot_sync(0xffffffffu, to > lo);
        if (past) {
            const int l = __ffs(past) - 1;
            part.seq = r0 + 4 * l;
            part.off = lo - __shfl_sync(0xffffffffu, to - mine, l);
            for (int i = 0; i < 3; ++i) {
                const int64_t of_seq = tiles_of(part.seq);
                if (part.off < of_seq) break;
                part.off -= of_seq;
                ++part.seq;
            }
            part.s = packed_seq<7>(p, part.seq, rows_per_chunk);
            break;
        }
        base = __shfl_sync(0xffffffffu, to, 31);
    }
    return part;
}

template <int D>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTileThreads, 1) packed_tile_kernel(const __grid_constant__ PackedAttnParams p) {
    using L = PackedTileLayout<D>;
    extern __shared__ uint8_t smem_raw[];
    struct Bars {
        uint64_t item_full[kTileItems], item_free[kTileItems];  // both: each CTA has its own
        uint64_t raw_full[kRawRing], raw_free[kRawRing];        // both
        uint64_t q_full, k_full[kFeedRing], v_full[kFeedRing];  // both: the CTA's feeder has written; first: and the other's (see the hand-over)
        uint64_t q_free;                                        // both
        uint64_t fed[kFedRing];                                 // both: the tile's mask (and its item's scales) are there
        uint64_t s_full[kFeedRing], pv_done[kFeedRing];         // both: QK(t), PV(t) are complete
        uint64_t s_read[2], p_full[2], o_free;                  // first
        uint64_t sums_full[kTileSums];                          // both
    };
    __shared__ Bars bars;
    __shared__ uint32_t tmem_base_slot;
    __shared__ WaitState wait_state;
    __shared__ unsigned s_published;
    __shared__ TileItem s_items[kTileItems];
    __shared__ float s_max[2][kTile];
    __shared__ float2 s_sums[kTileSums][2][kTile];
    __shared__ float s_scale[4][kTile];       // softmax scale of the rows in units of log2, items in turn
    __shared__ unsigned s_raw_there[kRawRing], s_there[kFedRing];  // of a tile's 16-key parts, which exist
    __shared__ __align__(4) uint16_t s_raw_seen[kRawRing][8];  // of each part's keys, those that a row of the item can see

    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = same_in_warp(tid >> 5);
    const uint32_t rank = cluster_ctarank();
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (smem_base - smem_u32(smem_raw));
    constexpr unsigned kNoMore = 1u << 31;

    if (tid == 0) {
        wait_state.tries = kDefaultWaitTries;
        wait_state.expired = 0;
        s_published = 0;
        for (int i = 0; i < kTileItems; ++i) {
            mbar_init(smem_u32(&bars.item_full[i]), 1);
            mbar_init(smem_u32(&bars.item_free[i]), 1 + 8 + 4 + 2);
        }
        for (int i = 0; i < kRawRing; ++i) {
            mbar_init(smem_u32(&bars.raw_full[i]), 1);
            mbar_init(smem_u32(&bars.raw_free[i]), 4);
        }
        for (int i = 0; i < kFeedRing; ++i) {
            mbar_init(smem_u32(&bars.k_full[i]), rank == 0 ? 4 + 1 : 4);
            mbar_init(smem_u32(&bars.v_full[i]), rank == 0 ? 4 + 1 : 4);
            mbar_init(smem_u32(&bars.s_full[i]), 1);
            mbar_init(smem_u32(&bars.pv_done[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars.s_read[i]), 8);
            mbar_init(smem_u32(&bars.p_full[i]), 8);
        }
        for (int i = 0; i < kFedRing; ++i) mbar_init(smem_u32(&bars.fed[i]), 4);
        for (int i = 0; i < kTileSums; ++i) mbar_init(smem_u32(&bars.sums_full[i]), 8);
        mbar_init(smem_u32(&bars.q_full), rank == 0 ? 4 + 1 : 4);
        mbar_init(smem_u32(&bars.q_free), 1);
        mbar_init(smem_u32(&bars.o_free), 8);
        fence_mbar_init();
    }
    if (warp == 12) {
        __syncwarp();
        tmem_alloc_pair(smem_u32(&tmem_base_slot), 512);
    }
    tc_fence_before_sync();
    cluster_sync_all();
    tc_fence_after_sync();
    const uint32_t tmem_base = same_in_warp(tmem_base_slot);
    grid_wait();
    grid_launch_dependents();
    if (blockIdx.x == 0 && tid == 0) p.hdr->status = p.hdr->detail = 0;  // of the call before; no wait has run out yet

    auto wait = [&](const uint64_t& bar, uint32_t parity, int which) { mbar_wait(smem_u32(&bar), parity, wait_state, which); };
    auto wait_asleep = [&](const uint64_t& bar, uint32_t parity, int which) { mbar_wait<100>(smem_u32(&bar), parity, wait_state, which); };
    // k-th item: the same answer in every warp, a timeout included (see item_ready in attn_kernel.cu)
    auto item_ready = [&](int k) {
        wait(bars.item_full[k % kTileItems], (k / kTileItems) & 1, kTwItem);
        if (static_cast<int>(*static_cast<volatile unsigned*>(&s_published) & ~kNoMore) > k) return true;
        return static_cast<int>(atomicOr(&s_published, kNoMore) & ~kNoMore) > k;
    };
    auto item_release = [&](int k) { mbar_arrive(smem_u32(&bars.item_free[k % kTileItems])); };
    auto wait_s_full = [&](uint32_t t, int which) { wait(bars.s_full[t % kFeedRing], (t / kFeedRing) & 1, which); };
    auto wait_pv_done = [&](uint32_t t, int which) { wait(bars.pv_done[t % kFeedRing], (t / kFeedRing) & 1, which); };

    // registers: 2 x 184 + 96 + 48 = 4 x 128
    if (warp >= 12) {
        reg_dealloc<48>();
        if (warp == 15) {
            // ------------------------------------------------------------- work items
            const int me = static_cast<int>(blockIdx.x >> 1);
            const PackedPart part = part_by_warp(p, L::kRows, me, static_cast<int>(gridDim.x >> 1));
            const int64_t lo = part.deal.start(me), hi = part.deal.start(me + 1);
            PackedJoin join{0, 0, 0, 0, 0, 0};
            int published = 0;
            bool stop = false;
            if (lo < hi) {
                int at;
                PackedUnit<7> u(part, at);
                int64_t unit0 = lo - at + kUnitTiles<7>;
                int first = max(at - kUnitTiles<7>, 0);
                while (unit0 < hi && !stop) {
                    // the unit's own tiles: up to its last row's position, from where its first row's window begins
                    TileItem it;
                    const int row_a = u.chunk * L::kRows, row_b = min(row_a + L::kRows, u.s.n * p.G) - 1;
                    const int pos_a = u.s.len - u.s.n + quotient(row_a, p.div_g), pos_b = u.s.len - u.s.n + quotient(row_b, p.div_g);
                    const int tiles = pos_b >= 0 ? (pos_b >> 7) + 1 : 0;
                    it.ns = min(u.s.ns, tiles);
                    it.skip = p.window > 0 ? min(max((max(pos_a - p.window + 1, 0) >> 7) - it.ns, 0), tiles - it.ns) : 0;
                    const int cnt = max(tiles - it.skip, 1);
                    it.t0 = first;
                    it.nt = static_cast<int>(max(min(hi - unit0, static_cast<int64_t>(cnt)), static_cast<int64_t>(0))) - first;
                    if (it.nt > 0) {
                        it.len = u.s.len; it.n = u.s.n; it.row0 = u.s.row0; it.head = u.head; it.chunk = u.chunk;
                        it.seq = u.r;
                        it.whole = it.t0 == 0 && it.nt == cnt;
                        it.second = unit0 > lo;
                        if (!it.whole && it.t0 == 0) join = {part.deal.worker_of(unit0 + cnt - 1), it.second, it.row0, it.n, it.head, it.chunk};
                        const int slot = published % kTileItems;
                        if (published >= kTileItems) {
                            wait_asleep(bars.item_free[slot], (published / kTileItems - 1) & 1, kTwItemFree);
                            if (!mbar_try_wait(smem_u32(&bars.item_free[slot]), (published / kTileItems - 1) & 1)) stop = true;  // may still be read
                        }
                        stop = __any_sync(0xffffffffu, stop);
                        if (!stop) {
                            if (lane == 0) {
                                s_items[slot] = it;
                                __threadfence_block();
                                if (atomicCAS(&s_published, published, published + 1) != static_cast<unsigned>(published)) stop = true;
                                else mbar_arrive(smem_u32(&bars.item_full[slot]));
                            }
                            stop = __shfl_sync(0xffffffffu, stop, 0);
                            ++published;
                        }
                    }
                    unit0 += u.s.cnt + kUnitTiles<7>;
                    first = 0;
                    if (unit0 < hi) u.next(p, L::kRows, nullptr);
                }
            }
            // the end takes a place like an item: its phase must not pass a warp that has yet to see the one before in that place
            if (published >= kTileItems) wait_asleep(bars.item_free[published % kTileItems], (published / kTileItems - 1) & 1, kTwItemFree);
            if (lane == 0) {
                atomicOr(&s_published, kNoMore);
                mbar_arrive(smem_u32(&bars.item_full[published % kTileItems]));
                if (rank == 0) p.joins[me] = join;
            }
        } else if (warp == 13) {
            // ------------------------------------------------------------- packed tiles: lane i fetches its i-th 16 keys
            uint32_t u = 0;
#pragma unroll 1
            for (int k = 0; same_in_warp(item_ready(k)); ++k) {
                const TileItem& it = s_items[k % kTileItems];
                const int nt = it.nt, t0 = it.t0, ns = it.ns, skip = it.skip, len = it.len, head = it.head, seq = it.seq;
                const int low = p.window > 0 ? len - it.n + quotient(it.chunk * L::kRows, p.div_g) - p.window + 1 : 0;  // of the first row's window
                __syncwarp();
                if (lane == 0) item_release(k);
                auto sub = [&](int j) { return (j < ns ? j : j + skip) * 8 + lane; };  // of the sequence's 16-key tiles
                int page = lane < 8 ? packed_page(p, seq, len, sub(t0)) : -1;
#pragma unroll 1
                for (int j = t0; j < t0 + nt; ++j, ++u) {
                    const int place = u % kRawRing;
                    const int page_next = lane < 8 && j + 1 < t0 + nt ? packed_page(p, seq, len, sub(j + 1)) : -1;
                    if (u >= kRawRing) wait(bars.raw_free[place], (u / kRawRing - 1) & 1, kTwRawFree);
                    const uint32_t at = lane < 8 ? packed_place(p, page, head, sub(j), L::kSubBytes / 128) : kNoTile;
                    const unsigned there = __ballot_sync(0xffffffffu, at != kNoTile);
                    const uint32_t bar = smem_u32(&bars.raw_full[place]);
                    if (lane < 8) {
                        const int key0 = sub(j) << 4;
                        auto first = [&](int end) { return (1u << min(max(end - key0, 0), 16)) - 1u; };  // keys before `end`
                        s_raw_seen[place][lane] = static_cast<uint16_t>(at != kNoTile ? first(len) & (first(p.sink) | ~first(low)) : 0u);
                    }
                    __syncwarp();
                    if (lane == 0) {
                        s_raw_there[place] = there;
                        mbar_arrive_expect_tx(bar, __popc(there) * L::kSubBytes);
                    }
                    __syncwarp();
                    if (at != kNoTile)
                        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                                     ::"r"(smem_base + L::kRaw + place * L::kRawBytes + lane * L::kSubBytes), "l"(p.cache + static_cast<uint64_t>(at) * 128),
                                       "r"(L::kSubBytes), "r"(bar) : "memory");
                    page = page_next;
                }
            }
        } else if (rank == 0 && warp == 12) {
            // ------------------------------------------------------------- S = Q K^T of the pair
            uint32_t t = 0;
#pragma unroll 1
            for (int k = 0; same_in_warp(item_ready(k)); ++k) {
                const int nt = same_in_warp(s_items[k % kTileItems].nt);
                __syncwarp();
                if (lane == 0) item_release(k);
                const uint32_t q_lo = desc_lo(smem_base + L::kQ, 16);
                mbar_wait_cluster(smem_u32(&bars.q_full), k & 1, wait_state, kTwQ);
#pragma unroll 1
                for (int j = 0; j < nt; ++j, ++t) {
                    const uint32_t slot = t % kFeedRing;
                    mbar_wait_cluster(smem_u32(&bars.k_full[slot]), (t / kFeedRing) & 1, wait_state, kTwK);
                    if (t >= 2) wait(bars.s_read[t & 1], ((t >> 1) - 1) & 1, kTwSRead);
                    tc_fence_after_sync();
                    mma_ss_batch<D / 16>(tmem_base + (t & 1) * kTile, q_lo, desc_lo(smem_base + L::kK + slot * L::kKBytes, 16),
                                         make_idesc_f16(2 * kTile, kTile, false));
                    mma_commit_pair(smem_u32(&bars.s_full[slot]));
                }
                mma_commit_pair(smem_u32(&bars.q_free));
            }
        } else if (rank == 0 && warp == 14) {
            // ------------------------------------------------------------- O += P V of the pair
            constexpr uint32_t kIdescPv = make_idesc_f16(2 * kTile, D, true);
            const uint32_t d_tmem = tmem_base + kTileTmemO;
            uint32_t t = 0;
#pragma unroll 1
            for (int k = 0; same_in_warp(item_ready(k)); ++k) {
                const int nt = same_in_warp(s_items[k % kTileItems].nt);
                __syncwarp();
                if (lane == 0) item_release(k);
                if (k > 0) wait(bars.o_free, (k - 1) & 1, kTwOFree);  // the previous output has left TMEM
#pragma unroll 1
                for (int j = 0; j < nt; ++j, ++t) {
                    const uint32_t slot = t % kFeedRing;
                    const uint32_t v_lo = desc_lo(smem_base + L::kV + slot * L::kVBytes, 0);
                    const uint32_t a_tmem = tmem_base + kTileTmemP + (t & 1) * (kTile / 2);
                    mbar_wait_cluster(smem_u32(&bars.v_full[slot]), (t / kFeedRing) & 1, wait_state, kTwV);
                    wait(bars.p_full[t & 1], (t >> 1) & 1, kTwP);
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int ks = 0; ks < kTile / 16; ++ks) mma_ts_step<D>(d_tmem, a_tmem + ks * 8, v_lo + ks * kVDescStep<D>, kIdescPv, j + ks);
                    mma_commit_pair(smem_u32(&bars.pv_done[slot]));
                }
            }
        } else if (warp == 12 || warp == 14) {
            // ------------------------------------------------------------- hand-over: tells the first CTA what the second's feeder has written,
            // warp 12 of Q and K, warp 14 of V.  (An arrival that releases this CTA's writes to the other one takes 650 cycles of the warp that
            // makes it; two of them a tile in the feeder were half of its time.)
            const uint64_t* const full = warp == 12 ? bars.k_full : bars.v_full;
            uint32_t t = 0;
#pragma unroll 1
            for (int k = 0; same_in_warp(item_ready(k)); ++k) {
                const int nt = same_in_warp(s_items[k % kTileItems].nt);
                __syncwarp();
                if (lane == 0) item_release(k);
                if (warp == 12) {
                    wait(bars.q_full, k & 1, kTwQ);
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release_cluster(map_to_cta(smem_u32(&bars.q_full), 0));
                }
#pragma unroll 1
                for (int j = 0; j < nt; ++j, ++t) {
                    wait(full[t % kFeedRing], (t / kFeedRing) & 1, warp == 12 ? kTwK : kTwV);
                    __syncwarp();
                    if (lane == 0) mbar_arrive_release_cluster(map_to_cta(smem_u32(&full[t % kFeedRing]), 0));
                }
            }
        }
    } else if (warp >= 8) {
        // ----------------------------------------------------------------- feeder and epilogue
        reg_dealloc<96>();
        const int fw = warp - 8, g = lane >> 2, c4 = lane & 3;  // K: key g (and g + 8), quarter c4 of the head
        const int k8 = lane & 7, e4 = lane >> 3;                // V: key k8 (and k8 + 8), eighth 4 rank + e4 of the head
        const int eighth = 4 * static_cast<int>(rank) + e4;
        const int row = tid & 127;
        const uint32_t tO = tmem_base + kTileTmemO + (static_cast<uint32_t>(fw * 32) << 16);
        const uint32_t o_free_bar = map_to_cta(smem_u32(&bars.o_free), 0);
        uint32_t t = 0, v = 0;              // tiles whose K, whose V has been fed
        int started = 0, out_k = 0;         // items whose tiles are being fed or have been; the oldest that is not written out,
        uint32_t out_end = 0;               // and the tiles up to its end

        // Writes item k out, its PVs being complete once its last tile's, t_end - 1, is.
        auto epilogue = [&](int k, uint32_t t_end) {
            const TileItem& done = s_items[k % kTileItems];
            const int rr = done.chunk * L::kRows + static_cast<int>(rank) * kTile + row;
            const bool row_ok = rr < done.n * p.G;
            const float scale = s_scale[k & 3][row];
            wait_asleep(bars.sums_full[k % kTileSums], (k / kTileSums) & 1, kTwSum);
            const float2 sa = s_sums[k % kTileSums][0][row], sb = s_sums[k % kTileSums][1][row];
            const float m = fmaxf(sa.y, sb.y);
            const float l = m == -INFINITY ? 0.f : sa.x * fast_exp2((sa.y - m) * scale) + sb.x * fast_exp2((sb.y - m) * scale);
            const float inv = !done.whole ? 1.f : l > 0.f ? 1.f / l : 0.f;
            wait_pv_done(t_end - 1, kTwODone);
            tc_fence_after_sync();
            const PackedRow at = packed_row(p, done.row0, done.head, row_ok ? rr : 0, D);
            float* const share = p.part + (2 * static_cast<int64_t>(blockIdx.x >> 1) + done.second) * L::kShareFloats;
            const int in_unit = static_cast<int>(rank) * kTile + row;
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                tmem_ld32(tO + c * 32, o);
                tmem_wait_ld();
                if (c == D / 32 - 1) {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(o_free_bar);
                }
                if (row_ok && done.whole) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = pack_bf16x2(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv);
#pragma unroll
                    for (int v = 0; v < 2; ++v) st_global_v8(p.o + at.o + c * 32 + v * 16, *reinterpret_cast<uint32_t(*)[8]>(&w[8 * v]));
                } else if (row_ok) {
#pragma unroll
                    for (int v = 0; v < 8; ++v)
                        reinterpret_cast<uint4*>(share + in_unit * D + c * 32)[v] = make_uint4(o[4 * v], o[4 * v + 1], o[4 * v + 2], o[4 * v + 3]);
                }
                __syncwarp();
            }
            if (row_ok) {
                const float m_log2 = m == -INFINITY ? kNoMax : m * scale - kHeadroom;
                if (!done.whole) {
                    share[L::kRows * D + in_unit] = m_log2;
                    share[L::kRows * (D + 1) + in_unit] = l;
                } else if (p.lse) {
                    p.lse[at.lse] = l > 0.f ? (m_log2 + log2f(l)) * 0.693147180559945309f : -INFINITY;
                }
            }
            __syncwarp();
            if (lane == 0) item_release(k);
        };

        // Codes of a tile in registers: K's of keys g and g + 8 of this warp's 16 (heads of 64: two words of each are used), V's of keys k8 and
        // k8 + 8 of two parts of 16, and their scales.  V's scales are 0 for keys behind the end, not there or seen by no row, whose bytes may be
        // anything.
        struct VCodes {
            uint2 c[2][2];
            uint32_t s[2];
        };
        uint4 kc[2];
        uint32_t ks = 0;
        unsigned there = 0;
        VCodes v_now, v_one, v_two;  // of the tile just loaded, and of the one and two before
        auto load = [&]() {
            const uint32_t place = t % kRawRing;
            wait(bars.raw_full[place], (t / kRawRing) & 1, kTwRaw);
            there = s_raw_there[place];
            const uint32_t raw = smem_base + L::kRaw + place * L::kRawBytes;
            const uint32_t sub = raw + (4 * rank + fw) * L::kSubBytes;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (D == 128) kc[h] = ld_shared<uint4>(sub + h * 512 + lane * 16);
                else *reinterpret_cast<uint2*>(&kc[h]) = ld_shared<uint2>(sub + h * 256 + lane * 8);
            }
            ks = D == 128 ? ld_shared<uint32_t>(sub + 16 * D + lane * 4) : ld_shared<uint32_t>(sub + 16 * D + (lane >> 1) * 4) >> (lane & 1) * 16;
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                const uint32_t from = raw + (2 * fw + s2) * L::kSubBytes;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (D == 128) v_now.c[s2][h] = ld_shared<uint2>(from + 8 * D + ((h * 8 + eighth) * 8 + k8) * 8);
                    else v_now.c[s2][h].x = ld_shared<uint32_t>(from + 8 * D + ((h * 8 + eighth) * 8 + k8) * 4);
                }
                v_now.s[s2] = ld_shared<uint32_t>(from + 17 * D + (D == 128 ? eighth : eighth >> 1) * 16 + (k8 >> 1) * 4);
            }
            const uint32_t seen = *reinterpret_cast<const uint32_t*>(&s_raw_seen[place][2 * fw]);
            if (seen != 0xffffffffu) {
                const uint32_t bytes = (seen >> k8 & 0x01010101u) * 0xffu;
                v_now.s[0] &= __byte_perm(bytes, 0u, 0x1100);
                v_now.s[1] &= __byte_perm(bytes, 0u, 0x3322);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.raw_free[place]));
        };
        // where this thread's chunks of 16 bytes go: eight lanes that store together hit all banks (of K's words the upper quarters of the head
        // take theirs in another order)
        const bool upper = D == 128 && c4 >= 2;
        const uint32_t k_to = smem_base + L::kK + (upper ? L::kKPanelBytes : 0) + (fw * 16 + g) * 128;
        const uint32_t k_chunk = D == 128 ? (4 * (c4 & 1)) ^ (upper ? 2 : 0) ^ g : (2 * c4) ^ g;
        const uint32_t v_to = smem_base + L::kV + (fw * 32 + k8) * (D == 128 ? 128 : 64);
        const uint32_t v_scale = k8 & 1 ? 0x11 : 0x00;  // byte of the word, twice
        const uint32_t v_chunk = D == 128 ? (2 * e4) ^ k8 : e4 ^ (k8 >> 1);
        // K of tile t, from the registers
        auto feed_k = [&]() {
            const uint32_t slot = t % kFeedRing, k_at = k_to + slot * L::kKBytes;
            if (t >= kFeedRing) wait_s_full(t - kFeedRing, kTwKFree);
            if (D == 128) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t two = scale_pair(ks >> (16 * h)), s0 = __byte_perm(two, 0, upper ? 0x3232 : 0x1010), s1 = __byte_perm(two, 0, upper ? 0x1010 : 0x3232);
                    st_shared_values(k_at + h * 1024 + ((k_chunk ^ 0) << 4), upper ? kc[h].z : kc[h].x, s0);
                    st_shared_values(k_at + h * 1024 + ((k_chunk ^ 1) << 4), upper ? kc[h].w : kc[h].y, s0);
                    st_shared_values(k_at + h * 1024 + ((k_chunk ^ 2) << 4), upper ? kc[h].x : kc[h].z, s1);
                    st_shared_values(k_at + h * 1024 + ((k_chunk ^ 3) << 4), upper ? kc[h].y : kc[h].w, s1);
                }
            } else {
                const uint32_t two = scale_pair(ks);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t s0 = __byte_perm(two, 0, h ? 0x3232 : 0x1010);
                    st_shared_values(k_at + h * 1024 + ((k_chunk ^ 0) << 4), kc[h].x, s0);
                    st_shared_values(k_at + h * 1024 + ((k_chunk ^ 1) << 4), kc[h].y, s0);
                }
            }
            if (warp == 8 && lane == 0) s_there[t % kFedRing] = there;
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&bars.k_full[slot]));
                mbar_arrive(smem_u32(&bars.fed[t % kFedRing]));
            }
            ++t;
        };
        // V of tile v, from registers, and whatever is complete with it
        auto feed_v = [&](const VCodes& x) {
            const uint32_t slot = v % kFeedRing, v_at = v_to + slot * L::kVBytes;
            if (v >= kFeedRing) wait_pv_done(v - kFeedRing, kTwVFree);
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t sc = scale_pair(__byte_perm(x.s[s2], 0, h ? v_scale + 0x22 : v_scale));
                    const uint32_t at = v_at + (s2 * 16 + h * 8) * (D == 128 ? 128 : 64);
                    st_shared_values(at + (v_chunk << 4), x.c[s2][h].x, sc);
                    if (D == 128) st_shared_values(at + ((v_chunk ^ 1) << 4), x.c[s2][h].y, sc);
                }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.v_full[slot]));
            ++v;
        };
        // An item is written out one tile behind its last V: that PV may be a tile or two away, and the tiles of the next one go on meanwhile.
        // (No later: the PVs after that wait for the accumulator, and a fourth item for this one's place.)
        auto write_out = [&](uint32_t behind) {
            while (out_k < started && v >= out_end + behind) {
                epilogue(out_k, out_end);
                if (++out_k < started) out_end += s_items[out_k % kTileItems].nt;
            }
        };

#pragma unroll 1
        for (int k = 0; same_in_warp(item_ready(k)); ++k) {
            const TileItem& it = s_items[k % kTileItems];
            const int nt = it.nt;
            if (out_k == k) out_end = t + nt;
            started = k + 1;
            // ---- Q: a row a thread, scaled by a power of two
            if (k > 0) wait(bars.q_free, (k - 1) & 1, kTwQFree);
            {
                const int rr = it.chunk * L::kRows + static_cast<int>(rank) * kTile + row;
                const bool some = rr < it.n * p.G;
                const int tok = quotient(some ? rr : 0, p.div_g), h = it.head * p.G + (some ? rr - tok * p.G : 0);
                const uint4* const src = reinterpret_cast<const uint4*>(p.q + (it.row0 + tok) * p.q_stride + h * D);
                uint32_t top2 = 0u;
#pragma unroll 4
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 x = some ? src[c] : make_uint4(0u, 0u, 0u, 0u);
                    uint32_t a, b;
                    asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(x.x & 0x7fff7fffu), "r"(x.y & 0x7fff7fffu));
                    asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(x.z & 0x7fff7fffu), "r"(x.w & 0x7fff7fffu));
                    asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
                    asm("max.bf16x2 %0, %1, %2;" : "=r"(top2) : "r"(a), "r"(top2));
                }
                const float top = fmaxf(__uint_as_float(top2 << 16), __uint_as_float(top2 & 0xffff0000u));
                const RowPower power(top);
                const float down = power.down();
                s_scale[k & 3][row] = power.up(p.scale_log2);
#pragma unroll 4
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 x = some ? src[c] : make_uint4(0u, 0u, 0u, 0u);
                    uint4 y;
                    y.x = pack_f16x2(__uint_as_float(x.x << 16) * down, __uint_as_float(x.x & 0xffff0000u) * down);
                    y.y = pack_f16x2(__uint_as_float(x.y << 16) * down, __uint_as_float(x.y & 0xffff0000u) * down);
                    y.z = pack_f16x2(__uint_as_float(x.z << 16) * down, __uint_as_float(x.z & 0xffff0000u) * down);
                    y.w = pack_f16x2(__uint_as_float(x.w << 16) * down, __uint_as_float(x.w & 0xffff0000u) * down);
                    *reinterpret_cast<uint4*>(smem + L::kQ + (c >> 3) * L::kQPanelBytes + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = y;
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.q_full));
#pragma unroll 1
            for (int j = 0; j < nt; ++j) {
                load();
                feed_k();
                if (t > 2) feed_v(v_two);
                v_two = v_one;
                v_one = v_now;
                write_out(1);
            }
        }
        if (t > 1) feed_v(v_two);
        if (t > 0) feed_v(v_one);
        write_out(0);
    } else {
        // ----------------------------------------------------------------- softmax, every other key tile
        reg_alloc<184>();
        const int wg = warp >> 2, quarter = warp & 3;
        const int row = tid & 127;
        constexpr int kPassMax = 0, kPassTurn = 8;
        const uint32_t lane_off = static_cast<uint32_t>(quarter * 32) << 16;
        const uint32_t p_bar = map_to_cta(smem_u32(&bars.p_full[wg]), 0), s_read_bar = map_to_cta(smem_u32(&bars.s_read[wg]), 0);
        const uint32_t tS = tmem_base + wg * kTile + lane_off, tP = tmem_base + kTileTmemP + wg * (kTile / 2) + lane_off;
        const uint32_t tO = tmem_base + kTileTmemO + lane_off;
        uint32_t t0 = 0;
#pragma unroll 1
        for (int k = 0; same_in_warp(item_ready(k)); ++k) {
            const TileItem& it = s_items[k % kTileItems];
            const int nt = same_in_warp(it.nt), first_tile = same_in_warp(it.t0), ns = same_in_warp(it.ns), skip = same_in_warp(it.skip);
            const int base = it.len - it.n, rr0 = it.chunk * L::kRows + static_cast<int>(rank) * kTile, rows = it.n * p.G;
            // positions of this thread's row and of the CTA's first and last; rows that do not exist go along with the last one
            const int pos = base + quotient(min(rr0 + row, rows - 1), p.div_g);
            const int pos_min = same_in_warp(base + quotient(min(rr0, rows - 1), p.div_g)), pos_max = same_in_warp(base + quotient(min(rr0 + kTile - 1, rows - 1), p.div_g));
            __syncwarp();
            if (lane == 0) item_release(k);
            float m_own = -INFINITY, l_run = 0.f, scale = 0.f;
            const int first = static_cast<int>((t0 ^ static_cast<uint32_t>(wg)) & 1u);
#pragma unroll 1
            for (int j = first; j < nt; j += 2) {
                const uint32_t t = t0 + j;
                const int key0 = (first_tile + j < ns ? first_tile + j : first_tile + j + skip) << 7;
                wait(bars.fed[t % kFedRing], (t / kFedRing) & 1, kTwFed);
                const unsigned there = same_in_warp(s_there[t % kFedRing]);
                if (j == first) scale = s_scale[k & 3][row];
                wait_s_full(t, kTwS);
                tc_fence_after_sync();
                uint32_t r[kTile];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&r[32 * c]));
                tmem_wait_ld();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(s_read_bar);
                if (key0 + kTile - 1 > pos_min) {  // some row's position is within the tile, or before it
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int cols = pos + 1 - key0 - c * 32;  // visible ones of this part
                        if (__all_sync(0xffffffffu, cols >= 32)) continue;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i >= cols) r[c * 32 + i] = 0xff800000u;  // -inf
                    }
                }
                if (p.window > 0 && key0 <= pos_max - p.window && key0 + kTile > p.sink) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int from = p.sink - key0 - c * 32, to = pos - p.window + 1 - key0 - c * 32;  // hidden ones of this part
                        if (__all_sync(0xffffffffu, to <= 0 || from >= 32)) continue;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i >= from && i < to) r[c * 32 + i] = 0xff800000u;
                    }
                }
                if (there != 0xffu) {  // pages that are not there
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if ((there >> (2 * c) & 3u) == 3u) continue;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (!(there >> (2 * c + i / 16) & 1u)) r[c * 32 + i] = 0xff800000u;
                    }
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int i = 0; i < kTile; i += 8) {
#pragma unroll
                    for (int a = 0; a < 4; ++a)
                        mx[a] = fmax3(mx[a], __uint_as_float(r[i + 2 * a]), __uint_as_float(r[i + 2 * a + 1]));
                }
                const float m_tile = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                float m_prev = -INFINITY;
                if (t > 0) {
                    turn_wait(kPassMax, wg, quarter);
                    if (j > 0) m_prev = s_max[wg ^ 1][row];
                }
                float m_ref = m_prev;
                if ((m_tile - m_prev) * scale > kTileRescaleLog2 || m_prev == -INFINITY) m_ref = fmaxf(m_prev, m_tile);
                s_max[wg][row] = m_ref;
                turn_pass(kPassMax, wg, quarter);
                if (j > 0 && __any_sync(0xffffffffu, m_ref != m_prev)) {
                    const float alpha = m_ref == m_prev ? 1.f : fast_exp2((m_prev - m_ref) * scale);
                    wait_pv_done(t - 1, kTwPV);
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        tmem_ld16(tO + c * 16, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                        tmem_st16(tO + c * 16, o);
                    }
                }
                if (t >= 2) wait_pv_done(t - 2, kTwPFree);
                if (t > 0) turn_wait(kPassTurn, wg, quarter);
                const float neg_ms = (m_ref == -INFINITY) ? 0.f : fmaf(-m_ref, scale, kHeadroom);
                const uint64_t scale2 = pack_f32x2(scale, scale);
                const uint64_t shift2 = pack_f32x2(neg_ms, neg_ms);
                uint64_t sm2[4] = {0ull, 0ull, 0ull, 0ull};
                uint32_t pk[kTile / 2];
#pragma unroll
                for (int i = 0; i < kTile / 2; ++i) {
                    const uint64_t t2 = fma_f32x2(pack_f32x2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), scale2, shift2);
                    float e0, e1;
                    unpack_f32x2(t2, e0, e1);
                    const float p0 = fast_exp2(e0), p1 = fast_exp2(e1);
                    sm2[i & 3] = add_f32x2(sm2[i & 3], pack_f32x2(p0, p1));
                    pk[i] = pack_probabilities(p0, p1);
                    if (i % 16 == 15) tmem_st16(tP + i - 15, &pk[i - 15]);
                    if (i == kTileTurn) turn_pass(kPassTurn, wg, quarter);
                }
                tmem_wait_st();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(p_bar);
                float a0, a1, b0, b1;
                unpack_f32x2(add_f32x2(sm2[0], sm2[1]), a0, a1);
                unpack_f32x2(add_f32x2(sm2[2], sm2[3]), b0, b1);
                const float sum = (a0 + a1) + (b0 + b1);
                l_run = (m_own == m_ref ? l_run : l_run * fast_exp2((m_own - m_ref) * scale)) + sum;
                m_own = m_ref;
            }
            t0 += nt;
            s_sums[k % kTileSums][first][row] = make_float2(l_run, m_own);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.sums_full[k % kTileSums]));
        }
        if (t0 > 0 && static_cast<uint32_t>(wg) == (t0 & 1u)) {  // the last tile's passes
            turn_wait(kPassMax, wg, quarter);
            turn_wait(kPassTurn, wg, quarter);
        }
    }
    // as in attn_kernel.cu: what an expired wait left in flight lands before anyone leaves
    if (*static_cast<volatile int*>(&wait_state.expired) != 0) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
    }
    tc_fence_before_sync();
    __syncwarp();
    cluster_sync_all();
    if (warp == 12) {
        __syncwarp();
        tmem_dealloc_pair(tmem_base, 512);
    }
    if (tid == 0 && wait_state.expired != 0) {
        const int detail = wait_state.expired * 1000000 + blockIdx.x;
        if (atomicCAS(&p.hdr->status, 0, PEVLM_ETIMEOUT) == 0) p.hdr->detail = detail;
    }
}

cudaError_t launch_packed_tile(const PackedAttnParams& p, int head_dim, cudaStream_t stream) {
    return head_dim == 128 ? launch_chained<packed_tile_kernel<128>>(dim3(kNumSms), kTileThreads, 1024 + PackedTileLayout<128>::kTotal, stream, p)
                           : launch_chained<packed_tile_kernel<64>>(dim3(kNumSms), kTileThreads, 1024 + PackedTileLayout<64>::kTotal, stream, p);
}

}  // namespace pevlm
