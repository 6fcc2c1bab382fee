// Attention over the packed cache (4-bit keys and values in pages) for a few rows per sequence and kv head: one generated token,
// drafted tokens, short questions.
//
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j  over the keys j <= pos_i that the window leaves
//
// Work is counted in tiles of 16 keys.  A unit is what one result needs: (sequence, kv head, chunk of 8 * NT rows); its tiles, and the
// units one after another, make one long list, of which every warp of the launch takes an equal part, whatever the
// lengths of the sequences are.  A unit that lies within a warp's part is written by the warp; the others leave the warp's
// share in shared memory (two at most: the unit its part begins with and the one it ends with), where the CTA joins them, and what then
// still crosses into another CTA goes to the workspace for the launch behind (packed_merge_kernel), which joins it in the order of the
// CTAs: results do not depend on timing.
//
// Inside a warp nothing waits for other warps: it fetches its tiles (a page of a kv head is a run of them, 2,304 bytes each at
// head_dim 128) into a ring of its own with cp.async and forms S^T = K Q^T and O^T += V^T P^T with mma.sync m16n8k16 in fp16,
// where both the keys' values (e2m1 x e4m3, at most 6 significant bits, 2^-10 .. 2688) and their products with the scales are exact.
// The 16 rows of an MMA are keys (or elements of the head), its 8 columns query rows: few of them are idle with the 7 or 8 heads of a
// group, where tcgen05's smallest tile has 128 rows.  The format keeps together what a thread holds: k-steps of S take
// elements 32 t + 4 s .. + 3 of the head (thread t of four; Q's fragments are cut the same way, the order of a sum's terms is
// free), the rows of V^T are elements 16 g + 2 i, + 1, so a thread needs 16 bytes of codes of two keys, 8 bytes of four, and one scale for
// all of them.  Probabilities change from the result's layout to the operand's by movmatrix.
// Rows of Q are scaled by a power of two, so that any bf16 values fit fp16: exactly, down to 2^-31 of the row's largest (RowPower in packed_list.cuh;
// with S in bf16, whose conversions of the keys take three instructions a pair more, the 64 sequences below took 85.7 us); sums, maxima and outputs are fp32.  Probabilities are rounded to fp16
// (2^-11 of each; 2^-32 of the running reference where smaller, see kHeadroom).
// What bounds it: large batches HBM (64 sequences of up to 16K keys, 28/4 heads: 304 MB at 6 TB/s while the warps are in their loops, 55 of 72 us;
// the start, the slowest warps, the join and the merge are the rest); small ones the chain lengths -> part -> pages -> tiles -> join -> merge
// and the instructions (277 of a warp a tile of 16 keys, 128 of them the conversions and the products with the scales; half of the ALU's
// throughput, which conversions share, is in use).  One token against 50K keys (29 MB) 17.8 us, of which 6 in the loop; 16 sequences of heads of
// 64 under a window (38 MB) 27.8.  Two tiles a step (two chains of dependent products): 116 -> 77.5 us for the 64 sequences.
#include "packed_list.cuh"

namespace pevlm {

template <int D, int NT>
struct PackedAttnLayout {
    static constexpr int kWarps = D == 128 ? (NT == 1 ? 12 : 8) : (NT == 1 ? 16 : 12);  // as many as the registers allow, the same for each scheduler
    static constexpr int kStages = D == 128 ? 3 + (NT == 2) : 5;  // steps (two tiles) in a warp's ring
    static constexpr int kTileBytes = 18 * D, kStepBytes = 2 * kTileBytes;
    static constexpr int kRows = 8 * NT;
    static constexpr int kShareFloats = kRows * (D + 2);          // O [rows][D], then m and l of each row
    static constexpr int kRing = kWarps * kStages * kStepBytes;
    static constexpr int kTotal = kRing + kWarps * kShareFloats * 4;
    static_assert(kShareFloats * 4 <= kStages * kStepBytes, "the second share of a warp is left in its ring");
};

constexpr int kSeqsPerLane = 4;  // up to 128 sequences are looked over by every warp for itself
constexpr int kTableSeqs = 32 * kSeqsPerLane;

// `table`: shared memory for the sequences' descriptions, where there are at most kTableSeqs (every warp writes the same).
template <int W>
__device__ __forceinline__ PackedPart my_part(const PackedAttnParams& p, int rows_per_chunk, PackedSeq* table) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, me = blockIdx.x * W + warp;
    if (p.num_seqs <= kTableSeqs) {  // each warp for itself, neighbouring sequences in a lane
        const int each = (p.num_seqs + 31) / 32, r0 = lane * each;
        PackedSeq s[kSeqsPerLane];
        int64_t upto[kSeqsPerLane], mine = 0;
        int len[kSeqsPerLane], start[kSeqsPerLane + 1];  // all in flight together
#pragma unroll
        for (int i = 0; i <= kSeqsPerLane; ++i) {
            if (i < kSeqsPerLane) len[i] = i < each && r0 + i < p.num_seqs ? p.lens[r0 + i] : 0;
            start[i] = i <= each && r0 + i <= p.num_seqs ? p.row_start[r0 + i] : 0;
        }
#pragma unroll
        for (int i = 0; i < kSeqsPerLane; ++i) {
            s[i] = {0, 0, 0, 0, 1, 0, 0};
            if (i < each && r0 + i < p.num_seqs) table[r0 + i] = s[i] = packed_seq<4>(p, len[i], start[i], start[i + 1], rows_per_chunk);
            mine += seq_tiles<4>(p, s[i]);
            upto[i] = mine;
        }
        __syncwarp();  // the table, for all lanes
        const int64_t to = warp_inclusive(mine), from = to - mine;
        PackedPart part{PackedDeal(__shfl_sync(0xffffffffu, to, 31), gridDim.x * W), 0, 0, s[0]};
        const int64_t lo = part.deal.start(me);
        const int owner = max(__ffs(__ballot_sync(0xffffffffu, to > lo)) - 1, 0);
        // in its owner's lane: which of its sequences
        part.seq = r0;
        part.off = lo - from;
#pragma unroll
        for (int i = 1; i < kSeqsPerLane; ++i)
            if (lo - from >= upto[i - 1]) {
                part.seq = r0 + i;
                part.off = lo - from - upto[i - 1];
                part.s = s[i];
            }
        part.seq = __shfl_sync(0xffffffffu, part.seq, owner);
        part.off = __shfl_sync(0xffffffffu, part.off, owner);
        part.s.len = __shfl_sync(0xffffffffu, part.s.len, owner);
        part.s.n = __shfl_sync(0xffffffffu, part.s.n, owner);
        part.s.row0 = __shfl_sync(0xffffffffu, part.s.row0, owner);
        part.s.chunks = __shfl_sync(0xffffffffu, part.s.chunks, owner);
        part.s.cnt = __shfl_sync(0xffffffffu, part.s.cnt, owner);
        part.s.ns = __shfl_sync(0xffffffffu, part.s.ns, owner);
        part.s.skip = __shfl_sync(0xffffffffu, part.s.skip, owner);
        return part;
    }
    // a thread for every sequence, W * 32 at a time
    __shared__ int64_t s_sum[W], s_off[W];
    __shared__ int s_seq[W];
    int64_t sum = 0;
    for (int r = threadIdx.x; r < p.num_seqs; r += W * 32) sum += seq_tiles<4>(p, packed_seq<4>(p, r, rows_per_chunk));
    sum = warp_inclusive(sum);
    if (lane == 31) s_sum[warp] = sum;
    __syncthreads();
    int64_t total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) total += s_sum[w];
    PackedPart part{PackedDeal(total, gridDim.x * W), 0, 0, {}};
    int64_t base = 0;
    for (int r0 = 0; r0 < p.num_seqs; r0 += W * 32) {
        const int r = r0 + threadIdx.x;
        const int64_t mine = r < p.num_seqs ? seq_tiles<4>(p, packed_seq<4>(p, r, rows_per_chunk)) : 0;
        int64_t to = warp_inclusive(mine);
        __syncthreads();
        if (lane == 31) s_sum[warp] = to;
        __syncthreads();
        int64_t all = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            if (w < warp) to += s_sum[w];
            all += s_sum[w];
        }
        to += base;
        const int64_t from = to - mine;
        if (from < part.deal.start(blockIdx.x * W + W) && to > part.deal.start(blockIdx.x * W)) {
            for (int w = 0; w < W; ++w) {
                const int64_t lo = part.deal.start(blockIdx.x * W + w);
                if (lo >= from && lo < to) {
                    s_seq[w] = r;
                    s_off[w] = lo - from;
                }
            }
        }
        base += all;
    }
    __syncthreads();
    if (part.deal.start(me) < total) {
        part.seq = s_seq[warp];
        part.off = s_off[warp];
        part.s = packed_seq<4>(p, part.seq, rows_per_chunk);
    }
    return part;
}

__device__ __forceinline__ void mma16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t m) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(m));
    return r;
}
template <int D, int NT>
__global__ void __launch_bounds__(PackedAttnLayout<D, NT>::kWarps * 32, 1) packed_attn_kernel(const __grid_constant__ PackedAttnParams p) {
    using L = PackedAttnLayout<D, NT>;
    constexpr int W = L::kWarps, KS = D / 16, MT = D / 16;  // k-steps of S, row tiles of V^T
    constexpr int kWords = D / 32;                          // words of codes: of a key in a thread of S; twice what an eighth of the head has
    constexpr int kChunks = L::kTileBytes / 16;             // of 16 bytes
    extern __shared__ __align__(128) uint8_t raw[];
    struct Share {       // a share left for the CTA to join
        int64_t u0, u1;  // tiles of its unit, counted over the whole list
        int r, head, chunk, row0, n;
    };
    __shared__ Share s_share[2 * W];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint8_t* const my_ring = raw + warp * L::kStages * L::kStepBytes;
    const uint32_t ring = smem_u32(my_ring);
    // a warp's first share has a place of its own, the second, with which its part ends, takes the ring
    auto share_at = [&](int slot) { return reinterpret_cast<float*>(slot & 1 ? raw + (slot >> 1) * L::kStages * L::kStepBytes : raw + L::kRing + (slot >> 1) * L::kShareFloats * 4); };
    if (lane < 2) s_share[2 * warp + lane].u1 = -1;
    __syncwarp();
    grid_wait();

    __shared__ PackedSeq s_seqs[kTableSeqs];
    const PackedSeq* const table = p.num_seqs <= kTableSeqs ? s_seqs : nullptr;
    const PackedPart part = my_part<W>(p, L::kRows, s_seqs);
    const PackedDeal& deal = part.deal;
    const int64_t lo = deal.start(blockIdx.x * W + warp), hi = deal.start(blockIdx.x * W + warp + 1);
    grid_launch_dependents();
    if (lo < hi) {
        // Fetching: steps of two tiles.  A lane holds the place of a tile, of 32 tiles, and the pages of the 32 behind them and of the
        // first 32 of the next unit (`after`), so that a page is looked up long before it is needed.
        int at;
        PackedUnit<4> cur(part, at), after(cur);
        // Places [from, from + kUnitTiles<4>) of the list belong to a unit, its tiles follow.  Those of it that are in the part:
        int64_t unit0 = lo - at + kUnitTiles<4>;  // of the unit's first tile
        int first_tile = max(at - kUnitTiles<4>, 0);
        auto tiles_of = [&](const PackedUnit<4>& u, int64_t tile0) { return static_cast<int>(max(min(hi - tile0, static_cast<int64_t>(u.s.cnt)), static_cast<int64_t>(0))); };
        // (a unit that the part does not reach is not looked for)
        auto to_next = [&](PackedUnit<4>& u, int64_t tile0) {
            if (tile0 < hi) u.next(p, L::kRows, table);
            else u.r = p.num_seqs;
        };
        to_next(after, unit0 + cur.s.cnt + kUnitTiles<4>);
        int64_t fetch0 = unit0;                          // the same of the unit that is fetched
        int left = tiles_of(cur, fetch0) - first_tile;   // and its tiles that are yet to be
        int in_block = 0, block = first_tile;            // of 32 places, and their first tile
        PackedUnit<4> ahead(cur);                           // the unit that is fetched
        auto page_of = [&](const PackedUnit<4>& u, int x) { return u.r < p.num_seqs && x < u.s.cnt ? packed_page(p, u.r, u.s.len, u.key0(x) >> 4) : -1; };
        auto place_of = [&](const PackedUnit<4>& u, int x, int page) { return packed_place(p, page, u.head, u.key0(x) >> 4, L::kTileBytes / 128); };
        int page = page_of(ahead, block + lane), page_next = page_of(ahead, block + 32 + lane), page_after = page_of(after, lane);
        // Rows of the unit: Q's fragments, the softmax scale in units of log2 and the positions of rows 2 t and 2 t + 1.
        uint32_t q[NT][KS][2];
        float sc[NT][2];
        int pos[NT][2];
        uint32_t raw_q[NT][KS * 2];
        auto ask_for_rows = [&]() {
            const int rows = min(cur.s.n * p.G - cur.chunk * L::kRows, L::kRows);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int rr = cur.chunk * L::kRows + 8 * j + g;
                if (8 * j + g < rows) {
                    const int tok = quotient(rr, p.div_g), h = cur.head * p.G + rr - tok * p.G;
                    const __nv_bfloat16* src = p.q + (cur.s.row0 + tok) * p.q_stride + h * D + t * (D / 4);
#pragma unroll
                    for (int c = 0; c < KS / 2; ++c) *reinterpret_cast<uint4*>(&raw_q[j][4 * c]) = reinterpret_cast<const uint4*>(src)[c];  // through L1: all warps of the SM read these rows
                } else {
#pragma unroll
                    for (int c = 0; c < KS * 2; ++c) raw_q[j][c] = 0u;
                }
            }
        };
        auto rows_of_unit = [&]() {
            const int rows = min(cur.s.n * p.G - cur.chunk * L::kRows, L::kRows);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                uint32_t (&x)[KS * 2] = raw_q[j];
                float top = 0.f;
#pragma unroll
                for (int c = 0; c < KS * 2; ++c) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(x[c] << 16)), fabsf(__uint_as_float(x[c] & 0xffff0000u))));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const RowPower power(top);
                const float down = power.down(), up = power.up(p.scale_log2);
#pragma unroll
                for (int c = 0; c < KS * 2; ++c)
                    q[j][c >> 1][c & 1] = pack_f16x2(__uint_as_float(x[c] << 16) * down, __uint_as_float(x[c] & 0xffff0000u) * down);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    sc[j][b] = __shfl_sync(0xffffffffu, up, 8 * t + 4 * b);
                    const int row = 8 * j + 2 * t + b;
                    pos[j][b] = row < rows ? cur.s.len - cur.s.n + quotient(cur.chunk * L::kRows + row, p.div_g) : -1;
                }
            }
        };
        // Q's rows of a unit that comes into L1, one line a lane
        auto prefetch_rows = [&](const PackedUnit<4>& u) {
            constexpr int kLines = D / 64;
            const int rows = min(u.s.n * p.G - u.chunk * L::kRows, L::kRows);
#pragma unroll
            for (int x = lane; x < L::kRows * kLines; x += 32) {
                if (x / kLines >= rows) break;
                const int rr = u.chunk * L::kRows + x / kLines, tok = quotient(rr, p.div_g), h = u.head * p.G + rr - tok * p.G;
                asm volatile("prefetch.global.L1 [%0];" ::"l"(p.q + (u.s.row0 + tok) * p.q_stride + h * D + x % kLines * 64));
            }
        };
        ask_for_rows();
        uint32_t places = place_of(ahead, block + lane, page);
        unsigned there = 0;  // two bits a step, the latest in the lowest: the tiles exist
        const uint8_t* const cache = p.cache + lane * 16;
        uint32_t into = 0;   // place in the ring
        auto fetch = [&]() {
            there <<= 2;
            if (left > 0) {
                const uint32_t at0 = __shfl_sync(0xffffffffu, places, in_block);
                uint32_t at1 = __shfl_sync(0xffffffffu, places, in_block + 1);
                if (left == 1) at1 = kNoTile;
                there |= (at0 != kNoTile ? 1u : 0u) | (at1 != kNoTile ? 2u : 0u);
                const uint8_t* const src0 = cache + static_cast<uint64_t>(at0) * 128;
                const uint8_t* const src1 = cache + static_cast<uint64_t>(at1) * 128 - kChunks % 32 * 16;
                const uint32_t dst = ring + lane * 16 + into;
                // the chunks of both tiles, 32 at a time: those in the middle are of one or the other (kChunks % 32 = 16 or 8)
#pragma unroll
                for (int c = 0; c < (2 * kChunks + 31) / 32; ++c) {
                    const bool first = c < kChunks / 32 || (c == kChunks / 32 && lane < kChunks % 32);
                    const uint8_t* const src = first ? src0 + c * 512 : src1 + (c - kChunks / 32) * 512;
                    const bool some = (first ? at0 : at1) != kNoTile && ((c + 1) * 32 <= 2 * kChunks || c * 32 + lane < 2 * kChunks);
                    if (some) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + c * 512), "l"(src) : "memory");
                }
                into = into + L::kStepBytes == L::kStages * L::kStepBytes ? 0 : into + L::kStepBytes;
                in_block += 2;
                left -= 2;
                if (left <= 0) {
                    fetch0 += ahead.s.cnt + kUnitTiles<4>;
                    if (fetch0 < hi) {
                        ahead = after;
                        left = tiles_of(ahead, fetch0);
                        in_block = block = 0;
                        places = place_of(ahead, lane, page_after);
                        page_next = page_of(ahead, 32 + lane);
                        to_next(after, fetch0 + ahead.s.cnt + kUnitTiles<4>);
                        page_after = page_of(after, lane);
                        prefetch_rows(ahead);
                    }
                } else if (in_block == 32) {
                    in_block = 0;
                    block += 32;
                    places = place_of(ahead, block + lane, page_next);
                    page_next = page_of(ahead, block + 32 + lane);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int i = 0; i < L::kStages - 1; ++i) fetch();
        rows_of_unit();

        uint32_t from_place = 0;
        bool first_unit = true;
        while (unit0 < hi) {
            // ------------------------------------------------ a unit, or the share of it that is in this part
            const int tiles = tiles_of(cur, unit0) - first_tile;
            const int rows = min(cur.s.n * p.G - cur.chunk * L::kRows, L::kRows);
            float m[NT][2], l[NT][2], o[NT][MT][4];
            if (!first_unit) {
                ask_for_rows();
                rows_of_unit();
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    m[j][b] = kNoMax;
                    l[j][b] = 0.f;
                }
#pragma unroll
                for (int c = 0; c < MT; ++c) o[j][c][0] = o[j][c][1] = o[j][c][2] = o[j][c][3] = 0.f;
            }
            const int pos_min = cur.s.len - cur.s.n + quotient(cur.chunk * L::kRows, p.div_g);
            const int pos_max = cur.s.len - cur.s.n + quotient(cur.chunk * L::kRows + rows - 1, p.div_g);
            int open_from, open_to;
            cur.open_tiles(p, pos_min, pos_max, open_from, open_to);
            for (int n = first_tile; n < first_tile + tiles; n += 2) {
                asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 2) : "memory");
                __syncwarp();  // this step is there for all lanes, and all have read the one before, whose place is filled again
                const unsigned exist = there >> (2 * (L::kStages - 2)) & 3u;
                fetch();
                const uint8_t* const step = my_ring + from_place;
                from_place = from_place + L::kStepBytes == L::kStages * L::kStepBytes ? 0 : from_place + L::kStepBytes;
                if (exist == 0) continue;
                // S^T: keys g and g + 8 of either tile, rows 2 t and 2 t + 1
                float s[NT][2][4];
                uint32_t vs[2][2];  // V's scales of keys 2 t, 2 t + 1 and 2 t + 8, 2 t + 9
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint8_t* const tile = step + x * L::kTileBytes;
#pragma unroll
                    for (int j = 0; j < NT; ++j) s[j][x][0] = s[j][x][1] = s[j][x][2] = s[j][x][3] = 0.f;
                    uint32_t kw[2][kWords], ks[2][2];  // codes and scales (twice in a word) of keys g and g + 8
                    if (D == 128) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) *reinterpret_cast<uint4*>(&kw[h][0]) = *reinterpret_cast<const uint4*>(tile + h * 512 + lane * 16);
                        const uint32_t sb = *reinterpret_cast<const uint32_t*>(tile + 16 * D + lane * 4);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t two = scale_pair(sb >> (16 * h));
                            ks[h][0] = __byte_perm(two, 0, 0x1010);
                            ks[h][1] = __byte_perm(two, 0, 0x3232);
                        }
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; ++h) *reinterpret_cast<uint2*>(&kw[h][0]) = *reinterpret_cast<const uint2*>(tile + h * 256 + lane * 8);
                        const uint32_t two = scale_pair(*reinterpret_cast<const uint16_t*>(tile + 16 * D + lane * 2));
                        ks[0][0] = ks[0][1] = __byte_perm(two, 0, 0x1010);
                        ks[1][0] = ks[1][1] = __byte_perm(two, 0, 0x3232);
                    }
#pragma unroll
                    for (int w = 0; w < kWords; ++w) {
                        uint32_t a[2][4];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            halves_of_word(kw[h][w], a[h]);
#pragma unroll
                            for (int b = 0; b < 4; ++b) a[h][b] = mul_f16x2(a[h][b], ks[h][w >> 1]);
                        }
#pragma unroll
                        for (int half = 0; half < 2; ++half)
#pragma unroll
                            for (int j = 0; j < NT; ++j)
                                mma16816_f16(s[j][x], a[0][2 * half], a[1][2 * half], a[0][2 * half + 1], a[1][2 * half + 1], q[j][2 * w + half][0], q[j][2 * w + half][1]);
                    }
                    const uint32_t vb = *reinterpret_cast<const uint32_t*>(tile + 17 * D + (D == 128 ? lane * 4 : (g >> 1) * 16 + t * 4));
                    vs[x][0] = scale_pair(vb);
                    vs[x][1] = scale_pair(vb >> 16);
                }
                // masks, and scales of 0 for V of keys that no row sees, whose bytes may be anything
                if (exist != 3u || n < open_from || n + 1 >= open_to) {
                    const int key0[2] = {cur.key0(n), cur.key0(n + 1)};
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const bool is_there = exist >> x & 1;
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int key = key0[x] + g + (e >> 1) * 8, at = pos[j][e & 1];
                                if (!is_there || key > at || (p.window > 0 && key <= at - p.window && key >= p.sink)) s[j][x][e] = -INFINITY;
                            }
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int key = key0[x] + 8 * h + 2 * t;
                            auto nobody_sees = [&](int k) { return !is_there || k >= cur.s.len || (p.window > 0 && k <= pos_min - p.window && k >= p.sink); };
                            if (nobody_sees(key)) vs[x][h] &= 0xffff0000u;
                            if (nobody_sees(key + 1)) vs[x][h] &= 0x0000ffffu;
                        }
                    }
                }
                uint32_t pb[NT][2][2];
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    float y[2][4], most = -INFINITY;
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            y[x][e] = fmaf(s[j][x][e], sc[j][e & 1], -m[j][e & 1]);
                            most = fmaxf(most, y[x][e]);
                        }
                    // m, which stands kHeadroom below the reference maximum, moves when a score is more than 2^8 above that
                    if (__any_sync(0xffffffffu, most > 8.f + kHeadroom)) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            float top = fmaxf(fmaxf(s[j][0][b], s[j][0][2 + b]), fmaxf(s[j][1][b], s[j][1][2 + b])) * sc[j][b];
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                            const float to = fmaxf(m[j][b], top - kHeadroom), alpha = fast_exp2(m[j][b] - to);
                            m[j][b] = to;
                            l[j][b] *= alpha;
#pragma unroll
                            for (int c = 0; c < MT; ++c) {
                                o[j][c][b] *= alpha;
                                o[j][c][2 + b] *= alpha;
                            }
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                y[x][b] = fmaf(s[j][x][b], sc[j][b], -to);
                                y[x][2 + b] = fmaf(s[j][x][2 + b], sc[j][b], -to);
                            }
                        }
                    }
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[x][e] = fast_exp2(y[x][e]);
                        pb[j][x][0] = transposed(pack_probabilities(y[x][0], y[x][1]));
                        pb[j][x][1] = transposed(pack_probabilities(y[x][2], y[x][3]));
                    }
                    l[j][0] += (y[0][0] + y[0][2]) + (y[1][0] + y[1][2]);
                    l[j][1] += (y[0][1] + y[0][3]) + (y[1][1] + y[1][3]);
                }
                // O^T: elements 16 g + 2 i, + 1 (8 g at head_dim 64) of keys 2 t, 2 t + 1 and those 8 further on
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint8_t* const tile = step + x * L::kTileBytes;
                    uint32_t vw[2][2][kWords / 2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (D == 128) {
                            const uint4 v = *reinterpret_cast<const uint4*>(tile + 8 * D + h * 512 + lane * 16);
                            vw[h][0][0] = v.x; vw[h][0][kWords / 2 - 1] = v.y; vw[h][1][0] = v.z; vw[h][1][kWords / 2 - 1] = v.w;
                        } else {
                            const uint2 v = *reinterpret_cast<const uint2*>(tile + 8 * D + h * 256 + lane * 8);
                            vw[h][0][0] = v.x; vw[h][1][0] = v.y;
                        }
                    }
#pragma unroll
                    for (int w = 0; w < kWords / 2; ++w) {
                        uint32_t a[2][2][4];  // [keys][even, odd element]
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t lo = vw[h][0][w], hi = vw[h][1][w];
                            halves_of_word((lo & 0x0f0f0f0fu) | (hi << 4 & 0xf0f0f0f0u), a[h][0]);
                            halves_of_word((lo >> 4 & 0x0f0f0f0fu) | (hi & 0xf0f0f0f0u), a[h][1]);
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                a[h][0][b] = mul_f16x2(a[h][0][b], vs[x][h]);
                                a[h][1][b] = mul_f16x2(a[h][1][b], vs[x][h]);
                            }
                        }
#pragma unroll
                        for (int b = 0; b < 4; ++b)
#pragma unroll
                            for (int j = 0; j < NT; ++j) mma16816_f16(o[j][4 * w + b], a[0][0][b], a[0][1][b], a[1][0][b], a[1][1][b], pb[j][x][0], pb[j][x][1]);
                    }
                }
            }
            __syncwarp();

            // ------------------------------------------------ its end
            const bool ends = first_tile + tiles == cur.s.cnt, whole = first_tile == 0 && ends;
            const int slot = 2 * warp + (first_unit ? 0 : 1);  // the part begins with it, or ends with it
            float* const share = share_at(slot);
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    float sum = l[j][b];
                    sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                    const int row = 8 * j + 2 * t + b;
                    if (whole) {
                        if (row >= rows) continue;
                        const PackedRow at = packed_row(p, cur.s.row0, cur.head, cur.chunk * L::kRows + row, D);
                        const float inv = sum > 0.f ? 1.f / sum : 0.f;
                        uint32_t w[MT];
#pragma unroll
                        for (int c = 0; c < MT; ++c) w[c] = pack_bf16x2(o[j][c][b] * inv, o[j][c][2 + b] * inv);
                        uint4* const to = reinterpret_cast<uint4*>(p.o + at.o + g * (D / 8));
#pragma unroll
                        for (int c = 0; c < MT / 4; ++c) to[c] = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
                        if (g == 0 && p.lse) p.lse[at.lse] = sum > 0.f ? (m[j][b] + log2f(sum)) * 0.693147180559945309f : -INFINITY;
                    } else {
                        float4* const to = reinterpret_cast<float4*>(share + row * D + g * (D / 8));
#pragma unroll
                        for (int c = 0; c < MT / 2; ++c) to[c] = make_float4(o[j][2 * c][b], o[j][2 * c][2 + b], o[j][2 * c + 1][b], o[j][2 * c + 1][2 + b]);
                        if (g == 0) {
                            share[L::kRows * D + row] = m[j][b];
                            share[L::kRows * (D + 1) + row] = sum;
                        }
                    }
                }
            if (!whole && lane == 0) s_share[slot] = {unit0, unit0 + cur.s.cnt, cur.r, cur.head, cur.chunk, cur.s.row0, cur.s.n};
            unit0 += cur.s.cnt + kUnitTiles<4>;
            first_unit = false;
            first_tile = 0;
            to_next(cur, unit0);
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    __syncthreads();

    // ---------------------------------------------------- shares of one unit stand one after another
    const int64_t cta_lo = deal.start(blockIdx.x * W), cta_hi = deal.start(blockIdx.x * W + W);
    PackedJoin join{0, 0, 0, 0, 0, 0};
    __shared__ float s_factor[2 * W][L::kRows];  // what each share of a row counts
    __shared__ int s_list[2 * W];                // the shares of the unit
    const int64_t u0_of = lane < 2 * W && s_share[lane].u1 >= 0 ? s_share[lane].u0 : -1;
    unsigned left_over = __ballot_sync(0xffffffffu, u0_of >= 0);
    while (left_over != 0) {
        const int a = __ffs(left_over) - 1;
        const Share u = s_share[a];
        const unsigned group = __ballot_sync(0xffffffffu, u0_of == u.u0);
        left_over &= ~group;
        const bool done = u.u0 >= cta_lo && u.u1 <= cta_hi;
        const int rows = min(u.n * p.G - u.chunk * L::kRows, L::kRows), count = __popc(group);
        // the place in the workspace: the first if this CTA's part begins with the unit
        const int second = u.u0 > cta_lo;
        float* const left = p.part + (2 * static_cast<int64_t>(blockIdx.x) + second) * L::kShareFloats;
        if (!done && u.u0 >= cta_lo) join = {deal.worker_of(u.u1 - 1) / W, second, u.row0, u.n, u.head, u.chunk};
        // a warp for a row, a lane for a share
        const bool in = group >> lane & 1;
        const int at = __popc(group & ((1u << lane) - 1));
        if (warp == 0 && in) s_list[at] = lane;
        for (int row = warp; row < rows; row += W) {
            const float m = in ? share_at(lane)[L::kRows * D + row] : kNoMax, l = in ? share_at(lane)[L::kRows * (D + 1) + row] : 0.f;
            float top = m;
#pragma unroll
            for (int by = 16; by > 0; by /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, by));
            const float f = fast_exp2(m - top);
            float sum = f * l;
#pragma unroll
            for (int by = 16; by > 0; by /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, by);
            if (in) s_factor[at][row] = done ? (sum > 0.f ? f / sum : 0.f) : f;
            if (lane == 0) {
                if (!done) {
                    left[L::kRows * D + row] = top;
                    left[L::kRows * (D + 1) + row] = sum;
                } else if (p.lse) {
                    p.lse[packed_row(p, u.row0, u.head, u.chunk * L::kRows + row, D).lse] = sum > 0.f ? (top + log2f(sum)) * 0.693147180559945309f : -INFINITY;
                }
            }
        }
        __syncthreads();
        for (int x = threadIdx.x; x < rows * (D / 4); x += W * 32) {
            const int row = x / (D / 4), c = x % (D / 4);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int i = 0; i < count; ++i) {
                const float f = s_factor[i][row];
                const float4 v = reinterpret_cast<const float4*>(share_at(s_list[i]) + row * D)[c];
                acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
            }
            if (done)
                reinterpret_cast<uint2*>(p.o + packed_row(p, u.row0, u.head, u.chunk * L::kRows + row, D).o)[c] = make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
            else
                reinterpret_cast<float4*>(left + row * D)[c] = acc;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) p.joins[blockIdx.x] = join;
    if (blockIdx.x == 0 && threadIdx.x == 0) p.hdr->status = p.hdr->detail = 0;  // of a call before
}

// Units that cross from one worker (a CTA of packed_attn_kernel, a pair of packed_tile_kernel) into the next: blocks (c, y) take the one
// that worker c - the first of it - ends with, RPB of its rows each.  A warp for every row and every TURNS-th of the workers, lanes are
// columns; the warps of a row meet in shared memory.
// AT_ONCE: of a warp's shares, in flight together, with the first maxima.
template <int D, int ROWS, int RPB, int TURNS, int AT_ONCE>
__global__ void __launch_bounds__(RPB * TURNS * 32) packed_merge_kernel(const __grid_constant__ PackedAttnParams p) {
    constexpr int kTurns = TURNS, kShareFloats = ROWS * (D + 2);
    __shared__ float4 s_acc[kTurns][RPB][32];
    __shared__ float s_sum[kTurns][RPB];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, at_row = warp % RPB, turn = warp / RPB, c0 = blockIdx.x;
    const int row = blockIdx.y * RPB + at_row;
    grid_wait();
    grid_launch_dependents();
    const PackedJoin join = p.joins[c0];
    const int c1 = join.last;
    if (c1 <= c0) return;
    const bool some = row < min(join.n * p.G - join.chunk * ROWS, ROWS);
    auto share_of = [&](int c) { return p.part + (2 * static_cast<int64_t>(c) + (c == c0 ? join.second : 0)) * kShareFloats; };
    float top = kNoMax, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (some) {
        float4 v[AT_ONCE];
        float m[AT_ONCE], l[AT_ONCE];
        auto load = [&](int first) {
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int c = min(first + i * kTurns, c1);
                const float* const share = share_of(c);
                m[i] = __ldcg(share + ROWS * D + row);
                l[i] = __ldcg(share + ROWS * (D + 1) + row);
                v[i] = __ldcg(reinterpret_cast<const float4*>(share + row * D) + lane % (D / 4));
            }
        };
        load(c0 + turn);
        for (int c = c0 + lane; c <= c1; c += 32) top = fmaxf(top, __ldcg(share_of(c) + ROWS * D + row));
#pragma unroll
        for (int by = 16; by > 0; by /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, by));
        for (int c = c0 + turn; c <= c1; c += AT_ONCE * kTurns) {
            if (c > c0 + turn) load(c);
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const float f = c + i * kTurns <= c1 ? fast_exp2(m[i] - top) : 0.f;
                sum += f * l[i];
                acc.x += f * v[i].x; acc.y += f * v[i].y; acc.z += f * v[i].z; acc.w += f * v[i].w;
            }
        }
    }
    s_acc[turn][at_row][lane] = acc;
    if (lane == 0) s_sum[turn][at_row] = sum;
    __syncthreads();
    if (turn != 0 || !some) return;
#pragma unroll
    for (int w = 1; w < kTurns; ++w) {
        const float4 v = s_acc[w][at_row][lane];
        acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
        sum += s_sum[w][at_row];
    }
    const PackedRow at = packed_row(p, join.row0, join.head, join.chunk * ROWS + row, D);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    if (lane < D / 4) reinterpret_cast<uint2*>(p.o + at.o)[lane] = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (lane == 0 && p.lse) p.lse[at.lse] = sum > 0.f ? (top + log2f(sum)) * 0.693147180559945309f : -INFINITY;
}

template <int D, int NT>
static cudaError_t launch_rows(const PackedAttnParams& p, cudaStream_t stream) {
    using L = PackedAttnLayout<D, NT>;
    const cudaError_t e = launch_chained<packed_attn_kernel<D, NT>>(dim3(kNumSms), L::kWarps * 32, L::kTotal, stream, p);
    if (e != cudaSuccess) return e;
    // Few units have many shares each (a unit alone those of all CTAs): ten of a row in flight, whose registers leave a CTA to an SM, i.e. two rounds
    // of them.  Many units have two or three: five, and one round.  Measured, ten against five: one token against 50K keys 17.5 / 18.1 us, 64 sequences
    // of up to 16K 75.0 / 72.5, 4 sequences of 12K 17.6 / 16.9, one with rows among 1,000 of a table 20.5 / 20.9: the rule goes by the table, since which of its sequences have rows
    // only the GPU knows, and is worth half a microsecond either way.  (8 rows as a whole with two turns 18.9 and 16 rows in halves with four 30.7 us for 16 sequences under a
    // window, as a whole with one turn 27.4.)
    if (NT == 2) return launch_chained<packed_merge_kernel<D, 16, 16, 1, 10>>(dim3(kNumSms - 1), 512, 0, stream, p);
    if (static_cast<int64_t>(p.num_seqs) * p.Hkv <= 32) return launch_chained<packed_merge_kernel<D, 8, 4, 4, 10>>(dim3(kNumSms - 1, 2), 512, 0, stream, p);
    return launch_chained<packed_merge_kernel<D, 8, 4, 4, 5>>(dim3(kNumSms - 1, 2), 512, 0, stream, p);
}

template <int D>
static cudaError_t launch_tiles(const PackedAttnParams& p, cudaStream_t stream) {
    const cudaError_t e = launch_packed_tile(p, D, stream);
    if (e != cudaSuccess) return e;
    return launch_chained<packed_merge_kernel<D, 2 * kTile, 8, 1, 5>>(dim3(kNumSms / 2 - 1, 2 * kTile / 8), 8 * 32, 0, stream, p);
}

// Measured, few rows against tiles: 28/4 heads of 128, 50K keys 28 rows 29.7 / 34.6 us, 35 rows 36.6 / 34.7, 56 rows 43.6 / 35.9; 64 sequences of
// 1 to 4K keys 28 rows 72.0 / 91.5, 35 rows 94.7 / 91.7.  32/8 heads of 64, 50K keys 48 rows 41.1 / 48.0, 64 rows 49.9 / 48.2; 64 sequences
// 48 rows 115 / 144, 64 rows 143 / 146.
static int most_few(int head_dim) { return head_dim == 128 ? 32 : 48; }
static bool takes_tiles(int64_t rows, int head_dim) { return rows > most_few(head_dim); }

size_t packed_attn_workspace_bytes(int head_dim, int64_t rows) {
    const int unit = takes_tiles(rows, head_dim) ? kTile : 16;  // rows for each CTA
    return sizeof(PackedJoin) * kNumSms + 2 * static_cast<size_t>(kNumSms) * unit * (head_dim + 2) * sizeof(float);
}

static cudaError_t launch_few(const PackedAttnParams& p, int head_dim, int64_t rows, cudaStream_t stream) {
    if (head_dim == 128) return rows > 8 ? launch_rows<128, 2>(p, stream) : launch_rows<128, 1>(p, stream);
    return rows > 8 ? launch_rows<64, 2>(p, stream) : launch_rows<64, 1>(p, stream);
}

cudaError_t launch_packed_attn(PackedAttnParams p, int head_dim, int64_t max_rows, cudaStream_t stream) {
    p.n_from = 1;
    p.n_to = INT32_MAX;
    if (!takes_tiles(max_rows * p.G, head_dim)) return launch_few(p, head_dim, max_rows * p.G, stream);
    // Sequences with few rows beside some with many, or a caller who does not know: a launch for either kind, unless n_rows can only be so
    // many if all have more than a few.  64 sequences of 4K keys (28/4 heads of 128): 63 single tokens beside a question of 64 137 -> 80 us, 64
    // single tokens that are said to be up to 64 rows 129 -> 61 (40 if said to be one); launches without work take 12.
    const int few = most_few(head_dim) / p.G;  // rows of a sequence that are not worth a tile
    if (few > 0 && p.n_rows <= (p.num_seqs - 1) * max_rows + few) {
        p.n_to = few;
        const cudaError_t e = launch_few(p, head_dim, few * p.G, stream);
        if (e != cudaSuccess) return e;
        p.n_from = few + 1;
        p.n_to = INT32_MAX;
    }
    return head_dim == 128 ? launch_tiles<128>(p, stream) : launch_tiles<64>(p, stream);
}

}  // namespace pevlm
