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
// Rows of Q are scaled by a power of two to at most 2 in magnitude, so that any bf16 values fit fp16 (what is below 2^-24 of the
// row's largest is lost, far below fp32's rounding of the sum); sums, maxima and outputs are fp32.  Probabilities are rounded to fp16
// (2^-11 of each; 2^-24 of the row's largest where smaller).
#include "internal.h"
#include "ptx.cuh"

namespace pevlm {

constexpr uint32_t kNoTile = 0xffffffffu;
constexpr float kNoMax = -3.0e38f;  // running maximum of a row that has seen no key: any score raises it

template <int D, int NT>
struct PackedAttnLayout {
    static constexpr int kWarps = NT == 1 ? 12 : 8;
    static constexpr int kStages = D == 128 ? 3 + (NT == 2) : 6;  // steps (two tiles) in a warp's ring
    static constexpr int kTileBytes = 18 * D, kStepBytes = 2 * kTileBytes;
    static constexpr int kRows = 8 * NT;
    static constexpr int kShareFloats = kRows * (D + 2);          // O [rows][D], then m and l of each row
    static constexpr int kRing = kWarps * kStages * kStepBytes;
    static constexpr int kTotal = kRing + kWarps * kShareFloats * 4;
    static_assert(kShareFloats * 4 <= kStages * kStepBytes, "the second share of a warp is left in its ring");
};

// One sequence of the call as the tiles see it.
struct PackedSeq {
    int len, n, row0;      // keys, rows, first row
    int chunks, cnt;       // units of a kv head, tiles of a unit
    int ns, skip;          // tiles from ns on are skip tiles further on in the sequence (between sink and window nobody looks)
};

__device__ __forceinline__ PackedSeq packed_seq(const PackedAttnParams& p, int r, int rows_per_chunk) {
    PackedSeq s;
    s.len = min(max(p.lens[r], 0), p.max_pages << p.page_shift);
    s.row0 = min(max(p.row_start[r], 0), p.n_rows);
    s.n = max(min(p.row_start[r + 1], p.n_rows) - s.row0, 0);
    s.chunks = (s.n * p.G + rows_per_chunk - 1) / rows_per_chunk;
    s.ns = s.skip = 0;
    const int tiles = (s.len + 15) >> 4;
    if (p.window > 0) {
        s.ns = (min(p.sink, s.len) + 15) >> 4;
        const int lo = max(s.len - s.n - p.window + 1, 0) >> 4;  // tile of the first key that the first row's window shows
        s.skip = min(max(lo - s.ns, 0), tiles - s.ns);
    }
    s.cnt = max(tiles - s.skip, 1);  // a sequence without keys has a tile that nothing is visible in
    return s;
}

// Where the part of warp w of the launch begins, of n_workers warps and all `total` tiles.
__device__ __forceinline__ int64_t part_start(int64_t w, int64_t total, int n_workers) { return w * total / n_workers; }
// The warp whose part a tile is in.
__device__ __forceinline__ int worker_of(int64_t tile, int64_t total, int n_workers) { return static_cast<int>(((tile + 1) * n_workers - 1) / total); }
__device__ __forceinline__ int workers_for(int64_t total, int most) { return static_cast<int>(min(static_cast<int64_t>(most), (total + 1) / 2)); }

__device__ __forceinline__ int64_t seq_tiles(const PackedAttnParams& p, int r, int rows_per_chunk) {
    if (r >= p.num_seqs) return 0;
    const PackedSeq s = packed_seq(p, r, rows_per_chunk);
    return static_cast<int64_t>(s.chunks) * s.cnt * p.Hkv;
}

__device__ __forceinline__ int64_t warp_inclusive(int64_t x) {
#pragma unroll
    for (int by = 1; by < 32; by *= 2) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, by);
        if ((threadIdx.x & 31) >= static_cast<unsigned>(by)) x += y;
    }
    return x;
}

// The calling warp's part of the list: tiles [lo, hi) of `total`, beginning `off` tiles into those of sequence seq.
struct PackedPart {
    int64_t total, lo, hi, off;
    int seq, n_workers;
};

template <int W>
__device__ __forceinline__ PackedPart my_part(const PackedAttnParams& p, int rows_per_chunk) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, me = blockIdx.x * W + warp;
    PackedPart part;
    part.seq = 0;
    part.off = 0;
    auto bounds = [&](int64_t total) {
        part.total = total;
        part.n_workers = workers_for(total, gridDim.x * W);
        part.lo = me < part.n_workers ? part_start(me, total, part.n_workers) : total;
        part.hi = me < part.n_workers ? part_start(me + 1, total, part.n_workers) : total;
    };
    if (p.num_seqs <= 32) {  // each warp for itself
        const int64_t mine = seq_tiles(p, lane, rows_per_chunk), to = warp_inclusive(mine);
        bounds(__shfl_sync(0xffffffffu, to, 31));
        const unsigned past = __ballot_sync(0xffffffffu, to > part.lo);
        if (past) {
            part.seq = __ffs(past) - 1;
            part.off = part.lo - __shfl_sync(0xffffffffu, to - mine, part.seq);
        }
        return part;
    }
    // a thread for every sequence, W * 32 at a time
    __shared__ int64_t s_sum[W], s_off[W];
    __shared__ int s_seq[W];
    int64_t sum = 0;
    for (int r = threadIdx.x; r < p.num_seqs; r += W * 32) sum += seq_tiles(p, r, rows_per_chunk);
    sum = warp_inclusive(sum);
    if (lane == 31) s_sum[warp] = sum;
    __syncthreads();
    int64_t total = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) total += s_sum[w];
    bounds(total);
    int64_t base = 0;
    for (int r0 = 0; r0 < p.num_seqs; r0 += W * 32) {
        const int r = r0 + threadIdx.x;
        const int64_t mine = seq_tiles(p, r, rows_per_chunk);
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
        if (mine > 0) {
            for (int w = 0; w < W; ++w) {
                const int worker = blockIdx.x * W + w;
                if (worker >= part.n_workers) break;
                const int64_t lo = part_start(worker, total, part.n_workers);
                if (lo >= to - mine && lo < to) {
                    s_seq[w] = r;
                    s_off[w] = lo - (to - mine);
                }
            }
        }
        base += all;
    }
    __syncthreads();
    if (part.hi > part.lo) {
        part.seq = s_seq[warp];
        part.off = s_off[warp];
    }
    return part;
}

// A place on the list.
struct PackedCursor {
    PackedSeq s;
    int r, head, chunk, t;
    __device__ __forceinline__ void at(const PackedAttnParams& p, int rows_per_chunk, int seq, int64_t off) {
        r = seq;
        s = packed_seq(p, r, rows_per_chunk);
        const int64_t unit = off / s.cnt;
        t = static_cast<int>(off - unit * s.cnt);
        head = static_cast<int>(unit / s.chunks);
        chunk = static_cast<int>(unit - static_cast<int64_t>(head) * s.chunks);
    }
    __device__ __forceinline__ void next_unit(const PackedAttnParams& p, int rows_per_chunk) {
        t = 0;
        if (++chunk < s.chunks) return;
        chunk = 0;
        if (++head < p.Hkv) return;
        head = 0;
        do {
            if (++r >= p.num_seqs) return;
            s = packed_seq(p, r, rows_per_chunk);
        } while (s.chunks == 0);
    }
    __device__ __forceinline__ int key0(int x) const { return (x < s.ns ? x : x + s.skip) << 4; }
    // Where tile x of the unit stands in the cache, in units of 128 bytes (which tile_units of them make); kNoTile where there is nothing to read.
    __device__ __forceinline__ uint32_t place(const PackedAttnParams& p, int x, int tile_units) const {
        const int tile = x < s.ns ? x : x + s.skip;
        if (x >= s.cnt || tile << 4 >= s.len) return kNoTile;
        const int page = __ldcg(p.page_table + static_cast<int64_t>(r) * p.max_pages + (tile >> (p.page_shift - 4)));
        if (page < 0 || page >= p.num_pages) return kNoTile;
        return static_cast<uint32_t>((((static_cast<int64_t>(page) * p.Hkv + head) << (p.page_shift - 4)) + (tile & ((1 << (p.page_shift - 4)) - 1))) * tile_units);
    }
};

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
// The eight codes of a word as four pairs of fp16, byte by byte.
__device__ __forceinline__ void halves_of_word(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
__device__ __forceinline__ uint32_t scale_pair(uint32_t two_bytes) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(two_bytes)));
    return r;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Where row rr (of a sequence and kv head: token rr / G, head rr % G of the group) of the result goes.
struct PackedRow {
    int64_t o, lse;
};
__device__ __forceinline__ PackedRow packed_row(const PackedAttnParams& p, int row0, int head, int rr, int d) {
    const int tok = quotient(rr, p.div_g), h = head * p.G + rr - tok * p.G;
    return {(static_cast<int64_t>(row0 + tok) * p.Hq + h) * d, static_cast<int64_t>(h) * p.n_rows + row0 + tok};
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

    const PackedPart part = my_part<W>(p, L::kRows);
    const int mine = static_cast<int>(part.hi - part.lo);
    grid_launch_dependents();
    if (mine > 0) {
        PackedCursor cur, ahead;
        cur.at(p, L::kRows, part.seq, part.off);
        ahead = cur;
        // Fetching: steps of two tiles.  A lane holds the place of a tile, 32 tiles at a time and the 32 behind them, so that a page
        // is looked up long before it is needed.
        int to_fetch = mine, left = min(ahead.s.cnt - ahead.t, to_fetch);  // of the part, and of it in this unit
        int block = ahead.t;
        uint32_t places = ahead.place(p, block + lane, L::kTileBytes / 128), places_next = ahead.place(p, block + 32 + lane, L::kTileBytes / 128);
        unsigned there = 0;  // two bits a place in the ring: the tiles exist
        int stage_in = 0;
        auto fetch = [&]() {
            if (to_fetch > 0) {
                if (ahead.t - block == 32) {
                    block += 32;
                    places = places_next;
                    places_next = ahead.place(p, block + 32 + lane, L::kTileBytes / 128);
                }
                const uint32_t at0 = __shfl_sync(0xffffffffu, places, ahead.t - block), at1 = left > 1 ? __shfl_sync(0xffffffffu, places, ahead.t - block + 1) : kNoTile;
                there = (there & ~(3u << (2 * stage_in))) | ((at0 != kNoTile ? 1u : 0u) | (at1 != kNoTile ? 2u : 0u)) << (2 * stage_in);
                const uint8_t* const src0 = p.cache + static_cast<uint64_t>(at0) * 128 + lane * 16;
                const uint8_t* const src1 = p.cache + static_cast<uint64_t>(at1) * 128 + lane * 16 - kChunks % 32 * 16;
                const uint32_t dst = ring + stage_in * L::kStepBytes + lane * 16;
                // the chunks of both tiles, 32 at a time: those in the middle are of one or the other (kChunks % 32 = 16 or 8)
#pragma unroll
                for (int c = 0; c < (2 * kChunks + 31) / 32; ++c) {
                    const bool first = c * 32 + lane < kChunks;
                    const uint8_t* const src = first ? src0 + c * 512 : src1 + (c - kChunks / 32) * 512;
                    const bool some = (first ? at0 : at1) != kNoTile && ((c + 1) * 32 <= 2 * kChunks || c * 32 + lane < 2 * kChunks);
                    if (some) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + c * 512), "l"(src) : "memory");
                }
                stage_in = stage_in + 1 == L::kStages ? 0 : stage_in + 1;
                const int step = min(left, 2);
                to_fetch -= step;
                left -= step;
                ahead.t += step;
                if (left == 0 && to_fetch > 0) {
                    ahead.next_unit(p, L::kRows);
                    left = min(ahead.s.cnt, to_fetch);
                    block = 0;
                    places = ahead.place(p, lane, L::kTileBytes / 128);
                    places_next = ahead.place(p, 32 + lane, L::kTileBytes / 128);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int i = 0; i < L::kStages - 1; ++i) fetch();

        int64_t unit0 = part.lo - cur.t;  // of this unit on the list
        int stage = 0, done_tiles = 0;
        while (done_tiles < mine) {
            // ------------------------------------------------ a unit, or the share of it that is in this part
            const int first_tile = cur.t, tiles = min(cur.s.cnt - cur.t, mine - done_tiles);
            const int rows = min(cur.s.n * p.G - cur.chunk * L::kRows, L::kRows);
            uint32_t q[NT][KS][2];
            float sc[NT][2];                // softmax scale, in units of log2, of rows 2 t and 2 t + 1
            int pos[NT][2];
            float m[NT][2], l[NT][2], o[NT][MT][4];
            int pos_min = INT32_MAX, pos_max = -1;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int rr = cur.chunk * L::kRows + 8 * j + g;
                uint32_t x[KS * 2];
                float top = 0.f;
                if (8 * j + g < rows) {
                    const int tok = quotient(rr, p.div_g), h = cur.head * p.G + rr - tok * p.G;
                    const __nv_bfloat16* src = p.q + (cur.s.row0 + tok) * p.q_stride + h * D + t * (D / 4);
#pragma unroll
                    for (int c = 0; c < KS / 2; ++c) *reinterpret_cast<uint4*>(&x[4 * c]) = __ldcg(reinterpret_cast<const uint4*>(src) + c);
                } else {
#pragma unroll
                    for (int c = 0; c < KS * 2; ++c) x[c] = 0u;
                }
#pragma unroll
                for (int c = 0; c < KS * 2; ++c) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(x[c] << 16)), fabsf(__uint_as_float(x[c] & 0xffff0000u))));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // 2^e <= top < 2^(e + 1); down by 2^e, the softmax scale up by it
                const int e = min(max(static_cast<int>(__float_as_uint(top) >> 23), 1), 253);
                const float down = __uint_as_float(static_cast<uint32_t>(254 - e) << 23), up = __uint_as_float(static_cast<uint32_t>(e) << 23) * p.scale_log2;
#pragma unroll
                for (int c = 0; c < KS * 2; ++c)
                    q[j][c >> 1][c & 1] = pack_f16x2(__uint_as_float(x[c] << 16) * down, __uint_as_float(x[c] & 0xffff0000u) * down);
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    sc[j][b] = __shfl_sync(0xffffffffu, up, 8 * t + 4 * b);
                    const int row = 8 * j + 2 * t + b;
                    pos[j][b] = row < rows ? cur.s.len - cur.s.n + quotient(cur.chunk * L::kRows + row, p.div_g) : -1;
                    m[j][b] = kNoMax;
                    l[j][b] = 0.f;
                }
#pragma unroll
                for (int c = 0; c < MT; ++c) o[j][c][0] = o[j][c][1] = o[j][c][2] = o[j][c][3] = 0.f;
            }
            pos_min = cur.s.len - cur.s.n + quotient(cur.chunk * L::kRows, p.div_g);
            pos_max = cur.s.len - cur.s.n + quotient(cur.chunk * L::kRows + rows - 1, p.div_g);

            for (int n = 0; n < tiles; n += 2) {
                fetch();
                asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 1) : "memory");
                __syncwarp();
                const uint8_t* const step = my_ring + stage * L::kStepBytes;
                const unsigned exist = there >> (2 * stage) & 3u;
                stage = stage + 1 == L::kStages ? 0 : stage + 1;
                const int key0[2] = {cur.key0(first_tile + n), cur.key0(first_tile + n + 1)};
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
                // masks, and scales of 0 for what is behind the end or not there (its bytes may be anything)
                const int last0 = max(key0[0], key0[1]);
                if (exist != 3u || last0 + 15 > pos_min || (p.window > 0 && key0[0] <= pos_max - p.window && last0 + 15 >= p.sink)) {
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
                            if (!is_there || key0[x] + 8 * h + 2 * t >= cur.s.len) vs[x][h] = 0u;
                            else if (key0[x] + 8 * h + 2 * t + 1 >= cur.s.len) vs[x][h] &= 0xffffu;
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
                    // the reference maximum moves when a score is more than 2^8 above it
                    if (__any_sync(0xffffffffu, most > 8.f)) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            float top = fmaxf(fmaxf(s[j][0][b], s[j][0][2 + b]), fmaxf(s[j][1][b], s[j][1][2 + b])) * sc[j][b];
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                            const float to = fmaxf(m[j][b], top), alpha = fast_exp2(m[j][b] - to);
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
                        pb[j][x][0] = transposed(pack_f16x2(y[x][0], y[x][1]));
                        pb[j][x][1] = transposed(pack_f16x2(y[x][2], y[x][3]));
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
                __syncwarp();  // every lane has read the place before it is filled again
            }
            cur.t += tiles;
            done_tiles += tiles;

            // ------------------------------------------------ its end
            const bool whole = first_tile == 0 && cur.t == cur.s.cnt;
            const int slot = 2 * warp + (done_tiles == tiles ? 0 : 1);  // the part begins with it, or ends with it
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
            if (cur.t == cur.s.cnt) {
                unit0 += cur.s.cnt;
                if (done_tiles < mine) cur.next_unit(p, L::kRows);
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    __syncthreads();

    // ---------------------------------------------------- shares of one unit stand one after another
    const int workers = max(part.n_workers, 1);
    const int64_t cta_lo = part_start(min(static_cast<int>(blockIdx.x) * W, part.n_workers), part.total, workers);
    const int64_t cta_hi = part_start(min(static_cast<int>(blockIdx.x + 1) * W, part.n_workers), part.total, workers);
    PackedJoin join{0, 0, 0, 0, 0, 0};
    for (int a = 0; a < 2 * W; ++a) {
        if (s_share[a].u1 < 0) continue;
        const Share u = s_share[a];
        int end = a + 1;
        while (end < 2 * W && (s_share[end].u1 < 0 || s_share[end].u0 == u.u0)) ++end;
        const bool done = u.u0 >= cta_lo && u.u1 <= cta_hi;
        const int rows = min(u.n * p.G - u.chunk * L::kRows, L::kRows);
        // the place in the workspace: the first if this CTA's part begins with the unit
        const int second = u.u0 > cta_lo;
        float* const left = p.part + (2 * static_cast<int64_t>(blockIdx.x) + second) * L::kShareFloats;
        if (!done && u.u0 >= cta_lo) join = {worker_of(u.u1 - 1, part.total, workers) / W, second, u.row0, u.n, u.head, u.chunk};
        for (int x = threadIdx.x; x < rows * (D / 4); x += W * 32) {
            const int row = x / (D / 4), c = x % (D / 4);
            float top = kNoMax;
            for (int b = a; b < end; ++b)
                if (s_share[b].u1 >= 0) top = fmaxf(top, share_at(b)[L::kRows * D + row]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            float sum = 0.f;
            for (int b = a; b < end; ++b) {
                if (s_share[b].u1 < 0) continue;
                const float* const share = share_at(b);
                const float f = fast_exp2(share[L::kRows * D + row] - top);
                const float4 v = reinterpret_cast<const float4*>(share + row * D)[c];
                sum += f * share[L::kRows * (D + 1) + row];
                acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
            }
            if (done) {
                const PackedRow at = packed_row(p, u.row0, u.head, u.chunk * L::kRows + row, D);
                const float inv = sum > 0.f ? 1.f / sum : 0.f;
                reinterpret_cast<uint2*>(p.o + at.o)[c] = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
                if (c == 0 && p.lse) p.lse[at.lse] = sum > 0.f ? (top + log2f(sum)) * 0.693147180559945309f : -INFINITY;
            } else {
                reinterpret_cast<float4*>(left + row * D)[c] = acc;
                if (c == 0) {
                    left[L::kRows * D + row] = top;
                    left[L::kRows * (D + 1) + row] = sum;
                }
            }
        }
        a = end - 1;
    }
    if (threadIdx.x == 0) p.joins[blockIdx.x] = join;
}

// Units that cross from one CTA into the next: block (c, row) takes the one that CTA c - the first of it - ends with.  Lanes are
// columns, the warps take the CTAs in turn and meet in shared memory.
constexpr int kPackedMergeWarps = 8;

template <int D, int NT>
__global__ void __launch_bounds__(kPackedMergeWarps * 32) packed_merge_kernel(const __grid_constant__ PackedAttnParams p) {
    using L = PackedAttnLayout<D, NT>;
    __shared__ float4 s_acc[kPackedMergeWarps][32];
    __shared__ float2 s_ml[kPackedMergeWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.y, c0 = blockIdx.x;
    grid_wait();
    grid_launch_dependents();
    const PackedJoin join = p.joins[c0];
    const int c1 = join.last;
    if (c1 <= c0 || row >= min(join.n * p.G - join.chunk * L::kRows, L::kRows)) return;
    auto share_of = [&](int c) { return p.part + (2 * static_cast<int64_t>(c) + (c == c0 ? join.second : 0)) * L::kShareFloats; };
    float top = kNoMax;
    for (int c = c0 + lane; c <= c1; c += 32) top = fmaxf(top, __ldcg(share_of(c) + L::kRows * D + row));
#pragma unroll
    for (int by = 16; by > 0; by /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, by));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll 4
    for (int c = c0 + warp; c <= c1; c += kPackedMergeWarps) {
        const float* const share = share_of(c);
        const float f = fast_exp2(__ldcg(share + L::kRows * D + row) - top);
        sum += f * __ldcg(share + L::kRows * (D + 1) + row);
        if (lane < D / 4) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(share + row * D) + lane);
            acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
        }
    }
    s_acc[warp][lane] = acc;
    if (lane == 0) s_ml[warp] = make_float2(top, sum);
    __syncthreads();
    if (warp != 0) return;
    for (int w = 1; w < kPackedMergeWarps; ++w) {
        const float4 v = s_acc[w][lane];
        acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
        sum += s_ml[w].y;
    }
    const PackedRow at = packed_row(p, join.row0, join.head, join.chunk * L::kRows + row, D);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    if (lane < D / 4) reinterpret_cast<uint2*>(p.o + at.o)[lane] = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (lane == 0 && p.lse) p.lse[at.lse] = sum > 0.f ? (top + log2f(sum)) * 0.693147180559945309f : -INFINITY;
}

template <int D, int NT>
static cudaError_t launch_rows(const PackedAttnParams& p, cudaStream_t stream) {
    using L = PackedAttnLayout<D, NT>;
    const cudaError_t e = launch_chained<packed_attn_kernel<D, NT>>(dim3(kNumSms), L::kWarps * 32, L::kTotal, stream, p);
    if (e != cudaSuccess) return e;
    return launch_chained<packed_merge_kernel<D, NT>>(dim3(kNumSms - 1, L::kRows), kPackedMergeWarps * 32, 0, stream, p);
}

size_t packed_attn_workspace_bytes(int head_dim) { return sizeof(PackedJoin) * kNumSms + 2 * static_cast<size_t>(kNumSms) * 16 * (head_dim + 2) * 4; }

cudaError_t launch_packed_attn(const PackedAttnParams& p, int head_dim, int max_rows, cudaStream_t stream) {
    const bool two = static_cast<int64_t>(max_rows) * p.G > 8;
    if (head_dim == 128) return two ? launch_rows<128, 2>(p, stream) : launch_rows<128, 1>(p, stream);
    return two ? launch_rows<64, 2>(p, stream) : launch_rows<64, 1>(p, stream);
}

}  // namespace pevlm
