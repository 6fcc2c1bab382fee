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

constexpr float kNoMax = -3.0e38f;  // running maximum of a row that has seen no key: any score raises it

template <int D, int NT>
struct PackedAttnLayout {
    static constexpr int kWarps = NT == 1 ? 12 : 8;
    static constexpr int kStages = D == 128 ? 4 : 8;
    static constexpr int kTileBytes = 18 * D;
    static constexpr int kRows = 8 * NT;
    static constexpr int kShareFloats = kRows * (D + 2);          // O [rows][D], then m and l of each row
    static constexpr int kRing = kWarps * kStages * kTileBytes;
    static constexpr int kTotal = kRing + kWarps * 2 * kShareFloats * 4;
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

// By a whole warp: tiles of all sequences; with `tile` >= 0 also the sequence that it belongs to and the tiles before that sequence.
__device__ __forceinline__ int64_t find_seq(const PackedAttnParams& p, int rows_per_chunk, int64_t tile, int& seq, int64_t& before) {
    const int lane = threadIdx.x & 31;
    int64_t base = 0;
    for (int r0 = 0; r0 < p.num_seqs; r0 += 32) {
        int64_t mine = 0;
        if (r0 + lane < p.num_seqs) {
            const PackedSeq s = packed_seq(p, r0 + lane, rows_per_chunk);
            mine = static_cast<int64_t>(s.chunks) * s.cnt * p.Hkv;
        }
        int64_t to = mine;
#pragma unroll
        for (int by = 1; by < 32; by *= 2) {
            const int64_t y = __shfl_up_sync(0xffffffffu, to, by);
            if (lane >= by) to += y;
        }
        if (tile >= 0) {
            const unsigned past = __ballot_sync(0xffffffffu, base + to > tile);
            if (past) {
                const int l = __ffs(past) - 1;
                seq = r0 + l;
                before = base + __shfl_sync(0xffffffffu, to - mine, l);
                return 0;
            }
        }
        base += __shfl_sync(0xffffffffu, to, 31);
    }
    return base;
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
    __device__ __forceinline__ int key_tile() const { return t < s.ns ? t : t + s.skip; }
    // Page of the tile, -1 where there is nothing to read.
    __device__ __forceinline__ int page(const PackedAttnParams& p) const {
        const int key0 = key_tile() << 4;
        if (key0 >= s.len) return -1;
        const int pg = __ldcg(p.page_table + static_cast<int64_t>(r) * p.max_pages + (key0 >> p.page_shift));
        return pg >= 0 && pg < p.num_pages ? pg : -1;
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
    extern __shared__ __align__(128) uint8_t raw[];
    struct Share {       // a share left for the CTA to join
        int64_t u0, u1;  // tiles of its unit, counted over the whole list
        int r, head, chunk, row0, n;
        int from_start;  // the part of the warp begins with it
    };
    __shared__ Share s_share[2 * W];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t ring = smem_u32(raw) + warp * L::kStages * L::kTileBytes;
    float* const shares = reinterpret_cast<float*>(raw + L::kRing);
    if (lane < 2) s_share[2 * warp + lane].u1 = -1;
    grid_wait();

    int seq = 0;
    int64_t before = 0;
    const int64_t total = find_seq(p, L::kRows, -1, seq, before);
    const int n_workers = workers_for(total, gridDim.x * W);
    const int me = blockIdx.x * W + warp;
    const int64_t lo = me < n_workers ? part_start(me, total, n_workers) : total;
    const int64_t hi = me < n_workers ? part_start(me + 1, total, n_workers) : total;
    const int mine = static_cast<int>(hi - lo);
    grid_launch_dependents();
    if (mine > 0) {
        find_seq(p, L::kRows, lo, seq, before);
        PackedCursor cur, ahead;
        cur.at(p, L::kRows, seq, lo - before);
        ahead = cur;
        int next_page = ahead.page(p);
        unsigned there = 0;  // of the ring's places: the tile exists
        const int tiles_per_page = 1 << (p.page_shift - 4);
        auto fetch = [&](int i) {
            if (i < mine) {
                const int place = i % L::kStages;
                there &= ~(1u << place);
                if (next_page >= 0) {
                    there |= 1u << place;
                    const uint8_t* src = p.cache + ((static_cast<int64_t>(next_page) * p.Hkv + ahead.head) * tiles_per_page + (ahead.key_tile() & (tiles_per_page - 1))) * L::kTileBytes;
                    const uint32_t dst = ring + place * L::kTileBytes;
#pragma unroll
                    for (int c = lane; c < L::kTileBytes / 16; c += 32)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + c * 16), "l"(src + c * 16) : "memory");
                }
                if (++ahead.t == ahead.s.cnt) ahead.next_unit(p, L::kRows);
                if (i + 1 < mine) next_page = ahead.page(p);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        for (int i = 0; i < L::kStages - 1; ++i) fetch(i);

        int64_t unit0 = lo - cur.t;  // of this unit on the list
        int i = 0;
        while (i < mine) {
            // ------------------------------------------------ a unit, or the share of it that is in this part
            const int first_tile = cur.t, tiles = min(cur.s.cnt - cur.t, mine - i);
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

            for (int n = 0; n < tiles; ++n, ++i) {
                fetch(i + L::kStages - 1);
                asm volatile("cp.async.wait_group %0;" ::"n"(L::kStages - 1) : "memory");
                __syncwarp();
                const int place = i % L::kStages;
                const int key0 = cur.key_tile() << 4;
                ++cur.t;
                if (!(there >> place & 1)) continue;
                const uint8_t* const tile = raw + (warp * L::kStages + place) * L::kTileBytes;
                // S^T: keys g and g + 8, rows 2 t and 2 t + 1
                float s[NT][4];
#pragma unroll
                for (int j = 0; j < NT; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
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
                            mma16816_f16(s[j], a[0][2 * half], a[1][2 * half], a[0][2 * half + 1], a[1][2 * half + 1], q[j][2 * w + half][0], q[j][2 * w + half][1]);
                }
                // V's scales of keys 2 t, 2 t + 1 and 2 t + 8, 2 t + 9; of keys behind the end, whose bytes may be anything, 0
                uint32_t vs[2];
                const uint32_t vb = *reinterpret_cast<const uint32_t*>(tile + 17 * D + (D == 128 ? lane * 4 : (g >> 1) * 16 + t * 4));
                vs[0] = scale_pair(vb);
                vs[1] = scale_pair(vb >> 16);
                const bool edge = key0 + 15 > pos_min || (p.window > 0 && key0 <= pos_max - p.window && key0 + 15 >= p.sink);
                if (edge) {
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int key = key0 + g + (e >> 1) * 8, at = pos[j][e & 1];
                            if (key > at || (p.window > 0 && key <= at - p.window && key >= p.sink)) s[j][e] = -INFINITY;
                        }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (key0 + 8 * h + 2 * t >= cur.s.len) vs[h] = 0u;
                        else if (key0 + 8 * h + 2 * t + 1 >= cur.s.len) vs[h] &= 0xffffu;
                    }
                }
                uint32_t pb[NT][2];
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = fmaf(s[j][e], sc[j][e & 1], -m[j][e & 1]);
                    // the reference maximum moves when a score is more than 2^8 above it
                    if (__any_sync(0xffffffffu, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) > 8.f)) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            float top = fmaxf(s[j][b], s[j][2 + b]) * sc[j][b];
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
                            x[b] = fmaf(s[j][b], sc[j][b], -to);
                            x[2 + b] = fmaf(s[j][2 + b], sc[j][b], -to);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = fast_exp2(x[e]);
                    l[j][0] += x[0] + x[2];
                    l[j][1] += x[1] + x[3];
                    pb[j][0] = transposed(pack_f16x2(x[0], x[1]));
                    pb[j][1] = transposed(pack_f16x2(x[2], x[3]));
                }
                // O^T: elements 16 g + 2 i, + 1 (8 g at head_dim 64) of keys 2 t, 2 t + 1 and those 8 further on
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
                        const uint32_t x = vw[h][0][w], y = vw[h][1][w];
                        halves_of_word((x & 0x0f0f0f0fu) | (y << 4 & 0xf0f0f0f0u), a[h][0]);
                        halves_of_word((x >> 4 & 0x0f0f0f0fu) | (y & 0xf0f0f0f0u), a[h][1]);
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            a[h][0][b] = mul_f16x2(a[h][0][b], vs[h]);
                            a[h][1][b] = mul_f16x2(a[h][1][b], vs[h]);
                        }
                    }
#pragma unroll
                    for (int b = 0; b < 4; ++b)
#pragma unroll
                        for (int j = 0; j < NT; ++j) mma16816_f16(o[j][4 * w + b], a[0][0][b], a[0][1][b], a[1][0][b], a[1][1][b], pb[j][0], pb[j][1]);
                }
                __syncwarp();  // every lane has read the place before it is filled again
            }

            // ------------------------------------------------ its end
            const bool whole = first_tile == 0 && cur.t == cur.s.cnt;
            const bool from_start = i == tiles;  // the part begins with it
            const int slot = 2 * warp + (from_start ? 0 : 1);
            float* const share = shares + slot * L::kShareFloats;
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
            if (!whole && lane == 0) s_share[slot] = {unit0, unit0 + cur.s.cnt, cur.r, cur.head, cur.chunk, cur.s.row0, cur.s.n, from_start};
            if (cur.t == cur.s.cnt) {
                unit0 += cur.s.cnt;
                if (i < mine) cur.next_unit(p, L::kRows);
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
    __syncthreads();

    // ---------------------------------------------------- shares of one unit stand one after another
    const int64_t cta_lo = part_start(min(static_cast<int>(blockIdx.x) * W, n_workers), total, max(n_workers, 1));
    const int64_t cta_hi = part_start(min(static_cast<int>(blockIdx.x + 1) * W, n_workers), total, max(n_workers, 1));
    for (int a = 0; a < 2 * W; ++a) {
        if (s_share[a].u1 < 0) continue;
        const Share u = s_share[a];
        int end = a + 1;
        while (end < 2 * W && (s_share[end].u1 < 0 || s_share[end].u0 == u.u0)) ++end;
        const bool done = u.u0 >= cta_lo && u.u1 <= cta_hi;
        const int rows = min(u.n * p.G - u.chunk * L::kRows, L::kRows);
        // the place in the workspace: the first if this CTA's part begins with the unit
        float* const part = p.part + (2 * static_cast<int64_t>(blockIdx.x) + (u.u0 <= cta_lo ? 0 : 1)) * L::kShareFloats;
        for (int x = threadIdx.x; x < rows * (D / 4); x += W * 32) {
            const int row = x / (D / 4), c = x % (D / 4);
            float top = kNoMax;
            for (int b = a; b < end; ++b)
                if (s_share[b].u1 >= 0) top = fmaxf(top, shares[b * L::kShareFloats + L::kRows * D + row]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            float sum = 0.f;
            for (int b = a; b < end; ++b) {
                if (s_share[b].u1 < 0) continue;
                const float* const share = shares + b * L::kShareFloats;
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
                reinterpret_cast<float4*>(part + row * D)[c] = acc;
                if (c == 0) {
                    part[L::kRows * D + row] = top;
                    part[L::kRows * (D + 1) + row] = sum;
                }
            }
        }
        a = end - 1;
    }
}

// Units that cross from one CTA into the next: block (c, row) takes the one that CTA c - the first of it - ends with.  Lanes are
// columns, the warps take the CTAs in turn and meet in shared memory.
constexpr int kPackedMergeWarps = 8;

template <int D, int NT>
__global__ void __launch_bounds__(kPackedMergeWarps * 32) packed_merge_kernel(const __grid_constant__ PackedAttnParams p, int ctas) {
    using L = PackedAttnLayout<D, NT>;
    constexpr int W = L::kWarps;
    __shared__ float4 s_acc[kPackedMergeWarps][32];
    __shared__ float2 s_ml[kPackedMergeWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.y;
    grid_wait();
    grid_launch_dependents();
    int seq = 0;
    int64_t before = 0;
    const int64_t total = find_seq(p, L::kRows, -1, seq, before);
    if (total == 0) return;
    const int n_workers = workers_for(total, ctas * W);
    const int c0 = blockIdx.x;
    if ((c0 + 1) * W >= n_workers) return;  // nothing behind it
    const int64_t lo = part_start(c0 * W, total, n_workers), hi = part_start((c0 + 1) * W, total, n_workers);
    find_seq(p, L::kRows, hi - 1, seq, before);
    PackedCursor cur;
    cur.at(p, L::kRows, seq, hi - 1 - before);
    const int64_t u0 = hi - 1 - cur.t, u1 = u0 + cur.s.cnt;
    if (u1 <= hi || u0 < lo) return;  // ends here, or began before
    const int rows = min(cur.s.n * p.G - cur.chunk * L::kRows, L::kRows);
    if (row >= rows) return;
    const int c1 = worker_of(u1 - 1, total, n_workers) / W;
    auto share_of = [&](int c) { return p.part + (2 * static_cast<int64_t>(c) + (c == c0 && u0 > lo ? 1 : 0)) * L::kShareFloats; };
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
    const PackedRow at = packed_row(p, cur.s.row0, cur.head, cur.chunk * L::kRows + row, D);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    if (lane < D / 4) reinterpret_cast<uint2*>(p.o + at.o)[lane] = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (lane == 0 && p.lse) p.lse[at.lse] = sum > 0.f ? (top + log2f(sum)) * 0.693147180559945309f : -INFINITY;
}

template <int D, int NT>
static cudaError_t launch_rows(const PackedAttnParams& p, cudaStream_t stream) {
    using L = PackedAttnLayout<D, NT>;
    const cudaError_t e = launch_chained<packed_attn_kernel<D, NT>>(dim3(kNumSms), L::kWarps * 32, L::kTotal, stream, p);
    if (e != cudaSuccess) return e;
    return launch_chained<packed_merge_kernel<D, NT>>(dim3(kNumSms - 1, L::kRows), kPackedMergeWarps * 32, 0, stream, p, kNumSms);
}

size_t packed_attn_workspace_bytes(int head_dim) { return 2 * static_cast<size_t>(kNumSms) * 16 * (head_dim + 2) * 4; }

cudaError_t launch_packed_attn(const PackedAttnParams& p, int head_dim, int max_rows, cudaStream_t stream) {
    const bool two = static_cast<int64_t>(max_rows) * p.G > 8;
    if (head_dim == 128) return two ? launch_rows<128, 2>(p, stream) : launch_rows<128, 1>(p, stream);
    return two ? launch_rows<64, 2>(p, stream) : launch_rows<64, 1>(p, stream);
}

}  // namespace pevlm
