// What the kernels of the attention over the packed cache share: the list of work and the conversions of the format.
#pragma once
#include "internal.h"
#include "ptx.cuh"

namespace pevlm {

// The list.  A unit is what one result needs: (sequence, kv head, chunk of query rows).  Its tiles of 1 << TS keys stand one after another, the
// units behind one another, and every worker (a warp, or a pair of CTAs) has an equal part of the list.
constexpr uint32_t kNoTile = 0xffffffffu;
constexpr float kNoMax = -3.0e38f;  // running maximum of a row that has seen no key: any score raises it
// What a worker does at the start and the end of a unit takes it as long as so many tiles: they stand on the list in front of the unit's
// own, so that workers with several short units have fewer tiles.  Measured with tiles of 16 keys: 1.9 us where a tile takes 0.7, 4.5 us with 16
// rows and heads of 64, a tile 0.46 (64 sequences of 1 to 16K keys, one warp with five units: 64 us where the others took 55).
template <int TS>
constexpr int kUnitTiles = TS == 4 ? 4 : 2;

// One sequence of the call as the tiles see it.
struct PackedSeq {
    int len, n, row0;      // keys, rows, first row
    int chunks, cnt;       // units of a kv head, tiles of a unit
    int ns, skip;          // tiles from ns on are skip tiles further on in the sequence (between sink and window nobody looks)
};

// From what the sequence's lens[r], row_start[r] and row_start[r + 1] hold.
template <int TS>
__device__ __forceinline__ PackedSeq packed_seq(const PackedAttnParams& p, int len, int from, int to, int rows_per_chunk) {
    PackedSeq s;
    // rows that are not all there: where they stand in the sequence would have to be guessed, so they see no key
    s.len = to > p.n_rows ? 0 : min(max(len, 0), p.max_pages << p.page_shift);
    s.row0 = min(max(from, 0), p.n_rows);
    s.n = max(min(to, p.n_rows) - s.row0, 0);
    if (s.n < p.n_from || s.n > p.n_to) s.n = 0;
    s.chunks = (s.n * p.G + rows_per_chunk - 1) / rows_per_chunk;
    s.ns = s.skip = 0;
    constexpr int kKeys = 1 << TS;
    const int tiles = (s.len + kKeys - 1) >> TS;
    if (p.window > 0) {
        s.ns = (min(p.sink, s.len) + kKeys - 1) >> TS;
        const int lo = max(s.len - s.n - p.window + 1, 0) >> TS;  // tile of the first key that the first row's window shows
        s.skip = min(max(lo - s.ns, 0), tiles - s.ns);
    }
    s.cnt = max(tiles - s.skip, 1);  // a sequence without keys has a tile that nothing is visible in
    return s;
}

template <int TS>
__device__ __forceinline__ PackedSeq packed_seq(const PackedAttnParams& p, int r, int rows_per_chunk) {
    return packed_seq<TS>(p, p.lens[r], p.row_start[r], p.row_start[r + 1], rows_per_chunk);
}

// a / b for a >= 0, b > 0: 32 bits wherever they do (a 64-bit division is a subroutine of a hundred instructions).
__device__ __forceinline__ int64_t divided(int64_t a, int64_t b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// How `total` tiles are dealt to n workers: the first `more` of them have each + 1 tiles, the others each.
struct PackedDeal {
    int64_t total, each;
    int n, more;
    __device__ __forceinline__ PackedDeal(int64_t tiles, int most) {
        total = tiles;
        n = static_cast<int>(min(static_cast<int64_t>(most), (tiles + 1) / 2));
        each = n > 0 ? divided(tiles, n) : 0;
        more = static_cast<int>(tiles - each * n);
    }
    __device__ __forceinline__ int64_t start(int w) const { return w < n ? w * each + min(w, more) : total; }
    __device__ __forceinline__ int worker_of(int64_t tile) const {
        const int64_t head = more * (each + 1);
        return static_cast<int>(tile < head ? divided(tile, each + 1) : more + divided(tile - head, each));
    }
};

template <int TS>
__device__ __forceinline__ int64_t seq_tiles(const PackedAttnParams& p, const PackedSeq& s) {
    return static_cast<int64_t>(s.chunks) * (s.cnt + kUnitTiles<TS>) * p.Hkv;
}

__device__ __forceinline__ int64_t warp_inclusive(int64_t x) {
#pragma unroll
    for (int by = 1; by < 32; by *= 2) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, by);
        if ((threadIdx.x & 31) >= static_cast<unsigned>(by)) x += y;
    }
    return x;
}

// A worker's part of the list begins `off` tiles into those of sequence seq.
struct PackedPart {
    PackedDeal deal;
    int64_t off;
    int seq;
    PackedSeq s;  // that sequence
};

// Rows of Q are held in fp16, scaled by a power of two so that their largest element (of exponent field e) has a magnitude in [2^14, 2^15): what is at
// least 2^-31 of it is exact then, and what is smaller off by at most 2^-39 of it.  (A score is off by at most 2^-39 max|q| * sum|k| for that, over the
// keys' elements beside such small ones: visible only where scale * max|q| * sum|k| is some 10^7.)  Sums of 128 products with values up to 2688 are below 2^34.
struct RowPower {
    int e;
    __device__ __forceinline__ explicit RowPower(float top) { e = min(max(static_cast<int>(__float_as_uint(top) >> 23), 15), 254); }
    __device__ __forceinline__ float down() const { return __uint_as_float(static_cast<uint32_t>(268 - e) << 23); }
    // Softmax scale, in units of log2, of the row as it is held.  Kept within the normal numbers: the scores it goes with are below 2^34, which makes
    // nothing of the smallest, but -inf of a hidden key times 0 would be no number.
    __device__ __forceinline__ float up(float scale_log2) const {
        return fminf(fmaxf(__uint_as_float(static_cast<uint32_t>(e) << 23) * 0x1p-14f * scale_log2, 1.17549435e-38f), 3.40282347e38f);
    }
};

// Probabilities are formed 2^kHeadroom times larger than the softmax of the running reference has them (the row sums with them, so that it cancels): with the
// reference up to 2^8 below the largest they are at most 2^15, and what fp16 loses of the smallest is 2^-32 of the reference instead of 2^-25.
constexpr float kHeadroom = 7.f;

// First sequence from r on that has rows (num_seqs: none has), for a whole warp: 128 are looked at together, since a server's table may hold many
// that have none in this call.
__device__ __forceinline__ int seq_with_rows(const PackedAttnParams& p, int r) {
    const int lane = threadIdx.x & 31;
    for (; r < p.num_seqs; r += 128) {
        int from[4], to[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = min(r + 32 * i + lane, p.num_seqs - 1);
            from[i] = p.row_start[x];
            to[i] = p.row_start[x + 1];
        }
        int found = p.num_seqs;
#pragma unroll
        for (int i = 3; i >= 0; --i) {
            const int n = min(to[i], p.n_rows) - max(from[i], 0);
            const unsigned some = __ballot_sync(0xffffffffu, r + 32 * i + lane < p.num_seqs && n > 0 && n >= p.n_from && n <= p.n_to);
            if (some != 0) found = r + 32 * i + __ffs(some) - 1;
        }
        if (found < p.num_seqs) return found;
    }
    return p.num_seqs;
}

// A unit on the list.
template <int TS>
struct PackedUnit {
    PackedSeq s;
    int r, head, chunk;
    // The part's first one, and the part's first place in it.
    __device__ __forceinline__ PackedUnit(const PackedPart& part, int& at) : s(part.s), r(part.seq) {
        const int64_t unit = divided(part.off, s.cnt + kUnitTiles<TS>);
        at = static_cast<int>(part.off - unit * (s.cnt + kUnitTiles<TS>));
        head = static_cast<int>(divided(unit, s.chunks));
        chunk = static_cast<int>(unit - static_cast<int64_t>(head) * s.chunks);
    }
    // The next one, for a whole warp; past the last, r = num_seqs.  `table`: the sequences' descriptions in shared memory, or NULL.
    __device__ __forceinline__ void next(const PackedAttnParams& p, int rows_per_chunk, const PackedSeq* table) {
        if (++chunk < s.chunks) return;
        chunk = 0;
        if (++head < p.Hkv) return;
        head = 0;
        if (++r >= p.num_seqs) return;
        s = table ? table[r] : packed_seq<TS>(p, r, rows_per_chunk);
        if (s.chunks > 0) return;
        r = seq_with_rows(p, r + 1);
        if (r < p.num_seqs) s = table ? table[r] : packed_seq<TS>(p, r, rows_per_chunk);
    }
    __device__ __forceinline__ int key0(int x) const { return (x < s.ns ? x : x + s.skip) << TS; }
    // Tiles [from, to) of the unit, of whose keys every row at positions pos_min .. pos_max sees all.
    __device__ __forceinline__ void open_tiles(const PackedAttnParams& p, int pos_min, int pos_max, int& from, int& to) const {
        from = 0;
        to = max((pos_min + 1) >> TS, 0) - s.skip;
        if (p.window > 0) from = max(((pos_max - p.window + (1 << TS)) >> TS) - s.skip, s.ns);  // the sink's few are looked at one by one
    }
};

// Page of 16 keys (the tile-th of sequence r, that has len) as the table has it, -1 behind the end; to be looked at only once it is
// needed: until then the load is in flight.
__device__ __forceinline__ int packed_page(const PackedAttnParams& p, int r, int len, int tile) {
    if (tile << 4 >= len) return -1;
    return __ldcg(p.page_table + static_cast<int64_t>(r) * p.max_pages + (tile >> (p.page_shift - 4)));
}
// Where those 16 keys of a head stand in the cache, in units of 128 bytes (which tile_units of them make); kNoTile where there is nothing to read.
__device__ __forceinline__ uint32_t packed_place(const PackedAttnParams& p, int page, int head, int tile, int tile_units) {
    if (page < 0 || page >= p.num_pages) return kNoTile;
    return static_cast<uint32_t>((((static_cast<int64_t>(page) * p.Hkv + head) << (p.page_shift - 4)) + (tile & ((1 << (p.page_shift - 4)) - 1))) * tile_units);
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
// The same of probabilities: at most 2^15 by kHeadroom, unless scores are so large (2^25 and more in units of log2) that their own rounding moves them by
// whole powers of two.  Then the largest number there is, where an infinity would make the row no number.
__device__ __forceinline__ uint32_t pack_probabilities(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
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

}  // namespace pevlm
