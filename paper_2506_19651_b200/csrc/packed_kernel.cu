// Rows of K and V into the packed cache and back (the format stands in include/pevlm.h).
//
// Bound by HBM: a value is 2 bytes of bf16 on one side and 4.5 bits on the other.  A thread takes one group of 16 values, i.e.
// 32 bytes of a row, so nothing is exchanged between threads; the lanes of a warp are the groups of a head, then the next rows, so that
// the codes of neighbouring tokens (V's stand 8 bytes a token side by side) fill whole sectors.  The instructions count beside the memory (60 % of the
// issue slots in use, about 9 a value each way).  60K rows of 8 heads of 64, stored and read back: 315 MB in 60.5 us = 5.2 TB/s.
//
// Rounding, without a division.  The scale s is the e4m3 number nearest to m / 6 in exact arithmetic: a point halfway between two e4m3
// numbers has 5 significant bits, so a quotient in its place is 6 times it exactly (7 bits, a bf16 number), and any other bf16 m is off by
// at least 2^-9 of it.  m * (1 / 6) in fp32 is off by 2^-23 of it; rounded to fp16 (11 bits; m / 6 is clamped to 2^-9 .. 448 before) an exact
// halfway point is one again, and every other value stays on its side of it.  In the same way x / s against a halfway point t of e2m1: t * s
// has at most 7 significant bits, x has 8, so x = t * s or they are at least 1/256 of t (2^-10 for the smallest, 0.25) apart.  x * (1 / s) in
// fp32 is off by 2^-22 of it at most; rounded to multiples of 2^-11, which the addition of 6144 does on the way, an exact halfway point is one
// again and every other value stays on its side of it.
#include "internal.h"
#include "ptx.cuh"

namespace pevlm {

constexpr int kPackedThreads = 256;

// Byte offsets in the cache of what the group i (of n = D / 16) of a token's head has.
template <int D>
struct PackedPlace {
    static constexpr int n = D / 16, w = D / 64, kTileBytes = 18 * D;
    int64_t tile;
    int u;
    __device__ __forceinline__ PackedPlace(int slot, int head, int heads, int page_shift) {
        const int page = slot >> page_shift, in_page = slot & ((1 << page_shift) - 1);
        tile = ((static_cast<int64_t>(page) * heads + head) * (1 << (page_shift - 4)) + (in_page >> 4)) * kTileBytes;
        u = in_page & 15;
    }
    __device__ __forceinline__ int64_t k_codes(int i) const { return tile + u * (D / 2) + i * 8; }
    // 16 values are the 2 / w eighths from 2 i / w on: 8 bytes, together where an eighth has 16 values
    __device__ __forceinline__ int64_t v_codes(int c) const { return tile + 8 * D + (((u >> 3) * 8 + c) * 8 + (u & 7)) * n; }
    __device__ __forceinline__ int64_t k_scale(int i) const { return tile + 16 * D + (u & 7) * 2 * n + (i / w) * 2 * w + (u >> 3) * w + i % w; }
    __device__ __forceinline__ int64_t v_scale(int i) const { return tile + 17 * D + i * 16 + ((u & 7) >> 1) * 4 + (u >> 3) * 2 + (u & 1); }
};

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Eight values to eight codes, the first in the lowest bits; scaled by 1 / s and rounded to multiples of 2^-11 on the way.
__device__ __forceinline__ uint32_t codes_of(const uint4& x, uint64_t inv2) {
    const uint64_t grid = pack_f32x2(6144.f, 6144.f), back = pack_f32x2(-6144.f, -6144.f);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        unpack_f32x2(add_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), inv2, grid), back), lo[i], hi[i]);
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(lo[0]), "f"(hi[0]), "f"(lo[1]), "f"(hi[1]), "f"(lo[2]), "f"(hi[2]), "f"(lo[3]), "f"(hi[3]));
    return r;
}

// 16 values: their codes in 8 bytes and the bits of their scale.
__device__ __forceinline__ uint2 quantise(const uint4& a, const uint4& b, uint8_t& scale) {
    constexpr uint32_t kAbs = 0x7fff7fffu;
    const uint32_t m = max_bf16x2(max_bf16x2(max_bf16x2(a.x & kAbs, a.y & kAbs), max_bf16x2(a.z & kAbs, a.w & kAbs)),
                                  max_bf16x2(max_bf16x2(b.x & kAbs, b.y & kAbs), max_bf16x2(b.z & kAbs, b.w & kAbs)));
    const float top = fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    const float want = fminf(fmaxf(top * (1.f / 6.f), 1.f / 512.f), 448.f);
    uint32_t halves;
    uint16_t bits;
    asm("cvt.rn.f16x2.f32 %0, %1, %1;" : "=r"(halves) : "f"(want));
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(bits) : "r"(halves));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(halves) : "h"(bits));
    scale = static_cast<uint8_t>(bits);
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(__half2float(__ushort_as_half(static_cast<unsigned short>(halves)))));
    const uint64_t inv2 = pack_f32x2(inv, inv);
    return make_uint2(codes_of(a, inv2), codes_of(b, inv2));
}

// The heads of the same rows, K's first, are neighbouring blocks, so that what runs at the same time reads and writes the memory's rows as a whole
// (60K rows of 8 heads of 64, one head after another: 65 us for both calls instead of 60).  A thread has ROWS rows, kPackedThreads / n apart,
// all of whose loads are in flight together.
template <int D, int ROWS>
__global__ void __launch_bounds__(kPackedThreads) packed_store_kernel(const __grid_constant__ PackedRows p) {
    constexpr int n = D / 16, kApart = kPackedThreads / n;
    const int i = threadIdx.x % n;
    const int block = quotient(blockIdx.x, p.div_heads), h = blockIdx.x - block * 2 * p.Hkv;
    const int64_t row0 = static_cast<int64_t>(block) * (ROWS * kApart) + threadIdx.x / n;
    const bool is_v = h >= p.Hkv;
    const int head = is_v ? h - p.Hkv : h;
    const int64_t stride = is_v ? p.v_stride : p.k_stride;
    const __nv_bfloat16* const x = (is_v ? p.v : p.k) + head * D + i * 16;
    grid_wait();
    grid_launch_dependents();
    int slot[ROWS];
    uint4 a[ROWS], b[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t row = row0 + r * kApart;
        slot[r] = -1;
        a[r] = b[r] = make_uint4(0u, 0u, 0u, 0u);
        if (row >= p.n_rows) continue;
        slot[r] = p.slots[row];
        a[r] = __ldcs(reinterpret_cast<const uint4*>(x + row * stride));
        b[r] = __ldcs(reinterpret_cast<const uint4*>(x + row * stride) + 1);
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (slot[r] < 0 || slot[r] >= p.n_slots) continue;
        const PackedPlace<D> at(slot[r], head, p.Hkv, p.page_shift);
        uint8_t scale;
        const uint2 c = quantise(a[r], b[r], scale);
        if (!is_v) {
            *reinterpret_cast<uint2*>(p.cache + at.k_codes(i)) = c;
            p.cache[at.k_scale(i)] = scale;
        } else {
            if (D == 128) {
                *reinterpret_cast<uint2*>(p.cache + at.v_codes(i)) = c;
            } else {
                *reinterpret_cast<uint32_t*>(p.cache + at.v_codes(2 * i)) = c.x;
                *reinterpret_cast<uint32_t*>(p.cache + at.v_codes(2 * i + 1)) = c.y;
            }
            p.cache[at.v_scale(i)] = scale;
        }
    }
}

// Eight codes times the scale (twice in a word), as bf16: both products are exact in fp16 and in bf16.
__device__ __forceinline__ void values_of_word(uint32_t codes, uint32_t scale2, uint32_t* x) {
    uint32_t h[4];
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(h[i]) : "r"(h[i]), "r"(scale2));
        const __half2 v = *reinterpret_cast<const __half2*>(&h[i]);
        x[i] = pack_bf16x2(__low2float(v), __high2float(v));
    }
}

template <int D, int ROWS>
__global__ void __launch_bounds__(kPackedThreads) packed_load_kernel(const __grid_constant__ PackedRows p) {
    constexpr int n = D / 16, kApart = kPackedThreads / n;
    const int i = threadIdx.x % n;
    const int block = quotient(blockIdx.x, p.div_heads), h = blockIdx.x - block * 2 * p.Hkv;
    const int64_t row0 = static_cast<int64_t>(block) * (ROWS * kApart) + threadIdx.x / n;
    const bool is_v = h >= p.Hkv;
    const int head = is_v ? h - p.Hkv : h;
    __nv_bfloat16* const out = (is_v ? p.v_out : p.k_out) + head * D + i * 16;
    grid_wait();
    grid_launch_dependents();
    int slot[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) slot[r] = row0 + r * kApart < p.n_rows ? p.slots[row0 + r * kApart] : -1;
    uint2 c[ROWS];
    uint32_t bits[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        c[r] = make_uint2(0u, 0u);  // zeros for a slot out of range
        bits[r] = 0u;
        if (slot[r] < 0 || slot[r] >= p.n_slots) continue;
        const PackedPlace<D> at(slot[r], head, p.Hkv, p.page_shift);
        if (!is_v || D == 128) c[r] = __ldcg(reinterpret_cast<const uint2*>(p.cache + (is_v ? at.v_codes(i) : at.k_codes(i))));
        else c[r] = make_uint2(__ldcg(reinterpret_cast<const uint32_t*>(p.cache + at.v_codes(2 * i))), __ldcg(reinterpret_cast<const uint32_t*>(p.cache + at.v_codes(2 * i + 1))));
        bits[r] = __ldcg(p.cache + (is_v ? at.v_scale(i) : at.k_scale(i)));
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t row = row0 + r * kApart;
        if (row >= p.n_rows) continue;
        uint32_t scale2, x[8];
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(scale2) : "h"(static_cast<uint16_t>(bits[r] << 8 | bits[r])));
        values_of_word(c[r].x, scale2, x);
        values_of_word(c[r].y, scale2, x + 4);
        st_global_v8(out + row * p.Hkv * D, x);
    }
}

// Rows of a thread: one where there are few blocks (every SM should have some), else two.  Both calls, one / two / three / four rows: 12.6K rows of 4
// heads of 128 15.1 / 15.0 / 15.6 / 16.1 us, 60K of 8 heads of 64 62.4 / 60.5 / 60.8 / 61.0.
template <int D>
static cudaError_t launch_packed_rows(PackedRows p, bool store, cudaStream_t stream) {
    constexpr int kRows = kPackedThreads / (D / 16);
    const int64_t heads = 2 * p.Hkv, blocks = (p.n_rows + kRows - 1) / kRows;
    p.div_heads = make_divisor(static_cast<int>(heads));
    if (blocks * heads < 16 * kNumSms) {
        const dim3 grid(static_cast<unsigned>(blocks * heads));
        return store ? launch_chained<packed_store_kernel<D, 1>>(grid, kPackedThreads, 0, stream, p) : launch_chained<packed_load_kernel<D, 1>>(grid, kPackedThreads, 0, stream, p);
    }
    const dim3 grid(static_cast<unsigned>((blocks + 1) / 2 * heads));
    return store ? launch_chained<packed_store_kernel<D, 2>>(grid, kPackedThreads, 0, stream, p) : launch_chained<packed_load_kernel<D, 2>>(grid, kPackedThreads, 0, stream, p);
}

cudaError_t launch_packed_store(const PackedRows& p, int head_dim, cudaStream_t stream) {
    return head_dim == 128 ? launch_packed_rows<128>(p, true, stream) : launch_packed_rows<64>(p, true, stream);
}

cudaError_t launch_packed_load(const PackedRows& p, int head_dim, cudaStream_t stream) {
    return head_dim == 128 ? launch_packed_rows<128>(p, false, stream) : launch_packed_rows<64>(p, false, stream);
}

}  // namespace pevlm
