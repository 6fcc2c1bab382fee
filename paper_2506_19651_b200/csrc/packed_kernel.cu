// Rows of K and V into the packed cache and back (the format stands in include/pevlm.h).
//
// Bound by HBM: a value is 2 bytes of bf16 on one side and 4.5 bits on the other.  A thread takes one group of 16 values, i.e.
// 32 bytes of a row, so nothing is exchanged between threads; the lanes of a warp are the groups of a head, then the next rows, so that
// the codes of neighbouring tokens (V's stand 8 bytes a token side by side) fill whole sectors.
//
// Rounding, without a division for each value.  The scale s is the e4m3 number nearest to m / 6 in exact arithmetic although the quotient is
// formed in fp32: a point halfway between two e4m3 numbers has 5 significant bits, so a quotient in its place is 6 times it
// exactly (7 bits, a bf16 number), and any other bf16 m is off by at least 2^-9 of it.  In the same way x / s against a
// halfway point t of e2m1: t * s has at most 7 significant bits, x has 8, so x = t * s or they are at least 1/256 of t (2^-10 for the
// smallest, 0.25) apart.  x * (1 / s) in fp32 is off by 2^-23 of it; rounded to multiples of 2^-11, which the addition of 6144 does on
// the way, an exact halfway point is one again and every other value stays on its side of it.
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

__device__ __forceinline__ uint32_t abs_max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a & 0x7fff7fffu), "r"(b & 0x7fff7fffu));
    return r;
}

// Four values to four codes, the first in the lowest bits; scaled by 1 / s and rounded to multiples of 2^-11 on the way.
__device__ __forceinline__ uint32_t codes_of_four(uint32_t x01, uint32_t x23, float inv) {
    constexpr float kGrid = 6144.f;
    const float a = __fmaf_rn(__uint_as_float(x01 << 16), inv, kGrid) - kGrid, b = __fmaf_rn(__uint_as_float(x01 & 0xffff0000u), inv, kGrid) - kGrid;
    const float c = __fmaf_rn(__uint_as_float(x23 << 16), inv, kGrid) - kGrid, d = __fmaf_rn(__uint_as_float(x23 & 0xffff0000u), inv, kGrid) - kGrid;
    uint32_t r;
    asm("{\n\t.reg .b8 lo, hi;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi, 0, 0};\n\t}"
        : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// The 16 values at x, 16-byte aligned: their codes in 8 bytes and the bits of their scale.
__device__ __forceinline__ uint2 quantise(const __nv_bfloat16* x, uint8_t& scale) {
    const uint4 a = __ldcs(reinterpret_cast<const uint4*>(x)), b = __ldcs(reinterpret_cast<const uint4*>(x) + 1);
    const uint32_t m = abs_max_bf16x2(abs_max_bf16x2(abs_max_bf16x2(a.x, a.y), abs_max_bf16x2(a.z, a.w)),
                                      abs_max_bf16x2(abs_max_bf16x2(b.x, b.y), abs_max_bf16x2(b.z, b.w)));
    const float top = fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    const float want = fminf(fmaxf(__fdiv_rn(top, 6.f), 1.f / 512.f), 448.f);
    uint16_t bits;
    uint32_t halves;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %1;" : "=h"(bits) : "f"(want));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(halves) : "h"(bits));
    scale = static_cast<uint8_t>(bits);
    const float inv = __frcp_rn(__half2float(__ushort_as_half(static_cast<unsigned short>(halves))));
    return make_uint2(codes_of_four(a.x, a.y, inv) | codes_of_four(a.z, a.w, inv) << 16, codes_of_four(b.x, b.y, inv) | codes_of_four(b.z, b.w, inv) << 16);
}

// blockIdx.y: head, K heads first.
template <int D>
__global__ void __launch_bounds__(kPackedThreads) packed_store_kernel(const __grid_constant__ PackedRows p) {
    constexpr int n = D / 16;
    const int i = threadIdx.x % n;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kPackedThreads / n) + threadIdx.x / n;
    const bool is_v = blockIdx.y >= static_cast<unsigned>(p.Hkv);
    const int head = is_v ? blockIdx.y - p.Hkv : blockIdx.y;
    grid_wait();
    grid_launch_dependents();
    if (row >= p.n_rows) return;
    const int slot = p.slots[row];
    if (slot < 0 || slot >= p.n_slots) return;
    const PackedPlace<D> at(slot, head, p.Hkv, p.page_shift);
    uint8_t scale;
    const uint2 c = quantise((is_v ? p.v + row * p.v_stride : p.k + row * p.k_stride) + head * D + i * 16, scale);
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

// Two codes (a byte) times the scale, as bf16: both products are exact in fp16 and in bf16.
__device__ __forceinline__ uint32_t values_of_byte(uint32_t byte, uint32_t scale2) {
    uint32_t h, r;
    asm("{\n\t.reg .b8 c, z0, z1, z2;\n\t"
        "mov.b32 {c, z0, z1, z2}, %1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(h) : "r"(byte));
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(h), "r"(scale2));
    const __half2 v = *reinterpret_cast<const __half2*>(&r);
    return pack_bf16x2(__low2float(v), __high2float(v));
}

template <int D>
__global__ void __launch_bounds__(kPackedThreads) packed_load_kernel(const __grid_constant__ PackedRows p) {
    constexpr int n = D / 16;
    const int i = threadIdx.x % n;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kPackedThreads / n) + threadIdx.x / n;
    const bool is_v = blockIdx.y >= static_cast<unsigned>(p.Hkv);
    const int head = is_v ? blockIdx.y - p.Hkv : blockIdx.y;
    grid_wait();
    grid_launch_dependents();
    if (row >= p.n_rows) return;
    const int slot = p.slots[row];
    uint32_t out[8] = {};
    if (slot >= 0 && slot < p.n_slots) {
        const PackedPlace<D> at(slot, head, p.Hkv, p.page_shift);
        uint2 c;
        if (!is_v || D == 128) c = __ldcg(reinterpret_cast<const uint2*>(p.cache + (is_v ? at.v_codes(i) : at.k_codes(i))));
        else c = make_uint2(__ldcg(reinterpret_cast<const uint32_t*>(p.cache + at.v_codes(2 * i))), __ldcg(reinterpret_cast<const uint32_t*>(p.cache + at.v_codes(2 * i + 1))));
        const uint32_t bits = __ldcg(p.cache + (is_v ? at.v_scale(i) : at.k_scale(i)));
        uint32_t scale2;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(scale2) : "h"(static_cast<uint16_t>(bits << 8 | bits)));
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            out[b] = values_of_byte(c.x >> (8 * b) & 0xffu, scale2);
            out[4 + b] = values_of_byte(c.y >> (8 * b) & 0xffu, scale2);
        }
    }
    uint4* const to = reinterpret_cast<uint4*>((is_v ? p.v_out : p.k_out) + (row * p.Hkv + head) * D + i * 16);
    to[0] = make_uint4(out[0], out[1], out[2], out[3]);
    to[1] = make_uint4(out[4], out[5], out[6], out[7]);
}

static dim3 packed_grid(const PackedRows& p, int head_dim) {
    const int64_t rows = kPackedThreads / (head_dim / 16);
    return dim3(static_cast<unsigned>((p.n_rows + rows - 1) / rows), static_cast<unsigned>(2 * p.Hkv));
}

cudaError_t launch_packed_store(const PackedRows& p, int head_dim, cudaStream_t stream) {
    return head_dim == 128 ? launch_chained<packed_store_kernel<128>>(packed_grid(p, 128), kPackedThreads, 0, stream, p)
                           : launch_chained<packed_store_kernel<64>>(packed_grid(p, 64), kPackedThreads, 0, stream, p);
}

cudaError_t launch_packed_load(const PackedRows& p, int head_dim, cudaStream_t stream) {
    return head_dim == 128 ? launch_chained<packed_load_kernel<128>>(packed_grid(p, 128), kPackedThreads, 0, stream, p)
                           : launch_chained<packed_load_kernel<64>>(packed_grid(p, 64), kPackedThreads, 0, stream, p);
}

}  // namespace pevlm
