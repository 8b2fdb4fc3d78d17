// The 4-bit cache's format (include/radar.h) in device code: where the parts of a block are, and how codes become bf16 pairs.
#pragma once
#include "common.cuh"

namespace radar {
namespace cache4 {

constexpr int kBlock = 16;               // tokens of a block, and channels of a group
// byte offsets of the parts of a block of head dimension D
template <int D>
struct Layout {
    static constexpr int kKScales = 8 * D, kVCodes = 9 * D, kVScales = 17 * D, kBytes = 18 * D;
    static constexpr int kRow = D / 2;   // bytes of a row's codes
    static constexpr int kW = D / 64;
};

inline bool page_size_ok(int p) { return p == 16 || p == 32 || p == 64 || (p > 0 && p % 128 == 0); }
inline int64_t page_bytes(int Hkv, int d, int page_size) { return (int64_t)Hkv * (page_size / kBlock) * 18 * d; }

__host__ __device__ constexpr int v_place(int r) { return (r & 1) * 4 + ((r & 7) >> 1) + (r & 8); }
template <int D>
__host__ __device__ constexpr int k_scale_at(int r, int g) {
    constexpr int w = D / 64;
    return Layout<D>::kKScales + (r & 7) * (D / 8) + g / w * 2 * w + (r >> 3) * w + g % w;
}
template <int D>
__host__ __device__ constexpr int v_scale_at(int r, int g) {
    return Layout<D>::kVScales + g * 16 + (v_place(r) & 3) * 4 + (v_place(r) >> 2);
}
// codes of the eight bytes `unit` (16 channels) of row r
template <int D>
__host__ __device__ constexpr int k_codes_at(int r, int unit) { return r * Layout<D>::kRow + unit * 8; }
template <int D>
__host__ __device__ constexpr int v_codes_at(int r, int unit) {
    const int p = v_place(r);
    return Layout<D>::kVCodes + p * Layout<D>::kRow + ((unit * 8) ^ (D == 128 && (p & 2) ? 32 : 0));
}

// Decoding.  A scale byte times 16 plus 107 << 7 is the bf16 number s.  A code or'ed into the low mantissa bits of 128 is
// the bf16 number 128 + (q + 8), and fma(128 + (q + 8), s, -136 s) is q s: 136 s is 17 times eight, and s has four significant
// bits, so the addend is a bf16 number, the result too, and nothing is rounded.
__device__ __forceinline__ uint32_t scale_pair(uint32_t bytes_0x0x) { return bytes_0x0x * 16u + 0x35803580u; }
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t offset_pair(uint32_t s) {           // -136 s
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(s), "r"(0xC308C308u));
    return d;
}
// the codes in bits 4 i .. 4 i + 3 of the two halves of w
template <int I>
__device__ __forceinline__ uint32_t decode(uint32_t w, uint32_t s, uint32_t off) {
    uint32_t x;
    asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(x) : "r"(I ? w >> (4 * I) : w));      // (a & b) | c
    return fma_bf16x2(x, s, off);
}

}  // namespace cache4
}  // namespace radar
