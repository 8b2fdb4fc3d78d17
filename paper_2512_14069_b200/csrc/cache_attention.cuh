// What the kernels of the attention over the 4-bit cache share.
#pragma once
#include "cache.cuh"

namespace radar {

struct CacheAttnParams {
    radar_cache_attn_args a;
    int G;
    int n_tiles, n_splits, split_len;            // row tiles, splits of a unit, keys of a split
    int blocks_per_page, page_shift_blocks;      // log2 of it, -1: no power of two
    int64_t page_bytes;
    float scale_log2;
    float2* part_ml;                             // [B][rows][Hq][n_splits] (maximum in log2 units, sum)
    float* part_o;                               // ... [D], not normalised
    int* status;
};

// m ln 2 + ln l, m in log2 units
__device__ __forceinline__ float lse_of(float m, float l) {
    constexpr float kHi = 0.693147182f, kLo = (float)(0.6931471805599453 - (double)kHi);
    return fmaf(m, kHi, fmaf(m, kLo, logf(l)));
}
// eight channels of a finished row: O and, from one of its threads, lse
__device__ __forceinline__ void write_row(const radar_cache_attn_args& a, int b, int node, int hq, int c, int D, const float (&o)[8], float m, float l, bool first) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(o[2 * e] * inv, o[2 * e + 1] * inv);
        w[e] = *reinterpret_cast<const uint32_t*>(&t);
    }
    *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(a.O) + (((int64_t)b * a.rows + node) * a.Hq + hq) * D + c) = make_uint4(w[0], w[1], w[2], w[3]);
    if (first && a.lse != nullptr) a.lse[((int64_t)b * a.Hq + hq) * a.rows + node] = l > 0.f ? lse_of(m, l) : -CUDART_INF_F;
}

}  // namespace radar
