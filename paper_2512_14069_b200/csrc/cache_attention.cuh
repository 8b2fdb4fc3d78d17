// What the kernels of the attention over the 4-bit cache share.
#pragma once
#include "cache.cuh"

namespace radar {

struct CacheAttnParams {
    radar_cache_attn_args a;
    int G;
    int blocks, cluster;                         // of the launch; of a unit, in the form for little work
    int blocks_per_page, page_shift_blocks;      // log2 of it, -1: no power of two
    float scale_log2;
    // [blocks][2][8 or 16 rows]: a block's share of the unit that its range begins in, and of the one that it ends in
    float2* part_ml;                             // (maximum in log2 units, sum)
    float* part_o;                               // ... [D], not normalised
    int* status;
};

// a contiguous piece of global memory into shared memory; 16-byte aligned, a multiple of 16 bytes
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_addr(dst)), "l"(src), "r"(bytes), "r"(smem_addr(bar)) : "memory");
}

// --- the form for many query rows (cache_attention_tc.cu); its workspace serves every size -------
size_t cache_attn_tc_workspace_bytes(const radar_ctx* ctx, int d);
int cache_attn_tc_launch(radar_ctx* ctx, const radar_cache_attn_args* a, cudaStream_t stream);
}  // namespace radar
