// Chunk attention of few rows (single tokens above all) over the paged cache, where there is little to read: what bounds such a call is the
// way from the block table to a key and back, so every warp of the machine takes a few keys at once and a unit's blocks merge in
// their cluster's shared memory, in one launch.
//
// A unit (request, KV head) has up to 8 NT rows (token * G + head in group).  bf16: a warp takes 16 keys at a time, keys and values straight from
// memory into the fragments of mma.sync (m16n8k16), keys as M, rows as N:
//   S^T (16 keys x 8 rows) = K Q^T.  The sum over channels may run in any order, so lane (g, q) = (lane / 4, lane % 4) holds of keys g and
//       g + 8 the 16 channels from 16 q on of every 64, 32 bytes that lie together, and of row g the same channels.
//   P^T: two 8 x 8 transpositions (movmatrix) take the scores' fragment to the other operand's.
//   O^T (16 channels x 8 rows) += V^T P^T.  The channels may stand in any order, so lane (g, q) holds of keys 2 q, 2 q + 1, 2 q + 8 and
//       2 q + 9 the D / 8 channels from D g / 8 on; two keys' halves are put together by byte permutation.  A lane ends with these channels
//       of rows 2 q and 2 q + 1.
// fp32: a warp takes 8 keys at a time on the FMA units, four lanes to a key for the scores (queries from shared memory, two exchanges a row), then
// all lanes to a value's channels (a probability by one exchange).
// The reference of a row's exponentials moves only when a score passes it by 2^8 (for all lanes at once), so the loop has one vote and no
// exchange.  Sums are fp32; a probability enters its product as bf16.
#include <type_traits>

#include "attn_tiles.cuh"
#include "chunk_attention.cuh"

namespace radar {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps, kChunk = 16;        // keys of a chunk: they lie in one page
constexpr int kMostSplit = 16;                                        // blocks of a unit: a cluster

template <int D, int R>
struct RowsSmem {
    static constexpr int kRows = R;
    float o[kWarps][kRows][D];           // of each warp
    float2 ml[kWarps][kRows];            // (m in log2 units, l)
    float block_o[kRows][D];             // of the block, for its cluster
    float2 block_ml[kRows];
};

template <int W>
__device__ __forceinline__ void load_words(const void* p, bool on, uint32_t (&w)[W]) {
    static_assert(W == 8 || W == 4, "32 or 16 bytes");
    if (!on) {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
        return;
    }
    if constexpr (W == 8)
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
    else
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
}
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed_8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float4 load_cluster4(uint32_t at) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ float2 load_cluster2(uint32_t at) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
    return v;
}
// weight of a part with maximum m in a whole with maximum top (-inf: nothing there)
__device__ __forceinline__ float part_weight(float m, float top) { return ex2(m - (top == -CUDART_INF_F ? 0.f : top)); }

// The unit's output from its warps' parts, by all threads of its blocks.
template <typename T, int D, int R>
__device__ __forceinline__ void merge_parts(RowsSmem<D, R>& sm, const ChunkParams& P, const ChunkSeq& s, int g, int rows, int rank, int split) {
    const radar_chunk_attn_args& a = P.a;
    const int tid = threadIdx.x;
    __syncthreads();
    auto write = [&](int r, int c4, float4 v, float top, float sum) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int token = r / P.G;
        const int64_t out_row = (int64_t)(s.q0 + token) * a.Hq + g * P.G + r - token * P.G;
        T* const to = reinterpret_cast<T*>(a.O) + out_row * D + c4 * 4;
        if constexpr (sizeof(T) == 2) {
            const __nv_bfloat162 x = __floats2bfloat162_rn(v.x * inv, v.y * inv), y = __floats2bfloat162_rn(v.z * inv, v.w * inv);
            *reinterpret_cast<uint2*>(to) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
        } else {
            *reinterpret_cast<float4*>(to) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        }
        if (c4 == 0 && a.lse != nullptr) a.lse[out_row] = sum == 0.f ? -CUDART_INF_F : lse_of(top, sum);
    };
    // parts: their (m, l) and four channels; added up in order.  A part that saw no key has l = 0 and O = 0; one whose sum is NaN makes the row NaN
    auto merge = [&](int n, auto ml_of, auto o_of, float4& v, float& top, float& sum) {
        top = -CUDART_INF_F;
        for (int i = 0; i < n; ++i) top = fmaxf(top, ml_of(i).x);
        v = make_float4(0.f, 0.f, 0.f, 0.f);
        sum = 0.f;
        for (int i = 0; i < n; ++i) {
            const float2 ml = ml_of(i);
            const float4 x = o_of(i);
            const float w = part_weight(ml.x, top);
            sum = fmaf(ml.y, w, sum);
            v.x = fmaf(x.x, w, v.x); v.y = fmaf(x.y, w, v.y); v.z = fmaf(x.z, w, v.z); v.w = fmaf(x.w, w, v.w);
        }
    };
    for (int e = tid; e < rows * (D / 4); e += kThreads) {
        const int r = e / (D / 4), c4 = e % (D / 4);
        float4 v;
        float top, sum;
        merge(kWarps, [&](int i) { return sm.ml[i][r]; }, [&](int i) { return *reinterpret_cast<const float4*>(&sm.o[i][r][c4 * 4]); }, v, top, sum);
        if (split == 1) {
            write(r, c4, v, top, sum);
        } else {
            *reinterpret_cast<float4*>(&sm.block_o[r][c4 * 4]) = v;
            if (c4 == 0) sm.block_ml[r] = make_float2(top, sum);
        }
    }
    if (split == 1) return;
    cluster_barrier();
    for (int e = rank * kThreads + tid; e < rows * (D / 4); e += split * kThreads) {
        const int r = e / (D / 4), c4 = e % (D / 4);
        float4 v;
        float top, sum;
        merge(split, [&](int i) { return load_cluster2(cluster_addr(&sm.block_ml[r], i)); }, [&](int i) { return load_cluster4(cluster_addr(&sm.block_o[r][c4 * 4], i)); }, v, top, sum);
        write(r, c4, v, top, sum);
    }
    cluster_barrier();                                       // nobody leaves while its shared memory is read
}

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 2 : 1) chunk_attn_rows_kernel(const ChunkParams P, const int split) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    using Smem = RowsSmem<D, 8 * NT>;
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
    constexpr int kBlocks = D / 64, MT = D / 16, kVWords = D / 16;     // 64-channel blocks, 16-channel tiles of O, words of a lane's values
    const radar_chunk_attn_args& a = P.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lg = lane >> 2, lq = lane & 3;
    const int rank = blockIdx.x % split, unit = blockIdx.x / split, b = unit / a.Hkv, g = unit - b * a.Hkv;
    chain_wait();
    bool seq_ok;
    const ChunkSeq s = chunk_seq(a, b, seq_ok);
    if (!seq_ok && rank == 0 && g == 0 && tid == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
    const int rows = s.n * P.G;                              // (at most 8 NT: the host has looked at max_new)
    if (rows == 0) return;                                   // (the whole cluster)
    const int chunks = (s.len + kChunk - 1) / kChunk, step = split * kWarps, per_page = a.page_size / kChunk;
    const int n_cache_pages = (int)(a.cache_rows / a.page_size);
    const int* const table = a.block_table + (int64_t)b * a.max_pages;
    const int64_t row_elems = (int64_t)a.Hkv * D;
    const __nv_bfloat16 *const Kc = reinterpret_cast<const __nv_bfloat16*>(a.Kc) + g * D, *const Vc = reinterpret_cast<const __nv_bfloat16*>(a.Vc) + g * D;
    auto page_of = [&](int chunk) { return chunk < chunks ? table[chunk / per_page] : 0; };

    int chunk = rank * kWarps + warp;
    int page = page_of(chunk);
    // the rows' queries
    uint32_t qw[NT][kBlocks][8];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = t * 8 + lg, token = r / P.G;
        const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.Q) + (int64_t)(s.q0 + token) * a.q_row_stride + (int64_t)(g * P.G + r - token * P.G) * D + lq * 16;
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t w[4];
                load_words<4>(q + k * 64 + h * 8, r < rows, w);
#pragma unroll
                for (int i = 0; i < 4; ++i) qw[t][k][h * 4 + i] = w[i];
            }
    }
    // keys that rows 2 lq and 2 lq + 1 of each tile see
    int lim[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) lim[t][i] = s.len - s.n + (t * 8 + 2 * lq + i) / P.G + 1;
    float o[NT][MT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int i = 0; i < 2; ++i) { m[t][i] = -CUDART_INF_F; l[t][i] = 0.f; }
#pragma unroll
        for (int j = 0; j < MT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[t][j][i] = 0.f;
    }
#pragma unroll 1
    for (; chunk < chunks; chunk += step) {
        if (page < 0 || page >= n_cache_pages) { if (lane == 0) set_status(P.status, RADAR_ERR_INVALID_ARG); page = 0; }
        const int first = chunk * kChunk;
        const int64_t row0 = (int64_t)page * a.page_size + (chunk % per_page) * kChunk;
        // (a cache of less than one page has no page at all: rows behind its end are not read)
        const int there = (int)min((int64_t)(s.len - first), a.cache_rows - row0);
        uint32_t kw[2][kBlocks][8], vw[4][kVWords];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int k = 0; k < kBlocks; ++k) load_words<8>(Kc + (row0 + lg + 8 * h) * row_elems + k * 64 + lq * 16, lg + 8 * h < there, kw[h][k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = 2 * lq + (i & 1) + 8 * (i >> 1);
            load_words<kVWords>(Vc + (row0 + key) * row_elems + lg * (D / 8), key < there, vw[i]);
        }
        page = page_of(chunk + step);
        float c[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) c[t][i] = 0.f;
#pragma unroll
            for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) mma_16x8x16(c[t], kw[0][k][2 * i], kw[1][k][2 * i], kw[0][k][2 * i + 1], kw[1][k][2 * i + 1], qw[t][k][2 * i], qw[t][k][2 * i + 1]);
        }
        // ---- c: (key lg, row 2 lq), (lg, 2 lq + 1), (lg + 8, 2 lq), (lg + 8, 2 lq + 1) ----
        bool passed = false;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[t][i] = first + lg + 8 * (i >> 1) < lim[t][i & 1] ? c[t][i] * P.scale_log2 : -CUDART_INF_F;
                passed |= c[t][i] > m[t][i & 1] + kRescaleThreshold;
            }
        if (__any_sync(kFull, passed)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float top = fmaxf(c[t][i], c[t][i + 2]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
                    top = fmaxf(top, m[t][i]);
                    const float factor = part_weight(m[t][i], top);
                    m[t][i] = top;
                    l[t][i] *= factor;
#pragma unroll
                    for (int j = 0; j < MT; ++j) { o[t][j][i] *= factor; o[t][j][i + 2] *= factor; }
                }
        }
        uint32_t p[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float top = m[t][i & 1];
                c[t][i] = ex2(c[t][i] - (top == -CUDART_INF_F ? 0.f : top));
                l[t][i & 1] += c[t][i];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const __nv_bfloat162 two = __floats2bfloat162_rn(c[t][2 * h], c[t][2 * h + 1]);
                p[t][h] = transposed_8x8(*reinterpret_cast<const uint32_t*>(&two));       // keys 2 lq + 8 h and the next of row lg
            }
        }
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            const uint32_t a0 = __byte_perm(vw[0][j], vw[1][j], 0x5410), a1 = __byte_perm(vw[0][j], vw[1][j], 0x7632);
            const uint32_t a2 = __byte_perm(vw[2][j], vw[3][j], 0x5410), a3 = __byte_perm(vw[2][j], vw[3][j], 0x7632);
#pragma unroll
            for (int t = 0; t < NT; ++t) mma_16x8x16(o[t][j], a0, a1, a2, a3, p[t][0], p[t][1]);
        }
    }
    // ---- the warps' parts; a lane has channels D lg / 8 + 2 j and the next of rows 2 lq and 2 lq + 1 ----
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[t][i] += __shfl_xor_sync(kFull, l[t][i], d);
            const int r = t * 8 + 2 * lq + i;
            if (lg == 0) sm.ml[warp][r] = make_float2(m[t][i], l[t][i]);
#pragma unroll
            for (int j = 0; j < MT; ++j) *reinterpret_cast<float2*>(&sm.o[warp][r][lg * (D / 8) + 2 * j]) = make_float2(o[t][j][i], o[t][j][i + 2]);
        }
    merge_parts<__nv_bfloat16>(sm, P, s, g, rows, rank, split);
}

constexpr int kChunkF32 = 8;             // keys of a chunk

template <int D, int R>
__global__ void __launch_bounds__(kThreads, R <= 8 ? 2 : 1) chunk_attn_rows_f32_kernel(const ChunkParams P, const int split) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    using Smem = RowsSmem<D, R>;
    Smem& sm = *reinterpret_cast<Smem*>(smem_raw);
    float (*const sq)[D] = sm.block_o;                       // the queries, until the warps' parts are merged
    constexpr int kBlocks = D / 32, E = D / 32;              // 32-channel blocks, channels of a lane's values
    const radar_chunk_attn_args& a = P.a;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lg = lane >> 2, lq = lane & 3;
    const int rank = blockIdx.x % split, unit = blockIdx.x / split, b = unit / a.Hkv, g = unit - b * a.Hkv;
    chain_wait();
    bool seq_ok;
    const ChunkSeq s = chunk_seq(a, b, seq_ok);
    if (!seq_ok && rank == 0 && g == 0 && tid == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
    const int rows = s.n * P.G;                              // (at most R: the host has looked at max_new)
    if (rows == 0) return;                                   // (the whole cluster)
    const int chunks = (s.len + kChunkF32 - 1) / kChunkF32, step = split * kWarps, per_page = a.page_size / kChunkF32;
    const int n_cache_pages = (int)(a.cache_rows / a.page_size);
    const int* const table = a.block_table + (int64_t)b * a.max_pages;
    const int64_t row_elems = (int64_t)a.Hkv * D;
    const float *const Kc = reinterpret_cast<const float*>(a.Kc) + g * D, *const Vc = reinterpret_cast<const float*>(a.Vc) + g * D;
    auto page_of = [&](int chunk) { return chunk < chunks ? table[chunk / per_page] : 0; };
    int chunk = rank * kWarps + warp;
    int page = page_of(chunk);
    for (int e = tid; e < R * (D / 4); e += kThreads) {
        const int r = e / (D / 4), c = e % (D / 4) * 4, token = r / P.G;
        float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < rows) q = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(a.Q) + (int64_t)(s.q0 + token) * a.q_row_stride + (int64_t)(g * P.G + r - token * P.G) * D + c);
        *reinterpret_cast<float4*>(&sq[r][c]) = q;
    }
    __syncthreads();
    const int seen = s.len - s.n + 1;                        // keys that the first token sees
    float o[R][E], m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = -CUDART_INF_F;
        l[r] = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[r][e] = 0.f;
    }
#pragma unroll 1
    for (; chunk < chunks; chunk += step) {
        if (page < 0 || page >= n_cache_pages) { if (lane == 0) set_status(P.status, RADAR_ERR_INVALID_ARG); page = 0; }
        const int first = chunk * kChunkF32;
        const int64_t row0 = (int64_t)page * a.page_size + (chunk % per_page) * kChunkF32;
        const int there = (int)min((int64_t)(s.len - first), a.cache_rows - row0);
        uint32_t kw[kBlocks][8], vw[kChunkF32][E];
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) load_words<8>(Kc + (row0 + lg) * row_elems + k * 32 + lq * 8, lg < there, kw[k]);
#pragma unroll
        for (int i = 0; i < kChunkF32; ++i) {
            const float* at = Vc + (row0 + i) * row_elems + lane * E;
            if constexpr (E == 4) {
                load_words<4>(at, i < there, vw[i]);
            } else {
                const float2 x = i < there ? *reinterpret_cast<const float2*>(at) : make_float2(0.f, 0.f);
                vw[i][0] = __float_as_uint(x.x);
                vw[i][1] = __float_as_uint(x.y);
            }
        }
        page = page_of(chunk + step);
        // ---- scores of key lg, in its four lanes ----
        float c[R];
        bool passed = false;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float2 t = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 q = *reinterpret_cast<const float4*>(&sq[r][k * 32 + lq * 8 + h * 4]);
                    t.x = fmaf(q.x, __uint_as_float(kw[k][h * 4]), t.x);
                    t.y = fmaf(q.y, __uint_as_float(kw[k][h * 4 + 1]), t.y);
                    t.x = fmaf(q.z, __uint_as_float(kw[k][h * 4 + 2]), t.x);
                    t.y = fmaf(q.w, __uint_as_float(kw[k][h * 4 + 3]), t.y);
                }
            float x = t.x + t.y;
            x += __shfl_xor_sync(kFull, x, 1);
            x += __shfl_xor_sync(kFull, x, 2);
            c[r] = first + lg < seen + r / P.G ? x * P.scale_log2 : -CUDART_INF_F;
            passed |= c[r] > m[r] + kRescaleThreshold;
        }
        if (__any_sync(kFull, passed)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float top = c[r];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
                top = fmaxf(top, m[r]);
                const float factor = part_weight(m[r], top);
                m[r] = top;
                l[r] *= factor;
#pragma unroll
                for (int e = 0; e < E; ++e) o[r][e] *= factor;
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            c[r] = ex2(c[r] - (m[r] == -CUDART_INF_F ? 0.f : m[r]));
            l[r] += c[r];
        }
#pragma unroll
        for (int i = 0; i < kChunkF32; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float p = __shfl_sync(kFull, c[r], 4 * i);
#pragma unroll
                for (int e = 0; e < E; ++e) o[r][e] = fmaf(p, __uint_as_float(vw[i][e]), o[r][e]);
            }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[r] += __shfl_xor_sync(kFull, l[r], d);      // (four lanes have a key's)
        if (lane == 0) sm.ml[warp][r] = make_float2(m[r], l[r]);
#pragma unroll
        for (int e = 0; e < E; ++e) sm.o[warp][r][lane * E + e] = o[r][e];
    }
    merge_parts<float>(sm, P, s, g, rows, rank, split);
}

struct RowsLaunch {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    RowsLaunch(long long units, int split, size_t smem, cudaStream_t stream) : cfg{}, attr{} {
        cfg.gridDim = dim3((unsigned)(units * split));
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = stream;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)split;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = split > 1 ? 2 : 1;
    }
    RowsLaunch(const RowsLaunch&) = delete;
};

// Blocks of a unit: as many as leave every warp a chunk, in clusters that are all resident at once (the device is asked once for each
// size: clusters of 8 and 16 do not fill every part of the machine).
//
// Where a warp would go through many chunks, one load behind the other, the tensor cores' form with its copies in flight is the faster
// one: beyond 8 chunks a warp, 24 where the blocks fill the machine (which then has enough loads in flight).  One token, us, this form / that
// one (chunks a warp), 32 / 8 heads of 128: B = 1, 1024 tokens 6.3 / 11.6, 4096 (2) 10.8 / 15.1, 8192 (4) 16.3 / 18.0, 16384 (8) 25.7 / 24.0, 32768 (16)
// 42.8 / 34.5, 65536 (32) 75 / 54; B = 2, 4096 (4) 14.9 / 17.1, 8192 (8) 24.1 / 22.9, 16384 (16) 40.9 / 33.5; filled: B = 8, 4096 (8) 28.2 / 32.3, 8192
// (16) 48.8 / 51.9; B = 32, 1024 (8) 27.0 / 34.5, 4096 (32) 88.8 / 92.9, 8192 (64) 170.4 / 169.6; B = 128, 1024 (8) 98.5 / 96.3, 2048 (16) 183 / 174, 4096
// (32) 348 / 328; 16 / 1 heads: B = 1, 16384 (8) 16.5 / 18.9, 32768 (16) 25.7 / 23.6; B = 8, 8192 (8) 18.5 / 18.3, 16384 (16) 32.0 / 24.4; B = 64, 4096
// (16, filled) 31.6 / 33.4, 8192 (32) 55.2 / 53.1.  So the forms meet between 4 and 16 chunks, or between 8 and 64, and near the rule's bounds either may be
// up to 7 % ahead.
// fp32 against the form of whole tiles: up to 8 rows this one, but for a few units over very many keys, which that one spreads over the machine: 32 / 8
// heads of 128 (4 rows): B = 1, 1024 tokens 8.4 / 19.1, 65536 174 / 268; B = 32, 4096 180 / 517; 8 / 1 heads of 64 (8 rows): B = 1, 16384 (16 chunks a warp,
// 16 blocks) 30 / 54, 65536 112 / 72; B = 4, 16384 33 / 40.  (From a quarter of the SMs' number of blocks on the rule asks no more for the length, which
// costs where 8 rows meet a very long cache: B = 4, 65536 117 / 88; B = 8 166 / 145.)  16 rows, one block an SM: this one up to 8 chunks a warp or where
// the blocks fill the machine: 16 / 1 heads of 128: B = 1, 8192 tokens (8) 38 / 43, 16384 (16) 67 / 61, 65536 (64) 252 / 93; B = 4, 8192 (8) 40 / 42, 16384 (16)
// 72 / 60; B = 16, 2048 (8) 38 / 33, 4096 (16) 70 / 52; B = 32, 2048 (8, filled) 40 / 51, 16384 (64, filled) 254 / 266.
template <typename T, int D, int R>
int launch_rows(radar_ctx* ctx, const ChunkParams& P, cudaStream_t stream, bool& taken) {
    void (*kernel)(ChunkParams, int);
    if constexpr (sizeof(T) == 2) kernel = chunk_attn_rows_kernel<D, (R + 7) / 8>;
    else kernel = chunk_attn_rows_f32_kernel<D, R>;
    constexpr int kKeys = sizeof(T) == 2 ? kChunk : kChunkF32;
    const size_t smem = sizeof(RowsSmem<D, R>);
    constexpr int variant = sizeof(T) == 2 ? 2 * (D == 128) + R / 8 - 1 : 4 + 3 * (D == 128) + (R == 4 ? 0 : R / 8);
    const bool first = ctx->smem_room[RADAR_SMEM_CHUNK_ROWS + variant] == 0;
    RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, RADAR_SMEM_CHUNK_ROWS + variant, kernel, smem));
    if (first) RADAR_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    const long long units = (long long)P.a.B * P.a.Hkv;
    int split = 1;
    for (int i = 0; 2 * split <= kMostSplit && (long long)split * kWarps * kKeys < P.a.max_cache_len; ++i) {
        int& clusters = ctx->chunk_clusters[variant][i];     // of 2 * split blocks
        if (clusters == 0) {
            RowsLaunch l(1, 2 * split, smem, stream);
            RADAR_CUDA_CHECK(cudaOccupancyMaxActiveClusters(&clusters, kernel, &l.cfg));
            if (clusters == 0) clusters = -1;
        }
        if (units > clusters) break;
        split *= 2;
    }
    const bool filled = units * split * 5 >= 4ll * ctx->sm_count * (R <= 8 ? 2 : 1);
    if (sizeof(T) == 2) taken = P.a.max_cache_len <= (filled ? 24ll : 8ll) * split * kWarps * kKeys;
    else taken = (R <= 8 ? units * split * 4 >= ctx->sm_count : filled) || P.a.max_cache_len <= (R <= 8 ? 16ll : 8ll) * split * kWarps * kKeys;
    if (!taken) return RADAR_OK;
    RowsLaunch l(units, split, smem, stream);
    radar_launch_scope scope(ctx, RADAR_K_CHUNK_ATTN, stream);
    RADAR_CUDA_CHECK(cudaLaunchKernelEx(&l.cfg, kernel, P, split));
    return RADAR_OK;
}

}  // namespace

int chunk_rows_launch(radar_ctx* ctx, const radar_chunk_attn_args* a, cudaStream_t stream, bool& taken) {
    const int G = a->Hq / a->Hkv;
    const long long rows = (long long)a->max_new * G;
    taken = false;
    if (rows > 16 || (long long)a->B * a->Hkv > INT32_MAX / kMostSplit || ((reinterpret_cast<uintptr_t>(a->Kc) | reinterpret_cast<uintptr_t>(a->Vc)) & 31) != 0) return RADAR_OK;
    const ChunkParams P = chunk_params(ctx, *a, G, 128, 1);
    auto go = [&](auto t, auto d) {
        using T = decltype(t);
        constexpr int D = decltype(d)::value;
        if constexpr (sizeof(T) == 4)
            if (rows <= 4) return launch_rows<T, D, 4>(ctx, P, stream, taken);
        return rows > 8 ? launch_rows<T, D, 16>(ctx, P, stream, taken) : launch_rows<T, D, 8>(ctx, P, stream, taken);
    };
    using d64 = std::integral_constant<int, 64>;
    using d128 = std::integral_constant<int, 128>;
    if (a->dtype == RADAR_F32) return a->d == 128 ? go(0.f, d128{}) : go(0.f, d64{});
    return a->d == 128 ? go(__nv_bfloat16{}, d128{}) : go(__nv_bfloat16{}, d64{});
}

}  // namespace radar
