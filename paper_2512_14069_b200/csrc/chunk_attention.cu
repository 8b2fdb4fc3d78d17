// radar_chunk_attention: the entry point, and the form for fp32 rows, on the FMA units.
//
// Scores s = scale q.k of the keys a row sees, online softmax over tiles of 64 keys: m = a row's maximum so far, moved (and l = sum exp(s - m),
// O = sum exp(s - m) v with it) only where a score passes it by 2^8; everything in fp32.
//
// A head group is a KV head's G query heads (one query head where G is above 64, so that a unit holds a whole token), a unit 64 rows.  A block of
// 128 threads, two to an SM, has Q (64 rows), K and V (64 keys each) and P in shared memory; a thread holds 8 rows x 4 keys of the scores, then 8
// rows x d / 16 channels of O, in pairs of rows that one instruction multiplies by a key's or value's channel.  A prompt of 2048 tokens, 32 / 8 heads
// of 128: 842 us; 888 with scores one by one from rows side by side, 924 with O one by one too, 1191 with one block an SM, a row of padding in P
// and every tile rescaled.  A warp without live rows only fetches (8 requests of 16 rows over 16384 tokens 120 -> 87).  What bounds it: the issue of
// FMAs with two warps to a scheduler: 41 TFLOP/s of the 72 that FMAs alone reach (three blocks an SM, d = 64: no faster).
#include <algorithm>
#include <climits>

#include "attn_tiles.cuh"
#include "chunk_attention.cuh"

namespace radar {
namespace {

constexpr int kFmaThreads = 128, kFmaRows = 64, kFmaKeys = 64, kPStride = 4 * kFmaRows + 4;

struct FmaCosts {
    static constexpr int kTile = kFmaKeys, kOne = 1, kTwo = 1, kUnit = kFmaKeys;
};

template <int D>
struct FmaSmem {
    float q[kFmaRows * D], k[kFmaKeys * D], v[kFmaKeys * D];
    float p[16 * kPStride];              // [key % 16][key / 16][row]: writes of neighbouring keys meet in no bank, and two blocks fit an SM
    int at[2][kFmaKeys];                 // cache rows of a tile's keys; below 0: there is none
};

// two fp32 numbers in a register pair, and the arithmetic on both at once
typedef unsigned long long Two;
__device__ __forceinline__ Two two_of(float x, float y) {
    Two t;
    asm("mov.b64 %0, {%1, %2};" : "=l"(t) : "f"(x), "f"(y));
    return t;
}
__device__ __forceinline__ float2 both(Two t) {
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(t));
    return v;
}
__device__ __forceinline__ Two fma_two(Two a, Two b, Two c) {
    Two d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ Two mul_two(Two a, Two b) {
    Two d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ void copy16(float* to, const float* from, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(to)), "l"(from), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int D>
__global__ void __launch_bounds__(kFmaThreads, 2) chunk_attn_fma_kernel(const ChunkParams P) {
    chain_wait();
    extern __shared__ __align__(16) unsigned char smem_raw[];
    FmaSmem<D>& sm = *reinterpret_cast<FmaSmem<D>*>(smem_raw);
    constexpr int kVec = D / 4, kCols = D / 64;              // float4s of a row, and of a thread's channels
    const radar_chunk_attn_args& a = P.a;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const float* const Q = reinterpret_cast<const float*>(a.Q);
    const int64_t row_elems = (int64_t)a.Hkv * D;
    const int n_cache_pages = (int)(a.cache_rows / a.page_size);
    long long tot;
    Walk<FmaCosts> cur = first_segment<FmaCosts>(P, blockIdx.x, tot);
    ChunkPieces cut;
    cut.unit.valid = 0;
    cut.tot = tot;
    for (int seg = 0; cur.valid(); ++seg) {
        const Unit<FmaCosts> u = cur.u;
        const int b = cur.b, g = cur.g, t0 = cur.t0, n = cur.t1 - cur.t0;
        const int keys = max(u.seen + u.tokens - 1, 0), kv_head = g * P.G / (a.Hq / a.Hkv);
        if (t0 == 0 && n < u.nt) {
            cut.unit.valid = 1; cut.unit.row0 = u.row0; cut.unit.g = g; cut.unit.slot = seg == 0 ? 0 : 1; cut.unit.rows = u.rows;
            cut.nt = u.nt; cut.w = u.w; cut.size_keys = u.keys; cut.u0 = cur.U;
        }
        cur.next(P);
        auto look_up = [&](int t, int buffer) {
            if (tid < kFmaKeys) {
                const int j = t * kFmaKeys + tid;
                int at = -1;
                if (j < keys) {
                    int page = a.block_table[(int64_t)b * a.max_pages + j / a.page_size];
                    if (page < 0 || page >= n_cache_pages) { set_status(P.status, RADAR_ERR_INVALID_ARG); page = 0; }
                    const int64_t row = (int64_t)page * a.page_size + j % a.page_size;
                    if (row < a.cache_rows) at = (int)row;   // (a cache of less than one page; cache_rows: below 2^31)
                }
                sm.at[buffer][tid] = at;
            }
        };
        // keys are stored with their float4s exchanged by the row, so that 16 rows at one channel meet in no bank
        auto fetch = [&](const void* base, float* to, int buffer, bool exchange) {
#pragma unroll 4
            for (int i = tid; i < kFmaKeys * kVec; i += kFmaThreads) {
                const int r = i / kVec, c = i % kVec;
                const int at = sm.at[buffer][r];
                copy16(to + r * D + (exchange ? c ^ (r & 7) : c) * 4, reinterpret_cast<const float*>(base) + max(at, 0) * row_elems + (int64_t)kv_head * D + c * 4, at >= 0);
            }
            copies_end();
        };
        __syncthreads();                                     // the segment before has read its rows
        look_up(t0, 0);
        // queries are stored channel by channel, so that a thread has rows side by side
        for (int i = tid; i < kFmaRows * kVec; i += kFmaThreads) {
            const int r = i % kFmaRows, c = i / kFmaRows, token = (int)(((uint32_t)r * P.g_magic) >> 16);
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < u.rows) x = *reinterpret_cast<const float4*>(Q + (int64_t)(u.row0 + token) * a.q_row_stride + (int64_t)(g * P.G + r - token * P.G) * D + c * 4);
            float* const to = sm.q + c * 4 * kFmaRows + r;
            to[0] = x.x; to[kFmaRows] = x.y; to[2 * kFmaRows] = x.z; to[3 * kFmaRows] = x.w;
        }
        __syncthreads();
        fetch(a.Kc, sm.k, 0, true);
        fetch(a.Vc, sm.v, 0, false);
        Two o[4][4 * kCols];                                 // of rows 2 i and 2 i + 1
        float m[8], l[8];
        int lim[8];
        const bool live = (ty & ~1) * 8 < u.rows;            // the warp has live rows; one that has none only fetches
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = -CUDART_INF_F;
            l[i] = 0.f;
            lim[i] = u.seen + (int)(((uint32_t)(ty * 8 + i) * P.g_magic) >> 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4 * kCols; ++e) o[i][e] = 0;
#pragma unroll 1
        for (int t = t0; t < t0 + n; ++t) {
            const bool more = t + 1 < t0 + n;
            if (more) look_up(t + 1, (t + 1 - t0) & 1);
            copies_wait<1>();
            __syncthreads();
            // ---- 8 rows x 4 keys of S: the keys tx, tx + 16, .. ----
            Two part[4][4];                                  // of rows 2 i and 2 i + 1
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) part[i][j] = 0;
#pragma unroll 8
            for (int c = 0; c < (live ? kVec : 0); ++c) {
                float k4[4][4];
#pragma unroll
                for (int j = 0; j < 4; ++j) *reinterpret_cast<float4*>(k4[j]) = *reinterpret_cast<const float4*>(sm.k + (tx + 16 * j) * D + (c ^ (tx & 7)) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float* at = sm.q + (c * 4 + e) * kFmaRows + ty * 8;
                    const ulonglong2 q0 = *reinterpret_cast<const ulonglong2*>(at), q1 = *reinterpret_cast<const ulonglong2*>(at + 4);
                    const Two q[4] = {q0.x, q0.y, q1.x, q1.y};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const Two k2 = two_of(k4[j][e], k4[j][e]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) part[i][j] = fma_two(q[i], k2, part[i][j]);
                    }
                }
            }
            __syncthreads();
            if (more) fetch(a.Kc, sm.k, (t + 1 - t0) & 1, true);
            else copies_end();
            if (live) {
                // ---- softmax ----
                float s[8][4];
                bool passed = false;
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[i][j] = t * kFmaKeys + tx + 16 * j < lim[i] ? (i & 1 ? both(part[i >> 1][j]).y : both(part[i >> 1][j]).x) * P.scale_log2 : -CUDART_INF_F;
                        passed |= s[i][j] > m[i] + kRescaleThreshold;
                    }
                if (__any_sync(kFull, passed)) {
                    float factor[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float top = fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3]));
#pragma unroll
                        for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
                        top = fmaxf(top, m[i]);
                        factor[i] = ex2(m[i] - (top == -CUDART_INF_F ? 0.f : top));
                        m[i] = top;
                        l[i] *= factor[i];
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const Two f = two_of(factor[2 * i], factor[2 * i + 1]);
#pragma unroll
                        for (int e = 0; e < 4 * kCols; ++e) o[i][e] = mul_two(o[i][e], f);
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[i][j] = ex2(s[i][j] - (m[i] == -CUDART_INF_F ? 0.f : m[i]));
                        l[i] += s[i][j];
                    }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float* to = sm.p + tx * kPStride + j * kFmaRows + ty * 8;
                    *reinterpret_cast<float4*>(to) = make_float4(s[0][j], s[1][j], s[2][j], s[3][j]);
                    *reinterpret_cast<float4*>(to + 4) = make_float4(s[4][j], s[5][j], s[6][j], s[7][j]);
                }
            }
            copies_wait<1>();
            __syncthreads();
            // ---- O += P V ----
#pragma unroll 8
            for (int h = 0; h < (live ? 16 : 0); ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float* at = sm.p + h * kPStride + j * kFmaRows + ty * 8;
                    const ulonglong2 p0 = *reinterpret_cast<const ulonglong2*>(at), p1 = *reinterpret_cast<const ulonglong2*>(at + 4);
                    const Two p[4] = {p0.x, p0.y, p1.x, p1.y};
#pragma unroll
                    for (int c = 0; c < kCols; ++c) {
                        const float4 v4 = *reinterpret_cast<const float4*>(sm.v + (h + 16 * j) * D + c * 64 + tx * 4);
                        const Two v[4] = {two_of(v4.x, v4.x), two_of(v4.y, v4.y), two_of(v4.z, v4.z), two_of(v4.w, v4.w)};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[i][4 * c + e] = fma_two(p[i], v[e], o[i][4 * c + e]);
                    }
                }
            __syncthreads();
            if (more) fetch(a.Vc, sm.v, (t + 1 - t0) & 1, false);
            else copies_end();
        }
        // ---- the rows' results: final ones, or a piece's partials ----
        const bool final_rows = n == u.nt;
        const int slot = seg == 0 ? 0 : 1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) l[i] += __shfl_xor_sync(kFull, l[i], d);
            const int r = ty * 8 + i;
            if (r >= u.rows) continue;
            const int token = (int)(((uint32_t)r * P.g_magic) >> 16);
            const int64_t out_row = (int64_t)(u.row0 + token) * a.Hq + g * P.G + r - token * P.G;
            const int64_t rec = ((int64_t)blockIdx.x * 2 + slot) * P.unit_records + r;
            const float inv = !final_rows ? 1.f : l[i] == 0.f ? 0.f : 1.f / l[i];
            float* to = final_rows ? reinterpret_cast<float*>(a.O) + out_row * D : P.part_o + rec * D;
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (i & 1 ? both(o[i >> 1][4 * c + e]).y : both(o[i >> 1][4 * c + e]).x) * inv;
                *reinterpret_cast<float4*>(to + c * 64 + tx * 4) = make_float4(x[0], x[1], x[2], x[3]);
            }
            if (tx == 0) {
                if (!final_rows) P.part_ml[rec] = make_float2(l[i] == 0.f ? -CUDART_INF_F : m[i], l[i]);
                else if (a.lse != nullptr) a.lse[out_row] = l[i] == 0.f ? -CUDART_INF_F : lse_of(m[i], l[i]);
            }
        }
    }
    copies_wait<0>();
    if (tid < 32) write_cut<FmaCosts>(P, blockIdx.x, cut);
}

// query heads of a group: a unit holds whole tokens
int fma_group(int Hq, int Hkv) { return Hq / Hkv <= kFmaRows ? Hq / Hkv : 1; }
int fma_most_ctas(const radar_ctx* ctx) { return std::min(2 * ctx->sm_count, kMaxCtas); }

template <int D>
int fma_launch(radar_ctx* ctx, const radar_chunk_attn_args& a, cudaStream_t stream) {
    ChunkParams P = chunk_params(ctx, a, fma_group(a.Hq, a.Hkv), kFmaRows, 1);
    P.n_cta = chunk_ctas(P, fma_most_ctas(ctx), std::max(1, (a.max_cache_len + kFmaKeys - 1) / kFmaKeys));
    chunk_carve(P);
    RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, RADAR_SMEM_CHUNK_FMA + (D == 128), chunk_attn_fma_kernel<D>, sizeof(FmaSmem<D>)));
    {
        radar_launch_scope scope(ctx, RADAR_K_CHUNK_ATTN, stream);
        RADAR_CUDA_CHECK(launch_chained(chunk_attn_fma_kernel<D>, dim3((unsigned)P.n_cta), dim3(kFmaThreads), sizeof(FmaSmem<D>), stream, P));
    }
    return chunk_combine<float, D>(ctx, P, stream);
}

bool sizes_ok(int B, int Hq, int Hkv, int d, int dtype) {
    return B > 0 && Hq > 0 && Hkv > 0 && Hq % Hkv == 0 && (d == 64 || d == 128) && (dtype == RADAR_F32 || dtype == RADAR_BF16);
}
constexpr int kMaxLen = INT_MAX - (1 << 14);

}  // namespace
}  // namespace radar

using namespace radar;

extern "C" size_t radar_chunk_attn_workspace_bytes(const radar_ctx* ctx, int B, int Hq, int Hkv, int d, int dtype, int max_new, int max_cache_len) {
    if (!ctx || !sizes_ok(B, Hq, Hkv, d, dtype) || max_new < 0 || max_cache_len < 0) return 0;
    // the largest launch's: the pieces of a launch are no more than its CTAs, whatever the requests
    return dtype == RADAR_BF16 ? chunk_tc_workspace_bytes(ctx, d) : chunk_partial_bytes((size_t)fma_most_ctas(ctx), kFmaRows, d);
}

extern "C" int radar_chunk_attention(radar_ctx* ctx, const radar_chunk_attn_args* a, void* stream_) {
    if (!ctx || !a || a->B <= 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv != 0 || a->n_rows < 0 || a->max_new < 0 || a->max_cache_len < 0 || a->max_pages < 0)
        return RADAR_ERR_INVALID_ARG;
    if (!sizes_ok(a->B, a->Hq, a->Hkv, a->d, a->dtype) || a->Hq / a->Hkv > 128 || a->B > 65535 || a->n_rows > INT_MAX || a->cache_rows > INT_MAX || a->max_cache_len > kMaxLen)
        return RADAR_ERR_UNSUPPORTED;
    const bool page_ok = a->page_size == 16 || a->page_size == 32 || a->page_size == 64 || (a->page_size > 0 && a->page_size % 128 == 0);
    if (!page_ok || a->cache_rows <= 0 || (int64_t)a->max_pages * a->page_size < a->max_cache_len) return RADAR_ERR_INVALID_ARG;
    if (a->n_rows == 0 || a->max_new == 0) return RADAR_OK;
    if (!a->Q || !a->q_start || !a->Kc || !a->Vc || (!a->block_table && a->max_cache_len > 0) || !a->cache_len || !a->O || a->q_row_stride < (int64_t)a->Hq * a->d) return RADAR_ERR_INVALID_ARG;
    const uintptr_t tensors = reinterpret_cast<uintptr_t>(a->Q) | reinterpret_cast<uintptr_t>(a->Kc) | reinterpret_cast<uintptr_t>(a->Vc) | reinterpret_cast<uintptr_t>(a->O);
    if ((tensors & 15) != 0 || a->q_row_stride % (a->dtype == RADAR_F32 ? 4 : 8) != 0) return RADAR_ERR_INVALID_ARG;
    if (!a->workspace || (reinterpret_cast<uintptr_t>(a->workspace) & 255) != 0 ||
        a->workspace_bytes < radar_chunk_attn_workspace_bytes(ctx, a->B, a->Hq, a->Hkv, a->d, a->dtype, a->max_new, a->max_cache_len))
        return RADAR_ERR_WORKSPACE;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    bool taken;
    const int status = chunk_rows_launch(ctx, a, stream, taken);
    if (taken || status != RADAR_OK) return status;
    if (a->dtype == RADAR_F32) return a->d == 128 ? fma_launch<128>(ctx, *a, stream) : fma_launch<64>(ctx, *a, stream);
    if (!chunk_tc_supported(a)) return RADAR_ERR_CUDA;
    return chunk_tc_launch(ctx, a, stream);
}
