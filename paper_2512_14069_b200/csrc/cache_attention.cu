// Attention over the 4-bit paged cache for few query rows (a single token of a few heads, a small tree): bound by the cache's
// bytes and by what it takes to make numbers of them.
//
// The G query heads of a KV head, for all tree rows, are R = n_nodes * G query rows (row r = node * G + head in group), in tiles of
// 8 NT.  A warp works on its own: it takes blocks of 16 keys as they lie in the cache from a ring of bulk copies, decodes them
// in registers and multiplies them there; no two warps meet before the end.
//   S^T = K Q^T    keys are the rows of the product (m = 16), query rows its columns (n = 8), so that eight rows cost half of what
//                  sixteen do: a thread (g = lane / 4, q = lane % 4) decodes D / 4 consecutive channels of keys g and 8 + g, which
//                  are the k slots of its A fragments in an order that Q's fragments share.
//   P^T            exp2 of the scores in the accumulators' layout; a transpose of 8 x 8 tiles makes it the B fragment of
//   O^T = V^T P^T  channels are the rows: a thread decodes D / 8 consecutive channels of keys 2q, 2q + 1, 8 + 2q, 9 + 2q.  The words
//                  of two keys are interleaved by halves before they are decoded, so that a decoded pair is two keys of a
//                  channel, what a fragment holds.
// The running maximum is a reference that is moved when some score exceeds it by 2^8: in between there is nothing but a vote.
// Sums are per thread until the end.
// A unit (sequence, KV head, row tile) is cut into splits of keys, a block of four warps each; the four are merged in shared
// memory, the splits by the combine kernel.  Split 0 takes the tree's own rows, 16 a warp.
#include <algorithm>
#include <cmath>

#include "cache.cuh"
#include "cache_attention.cuh"
#include "tc05.cuh"

namespace radar {
namespace {

using namespace cache4;
using tc05::mbar_init;
using tc05::mbar_arrive_expect_tx;
using tc05::mbar_wait_while;
using tc05::mbar_drain;

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kStageKeys = 32;       // keys of a stage: two blocks
constexpr float kMove = 8.f;         // log2 units
constexpr int kTensorRows = 48;      // query rows of a KV head from which on the form of cache_attention_tc.cu takes them

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
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

// What a warp keeps of its rows.  Thread (g, q) has rows 2q and 2q + 1 of each tile of eight.
template <int D, int NT>
struct State {
    static constexpr int kSteps = D / 16;        // k steps of S, and m tiles of O
    uint32_t q[NT][kSteps][2];
    float o[NT][kSteps][4];                      // channels D/8 g + 2u + {0, 1}, rows 2q, 2q + 1: (c0 r0, c0 r1, c1 r0, c1 r1)
    float m[NT][2], l[NT][2];                    // log2 units; l of this thread's keys
};

// S^T of 16 keys from A fragments given by k step
template <int D, int NT, typename F>
__device__ __forceinline__ void scores(const State<D, NT>& st, float (&s)[NT][4], F fragment) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
        uint32_t a[4];
        fragment(j, a);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma(s[n], a[0], a[1], a[2], a[3], st.q[n][j][0], st.q[n][j][1]);
    }
}

// S^T of a cached block
template <int D, int NT>
__device__ __forceinline__ void cached_scores(const State<D, NT>& st, float (&s)[NT][4], const unsigned char* block) {
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    uint32_t w0[D / 32], w1[D / 32], sc;                     // words of keys g and 8 + g
    if (D == 128) {
        const uint4 x = *reinterpret_cast<const uint4*>(block + g * 64 + q * 16), y = *reinterpret_cast<const uint4*>(block + (g + 8) * 64 + q * 16);
        w0[0] = x.x; w0[1] = x.y; w0[D / 32 - 2] = x.z; w0[D / 32 - 1] = x.w;
        w1[0] = y.x; w1[1] = y.y; w1[D / 32 - 2] = y.z; w1[D / 32 - 1] = y.w;
        sc = *reinterpret_cast<const uint32_t*>(block + Layout<D>::kKScales + g * 16 + q * 4);
    } else {
        const uint2 x = *reinterpret_cast<const uint2*>(block + g * 32 + q * 8), y = *reinterpret_cast<const uint2*>(block + (g + 8) * 32 + q * 8);
        w0[0] = x.x; w0[1] = x.y;
        w1[0] = y.x; w1[1] = y.y;
        sc = *reinterpret_cast<const uint16_t*>(block + Layout<D>::kKScales + g * 8 + q * 2);
    }
    uint32_t s0[D / 64], s1[D / 64], f0[D / 64], f1[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        s0[i] = scale_pair(__byte_perm(sc, 0, i == 0 ? 0x4040 : 0x4141));
        s1[i] = scale_pair(__byte_perm(sc, 0, D == 128 ? (i == 0 ? 0x4242 : 0x4343) : 0x4141));
        f0[i] = offset_pair(s0[i]);
        f1[i] = offset_pair(s1[i]);
    }
    scores<D, NT>(st, s, [&](const int j, uint32_t (&a)[4]) {
        const int w = j >> 1, i = j >> 2;                    // 16 channels of a word pair are a group: 4 k steps
        if ((j & 1) == 0) {
            a[0] = decode<0>(w0[w], s0[i], f0[i]); a[1] = decode<0>(w1[w], s1[i], f1[i]);
            a[2] = decode<1>(w0[w], s0[i], f0[i]); a[3] = decode<1>(w1[w], s1[i], f1[i]);
        } else {
            a[0] = decode<2>(w0[w], s0[i], f0[i]); a[1] = decode<2>(w1[w], s1[i], f1[i]);
            a[2] = decode<3>(w0[w], s0[i], f0[i]); a[3] = decode<3>(w1[w], s1[i], f1[i]);
        }
    });
}

// O^T += V^T P^T of a cached block
template <int D, int NT>
__device__ __forceinline__ void cached_values(State<D, NT>& st, const uint32_t (&p)[NT][2], const unsigned char* block) {
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    constexpr int W = D / 64;                                // words of a key
    uint32_t v[4][W];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const unsigned char* at = block + Layout<D>::kVCodes + (q + 4 * k) * Layout<D>::kRow;
        if (D == 128) {
            const uint2 x = *reinterpret_cast<const uint2*>(at + ((g * 8) ^ ((q >> 1) * 32)));
            v[k][0] = x.x; v[k][W - 1] = x.y;
        } else {
            v[k][0] = *reinterpret_cast<const uint32_t*>(at + g * 4);
        }
    }
    const uint32_t sc = *reinterpret_cast<const uint32_t*>(block + Layout<D>::kVScales + (D == 128 ? g : g >> 1) * 16 + q * 4);
    const uint32_t s01 = scale_pair(__byte_perm(sc, 0, 0x4140)), s23 = scale_pair(__byte_perm(sc, 0, 0x4342));
    const uint32_t f01 = offset_pair(s01), f23 = offset_pair(s23);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const uint32_t a_lo = __byte_perm(v[0][w], v[1][w], 0x5410), a_hi = __byte_perm(v[0][w], v[1][w], 0x7632);
        const uint32_t b_lo = __byte_perm(v[2][w], v[3][w], 0x5410), b_hi = __byte_perm(v[2][w], v[3][w], 0x7632);
        auto step = [&](auto ic) {
            constexpr int I = decltype(ic)::value;
            const uint32_t a0 = decode<I>(a_lo, s01, f01), a1 = decode<I>(a_hi, s01, f01), a2 = decode<I>(b_lo, s23, f23), a3 = decode<I>(b_hi, s23, f23);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma(st.o[n][4 * w + I], a0, a1, a2, a3, p[n][0], p[n][1]);
        };
        step(std::integral_constant<int, 0>{}); step(std::integral_constant<int, 1>{}); step(std::integral_constant<int, 2>{}); step(std::integral_constant<int, 3>{});
    }
}

// Scores to probabilities: moves the reference maximum where it has to.  s are raw scores (-inf: masked).
template <int D, int NT, int NB>
__device__ __forceinline__ void probabilities(State<D, NT>& st, float (&s)[NB][NT][4], uint32_t (&p)[NB][NT][2], float scale_log2) {
    bool move = false;
    float top[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float t = s[0][n][e];
#pragma unroll
            for (int b = 0; b < NB; ++b) t = fmaxf(fmaxf(t, s[b][n][e]), s[b][n][e + 2]);
            top[n][e] = t * scale_log2;
            move |= top[n][e] > st.m[n][e] + kMove;
        }
    if (__any_sync(kFull, move)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float t = top[n][e];
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) t = fmaxf(t, __shfl_xor_sync(kFull, t, o));
                const float m = fmaxf(st.m[n][e], t), f = m == -CUDART_INF_F ? 1.f : ex2(st.m[n][e] - m);
                st.m[n][e] = m;
                st.l[n][e] *= f;
#pragma unroll
                for (int u = 0; u < D / 16; ++u) { st.o[n][u][e] *= f; st.o[n][u][e + 2] *= f; }
            }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float m0 = st.m[n][0] == -CUDART_INF_F ? 0.f : st.m[n][0], m1 = st.m[n][1] == -CUDART_INF_F ? 0.f : st.m[n][1];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const float p0 = ex2(fmaf(s[b][n][0], scale_log2, -m0)), p1 = ex2(fmaf(s[b][n][1], scale_log2, -m1));
            const float p2 = ex2(fmaf(s[b][n][2], scale_log2, -m0)), p3 = ex2(fmaf(s[b][n][3], scale_log2, -m1));
            st.l[n][0] += p0 + p2;
            st.l[n][1] += p1 + p3;
            p[b][n][0] = transposed(pack(p0, p1));
            p[b][n][1] = transposed(pack(p2, p3));
        }
    }
}

template <int D, int NT>
struct SmemPlan {
    static constexpr int kStageBytes = kStageKeys / kBlock * Layout<D>::kBytes;
    static constexpr int kStages = 4;
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kMergeO = kWarps * 8 * NT * (D + 4) * 4;     // rows padded: eight lanes of a column write to different banks
    static constexpr int kDynamic = kRing > kMergeO ? kRing : kMergeO;
};

template <int D, int NT>
__global__ void __launch_bounds__(kThreads) cache_attn_kernel(const CacheAttnParams P) {
    using SP = SmemPlan<D, NT>;
    chain_wait();
    extern __shared__ __align__(128) unsigned char s_dyn[];
    __shared__ uint64_t s_full[kWarps][SP::kStages];
    __shared__ float2 s_ml[kWarps][8 * NT];
    const radar_cache_attn_args& a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    // block -> row tile (fastest, so that the tiles of a unit share its keys in L2), split, KV head, sequence
    unsigned x = blockIdx.x;
    const int tile = x % P.n_tiles; x /= P.n_tiles;
    const int h = x % a.Hkv; x /= a.Hkv;
    const int split = x % P.n_splits, b = x / P.n_splits;
    const int M = a.n_nodes != nullptr ? a.n_nodes[b] : a.rows, len = a.cache_len[b];
    if (M < 0 || M > a.rows || len < 0 || len > a.max_cache_len) {
        if (tile == 0 && h == 0 && split == 0 && tid == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
        return;
    }
    const int R = M * P.G, row0 = tile * 8 * NT;
    if (row0 >= R || (split > 0 && split * P.split_len >= len)) return;

    // ---- the ring: every warp its own ----
    unsigned char* ring = s_dyn + warp * SP::kStages * SP::kStageBytes;
    if (lane == 0)
        for (int i = 0; i < SP::kStages; ++i) mbar_init(&s_full[warp][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    const int k0 = split * P.split_len, k1 = min(len, k0 + P.split_len);
    // stages of this warp: every fourth of the split
    const int n_stages = max(k1 - k0 + kStageKeys - 1, 0) / kStageKeys;
    const int mine = n_stages > warp ? (n_stages - warp - 1) / kWarps + 1 : 0;
    const int64_t page_bytes = P.page_bytes;
    const int32_t* table = a.block_table + (int64_t)b * a.max_pages;
    auto fetch = [&](int i) {                                // lane 0: the warp's i-th stage
        const int key = k0 + (i * kWarps + warp) * kStageKeys, slot = i % SP::kStages;
        const int blocks = min(2, (k1 - key + kBlock - 1) / kBlock);
        uint64_t* bar = &s_full[warp][slot];
        unsigned char* to = ring + slot * SP::kStageBytes;
        mbar_arrive_expect_tx(bar, blocks * Layout<D>::kBytes);
        const int per = P.blocks_per_page >= 2 ? blocks : 1;          // blocks of a copy
        for (int c = 0; c < blocks; c += per) {
            const int blk = (key >> 4) + c, index = P.page_shift_blocks >= 0 ? blk >> P.page_shift_blocks : blk / P.blocks_per_page;
            int page = table[index];
            if (page < 0 || page >= a.n_pages) { set_status(P.status, RADAR_ERR_INVALID_ARG); page = 0; }
            const int in = blk - index * P.blocks_per_page;
            bulk_load(to + c * Layout<D>::kBytes,
                      reinterpret_cast<const unsigned char*>(a.pages) + page * page_bytes + ((int64_t)h * P.blocks_per_page + in) * Layout<D>::kBytes,
                      per * Layout<D>::kBytes, bar);
        }
    };
    if (lane == 0)
        for (int i = 0; i < min(mine, SP::kStages - 1); ++i) fetch(i);

    // ---- Q ----
    State<D, NT> st;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = row0 + n * 8 + g, node = r / P.G, hq = h * P.G + r - node * P.G;
        const bool on = r < R;
        const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(a.Q) + ((int64_t)b * a.rows + (on ? node : 0)) * a.q_row_stride + (on ? hq : 0) * D + q * (D / 4);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const uint4 t = on ? *reinterpret_cast<const uint4*>(src + 8 * i) : make_uint4(0, 0, 0, 0);
            st.q[n][2 * i][0] = t.x; st.q[n][2 * i][1] = t.y; st.q[n][2 * i + 1][0] = t.z; st.q[n][2 * i + 1][1] = t.w;
        }
#pragma unroll
        for (int u = 0; u < D / 16; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) st.o[n][u][e] = 0.f;
        st.m[n][0] = st.m[n][1] = -CUDART_INF_F;
        st.l[n][0] = st.l[n][1] = 0.f;
    }

    // ---- the cached keys ----
    bool ok = true;
    int i = 0;
#pragma unroll 1
    for (; i < mine; ++i) {
        if (lane == 0 && i + SP::kStages - 1 < mine) fetch(i + SP::kStages - 1);
        const int slot = i % SP::kStages;
        ok = mbar_wait_while(ok, &s_full[warp][slot], (i / SP::kStages) & 1);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        const unsigned char* block = ring + slot * SP::kStageBytes;
        const int key = k0 + (i * kWarps + warp) * kStageKeys, left = k1 - key;
        float s[2][NT][4];
        uint32_t p[2][NT][2];
        cached_scores<D, NT>(st, s[0], block);
        cached_scores<D, NT>(st, s[1], block + Layout<D>::kBytes);
        if (left < kStageKeys) {                             // (a block that was not fetched holds old bytes: finite numbers)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (c * 16 + g + (e >> 1) * 8 >= left) s[c][n][e] = -CUDART_INF_F;
        }
        probabilities<D, NT, 2>(st, s, p, P.scale_log2);
        cached_values<D, NT>(st, p[0], block);
        cached_values<D, NT>(st, p[1], block + Layout<D>::kBytes);
        __syncwarp();                                        // the slot may be filled again
    }
    if (!ok && lane == 0) {                                  // nothing may land behind the block's end
        set_status(P.status, RADAR_ERR_TIMEOUT);
        for (const int end = min(mine, i + SP::kStages); i < end; ++i) mbar_drain(&s_full[warp][i % SP::kStages], (i / SP::kStages) & 1);
    }

    // ---- the tree's own rows: 16 a warp ----
    if (split == 0 && warp * 16 < M) {
        const int t0 = warp * 16;
        const __nv_bfloat16* kt = reinterpret_cast<const __nv_bfloat16*>(a.Kt) + (int64_t)b * a.rows * a.kv_row_stride + h * D;
        const __nv_bfloat16* vt = reinterpret_cast<const __nv_bfloat16*>(a.Vt) + (int64_t)b * a.rows * a.kv_row_stride + h * D;
        float s[1][NT][4];
        uint32_t p[1][NT][2], k[2][D / 8];
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const int t = t0 + g + 8 * r;
                const uint4 v = t < M ? *reinterpret_cast<const uint4*>(kt + t * a.kv_row_stride + q * (D / 4) + 8 * i) : make_uint4(0, 0, 0, 0);
                k[r][4 * i] = v.x; k[r][4 * i + 1] = v.y; k[r][4 * i + 2] = v.z; k[r][4 * i + 3] = v.w;
            }
        scores<D, NT>(st, s[0], [&](const int j, uint32_t (&f)[4]) { f[0] = k[0][2 * j]; f[1] = k[1][2 * j]; f[2] = k[0][2 * j + 1]; f[3] = k[1][2 * j + 1]; });
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = row0 + n * 8 + 2 * q + e, node = r / P.G;
                uint64_t see = 0;
                if (r < R) {
                    see = a.mask != nullptr ? a.mask[(int64_t)b * a.rows + node] : ~0ull >> (63 - node);
                    if (M < 64) see &= (1ull << M) - 1;
                }
                see >>= t0;
                if (!(see >> g & 1)) s[0][n][e] = -CUDART_INF_F;
                if (!(see >> (g + 8) & 1)) s[0][n][e + 2] = -CUDART_INF_F;
            }
        probabilities<D, NT, 1>(st, s, p, P.scale_log2);
        uint32_t v[4][D / 16];                               // keys 2q, 2q + 1, 8 + 2q, 9 + 2q: D / 8 channels
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const int t = t0 + 2 * q + (kk & 1) + 8 * (kk >> 1);
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                const uint4 y = t < M ? *reinterpret_cast<const uint4*>(vt + t * a.kv_row_stride + g * (D / 8) + 8 * i) : make_uint4(0, 0, 0, 0);
                v[kk][4 * i] = y.x; v[kk][4 * i + 1] = y.y; v[kk][4 * i + 2] = y.z; v[kk][4 * i + 3] = y.w;
            }
        }
#pragma unroll
        for (int u = 0; u < D / 16; ++u) {
            const uint32_t a0 = __byte_perm(v[0][u], v[1][u], 0x5410), a1 = __byte_perm(v[0][u], v[1][u], 0x7632);
            const uint32_t a2 = __byte_perm(v[2][u], v[3][u], 0x5410), a3 = __byte_perm(v[2][u], v[3][u], 0x7632);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma(st.o[n][u], a0, a1, a2, a3, p[0][n][0], p[0][n][1]);
        }
    }

    // ---- the four warps' shares of a row together ----
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float l = st.l[n][e];
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(kFull, l, o);
            if (g == 0) s_ml[warp][n * 8 + 2 * q + e] = make_float2(st.m[n][e], l);
        }
    __syncthreads();                                         // (the rings are read no more)
    float* s_o = reinterpret_cast<float*>(s_dyn);            // [warp][row][D + 4]
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = n * 8 + 2 * q + e;
            float m = s_ml[0][r].x;
#pragma unroll
            for (int w = 1; w < kWarps; ++w) m = fmaxf(m, s_ml[w][r].x);
            const float f = st.m[n][e] == -CUDART_INF_F ? 0.f : ex2(st.m[n][e] - m);
            float* to = s_o + (warp * 8 * NT + r) * (D + 4) + g * (D / 8);
#pragma unroll
            for (int u = 0; u < D / 16; u += 2)
                *reinterpret_cast<float4*>(to + 2 * u) = make_float4(st.o[n][u][e] * f, st.o[n][u][e + 2] * f, st.o[n][u + 1][e] * f, st.o[n][u + 1][e + 2] * f);
        }
    __syncthreads();
    for (int i = tid; i < 8 * NT * (D / 8); i += kThreads) {                 // eight channels of a row a thread
        const int r = i / (D / 8), c = i % (D / 8) * 8, row = row0 + r;
        if (row >= R) continue;
        float m = -CUDART_INF_F, l = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s_ml[w][r].x);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 ml = s_ml[w][r];
            l += ml.x == -CUDART_INF_F ? 0.f : ml.y * ex2(ml.x - m);
            const float4* from = reinterpret_cast<const float4*>(s_o + (w * 8 * NT + r) * (D + 4) + c);
            const float4 x = from[0], y = from[1];
            o[0] += x.x; o[1] += x.y; o[2] += x.z; o[3] += x.w; o[4] += y.x; o[5] += y.y; o[6] += y.z; o[7] += y.w;
        }
        const int node = row / P.G, hq = h * P.G + row - node * P.G;
        if (P.n_splits == 1) {
            write_row(a, b, node, hq, c, D, o, m, l, c == 0);
        } else {
            const int64_t rec = (((int64_t)b * a.rows + node) * a.Hq + hq) * P.n_splits + split;
            float4* to = reinterpret_cast<float4*>(P.part_o + rec * D + c);
            to[0] = make_float4(o[0], o[1], o[2], o[3]);
            to[1] = make_float4(o[4], o[5], o[6], o[7]);
            if (c == 0) P.part_ml[rec] = make_float2(m, l);
        }
    }
}

// A warp joins the splits of a row.
template <int D>
__global__ void __launch_bounds__(128) cache_combine_kernel(const CacheAttnParams P) {
    chain_wait();
    const radar_cache_attn_args& a = P.a;
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);       // (sequence, node, query head)
    if (item >= (int64_t)a.B * a.rows * a.Hq) return;
    const int hq = (int)(item % a.Hq), node = (int)(item / a.Hq % a.rows), b = (int)(item / a.Hq / a.rows);
    const int M = a.n_nodes != nullptr ? a.n_nodes[b] : a.rows, len = a.cache_len[b];
    if (node >= M || M > a.rows || len < 0 || len > a.max_cache_len) return;
    const int n = max(1, (len + P.split_len - 1) / P.split_len);
    constexpr int E = D / 32;
    const float2* ml = P.part_ml + item * P.n_splits;
    const float* po = P.part_o + item * P.n_splits * D + lane * E;
    float m = -CUDART_INF_F, l = 0.f;
    for (int s = lane; s < n; s += 32) m = fmaxf(m, ml[s].x);
    m = warp_max(m);
    for (int s = lane; s < n; s += 32) l += ml[s].x == -CUDART_INF_F ? 0.f : ml[s].y * ex2(ml[s].x - m);
    l = warp_sum(l);
    float o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll 4
    for (int s = 0; s < n; ++s) {
        const float w = ml[s].x == -CUDART_INF_F ? 0.f : ex2(ml[s].x - m);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(po[(int64_t)s * D + e], w, o[e]);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    uint32_t out[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) out[e] = pack(o[2 * e] * inv, o[2 * e + 1] * inv);
    uint32_t* to = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(a.O) + item * D + lane * E);
#pragma unroll
    for (int e = 0; e < E / 2; ++e) to[e] = out[e];
    if (lane == 0 && a.lse != nullptr) a.lse[((int64_t)b * a.Hq + hq) * a.rows + node] = l > 0.f ? lse_of(m, l) : -CUDART_INF_F;
}

// Splits of a unit: as many as fill the SMs several times over, a block of four warps and at least one stage a warp each.
struct Plan { int nt, n_tiles, n_splits, split_len; };
Plan plan(const radar_ctx* ctx, int B, int Hkv, int G, int rows, int max_len) {
    Plan p;
    const int R = rows * G;
    p.nt = R > 8 ? 2 : 1;
    p.n_tiles = (R + 8 * p.nt - 1) / (8 * p.nt);
    constexpr int kUnit = kWarps * kStageKeys;
    const int64_t units = (int64_t)B * Hkv * p.n_tiles;
    const int want = (int)std::max<int64_t>(1, (int64_t)ctx->sm_count * 12 / units), most = std::max(1, (max_len + kUnit - 1) / kUnit);
    const int n = std::min(want, most);
    p.split_len = std::max(1, ((max_len + n - 1) / n + kUnit - 1) / kUnit) * kUnit;
    p.n_splits = std::max(1, (max_len + p.split_len - 1) / p.split_len);
    return p;
}
size_t partial_bytes(int64_t records, int d) { return align_up(records * sizeof(float2), 256) + align_up(records * d * sizeof(float), 256); }

template <int D, int NT>
int launch(radar_ctx* ctx, const CacheAttnParams& P, cudaStream_t stream) {
    using SP = SmemPlan<D, NT>;
    const radar_cache_attn_args& a = P.a;
    const int64_t blocks = (int64_t)a.B * P.n_splits * a.Hkv * P.n_tiles;
    if (blocks > INT32_MAX) return RADAR_ERR_UNSUPPORTED;
    RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, RADAR_SMEM_CACHE_ATTN + 4 * (D == 128) + NT - 1, cache_attn_kernel<D, NT>, (size_t)SP::kDynamic));
    {
        radar_launch_scope scope(ctx, RADAR_K_CACHE_ATTN, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_attn_kernel<D, NT>, dim3((unsigned)blocks), dim3(kThreads), (size_t)SP::kDynamic, stream, P));
    }
    if (P.n_splits > 1) {
        const int64_t items = (int64_t)a.B * a.rows * a.Hq;
        radar_launch_scope scope(ctx, RADAR_K_CACHE_COMBINE, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_combine_kernel<D>, dim3((unsigned)((items + 3) / 4)), dim3(128), 0, stream, P));
    }
    RADAR_CUDA_CHECK(cudaGetLastError());
    return RADAR_OK;
}

}  // namespace
}  // namespace radar

using namespace radar;

extern "C" size_t radar_cache_attn_workspace_bytes(const radar_ctx* ctx, int B, int Hq, int Hkv, int d, int rows, int max_cache_len) {
    if (!ctx || B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || (d != 64 && d != 128) || rows <= 0 || rows > kMaxNodes || max_cache_len < 0) return 0;
    // B * n_splits is at most B * ceil(max / unit) and, where it is more than B, 12 SMs / (Hkv * tiles); fewer sequences or a
    // shorter prefix do not raise either
    const Plan p = plan(ctx, B, Hkv, Hq / Hkv, rows, max_cache_len);
    const int64_t most = std::max<int64_t>(1, (max_cache_len + kWarps * kStageKeys - 1) / (kWarps * kStageKeys));
    const int64_t cut = std::max<int64_t>(B, (int64_t)ctx->sm_count * 12 / ((int64_t)Hkv * p.n_tiles));
    return std::max(partial_bytes(std::min(B * most, cut) * rows * Hq, d), cache_attn_tc_workspace_bytes(ctx, d));
}

extern "C" int radar_cache_attention(radar_ctx* ctx, const radar_cache_attn_args* a, void* stream_) {
    if (!ctx || !a || a->B <= 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv != 0 || a->rows <= 0 || a->rows > kMaxNodes || a->max_cache_len < 0 ||
        a->n_pages < 0)
        return RADAR_ERR_INVALID_ARG;
    if ((a->d != 64 && a->d != 128) || a->dtype != RADAR_BF16 || a->Hq / a->Hkv > 128) return RADAR_ERR_UNSUPPORTED;
    if (!page_size_ok(a->page_size) || a->max_pages <= 0 || (int64_t)a->max_pages * a->page_size < a->max_cache_len) return RADAR_ERR_INVALID_ARG;
    if (!a->Q || !a->Kt || !a->Vt || !a->O || !a->cache_len || !a->block_table || !a->workspace || (a->max_cache_len > 0 && (!a->pages || a->n_pages == 0)))
        return RADAR_ERR_INVALID_ARG;
    if (a->q_row_stride < (int64_t)a->Hq * a->d || a->kv_row_stride < (int64_t)a->Hkv * a->d || a->q_row_stride % 8 != 0 || a->kv_row_stride % 8 != 0)
        return RADAR_ERR_INVALID_ARG;
    const uintptr_t al = reinterpret_cast<uintptr_t>(a->Q) | reinterpret_cast<uintptr_t>(a->Kt) | reinterpret_cast<uintptr_t>(a->Vt) |
                         reinterpret_cast<uintptr_t>(a->O) | reinterpret_cast<uintptr_t>(a->pages);
    if ((al & 15) != 0) return RADAR_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(a->workspace) & 255) != 0) return RADAR_ERR_WORKSPACE;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    CacheAttnParams P;
    P.a = *a;
    P.G = a->Hq / a->Hkv;
    if (a->rows * P.G >= kTensorRows) return cache_attn_tc_launch(ctx, a, stream);
    const Plan p = plan(ctx, a->B, a->Hkv, P.G, a->rows, a->max_cache_len);
    P.n_tiles = p.n_tiles;
    P.n_splits = p.n_splits;
    P.split_len = p.split_len;
    P.blocks_per_page = a->page_size / kBlock;
    P.page_shift_blocks = -1;
    for (int s = 0; s < 28; ++s)
        if (P.blocks_per_page == 1 << s) P.page_shift_blocks = s;
    P.page_bytes = page_bytes(a->Hkv, a->d, a->page_size);
    P.scale_log2 = (a->scale > 0.f ? a->scale : 1.f / sqrtf((float)a->d)) * 1.4426950408889634f;
    P.status = ctx->d_status;
    const int64_t records = (int64_t)a->B * a->rows * a->Hq * p.n_splits;
    if (p.n_splits > 1 && partial_bytes(records, a->d) > a->workspace_bytes) return RADAR_ERR_WORKSPACE;
    P.part_ml = reinterpret_cast<float2*>(a->workspace);
    P.part_o = reinterpret_cast<float*>(reinterpret_cast<char*>(a->workspace) + align_up(records * sizeof(float2), 256));
    if (a->d == 128) return p.nt == 2 ? launch<128, 2>(ctx, P, stream) : launch<128, 1>(ctx, P, stream);
    return p.nt == 2 ? launch<64, 2>(ctx, P, stream) : launch<64, 1>(ctx, P, stream);
}
