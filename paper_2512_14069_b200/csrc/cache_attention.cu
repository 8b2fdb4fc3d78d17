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
// Shares.  A unit is (sequence, KV head, row tile); its items are the tree's own rows, which come first, and the prefix in stages of 32
// keys.  The items of all units, with something for what a unit costs beside them, are laid end to end and cut into equal
// ranges, one for each block of four warps, as many blocks as are resident at once: whatever the mix of lengths, all end
// together, and a block's start is paid once.  A block's items of one unit are a segment: its warps take stages in turn and are
// merged in shared memory at its end, while the next segment's copies are under way.  Units that were cut are joined by the
// combine kernel from partial records, two at most a block.  Where there is little to do in all, finding shares and joining them
// is what takes the time: there a cluster of blocks takes a unit, and joins its shares through its shared memories.
// What bounds it, long caches: the warps' own chains of loads, decoding, products and votes.  No unit is full: an instruction is issued
// in 58 % of the cycles, the integer pipe, the busiest (seven of its instructions for eight values), works 63 % of the time; 16 warps an SM do not
// cover one another's waits, and there are no registers for more.  32 sequences of 4096 to 32768 tokens, 32 / 8 heads, one row: 160 us, 4.2 TB/s of the
// cache's 680 MB.  Two stages a warp and four blocks an SM; three stages 175 us, five blocks (96 registers, spilled) 216, three blocks 160;
// shifts by the multiplier were slower too.
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
// Of a unit beside its stages, in stages.  Lengths of 100 to 16384 tokens: 4 sequences, 40 heads, 16 rows 75 us (with 5: 128), 32
// sequences, 32 / 8 heads, 1 row 81 (88); equal lengths do not depend on it.
constexpr int kUnitCost = 16;
// Stages a warp, at most, in the form for little work.  One sequence, 32 / 8 heads, 1 row, 7000 tokens: 12 us (in ranges 18), 9000 tokens
// 14 (22); 8 rows (two row tiles), 12000 tokens 25 (24), 16384 tokens 32 (27).
constexpr int kSmallStages = 12;
// Blocks of a cluster; more than 8 where all clusters have an SM for each block.  One sequence, 32 / 8 heads, 1 row, 16384 tokens: 16 us
// (with 8: 23), 9000 tokens 13 (14), below that the same; 8 rows, two clusters' blocks an SM, 9000 tokens 29 (20).
constexpr int kMaxCluster = 16;
constexpr int blocks_per_sm(int nt) { return nt == 1 ? 4 : 2; }
constexpr float kMove = 8.f;         // log2 units
// Query rows of a KV head up to which this form takes all work; above, only what is little, and cache_attention_tc.cu the rest.  8
// sequences of 4096 to 16384 tokens, 32 / 8 heads of 128: 16 rows 42 us (there 65), 32 rows 68 (65), 48 rows 95 (68), 64 rows 120 (68); of
// 2048 tokens: 32 rows 20 us (32), 48 rows 32 (33), 64 rows 37 (33).  (17 to 32 rows over long caches are up to 18 % faster there, 64 sequences
// of 4096 to 32768 tokens 766 us (627), but the lengths are the GPU's, and the bound that the host has may be far off.)  Little work: 64
// rows over 300 tokens 11 us (20), one sequence of 1000 tokens, 256 rows 14 us (17).
constexpr int kTokenRows = 32;
// The longest bound: keys are counted in int, and pages are looked up as far as 2 x 4096 keys ahead of a position (two windows of 32 pieces
// of at most a tile), rounded up to tiles.
constexpr int kMaxLen = INT32_MAX - (1 << 14);

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
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
// A row that attends to nothing (l = 0) has 0 in O and lse = -inf.  A score that is NaN makes l NaN, and where shares are joined a weight of 0 keeps it so, whatever their maxima
// (which a NaN does not move): the row's O and lse are NaN however its keys were shared out.
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? -CUDART_INF_F : lse_of(m, l); }
// What a warp keeps of its rows.  Thread (g, q) has rows 2q and 2q + 1 of each tile of eight.
template <int D, int NT>
struct State {
    static constexpr int kSteps = D / 16;        // k steps of S, and m tiles of O
    uint32_t q[NT][kSteps][2];
    float o[NT][kSteps][4];                      // channels D/8 g + 2u + {0, 1}, rows 2q, 2q + 1: (c0 r0, c0 r1, c1 r0, c1 r1)
    float m[NT][2], l[NT][2];                    // log2 units; l of this thread's keys
};

// A tile's rows of Q, and nothing summed up.
template <int D, int NT>
__device__ __forceinline__ void begin_rows(const CacheAttnParams& P, State<D, NT>& st, int b, int h, int R, int row0) {
    const radar_cache_attn_args& a = P.a;
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
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
}

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

// Scores to probabilities: moves the reference maximum where it has to.  s are raw scores (-inf: masked).  They are rounded to bf16 for
// the product with values that are bf16 already; their sum is taken in fp32 before that.  It costs as much as O's own rounding (O is off by
// 0.0023 of its size, 0.0017 with fp32 probabilities), and a second bf16 part would double the products of P V.
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

// A stage of 32 cached keys, of which `left` are there.
template <int D, int NT>
__device__ __forceinline__ void cached_stage(const CacheAttnParams& P, State<D, NT>& st, const unsigned char* block, int left) {
    const int g = (threadIdx.x & 31) >> 2;
    float s[2][NT][4];
    uint32_t p[2][NT][2];
    cached_scores<D, NT>(st, s[0], block);
    cached_scores<D, NT>(st, s[1], block + Layout<D>::kBytes);
    if (left < kStageKeys) {                         // (a block that was not fetched holds old bytes: finite numbers)
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
}

// The products of 16 of the tree's own rows, from row t0 on.
template <int D, int NT>
__device__ __forceinline__ void tree_rows(const CacheAttnParams& P, State<D, NT>& st, int b, int h, int M, int R, int row0, int t0) {
    const radar_cache_attn_args& a = P.a;
    const int lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
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

// ---- units, items and ranges ---------------------------------------------------------------------------------------------
struct Unit {
    int b, h, tile;
    int M, len, stages;                  // of the sequence
    long long start;                     // of the unit, in the space of all
    int k0, k1;                          // items of the segment: 0 the tree's rows, 1 .. stages the prefix
};
struct Sequence { int M, len, stages, tiles; };
template <int NT>
__device__ __forceinline__ Sequence sequence(const CacheAttnParams& P, int b) {
    const radar_cache_attn_args& a = P.a;
    Sequence s;
    s.M = a.n_nodes != nullptr ? a.n_nodes[b] : a.rows;
    s.len = a.cache_len[b];
    const bool ok = s.M >= 0 && s.M <= a.rows && s.len >= 0 && s.len <= a.max_cache_len;
    s.tiles = ok ? (s.M * P.G + 8 * NT - 1) / (8 * NT) : 0;
    s.stages = ok ? (s.len + kStageKeys - 1) / kStageKeys : 0;
    return s;
}
__device__ __forceinline__ long long cost(const CacheAttnParams& P, const Sequence& s) { return (long long)P.a.Hkv * s.tiles * (s.stages + kUnitCost); }
// items of a unit that lie before position x
__device__ __forceinline__ int items_before(long long x, long long start, int stages) {
    const long long d = x - start;
    return d <= 0 ? 0 : 1 + (int)max(0ll, min(d - kUnitCost, (long long)stages));
}
// by a whole warp: the size of the space, and the sequence that holds position x with what lies before it
template <int NT>
__device__ __forceinline__ long long space(const CacheAttnParams& P) {
    const int lane = threadIdx.x & 31;
    long long n = 0;
    for (int b = lane; b < P.a.B; b += 32) n += cost(P, sequence<NT>(P, b));
    return warp_sum(n);
}
template <int NT>
__device__ __forceinline__ int find_sequence(const CacheAttnParams& P, long long x, long long& before) {
    const int lane = threadIdx.x & 31;
    before = 0;
    for (int b0 = 0; b0 < P.a.B; b0 += 32) {
        const int b = b0 + lane;
        const long long n = b < P.a.B ? cost(P, sequence<NT>(P, b)) : 0;
        long long incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(kFull, incl, o);
            if (lane >= o) incl += v;
        }
        const unsigned hit = __ballot_sync(kFull, before + incl > x);
        if (hit) {
            const int src = __ffs(hit) - 1;
            before += __shfl_sync(kFull, incl - n, src);
            return b0 + src;
        }
        before += __shfl_sync(kFull, incl, 31);
    }
    return P.a.B;
}
// x / n for x >= 0, n > 0: 32 bits nearly always
__device__ __forceinline__ long long quotient(long long x, long long n) { return (x | n) < (1ll << 31) ? (long long)((unsigned)x / (unsigned)n) : x / n; }
// Block i's range begins at i times this.
__device__ __forceinline__ long long range_size(long long all, int blocks) { return quotient(all + blocks - 1, blocks); }

template <int D, int NT>
struct SmemPlan {
    static constexpr int kStageBytes = kStageKeys / kBlock * Layout<D>::kBytes;
    static constexpr int kStages = 2;
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kHalf = D / 2 + 4;              // channels that are merged at a time; padded: eight lanes of a column write to different banks
    static constexpr int kMerge = kWarps * 8 * NT * kHalf * 4;
    static constexpr int kDynamic = kRing + kMerge;
};

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(NT)) cache_attn_kernel(const CacheAttnParams P) {
    using SP = SmemPlan<D, NT>;
    extern __shared__ __align__(128) unsigned char s_dyn[];
    __shared__ uint64_t s_full[kWarps][SP::kStages];
    __shared__ float2 s_ml[kWarps][8 * NT];
    const radar_cache_attn_args& a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    unsigned char* ring = s_dyn + warp * SP::kStages * SP::kStageBytes;
    float* s_o = reinterpret_cast<float*>(s_dyn + SP::kRing);               // [warp][row][kHalf]
    if (lane == 0)
        for (int i = 0; i < SP::kStages; ++i) mbar_init(&s_full[warp][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    chain_wait();

    if (blockIdx.x == 0 && warp == 0)
        for (int b = lane; b < a.B; b += 32) {
            const int M = a.n_nodes != nullptr ? a.n_nodes[b] : a.rows, len = a.cache_len[b];
            if (M < 0 || M > a.rows || len < 0 || len > a.max_cache_len) set_status(P.status, RADAR_ERR_INVALID_ARG);
        }
    // ---- the block's range and its first segment; every warp for itself ----
    const long long all = space<NT>(P), range = range_size(all, gridDim.x), lo = min(range * blockIdx.x, all), hi = min(lo + range, all);
    auto next_unit = [&](Unit& u) {                  // k1 == k0: there is none in the range
        u.start += u.stages + kUnitCost;
        if (++u.tile == (u.M * P.G + 8 * NT - 1) / (8 * NT)) {
            u.tile = 0;
            if (++u.h == a.Hkv) {
                u.h = 0;
                Sequence s;
                do {
                    if (++u.b >= a.B) { u.k0 = u.k1 = 0; return; }
                    s = sequence<NT>(P, u.b);
                } while (s.tiles == 0);
                u.M = s.M; u.len = s.len; u.stages = s.stages;
            }
        }
        u.k0 = 0;
        u.k1 = items_before(hi, u.start, u.stages);
    };
    auto next_segment = [&](Unit& u) {
        if (u.k1 < u.stages + 1) u.k0 = u.k1 = 0;    // the range ended inside the unit
        else next_unit(u);
    };
    Unit cur;
    cur.k0 = cur.k1 = 0;
    if (hi > lo) {
        long long before;
        cur.b = find_sequence<NT>(P, lo, before);
        const Sequence s = sequence<NT>(P, cur.b);
        cur.M = s.M; cur.len = s.len; cur.stages = s.stages;
        const int index = (int)quotient(lo - before, s.stages + kUnitCost);
        cur.h = index / s.tiles;
        cur.tile = index - cur.h * s.tiles;
        cur.start = before + (long long)index * (s.stages + kUnitCost);
        cur.k0 = items_before(lo, cur.start, cur.stages);
        cur.k1 = items_before(hi, cur.start, cur.stages);
        if (cur.k0 == cur.stages + 1) next_unit(cur);
        else if (cur.k0 == cur.k1) cur.k0 = cur.k1 = 0;
    }

    // ---- copies: the warp's stages of this segment and the next ones, as far as the ring reaches.  Pages are looked up 32 stages at a
    // time, by a lane each, ahead of need ----
    Unit far = cur;                                      // the segment that is being fetched
    int far_i = 0, far_n = 0;                            // next stage of the warp in it, and how many there are
    int window[2], ahead[2];                             // blocks of the pool that the stages' two blocks are
    auto own_stages = [&](const Unit& u) { const int n = u.k1 - max(u.k0, 1); return n > warp ? (n - warp + kWarps - 1) / kWarps : 0; };
    auto own_stage = [&](const Unit& u, int i) { return max(u.k0, 1) - 1 + warp + kWarps * i; };
    auto look_up = [&](int i, int (&out)[2]) {
        const int blk = own_stage(far, i + lane) * 2;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            out[c] = 0;
            if (i + lane < far_n && (blk + c) * kBlock < far.len) {
                const int index = P.page_shift_blocks >= 0 ? (blk + c) >> P.page_shift_blocks : (blk + c) / P.blocks_per_page;
                int page = a.block_table[(int64_t)far.b * a.max_pages + index];
                if (page < 0 || page >= a.n_pages) { set_status(P.status, RADAR_ERR_INVALID_ARG); page = 0; }
                out[c] = (page * a.Hkv + far.h) * P.blocks_per_page + blk + c - index * P.blocks_per_page;
            }
        }
    };
    auto begin_far = [&]() {
        far_i = 0;
        far_n = own_stages(far);
        look_up(0, window);
        look_up(32, ahead);
    };
    int fetched = 0, used = 0;                           // stages of this warp
    bool ok = true;
    auto fetch = [&]() {
        if (!ok) return;
        while (far_i == far_n) {
            if (far.k1 == far.k0) return;
            next_segment(far);
            if (far.k1 == far.k0) return;
            begin_far();
        }
        if ((far_i & 31) == 0 && far_i > 0) {
            window[0] = ahead[0]; window[1] = ahead[1];
            look_up(far_i + 32, ahead);
        }
        const int at0 = __shfl_sync(kFull, window[0], far_i & 31), at1 = __shfl_sync(kFull, window[1], far_i & 31);
        const int key = own_stage(far, far_i) * kStageKeys, slot = fetched % SP::kStages;
        const bool two = far.len - key > kBlock, together = P.blocks_per_page > 1;
        ++far_i;
        ++fetched;
        if (lane == 0) {
            uint64_t* bar = &s_full[warp][slot];
            unsigned char* to = ring + slot * SP::kStageBytes;
            const unsigned char* pages = reinterpret_cast<const unsigned char*>(a.pages);
            mbar_arrive_expect_tx(bar, (two ? 2 : 1) * Layout<D>::kBytes);
            bulk_load(to, pages + (int64_t)at0 * Layout<D>::kBytes, (two && together ? 2 : 1) * Layout<D>::kBytes, bar);
            if (two && !together) bulk_load(to + Layout<D>::kBytes, pages + (int64_t)at1 * Layout<D>::kBytes, Layout<D>::kBytes, bar);
        }
    };
    if (cur.k1 > cur.k0) begin_far();
    for (int i = 0; i < SP::kStages - 1; ++i) fetch();

    // ---- segments ----
#pragma unroll 1
    for (; cur.k1 > cur.k0; next_segment(cur)) {
        const int b = cur.b, h = cur.h, M = cur.M, R = M * P.G, row0 = cur.tile * 8 * NT;
        State<D, NT> st;
        begin_rows<D, NT>(P, st, b, h, R, row0);

        // ---- the cached keys ----
        const int mine = own_stages(cur);
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
            fetch();
            const int slot = used % SP::kStages;
            ok = mbar_wait_while(ok, &s_full[warp][slot], (used / SP::kStages) & 1);
            ok = __all_sync(kFull, ok);
            if (!ok) break;
            ++used;
            const unsigned char* block = ring + slot * SP::kStageBytes;
            const int left = cur.len - own_stage(cur, i) * kStageKeys;
            cached_stage<D, NT>(P, st, block, left);
            __syncwarp();                                    // the slot may be filled again
        }

        // ---- the tree's own rows: 16 a warp ----
        if (cur.k0 == 0 && warp * 16 < M) tree_rows<D, NT>(P, st, b, h, M, R, row0, warp * 16);

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
        __syncthreads();
        float f[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = n * 8 + 2 * q + e;
                float m = s_ml[0][r].x;
#pragma unroll
                for (int w = 1; w < kWarps; ++w) m = fmaxf(m, s_ml[w][r].x);
                f[n][e] = st.m[n][e] == -CUDART_INF_F ? 0.f : ex2(st.m[n][e] - m);
            }
        const bool whole = cur.k0 == 0 && cur.k1 == cur.stages + 1;
        // channels D/8 g + 2u + {0, 1}: those with u in the first half of the steps of every lane, then the others
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            constexpr int kU = D / 32, kC = D / 16;          // steps and channels of a lane in a half
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float* to = s_o + (warp * 8 * NT + n * 8 + 2 * q + e) * SP::kHalf + g * kC;
#pragma unroll
                    for (int u = 0; u < kU; u += 2) {
                        const float(&x)[4] = st.o[n][half * kU + u], (&y)[4] = st.o[n][half * kU + u + 1];
                        *reinterpret_cast<float4*>(to + 2 * u) = make_float4(x[e] * f[n][e], x[e + 2] * f[n][e], y[e] * f[n][e], y[e + 2] * f[n][e]);
                    }
                }
            __syncthreads();
            for (int i = tid; i < 8 * NT * (D / 8); i += kThreads) {             // four channels of a row a thread
                const int r = i / (D / 8), c4 = i % (D / 8) * 4, row = row0 + r;
                if (row >= R) continue;
                float m = -CUDART_INF_F, l = 0.f;
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s_ml[w][r].x);
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float2 ml = s_ml[w][r];
                    l = fmaf(ml.y, ml.x == -CUDART_INF_F ? 0.f : ex2(ml.x - m), l);
                    const float4 x = *reinterpret_cast<const float4*>(s_o + (w * 8 * NT + r) * SP::kHalf + c4);
                    o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
                }
                const int c = c4 / kC * (D / 8) + half * kC + c4 % kC;           // the channel
                const int node = row / P.G, hq = h * P.G + row - node * P.G;
                const bool first = half == 0 && c4 == 0;
                if (whole) {
                    const float inv = inverse(l);
                    *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.O) + (((int64_t)b * a.rows + node) * a.Hq + hq) * D + c) =
                        make_uint2(pack(o.x * inv, o.y * inv), pack(o.z * inv, o.w * inv));
                    if (first && a.lse != nullptr) a.lse[((int64_t)b * a.Hq + hq) * a.rows + node] = row_lse(m, l);
                } else {
                    const int64_t rec = ((int64_t)blockIdx.x * 2 + (cur.k0 == 0)) * (8 * NT) + r;
                    *reinterpret_cast<float4*>(P.part_o + rec * D + c) = o;
                    if (first) P.part_ml[rec] = make_float2(m, l);
                }
            }
            __syncthreads();                                 // (the next half, or segment, may be written)
        }
    }
    if (!ok) {                                               // nothing may land behind the block's end
        if (lane == 0) {
            set_status(P.status, RADAR_ERR_TIMEOUT);
            for (; used < fetched; ++used) mbar_drain(&s_full[warp][used % SP::kStages], (used / SP::kStages) & 1);
        }
        __syncwarp();
    }
}

// The form for little work: a cluster of blocks a unit, whose warps take stages in turn.
template <int D, int NT>
struct SmallPlan {
    static constexpr int kRow = D + 4;                   // padded
    static constexpr int kRing = SmemPlan<D, NT>::kRing;
    static constexpr int kOut = 8 * NT * kRow * 4;       // a warp's, or a block's, sums
    static constexpr int kDynamic = kRing + (kWarps + 1) * kOut;
};
template <int D, int NT>
__global__ void __launch_bounds__(kThreads) cache_attn_small_kernel(const CacheAttnParams P) {
    using SP = SmemPlan<D, NT>;
    using PL = SmallPlan<D, NT>;
    extern __shared__ __align__(128) unsigned char s_dyn[];
    __shared__ uint64_t s_full[kWarps][SP::kStages];
    __shared__ float2 s_ml[kWarps + 1][8 * NT];
    const radar_cache_attn_args& a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const int size = P.cluster, rank = (int)(blockIdx.x % size), tiles = (a.rows * P.G + 8 * NT - 1) / (8 * NT);
    unsigned x = blockIdx.x / size;
    const int tile = x % tiles; x /= tiles;
    const int h = x % a.Hkv, b = x / a.Hkv;
    unsigned char* ring = s_dyn + warp * SP::kStages * SP::kStageBytes;
    float* const s_o = reinterpret_cast<float*>(s_dyn + PL::kRing);          // [warp][row][kRow], then the block's
    float* const s_sum = s_o + kWarps * 8 * NT * PL::kRow;
    if (lane == 0)
        for (int i = 0; i < SP::kStages; ++i) mbar_init(&s_full[warp][i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncwarp();
    chain_wait();
    const int M = a.n_nodes != nullptr ? a.n_nodes[b] : a.rows, len = a.cache_len[b], row0 = tile * 8 * NT;
    const bool valid = M >= 0 && M <= a.rows && len >= 0 && len <= a.max_cache_len;
    if (!valid && rank == 0 && tile == 0 && h == 0 && tid == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
    const int R = M * P.G;
    if (!valid || row0 >= R) return;                     // (all of the cluster)

    const int stages = (len + kStageKeys - 1) / kStageKeys, me = rank * kWarps + warp, all = size * kWarps;
    const int mine = stages > me ? (stages - me - 1) / all + 1 : 0;
    int fetched = 0;
    bool ok = true;
    auto fetch = [&]() {
        if (fetched == mine || !ok) return;
        const int key = (me + all * fetched) * kStageKeys, slot = fetched % SP::kStages;
        const int blocks = len - key > kBlock ? 2 : 1;
        if (lane == 0) mbar_arrive_expect_tx(&s_full[warp][slot], blocks * Layout<D>::kBytes);
        __syncwarp();
        const int copies = P.blocks_per_page > 1 ? 1 : blocks;
        if (lane < copies) {
            const int blk = key / kBlock + lane, index = P.page_shift_blocks >= 0 ? blk >> P.page_shift_blocks : blk / P.blocks_per_page;
            int page = a.block_table[(int64_t)b * a.max_pages + index];
            if (page < 0 || page >= a.n_pages) { set_status(P.status, RADAR_ERR_INVALID_ARG); page = 0; }
            const int64_t at = ((int64_t)page * a.Hkv + h) * P.blocks_per_page + blk - index * P.blocks_per_page;
            bulk_load(ring + slot * SP::kStageBytes + lane * Layout<D>::kBytes, reinterpret_cast<const unsigned char*>(a.pages) + at * Layout<D>::kBytes,
                      blocks / copies * Layout<D>::kBytes, &s_full[warp][slot]);
        }
        __syncwarp();
        ++fetched;
    };
    for (int i = 0; i < SP::kStages; ++i) fetch();
    State<D, NT> st;
    begin_rows<D, NT>(P, st, b, h, R, row0);
    // the tree's own rows, 16 a warp, one block after the other
    const int t0 = (rank + size * warp) * 16;
    if (t0 < M) tree_rows<D, NT>(P, st, b, h, M, R, row0, t0);
    int used = 0;
#pragma unroll 1
    for (; used < mine; ++used) {
        const int slot = used % SP::kStages;
        ok = mbar_wait_while(ok, &s_full[warp][slot], (used / SP::kStages) & 1);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        cached_stage<D, NT>(P, st, ring + slot * SP::kStageBytes, len - (me + all * used) * kStageKeys);
        __syncwarp();
        fetch();
    }
    if (!ok && lane == 0) {                              // nothing may land behind the block's end
        set_status(P.status, RADAR_ERR_TIMEOUT);
        for (; used < fetched; ++used) mbar_drain(&s_full[warp][used % SP::kStages], (used / SP::kStages) & 1);
    }

    // ---- the block's four shares, then the cluster's ----
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = n * 8 + 2 * q + e;
            float l = st.l[n][e];
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(kFull, l, o);
            if (g == 0) s_ml[warp][r] = make_float2(st.m[n][e], l);
            float* to = s_o + (warp * 8 * NT + r) * PL::kRow + g * (D / 8);
#pragma unroll
            for (int u = 0; u < D / 16; u += 2)
                *reinterpret_cast<float4*>(to + 2 * u) = make_float4(st.o[n][u][e], st.o[n][u][e + 2], st.o[n][u + 1][e], st.o[n][u + 1][e + 2]);
        }
    __syncthreads();
    // sums over n shares of four channels of a row, each with its (m, l); the weight of a share is 2^(its m - the largest)
    auto join = [&](const int n, auto get_ml, auto get_o, float& m, float& l, float4& o) {
        m = -CUDART_INF_F;
        l = 0.f;
        o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 0; w < n; ++w) m = fmaxf(m, get_ml(w).x);
#pragma unroll 4
        for (int w = 0; w < n; ++w) {
            const float2 ml = get_ml(w);
            const float4 v = get_o(w);
            const float f = ml.x == -CUDART_INF_F ? 0.f : ex2(ml.x - m);
            l = fmaf(ml.y, f, l);
            o.x = fmaf(v.x, f, o.x); o.y = fmaf(v.y, f, o.y); o.z = fmaf(v.z, f, o.z); o.w = fmaf(v.w, f, o.w);
        }
    };
    auto write = [&](int r, int c, float m, float l, const float4& o) {
        const int row = row0 + r;
        if (row >= R) return;
        const int node = row / P.G, hq = h * P.G + row - node * P.G;
        const float inv = inverse(l);
        *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.O) + (((int64_t)b * a.rows + node) * a.Hq + hq) * D + c) =
            make_uint2(pack(o.x * inv, o.y * inv), pack(o.z * inv, o.w * inv));
        if (c == 0 && a.lse != nullptr) a.lse[((int64_t)b * a.Hq + hq) * a.rows + node] = row_lse(m, l);
    };
    for (int i = tid; i < 8 * NT * (D / 4); i += kThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float m, l;
        float4 o;
        join(kWarps, [&](int w) { return s_ml[w][r]; }, [&](int w) { return *reinterpret_cast<const float4*>(s_o + (w * 8 * NT + r) * PL::kRow + c); }, m, l, o);
        if (size == 1) {
            write(r, c, m, l, o);
        } else {
            *reinterpret_cast<float4*>(s_sum + r * PL::kRow + c) = o;
            if (c == 0) s_ml[kWarps][r] = make_float2(m, l);
        }
    }
    if (size == 1) return;
    cluster_barrier();
    for (int i = rank * kThreads + tid; i < 8 * NT * (D / 4); i += size * kThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float m, l;
        float4 o;
        join(size,
             [&](int w) {
                 float2 v;
                 asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(cluster_addr(&s_ml[kWarps][r], w)));
                 return v;
             },
             [&](int w) {
                 float4 v;
                 asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_addr(s_sum + r * PL::kRow + c, w)));
                 return v;
             },
             m, l, o);
        write(r, c, m, l, o);
    }
    cluster_barrier();                                   // (nobody leaves while its sums are read)
}

// A warp joins the pieces of a row whose unit was cut.
template <int D, int NT>
__global__ void __launch_bounds__(128) cache_combine_kernel(const CacheAttnParams P) {
    chain_wait();
    const radar_cache_attn_args& a = P.a;
    const int lane = threadIdx.x & 31;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);       // (sequence, node, query head)
    if (item >= (int64_t)a.B * a.rows * a.Hq) return;
    const int hq = (int)(item % a.Hq), node = (int)(item / a.Hq % a.rows), b = (int)(item / a.Hq / a.rows);
    const Sequence s = sequence<NT>(P, b);
    if (node >= s.M || s.tiles == 0) return;
    long long all = 0, before = 0;
    for (int i = lane; i < a.B; i += 32) {
        const long long n = cost(P, sequence<NT>(P, i));
        all += n;
        if (i < b) before += n;
    }
    all = warp_sum(all);
    before = warp_sum(before);
    const int h = hq / P.G, row = node * P.G + hq - h * P.G, tile = row / (8 * NT), r = row - tile * 8 * NT;
    const long long start = before + ((long long)h * s.tiles + tile) * (s.stages + kUnitCost);
    const long long range = range_size(all, P.blocks);
    const int first = (int)quotient(start, range), last = (int)quotient(start + (s.stages > 0 ? kUnitCost + s.stages - 1 : 0), range);
    if (first == last) return;                                               // it was not cut
    constexpr int E = D / 32;
    float m = -CUDART_INF_F, l = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
    for (int j0 = first; j0 <= last; j0 += 32) {                             // a lane looks after a piece
        const int j = j0 + lane;
        float2 ml = make_float2(-CUDART_INF_F, 0.f);
        if (j <= last && (j == first || items_before(range * j, start, s.stages) < items_before(range * (j + 1), start, s.stages)))
            ml = P.part_ml[((int64_t)j * 2 + (j == first)) * (8 * NT) + r];
        const float m2 = fmaxf(m, warp_max(ml.x));
        const float old = m == -CUDART_INF_F ? 0.f : ex2(m - m2), w = ml.x == -CUDART_INF_F ? 0.f : ex2(ml.x - m2);
        m = m2;
        l = l * old + warp_sum(ml.y * w);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= old;
        const int n = min(32, last - j0 + 1);
        for (int k0 = 0; k0 < n; k0 += 8) {                                  // eight pieces in flight (one that is not there has weight 0)
            float v[8][E], wk[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                wk[k] = __shfl_sync(kFull, w, k0 + k);
                const float* from = P.part_o + (((int64_t)(j0 + k0 + k) * 2 + (j0 + k0 + k == first)) * (8 * NT) + r) * D + lane * E;
#pragma unroll
                for (int e = 0; e < E; ++e) v[k][e] = 0.f;
                if (wk[k] != 0.f) {
                    if (E == 4) {
                        const float4 t = *reinterpret_cast<const float4*>(from);
                        v[k][0] = t.x; v[k][1] = t.y; v[k][E - 2] = t.z; v[k][E - 1] = t.w;
                    } else {
                        const float2 t = *reinterpret_cast<const float2*>(from);
                        v[k][0] = t.x; v[k][1] = t.y;
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = fmaf(v[k][e], wk[k], o[e]);
        }
    }
    const float inv = inverse(l);
    uint32_t* to = reinterpret_cast<uint32_t*>(reinterpret_cast<__nv_bfloat16*>(a.O) + item * D + lane * E);
#pragma unroll
    for (int e = 0; e < E / 2; ++e) to[e] = pack(o[2 * e] * inv, o[2 * e + 1] * inv);
    if (lane == 0 && a.lse != nullptr) a.lse[((int64_t)b * a.Hq + hq) * a.rows + node] = row_lse(m, l);
}

// Row tiles of eight in a warp, and blocks: as many as are resident, each with a stage for every warp at least.
struct Plan { int nt, blocks, cluster; };              // cluster > 0: the form for little work
Plan plan(const radar_ctx* ctx, int B, int Hkv, int G, int rows, int max_len) {
    Plan p;
    const int R = rows * G;
    p.nt = R > 8 ? 2 : 1;
    const int64_t units = (int64_t)B * Hkv * ((R + 8 * p.nt - 1) / (8 * p.nt)), stages = units * ((max_len + kStageKeys - 1) / kStageKeys + 1);
    p.blocks = (int)std::max<int64_t>(1, std::min<int64_t>(ctx->sm_count * blocks_per_sm(p.nt), (stages + kWarps - 1) / kWarps));
    // A cluster a unit, as large as gives every warp about two stages, where that leaves no more than kSmallStages a warp and the
    // blocks fit the SMs together.
    const int unit_stages = (max_len + kStageKeys - 1) / kStageKeys;
    int size = 1;
    while (size < kMaxCluster && unit_stages > 2 * kWarps * size && 2 * size * units <= (int64_t)ctx->sm_count * (size < 8 ? 2 : 1)) size *= 2;
    p.cluster = unit_stages <= kSmallStages * kWarps * size && size * units <= (int64_t)ctx->sm_count * 3 ? size : 0;
    return p;
}
int64_t records(const radar_ctx* ctx, int nt) { return (int64_t)ctx->sm_count * blocks_per_sm(nt) * 2 * 8 * nt; }
size_t partial_bytes(int64_t records, int d) { return align_up(records * sizeof(float2), 256) + align_up(records * d * sizeof(float), 256); }

template <int D, int NT>
int launch(radar_ctx* ctx, const CacheAttnParams& P, cudaStream_t stream) {
    using SP = SmemPlan<D, NT>;
    const radar_cache_attn_args& a = P.a;
    if (P.cluster > 0) {
        auto* const kernel = cache_attn_small_kernel<D, NT>;
        constexpr size_t smem = SmallPlan<D, NT>::kDynamic;
        constexpr int slot = RADAR_SMEM_CACHE_SMALL + 2 * (D == 128) + NT - 1;
        if (ctx->smem_room[slot] == 0) RADAR_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
        RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, slot, kernel, smem));
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)((int64_t)a.B * a.Hkv * ((a.rows * P.G + 8 * NT - 1) / (8 * NT)) * P.cluster));
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)P.cluster;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        radar_launch_scope scope(ctx, RADAR_K_CACHE_ATTN, stream);
        RADAR_CUDA_CHECK(cudaLaunchKernelEx(&cfg, kernel, P));
        return RADAR_OK;
    }
    RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, RADAR_SMEM_CACHE_ATTN + 2 * (D == 128) + NT - 1, cache_attn_kernel<D, NT>, (size_t)SP::kDynamic));
    {
        radar_launch_scope scope(ctx, RADAR_K_CACHE_ATTN, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_attn_kernel<D, NT>, dim3((unsigned)P.blocks), dim3(kThreads), (size_t)SP::kDynamic, stream, P));
    }
    if (P.blocks > 1) {
        const int64_t items = (int64_t)a.B * a.rows * a.Hq;
        radar_launch_scope scope(ctx, RADAR_K_CACHE_COMBINE, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_combine_kernel<D, NT>, dim3((unsigned)((items + 3) / 4)), dim3(128), 0, stream, P));
    }
    RADAR_CUDA_CHECK(cudaGetLastError());
    return RADAR_OK;
}

}  // namespace
}  // namespace radar

using namespace radar;

extern "C" size_t radar_cache_attn_workspace_bytes(const radar_ctx* ctx, int B, int Hq, int Hkv, int d, int rows, int max_cache_len) {
    if (!ctx || B <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || (d != 64 && d != 128) || rows <= 0 || rows > kMaxNodes || max_cache_len < 0) return 0;
    return std::max(partial_bytes(records(ctx, 2), d), cache_attn_tc_workspace_bytes(ctx, d));       // of every size
}

extern "C" int radar_cache_attention(radar_ctx* ctx, const radar_cache_attn_args* a, void* stream_) {
    if (!ctx || !a || a->B <= 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv != 0 || a->rows <= 0 || a->rows > kMaxNodes || a->max_cache_len < 0 ||
        a->n_pages < 0)
        return RADAR_ERR_INVALID_ARG;
    if ((a->d != 64 && a->d != 128) || a->dtype != RADAR_BF16 || a->Hq / a->Hkv > 128) return RADAR_ERR_UNSUPPORTED;
    if (!page_size_ok(a->page_size) || a->max_pages <= 0 || (int64_t)a->max_pages * a->page_size < a->max_cache_len || a->max_cache_len > kMaxLen) return RADAR_ERR_INVALID_ARG;
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
    const Plan p = plan(ctx, a->B, a->Hkv, P.G, a->rows, a->max_cache_len);
    if (a->rows * P.G > kTokenRows && p.cluster == 0) return cache_attn_tc_launch(ctx, a, stream);
    P.blocks = p.blocks;
    P.cluster = p.cluster;
    P.blocks_per_page = a->page_size / kBlock;
    P.page_shift_blocks = -1;
    for (int s = 0; s < 28; ++s)
        if (P.blocks_per_page == 1 << s) P.page_shift_blocks = s;
    P.scale_log2 = (a->scale > 0.f ? a->scale : 1.f / sqrtf((float)a->d)) * 1.4426950408889634f;
    P.status = ctx->d_status;
    const int64_t n = records(ctx, p.nt);
    if (partial_bytes(n, a->d) > a->workspace_bytes) return RADAR_ERR_WORKSPACE;
    P.part_ml = reinterpret_cast<float2*>(a->workspace);
    P.part_o = reinterpret_cast<float*>(reinterpret_cast<char*>(a->workspace) + align_up(n * sizeof(float2), 256));
    if (a->d == 128) return p.nt == 2 ? launch<128, 2>(ctx, P, stream) : launch<128, 1>(ctx, P, stream);
    return p.nt == 2 ? launch<64, 2>(ctx, P, stream) : launch<64, 1>(ctx, P, stream);
}
