// Attention over the 4-bit paged cache for many query rows (whole draft trees), on the tensor cores.
//
// The tile space, the softmax groups, the issuing warp and the epilogue are those of tree_attention_tc.cu: units of (sequence, KV head,
// pair of row blocks of 128 query rows), their tiles of 128 keys laid end to end and cut into equal ranges, one thread a query
// row.  What differs is where a tile comes from: the producer fetches a tile's keys, then its values, as they lie in the cache (by TMA:
// a block's keys, or its values, are a row of bytes), and eight warps decode them into the bf16 tiles that the products read,
// exactly (cache.cuh).
//   warps 0-3 / 4-7  softmax groups 0 / 1
//   warps 8-11       decoders of values, two blocks of a tile each; the tree's V by TMA; epilogue
//   warps 12-15      decoders of keys, the same; the tree's K by TMA
//   warp 16          producer: segments, stages, Q
//   warp 17          issues the products
// What bounds the kernel with two row blocks a tile is the warp that issues the products: 32 MMAs, which the tensor pipe takes at 64 to 70
// cycles each, and waits and commits between them in which it runs dry (4500 cycles a tile); and the softmax behind it, half as
// long.  8 sequences of 8192 tokens, 64 / 8 heads, 64 rows: 158 us; the same over bf16 rows takes 152.  With one row block a tile takes
// about 3000 cycles (8 sequences of 16384 tokens, 32 / 8 heads, 32 rows: 94 us, where the cache's bytes take 23), with 64 live rows
// as with 128, and its 16 MMAs some 1070 of them: neither products nor softmax.  What is left is the decoding (twelve instructions for eight
// values, a decoder's two blocks one after the other); its part has not been measured by itself.  A thread takes its row's scores 64
// at a time, against the maximum so far, and waits for each load at once, which makes room for eight decoders at 96 registers;
// keys and values are decoded by the same small loop.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cache_attention.cuh"
#include "tree_tiles.cuh"

namespace radar {
namespace {

using namespace cache4;

constexpr int kTcThreads = 576;      // 18 warps are allocated as 20: 96 registers a thread
constexpr int kEpilogueWarp = 8, kKeyWarp = 12, kProducerWarp = 16, kMmaWarp = 17, kDecoders = 4;    // decoders of either kind
// What a tile of one and of two row blocks and a unit beside its tiles cost here (decoding takes as long for one row block as for two).
// us, with these and with 5, 9, 24: 32 sequences of 16384 tokens, 32 / 8 heads, 64 and 32 rows in turn 444 (479), ragged trees of 9 to 64
// rows, 4096 to 32768 tokens 513 (560).
constexpr TileCosts kCosts = {5, 8, 24};
constexpr int kStaticSmem = 3072;
constexpr int kTileBlocks = kTileKeys / kBlock;
static_assert(kTileBlocks == 2 * kDecoders, "two blocks of a tile a decoder");

template <int D, bool TWO>
struct Smem {
    static constexpr int kHalves = D / 64;
    static constexpr int kQBlock = 128 * D * 2;
    static constexpr int kQBytes = (TWO ? 2 : 1) * kQBlock;
    static constexpr int kTileBytes = kTileKeys * D * 2;
    static constexpr int kPartBytes = Layout<D>::kBytes / 2;             // a block's keys, or its values
    // A copy's target is on a 128-byte boundary: where every part is a copy of its own (pages of one block) they lie this far apart.
    static constexpr int kSinglePitch = (kPartBytes + 127) / 128 * 128;
    static_assert(2 * kPartBytes % 128 == 0, "two parts end on a boundary");
    static constexpr int kStageBytes = kTileBlocks * kSinglePitch;      // a tile's keys, or its values
    static constexpr int kRingK = 2, kRingV = 2;
    static constexpr int kRoom = (227 * 1024 - kStaticSmem - kQBytes - (kRingK + kRingV) * kTileBytes) / kStageBytes;
    static constexpr int kStages = kRoom < 8 ? kRoom : 8;
    static_assert(kStages >= 3, "keys and values of a tile, and a stage to go on with");
    static constexpr int kDynamic = kQBytes + (kRingK + kRingV) * kTileBytes + kStages * kStageBytes;
};

// Place in a ring and the phase to wait for.
template <int N>
struct Ring {
    uint32_t slot = 0, par;
    __device__ __forceinline__ explicit Ring(uint32_t p) : par(p) {}
    __device__ __forceinline__ void next() { if (++slot == N) { slot = 0; par ^= 1; } }
    __device__ __forceinline__ void next_but_one() { slot += 2; if (slot >= N) { slot -= N; par ^= 1; } }
};

// A decoder's lane takes 32 channels of a row of a block's keys or values (at D = 128 of rows `row` and row + 8), which it stores as
// four chunks of the 128-byte swizzle.  The lanes are dealt out over rows and channels so that the eight lanes of a phase of a
// 16-byte store write to eight different chunks.
struct Share {
    int codes, scale0, scale1;       // offsets in the block's part: codes, the words with the scales of the two groups
    int pick0, pick1;                // selectors of their bytes (two further on for the second row)
    uint32_t to[4];                  // offsets of the chunks in the tile, from the row of the block's first key
};
template <int D>
__device__ __forceinline__ Share share_of(const bool values) {
    const int lane = threadIdx.x & 31, q = D == 128 ? (lane & 1) | (lane >> 4) << 1 : lane & 1;      // channels 32q ..
    // keys lie row by row; a value's place p is where its row stands
    const int p = values ? ((lane >> 1) & 1) | ((lane >> 2) & 1) << 2 | ((lane >> 3) & 1) << 1 | (D == 64 ? (lane >> 4) << 3 : 0) : (D == 128 ? (lane >> 1) & 7 : lane >> 1);
    const int row = values ? (p & 3) << 1 | ((p >> 2) & 1) | (p & 8) : p;
    Share s;
    s.codes = p * Layout<D>::kRow + ((q * 16) ^ (values && D == 128 && (p & 2) ? 32 : 0));
    s.scale0 = Layout<D>::kKScales + (values ? q * 32 + (p & 3) * 4 : (row & 7) * (D / 8) + q * 4);
    s.scale1 = s.scale0 + (values ? 16 : 0);
    s.pick0 = 0x4040 + 0x101 * (values ? p >> 2 : row >> 3);
    s.pick1 = 0x4040 + 0x101 * (values ? p >> 2 : D == 128 ? 1 : 2 + (row >> 3));
    for (int c = 0; c < 4; ++c) s.to[c] = (q >> 1) * (kTileKeys * 128) + row * 128 + ((((q & 1) * 4 + c) ^ (row & 7)) << 4);
    return s;
}
// A block's keys or values into the tile whose row of the block's first key is at `tile_at_key0`.
template <int D>
__device__ __forceinline__ void decode_part(const unsigned char* part, uint32_t tile_at_key0, const Share& sh) {
    constexpr int kRows = D / 64;
    uint4 w[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) w[i] = *reinterpret_cast<const uint4*>(part + sh.codes + 8 * i * Layout<D>::kRow);
    uint32_t sc0 = *reinterpret_cast<const uint32_t*>(part + sh.scale0), sc1 = *reinterpret_cast<const uint32_t*>(part + sh.scale1);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t s0 = scale_pair(__byte_perm(sc0, 0, sh.pick0)), s1 = scale_pair(__byte_perm(sc1, 0, sh.pick1)), f0 = offset_pair(s0), f1 = offset_pair(s1);
        auto put = [&](const uint32_t at, uint32_t x, uint32_t s, uint32_t f) {
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + i * 8 * 128), "r"(decode<0>(x, s, f)), "r"(decode<1>(x, s, f)), "r"(decode<2>(x, s, f)),
                         "r"(decode<3>(x, s, f)) : "memory");
        };
        put(tile_at_key0 + sh.to[0], w[i].x, s0, f0);
        put(tile_at_key0 + sh.to[1], w[i].y, s0, f0);
        put(tile_at_key0 + sh.to[2], w[i].z, s1, f1);
        put(tile_at_key0 + sh.to[3], w[i].w, s1, f1);
        sc0 >>= 16;
        sc1 >>= 16;
    }
}

// TWO: the launch may contain units with two live row blocks; decides the shared-memory layout
template <int D, bool TWO>
__global__ void __launch_bounds__(kTcThreads, 1)
cache_attn_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmKt,
                     const __grid_constant__ CUtensorMap tmVt, const __grid_constant__ CUtensorMap tmCache, const TcParams P) {
    chain_trigger();                     // every warp waits for the predecessor where its role begins; the barrier,
                                         // tensor-memory and descriptor set-up needs nothing from global memory
    using SM = Smem<D, TWO>;
    constexpr int H = SM::kHalves;
    constexpr int RK = SM::kRingK, RV = SM::kRingV, RS = SM::kStages;
    const radar_attn_args& a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int pp = blockIdx.x % P.n_cls;                    // class
    const int ci = blockIdx.x / P.n_cls;
    const int G = P.G;

    // Static block first (padded to a multiple of 1024 bytes and aligned to it), the tiles behind it: the
    // swizzled tiles need a 1024-byte boundary and there is no room left for alignment slack.
    struct __align__(1024) Static {
        uint64_t bar_qfull, bar_qempty, bar_kfull[RK], bar_kempty[RK], bar_vfull[RV], bar_vempty[RV];
        // stages: the cache's bytes as they lie there, keys and values in turn.  Whoever waits for a phase must have seen the one before it
        // complete, or takes the one before that for it: a slot has a barrier for what it holds as keys and one for values.
        uint64_t bar_stfull[2][RS], bar_stempty[RS];
        uint64_t bar_sfull[2], bar_odone[2], bar_ofree[2];
        uint64_t bar_idle;               // every product issued has run
        uint64_t bar_pready[2];          // the tile's probabilities are there
        uint64_t bar_mlfull, bar_mlempty, bar_epilogue;
        uint64_t bar_segfull[kSegRing], bar_segempty[kSegRing];
        Segment seg[kSegRing];
        float2 ml[2][128];               // per group: (m in log2 units, l) of the rows at the end of a segment
        uint32_t q_last, st_armed[2], k_tree, v_tree;   // phase parity of the last Q, parities of the stages' next phases (a bit a slot), the last tree tiles
        uint32_t tmem_base;
        int abort;
    };
    static_assert(sizeof(Static) <= kStaticSmem, "static shared-memory block");
    __shared__ union { Static st; unsigned char bytes[kStaticSmem]; } s_static;
    Static& st = s_static.st;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* sQ = smem_raw;
    unsigned char* sK = sQ + SM::kQBytes;
    unsigned char* sV = sK + RK * SM::kTileBytes;
    unsigned char* sS = sV + RV * SM::kTileBytes;
    const int pitch = P.blocks_per_page == 1 ? SM::kSinglePitch : SM::kPartBytes;

    // ---- set-up ----
    if (warp == 0) {
        if (lane == 0) {
            st.abort = 0;
            mbar_init(&st.bar_qfull, 1);
            mbar_init(&st.bar_qempty, 1);
            for (int i = 0; i < RK; ++i) { mbar_init(&st.bar_kfull[i], kDecoders); mbar_init(&st.bar_kempty[i], 1); }
            for (int i = 0; i < RV; ++i) { mbar_init(&st.bar_vfull[i], kDecoders); mbar_init(&st.bar_vempty[i], 1); }
            for (int i = 0; i < RS; ++i) { mbar_init(&st.bar_stfull[0][i], 1); mbar_init(&st.bar_stfull[1][i], 1); mbar_init(&st.bar_stempty[i], kDecoders); }
            for (int i = 0; i < 2; ++i) {
                mbar_init(&st.bar_sfull[i], 1); mbar_init(&st.bar_pready[i], 4);
                mbar_init(&st.bar_odone[i], 1); mbar_init(&st.bar_ofree[i], 4);
            }
            for (int i = 0; i < kSegRing; ++i) { mbar_init(&st.bar_segfull[i], 1); mbar_init(&st.bar_segempty[i], kProducerWarp + 1); }
            mbar_init(&st.bar_idle, 1);
            st.q_last = 1;
            st.st_armed[0] = st.st_armed[1] = st.k_tree = st.v_tree = 0;
            mbar_init(&st.bar_mlfull, 8);
            mbar_init(&st.bar_mlempty, 4);
            mbar_init(&st.bar_epilogue, 4);
            fence_barrier_init();
        }
    } else if (warp == kMmaWarp) {
        tmem_alloc(&st.tmem_base, 512);
        tmem_relinquish();
        if (lane == 0) {
            tma_prefetch_desc(&tmQ); tma_prefetch_desc(&tmCache); tma_prefetch_desc(&tmKt); tma_prefetch_desc(&tmVt);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    // All of tensor memory is this CTA's, so its addresses are constants (the producer checks): S/P buffers in columns 0 and
    // 128, O accumulators in 256 and 384.  An address that the compiler does not know to be the same in every lane costs the
    // issuing warp a handful of instructions for every product.
    constexpr uint32_t tmem = 0;
    bool ok = true;                         // no wait of this thread has run out
    // Each role starts with chain_sync(): the bounds of the waits behind it are for this kernel's own work.  (A warp that went
    // straight to its first wait would spend them on whatever is left of the predecessor.)
    // the producer's next segment; false behind the last one
    auto take_segment = [&](uint32_t seg, Segment& s) {
        ok = mbar_wait_while(ok, &st.bar_segfull[seg % kSegRing], (seg / kSegRing) & 1);
        ok = __all_sync(kFull, ok);
        s = st.seg[seg % kSegRing];
        __syncwarp();
        if (lane == 0) mbar_arrive(&st.bar_segempty[seg % kSegRing]);
        return ok && s.n > 0;
    };

    // The tree's own keys or values, by one lane of the decoders: `last` keeps slot and phase of what is in flight.
    auto tree_tile = [&](unsigned char* to, const CUtensorMap* tm, uint64_t* full, const Segment& s, const bool issues, uint32_t& last, const uint32_t where) {
        ok = __all_sync(kFull, ok);
        if (lane != 0 || !ok) return;
        if (issues) {
            mbar_arrive_expect_tx(full, kTreeKeys * D * 2);
            for (int h = 0; h < H; ++h) tma_load_4d(to + h * (kTreeKeys * 128), tm, full, h * 64, s.g, s.b * P.nodes, 0);
            last = 1u << 16 | where;
        } else {
            mbar_arrive(full);
        }
    };

    if (warp < kEpilogueWarp) {
        chain_sync();
        // =================================== softmax groups ===================================
        // One thread per query row.
        const int grp = warp >> 2;
        const int row = (warp & 3) * 32 + lane;                 // row of the block == tensor-memory lane
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + grp * 128 + lane_addr;
        const uint32_t tO = tmem + 256 + grp * 128 + lane_addr;
        const int rb_node = (int)(((uint32_t)row * P.g_magic) >> 16);        // row / G
        uint32_t sc = 0;                         // S tiles this group has waited for
        Segment s;
        for (uint32_t seg = 0; take_segment(seg, s); ++seg) {
            const bool two = TWO && s.rows > P.rb_rows;
            const int blk = two ? grp : 0;                       // row block within the unit
            const int node = (pp * P.n_blk + blk) * P.nodes_per_rb + rb_node;
            const int rows_here = min(s.rows - blk * P.rb_rows, P.rb_rows);  // live rows of this row block
            // A warp none of whose 32 rows is live does no arithmetic (the products of its rows are never read):
            // it only keeps the barriers going.
            const bool warp_live = row - lane < rows_here;
            // the row's ancestor word is needed by the tree tile only (the unit's last): it is loaded here and first
            // touched there, so that the segment does not start with a wait for global memory
            uint32_t mask_lo, mask_hi;
            if (a.mask != nullptr) {
                asm volatile("ld.global.v2.u32 {%0, %1}, [%2];" : "=r"(mask_lo), "=r"(mask_hi) : "l"(a.mask + (int64_t)s.b * P.nodes + min(node, P.nodes - 1)));
            } else {                             // a chain
                mask_lo = node >= 31 ? 0xffffffffu : (2u << node) - 1u;
                mask_hi = node < 32 ? 0u : node >= 63 ? 0xffffffffu : (2u << (node - 32)) - 1u;
            }
            const int n_my = two ? s.n : (s.n - grp + 1) >> 1;
            float m_run = -CUDART_INF_F, l_run = 0.f;

#pragma unroll 1
            for (int j = 0; j < n_my; ++j) {
                const int t = s.t0 + (two ? j : 2 * j + grp);
                ok = mbar_wait_while(ok, &st.bar_sfull[grp], sc & 1);
                ok = __all_sync(kFull, ok);                      // warp-uniform: guards .aligned ops
                ++sc;
                tc_fence_after_sync();
                const int keys = t == s.nt - 1 ? s.M : min(kTileKeys, s.Pb - t * kTileKeys);
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    const int valid = keys - half * kFirstKeys;
                    if (ok && warp_live && valid > 0) {
                        const uint32_t tH = tS + half * kFirstKeys;
                        uint32_t va[32], vb[32];
                        if (t == s.nt - 1 || valid < kFirstKeys) {
                            // Keys that the row may not attend to, and columns that are stale, become -inf in tensor memory.
#pragma unroll 1
                            for (int c = 0; c < 2; ++c) {
                                const int lim = valid - c * 32;
                                uint32_t al = lim >= 32 ? 0xffffffffu : (lim <= 0 ? 0u : ((1u << lim) - 1u));
                                if (t == s.nt - 1) al &= row < rows_here ? (c == 0 ? mask_lo : mask_hi) : 0u;
                                tmem_ld32(tH + c * 32, va);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (!((al >> e) & 1u)) va[e] = 0xff800000u;     // -inf
                                tmem_st32(tH + c * 32, va);
                            }
                            tmem_wait_st();
                        }
                        // ---- P = exp2(s * scale - m) against the maximum so far, and the half's own maximum beside it; once more where a row's
                        // exceeds the reference by 2^8 (nearly never behind the first tile), behind a rescaling of the accumulator ----
                        // Probabilities are rounded to bf16 for the product, and their sum is taken before that: each is off by up to 2^-8 of
                        // itself, like O by its own rounding.  (A second bf16 part would double the P V products, which bound the kernel.)
                        // (the scaling and the row sum work on pairs: one packed fp32x2 instruction per two values.  The warp issues in
                        // order and an exponential takes its unit 8 cycles: what else there is to do stands between two of them.)
                        float2 ls[2];
                        uint32_t pa[16], pb[16];
#pragma unroll 1
                        for (;;) {
                            tmem_ld32(tH, va);
                            tmem_ld32(tH + 32, vb);
                            tmem_wait_ld();
                            const float m_use = m_run == -CUDART_INF_F ? 0.f : m_run;
                            const float2 sc2 = make_float2(P.scale_log2, P.scale_log2), nm2 = make_float2(-m_use, -m_use);
                            float mx0 = -CUDART_INF_F, mx1 = -CUDART_INF_F;
                            ls[0] = ls[1] = make_float2(0.f, 0.f);
                            auto exponentials = [&](uint32_t (&v)[32], uint32_t (&pk)[16]) {
                                auto scale = [&](const int p) {
                                    float& mx = p & 1 ? mx1 : mx0;
                                    mx = max3(mx, __uint_as_float(v[2 * p]), __uint_as_float(v[2 * p + 1]));
                                    const float2 t2 = fma2_in_order(make_float2(__uint_as_float(v[2 * p]), __uint_as_float(v[2 * p + 1])), sc2, nm2);
                                    v[2 * p] = __float_as_uint(t2.x);
                                    v[2 * p + 1] = __float_as_uint(t2.y);
                                };
                                auto finish = [&](const int p) {
                                    const float p0 = __uint_as_float(v[2 * p]), p1 = __uint_as_float(v[2 * p + 1]);
                                    ls[p & 1] = add2_in_order(ls[p & 1], make_float2(p0, p1));
                                    pk[p] = bf16x2_in_order(p0, p1);
                                };
                                // pairs that the scaling is ahead, and that the rest is behind
                                constexpr int kAhead = 2, kLag = 3;
#pragma unroll
                                for (int p = 0; p < kAhead; ++p) scale(p);
#pragma unroll
                                for (int p = 0; p < 16 + kLag; ++p) {
                                    if (p < 16) v[2 * p] = __float_as_uint(ex2_in_order(__uint_as_float(v[2 * p])));
                                    if (p + kAhead < 16) scale(p + kAhead);
                                    if (p < 16) v[2 * p + 1] = __float_as_uint(ex2_in_order(__uint_as_float(v[2 * p + 1])));
                                    if (p >= kLag) finish(p - kLag);
                                }
                            };
                            exponentials(va, pa);
                            exponentials(vb, pb);
                            const float m_half = fmaxf(mx0, mx1) * P.scale_log2;
                            const bool move = m_half > m_run + kRescaleThreshold;       // (m_run may be -inf)
                            if (!__any_sync(kFull, move)) break;
                            // The reference moves by a whole number, so that the factor is a power of two and scales probabilities that
                            // are bf16 already, those of the tile's first half, without another rounding.
                            float factor = 1.f;
                            if (move) {
                                const float by = ceilf(m_half - m_run);                     // infinite: factor 0 clears O and l
                                factor = by < 126.f ? __uint_as_float((uint32_t)(127 - (int)by) << 23) : 0.f;
                                m_run = by < 126.f ? m_run + by : m_half;
                            }
                            l_run *= factor;
                            if (half == 1) {
                                const uint32_t f2 = (__float_as_uint(factor) >> 16) * 0x10001u;
                                uint32_t first[32];
                                tmem_wait_st();
                                tmem_ld32(tS, first);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 32; ++e) asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(first[e]) : "r"(f2));
                                tmem_st32(tS, first);
                            }
                            if (j > 0) {
#pragma unroll 1
                                for (int c = 0; c < D; c += 16) {
                                    uint32_t o[16];
                                    tmem_ld16(tO + c, o);
                                    tmem_wait_ld();
#pragma unroll
                                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
                                    tmem_st16(tO + c, o);
                                }
                            }
                        }
                        tmem_st16(tS + half * 32, pa);
                        tmem_st16(tS + half * 32 + 16, pb);
                        l_run += (ls[0].x + ls[0].y) + (ls[1].x + ls[1].y);
                    }
                }
                tmem_wait_st();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&st.bar_pready[grp]);
                __syncwarp();
            }

            // the rows' (m, l) go to the epilogue, which has taken those of the segment before
            ok = mbar_wait_while(ok, &st.bar_mlempty, (seg & 1) ^ 1);
            st.ml[grp][row] = make_float2(m_run, l_run);
            __syncwarp();
            if (lane == 0) mbar_arrive(&st.bar_mlfull);
        }
    } else if (warp < kProducerWarp) {
        chain_sync();                            // every global access of the CTA comes behind one
        // =================================== decoders, and epilogue ===================================
        // The epilogue of a segment, by the decoders of values, comes behind the first tile of the next one, when its last product is
        // about done: the products have a tile to go on with.
        const int row = (warp - kEpilogueWarp) * 32 + lane;
        const uint32_t tO = tmem + 256 + ((uint32_t)((warp - kEpilogueWarp) * 32) << 16);
        const int rb_node = (int)(((uint32_t)row * P.g_magic) >> 16);        // row / G
        uint32_t oc[2] = {0, 0};             // accumulators waited for
        auto epilogue = [&](const Segment& s, const uint32_t seg) {
            const bool two = TWO && s.rows > P.rb_rows;
            const bool final_rows = s.n == s.nt;                 // the whole unit
            const int slot = seg == 0 ? 0 : 1;                   // a CTA has at most a cut first and a cut last segment
            // No warp gives back an accumulator of this segment while another reads it for the one before: behind a unit of two row blocks there
            // may be a single tile of one, whose second accumulator is given back unread.
            ok = mbar_wait_while(ok, &st.bar_epilogue, (seg & 1) ^ 1);
            ok = mbar_wait_lazy(ok, &st.bar_mlfull, seg & 1);
            const float2 ml0 = st.ml[0][row], ml1 = st.ml[1][row];
            __syncwarp();
            if (lane == 0) mbar_arrive(&st.bar_mlempty);
#pragma unroll 1
            for (int blk = 0; blk < 2; ++blk) {
                // two live row blocks: accumulator blk is row block blk; one: both belong to it, merged in the first trip
                if (blk == 1 && !two) {
                    if (lane == 0) mbar_arrive(&st.bar_ofree[1]);
                    break;
                }
                ok = mbar_wait_while(ok, &st.bar_odone[blk], oc[blk] & 1);
                ++oc[blk];
                const bool merge = !two && s.n > 1;
                if (merge) {
                    ok = mbar_wait_while(ok, &st.bar_odone[1], oc[1] & 1);
                    ++oc[1];
                }
                ok = __all_sync(kFull, ok);
                tc_fence_after_sync();
                const int rows_here = min(s.rows - blk * P.rb_rows, P.rb_rows);  // live rows of this row block
                const bool row_live = row < rows_here;
                if (ok && row - lane < rows_here) {
                    float m_out = blk == 0 ? ml0.x : ml1.x, l_out = blk == 0 ? ml0.y : ml1.y, w0 = 1.f, w1 = 0.f;
                    if (merge) {
                        m_out = fmaxf(ml0.x, ml1.x);
                        const float ms = m_out == -CUDART_INF_F ? 0.f : m_out;
                        w0 = ex2(ml0.x - ms);                        // exp2(-inf) = 0
                        w1 = ex2(ml1.x - ms);
                        l_out = ml0.y * w0 + ml1.y * w1;
                    }
                    const float m_safe = m_out == -CUDART_INF_F ? 0.f : m_out;
                    const float inv = final_rows ? (l_out == 0.f ? 0.f : 1.f / l_out) : 1.f;        // (NaN stays NaN)
                    const int node = (pp * P.n_blk + blk) * P.nodes_per_rb + rb_node;
                    const int hq = s.g * G + row - rb_node * G;
                    const int64_t out_row = ((int64_t)s.b * P.nodes + node) * a.Hq + hq;
                    const int64_t rec = ((int64_t)blockIdx.x * 2 + slot) * kPairRows + blk * 128 + row;
                    __nv_bfloat16* dst_o = reinterpret_cast<__nv_bfloat16*>(a.O) + out_row * D;
                    float* dst_p = P.part_o + rec * D;                  // 128-byte aligned (workspace carve)
                    const bool wide = (reinterpret_cast<uintptr_t>(dst_o) & 31) == 0;
#pragma unroll 1
                    for (int col = 0; col < D; col += 16) {
                        uint32_t o[16], o2[16];
                        tmem_ld16(tO + blk * 128 + col, o);
                        if (merge) tmem_ld16(tO + 128 + col, o2);
                        tmem_wait_ld();
                        float v[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(o[e]) * w0;
                        if (merge) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) v[e] = fmaf(__uint_as_float(o2[e]), w1, v[e]);
                        }
                        if (row_live) {
                            uint32_t w[8];
                            if (final_rows) {
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    const __nv_bfloat162 t2 = __floats2bfloat162_rn(v[2 * e] * inv, v[2 * e + 1] * inv);
                                    w[e] = *reinterpret_cast<const uint32_t*>(&t2);
                                }
                                if (wide) {
                                    st_global_32b(dst_o + col, w);
                                } else {
                                    *reinterpret_cast<uint4*>(dst_o + col) = make_uint4(w[0], w[1], w[2], w[3]);
                                    *reinterpret_cast<uint4*>(dst_o + col + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                                }
                            } else {
#pragma unroll
                                for (int q = 0; q < 2; ++q) {
#pragma unroll
                                    for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(v[q * 8 + e]);
                                    st_global_32b(dst_p + col + q * 8, w);
                                }
                            }
                        }
                    }
                    if (row_live) {
                        const float m_nat = m_safe * 0.6931471805599453f;
                        if (final_rows) {
                            if (a.lse != nullptr) a.lse[((int64_t)s.b * a.Hq + hq) * P.nodes + node] = l_out == 0.f ? -CUDART_INF_F : m_nat + logf(l_out);
                        } else {
                            P.part_ml[rec] = make_float2(m_out == -CUDART_INF_F ? m_out : m_nat, l_out);
                        }
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&st.bar_ofree[blk]);
            }
            if (lane == 0) mbar_arrive(&st.bar_epilogue);
        };
        const bool values = warp < kKeyWarp;
        const int mine = (warp - kEpilogueWarp) & (kDecoders - 1);
        const Share share = share_of<D>(values);
        uint64_t* const tiles_full = values ? st.bar_vfull : st.bar_kfull;
        uint64_t* const tiles_empty = values ? st.bar_vempty : st.bar_kempty;
        unsigned char* const tiles = values ? sV : sK;
        static_assert(RK == RV, "one ring's length for both");
        Ring<RV> out(1);
        Ring<RS> in(0);
        if (values) in.next();
        uint32_t stage_par = 0;              // phase parities of this kind's stages, a bit a slot
        Segment s, done;
        done.n = 0;
        uint32_t seg = 0;
        for (; take_segment(seg, s); ++seg) {
#pragma unroll 1
            for (int i = 0; i < s.n; ++i) {
                const int t = s.t0 + i;
                ok = mbar_wait_while(ok, &tiles_empty[out.slot], out.par);
                unsigned char* to = tiles + out.slot * SM::kTileBytes;
                if (t == s.nt - 1) {
                    tree_tile(to, values ? &tmVt : &tmKt, &tiles_full[out.slot], s, mine == 0, values ? st.v_tree : st.k_tree, out.slot | (out.par ^ 1) << 8);
                } else {
                    const int blocks = min((s.Pb - t * kTileKeys + kBlock - 1) / kBlock, kTileBlocks);
                    ok = mbar_wait_while(ok, &st.bar_stfull[values][in.slot], stage_par >> in.slot & 1);
                    stage_par ^= 1u << in.slot;
                    const uint32_t at = smem_addr(to);
                    const unsigned char* from = sS + in.slot * SM::kStageBytes;
#pragma unroll 1
                    for (int k = mine; k < blocks; k += kDecoders) decode_part<D>(from + k * pitch, at + k * (kBlock * 128), share);
                    fence_proxy_async_smem();
                    ok = __all_sync(kFull, ok);
                    __syncwarp();                            // lane 0 speaks for all lanes' reads and writes, which a vote does not order
                    if (lane == 0) {
                        mbar_arrive(&st.bar_stempty[in.slot]);
                        if (ok) mbar_arrive(&tiles_full[out.slot]);
                    }
                    in.next_but_one();
                }
                out.next();
                if (i == 0 && values && seg > 0) epilogue(done, seg - 1);
            }
            if (values) done = s;
        }
        if (values && seg > 0) epilogue(done, seg - 1);
    } else {
        chain_sync();
        if (warp == kProducerWarp) {
            // =================================== TMA producer ===================================
            // The whole warp walks the tiles: lane c looks up and fetches piece c of a stage (the blocks of one page), the leading lane
            // does the waits, the byte counts and Q.
            const bool lead = lane == 0;
            const bool usable = (smem_u32(smem_raw) & 1023u) == 0 && st.tmem_base == 0;     // (else the tiles would not sit on their swizzle boundary)
            if (!usable && lead) set_status(P.status, RADAR_ERR_CUDA);
            long long tot_all;
            Cursor<kFourBit> cur = first_segment<kFourBit>(P, pp, ci, tot_all);
            if (!usable) cur.t0 = cur.t1 = 0;
            Cut cut;
            cut.unit.valid = 0;
            cut.tot = tot_all;
            Ring<RS> out(1);
            uint32_t armed[2] = {0, 0};
            const int per = min(P.blocks_per_page, kTileBlocks);         // blocks of a piece
            // Where the pieces are: lane l looks up piece l of a window of 32, the window after next at a time (a lookup is a trip to L2,
            // and one on the way of every stage was what bounded the kernel).
            const int tile_pieces = kTileBlocks / per, window_tiles = 32 / tile_pieces;
            auto look_up = [&](int b, int g, int key0, int key_end) {    // of the window that begins with key0
                const int blk = key0 / kBlock + lane * per;
                if (blk * kBlock >= key_end) return 0;
                const int index = P.page_shift_blocks >= 0 ? blk >> P.page_shift_blocks : blk / P.blocks_per_page;
                int page = a.block_table[(long long)b * a.max_pages + index];
                if (page < 0 || page >= P.n_pages) { set_status(P.status, RADAR_ERR_INVALID_ARG); page = 0; }
                return (page * a.Hkv + g) * P.blocks_per_page + blk - index * P.blocks_per_page;
            };
            int next_window = cur.valid() ? look_up(cur.b, cur.g, cur.t0 * kTileKeys, min(cur.t1 * kTileKeys, cur.s.Pb)) : 0;    // the next segment's first
            for (uint32_t seg = 0;; ++seg) {
                const bool on = cur.valid();
                const int b = cur.b, g = cur.g, n = cur.t1 - cur.t0, t0 = cur.t0, nt = cur.s.nt, Pb = cur.s.Pb;
                const bool two = TWO && cur.two_rb(P);
                if (lead) {
                    ok = mbar_wait_while(ok, &st.bar_segempty[seg % kSegRing], ((seg / kSegRing) & 1) ^ 1);
                    Segment s;                       // (behind a wait that ran out the others are sent home)
                    s.n = on && ok ? n : 0; s.t0 = t0; s.nt = nt; s.Pb = Pb; s.M = cur.s.M; s.rows = cur.s.rows; s.b = b; s.g = g; s.layer = 0;
                    st.seg[seg % kSegRing] = s;
                    mbar_arrive(&st.bar_segfull[seg % kSegRing]);
                }
                ok = __shfl_sync(kFull, ok, 0);
                if (!on) break;
                if (t0 == 0 && n < nt) {                             // necessarily the last segment of this CTA
                    cut.unit.valid = 1; cut.unit.b = b; cut.unit.g = g; cut.unit.slot = seg == 0 ? 0 : 1; cut.unit.layer = 0; cut.unit.rows = cur.s.rows;
                    cut.nt = nt; cut.w = cur.s.w; cut.u0 = cur.U;
                }
                cur.next(P, pp);
                const int key_end = min((t0 + n) * kTileKeys, Pb);
                int window = next_window, window2 = look_up(b, g, (t0 + window_tiles) * kTileKeys, key_end);
                if (cur.valid()) next_window = look_up(cur.b, cur.g, cur.t0 * kTileKeys, min(cur.t1 * kTileKeys, cur.s.Pb));
                // The segment's first tile, then Q (its slot is free only behind the last S of the segment before), then the rest.
#pragma unroll 1
                for (int i = 0; i < n && ok; ++i) {
                    const int key = (t0 + i) * kTileKeys, left = t0 + i == nt - 1 ? 0 : min(kTileKeys, Pb - key);
                    if (left > 0) {
                        const int in_window = i & (window_tiles - 1);
                        if (in_window == 0 && i > 0) {
                            window = window2;
                            window2 = look_up(b, g, key + window_tiles * kTileKeys, key_end);
                        }
                        const int at = __shfl_sync(kFull, window, (in_window * tile_pieces + lane) & 31);     // block of the pool
                        const int pieces = per == kTileBlocks ? 1 : (left + per * kBlock - 1) / (per * kBlock);
#pragma unroll 1
                        for (int v = 0; v < 2; ++v) {                    // keys, then values
                            ok = mbar_wait_while(ok, &st.bar_stempty[out.slot], out.par);
                            ok = __all_sync(kFull, ok);
                            if (!ok) break;                              // (the ring's position stays that of the last load)
                            if (lead) mbar_arrive_expect_tx(&st.bar_stfull[v][out.slot], pieces * per * SM::kPartBytes);
                            __syncwarp();
                            if (lane < pieces) tma_load_3d(sS + out.slot * SM::kStageBytes + lane * per * pitch, &tmCache, &st.bar_stfull[v][out.slot], 0, v, at);
                            armed[v] ^= 1u << out.slot;
                            out.next();
                        }
                    }
                    if (i == 0 && lead) {
                        ok = mbar_wait_while(ok, &st.bar_qempty, (seg & 1) ^ 1);
                        const int blocks = two ? 2 : 1, node0 = b * P.nodes + pp * P.n_blk * P.nodes_per_rb;
                        if (ok) {
                            st.q_last = seg & 1;
                            mbar_arrive_expect_tx(&st.bar_qfull, blocks * P.rb_rows * D * 2);   // rows past rb_rows stay stale: never read back
                            for (int q = 0; q < blocks; ++q)
                                for (int h = 0; h < H; ++h)
                                    tma_load_4d(sQ + q * SM::kQBlock + h * (128 * 128), &tmQ, &st.bar_qfull, h * 64, g * G, node0 + q * P.nodes_per_rb, 0);
                        }
                        // ... so the next segment's Q waits for it in L2
                        if (cur.valid()) {
                            const int next0 = cur.b * P.nodes + pp * P.n_blk * P.nodes_per_rb;
                            for (int q = 0; q < (TWO && cur.two_rb(P) ? 2 : 1); ++q)
                                for (int h = 0; h < H; ++h) tma_prefetch_4d(&tmQ, h * 64, cur.g * G, next0 + q * P.nodes_per_rb, 0);
                        }
                    }
                    ok = __shfl_sync(kFull, ok, 0);
                }
            }
            __syncwarp();
            write_cut_unit(P, ci, cut);
            if (lead) { st.st_armed[0] = armed[0]; st.st_armed[1] = armed[1]; }
            __syncwarp();
        } else if (warp == kMmaWarp) {
            // =================================== MMA issuer ===================================
            // The warp runs converged: every lane waits on the barriers and executes the same straight-line issue
            // sequences with warp-uniform descriptor words, and the elected lane issues the instructions and the
            // commits (predicated, no branch around them).  Whatever this warp executes between two MMAs costs
            // tensor-pipe time, so no control flow depends on a wait's outcome: after a wait that ran out the
            // predicate is off and the loops run dry.
            constexpr uint32_t idesc_s128 = idesc_bf16_f32(128, kTileKeys, false, false);
            constexpr uint32_t idesc_s64 = idesc_bf16_f32(128, kTreeKeys, false, false);
            constexpr uint32_t idesc_pv = idesc_bf16_f32(128, D, false, true);
            // high word of every shared-memory descriptor (stride between 8-row groups 1024 B, version, swizzle)
            constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
            const uint32_t q_lo = ((smem_u32(sQ) & 0x3ffff) >> 4) | (1u << 16);
            const uint32_t k_lo = ((smem_u32(sK) & 0x3ffff) >> 4) | (1u << 16);
            const uint32_t v_lo = (smem_u32(sV) & 0x3ffff) >> 4;
            const uint32_t elected = elect_one();
            uint32_t k_next = 0, k_par = 0, v_next = 0, v_par = 0;   // ring slot to take next and its phase parity
            uint32_t p_par[2] = {0, 0};              // phase parity of the next P tile per group
            // The segment's shape comes from memory; passing it through a broadcast from lane 0 tells the
            // compiler that it is the same in every lane, so that the loops below and the descriptor arithmetic in
            // them stay on the uniform datapath (this warp's own instruction stream is what bounds the issue rate).
            auto uni = [](int v) { return __shfl_sync(kFull, v, 0); };
            // a wait that nearly always is over when it begins
            auto wait = [&](uint64_t* bar, const uint32_t parity) {
                if (!__all_sync(kFull, mbar_try_wait(bar, parity))) ok = mbar_wait_while(ok, bar, parity);
            };
            Segment s;
            for (uint32_t seg = 0; take_segment(seg, s); ++seg) {
                const int seg_t0 = uni(s.t0), n = uni(s.n), M = uni(s.M), Pb = uni(s.Pb), last = uni(s.nt) - 1;
                const bool two = TWO && uni(s.rows) > P.rb_rows;
                ok = mbar_wait_while(ok, &st.bar_qfull, seg & 1);
                uint32_t k_slot = 0, v_slot = 0;      // ring slots of the K and V tiles in use
                bool acc[2] = {false, false};         // accumulator holds a product of this segment
                auto take_v = [&]() {
                    v_slot = v_next;
                    wait(&st.bar_vfull[v_slot], v_par);
                    if (++v_next == RV) { v_next = 0; v_par ^= 1; }
                };
                auto take_k = [&]() {
                    k_slot = k_next;
                    wait(&st.bar_kfull[k_slot], k_par);
                    if (++k_next == RK) { k_next = 0; k_par ^= 1; }
                };
                // the accumulator's first product of the segment: the epilogue of the previous one has read it
                auto take_o = [&](const int q) {
                    if (!acc[q]) ok = mbar_wait_while(ok, &st.bar_ofree[q], (seg & 1) ^ 1);
                };

                // ---- O[q] (+)= P[q] V for tile i (q is a literal at every call site) ----
                auto pv = [&](const int q, const int i, const bool fresh_v, const bool release_v) {
                    const bool tree = seg_t0 + i == last;
                    const int nk = tree ? kTreeKeys : kTileKeys;
                    const int valid = tree ? M : min(kTileKeys, Pb - (seg_t0 + i) * kTileKeys);
                    const int ksteps = (valid + 15) >> 4;
                    if (fresh_v) {
                        take_v();
                        if (tree && valid < ksteps * 16) {
                            // rows past the last live key meet P = 0; they must not hold NaN/Inf bit patterns
                            unsigned char* vtile = sV + v_slot * SM::kTileBytes;
                            const int nrows = ksteps * 16 - valid;
#pragma unroll 1
                            for (int e = lane; e < nrows * 8 * H; e += 32) {
                                const int h = e / (nrows * 8), rem = e % (nrows * 8);
                                const int r = valid + rem / 8, c = rem % 8;
                                *reinterpret_cast<uint4*>(vtile + h * (nk * 128) + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
                            }
                            fence_proxy_async_smem();
                            __syncwarp();
                        }
                    }
                    take_o(q);
                    ok = mbar_wait_while(ok, &st.bar_pready[q], p_par[q]);
                    p_par[q] ^= 1;
                    tc_fence_after_sync();
                    const uint32_t go = ok ? elected : 0u;
                    // V is consumed N-major: 16 keys are 2048 B; 64-column blocks are nk * 128 B apart
                    const uint32_t b_lo = (v_lo + v_slot * (SM::kTileBytes >> 4)) | ((uint32_t)(nk * 128 >> 4) << 16);
                    mma_ts_x4(go, ksteps, tmem + 256 + q * 128, tmem + q * 128, b_lo, kDescHi, idesc_pv, acc[q]);
                    mma_ts_x4(go, ksteps - 4, tmem + 256 + q * 128, tmem + q * 128 + 32, b_lo + 4 * 128, kDescHi, idesc_pv, true);
                    acc[q] = true;
                    if (release_v) mma_commit_if(go, &st.bar_vempty[v_slot]);
                    if (two ? i == n - 1 : i + 2 >= n) mma_commit_if(go, &st.bar_odone[q]);
                };
                // ---- S[q] = Q K^T for tile si.  Nothing in tensor memory changes hands here: K arrives through the
                // async proxy, and the buffer was last read by this thread's own P V, which runs first. ----
                auto qk = [&](const int q, const int si, const bool fresh_k, const bool release_k) {
                    if (fresh_k) take_k();
                    const uint32_t go = ok ? elected : 0u;
                    const bool tree = seg_t0 + si == last;
                    const uint32_t a0 = q_lo + (two ? q : 0) * (SM::kQBlock >> 4);
                    const uint32_t b0 = k_lo + k_slot * (SM::kTileBytes >> 4);
                    const uint32_t idesc = tree ? idesc_s64 : idesc_s128;
                    mma_ss_x4(go, tmem + q * 128, a0, b0, kDescHi, idesc, false);
                    if (D == 128)                     // second 64-column block of Q and K
                        mma_ss_x4(go, tmem + q * 128, a0 + (128 * 128 >> 4), b0 + ((uint32_t)((tree ? kTreeKeys : kTileKeys) * 128) >> 4),
                                  kDescHi, idesc, true);
                    if (release_k) mma_commit_if(go, &st.bar_kempty[k_slot]);
                    mma_commit_if(go, &st.bar_sfull[q]);
                    // the last S of the segment: Q may be overwritten once it has run
                    if (si == n - 1 && release_k) mma_commit_if(go, &st.bar_qempty);
                };
                // Schedule.  Two live row blocks: group s owns row block s; per tile PV0(i) S0(i+1) PV1(i) S1(i+1),
                // both groups sharing K(i+1) and V(i).  One live row block: the groups take alternate tiles,
                // PV(i) S(i+2) for group i & 1.  S of the first tile(s) comes from the iterations with i < 0.
                // Steady state (behind the first tiles, and all tiles involved are full prefix tiles): the same steps with nothing to decide,
                // so that the issuing warp executes as few instructions per MMA as possible.  (It is what the groups wait for: 32 MMAs a
                // tile take it 2300 cycles, so everything else counts.)
                auto full = [&](const int q, const uint32_t a0, const bool fresh, const bool release) {
                    static_assert(kTileKeys == 128, "eight steps");
                    const uint32_t o_col = tmem + 256 + q * 128, p_col = tmem + q * 128;
                    if (fresh) {
                        take_v();
                        take_k();
                    }
                    const uint32_t b_lo = (v_lo + v_slot * (SM::kTileBytes >> 4)) | ((uint32_t)(kTileKeys * 128 >> 4) << 16);
                    const uint32_t b0 = k_lo + k_slot * (SM::kTileBytes >> 4);
                    wait(&st.bar_pready[q], p_par[q]);
                    p_par[q] ^= 1;
                    tc_fence_after_sync();
                    const uint32_t go = ok ? elected : 0u;
                    mma_ts_x4(go, o_col, p_col, b_lo, kDescHi, idesc_pv, true);
                    mma_ts_x4(go, o_col, p_col + 32, b_lo + 4 * 128, kDescHi, idesc_pv, true);
                    if (release) mma_commit_if(go, &st.bar_vempty[v_slot]);
                    mma_ss_x4(go, p_col, a0, b0, kDescHi, idesc_s128, false);
                    if (D == 128) mma_ss_x4(go, p_col, a0 + (128 * 128 >> 4), b0 + (kTileKeys * 128 >> 4), kDescHi, idesc_s128, true);
                    mma_commit_if(go, &st.bar_sfull[q]);
                    if (release) mma_commit_if(go, &st.bar_kempty[k_slot]);
                };
                const uint32_t a_q0 = q_lo, a_q1 = q_lo + (SM::kQBlock >> 4);
                const int n_full = min(n, Pb / kTileKeys - seg_t0);   // tiles [0, n_full) of the segment are full prefix tiles
                if (two) {
#pragma unroll 1
                    for (int i = -1; i < n; ++i) {
                        if (i > 0 && i + 2 < n_full) {            // tiles i and i+1 full, and S(i+1) is not the segment's last
                            full(0, a_q0, true, false);
                            full(1, a_q1, false, true);
                        } else {
                            if (i >= 0) pv(0, i, true, false);
                            if (i + 1 < n) qk(0, i + 1, true, false);
                            if (i >= 0) pv(1, i, false, true);
                            if (i + 1 < n) qk(1, i + 1, false, true);
                        }
                    }
                } else {
#pragma unroll 1
                    for (int i = -2; i < n; i += 2) {
                        if (i > 0 && i + 4 < n_full) {            // tiles i to i+3 full, S(i+3) not the last
                            full(0, a_q0, true, true);
                            full(1, a_q0, true, true);
                        } else {
                            if (i >= 0) pv(0, i, true, true);
                            if (i + 2 < n) qk(0, i + 2, true, true);
                            if (i >= 0 && i + 1 < n) pv(1, i + 1, true, true);
                            if (i + 3 < n) qk(1, i + 3, true, true);
                        }
                    }
                }
            }
            // no product may read shared memory or write tensor memory that the CTA has given back
            mma_commit_if(elected, &st.bar_idle);
            ok &= mbar_drain(&st.bar_idle, 0);
            __syncwarp();
        }
    }

    // ---- teardown ----
    if (!ok) st.abort = 1;
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) {
        if (lane == 0 && st.abort) {
            // No load may land in shared memory that the CTA has left.  (Without an abort the roles have waited for every
            // one.)
            mbar_drain(&st.bar_qfull, st.q_last);
            for (int i = 0; i < 2 * RS; ++i) mbar_drain(&st.bar_stfull[i % 2][i / 2], ~(st.st_armed[i % 2] >> i / 2) & 1);     // (one that never was is open)
            if (st.k_tree >> 16) mbar_drain(&st.bar_kfull[st.k_tree & 255], st.k_tree >> 8 & 1);
            if (st.v_tree >> 16) mbar_drain(&st.bar_vfull[st.v_tree & 255], st.v_tree >> 8 & 1);
            set_status(P.status, RADAR_ERR_TIMEOUT);
        }
        __syncwarp();
        tmem_dealloc(st.tmem_base, 512);
    }
}


// Joins the pieces of the units that were cut: blocks (c, *) those of the unit whose first piece CTA c holds.  A warp takes a row at a time,
// four of its pieces in flight.  What bounds it, large launches: the partial sums, written and read (8 sequences of 8192 tokens, 64 / 8 heads, 64 rows:
// 36 MB each way, 15 of the attention's 157 us); small ones, the waves of blocks, so there are two of those and not a block for
// each eight rows (4 sequences of 300 tokens, 40 / 40 heads, 64 rows 24 us, with 4736 blocks 26; two rows a warp spill, 30).
template <int D>
__global__ void __launch_bounds__(256, 6) cache_tc_combine_kernel(const TcParams P) {
    chain_wait();
    const radar_attn_args& a = P.a;
    const CutUnit& cu = P.cut[blockIdx.x];
    const int valid = cu.valid, b = cu.b, g = cu.g, slot = cu.slot, rows = cu.rows, n_pieces = cu.n_pieces;
    const uint32_t live0 = cu.live[0];
    if (!valid) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int E = D / 32, kPieces = 4;                   // elements of a lane; pieces in flight together
    using Part = std::conditional_t<E == 4, float4, float2>;
    for (int r = blockIdx.y * 8 + warp; r < rows; r += gridDim.y * 8) {
        const int blk = r < P.rb_rows ? 0 : 1, in_blk = r - blk * P.rb_rows;       // row blocks start 128 records apart, whatever part of them is live
        float m = -CUDART_INF_F, l = 0.f, o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = 0.f;
        for (int j0 = 0; j0 < n_pieces; j0 += kPieces) {
            const uint32_t live = (j0 < 32 ? live0 : cu.live[j0 >> 5]) >> (j0 & 31);
            float2 ml[kPieces];
            Part v[kPieces];
            float m2 = m;
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                ml[j] = make_float2(-CUDART_INF_F, 0.f);
                if (j0 + j < n_pieces && (live >> j & 1u)) {                       // (a range that holds no tile's start has no piece)
                    const int64_t cta = (int64_t)blockIdx.x + (int64_t)(j0 + j) * P.n_cls;
                    const int64_t rec = (cta * 2 + (j0 + j == 0 ? slot : 0)) * kPairRows + blk * 128 + in_blk;
                    ml[j] = P.part_ml[rec];
                    v[j] = *reinterpret_cast<const Part*>(P.part_o + rec * D + lane * E);
                }
            }
#pragma unroll
            for (int j = 0; j < kPieces; ++j) m2 = fmaxf(m2, ml[j].x);
            if (m2 == -CUDART_INF_F) {                                             // all sums are 0, or NaN from a NaN among the scores
#pragma unroll
                for (int j = 0; j < kPieces; ++j) l += ml[j].y;
                continue;
            }
            const float old = __expf(m - m2);
            m = m2;
            l *= old;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] *= old;
#pragma unroll
            for (int j = 0; j < kPieces; ++j) {
                if (ml[j].x == -CUDART_INF_F) {
                    l += ml[j].y;
                    continue;
                }
                const float w = __expf(ml[j].x - m);
                l = fmaf(ml[j].y, w, l);
                const float* x = reinterpret_cast<const float*>(&v[j]);
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = fmaf(x[e], w, o[e]);
            }
        }
        const int rb_node = (int)(((uint32_t)in_blk * P.g_magic) >> 16);
        const int node = ((blockIdx.x % P.n_cls) * P.n_blk + blk) * P.nodes_per_rb + rb_node, hq = g * P.G + in_blk - rb_node * P.G;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        __nv_bfloat162 w[E / 2];
#pragma unroll
        for (int e = 0; e < E; e += 2) w[e / 2] = __floats2bfloat162_rn(o[e] * inv, o[e + 1] * inv);
        __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(a.O) + (((int64_t)b * P.nodes + node) * a.Hq + hq) * D + lane * E;
        if (E == 4) *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(w);
        else *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(w);
        if (a.lse != nullptr && lane == 0) a.lse[((int64_t)b * a.Hq + hq) * P.nodes + node] = l == 0.f ? -CUDART_INF_F : m + logf(l);
    }
}

// a pool as [blocks][keys or values][bytes], in numbers of eight bytes; box: that of `box_blocks` blocks
template <int D>
bool make_cache_map(CUtensorMap* tm, const void* pages, long long blocks, int box_blocks) {
    constexpr int kPart = Layout<D>::kBytes / 2;
    cuuint64_t dims[3] = {kPart / 8, 2, (cuuint64_t)blocks}, strides[2] = {kPart, 2 * kPart};
    cuuint32_t box[3] = {kPart / 8, 1, (cuuint32_t)box_blocks}, es[3] = {1, 1, 1};
    return encode_fn()(tm, CU_TENSOR_MAP_DATA_TYPE_FLOAT64, 3, const_cast<void*>(pages), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool TWO>
int launch_tc(radar_ctx* ctx, const radar_cache_attn_args& c, TcParams& P, cudaStream_t stream) {
    using SM = Smem<D, TWO>;
    CUtensorMap tmQ, tmKt, tmVt, tmCache;
    const long long tree_rows = (long long)c.B * c.rows;
    // Without a pool nothing is loaded through its map, which still has to lie over memory that is there: some of the tree's keys.
    const bool pool = c.pages != nullptr && c.n_pages > 0;
    const long long blocks = pool ? (long long)c.n_pages * c.Hkv * P.blocks_per_page : 1;
    if (!make_map(&tmQ, c.Q, D, c.Hq, tree_rows, P.G, P.nodes_per_rb, 1, 0, c.q_row_stride) ||
        !make_map(&tmKt, c.Kt, D, c.Hkv, tree_rows, 1, kTreeKeys, 1, 0, c.kv_row_stride) ||
        !make_map(&tmVt, c.Vt, D, c.Hkv, tree_rows, 1, kTreeKeys, 1, 0, c.kv_row_stride) ||
        !make_cache_map<D>(&tmCache, pool ? c.pages : c.Kt, blocks, std::min(P.blocks_per_page, kTileBlocks)))
        return RADAR_ERR_CUDA;
    auto* const kernel = cache_attn_tc_kernel<D, TWO>;
    RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, RADAR_SMEM_CACHE_ATTN_TC + 2 * (D == 128) + TWO, kernel, (size_t)SM::kDynamic));
    {
        radar_launch_scope scope(ctx, RADAR_K_CACHE_ATTN, stream);
        RADAR_CUDA_CHECK(launch_chained(kernel, dim3((unsigned)(P.n_cls * P.ncc)), dim3(kTcThreads), (size_t)SM::kDynamic, stream, tmQ, tmKt, tmVt, tmCache, P));
    }
    {
        radar_launch_scope scope(ctx, RADAR_K_CACHE_COMBINE, stream);
        // two waves of blocks share out the units that can be cut
        const int grid = P.n_cls * P.ncc, cut = (int)std::min<long long>(grid, (long long)c.B * c.Hkv * P.n_cls);
        const int per = std::clamp((12 * ctx->sm_count + cut - 1) / cut, 1, kPairRows / 8);
        RADAR_CUDA_CHECK(launch_chained(cache_tc_combine_kernel<D>, dim3((unsigned)grid, (unsigned)per), dim3(256), 0, stream, P));
    }
    RADAR_CUDA_CHECK(cudaGetLastError());
    return RADAR_OK;
}

size_t tc_partial_bytes(size_t grid, int d) {
    const size_t rec = grid * 2 * kPairRows;
    return align_up(rec * sizeof(float2), 256) + align_up(rec * d * sizeof(float), 256) + align_up(grid * sizeof(CutUnit), 256);
}

}  // namespace

size_t cache_attn_tc_workspace_bytes(const radar_ctx* ctx, int d) { return tc_partial_bytes((size_t)ctx->sm_count, d); }

int cache_attn_tc_launch(radar_ctx* ctx, const radar_cache_attn_args* c, cudaStream_t stream) {
    if (!encode_fn()) return RADAR_ERR_CUDA;
    TcParams P = {};
    radar_attn_args& a = P.a;
    a.B = c->B; a.Hq = c->Hq; a.Hkv = c->Hkv; a.d = c->d;
    a.n_nodes = c->n_nodes; a.mask = c->mask; a.O = c->O; a.lse = c->lse;
    a.prefix_len = c->cache_len; a.max_prefix_len = c->max_cache_len;
    a.block_table = c->block_table; a.max_pages = c->max_pages; a.page_size = c->page_size;
    P.G = c->Hq / c->Hkv;
    P.g_magic = (65536u + P.G - 1) / P.G;
    P.nodes_per_rb = 128 / P.G;
    P.rb_rows = P.nodes_per_rb * P.G;
    P.scale_log2 = (c->scale > 0.f ? c->scale : 1.f / sqrtf((float)c->d)) * 1.4426950408889634f;
    P.status = ctx->d_status;
    P.n_layers = 1;
    P.nodes = c->rows;
    P.n_pages = c->n_pages;
    P.blocks_per_page = c->page_size / kBlock;
    P.page_shift_blocks = -1;
    for (int s = 0; s < 28; ++s)
        if (P.blocks_per_page == 1 << s) P.page_shift_blocks = s;
    bool whole;
    plan_grid(ctx, c->B, c->Hq, c->Hkv, c->max_cache_len, 1, &P.n_blk, &P.n_cls, &P.ncc, &whole, c->rows);
    P.pair_rows = P.n_blk * P.rb_rows;
    P.cost_one = kCosts.one; P.cost_two = kCosts.two; P.unit_cost = whole ? 0 : kCosts.unit;
    const size_t grid = (size_t)P.n_cls * P.ncc;
    if (tc_partial_bytes(grid, c->d) > c->workspace_bytes) return RADAR_ERR_WORKSPACE;
    const size_t rec = grid * 2 * kPairRows;
    P.part_ml = reinterpret_cast<float2*>(c->workspace);
    P.part_o = reinterpret_cast<float*>(reinterpret_cast<char*>(c->workspace) + align_up(rec * sizeof(float2), 256));
    P.cut = reinterpret_cast<CutUnit*>(reinterpret_cast<char*>(P.part_o) + align_up(rec * c->d * sizeof(float), 256));
    const bool two = P.n_blk > 1 && P.nodes_per_rb < c->rows;         // some unit can have two live row blocks
    if (c->d == 128) return two ? launch_tc<128, true>(ctx, *c, P, stream) : launch_tc<128, false>(ctx, *c, P, stream);
    return two ? launch_tc<64, true>(ctx, *c, P, stream) : launch_tc<64, false>(ctx, *c, P, stream);
}

}  // namespace radar
