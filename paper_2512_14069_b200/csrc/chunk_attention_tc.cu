// Attention of chunks of new tokens over the paged bf16 cache on the 5th-generation tensor cores (tcgen05 + tensor memory), K/V tiles
// staged by TMA.  The machine is that of the tree attention (tree_attention_tc.cu); its units and masks are not.
//
// A head group is a KV head's, a row block up to 128 rows (the MMA M dimension), a unit a pair of row blocks, a tile 128 keys; one CTA per SM.
//
// Inside the CTA (16 warps; the registers are shared out by warpgroup):
//   warp 12    TMA producer: works out the CTA's segments (unit, tile range) for itself and, through a ring in shared memory, for the others;
//              per segment the Q rows, and K tiles into a ring (128-byte swizzle), page by page.
//   warp 14    V tiles into theirs.  (With pages of 16 tokens a tile is 16 copies, and one warp issues them one behind the other.)
//   warp 13    MMA issuer: S = Q K^T into one of two tensor-memory score buffers, and O (+)= P V with P read back from
//              tensor memory (bf16, overlaying S) and V consumed N-major straight from the row-major tile.
//   warps 0-3 / 4-7  softmax groups 0 / 1, one thread per query row.  Unit with two live row blocks: group s owns row block s and sees
//              every tile, so each K/V tile is loaded once for 256 query rows.  Unit with one: the groups take alternate
//              tiles with separate (m, l, O) and are merged at the end.  Either way one group's softmax overlaps the other's MMAs.
//   warps 8-11 epilogue: a finished accumulator to O or to the partials, while the others are in the next segment.
//   warp 15 only fills up the producer's warpgroup.
// Every mbarrier wait is bounded; a wait that runs out sets RADAR_ERR_TIMEOUT on the device status word, the CTA drains, frees its
// tensor memory and returns.
#include <algorithm>
#include <cmath>
#include <cstddef>

#include "attn_tiles.cuh"
#include "chunk_attention.cuh"

namespace radar {
namespace {

constexpr int kChunkThreads = 512;
constexpr int kEpilogueWarp = 8, kProducerWarp = 12, kMmaWarp = 13, kValueWarp = 14;
// Registers a thread: 128 at launch, then shared out by warpgroup (two of softmax; what they take the other two give).
constexpr int kSoftmaxRegs = 176, kEpilogueRegs = 88, kIssueRegs = 72;
static_assert(2 * kSoftmaxRegs + kEpilogueRegs + kIssueRegs <= 512, "a block shares out the registers it was launched with");
constexpr int kStaticSmem = 3 * 1024;    // barriers and exchange arrays: with the tiles exactly the 227 KB a block may have

template <int N> __device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

template <int D>
struct Smem {
    static constexpr int kHalves = D / 64;
    static constexpr int kQBlock = 128 * D * 2;
    static constexpr int kQBytes = 2 * kQBlock;
    static constexpr int kTileBytes = kTileKeys * D * 2;
    static constexpr int kRingK = 3, kRingV = 2;
    static constexpr int kDynamic = kQBytes + (kRingK + kRingV) * kTileBytes;     // starts on a 1024-byte boundary behind the static block
};

constexpr int kFirstKeys = 64, kFirstSteps = kFirstKeys / 16;   // keys of a tile whose products start before the rest of its probabilities is there

struct Costs {
    static constexpr int kTile = kTileKeys, kOne = 3, kTwo = 5, kUnit = 15 * kTileKeys;
};

// What the other warps know of a segment.
struct __align__(16) Segment {
    int n;                               // tiles; 0: there is no further segment
    int t0, nt;                          // first tile, tiles of the unit
    int seen, keys, rows, row0, b, g;    // of the unit (keys: 0 where its last token sees none)
};

// Units of up to kSmallRows rows are products of 64 rows, of which a warp has 16, in its first lanes (what the others hold is never read); a larger
// row block is one of 128, 32 to a warp.  Half the rows are half the tensor cores' energy.  Over and over, under the power limit, 32 / 8 heads of
// 128, 64 / 128 rows: 64 requests of 1000 to 16384 tokens, one row each, 372 us (clock 1.3 GHz) / 412 (1.0); 32 of 8192 tokens, 8 new ones 184 / 191;
// 64 / 8 heads, 7 new ones 193 / 204.
constexpr int kSmallRows = 64;
__device__ __forceinline__ int row_at(const Segment& s, int quarter, int lane) { return quarter * (s.rows <= kSmallRows ? 16 : 32) + lane; }

// The pages of a tile: lane p of a warp looks up and fetches page p, up to eight boxes of a tile (one where a page holds whole tiles).  Only
// pages that hold keys which the unit sees are fetched; what stays stale in the slot is masked or never read.
struct Pages {
    int n_cache_pages, per, box_shift, tiles_per_page;
    __device__ __forceinline__ explicit Pages(const radar_chunk_attn_args& a)
        : n_cache_pages((int)(a.cache_rows / a.page_size)), per(min(a.page_size, kTileKeys)), box_shift(a.page_size == 16 ? 4 : a.page_size == 32 ? 5 : a.page_size == 64 ? 6 : 7),
          tiles_per_page(max(a.page_size / kTileKeys, 1)) {}       // (cache_rows: below 2^31)
    __device__ __forceinline__ int boxes(const Segment& s, int t) const { return (min(kTileKeys, s.keys - t * kTileKeys) + per - 1) >> box_shift; }
    // the lane's page of a tile, and the cache row that it begins at
    __device__ __forceinline__ int index_of(int t, int lane) const { return (tiles_per_page > 1 ? t / tiles_per_page : t << (7 - box_shift)) + lane; }
    __device__ __forceinline__ int page_of(const ChunkParams& P, const Segment& s, int t, int lane) const {
        return lane < boxes(s, t) ? P.a.block_table[(long long)s.b * P.a.max_pages + index_of(t, lane)] : 0;
    }
    __device__ __forceinline__ int row_of(const ChunkParams& P, const Segment& s, int page, int t, int lane) const {
        if (page < 0 || page >= n_cache_pages) {
            if (lane < boxes(s, t)) set_status(P.status, RADAR_ERR_INVALID_ARG);
            page = 0;
        }
        return page * P.a.page_size + (tiles_per_page > 1 ? (t - index_of(t, lane) * tiles_per_page) * kTileKeys : 0);   // (below cache_rows)
    }
    template <int D>
    __device__ __forceinline__ void fetch(const Segment& s, int t, int row, unsigned char* dst, const CUtensorMap* tm, uint64_t* full, int lane) const {
        const int n = boxes(s, t);
        if (lane == 0) mbar_arrive_expect_tx(full, n * per * D * 2);
        __syncwarp();
        if (lane < n)
            for (int h = 0; h < D / 64; ++h) tma_load_3d(dst + h * (kTileKeys * 128) + lane * per * 128, tm, full, h * 64, s.g, row);
        __syncwarp();
    }
};

template <int D>
__global__ void __launch_bounds__(kChunkThreads, 1)
chunk_attn_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const ChunkParams P) {
    chain_trigger();                     // every warp waits for the predecessor where its role begins; the barrier,
                                         // tensor-memory and descriptor set-up needs nothing from global memory
    using SM = Smem<D>;
    constexpr int H = SM::kHalves, RK = SM::kRingK, RV = SM::kRingV;
    const radar_chunk_attn_args& a = P.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = P.G;

    // Static block first (padded to a multiple of 1024 bytes and aligned to it), the tiles behind it: the
    // swizzled tiles need a 1024-byte boundary and there is no room left for alignment slack.
    struct Shared {
        // (in the order of barrier_arrivals)
        uint64_t bar_qfull, bar_qempty, bar_kfull[RK], bar_kempty[RK], bar_vfull[RV], bar_vempty[RV];
        uint64_t bar_sfull[2], bar_odone[2];
        uint64_t bar_idle;               // every product issued has run
        uint64_t bar_segfull[kSegRing];
        uint64_t bar_pfirst[2];          // the probabilities of the tile's first kFirstKeys keys are there
        uint64_t bar_pready[2];          // ... all of them
        uint64_t bar_ofree[2], bar_mlempty;
        uint64_t bar_mlfull;
        uint64_t bar_segempty[kSegRing];
        uint32_t q_last, k_next, v_next; // the producer's: phase parity of the last Q, slot and parity of the next K and V
        uint32_t tmem_base;
        int abort;
        Segment seg[kSegRing];
        ChunkPieces cut;                 // the producer's
        float2 ml[2][128];               // per group: (m in log2 units, l) of the rows at the end of a segment
    };
    static_assert(sizeof(Shared) <= kStaticSmem, "static shared-memory block");
    struct __align__(1024) Static {
        Shared s;
        unsigned char pad[kStaticSmem - sizeof(Shared)];
    };
    static_assert(sizeof(Static) == kStaticSmem, "static shared-memory block");
    __shared__ Static block;
    Shared& st = block.s;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* sQ = smem_raw;
    unsigned char* sK = sQ + SM::kQBytes;
    unsigned char* sV = sK + RK * SM::kTileBytes;

    // ---- set-up ----
    if (warp == 0) {
        constexpr int kOnes = 2 + 2 * RK + 2 * RV + 5 + kSegRing, kFours = 7, kBarriers = kOnes + kFours + 1 + kSegRing;
        static_assert(offsetof(Shared, bar_pfirst) == 8 * kOnes && offsetof(Shared, bar_mlfull) == 8 * (kOnes + kFours) && offsetof(Shared, q_last) == 8 * kBarriers, "barriers in order");
        for (int i = lane; i < kBarriers; i += 32)
            mbar_init(&st.bar_qfull + i, i < kOnes ? 1 : i < kOnes + kFours ? 4 : i == kOnes + kFours ? 8 : kProducerWarp + 2);
        fence_barrier_init();
        if (lane == 0) {
            st.abort = 0;
            st.q_last = 1;
        }
    } else if (warp == kMmaWarp) {
        tmem_alloc(&st.tmem_base, 512);
        tmem_relinquish();
        if (lane == 0) { tma_prefetch_desc(&tmQ); tma_prefetch_desc(&tmK); tma_prefetch_desc(&tmV); }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    // All of tensor memory is this CTA's, so its addresses are constants (the producer checks): S/P buffers in columns 0 and
    // 128, O accumulators in 256 and 384.
    constexpr uint32_t tmem = 0;
    bool ok = true;                         // no wait of this thread has run out
    // Each role starts with chain_sync(): the bounds of the waits behind it are for this kernel's own work.
    // the producer's next segment; false behind the last one
    auto take_segment = [&](uint32_t seg, Segment& s) {
        ok = mbar_wait_while(ok, &st.bar_segfull[seg % kSegRing], (seg / kSegRing) & 1);
        ok = __all_sync(kFull, ok);
        s = st.seg[seg % kSegRing];
        __syncwarp();
        if (lane == 0) mbar_arrive(&st.bar_segempty[seg % kSegRing]);
        return ok && s.n > 0;
    };

    if (warp < kEpilogueWarp) {
        regs_inc<kSoftmaxRegs>();
        chain_sync();
        // =================================== softmax groups ===================================
        // One thread per query row, which holds the tile's 128 scores in registers.
        const int grp = warp >> 2;
        const int place = (warp & 3) * 32 + lane;                // tensor-memory lane
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + grp * 128 + lane_addr;
        const uint32_t tO = tmem + 256 + grp * 128 + lane_addr;
        uint32_t sc = 0;                         // S tiles this group has waited for
        Segment s;
        for (uint32_t seg = 0; take_segment(seg, s); ++seg) {
            const bool two = s.rows > P.rb_rows;
            const int blk = two ? grp : 0;                       // row block within the unit
            const int row0 = row_at(s, warp & 3, 0), row = row0 + lane;      // rows of the block: the warp's first one, the thread's
            const int rows_here = min(s.rows - blk * P.rb_rows, P.rb_rows);  // live rows of this row block
            // A warp none of whose 32 rows is live does no arithmetic (the products of its rows are never read):
            // it only keeps the barriers going.
            const bool warp_live = row0 < rows_here;
            const int lim = s.seen + blk * P.tokens_per_rb + (int)(((uint32_t)row * P.g_magic) >> 16);       // keys that this row sees (more than there are for rows that are not live)
            const int lim_warp = s.seen + blk * P.tokens_per_rb + (int)(((uint32_t)row0 * P.g_magic) >> 16);    // ... and the warp's first one
            const int n_my = two ? s.n : (s.n - grp + 1) >> 1;
            float m_run = -CUDART_INF_F, l_run = 0.f;

#pragma unroll 1
            for (int j = 0; j < n_my; ++j) {
                const int t = s.t0 + (two ? j : 2 * j + grp);
                ok = mbar_wait_while(ok, &st.bar_sfull[grp], sc & 1);
                ok = __all_sync(kFull, ok);                      // warp-uniform: guards .aligned ops
                ++sc;
                tc_fence_after_sync();
                if (ok && warp_live) {
                    uint32_t sv[4][32];
                    if (lim_warp < (t + 1) * kTileKeys) {
                        // Keys that the row does not see become -inf in tensor memory, 32 at a time: the last tile or two of a unit need
                        // it, and an unrolled path for them would be fetched into the instruction cache anew each time.
                        const int valid = lim - t * kTileKeys;
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            const int in = valid - c * 32;
                            const uint32_t al = in >= 32 ? 0xffffffffu : (in <= 0 ? 0u : ((1u << in) - 1u));
                            tmem_ld32(tS + c * 32, sv[0]);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((al >> e) & 1u)) sv[0][e] = 0xff800000u;     // -inf
                            tmem_st32(tS + c * 32, sv[0]);
                        }
                        tmem_wait_st();
                    }
                    tmem_ld32(tS, sv[0]);
                    tmem_ld32(tS + 32, sv[1]);
                    tmem_wait_ld();
                    tmem_ld32(tS + 64, sv[2]);
                    tmem_ld32(tS + 96, sv[3]);
                    float mxa[8];
                    auto half_max = [&](const uint32_t (&u)[32], const uint32_t (&v)[32], const bool first) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8)                      // eight chains, three inputs an instruction
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const float x = __uint_as_float(u[e + c]), y = __uint_as_float(v[e + c]);
                                mxa[c] = first && e == 0 ? fmaxf(x, y) : max3(mxa[c], x, y);
                            }
                    };
                    half_max(sv[0], sv[1], true);
                    tmem_wait_ld();
                    half_max(sv[2], sv[3], false);
                    const float mx = max3(max3(mxa[0], mxa[1], mxa[2]), max3(mxa[3], mxa[4], mxa[5]), fmaxf(mxa[6], mxa[7]));
                    // ---- running max (log2 units), lazy rescale of the accumulator when some row of the warp moved its max ----
                    const float m_tile = mx * P.scale_log2;
                    float factor = 1.f;
                    if (j == 0) {
                        m_run = m_tile;
                    } else if (m_tile > m_run + kRescaleThreshold) {
                        factor = ex2(m_run - m_tile);           // m_run may be -inf: factor 0 clears O and l
                        m_run = m_tile;
                    }
                    const float m_use = m_run == -CUDART_INF_F ? 0.f : m_run;
                    if (j > 0 && __any_sync(kFull, factor != 1.f)) {
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
                    // ---- P = exp2(s * scale - m), row sum, bf16 pairs back to tensor memory ----
                    // (the scaling and the row sum work on pairs: one packed fp32x2 instruction per two values)
                    // The warp issues in order and an exponential takes its unit 8 cycles: what else there is to do stands between
                    // two of them.
                    float2 ls[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    const float2 sc2 = make_float2(P.scale_log2, P.scale_log2), nm2 = make_float2(-m_use, -m_use);
                    uint32_t pk[16];
                    auto scale = [&](const int p) {
                        uint32_t &x = sv[p >> 4][2 * (p & 15)], &y = sv[p >> 4][2 * (p & 15) + 1];
                        const float2 s2 = make_float2(__uint_as_float(x), __uint_as_float(y));
                        const float2 t2 = fma2_in_order(s2, sc2, nm2);
                        x = __float_as_uint(t2.x);
                        y = __float_as_uint(t2.y);
                    };
                    auto finish = [&](const int p) {
                        const float p0 = __uint_as_float(sv[p >> 4][2 * (p & 15)]), p1 = __uint_as_float(sv[p >> 4][2 * (p & 15) + 1]);
                        ls[p & 1] = add2_in_order(ls[p & 1], make_float2(p0, p1));
                        pk[p & 15] = bf16x2_in_order(p0, p1);
                        if ((p & 15) == 15) tmem_st16(tS + (p >> 4) * 16, pk);
                    };
                    // pairs that the scaling is ahead, that the rest is behind, and that the first stores are given to land in
                    constexpr int kAhead = 2, kLag = 4, kLanding = 4;
#pragma unroll
                    for (int p = 0; p < kAhead; ++p) scale(p);
#pragma unroll
                    for (int p = 0; p < 64 + kLag; ++p) {
                        if (p < 64) sv[p >> 4][2 * (p & 15)] = __float_as_uint(ex2_in_order(__uint_as_float(sv[p >> 4][2 * (p & 15)])));
                        if (p + kAhead < 64) scale(p + kAhead);
                        if (p < 64) sv[p >> 4][2 * (p & 15) + 1] = __float_as_uint(ex2_in_order(__uint_as_float(sv[p >> 4][2 * (p & 15) + 1])));
                        if (p >= kLag) finish(p - kLag);
                        if (p == kFirstKeys / 2 - 1 + kLag + kLanding) {
                            tmem_wait_st();
                            tc_fence_before_sync();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&st.bar_pfirst[grp]);
                        }
                    }
                    l_run = l_run * factor + ((ls[0].x + ls[0].y) + (ls[1].x + ls[1].y));
                    tmem_wait_st();
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    if (!(ok && warp_live)) mbar_arrive(&st.bar_pfirst[grp]);
                    mbar_arrive(&st.bar_pready[grp]);
                }
            }

            // the rows' (m, l) go to the epilogue, which has taken those of the segment before
            ok = mbar_wait_while(ok, &st.bar_mlempty, (seg & 1) ^ 1);
            st.ml[grp][place] = make_float2(m_run, l_run);
            __syncwarp();
            if (lane == 0) mbar_arrive(&st.bar_mlfull);
        }
    } else if (warp < kProducerWarp) {
        regs_dec<kEpilogueRegs>();
        chain_sync();
        // =================================== epilogue ===================================
        // One thread per tensor-memory lane takes the finished accumulators to O (or to the partials) while the softmax
        // groups and the tensor cores are already in the next segment; each accumulator is handed back as soon as it is read.
        const int place = (warp - kEpilogueWarp) * 32 + lane;
        const uint32_t tO = tmem + 256 + ((uint32_t)((warp - kEpilogueWarp) * 32) << 16);
        uint32_t oc[2] = {0, 0};             // accumulators waited for
        Segment s;
        for (uint32_t seg = 0; take_segment(seg, s); ++seg) {
            const bool two = s.rows > P.rb_rows;
            const bool final_rows = s.n == s.nt;                 // the whole unit
            const int slot = seg == 0 ? 0 : 1;                   // a CTA has at most a cut first and a cut last segment
            ok = mbar_wait_lazy(ok, &st.bar_mlfull, seg & 1);
            const int row = row_at(s, warp - kEpilogueWarp, lane), rb_token = (int)(((uint32_t)row * P.g_magic) >> 16);       // row / G
            const bool held = s.rows > kSmallRows || lane < 16;
            const float2 ml0 = st.ml[0][place], ml1 = st.ml[1][place];
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
                const bool row_live = held && row < rows_here;
                if (ok && row - lane < rows_here) {
                    float m_out = blk == 0 ? ml0.x : ml1.x, l_out = blk == 0 ? ml0.y : ml1.y, w0 = 1.f, w1 = 0.f;
                    if (merge) {
                        m_out = fmaxf(ml0.x, ml1.x);
                        const float ms = m_out == -CUDART_INF_F ? 0.f : m_out;
                        w0 = ex2(ml0.x - ms);                        // exp2(-inf) = 0
                        w1 = ex2(ml1.x - ms);
                        l_out = ml0.y * w0 + ml1.y * w1;
                    }
                    // a row that saw no key of these tiles (l = 0): O is 0, whatever its accumulator holds
                    const bool empty = l_out == 0.f;
                    const float inv = final_rows ? 1.f / l_out : 1.f;
                    const int token = blk * P.tokens_per_rb + rb_token;
                    const int hq = s.g * G + row - rb_token * G;
                    const int64_t out_row = (int64_t)(s.row0 + token) * a.Hq + hq;
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
                                    const __nv_bfloat162 t2 = __floats2bfloat162_rn(empty ? 0.f : v[2 * e] * inv, empty ? 0.f : v[2 * e + 1] * inv);
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
                        if (!final_rows) P.part_ml[rec] = make_float2(empty ? -CUDART_INF_F : m_out, l_out);
                        else if (a.lse != nullptr) a.lse[out_row] = empty ? -CUDART_INF_F : lse_of(m_out, l_out);
                    }
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&st.bar_ofree[blk]);
            }
        }
    } else {
        regs_dec<kIssueRegs>();
        chain_sync();                            // every global access of the CTA comes behind one
        if (warp == kProducerWarp) {
            // =================================== TMA producer ===================================
            const bool lead = lane == 0;
            const bool usable = (smem_u32(smem_raw) & 1023u) == 0 && st.tmem_base == 0;     // (else the tiles would not sit on their swizzle boundary)
            if (!usable && lead) set_status(P.status, RADAR_ERR_CUDA);
            ChunkPieces& cut = st.cut;
            long long tot;
            Walk<Costs> cur = first_segment<Costs>(P, blockIdx.x, tot);
            if (!usable) cur.t0 = cur.t1 = 0;
            __syncwarp();
            if (lead) { cut.unit.valid = 0; cut.tot = tot; }
            Pages pages(a);
            uint32_t slot = 0, par = 1;                              // ring slot to fill next and the phase that frees it
            for (uint32_t seg = 0;; ++seg) {
                const bool on = cur.valid();
                Segment s;                           // (behind a wait that ran out the others are sent home)
                s.n = cur.t1 - cur.t0; s.t0 = cur.t0; s.nt = cur.u.nt; s.seen = cur.u.seen; s.rows = cur.u.rows; s.row0 = cur.u.row0; s.b = cur.b; s.g = cur.g;
                s.keys = min(cur.u.keys, max(cur.u.seen + cur.u.tokens - 1, 0));
                if (lead) {
                    ok = mbar_wait_while(ok, &st.bar_segempty[seg % kSegRing], ((seg / kSegRing) & 1) ^ 1);
                    st.seg[seg % kSegRing] = s;
                    if (!(on && ok)) st.seg[seg % kSegRing].n = 0;
                    mbar_arrive(&st.bar_segfull[seg % kSegRing]);
                }
                if (!on) break;
                if (lead && s.t0 == 0 && s.n < s.nt) {               // necessarily the last segment of this CTA
                    cut.unit.valid = 1; cut.unit.row0 = s.row0; cut.unit.g = s.g; cut.unit.slot = seg == 0 ? 0 : 1; cut.unit.rows = s.rows;
                    cut.nt = s.nt; cut.w = cur.u.w; cut.size_keys = cur.u.keys; cut.u0 = cur.U;
                }
                auto fetch_q = [&]() {
                    ok = mbar_wait_while(ok, &st.bar_qempty, (seg & 1) ^ 1);
                    const int blocks = s.rows > P.rb_rows ? 2 : 1;
                    if (ok) {
                        st.q_last = seg & 1;
                        mbar_arrive_expect_tx(&st.bar_qfull, blocks * P.rb_rows * D * 2);   // rows past rb_rows stay stale: never read back
                        for (int q = 0; q < blocks; ++q)
                            for (int h = 0; h < H; ++h)
                                tma_load_3d(sQ + q * SM::kQBlock + h * (128 * 128), &tmQ, &st.bar_qfull, h * 64, s.g * G, s.row0 + q * P.tokens_per_rb);
                    }
                };
                // Q's slot is free only after the last S of the segment before, so the first K tiles go ahead of it; the CTA's first segment finds
                // it free, while its keys are looked up.
                int page = pages.page_of(P, s, s.t0, lane);
                if (seg == 0 && lead) fetch_q();
#pragma unroll 1
                for (int i = 0; i < s.n; ++i) {
                    const int here = pages.row_of(P, s, page, s.t0 + i, lane);
                    if (i + 1 < s.n) page = pages.page_of(P, s, s.t0 + i + 1, lane);     // (looked up while the slot is not free yet)
                    if (lead) ok = mbar_wait_while(ok, &st.bar_kempty[slot], par);
                    ok = __shfl_sync(kFull, ok, 0);
                    if (!ok) break;                                  // (the ring's position stays that of the last load)
                    pages.template fetch<D>(s, s.t0 + i, here, sK + slot * SM::kTileBytes, &tmK, &st.bar_kfull[slot], lane);
                    if (++slot == RK) { slot = 0; par ^= 1; }
                    if (i == min(s.n, 2) - 1 && seg > 0 && lead) fetch_q();
                }
                cur.next(P);
            }
            __syncwarp();
            write_cut<Costs>(P, blockIdx.x, cut);
            if (lead) st.k_next = slot | par << 8;
            __syncwarp();
        } else if (warp == kValueWarp) {
            // =================================== V tiles ===================================
            Pages pages(a);
            uint32_t slot = 0, par = 1;
            Segment s;
            for (uint32_t seg = 0; take_segment(seg, s); ++seg) {
                int page = pages.page_of(P, s, s.t0, lane);
#pragma unroll 1
                for (int i = 0; i < s.n; ++i) {
                    const int here = pages.row_of(P, s, page, s.t0 + i, lane);
                    if (i + 1 < s.n) page = pages.page_of(P, s, s.t0 + i + 1, lane);
                    if (lane == 0) ok = mbar_wait_while(ok, &st.bar_vempty[slot], par);
                    ok = __shfl_sync(kFull, ok, 0);
                    if (!ok) break;
                    pages.template fetch<D>(s, s.t0 + i, here, sV + slot * SM::kTileBytes, &tmV, &st.bar_vfull[slot], lane);
                    if (++slot == RV) { slot = 0; par ^= 1; }
                }
            }
            if (lane == 0) st.v_next = slot | par << 8;
            __syncwarp();
        } else if (warp == kMmaWarp) {
            // =================================== MMA issuer ===================================
            // Every lane waits on the barriers (and helps to clear what lies behind the last key), one issues the products and the commits.  No
            // control flow depends on a wait's outcome but that: after a wait that ran out nothing is issued and the loops run dry.
            // The vote on the waits comes first, and the branch of the one lane inside its branch: a product then takes 20 to 30 cycles to
            // issue, and 66 where one branch asks for both.  Some eight products queue up in front of the tensor cores, so that they have work
            // while this warp is in a wait.
            // descriptors: stride between 8-row groups 1024 B, version, swizzle; in units of 16 bytes
            constexpr uint64_t kDesc = (uint64_t)((1024u >> 4) | (1u << 14) | (2u << 29)) << 32;
            constexpr uint32_t kHalfTile = kTileKeys * 128 >> 4;     // between the 64-column blocks of a tile
            auto place = [](const void* p) { return (uint64_t)((smem_u32(p) & 0x3ffff) >> 4); };
            const uint64_t q_desc = kDesc | place(sQ) | (1u << 16), k_desc = kDesc | place(sK) | (1u << 16);
            const uint64_t v_desc = kDesc | place(sV) | (kHalfTile << 16);                 // N-major: 64-column blocks are a half tile apart
            const bool leader = elect_one() != 0;
            uint32_t k_next = 0, k_par = 0, v_next = 0, v_par = 0;   // ring slot to take next and its phase parity
            uint32_t p_par[2] = {0, 0};              // phase parity of the next P tile per group
            Segment s;
            for (uint32_t seg = 0; take_segment(seg, s); ++seg) {
                const int seg_t0 = s.t0, n = s.n, keys = s.keys;
                const bool two = s.rows > P.rb_rows;
                const uint32_t idesc_s = s.rows <= kSmallRows ? idesc_bf16_f32(64, kTileKeys, false, false) : idesc_bf16_f32(128, kTileKeys, false, false);
                const uint32_t idesc_pv = s.rows <= kSmallRows ? idesc_bf16_f32(64, D, false, true) : idesc_bf16_f32(128, D, false, true);
                ok = mbar_wait_while(ok, &st.bar_qfull, seg & 1);
                uint32_t k_slot = 0, v_slot = 0;      // ring slots of the K and V tiles in use
                uint32_t k_wait = 0, v_wait = 0;      // ... and the parities to wait for them with
                bool acc[2] = {false, false};         // accumulator holds a product of this segment
                auto take_v = [&]() {
                    v_slot = v_next;
                    v_wait = v_par;
                    if (++v_next == RV) { v_next = 0; v_par ^= 1; }
                };
                auto take_k = [&]() {
                    k_slot = k_next;
                    k_wait = k_par;
                    if (++k_next == RK) { k_next = 0; k_par ^= 1; }
                };
                // the accumulator's first product of the segment: the epilogue of the previous one has read it
                auto take_o = [&](const int q) {
                    if (!acc[q]) ok = mbar_wait_while(ok, &st.bar_ofree[q], (seg & 1) ^ 1);
                };
                // products of 16 keys each: O[q] (+)= P[q] V, steps [from, to) of tile v_slot
                auto issue_pv = [&](const int q, const int from, const int to, const bool first) {
                    const uint64_t b = v_desc + v_slot * (SM::kTileBytes >> 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i >= from && i < to) mma_ts(tmem + 256 + q * 128, tmem + q * 128 + 8 * i, b + 128 * i, idesc_pv, !first || i > 0);
                };
                // S[q] = Q K^T.  Nothing in tensor memory changes hands here: K arrives through the async proxy, and the buffer was
                // last read by this thread's own P V, which runs first.
                auto issue_s = [&](const int q, const int block) {
                    const uint64_t a0 = q_desc + block * (SM::kQBlock >> 4), b = k_desc + k_slot * (SM::kTileBytes >> 4);
#pragma unroll
                    for (int h = 0; h < H; ++h)
#pragma unroll
                        for (int i = 0; i < 4; ++i) mma_ss(tmem + q * 128, a0 + h * kHalfTile + 2 * i, b + h * kHalfTile + 2 * i, idesc_s, h + i > 0);
                };

                // ---- O[q] (+)= P[q] V for tile i (q is a literal at every call site) ----
                auto pv = [&](const int q, const int i, const bool fresh_v, const bool release_v) {
                    const int valid = min(kTileKeys, keys - (seg_t0 + i) * kTileKeys);
                    const int ksteps = (valid + 15) >> 4;
                    if (fresh_v) {
                        take_v();
                        ok = mbar_wait_while(ok, &st.bar_vfull[v_slot], v_wait);
                        if (valid < ksteps * 16) {
                            // rows past the last key meet P = 0; they must not hold NaN/Inf bit patterns
                            unsigned char* vtile = sV + v_slot * SM::kTileBytes;
                            const int nrows = ksteps * 16 - valid;
#pragma unroll 1
                            for (int e = lane; e < nrows * 8 * H; e += 32) {
                                const int h = e / (nrows * 8), rem = e % (nrows * 8);
                                const int r = valid + rem / 8, c = rem % 8;
                                *reinterpret_cast<uint4*>(vtile + h * (kTileKeys * 128) + r * 128 + c * 16) = make_uint4(0, 0, 0, 0);
                            }
                            fence_proxy_async_smem();
                            __syncwarp();
                        }
                    }
                    take_o(q);
                    ok = mbar_wait_while(ok, &st.bar_pready[q], p_par[q]);
                    p_par[q] ^= 1;
                    tc_fence_after_sync();
                    if (__all_sync(kFull, ok)) {
                        if (leader) {
                            issue_pv(q, 0, ksteps, !acc[q]);
                            if (release_v) mma_commit(&st.bar_vempty[v_slot]);
                            if (two ? i == n - 1 : i + 2 >= n) mma_commit(&st.bar_odone[q]);
                        }
                    }
                    __syncwarp();
                    acc[q] = true;
                };
                // ---- S[q] = Q K^T for tile si ----
                auto qk = [&](const int q, const int si, const bool fresh_k, const bool release_k) {
                    if (fresh_k) {
                        take_k();
                        ok = mbar_wait_while(ok, &st.bar_kfull[k_slot], k_wait);
                    }
                    if (__all_sync(kFull, ok)) {
                        if (leader) {
                            issue_s(q, two ? q : 0);
                            if (release_k) mma_commit(&st.bar_kempty[k_slot]);
                            mma_commit(&st.bar_sfull[q]);
                            // the last S of the segment: Q may be overwritten once it has run
                            if (si == n - 1 && release_k) mma_commit(&st.bar_qempty);
                        }
                    }
                    __syncwarp();
                };
                // Schedule.  Two live row blocks: group s owns row block s; per tile PV0(i) S0(i+1) PV1(i) S1(i+1),
                // both groups sharing K(i+1) and V(i).  One live row block: the groups take alternate tiles,
                // PV(i) S(i+2) for group i & 1.  S of the first tile(s) comes from the iterations with i < 0.
                // Steady state (all tiles involved are full): the same steps with nothing to decide and few waits.
                auto full = [&](const int q, const int block, const bool fresh, const bool release, const bool last_s) {
                    take_o(q);
                    if (fresh) {
                        take_v();
                        take_k();
                        ok = mbar_wait_both(ok, &st.bar_vfull[v_slot], v_wait, &st.bar_pfirst[q], p_par[q]);
                    } else {
                        ok = mbar_wait_while(ok, &st.bar_pfirst[q], p_par[q]);
                    }
                    tc_fence_after_sync();
                    if (__all_sync(kFull, ok)) {
                        if (leader) issue_pv(q, 0, kFirstSteps, !acc[q]);
                    }
                    __syncwarp();
                    if (fresh) ok = mbar_wait_both(ok, &st.bar_kfull[k_slot], k_wait, &st.bar_pready[q], p_par[q]);
                    else ok = mbar_wait_while(ok, &st.bar_pready[q], p_par[q]);
                    p_par[q] ^= 1;
                    acc[q] = true;
                    tc_fence_after_sync();
                    if (__all_sync(kFull, ok)) {
                        if (leader) {
                            issue_pv(q, kFirstSteps, 8, false);
                            if (release) mma_commit(&st.bar_vempty[v_slot]);
                            issue_s(q, block);
                            mma_commit(&st.bar_sfull[q]);
                            if (release) mma_commit(&st.bar_kempty[k_slot]);
                            if (last_s) mma_commit(&st.bar_qempty);
                        }
                    }
                    __syncwarp();
                };
                const int n_full = min(n, keys / kTileKeys - seg_t0);   // tiles [0, n_full) of the segment are full
                if (two) {
#pragma unroll 1
                    for (int i = -1; i < n; ++i) {
                        if (i >= 0 && i < n_full && i + 1 < n) {
                            full(0, 0, true, false, false);
                            full(1, 1, false, true, i + 2 == n);
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
                        if (i >= 0 && i + 1 < n_full && i + 3 < n) {
                            full(0, 0, true, true, false);
                            full(1, 0, true, true, i + 4 == n);
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
            if (leader) mma_commit(&st.bar_idle);
            __syncwarp();
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
            // No load may land in shared memory that the CTA has left.  (Without an abort the roles have waited for every one.)
            const uint32_t k = st.k_next, v = st.v_next;
            mbar_drain(&st.bar_qfull, st.q_last);
            for (int i = 0; i < RK; ++i) mbar_drain(&st.bar_kfull[i], last_armed_parity(i, k & 255, k >> 8));
            for (int i = 0; i < RV; ++i) mbar_drain(&st.bar_vfull[i], last_armed_parity(i, v & 255, v >> 8));
            set_status(P.status, RADAR_ERR_TIMEOUT);
        }
        __syncwarp();
        tmem_dealloc(st.tmem_base, 512);
    }
}

// [rows][heads][d] bf16, row_stride elements between rows; box = (64 elements, box_heads, box_rows), 128-byte swizzle, zero fill
bool make_map(CUtensorMap* tm, const void* base, int d, int heads, long long rows, long long row_stride, int box_heads, int box_rows) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows};
    cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)row_stride * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
    cuuint32_t es[3] = {1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int most_ctas(const radar_ctx* ctx) { return std::min(ctx->sm_count, kMaxCtas); }

template <int D>
int launch_d(radar_ctx* ctx, const ChunkParams& P, cudaStream_t stream) {
    const radar_chunk_attn_args& a = P.a;
    CUtensorMap tmQ, tmK, tmV;
    const int box = std::min(a.page_size, kTileKeys);          // rows of a box
    if (!make_map(&tmQ, a.Q, D, a.Hq, a.n_rows, a.q_row_stride, P.G, P.tokens_per_rb) ||
        !make_map(&tmK, a.Kc, D, a.Hkv, a.cache_rows, (long long)a.Hkv * D, 1, box) ||
        !make_map(&tmV, a.Vc, D, a.Hkv, a.cache_rows, (long long)a.Hkv * D, 1, box))
        return RADAR_ERR_CUDA;
    RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, RADAR_SMEM_CHUNK_TC + (D == 128), chunk_attn_tc_kernel<D>, (size_t)Smem<D>::kDynamic));
    {
        radar_launch_scope scope(ctx, RADAR_K_CHUNK_ATTN, stream);
        RADAR_CUDA_CHECK(launch_chained(chunk_attn_tc_kernel<D>, dim3((unsigned)P.n_cta), dim3(kChunkThreads), (size_t)Smem<D>::kDynamic, stream, tmQ, tmK, tmV, P));
    }
    return chunk_combine<__nv_bfloat16, D>(ctx, P, stream);
}

}  // namespace

bool chunk_tc_supported(const radar_chunk_attn_args* a) { return a->dtype == RADAR_BF16 && encode_fn() != nullptr; }

size_t chunk_tc_workspace_bytes(const radar_ctx* ctx, int d) { return chunk_partial_bytes((size_t)most_ctas(ctx), kPairRows, d); }

int chunk_tc_launch(radar_ctx* ctx, const radar_chunk_attn_args* a, cudaStream_t stream) {
    ChunkParams P = chunk_params(ctx, *a, a->Hq / a->Hkv, 128, 2);
    // One CTA per SM, but no more than make a unit of the bounds' size the fastest by itself: a CTA takes 0.8 us a tile, the merge 0.11 a piece, so
    // sqrt(7 tiles) pieces.  (us, half as many pieces as tiles / these: one unit of 63 tiles 16.4 / 15.4, of 250 33.0 / 23.4; 8 of 4 19.1 / 17.0; 16 of
    // one 12.8 / 9.9.)
    const long long tiles = std::max(1, (a->max_cache_len + kTileKeys - 1) / kTileKeys), pieces = std::min(tiles, (long long)std::ceil(std::sqrt(7.0 * tiles)));
    P.n_cta = chunk_ctas(P, most_ctas(ctx), pieces);
    chunk_carve(P);
    return a->d == 128 ? launch_d<128>(ctx, P, stream) : launch_d<64>(ctx, P, stream);
}

}  // namespace radar
