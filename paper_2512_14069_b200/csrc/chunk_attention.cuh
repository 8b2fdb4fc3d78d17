// What the forms of radar_chunk_attention share: the space of units, cut into equal ranges, and the merge of what was cut.
//
// All G query heads of a KV head of a request's n rows are rows (token * G + head in group), cut into units of whole tokens.  A
// unit visits the keys that its last token sees in tiles.  The units of all requests, each at the cost of its keys, are laid end to
// end and cut into equal ranges, one per CTA, so that chunks, whole prompts and single tokens share the machine evenly, and the
// diagonal costs what it holds.  A unit that falls into one CTA is normalised and written at once; the pieces of one that was cut are
// fp32 partials (m, l, O), merged by chunk_combine_kernel.
#pragma once
#include <algorithm>

#include "common.cuh"

namespace radar {
namespace {

constexpr int kMaxCtas = 320;        // of a launch

// The first piece of a unit that continues in the following CTAs, written by the CTA that has it, read by the combine kernel.
struct __align__(16) ChunkCut {
    int valid;           // 1: there is one
    int row0, g;         // first row of Q of the unit, head group
    int slot;            // partial slot of the first piece in this CTA (0 or 1)
    int rows;            // live query rows of the unit
    int n_pieces;        // CTAs from this one on whose range begins before the unit's end
    uint32_t live[kMaxCtas / 32];        // bit j: piece j's range holds the start of a tile of the unit
};

struct ChunkParams {
    radar_chunk_attn_args a;
    int G, groups;           // query heads of a head group, and groups: those of a KV head (see the form)
    int tokens_per_rb;       // a row block holds whole tokens
    int rb_rows;             // ... tokens_per_rb * G rows that can be live
    uint32_t g_magic;        // ceil(2^16 / G): row / G == row * g_magic >> 16 for row < 128 and G <= 128
    int unit_tokens;         // of one row block or a pair of them
    int unit_records;        // partial records of a unit; the second row block's start at half of it
    int n_cta;
    uint64_t cta_magic;      // floor(2^64 / n_cta): see bound_of
    float scale_log2;
    float2* part_ml;         // [n_cta][2][unit_records]     (m in log2 units, l)
    float* part_o;           // [n_cta][2][unit_records][D]
    ChunkCut* cut;           // [n_cta]
    int* status;
};

// A request of the call as its arguments have it: n rows from q0 on, len cached tokens; n = 0 where it is out of bounds.
struct ChunkSeq {
    int q0, n, len;
};
__device__ __forceinline__ ChunkSeq chunk_seq(const radar_chunk_attn_args& a, int b, bool& ok) {
    ChunkSeq s;
    s.q0 = a.q_start[b];
    const long long n = (long long)a.q_start[b + 1] - s.q0;
    s.len = a.cache_len[b];
    ok = s.q0 >= 0 && n >= 0 && n <= a.max_new && s.q0 + n <= a.n_rows && s.len >= 0 && s.len <= a.max_cache_len;
    s.n = ok ? (int)n : 0;
    return s;
}

// ---- the space of units -------------------------------------------------------------------------------------------------
// Positions are in cost units: a key of a unit with two live row blocks weighs C::kTwo, of a unit with one C::kOne, and every unit
// books C::kUnit in front of its first tile of C::kTile keys for what it costs beside its tiles (pipeline fill, epilogue).  A tile
// belongs to the CTA whose range contains the tile's start position.

// a unit's keys and what follows from them
template <class C>
struct Unit {
    int row0, tokens, rows;  // first row of Q, tokens, live query rows
    int seen;                // keys that its first token sees (0 or less: none)
    int keys;                // keys that its last token sees, 1 at least
    int nt, w;               // tiles, cost of a key
    __device__ __forceinline__ long long size() const { return (long long)keys * w + C::kUnit; }
};
__device__ __forceinline__ int units_of(const ChunkParams& P, const ChunkSeq& s) { return (s.n + P.unit_tokens - 1) / P.unit_tokens; }
template <class C>
__device__ __forceinline__ Unit<C> unit_of(const ChunkParams& P, const ChunkSeq& s, int i) {
    Unit<C> u;
    u.row0 = s.q0 + i * P.unit_tokens;
    u.tokens = min(s.n - i * P.unit_tokens, P.unit_tokens);
    u.rows = u.tokens * P.G;
    u.seen = s.len - s.n + i * P.unit_tokens + 1;
    u.keys = max(u.seen + u.tokens - 1, 1);
    u.nt = (u.keys + C::kTile - 1) / C::kTile;
    u.w = u.rows > P.rb_rows ? C::kTwo : C::kOne;
    return u;
}
// size of a request's first m units of one head group, none of them its last; unit i has max(base + (i + 1) T, 1) keys
template <class C>
__device__ __forceinline__ long long size_before(const ChunkParams& P, const ChunkSeq& s, int m) {
    const int T = P.unit_tokens, base = s.len - s.n;
    const long long none = base >= 0 ? 0 : min((unsigned)m, (unsigned)-base / (unsigned)T);       // units whose last token sees nothing (or one key)
    const long long keys = none + (m - none) * base + T * ((long long)m * (m + 1) - none * (none + 1)) / 2;
    return keys * (T > P.tokens_per_rb ? C::kTwo : C::kOne) + (long long)m * C::kUnit;
}
// ... of all of them
template <class C>
__device__ __forceinline__ long long head_size(const ChunkParams& P, const ChunkSeq& s) {
    if (s.n == 0) return 0;
    const int nq = units_of(P, s);
    return size_before<C>(P, s, nq - 1) + unit_of<C>(P, s, nq - 1).size();
}
// number of tiles of a unit at position U that start before position x
template <class C>
__device__ __forceinline__ int tiles_before(long long x, long long U, int nt, int w) {
    const long long d = x - U - C::kUnit;
    if (d <= 0) return 0;
    const long long t = (d + C::kTile - 1) / C::kTile;       // (a tile is kTile w; below nt w it fits an int)
    if (t >= (long long)nt * w) return nt;
    return w == C::kTwo ? ((unsigned)t + C::kTwo - 1) / C::kTwo : ((unsigned)t + C::kOne - 1) / C::kOne;
}
// where CTA c's range begins, for a space of size tot: tot c / n_cta or a little less, without a division
__device__ __forceinline__ long long bound_of(const ChunkParams& P, long long tot, int c) {
    return c >= P.n_cta ? tot : (long long)__umul64hi((unsigned long long)tot * (unsigned)c, P.cta_magic);
}

// One CTA's walk over its range [.., hi): segments (unit, tiles [t0, t1)).
template <class C>
struct Walk {
    int b, g, i, nq, t0, t1;
    long long U, hi;         // start position of the current unit, end of the CTA's range
    ChunkSeq s;
    Unit<C> u;
    __device__ __forceinline__ bool valid() const { return t1 > t0; }
    __device__ __forceinline__ void clip() { t1 = tiles_before<C>(hi, U, u.nt, u.w); }
    __device__ __forceinline__ void next_unit(const ChunkParams& P) {
        U += u.size();
        t0 = 0;
        if (++i == nq) {
            i = 0;
            if (++g == P.groups) {
                g = 0;
                bool ok;
                do {
                    if (++b >= P.a.B) { t1 = 0; return; }
                    s = chunk_seq(P.a, b, ok);
                } while (s.n == 0);
                nq = units_of(P, s);
            }
        }
        u = unit_of<C>(P, s, i);
        clip();
    }
    __device__ __forceinline__ void next(const ChunkParams& P) {
        if (t1 < u.nt) { t0 = t1; return; }                  // the range ended inside this unit
        next_unit(P);
    }
};

// The first segment of CTA ci, by a whole warp: the unit that contains the start of its range, from the unit's first tile that starts at
// or after it.  tot: size of the space.  (What a launch waits for before its first load: 3600 to 4600 cycles with 64-bit divisions and the sizes
// read twice.)
template <class C>
__device__ __forceinline__ Walk<C> first_segment(const ChunkParams& P, int ci, long long& tot) {
    const int lane = threadIdx.x & 31, B = P.a.B;
    bool ok = true;
    ChunkSeq mine;                       // of request lane, and its sizes: with up to 32 of them everything is read once
    mine.q0 = mine.n = mine.len = 0;
    if (lane < B) mine = chunk_seq(P.a, lane, ok);
    const long long my_head = head_size<C>(P, mine);
    auto running = [&](long long v) {    // sums over the lanes up to this one
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(kFull, v, o);
            if (lane >= o) v += x;
        }
        return v;
    };
    const long long my_incl = B == 1 ? my_head * P.groups : running(my_head * P.groups);
    tot = __shfl_sync(kFull, my_incl, B == 1 ? 0 : 31);
#pragma unroll 1
    for (int b0 = 32; b0 < B; b0 += 32) {
        const int b = b0 + lane;
        bool ok_b = true;
        const long long size = b < B ? head_size<C>(P, chunk_seq(P.a, b, ok_b)) * P.groups : 0;
        ok = ok && ok_b;
        tot += warp_sum(size);
    }
    if (!ok && ci == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
    Walk<C> cur;
    const long long lo = bound_of(P, tot, ci);
    cur.hi = bound_of(P, tot, ci + 1);
    cur.t0 = cur.t1 = 0;
    cur.b = -1;
    cur.g = cur.i = cur.nq = 0;
    cur.U = 0;
    cur.s.q0 = cur.s.n = cur.s.len = 0;
    cur.u.row0 = cur.u.tokens = cur.u.rows = cur.u.seen = cur.u.keys = cur.u.nt = cur.u.w = 0;
    long long cum = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < B && cur.b < 0; b0 += 32) {
        const int b = b0 + lane;
        bool ok_b;
        ChunkSeq s = mine;
        long long head = my_head, incl = my_incl;
        if (b0 > 0) {
            s.q0 = s.n = s.len = 0;
            if (b < B) s = chunk_seq(P.a, b, ok_b);
            head = head_size<C>(P, s);
            incl = running(head * P.groups);
        }
        const unsigned hit = __ballot_sync(kFull, b < B && cum + incl > lo);
        if (hit) {
            const int src = __ffs(hit) - 1;
            const long long size = __shfl_sync(kFull, head, src), at = lo - cum - __shfl_sync(kFull, incl - head * P.groups, src);
            cur.b = b0 + src;
            cur.s.q0 = __shfl_sync(kFull, s.q0, src); cur.s.n = __shfl_sync(kFull, s.n, src); cur.s.len = __shfl_sync(kFull, s.len, src);
            cur.nq = units_of(P, cur.s);
            int g = (int)((double)at / (double)size);            // (off by one at most)
            if (g * size > at) --g;
            else if ((g + 1) * size <= at) ++g;
            cur.g = g;
            const long long in_head = at - g * size;
            int m0 = 0, m1 = cur.nq - 1;                         // the last unit that starts at or before it
            while (m0 < m1) {
                const int m = m0 + (m1 - m0 + 1) / 2;
                if (size_before<C>(P, cur.s, m) <= in_head) m0 = m; else m1 = m - 1;
            }
            cur.i = m0;
            cur.U = lo - in_head + size_before<C>(P, cur.s, m0);
            cur.u = unit_of<C>(P, cur.s, m0);
        }
        cum += __shfl_sync(kFull, incl, 31);
    }
    if (cur.b >= 0) {
        cur.t0 = tiles_before<C>(lo, cur.U, cur.u.nt, cur.u.w);
        if (cur.t0 >= cur.u.nt) cur.next_unit(P);               // every tile of that unit starts before the range
        else cur.clip();
    }
    return cur;
}

// What a CTA leaves to the combine, by a whole warp that agrees on it.
struct ChunkPieces {
    ChunkCut unit;
    long long u0, tot;       // start of the unit, size of the space
    int nt, w, size_keys;
};
template <class C>
__device__ __forceinline__ void write_cut(const ChunkParams& P, int ci, const ChunkPieces& cut) {
    const int lane = threadIdx.x & 31;
    ChunkCut* out = P.cut + ci;
    int n_pieces = 0;
    if (cut.unit.valid) {
        const long long u0 = cut.u0, u1 = u0 + (long long)cut.size_keys * cut.w + C::kUnit;
#pragma unroll 1
        for (int k = 0; k < kMaxCtas / 32; ++k) {
            const int c = ci + k * 32 + lane;
            const long long lo = bound_of(P, cut.tot, c), hi = bound_of(P, cut.tot, c + 1);
            const bool piece = c < P.n_cta && lo < u1;
            const bool live = piece && tiles_before<C>(hi, u0, cut.nt, cut.w) > tiles_before<C>(lo, u0, cut.nt, cut.w);
            const uint32_t pieces = __ballot_sync(kFull, piece), bits = __ballot_sync(kFull, live);
            n_pieces += __popc(pieces);
            if (lane == 0) out->live[k] = bits;
            if (pieces != 0xffffffffu) break;
        }
    }
    if (lane == 0) {
        const ChunkCut& u = cut.unit;
        out->valid = u.valid; out->row0 = u.row0; out->g = u.g; out->slot = u.slot; out->rows = u.rows; out->n_pieces = n_pieces;
    }
}

// Merges the pieces of the units that were cut across CTAs.  Blocks (c, *): CTA c of the attention kernel holds the first
// piece of a cut unit (or the blocks exit); the following CTAs hold the rest, each as its first segment.  A warp merges one query row.
template <typename T, int D>
__global__ void __launch_bounds__(256) chunk_combine_kernel(const ChunkParams P) {
    chain_wait();
    const radar_chunk_attn_args& a = P.a;
    const ChunkCut& cu = P.cut[blockIdx.x];
    const int valid = cu.valid, row0 = cu.row0, g = cu.g, slot = cu.slot, rows = cu.rows, n_pieces = cu.n_pieces;
    const uint32_t live0 = cu.live[0];
    if (!valid) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r = blockIdx.y * 8 + warp;
    if (r >= rows) return;                                   // rows of a unit are live from 0 up
    constexpr int E = D / 32;                                // output elements per lane
    // the row's record in piece j's partials (row blocks start half a unit's records apart, whatever part of them is live)
    const int blk = r < P.rb_rows ? 0 : 1, in_blk = r - blk * P.rb_rows;
    auto rec_of = [&](int j) { return (((int64_t)blockIdx.x + j) * 2 + (j == 0 ? slot : 0)) * P.unit_records + blk * (P.unit_records / 2) + in_blk; };
    auto store_row = [&](const float (&o)[E], float mx, float den) {
        const float inv = den == 0.f ? 0.f : 1.f / den;      // (no piece live: o is 0)
        const int rb_token = (int)(((uint32_t)in_blk * P.g_magic) >> 16);
        const int token = blk * P.tokens_per_rb + rb_token, hq = g * P.G + in_blk - rb_token * P.G;
        const int64_t out_row = (int64_t)(row0 + token) * a.Hq + hq;
        T* dst = reinterpret_cast<T*>(a.O) + out_row * D + lane * E;
        if constexpr (sizeof(T) == 2) {
            __nv_bfloat162 w[E / 2];
#pragma unroll
            for (int q = 0; q < E; q += 2) w[q / 2] = __floats2bfloat162_rn(o[q] * inv, o[q + 1] * inv);
            if (E == 4) *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(w);
            else *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(w);
        } else {
            if (E == 4) *reinterpret_cast<float4*>(dst) = make_float4(o[0] * inv, o[1] * inv, o[E - 2] * inv, o[E - 1] * inv);
            else *reinterpret_cast<float2*>(dst) = make_float2(o[0] * inv, o[1] * inv);
        }
        if (a.lse != nullptr && lane == 0) a.lse[out_row] = den == 0.f ? -CUDART_INF_F : lse_of(mx, den);
    };
    auto load_row = [&](const float* src, float (&v)[E]) {
        if (E == 4) {
            const float4 t = *reinterpret_cast<const float4*>(src);
            v[0] = t.x; v[1] = t.y; v[E - 2] = t.z; v[E - 1] = t.w;
        } else {
            const float2 t = *reinterpret_cast<const float2*>(src);
            v[0] = t.x; v[1] = t.y;
        }
    };

    if (n_pieces <= 4) {
        // ---- the usual case: a unit spread over a few CTAs.  (A CTA whose range holds no tile start has no piece.) ----
        float2 ml[4];
        float v[4][E], o[E];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool on = ((live0 >> j) & 1u) && j < n_pieces;
            const int64_t rec = rec_of(on ? j : 0);
            ml[j] = P.part_ml[rec];
            load_row(P.part_o + rec * D + lane * E, v[j]);
            if (!on) ml[j] = make_float2(-CUDART_INF_F, 0.f);
        }
        const float mx = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
        float den = 0.f;
#pragma unroll
        for (int q = 0; q < E; ++q) o[q] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (ml[j].y == 0.f) continue;                    // (its accumulator may hold anything; a sum that is NaN makes the row NaN)
            const float w = ml[j].y != ml[j].y ? ml[j].y : ex2(ml[j].x - mx);
            den = fmaf(ml[j].y, w, den);
#pragma unroll
            for (int q = 0; q < E; ++q) o[q] = fmaf(v[j][q], w, o[q]);
        }
        store_row(o, mx, den);
        return;
    }

    // ---- a unit spread over many CTAs (few units, many keys): lane j holds piece j's (m, l) ----
    float den = 0.f, mx = -CUDART_INF_F, o[E];
    bool nan = false;                                        // a piece's sum is NaN, and so is the row
#pragma unroll
    for (int q = 0; q < E; ++q) o[q] = 0.f;
    for (int j0 = 0; j0 < n_pieces; j0 += 32) {
        const int jl = j0 + lane;
        const uint32_t live = cu.live[j0 >> 5];
        float2 ml = make_float2(-CUDART_INF_F, 0.f);
        if (jl < n_pieces && ((live >> lane) & 1u)) ml = P.part_ml[rec_of(jl)];
        if (__any_sync(kFull, ml.y != ml.y)) nan = true;
        const float mnew = fmaxf(mx, warp_max(ml.x));
        if (mnew == -CUDART_INF_F) continue;
        const float rescale = ex2(mx - mnew);                // 0 on the first live batch
        den *= rescale;
#pragma unroll
        for (int q = 0; q < E; ++q) o[q] *= rescale;
        mx = mnew;
        const float wl = ml.y == 0.f ? 0.f : ex2(ml.x - mx);
        den += warp_sum(ml.y * wl);
        const int nb = min(32, n_pieces - j0);
        for (int u0 = 0; u0 < nb; u0 += 4) {
            float v[4][E], w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                w[u] = u0 + u < nb ? __shfl_sync(kFull, wl, u0 + u) : 0.f;
                if (w[u] != 0.f) {
                    load_row(P.part_o + rec_of(j0 + u0 + u) * D + lane * E, v[u]);
                } else {
#pragma unroll
                    for (int q = 0; q < E; ++q) v[u][q] = 0.f;
                }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int q = 0; q < E; ++q) o[q] = fmaf(v[u][q], w[u], o[q]);
        }
    }
    store_row(o, mx, nan ? CUDART_NAN_F : den);
}

// partial records (two units' per CTA) and the table of cut units of a grid
inline size_t chunk_partial_bytes(size_t grid, int unit_records, int d) {
    const size_t rec = grid * 2 * unit_records;
    return align_up(rec * sizeof(float2), 256) + align_up(rec * d * sizeof(float), 256) + align_up(grid * sizeof(ChunkCut), 256);
}
inline void chunk_carve(ChunkParams& P) {
    P.cta_magic = P.n_cta > 1 ? ~0ull / (unsigned)P.n_cta : ~0ull;
    const size_t rec = (size_t)P.n_cta * 2 * P.unit_records;
    P.part_ml = reinterpret_cast<float2*>(P.a.workspace);
    P.part_o = reinterpret_cast<float*>(reinterpret_cast<char*>(P.a.workspace) + align_up(rec * sizeof(float2), 256));
    P.cut = reinterpret_cast<ChunkCut*>(reinterpret_cast<char*>(P.part_o) + align_up(rec * P.a.d * sizeof(float), 256));
}
// the arguments' part of the parameters, for head groups of G heads and row blocks of up to `rows` rows, `blocks` of them in a unit
inline ChunkParams chunk_params(const radar_ctx* ctx, const radar_chunk_attn_args& a, int G, int rows, int blocks) {
    ChunkParams P;
    P.a = a;
    P.G = G;
    P.groups = a.Hq / G;
    P.g_magic = (65536u + G - 1) / G;
    P.tokens_per_rb = rows / G;
    P.rb_rows = P.tokens_per_rb * G;
    P.unit_tokens = blocks * P.tokens_per_rb;
    P.unit_records = blocks * rows;
    P.scale_log2 = (a.scale > 0.f ? a.scale : 1.f / sqrtf((float)a.d)) * 1.4426950408889634f;
    P.status = ctx->d_status;
    return P;
}
// CTAs of a launch: `pieces` for every unit that the bounds allow, `most` of them at most (which cuts every step of the product, as the bounds may be
// any ints)
inline int chunk_ctas(const ChunkParams& P, int most, long long pieces) {
    long long n = 1;
    for (const long long x : {(long long)P.a.B, (long long)P.groups, ((long long)P.a.max_new + P.unit_tokens - 1) / P.unit_tokens, pieces}) n = std::min((long long)most, n * x);
    return (int)std::max(1ll, n);
}
template <typename T, int D>
int chunk_combine(radar_ctx* ctx, const ChunkParams& P, cudaStream_t stream) {
    const long long rows = min((long long)P.a.max_new * P.G, (long long)P.unit_tokens * P.G);
    radar_launch_scope scope(ctx, RADAR_K_CHUNK_COMBINE, stream);
    RADAR_CUDA_CHECK(launch_chained(chunk_combine_kernel<T, D>, dim3((unsigned)P.n_cta, (unsigned)((rows + 7) / 8)), dim3(256), 0, stream, P));
    return RADAR_OK;
}

}  // namespace

// --- tensor cores (chunk_attention_tc.cu) ---
bool chunk_tc_supported(const radar_chunk_attn_args* a);
size_t chunk_tc_workspace_bytes(const radar_ctx* ctx, int d);
int chunk_tc_launch(radar_ctx* ctx, const radar_chunk_attn_args* a, cudaStream_t stream);
// --- few rows (chunk_attention_rows.cu) ---
// taken: it was launched (or the launch failed); false: the call is the tensor cores'
int chunk_rows_launch(radar_ctx* ctx, const radar_chunk_attn_args* a, cudaStream_t stream, bool& taken);

}  // namespace radar
