// The tile space of the tensor-core attention kernels, shared by the bf16 caches (tree_attention_tc.cu) and the 4-bit cache
// (cache_attention_tc.cu): units of (layer, sequence, KV head, row-block pair), their tiles laid end to end and cut into equal
// ranges, the pieces' records, tensor maps and grid.
#pragma once
#include <cuda.h>

#include <algorithm>

#include "common.cuh"
#include "tc05.cuh"

namespace radar {
namespace {

using namespace tc05;

// how the prefix is held: what the tile space has to look up
enum CacheKind { kContiguous = 0, kPaged = 1, kFourBit = 2 };

constexpr int kTileKeys = 128;       // keys per prefix tile
constexpr int kFirstKeys = 64;       // keys of a tile whose products start before the rest of its probabilities is there
constexpr int kTreeKeys = 64;        // keys of the tree tile (RADAR_MAX_NODES)
constexpr int kPairRows = 256;       // query rows of a row-block pair (and the stride of partial records)
constexpr float kRescaleThreshold = 8.f;   // in log2 units: P stays below 2^8

// Written by every CTA of the attention kernel, read by the combine kernel: the pieces are worked out by the producer warp
// behind its last load, where nothing waits for it, and not by every warp of the combine (two 64-bit divisions a piece).
constexpr int kMaxPerClass = 160;    // CTAs of a class at most (plan_grid)
struct __align__(16) CutUnit {
    int valid;           // 1: this CTA's last segment starts a unit that continues in the following CTAs
    int b, g, layer;     // the unit
    int slot;            // partial slot of that first piece in this CTA (0 or 1)
    int rows;            // live query rows of the unit
    int n_pieces;        // CTAs of the class from this one on whose range begins before the unit's end
    uint32_t live[kMaxPerClass / 32];    // bit j: piece j's range holds the start of a tile of the unit
};

// ... and what its table of pieces follows from.
struct Cut {
    CutUnit unit;
    long long u0, tot;   // start of the unit, size of the class's space (all layers)
    int nt, w;           // tiles of the unit and their cost
};

struct TcParams {
    radar_attn_args a;
    int G, nodes_per_rb; // a row block holds whole nodes: nodes_per_rb = 128 / G (rounded down) of them
    int rb_rows;         // ... so rb_rows = nodes_per_rb * G of its 128 rows can be live (all of them if G divides 128)
    uint32_t g_magic;    // ceil(2^16 / G): row / G == row * g_magic >> 16 for row < 128 and G <= 128
    int n_blk;           // row blocks of a class's units: 2 (they share each K/V tile) or 1
    int pair_rows;       // query rows of a class's units: n_blk * rb_rows
    int n_layers;        // layers run by this launch (the same tree, masks and prefix lengths for all)
    long long o_ls, lse_ls;   // elements between consecutive layers of O and of lse
    int n_cls;           // classes = units per KV head
    int ncc;             // CTAs per class; grid = n_cls * ncc
    int cost_one, cost_two, unit_cost;   // tile_costs(n_cls)
    float scale_log2;
    float scale_log2_lo; // two parts of P: what scale_log2 is below the scale itself (positive)
    long long cache_rows;
    float2* part_ml;     // [grid][2][256]     (m in natural-log units, with two parts of P in log2 units; l)
    float* part_o;       // [grid][2][256][D]
    CutUnit* cut;        // [grid]
    int* status;
    // the 4-bit cache
    int nodes;           // tree rows of a sequence in Q, O, lse, mask and the tree's K and V (RADAR_MAX_NODES elsewhere)
    long long n_pages;
    int blocks_per_page, page_shift_blocks;      // blocks of 16 tokens of a page, log2 of it or -1
};

__device__ __forceinline__ float max3(float a, float b, float c) {
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
// one 32-byte store: a whole sector per lane (the epilogue's lanes write to different rows, so every store
// instruction is split into one transaction per lane; with 16-byte stores each of them filled half a sector)
__device__ __forceinline__ void st_global_32b(void* p, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}
// 2^x and the other steps of a probability, kept in the order in which they are written
__device__ __forceinline__ float ex2_in_order(float x) {
    float y;
    asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 fma2_in_order(float2 a, float2 b, float2 c) {
    float2 d;
    asm volatile("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
                 "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
                 : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2_in_order(float2 a, float2 b) {
    float2 d;
    asm volatile("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
                 : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ uint32_t bf16x2_in_order(float lo, float hi) {
    uint32_t d;
    asm volatile("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// ---- the tile space of one class (unit index pp within a KV head) ---------------------------------
// Positions are in cost units: a tile of a unit with two live row blocks (four MMAs) weighs cost_two, a tile of
// a unit with one live row block cost_one, and every unit books cost_unit in front of its first tile for what it
// costs beside its tiles (pipeline fill, epilogue), so that a CTA whose range holds several unit starts gets fewer
// tiles; equal position ranges are then about equal amounts of time.  A tile belongs to the CTA whose range
// contains the tile's start position.  The weights are measured, not derived (us a launch with its combine, against 3 : 5 without
// the unit term): several classes per KV head, 3 : 5 + 15: 32 / 8 heads, B = 1, 2048 tokens 18.7 -> 17.1; 64 / 8 heads, B = 8, 2000
// to 8192 tokens, trees of two calls 114 -> 111; one class, 2 : 4 + 12: 32 / 8 heads, B = 32, 4096 to 32768 tokens 780 -> 772.
// It is the unit term that counts; 2 : 4 + 12 everywhere gives 17.3, 103 to 108 and 764, other sets lie within 2 %.
struct TileCosts { int one, two, unit; };
inline TileCosts tile_costs(int n_cls) { return n_cls == 1 ? TileCosts{2, 4, 12} : TileCosts{3, 5, 15}; }

struct SeqInfo {
    int M, Pb, nt;       // tree rows, prefix length, tiles of a unit (prefix tiles + the tree tile)
    int rows;            // live query rows of this class's unit (0: it does not exist for this sequence)
    int w;               // cost of one tile
    long long kv0;
};

template <int KIND>
__device__ __forceinline__ SeqInfo seq_info(const TcParams& P, int b, int pp) {
    const radar_attn_args& a = P.a;
    SeqInfo s;
    const int nodes = KIND == kFourBit ? (a.n_nodes != nullptr ? a.n_nodes[b] : P.nodes) : a.n_nodes[b];
    s.M = min(max(nodes, 0), KIND == kFourBit ? P.nodes : kMaxNodes);
    s.Pb = a.prefix_len[b];
    s.kv0 = KIND != kContiguous ? 0 : a.kv_start[b];          // paged: the host has checked max_pages * page_size >= max_prefix_len
    const bool ok = s.Pb >= 0 && s.Pb <= a.max_prefix_len && (KIND == kFourBit ? nodes == s.M : s.kv0 >= 0 && s.kv0 + s.Pb <= P.cache_rows);
    s.rows = ok ? min(max(s.M * P.G - pp * P.pair_rows, 0), P.pair_rows) : 0;
    s.nt = (max(s.Pb, 0) + kTileKeys - 1) / kTileKeys + 1;
    s.w = s.rows > P.rb_rows ? P.cost_two : P.cost_one;
    return s;
}
template <int KIND>
__device__ __forceinline__ long long seq_cost(const TcParams& P, int b, int pp) {
    const SeqInfo s = seq_info<KIND>(P, b, pp);
    return s.rows > 0 ? (long long)P.a.Hkv * (s.nt * s.w + P.unit_cost) : 0;
}
// number of tiles of a unit (start position U, nt tiles of cost w) that start before position x
__device__ __forceinline__ int tiles_before(long long x, long long U, int nt, int w, int unit_cost) {
    const long long d = x - U - unit_cost;           // clamped first, so that the division is a 32-bit one
    if (d <= 0) return 0;
    if (d >= (long long)nt * w) return nt;
    return ((int)d + w - 1) / w;
}

// One CTA's walk over its range [.., hi) of the class's space: segments (sequence b, KV head g, tiles [t0, t1)).
template <int KIND>
struct Cursor {
    int b, g, t0, t1;
    int layer;           // layers follow one another in the space, each with the same sequence of units
    long long U, hi;     // start position of the current unit, end of the CTA's range
    int unit_cost;
    SeqInfo s;
    __device__ __forceinline__ bool valid() const { return t1 > t0; }
    __device__ __forceinline__ void clip() { t1 = tiles_before(hi, U, s.nt, s.w, unit_cost); }
    __device__ __forceinline__ void next_unit(const TcParams& P, int pp) {
        U += (long long)s.nt * s.w + unit_cost;
        t0 = 0;
        if (++g == P.a.Hkv) {
            g = 0;
            do {
                if (++b >= P.a.B) {                               // the next layer starts over at the first sequence
                    if (++layer >= P.n_layers) { t1 = 0; return; }
                    b = 0;
                }
                s = seq_info<KIND>(P, b, pp);
            } while (s.rows == 0);
        }
        clip();
    }
    __device__ __forceinline__ void next(const TcParams& P, int pp) {
        if (t1 < s.nt) { t0 = t1; return; }                  // the range ended inside this unit
        next_unit(P, pp);
    }
    __device__ __forceinline__ bool complete() const { return t0 == 0 && t1 == s.nt; }
    __device__ __forceinline__ bool two_rb(const TcParams& P) const { return s.rows > P.rb_rows; }
};

// The first segment of CTA ci of a class, by a whole warp: the unit that contains the start of its range, from the unit's first
// tile that starts at or after it.  tot_all: size of the class's space (all layers).
template <int KIND>
__device__ __forceinline__ Cursor<KIND> first_segment(const TcParams& P, int pp, int ci, long long& tot_all) {
    const radar_attn_args& a = P.a;
    const int lane = threadIdx.x & 31;
    long long tot = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < a.B; b0 += 32) {
        const int b = b0 + lane;
        if (pp == 0 && ci == 0 && b < a.B) {
            const int Pb = a.prefix_len[b];
            const long long kv0 = KIND != kContiguous ? 0 : a.kv_start[b];
            bool bad = Pb < 0 || Pb > a.max_prefix_len;
            if (KIND == kFourBit) bad |= a.n_nodes != nullptr && (a.n_nodes[b] < 0 || a.n_nodes[b] > P.nodes);
            else bad |= kv0 < 0 || kv0 + Pb > P.cache_rows;
            if (bad) set_status(P.status, RADAR_ERR_INVALID_ARG);
        }
        tot += warp_sum(b < a.B ? seq_cost<KIND>(P, b, pp) : 0ll);
    }
    // the space of all layers: layer l occupies [l * tot, (l + 1) * tot)
    tot_all = tot * P.n_layers;
    const long long lo_all = tot_all * ci / P.ncc;
    Cursor<KIND> cur;
    cur.hi = tot_all * (ci + 1) / P.ncc;
    cur.unit_cost = P.unit_cost;
    cur.layer = tot > 0 ? (int)(lo_all / tot) : 0;
    cur.t0 = cur.t1 = 0;
    cur.b = -1;
    cur.g = 0;
    cur.U = 0;
    const long long lo = lo_all - (long long)cur.layer * tot;
    long long cum = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < a.B && cur.b < 0; b0 += 32) {
        const int b = b0 + lane;
        const long long sz = b < a.B ? seq_cost<KIND>(P, b, pp) : 0;
        long long incl = sz;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(kFull, incl, o);
            if (lane >= o) incl += v;
        }
        const unsigned hit = __ballot_sync(kFull, cum + incl > lo);
        if (hit) {
            const int src = __ffs(hit) - 1;
            const long long before = cum + __shfl_sync(kFull, incl - sz, src);
            cur.b = b0 + src;
            cur.s = seq_info<KIND>(P, cur.b, pp);
            const long long unit = (long long)cur.s.nt * cur.s.w + P.unit_cost;
            cur.g = (int)((lo - before) / unit);
            cur.U = before + cur.g * unit + (long long)cur.layer * tot;
        }
        cum += __shfl_sync(kFull, incl, 31);
    }
    if (cur.b >= 0 && cur.layer < P.n_layers) {
        cur.t0 = tiles_before(lo_all, cur.U, cur.s.nt, cur.s.w, P.unit_cost);
        if (cur.t0 >= cur.s.nt) cur.next_unit(P, pp);       // every tile of that unit starts before the range
        else cur.clip();
    }
    return cur;
}

// What a CTA leaves to the combine, by a whole warp that agrees on `cut`.
__device__ __forceinline__ void write_cut_unit(const TcParams& P, int ci, const Cut& cut) {
    const int lane = threadIdx.x & 31;
    CutUnit* out = P.cut + blockIdx.x;
    int n_pieces = 0;
    if (cut.unit.valid) {
        const long long u0 = cut.u0, tot = cut.tot;
        const int nt = cut.nt, w = cut.w;
        const long long u1 = u0 + (long long)nt * w + P.unit_cost;
#pragma unroll 1
        for (int k = 0; k < kMaxPerClass / 32; ++k) {
            const int c = ci + k * 32 + lane;
            const long long lo = tot * c / P.ncc, hi = tot * (c + 1) / P.ncc;
            const bool piece = c < P.ncc && lo < u1;
            const bool live = piece && tiles_before(hi, u0, nt, w, P.unit_cost) > tiles_before(lo, u0, nt, w, P.unit_cost);
            const uint32_t pieces = __ballot_sync(kFull, piece), bits = __ballot_sync(kFull, live);
            n_pieces += __popc(pieces);
            if (lane == 0) out->live[k] = bits;
            if (pieces != 0xffffffffu) break;
        }
    }
    if (lane == 0) {
        const CutUnit& u = cut.unit;
        out->valid = u.valid; out->b = u.b; out->g = u.g; out->layer = u.layer;
        out->slot = u.slot; out->rows = u.rows; out->n_pieces = n_pieces;
    }
}

// What the other warps know of a segment.
constexpr int kSegRing = 4;
struct __align__(16) Segment {
    int n;                               // tiles; 0: there is no further segment
    int t0, nt, Pb, M, rows;             // first tile, tiles of the unit, prefix length, tree rows, live query rows
    int b, g, layer;
    int pad[3];
};

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = []() -> EncodeTiledFn {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess) return nullptr;
        return q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
    }();
    return fn;
}

// [layers][rows][heads][d] bf16 tensor (layer_stride elements between layers), box = (64 elements, box_heads,
// box_rows, one layer), 128-byte swizzle, zero fill
// row_stride: elements between rows, 0: they lie together
bool make_map(CUtensorMap* tm, const void* base, int d, int heads, long long rows, int box_heads, int box_rows, int layers,
              long long layer_stride, long long row_stride = 0) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    if (row_stride == 0) row_stride = (long long)heads * d;
    if (layers <= 1) { layers = 1; layer_stride = rows * row_stride; }
    cuuint64_t dims[4] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows, (cuuint64_t)layers};
    cuuint64_t strides[3] = {(cuuint64_t)d * 2, (cuuint64_t)row_stride * 2, (cuuint64_t)layer_stride * 2};
    cuuint32_t box[4] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows, 1};
    cuuint32_t es[4] = {1, 1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Grid shape.  A class is one row-block pair (256 query rows: both row blocks share every K/V tile in
// shared memory) or, when such fused units would leave most SMs without work, one row block (128 rows).
// CTAs per class: the grid is one CTA per SM, but at least two tiles per CTA when every sequence has the longest prefix (four
// instead of two, us: 32 / 8 heads, 1000 tokens 16.0 / 14.6; 4 / 4 heads, d = 64, 500 tokens 13.6 / 11.5; 16 / 16 heads, 1000 tokens
// 14.5 / 13.6; but 32 / 8 heads, 2048 tokens 16.5 / 17.1).  Both decisions look at the tiles of the whole launch, all its
// layers: 32 layers of one sequence with 2048 tokens (32 / 8 heads, d = 128) run as 148 CTAs of fused units, where one layer
// alone would be split into half units on 128 CTAs.
void plan_grid(const radar_ctx* ctx, int B, int Hq, int Hkv, int max_prefix_len, int layers, int* n_blk, int* n_cls, int* ncc,
               bool* whole, int nodes = kMaxNodes) {
    const int G = Hq / Hkv;
    const int blocks = (nodes + 128 / G - 1) / (128 / G);         // row blocks of a full tree
    const long long unit_tiles = (long long)layers * B * Hkv * ((max_prefix_len + kTileKeys - 1) / kTileKeys + 1);
    int nb = 2;
    if (blocks > 1 && unit_tiles * ((blocks + 1) / 2) < 4LL * ctx->sm_count) nb = 1;
    const int cls = (blocks + nb - 1) / nb;
    long long per = std::min(ctx->sm_count / cls, kMaxPerClass);
    const long long cap = (unit_tiles + 1) / 2;
    if (per > cap) per = cap;
    if (per < 1) per = 1;
    // All units of one sequence are alike, so where they are no more than the CTAs of a class a grid can be chosen in
    // which every CTA has one piece of one unit and pays for one segment (fill and epilogue, what tile_costs books per
    // unit) and not for two.  Not where that leaves so many CTAs unused that the pieces get longer than what it saves.
    // (Attention + combine, d = 128: 40 / 40 heads, 2048 tokens 22.9 -> 19.6 us; 16 / 16 heads, 1000 tokens 14.8 -> 13.6.  Measured over
    // bf16 rows, with that kernel's weights; the 4-bit cache's, which weighs its tiles otherwise, is planned by the same.)
    const long long units = (long long)layers * Hkv, tiles = unit_tiles / (B * units);
    *whole = false;
    if (B == 1 && units <= per) {
        const TileCosts tc = tile_costs(cls);
        const int w = nb > 1 && blocks > 1 ? tc.two : tc.one;
        const long long pieces = std::max(1ll, std::min(tiles / 2, per / units));
        *whole = (tiles + pieces - 1) / pieces * w <= units * (tiles * w + tc.unit) / per + 2 * tc.unit / 3;
        if (*whole) per = units * pieces;
    }
    *n_blk = nb;
    *n_cls = cls;
    *ncc = (int)per;
}

}  // namespace
}  // namespace radar
