// Rotary positions (radar_rotate) and the paged cache's writes with the rotation on the way (radar_paged_store): one kernel.
//
// (x, y) -> (x cos - y sin, y cos + x sin) for the pairs of a head, cos and sin of pos * inv_freq: one angle a row and pair, shared
// by all heads.  Every row is read and written once, so memory bounds it (and a launch behind a lookup where there is little).
#include <algorithm>
#include <climits>
#include <type_traits>

#include "common.cuh"

namespace radar {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 4;              // rows of a block
constexpr int kMaxPairs = 512;

struct PagedParams {
    // 0: Q, 1: K, 2: V (not turned)
    const void* in[3];
    void* out[3];
    int64_t in_row[3], out_row[3], in_layer[3], out_layer[3];      // strides, elements
    int heads[3];
    int d, rows;                         // channels of a head, rows of a block (at most kMaxRows)
    int turn_items, rest_items, copy_items;   // of a head: of its pairs, of the channels behind them, of a head that is not turned
    int rest_units, copy_units;          // ... the last two in units (an item is two of them, the last one perhaps one)
    int64_t n_tokens, n_rows, cache_rows;
    const int64_t* slots;                // NULL: token i goes to row i
    const int32_t* src_row;
    radar_rotation r;
    float sign;
    int* status;
};

// A unit is V elements, 16 bytes of them (or one element, for rows of any alignment).
template <typename T, int V>
struct Unit {
    T x[V];
};
template <typename T, int V>
__device__ __forceinline__ Unit<T, V> load_unit(const T* p) {
    Unit<T, V> u;
    if (V > 1) {
        const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p));
        *reinterpret_cast<uint4*>(&u) = w;
    } else {
        u.x[0] = *p;
    }
    return u;
}
template <typename T, int V>
__device__ __forceinline__ void store_unit(T* p, const Unit<T, V>& u) {
    if (V > 1) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&u);
    else *p = u.x[0];
}
__device__ __forceinline__ void from_float(float& y, float x) { y = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }

// cos and sin of pos * f.  The angle in turns, reduced to +- 1/2, is exact to 2^-50: pos * f and its product with 1 / (2 pi) (its double and
// what that lacks) are taken with their remainders.  fp32 has it to 2^-25 of a half turn.
__device__ __forceinline__ float2 turn_of(int pos, float f, float sign) {
    constexpr double kInv = 0.15915494309189535, kInvLow = -9.839338337591243e-18;      // 1 / (2 pi)
    const double a = (double)pos * (double)f, a_low = fma((double)pos, (double)f, -a);
    const double t = a * kInv, t_low = fma(a, kInv, -t) + fma(a, kInvLow, a_low * kInv);
    const double part = (t - rint(t)) + t_low;
    float s, c;
    sincospif((float)(2.0 * part), &s, &c);
    return make_float2(c, s * sign);
}

// A block takes P.rows rows of one layer, its threads first the rows' angles, one each, into shared memory, then the items: two units of
// a head that are turned together (or copied).  The first item is loaded ahead of the barrier.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 6) paged_rows_kernel(const PagedParams P) {
    __shared__ __align__(16) float s_cos[kMaxRows * kMaxPairs], s_sin[kMaxRows * kMaxPairs];
    chain_wait();
    const int pairs = P.r.n_pairs, layer = blockIdx.y;
    const int64_t first = (int64_t)blockIdx.x * P.rows;
    const int n = (int)min((int64_t)P.rows, P.n_tokens - first);
    const int turned = P.turn_items + P.rest_items;              // items of a head that is turned
    const int q_items = P.heads[0] * turned, qk_items = q_items + P.heads[1] * turned, row_items = qk_items + P.heads[2] * P.copy_items;
    const int total = n * row_items, step = gridDim.z * kThreads;

    struct Item {
        const T *a, *b;                  // b NULL: one unit
        T *to_a, *to_b;
        int row, pair;                   // pair < 0: copied
        Unit<T, V> x, y;
    };
    auto take = [&](int at, Item& it) {
        const int r = at / row_items, e = at - r * row_items;
        const int what = e < q_items ? 0 : e < qk_items ? 1 : 2;
        const int in_part = e - (what == 0 ? 0 : what == 1 ? q_items : qk_items), per = what == 2 ? P.copy_items : turned;
        const int head = in_part / per, item = in_part - head * per;
        const int64_t token = first + r;
        int64_t from = token, to = token;
        it.a = nullptr;
        if (P.src_row != nullptr) {
            from = P.src_row[token];
            if (from < 0 || from >= P.n_rows) { set_status(P.status, RADAR_ERR_INVALID_ARG); return; }
        }
        if (what > 0 && P.slots != nullptr) {
            to = P.slots[token];
            if (to < 0) return;
            if (to >= P.cache_rows) { set_status(P.status, RADAR_ERR_INVALID_ARG); return; }
        }
        int u0, u1;                      // the units' first elements
        it.row = r;
        it.pair = -1;
        if (what < 2 && item < P.turn_items) {
            it.pair = item;
            if (!P.r.neighbours) { u0 = item * V; u1 = u0 + pairs; }
            else if (V > 1) { u0 = item * V; u1 = u0 + pairs; }      // (units in the first and in the second half: neighbouring lanes read neighbouring units)
            else { u0 = 2 * item; u1 = u0 + 1; }
        } else {
            const int i = what < 2 ? item - P.turn_items : item, items = what < 2 ? P.rest_items : P.copy_items, units = what < 2 ? P.rest_units : P.copy_units;
            const int base = what < 2 ? 2 * pairs : 0;
            u0 = base + i * V;
            u1 = i + items < units ? u0 + items * V : -1;
        }
        const T* in = reinterpret_cast<const T*>(P.in[what]) + layer * P.in_layer[what] + from * P.in_row[what] + (int64_t)head * P.d;
        T* out = reinterpret_cast<T*>(P.out[what]) + layer * P.out_layer[what] + to * P.out_row[what] + (int64_t)head * P.d;
        it.a = in + u0; it.to_a = out + u0;
        it.b = u1 >= 0 ? in + u1 : nullptr; it.to_b = out + u1;
        it.x = load_unit<T, V>(it.a);
        if (it.b != nullptr) it.y = load_unit<T, V>(it.b);
    };
    auto finish = [&](Item& it) {
        if (it.a == nullptr) return;
        if (it.pair >= 0) {
            const float *co = s_cos + it.row * pairs, *si = s_sin + it.row * pairs;
            if (V > 1 && P.r.neighbours) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    Unit<T, V>& u = h ? it.y : it.x;
                    const int p = (it.pair * V + (h ? pairs : 0)) / 2;
#pragma unroll
                    for (int e = 0; e < V / 2; ++e) {
                        const float c = co[p + e], s = si[p + e], x = to_float(u.x[2 * e]), y = to_float(u.x[2 * e + 1]);
                        from_float(u.x[2 * e], fmaf(x, c, -(y * s)));
                        from_float(u.x[2 * e + 1], fmaf(y, c, x * s));
                    }
                }
            } else {
                const int p = it.pair * V;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float c = co[p + e], s = si[p + e], x = to_float(it.x.x[e]), y = to_float(it.y.x[e]);
                    from_float(it.x.x[e], fmaf(x, c, -(y * s)));
                    from_float(it.y.x[e], fmaf(y, c, x * s));
                }
            }
        }
        store_unit<T, V>(it.to_a, it.x);
        if (it.b != nullptr) store_unit<T, V>(it.to_b, it.y);
    };

    Item it;
    int at = (int)blockIdx.z * kThreads + (int)threadIdx.x;
    if (at < total) take(at, it);
    if (P.r.pos != nullptr) {
        for (int i = threadIdx.x; i < n * pairs; i += kThreads) {
            const int r = i / pairs, p = i - r * pairs;
            int axis = P.r.pair_axis != nullptr ? P.r.pair_axis[p] : 0;
            if (axis >= P.r.n_axes) { set_status(P.status, RADAR_ERR_INVALID_ARG); axis = 0; }
            const float2 cs = turn_of(P.r.pos[axis * P.r.pos_stride + first + r], P.r.inv_freq[p], P.sign);
            s_cos[i] = cs.x;
            s_sin[i] = cs.y;
        }
        __syncthreads();
    }
    for (; at < total; at += step) {
        finish(it);
        if (at + step < total) take(at + step, it);
    }
}

bool rotation_ok(const radar_rotation& r, int d, int64_t n) {
    return r.inv_freq != nullptr && r.n_axes >= 1 && r.n_pairs >= 1 && r.n_pairs <= d / 2 && (r.n_axes == 1 || r.pos_stride >= n);
}

int launch(radar_ctx* ctx, PagedParams& P, int dtype, int n_layers, int kernel_id, cudaStream_t stream) {
    const int es = dtype == RADAR_F32 ? 4 : 2, v = 16 / es;
    if (P.r.pos == nullptr) P.r.n_pairs = 0;
    bool wide = P.d % v == 0 && P.r.n_pairs % v == 0;
    for (int i = 0; i < 3; ++i)
        if (P.heads[i] > 0)
            wide = wide && ((reinterpret_cast<uintptr_t>(P.in[i]) | reinterpret_cast<uintptr_t>(P.out[i])) & 15) == 0 &&
                   ((P.in_row[i] | P.out_row[i] | (n_layers > 1 ? P.in_layer[i] | P.out_layer[i] : 0)) & (v - 1)) == 0;
    const int unit = wide ? v : 1;
    P.turn_items = P.r.n_pairs / unit;
    P.rest_units = (P.d - 2 * P.r.n_pairs) / unit;
    P.copy_units = P.d / unit;
    P.rest_items = (P.rest_units + 1) / 2;
    P.copy_items = (P.copy_units + 1) / 2;
    P.status = ctx->d_status;
    const int64_t row_items = (int64_t)(P.heads[0] + P.heads[1]) * (P.turn_items + P.rest_items) + (int64_t)P.heads[2] * P.copy_items;
    if (row_items * kMaxRows > INT_MAX) return RADAR_ERR_UNSUPPORTED;
    // Rows of a block: as many as there are threads for angles, unless that leaves SMs without one.
    const int64_t wave = 4ll * ctx->sm_count;
    int rows = kMaxRows;
    while (rows > 1 && (P.n_tokens + rows - 1) / rows * n_layers < wave) rows /= 2;
    P.rows = rows;
    const int64_t blocks = (P.n_tokens + rows - 1) / rows;
    // few rows: a row's items over several blocks, which take the angles each for themselves
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>((rows * row_items + kThreads - 1) / kThreads, 64));
    const int64_t split = std::max<int64_t>(1, std::min(most, wave / std::max<int64_t>(1, blocks * n_layers)));
    if (blocks > INT_MAX) return RADAR_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, (unsigned)n_layers, (unsigned)split);
    radar_launch_scope scope(ctx, kernel_id, stream);
    cudaError_t e;
    if (dtype == RADAR_F32) e = launch_chained(wide ? paged_rows_kernel<float, 4> : paged_rows_kernel<float, 1>, grid, dim3(kThreads), 0, stream, P);
    else e = launch_chained(wide ? paged_rows_kernel<__nv_bfloat16, 8> : paged_rows_kernel<__nv_bfloat16, 1>, grid, dim3(kThreads), 0, stream, P);
    RADAR_CUDA_CHECK(e);
    return RADAR_OK;
}

bool misaligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

}  // namespace
}  // namespace radar

using namespace radar;

extern "C" int radar_rotate(radar_ctx* ctx, const radar_rotate_args* a, void* stream_) {
    if (!ctx || !a || a->Hq < 0 || a->Hkv < 0 || a->Hq + (int64_t)a->Hkv == 0 || a->n_rows < 0 || a->d <= 0) return RADAR_ERR_INVALID_ARG;
    if ((a->dtype != RADAR_F32 && a->dtype != RADAR_BF16) || a->d > 2 * kMaxPairs || a->n_rows > INT_MAX) return RADAR_ERR_UNSUPPORTED;
    if (!a->rotation.pos || !rotation_ok(a->rotation, a->d, a->n_rows)) return RADAR_ERR_INVALID_ARG;
    if (a->n_rows == 0) return RADAR_OK;
    const size_t es = a->dtype == RADAR_F32 ? 4 : 2;
    PagedParams P = {};
    P.in[0] = a->Q; P.in[1] = a->K;
    P.out[0] = a->Q_out; P.out[1] = a->K_out;
    P.in_row[0] = a->q_row_stride; P.in_row[1] = a->k_row_stride;
    P.out_row[0] = a->q_out_row_stride; P.out_row[1] = a->k_out_row_stride;
    P.heads[0] = a->Hq; P.heads[1] = a->Hkv;
    for (int i = 0; i < 2; ++i)
        if (P.heads[i] > 0 && (!P.in[i] || !P.out[i] || misaligned(P.in[i], es) || misaligned(P.out[i], es) ||
                               (a->n_rows > 1 && (P.in_row[i] < (int64_t)P.heads[i] * a->d || P.out_row[i] < (int64_t)P.heads[i] * a->d)) ||
                               (P.in[i] == P.out[i] && a->n_rows > 1 && P.in_row[i] != P.out_row[i])))
            return RADAR_ERR_INVALID_ARG;
    P.d = a->d;
    P.n_tokens = P.n_rows = a->n_rows;
    P.r = a->rotation;
    P.sign = a->inverse ? -1.f : 1.f;
    return launch(ctx, P, a->dtype, 1, RADAR_K_ROTATE, reinterpret_cast<cudaStream_t>(stream_));
}

extern "C" int radar_paged_store(radar_ctx* ctx, const radar_paged_store_args* a, void* stream_) {
    if (!ctx || !a || a->n_layers <= 0 || a->Hq < 0 || a->Hkv <= 0 || a->d <= 0 || a->n_tokens < 0 || a->n_rows < 0 || a->cache_rows < 0) return RADAR_ERR_INVALID_ARG;
    if ((a->dtype != RADAR_F32 && a->dtype != RADAR_BF16) || a->d > 2 * kMaxPairs || a->n_layers > 65535 || a->n_tokens > INT_MAX || a->n_rows > INT_MAX) return RADAR_ERR_UNSUPPORTED;
    if (a->rotation.pos && !rotation_ok(a->rotation, a->d, a->n_tokens)) return RADAR_ERR_INVALID_ARG;
    if (!a->src_row && a->n_rows < a->n_tokens) return RADAR_ERR_INVALID_ARG;
    if (a->n_tokens == 0) return RADAR_OK;
    const int64_t kv = (int64_t)a->Hkv * a->d, q = (int64_t)a->Hq * a->d;
    const bool layers = a->n_layers > 1, rows = a->n_rows > 1;
    if (!a->K || !a->V || !a->Kc || !a->Vc || !a->slots || (rows && a->kv_row_stride < kv) || (layers && (a->kv_layer_stride <= 0 || a->cache_layer_stride < a->cache_rows * kv)))
        return RADAR_ERR_INVALID_ARG;
    const size_t es = a->dtype == RADAR_F32 ? 4 : 2;
    if (misaligned(a->K, es) || misaligned(a->V, es) || misaligned(a->Kc, es) || misaligned(a->Vc, es)) return RADAR_ERR_INVALID_ARG;
    if (a->Hq > 0) {
        if (!a->Q || !a->Q_out || (rows && a->q_row_stride < q) || (a->n_tokens > 1 && a->q_out_row_stride < q) || (layers && (a->q_layer_stride <= 0 || a->q_out_layer_stride <= 0)) ||
            misaligned(a->Q, es) || misaligned(a->Q_out, es))
            return RADAR_ERR_INVALID_ARG;
        if (a->Q == a->Q_out && (a->src_row || (rows && a->q_row_stride != a->q_out_row_stride) || (layers && a->q_layer_stride != a->q_out_layer_stride))) return RADAR_ERR_INVALID_ARG;
    }
    PagedParams P = {};
    P.in[0] = a->Q; P.in[1] = a->K; P.in[2] = a->V;
    P.out[0] = a->Q_out; P.out[1] = a->Kc; P.out[2] = a->Vc;
    P.in_row[0] = a->q_row_stride; P.in_row[1] = P.in_row[2] = a->kv_row_stride;
    P.in_layer[0] = a->q_layer_stride; P.in_layer[1] = P.in_layer[2] = a->kv_layer_stride;
    P.out_row[0] = a->q_out_row_stride; P.out_row[1] = P.out_row[2] = kv;
    P.out_layer[0] = a->q_out_layer_stride; P.out_layer[1] = P.out_layer[2] = a->cache_layer_stride;
    P.heads[0] = a->Hq; P.heads[1] = P.heads[2] = a->Hkv;
    P.d = a->d;
    P.n_tokens = a->n_tokens; P.n_rows = a->n_rows; P.cache_rows = a->cache_rows;
    P.slots = a->slots; P.src_row = a->src_row;
    P.r = a->rotation;
    P.sign = 1.f;
    return launch(ctx, P, a->dtype, a->n_layers, RADAR_K_PAGED_STORE, reinterpret_cast<cudaStream_t>(stream_));
}
