// Rotary positions (radar_rotate) and the paged cache's writes with the rotation on the way (radar_paged_store): one kernel.
//
// (x, y) -> (x cos - y sin, y cos + x sin) for the pairs of a head, cos and sin of pos * inv_freq: one angle a row and pair, shared
// by all heads.  Every row is read and written once, so memory bounds it (and a launch behind a lookup where there is little).
#include <algorithm>
#include <climits>
#include <cstring>
#include <type_traits>

#include "common.cuh"

namespace radar {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 2;                 // rows of a block, where there are many
constexpr int kMaxPairs = 512;

struct PagedParams {
    // 0: Q, 1: K, 2: V (not turned)
    const void* in[3];
    void* out[3];
    int64_t in_row[3], out_row[3], in_layer[3], out_layer[3];      // strides, elements
    int heads[3];
    int d;                               // channels of a head
    int turn_items, rest_items, copy_items;   // of a head: of its pairs, of the channels behind them, of a head that is not turned
    int rest_units, copy_units;          // ... the last two in units (an item is two of them, the last one perhaps one)
    int64_t n_tokens, n_rows, cache_rows;
    const int64_t* slots;                // NULL: token i goes to row i
    const int32_t* src_row;
    radar_rotation r;
    float sign;
    int* status;
};

// A unit is V elements that a thread moves in one access: 32, 16 or 8 bytes of them, or one element, by what the sizes and
// addresses are multiples of (us with the four: 8192 bf16 rows of 28 / 4 heads of 128 turned 25.1 / 27.3 / 35.1 / 89.3; 8192 tokens of 32 / 8
// heads stored 34.2 / 38.3 / 49.7 / 130; 5329 rows of 16 / 16 heads of 72, which 8 bytes divide, 15.3 and with elements 37.6).
template <typename T, int V>
struct Unit {
    T x[V];
};
template <typename T, int V>
__device__ __forceinline__ Unit<T, V> load_unit(const T* p) {
    Unit<T, V> u;
    if constexpr (sizeof(u) == 32) {
        uint32_t w[8];
        asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
        memcpy(&u, w, sizeof(u));
    } else if constexpr (V > 1) {
        using W = std::conditional_t<sizeof(u) == 16, uint4, uint2>;
        const W w = __ldcs(reinterpret_cast<const W*>(p));
        memcpy(&u, &w, sizeof(u));
    } else {
        u.x[0] = *p;
    }
    return u;
}
template <typename T, int V>
__device__ __forceinline__ void store_unit(T* p, const Unit<T, V>& u) {
    if constexpr (sizeof(u) == 32) {
        uint32_t w[8];
        memcpy(w, &u, sizeof(u));
        asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                     :: "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p) : "memory");
    } else if constexpr (V > 1) {
        using W = std::conditional_t<sizeof(u) == 16, uint4, uint2>;
        W w;
        memcpy(&w, &u, sizeof(u));
        *reinterpret_cast<W*>(p) = w;
    } else {
        *p = u.x[0];
    }
}
__device__ __forceinline__ void from_float(float& y, float x) { y = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }

// cos and sin of pos * f.  The angle in turns, reduced to +- 1/2, is exact to 2^-50: pos * f and its product with 1 / (2 pi) (its double and
// what that lacks) are taken with their remainders.  What fp32 drops of it (up to 2^-25 of a half turn, as much as the functions' own error) is
// put back by the first term of the series: an error of fp32 rows 0.93 times that of cos and sin rounded from fp64, 1.16 without it; of 20.7 million
// bf16 results 266 are not the exact ones rounded, 473 without it; the same times.
__device__ __forceinline__ float2 turn_of(int pos, float f, float sign) {
    constexpr double kInv = 0.15915494309189535, kInvLow = -9.839338337591243e-18;      // 1 / (2 pi)
    const double a = (double)pos * (double)f, a_low = fma((double)pos, (double)f, -a);
    const double t = a * kInv, t_low = fma(a, kInv, -t) + fma(a, kInvLow, a_low * kInv);
    const double part = 2.0 * ((t - rint(t)) + t_low);
    const float near = (float)part, rest = (float)(part - (double)near) * 3.14159265f;
    float s, c;
    sincospif(near, &s, &c);
    return make_float2(fmaf(-s, rest, c), fmaf(c, rest, s) * sign);
}

// A block takes up to R rows of one layer: its threads first load their items of all of these rows (two units of a head that are turned together, or
// copied), then take the rows' angles, one each, into shared memory, then turn and store.  A thread's items stand at the same place in every row,
// so where they lie is worked out once.  Two rows and 4 blocks of 256 threads an SM: 128 bytes a thread in flight (one row and 6 blocks 24.7 /
// 34.3 us for the first two above, but small calls 2.6 instead of 2.3; four rows of 16 bytes 26.1 / 37.4).
// What bounds it: memory.  The two above 5.3 and 5.9 TB/s, 157 accepted tokens in 40 layers of 40 heads 41.7 us, 6.2 TB/s.
template <typename T, int V, int R>
__global__ void __launch_bounds__(kThreads, 4) paged_rows_kernel(const PagedParams P) {
    extern __shared__ __align__(16) float s_angles[];
    chain_wait();
    const int pairs = P.r.n_pairs, layer = blockIdx.y;
    float *s_cos = s_angles, *s_sin = s_angles + R * pairs;
    const int64_t first = (int64_t)blockIdx.x * R;
    const int n = (int)min((int64_t)R, P.n_tokens - first);
    const int turned = P.turn_items + P.rest_items;              // items of a head that is turned
    const int q_items = P.heads[0] * turned, qk_items = q_items + P.heads[1] * turned, row_items = qk_items + P.heads[2] * P.copy_items;
    const int step = gridDim.z * blockDim.x;

    // the rows' places; from < 0: the row is left out
    int64_t from[R], to[R];
    bool bad = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int64_t token = first + r;
        from[r] = r < n ? token : -1;
        to[r] = token;
        bool lost = false;
        if (r < n && P.src_row != nullptr) {
            from[r] = P.src_row[token];
            if (from[r] < 0 || from[r] >= P.n_rows) { lost = true; from[r] = -1; }
        }
        if (r < n && P.slots != nullptr) {
            to[r] = P.slots[token];
            if (to[r] >= P.cache_rows) { bad = true; to[r] = -1; }
        }
        bad |= lost && (to[r] >= 0 || P.heads[0] > 0);       // (behind a slot below 0, where no query goes with it, stands nobody's row)
    }
    if (bad && threadIdx.x == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);

    const T* in;                         // of the thread's item: its head in row 0
    T* out;
    int64_t in_row, out_row;
    int u0, u1, pair;                    // first elements of its units (u1 < 0: it has one), its pairs' number (below 0: copied)
    bool queries;
    Unit<T, V> x[R], y[R];
    auto here = [&](int r) { return from[r] >= 0 && (queries || to[r] >= 0); };
    auto take = [&](int e) {
        const int what = e < q_items ? 0 : e < qk_items ? 1 : 2;
        const int in_part = e - (what == 0 ? 0 : what == 1 ? q_items : qk_items), per = what == 2 ? P.copy_items : turned;
        const int head = in_part / per, item = in_part - head * per;
        queries = what == 0;
        pair = -1;
        if (what < 2 && item < P.turn_items) {
            // (neighbours: a unit of the first and one of the second half of the pairs, so that neighbouring lanes have neighbouring units)
            pair = item;
            const bool lone = V == 1 && P.r.neighbours;
            u0 = lone ? 2 * item : item * V;
            u1 = lone ? u0 + 1 : u0 + pairs;
        } else {
            const int i = what < 2 ? item - P.turn_items : item, items = what < 2 ? P.rest_items : P.copy_items, units = what < 2 ? P.rest_units : P.copy_units;
            u0 = (what < 2 ? 2 * pairs : 0) + i * V;
            u1 = i + items < units ? u0 + items * V : -1;
        }
        in = reinterpret_cast<const T*>(P.in[what]) + layer * P.in_layer[what] + (int64_t)head * P.d;
        out = reinterpret_cast<T*>(P.out[what]) + layer * P.out_layer[what] + (int64_t)head * P.d;
        in_row = P.in_row[what];
        out_row = P.out_row[what];
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (here(r)) {
                x[r] = load_unit<T, V>(in + from[r] * in_row + u0);
                if (u1 >= 0) y[r] = load_unit<T, V>(in + from[r] * in_row + u1);
            }
    };
    auto finish = [&]() {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!here(r)) continue;
            if (pair >= 0) {
                const float *co = s_cos + r * pairs, *si = s_sin + r * pairs;
                if (V > 1 && P.r.neighbours) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        Unit<T, V>& u = h ? y[r] : x[r];
                        const int p = (pair * V + (h ? pairs : 0)) / 2;
#pragma unroll
                        for (int e = 0; e < V / 2; ++e) {
                            const float c = co[p + e], s = si[p + e], a = to_float(u.x[2 * e]), b = to_float(u.x[2 * e + 1]);
                            from_float(u.x[2 * e], fmaf(a, c, -(b * s)));
                            from_float(u.x[2 * e + 1], fmaf(b, c, a * s));
                        }
                    }
                } else {
                    const int p = pair * V;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float c = co[p + e], s = si[p + e], a = to_float(x[r].x[e]), b = to_float(y[r].x[e]);
                        from_float(x[r].x[e], fmaf(a, c, -(b * s)));
                        from_float(y[r].x[e], fmaf(b, c, a * s));
                    }
                }
            }
            T* const at = out + (queries ? first + r : to[r]) * out_row;
            store_unit<T, V>(at + u0, x[r]);
            if (u1 >= 0) store_unit<T, V>(at + u1, y[r]);
        }
    };

    int e = (int)(blockIdx.z * blockDim.x + threadIdx.x);
    if (e < row_items) take(e);
    if (P.r.pos != nullptr) {
        for (int i = threadIdx.x; i < n * pairs; i += blockDim.x) {
            const int r = i / pairs, p = i - r * pairs;
            int axis = P.r.pair_axis != nullptr ? P.r.pair_axis[p] : 0;
            if (axis >= P.r.n_axes) { set_status(P.status, RADAR_ERR_INVALID_ARG); axis = 0; }
            const float2 cs = turn_of(P.r.pos[axis * P.r.pos_stride + first + r], P.r.inv_freq[p], P.sign);
            s_cos[i] = cs.x;
            s_sin[i] = cs.y;
        }
        __syncthreads();
    }
    for (; e < row_items; e += step) {
        finish();
        if (e + step < row_items) take(e + step);
    }
}

bool rotation_ok(const radar_rotation& r, int d, int64_t n) {
    return r.inv_freq != nullptr && r.n_axes >= 1 && r.n_pairs >= 1 && r.n_pairs <= d / 2 && (r.n_axes == 1 || r.pos_stride >= n);
}

int launch(radar_ctx* ctx, PagedParams& P, int dtype, int n_layers, int kernel_id, cudaStream_t stream) {
    const int es = dtype == RADAR_F32 ? 4 : 2;
    if (P.r.pos == nullptr) P.r.n_pairs = 0;
    uint64_t all = (uint64_t)P.d * es | (uint64_t)P.r.n_pairs * es;          // sizes, addresses and strides: the powers of two that divide all of them
    for (int i = 0; i < 3; ++i)
        if (P.heads[i] > 0) {
            all |= reinterpret_cast<uintptr_t>(P.in[i]) | reinterpret_cast<uintptr_t>(P.out[i]) | (uint64_t)(P.in_row[i] | P.out_row[i]) * es;
            if (n_layers > 1) all |= (uint64_t)(P.in_layer[i] | P.out_layer[i]) * es;
        }
    const int bytes = all % 32 == 0 ? 32 : all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : es, unit = bytes / es;
    P.turn_items = P.r.n_pairs / unit;
    P.rest_units = (P.d - 2 * P.r.n_pairs) / unit;
    P.copy_units = P.d / unit;
    P.rest_items = (P.rest_units + 1) / 2;
    P.copy_items = (P.copy_units + 1) / 2;
    P.status = ctx->d_status;
    const int64_t row_items = (int64_t)(P.heads[0] + P.heads[1]) * (P.turn_items + P.rest_items) + (int64_t)P.heads[2] * P.copy_items;
    if (row_items > INT_MAX / 2) return RADAR_ERR_UNSUPPORTED;
    // few rows: one to a block, and a row's items over several blocks, which take the angles each for themselves
    const int64_t wave = 4ll * ctx->sm_count;
    const bool many = (P.n_tokens + kRows - 1) / kRows * n_layers >= wave;
    const int64_t blocks = many ? (P.n_tokens + kRows - 1) / kRows : P.n_tokens;
    const int64_t passes = (row_items + kThreads - 1) / kThreads;
    const int64_t split = std::max<int64_t>(1, std::min(std::min<int64_t>(passes, 64), wave / std::max<int64_t>(1, blocks * n_layers)));
    const int threads = (int)(((row_items + passes - 1) / passes + 31) / 32 * 32);      // the passes' items in equal parts
    if (blocks > INT_MAX) return RADAR_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks, (unsigned)n_layers, (unsigned)split);
    const size_t smem = 2 * (size_t)(many ? kRows : 1) * P.r.n_pairs * sizeof(float);
    auto go = [&](auto kernel) {
        radar_launch_scope scope(ctx, kernel_id, stream);
        return launch_chained(kernel, grid, dim3((unsigned)threads), smem, stream, P);
    };
    auto by_rows = [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value;
        return many ? go(paged_rows_kernel<T, V, kRows>) : go(paged_rows_kernel<T, V, 1>);
    };
    auto by_unit = [&](auto t) {
        constexpr int E = sizeof(t);
        return unit == 1 ? by_rows(t, std::integral_constant<int, 1>{}) : bytes == 8 ? by_rows(t, std::integral_constant<int, 8 / E>{}) :
               bytes == 16 ? by_rows(t, std::integral_constant<int, 16 / E>{}) : by_rows(t, std::integral_constant<int, 32 / E>{});
    };
    RADAR_CUDA_CHECK(dtype == RADAR_F32 ? by_unit(0.f) : by_unit(__nv_bfloat16{}));
    return RADAR_OK;
}

bool misaligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

}  // namespace
}  // namespace radar

using namespace radar;

extern "C" int radar_rotate(radar_ctx* ctx, const radar_rotate_args* a, void* stream_) {
    if (!ctx || !a || a->Hq < 0 || a->Hkv < 0 || a->Hq + (int64_t)a->Hkv == 0 || a->n_rows < 0 || a->d <= 0) return RADAR_ERR_INVALID_ARG;
    if ((a->dtype != RADAR_F32 && a->dtype != RADAR_BF16) || a->d > 2 * kMaxPairs || a->n_rows > INT_MAX) return RADAR_ERR_UNSUPPORTED;
    if (a->n_rows == 0) return RADAR_OK;
    if (!a->rotation.pos || !rotation_ok(a->rotation, a->d, a->n_rows)) return RADAR_ERR_INVALID_ARG;
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
    if (a->n_tokens == 0) return RADAR_OK;
    if (a->rotation.pos && !rotation_ok(a->rotation, a->d, a->n_tokens)) return RADAR_ERR_INVALID_ARG;
    if (!a->src_row && a->n_rows < a->n_tokens) return RADAR_ERR_INVALID_ARG;
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
