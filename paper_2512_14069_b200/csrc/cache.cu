// The 4-bit paged cache beside its attention: pages and slots for new tokens, rows into the cache and out of it.
#include <algorithm>
#include <type_traits>

#include "cache.cuh"

namespace radar {
namespace {

using namespace cache4;

// ---- radar_cache_extend -------------------------------------------------------------------------------------------------
// Three running sums over the requests (tokens added, pages lacked, pages given up) decide everything, and they are short: every
// block works them out for itself in shared memory, and the blocks then share out pages and slots, each of which looks up its
// request in the sums.  The stack as it is after the returns is never read back: an index at or beyond the old count is the
// returned page of some request, looked up in its table.  So no block waits for another one.  What may overwrite the inputs
// (lengths, free count) is written behind all reads: by the only block, or by a second kernel.
constexpr int kExtendThreads = 1024;
constexpr int kMaxRequests = 8192;
constexpr int kSlotsPerThread = 4;

struct ExtendParams {
    radar_cache_extend_args a;
    int shift;                       // log2(page_size), -1: no power of two
    int* status;
};

__device__ __forceinline__ int pages_of(const ExtendParams& P, int tokens) {
    return P.shift >= 0 ? (tokens + P.a.page_size - 1) >> P.shift : (int)((unsigned)(tokens + P.a.page_size - 1) / (unsigned)P.a.page_size);
}

struct Request { int len, n, have, want; bool ok; };
__device__ __forceinline__ Request request(const ExtendParams& P, int b) {
    Request r;
    r.len = P.a.cache_len[b];
    const long long n = (long long)P.a.new_len[b] + P.a.extra, most = min((long long)P.a.max_pages * P.a.page_size, (long long)INT32_MAX - P.a.page_size);
    r.ok = r.len >= 0 && r.len <= most && r.len + n >= 0 && r.len + n <= most;
    r.n = r.ok ? (int)n : 0;
    r.have = r.ok ? pages_of(P, r.len) : 0;
    r.want = r.ok ? pages_of(P, r.len + r.n) : 0;
    return r;
}

// exclusive sum of v over the block's threads, and the total
__device__ __forceinline__ long long block_scan(long long v, long long* s_warp, long long& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(kFull, incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    const long long w = s_warp[lane];                                 // 32 warps
    long long wi = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(kFull, wi, o);
        if (lane >= o) wi += u;
    }
    total = __shfl_sync(kFull, wi, 31);
    const long long before = __shfl_sync(kFull, wi - w, warp);
    __syncthreads();
    return before + incl - v;
}
// Sums are held up to here: behind the largest slot, and more pages than a stack can have.
__device__ __forceinline__ int clip(long long x) { return (int)min(x, (long long)INT32_MAX); }

// the request whose share of the running sum holds i: the last b with sum[b] <= i
__device__ __forceinline__ int owner(const int* sum, int B, int i) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

template <bool ALONE>
__global__ void __launch_bounds__(kExtendThreads) cache_extend_kernel(const ExtendParams P) {
    chain_wait();
    extern __shared__ int s_sums[];                                  // three times B + 1
    __shared__ long long s_warp[32];
    const radar_cache_extend_args& a = P.a;
    const int B = a.B, tid = threadIdx.x;
    int *s_tok = s_sums, *s_grow = s_tok + B + 1, *s_back = s_grow + B + 1;
    const bool first = blockIdx.x == 0;

    // a thread's consecutive requests
    const int per = (B + kExtendThreads - 1) / kExtendThreads, b0 = min(tid * per, B), b1 = min(b0 + per, B);
    long long tok = 0, grow = 0, back = 0, tok_sum, grow_sum, back_sum;
    for (int b = b0; b < b1; ++b) {
        const Request r = request(P, b);
        if (!r.ok && first) set_status(P.status, RADAR_ERR_INVALID_ARG);
        tok += max(r.n, 0); grow += max(r.want - r.have, 0); back += max(r.have - r.want, 0);
    }
    tok = block_scan(tok, s_warp, tok_sum);
    grow = block_scan(grow, s_warp, grow_sum);
    back = block_scan(back, s_warp, back_sum);
    for (int b = b0; b < b1; ++b) {
        const Request r = request(P, b);
        s_tok[b] = clip(tok); s_grow[b] = clip(grow); s_back[b] = clip(back);
        tok += max(r.n, 0); grow += max(r.want - r.have, 0); back += max(r.have - r.want, 0);
    }
    const int tok_all = clip(tok_sum), grow_all = clip(grow_sum);
    int back_all = clip(back_sum);
    if (tid == 0) { s_tok[B] = tok_all; s_grow[B] = grow_all; s_back[B] = back_all; }
    int n0 = *a.free_count;
    if (n0 < 0 || n0 > a.free_capacity) {
        if (first && tid == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
        n0 = max(0, min(n0, a.free_capacity));
    }
    if (back_all > a.free_capacity - n0) {                            // (what does not fit the stack is lost)
        if (first && tid == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
        back_all = a.free_capacity - n0;
    }
    const int n1 = n0 + back_all;
    __syncthreads();

    auto given_up = [&](int i) {                                       // the i-th page that comes back
        const int b = owner(s_back, B, i);
        return a.block_table[(int64_t)b * a.max_pages + request(P, b).want + i - s_back[b]];
    };
    auto taken = [&](int i) {                                          // the i-th page from the top
        const int at = n1 - 1 - i;
        return at < n0 ? a.free_pages[at] : given_up(at - n0);
    };
    auto granted = [&](int b, const Request& r) { return r.want <= r.have || s_grow[b + 1] <= n1; };
    const int step = gridDim.x * kExtendThreads, me = blockIdx.x * kExtendThreads + tid;
    // tokens of ungranted requests still count in `start`; slots beyond the capacity are not written
    if (first) {
        for (int b = tid; b <= B; b += kExtendThreads) {
            a.start[b] = s_tok[b];
            if (b < B) {
                const Request r = request(P, b);
                a.granted[b] = r.ok && granted(b, r);
            }
        }
        if (tok_all > a.slot_capacity && tid == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
    }
    // slots, four consecutive tokens a thread
    const long long tokens = min((long long)tok_all, (long long)a.slot_capacity);
    for (long long i0 = (long long)me * kSlotsPerThread; i0 < tokens; i0 += (long long)step * kSlotsPerThread) {
        int b = -1, end = 0, at = 0, page_at = -1, page = 0, have = 0;
        bool on = false;
        int64_t out[kSlotsPerThread];
#pragma unroll
        for (int k = 0; k < kSlotsPerThread; ++k) {
            const int i = (int)i0 + k;
            out[k] = -1;
            if (i >= tokens) continue;
            if (i >= end) {
                b = owner(s_tok, B, i);
                end = s_tok[b + 1];
                const Request r = request(P, b);
                at = r.len + i - s_tok[b];
                have = r.have;
                on = granted(b, r);
                page_at = -1;
            }
            if (on) {
                const int index = P.shift >= 0 ? at >> P.shift : at / a.page_size;
                if (index != page_at) {
                    page_at = index;
                    page = index < have ? a.block_table[(int64_t)b * a.max_pages + index] : taken(s_grow[b] + index - have);
                }
                out[k] = (int64_t)page * a.page_size + (at - index * a.page_size);
            }
            if (a.path_nodes != nullptr) {
                const int j = i - s_tok[b], row = j < a.path_stride ? a.path_nodes[(int64_t)b * a.path_stride + j] : -1;
                const bool ok = row >= 0 && row < a.rows;
                if (!ok) set_status(P.status, RADAR_ERR_INVALID_ARG);
                a.src_row[i] = ok ? b * a.rows + row : -1;
            }
            ++at;
        }
#pragma unroll
        for (int k = 0; k < kSlotsPerThread; ++k)
            if (i0 + k < tokens) a.slots[i0 + k] = out[k];
    }
    // returned pages onto the stack, new ones into the tables
    for (int i = me; i < back_all; i += step) a.free_pages[n0 + i] = given_up(i);
    for (int i = me; i < grow_all && i < n1; i += step) {
        const int b = owner(s_grow, B, i);
        const Request r = request(P, b);
        if (granted(b, r)) a.block_table[(int64_t)b * a.max_pages + r.have + i - s_grow[b]] = taken(i);
    }
    if (ALONE) {
        __syncthreads();
        long long used = 0, all;
        for (int b = b0; b < b1; ++b) {
            const Request r = request(P, b);
            const bool on = granted(b, r);
            if (on) used += max(r.want - r.have, 0);
            a.cache_len_out[b] = on ? r.len + r.n : r.len;
        }
        block_scan(used, s_warp, all);
        if (tid == 0) *a.free_count_out = n1 - (int)all;
    }
}

// Behind a launch of several blocks: what may overwrite their inputs.
__global__ void __launch_bounds__(kExtendThreads) cache_lengths_kernel(const ExtendParams P) {
    chain_wait();
    __shared__ long long s_warp[32];
    const radar_cache_extend_args& a = P.a;
    long long used = 0, back = 0, used_all, back_all;
    for (int b = threadIdx.x; b < a.B; b += kExtendThreads) {
        const Request r = request(P, b);
        const bool on = a.granted[b];
        if (on) used += max(r.want - r.have, 0);
        back += max(r.have - r.want, 0);
        a.cache_len_out[b] = on ? r.len + r.n : r.len;
    }
    block_scan(used, s_warp, used_all);
    block_scan(back, s_warp, back_all);
    if (threadIdx.x == 0) {
        const int n0 = max(0, min(*a.free_count, a.free_capacity));
        *a.free_count_out = n0 + (int)(min(back_all, (long long)(a.free_capacity - n0)) - used_all);
    }
}

// ---- radar_cache_store --------------------------------------------------------------------------------------------------
struct StoreParams {
    radar_cache_store_args a;
    int64_t page_bytes;
    int shift;
    int* status;
};

__device__ __forceinline__ void load_group(const float* p, float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 t = __ldcs(reinterpret_cast<const float4*>(p) + i);
        x[4 * i] = t.x; x[4 * i + 1] = t.y; x[4 * i + 2] = t.z; x[4 * i + 3] = t.w;
    }
}
__device__ __forceinline__ void load_group(const __nv_bfloat16* p, float (&x)[16]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 t = __ldcs(reinterpret_cast<const uint4*>(p) + i);
        const uint32_t w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[8 * i + 2 * k] = __uint_as_float(w[k] << 16);
            x[8 * i + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    }
}

// A group's codes (two words) and scale byte.
__device__ __forceinline__ uint2 quantise(float (&x)[16], uint32_t& scale, bool& nan) {
    float top = 0.f;
    nan = false;
#pragma unroll
    for (int i = 0; i < 16; ++i) nan |= x[i] != x[i];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (nan && x[i] != x[i]) x[i] = 0.f;
        top = fmaxf(top, fabsf(x[i]));
    }
    const uint32_t bits = __float_as_uint(__fdiv_rn(top, 7.f));
    const int number = (int)((bits + 0x7FFFFu + ((bits >> 20) & 1u)) >> 20) - 107 * 8;
    scale = (uint32_t)max(0, min(number, 255));
    const float s = __uint_as_float((scale + 107 * 8) << 20);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float q = fminf(fmaxf(rintf(__fdiv_rn(x[i], s)), -8.f), 7.f);
        const int c = i & 7, nibble = (c >> 1) + 4 * (c & 1);
        w[i >> 3] |= (uint32_t)((int)q + 8) << (4 * nibble);
    }
    return make_uint2(w[0], w[1]);
}

// One thread takes a group of K and the same of V.
template <typename T, int D>
__global__ void __launch_bounds__(256) cache_store_kernel(const StoreParams P) {
    chain_wait();
    const radar_cache_store_args& a = P.a;
    constexpr int kGroups = D / 16;
    const int per_token = a.Hkv * kGroups;
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t i = item / per_token;
    if (i >= a.n_tokens) return;
    const int u = (int)(item - i * per_token), h = u / kGroups, g = u % kGroups, l = blockIdx.y;
    const int64_t slot = a.slots[i], row = a.src_row != nullptr ? (int64_t)a.src_row[i] : i;
    if (slot < 0) return;
    const int64_t page = P.shift >= 0 ? slot >> P.shift : slot / a.page_size;
    if (page >= a.n_pages || row < 0 || row >= a.n_rows) {
        if (u == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
        return;
    }
    const int in_page = (int)(slot - page * a.page_size), r = in_page & 15;
    unsigned char* block = reinterpret_cast<unsigned char*>(a.pages) + l * a.page_layer_stride + page * P.page_bytes +
                           ((int64_t)h * (a.page_size / kBlock) + (in_page >> 4)) * Layout<D>::kBytes;
    const int64_t from = l * a.row_layer_stride + row * a.row_stride + h * D + g * 16;
    float x[16], y[16];
    load_group(reinterpret_cast<const T*>(a.K) + from, x);
    load_group(reinterpret_cast<const T*>(a.V) + from, y);
    uint32_t sk, sv;
    bool nan_k, nan_v;
    *reinterpret_cast<uint2*>(block + k_codes_at<D>(r, g)) = quantise(x, sk, nan_k);
    *reinterpret_cast<uint2*>(block + v_codes_at<D>(r, g)) = quantise(y, sv, nan_v);
    block[k_scale_at<D>(r, g)] = (unsigned char)sk;
    block[v_scale_at<D>(r, g)] = (unsigned char)sv;
    if (nan_k || nan_v) set_status(P.status, RADAR_ERR_NUMERIC);
}

// ---- radar_cache_load ---------------------------------------------------------------------------------------------------
struct LoadParams {
    radar_cache_load_args a;
    int64_t page_bytes;
    int shift;
    int* status;
};

__device__ __forceinline__ void store_group(float* p, const uint32_t (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        __stcs(reinterpret_cast<float4*>(p) + i, make_float4(__uint_as_float(v[2 * i] << 16), __uint_as_float(v[2 * i] & 0xffff0000u),
                                                             __uint_as_float(v[2 * i + 1] << 16), __uint_as_float(v[2 * i + 1] & 0xffff0000u)));
}
__device__ __forceinline__ void store_group(__nv_bfloat16* p, const uint32_t (&v)[8]) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<uint4*>(p) + 1, make_uint4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void decode_group(uint2 w, uint32_t byte, uint32_t (&v)[8]) {
    const uint32_t s = scale_pair(byte | byte << 16), off = offset_pair(s);
    v[0] = decode<0>(w.x, s, off); v[1] = decode<1>(w.x, s, off); v[2] = decode<2>(w.x, s, off); v[3] = decode<3>(w.x, s, off);
    v[4] = decode<0>(w.y, s, off); v[5] = decode<1>(w.y, s, off); v[6] = decode<2>(w.y, s, off); v[7] = decode<3>(w.y, s, off);
}

template <typename T, int D>
__global__ void __launch_bounds__(256) cache_load_kernel(const LoadParams P) {
    chain_wait();
    const radar_cache_load_args& a = P.a;
    constexpr int kGroups = D / 16;
    const int per_token = a.Hkv * kGroups;
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t i = item / per_token;
    const int64_t n = a.start[a.B];
    if (i >= n || i >= a.n_rows) {
        if (n > a.n_rows && item == a.n_rows * per_token) set_status(P.status, RADAR_ERR_INVALID_ARG);
        return;
    }
    const int u = (int)(item - i * per_token), h = u / kGroups, g = u % kGroups, l = blockIdx.y;
    const int b = owner(a.start, a.B, (int)i);
    const int64_t at = (int64_t)a.first[b] + (i - a.start[b]);
    if (at < 0 || at >= (int64_t)a.max_pages * a.page_size) { if (u == 0) set_status(P.status, RADAR_ERR_INVALID_ARG); return; }
    const int index = P.shift >= 0 ? (int)(at >> P.shift) : (int)(at / a.page_size);
    const int page = a.block_table[(int64_t)b * a.max_pages + index];
    if (page < 0 || page >= a.n_pages) { if (u == 0) set_status(P.status, RADAR_ERR_INVALID_ARG); return; }
    const int in_page = (int)(at - (int64_t)index * a.page_size), r = in_page & 15;
    const unsigned char* block = reinterpret_cast<const unsigned char*>(a.pages) + l * a.page_layer_stride + page * P.page_bytes +
                                 ((int64_t)h * (a.page_size / kBlock) + (in_page >> 4)) * Layout<D>::kBytes;
    const uint2 kc = *reinterpret_cast<const uint2*>(block + k_codes_at<D>(r, g)), vc = *reinterpret_cast<const uint2*>(block + v_codes_at<D>(r, g));
    const uint32_t ks = block[k_scale_at<D>(r, g)], vs = block[v_scale_at<D>(r, g)];
    const int64_t to = l * a.row_layer_stride + (i * a.Hkv + h) * D + g * 16;
    uint32_t v[8];
    decode_group(kc, ks, v);
    store_group(reinterpret_cast<T*>(a.K) + to, v);
    decode_group(vc, vs, v);
    store_group(reinterpret_cast<T*>(a.V) + to, v);
}

int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return (1 << s) == x ? s : -1;
}

template <typename F>
int by_type(int dtype, int d, F f) {
    using d64 = std::integral_constant<int, 64>;
    using d128 = std::integral_constant<int, 128>;
    if (dtype == RADAR_F32) return d == 128 ? f(0.f, d128{}) : f(0.f, d64{});
    return d == 128 ? f(__nv_bfloat16{}, d128{}) : f(__nv_bfloat16{}, d64{});
}

bool misaligned(const void* p, size_t n = 16) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }

}  // namespace
}  // namespace radar

using namespace radar;

extern "C" size_t radar_cache_page_bytes(int Hkv, int d, int page_size) {
    if (Hkv <= 0 || (d != 64 && d != 128) || !page_size_ok(page_size)) return 0;
    return (size_t)page_bytes(Hkv, d, page_size);
}

extern "C" int radar_cache_extend(radar_ctx* ctx, const radar_cache_extend_args* a, void* stream_) {
    if (!ctx || !a || a->B <= 0 || a->max_pages <= 0 || a->free_capacity <= 0 || a->free_capacity == INT32_MAX || a->slot_capacity < 0 || a->slot_capacity > INT32_MAX ||
        !page_size_ok(a->page_size))
        return RADAR_ERR_INVALID_ARG;
    if (!a->cache_len || !a->new_len || !a->block_table || !a->free_pages || !a->free_count || !a->cache_len_out || !a->free_count_out || !a->granted ||
        !a->start || (a->slot_capacity > 0 && !a->slots))
        return RADAR_ERR_INVALID_ARG;
    if (a->path_nodes && ((a->slot_capacity > 0 && !a->src_row) || a->path_stride <= 0 || a->rows <= 0 || (long long)a->B * a->rows > INT32_MAX))
        return RADAR_ERR_INVALID_ARG;
    if (a->B > kMaxRequests) return RADAR_ERR_UNSUPPORTED;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    ExtendParams P;
    P.a = *a;
    P.shift = log2_of(a->page_size);
    P.status = ctx->d_status;
    const size_t smem = 3 * (size_t)(a->B + 1) * sizeof(int);
    const int64_t per = kExtendThreads * kSlotsPerThread;
    const int blocks = (int)std::min<int64_t>(ctx->sm_count, (a->slot_capacity + per - 1) / per);
    if (blocks <= 1) {
        RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, RADAR_SMEM_CACHE_EXTEND, cache_extend_kernel<true>, smem));
        radar_launch_scope scope(ctx, RADAR_K_CACHE_EXTEND, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_extend_kernel<true>, dim3(1), dim3(kExtendThreads), smem, stream, P));
    } else {
        RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, RADAR_SMEM_CACHE_EXTEND + 1, cache_extend_kernel<false>, smem));
        {
            radar_launch_scope scope(ctx, RADAR_K_CACHE_EXTEND, stream);
            RADAR_CUDA_CHECK(launch_chained(cache_extend_kernel<false>, dim3((unsigned)blocks), dim3(kExtendThreads), smem, stream, P));
        }
        radar_launch_scope scope(ctx, RADAR_K_CACHE_LENGTHS, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_lengths_kernel, dim3(1), dim3(kExtendThreads), 0, stream, P));
    }
    RADAR_CUDA_CHECK(cudaGetLastError());
    return RADAR_OK;
}

extern "C" int radar_cache_store(radar_ctx* ctx, const radar_cache_store_args* a, void* stream_) {
    if (!ctx || !a || a->n_layers <= 0 || a->Hkv <= 0 || a->n_tokens < 0 || a->n_rows < 0 || a->n_pages < 0 || !page_size_ok(a->page_size))
        return RADAR_ERR_INVALID_ARG;
    if ((a->d != 64 && a->d != 128) || (a->dtype != RADAR_F32 && a->dtype != RADAR_BF16) || a->n_layers > 65535) return RADAR_ERR_UNSUPPORTED;
    if (a->n_tokens == 0) return RADAR_OK;
    const size_t es = a->dtype == RADAR_F32 ? 4 : 2;
    if (!a->K || !a->V || !a->slots || !a->pages || a->row_stride < (int64_t)a->Hkv * a->d || (a->n_layers > 1 && (a->row_layer_stride <= 0 || a->page_layer_stride <= 0)))
        return RADAR_ERR_INVALID_ARG;
    if (misaligned(a->K) || misaligned(a->V) || misaligned(a->pages) || (a->row_stride * es) % 16 != 0 || (a->row_layer_stride * es) % 16 != 0 ||
        a->page_layer_stride % 16 != 0)
        return RADAR_ERR_INVALID_ARG;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    StoreParams P;
    P.a = *a;
    P.page_bytes = page_bytes(a->Hkv, a->d, a->page_size);
    P.shift = log2_of(a->page_size);
    P.status = ctx->d_status;
    const int64_t items = a->n_tokens * a->Hkv * (a->d / 16), blocks = (items + 255) / 256;
    if (blocks > INT32_MAX) return RADAR_ERR_UNSUPPORTED;
    return by_type(a->dtype, a->d, [&](auto t, auto d) -> int {
        radar_launch_scope scope(ctx, RADAR_K_CACHE_STORE, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_store_kernel<decltype(t), decltype(d)::value>, dim3((unsigned)blocks, (unsigned)a->n_layers), dim3(256), 0, stream, P));
        return RADAR_OK;
    });
}

extern "C" int radar_cache_load(radar_ctx* ctx, const radar_cache_load_args* a, void* stream_) {
    if (!ctx || !a || a->n_layers <= 0 || a->B <= 0 || a->Hkv <= 0 || a->n_rows < 0 || a->n_rows > INT32_MAX || a->n_pages < 0 || a->max_pages <= 0 ||
        !page_size_ok(a->page_size))
        return RADAR_ERR_INVALID_ARG;
    if ((a->d != 64 && a->d != 128) || (a->dtype != RADAR_F32 && a->dtype != RADAR_BF16) || a->n_layers > 65535) return RADAR_ERR_UNSUPPORTED;
    if (a->n_rows == 0) return RADAR_OK;
    const size_t es = a->dtype == RADAR_F32 ? 4 : 2;
    if (!a->K || !a->V || !a->pages || !a->block_table || !a->first || !a->start || (a->n_layers > 1 && (a->row_layer_stride <= 0 || a->page_layer_stride <= 0)))
        return RADAR_ERR_INVALID_ARG;
    if (misaligned(a->K) || misaligned(a->V) || misaligned(a->pages) || (a->row_layer_stride * es) % 16 != 0 || a->page_layer_stride % 16 != 0)
        return RADAR_ERR_INVALID_ARG;
    cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
    LoadParams P;
    P.a = *a;
    P.page_bytes = page_bytes(a->Hkv, a->d, a->page_size);
    P.shift = log2_of(a->page_size);
    P.status = ctx->d_status;
    const int64_t items = a->n_rows * a->Hkv * (a->d / 16) + 1, blocks = (items + 255) / 256;    // (one more: it sees rows that do not fit)
    if (blocks > INT32_MAX) return RADAR_ERR_UNSUPPORTED;
    return by_type(a->dtype, a->d, [&](auto t, auto d) -> int {
        radar_launch_scope scope(ctx, RADAR_K_CACHE_LOAD, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_load_kernel<decltype(t), decltype(d)::value>, dim3((unsigned)blocks, (unsigned)a->n_layers), dim3(256), 0, stream, P));
        return RADAR_OK;
    });
}
