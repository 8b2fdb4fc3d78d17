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
// (lengths, free count) is written behind all reads: by the only block, or by a second kernel where there are several.
// What bounds it is the chain of loads, sums, searches and loads behind one another, not their number: 2.8 us for one request, 3.4 for 32
// that grow by 1 to 9 tokens, 10.9 for 512 admitted with 17 to 4096 tokens (a million slots; a launch that does nothing takes
// 2.2).  The three sums run side by side in 32 bits and each value is loaded once; with three sums of 64 bits behind one another, and four
// consecutive slots a thread, it was 5.7, 7.7 and 14.6 us.
constexpr int kExtendThreads = 1024;
constexpr int kMaxRequests = 8192;
// A warp takes 32 consecutive slots, or this many times 32 where every warp of the grid has some: it then looks up the first and
// the last one's request, and the others' between them.
constexpr int kSlotRuns = 4;
constexpr int kAloneSlots = 4096;        // that one block takes where a second kernel (2.2 us) would have to follow several

struct ExtendParams {
    radar_cache_extend_args a;
    int shift;                       // log2(page_size), -1: no power of two
    bool lengths_here;               // the first block writes lengths and free count
    int* status;
};

__device__ __forceinline__ int pages_of(const ExtendParams& P, int tokens) {
    return P.shift >= 0 ? (tokens + P.a.page_size - 1) >> P.shift : (int)((unsigned)(tokens + P.a.page_size - 1) / (unsigned)P.a.page_size);
}

// add: tokens that it counts in the running sum, also where it is refused (the caller's rows are laid out by new_len, whatever happens
// to a request)
struct Request { int len, n, add, have, want; bool ok; };
__device__ __forceinline__ Request request(const ExtendParams& P, int b) {
    Request r;
    r.len = P.a.cache_len[b];
    const long long n = (long long)P.a.new_len[b] + P.a.extra, most = min((long long)P.a.max_pages * P.a.page_size, (long long)INT32_MAX - P.a.page_size);
    r.ok = r.len >= 0 && r.len <= most && r.len + n >= 0 && r.len + n <= most;
    r.n = r.ok ? (int)n : 0;
    r.add = (int)max(0ll, min(n, (long long)INT32_MAX));
    r.have = r.ok ? pages_of(P, r.len) : 0;
    r.want = r.ok ? pages_of(P, r.len + r.n) : 0;
    return r;
}

// Sums end here: behind the largest slot, and more pages than a stack can have.
__device__ __forceinline__ int add_clipped(int a, int b) { return (int)min((unsigned)a + (unsigned)b, (unsigned)INT32_MAX); }

// what a request adds to the three sums
struct Sums {
    int v[3];                            // tokens, pages lacked, pages given up
    __device__ __forceinline__ explicit Sums(const Request& r) : v{r.add, max(r.want - r.have, 0), max(r.have - r.want, 0)} {}
};

// Exclusive sums over the block's threads, behind `carry`, which the block's own are added to.
__device__ __forceinline__ void block_scan(Sums& x, int (&carry)[3], int (*s_warp)[32]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int incl[3] = {x.v[0], x.v[1], x.v[2]};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int u = __shfl_up_sync(kFull, incl[k], o);
            if (lane >= o) incl[k] = add_clipped(incl[k], u);
        }
    int before[3] = {0, 0, 0}, all[3];
    if (warps == 1) {
#pragma unroll
        for (int k = 0; k < 3; ++k) all[k] = __shfl_sync(kFull, incl[k], 31);
    } else {
        if (lane == 31)
#pragma unroll
            for (int k = 0; k < 3; ++k) s_warp[k][warp] = incl[k];
        __syncthreads();
        int w[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) w[k] = lane < warps ? s_warp[k][lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1)
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const int u = __shfl_up_sync(kFull, w[k], o);
                if (lane >= o) w[k] = add_clipped(w[k], u);
            }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            all[k] = __shfl_sync(kFull, w[k], 31);
            before[k] = __shfl_sync(kFull, w[k], (warp - 1) & 31);
            if (warp == 0) before[k] = 0;
        }
        __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        const int u = __shfl_up_sync(kFull, incl[k], 1);
        x.v[k] = add_clipped(carry[k], add_clipped(before[k], lane > 0 ? u : 0));
        carry[k] = add_clipped(carry[k], all[k]);
    }
}

// the request whose share of the running sum holds i: the last one of b0 .. b1 - 1 with sum[b] <= i
__device__ __forceinline__ int owner(const int* sum, int b0, int b1, int i) {
    while (b1 - b0 > 1) {
        const int mid = (b0 + b1) >> 1;
        if (sum[mid] <= i) b0 = mid; else b1 = mid;
    }
    return b0;
}

template <int RUNS>
__global__ void __launch_bounds__(kExtendThreads) cache_extend_kernel(const ExtendParams P) {
    chain_wait();
    extern __shared__ int s_sums[];                                  // three times B + 1
    __shared__ int s_warp[3][32];
    const radar_cache_extend_args& a = P.a;
    const int B = a.B, tid = threadIdx.x, threads = blockDim.x;
    int *s_tok = s_sums, *s_grow = s_tok + B + 1, *s_back = s_grow + B + 1;
    const bool first = blockIdx.x == 0;
    int n0 = *a.free_count;

    int sum[3] = {0, 0, 0};
    for (int b0 = 0; b0 < B; b0 += threads) {
        const int b = b0 + tid;
        Request r = {0, 0, 0, 0, 0, true};
        if (b < B) r = request(P, b);
        if (!r.ok && first) set_status(P.status, RADAR_ERR_INVALID_ARG);
        Sums x(r);
        block_scan(x, sum, s_warp);
        if (b < B) { s_tok[b] = x.v[0]; s_grow[b] = x.v[1]; s_back[b] = x.v[2]; }
    }
    const int tok_all = sum[0], grow_all = sum[1];
    int back_all = sum[2];
    if (tid == 0) { s_tok[B] = tok_all; s_grow[B] = grow_all; s_back[B] = back_all; }
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
        const int b = owner(s_back, 0, B, i);
        return a.block_table[(int64_t)b * a.max_pages + request(P, b).want + i - s_back[b]];
    };
    auto taken = [&](int i) {                                          // the i-th page from the top
        const int at = n1 - 1 - i;
        return at < n0 ? a.free_pages[at] : given_up(at - n0);
    };
    // Pages and slots go to requests in order as long as there are enough: both sums only grow, so one request is the first that gets none.
    // (A sum that ended at the largest int has no slots.)
    const int room = (int)min(a.slot_capacity, (int64_t)INT32_MAX - 1);
    auto granted = [&](int b, const Request& r) { return r.ok && (r.n <= 0 || (s_tok[b + 1] <= room && (r.want <= r.have || s_grow[b + 1] <= n1))); };
    // tokens of requests that are not granted still count in `start`; slots beyond the capacity are not written
    const int64_t tokens = min((int64_t)tok_all, a.slot_capacity);
    const int lane = tid & 31, warps = threads >> 5;
    constexpr int kRun = 32 * RUNS;
    for (int64_t i0 = ((int64_t)blockIdx.x * warps + (tid >> 5)) * kRun; i0 < tokens; i0 += (int64_t)gridDim.x * warps * kRun) {
        int lo = 0, hi = B;
        if (RUNS > 1) {
            lo = owner(s_tok, 0, B, (int)i0);
            hi = owner(s_tok, 0, B, (int)min(i0 + kRun, tokens) - 1) + 1;
        }
        int b = -1, end = 0, tok = 0, grow = 0;                        // the request looked up last, if any, and its last slot's successor
        Request r;
        bool on = false;
#pragma unroll
        for (int k = 0; k < RUNS; ++k) {
            const int64_t i = i0 + 32 * k + lane;
            if (i >= tokens) continue;
            if (i >= end) {
                b = owner(s_tok, lo, hi, (int)i);
                tok = s_tok[b]; grow = s_grow[b]; end = s_tok[b + 1];
                r = request(P, b);
                on = granted(b, r);
            }
            const int j = (int)i - tok;
            if (a.path_nodes != nullptr) {
                const int row = j < a.path_stride ? a.path_nodes[(int64_t)b * a.path_stride + j] : -1;
                const bool ok = row >= 0 && row < a.rows;
                if (!ok) set_status(P.status, RADAR_ERR_INVALID_ARG);
                a.src_row[i] = ok ? b * a.rows + row : -1;
            }
            int64_t slot = -1;
            if (on) {
                const int at = r.len + j, index = P.shift >= 0 ? at >> P.shift : at / a.page_size;
                const int page = index < r.have ? a.block_table[(int64_t)b * a.max_pages + index] : taken(grow + index - r.have);
                slot = (int64_t)page * a.page_size + (at - index * a.page_size);
            }
            a.slots[i] = slot;
        }
    }
    // no slots behind the last token: whoever stores as many rows as there are slots stores nothing there
    const int step = gridDim.x * threads, me = blockIdx.x * threads + tid;
    for (int64_t i = tokens + me; i < a.slot_capacity; i += step) a.slots[i] = -1;
    // returned pages onto the stack, new ones into the tables
    for (int i = me; i < back_all; i += step) a.free_pages[n0 + i] = given_up(i);
    for (int i = me; i < grow_all && i < n1; i += step) {
        const int b = owner(s_grow, 0, B, i);
        const Request r = request(P, b);
        if (granted(b, r)) a.block_table[(int64_t)b * a.max_pages + r.have + i - s_grow[b]] = taken(i);
    }
    if (!first) return;
    if (tok_all > a.slot_capacity && tid == 0) set_status(P.status, RADAR_ERR_INVALID_ARG);
    if (P.lengths_here) __syncthreads();
    for (int b = tid; b <= B; b += threads) {
        a.start[b] = s_tok[b];
        // the pages of the requests before the first one that gets none are used up
        const bool before = s_grow[b] <= n1 && s_tok[b] <= room;
        if (P.lengths_here && before && (b == B || s_grow[b + 1] > n1 || s_tok[b + 1] > room)) *a.free_count_out = n1 - s_grow[b];
        if (b == B) break;
        const Request r = request(P, b);
        const bool on = granted(b, r);
        a.granted[b] = on;
        if (P.lengths_here) a.cache_len_out[b] = on ? r.len + r.n : r.len;
    }
}

// Behind a launch of several blocks: what overwrites their inputs.
__global__ void __launch_bounds__(kExtendThreads) cache_lengths_kernel(const ExtendParams P) {
    chain_wait();
    __shared__ int s_warp[3][32];
    const radar_cache_extend_args& a = P.a;
    int sum[3] = {0, 0, 0};
    for (int b0 = 0; b0 < a.B; b0 += kExtendThreads) {
        const int b = b0 + threadIdx.x;
        Request r = {0, 0, 0, 0, 0, true};
        if (b < a.B) r = request(P, b);
        Sums x(r);
        if (b < a.B) {
            const bool on = a.granted[b];
            if (!on) x.v[1] = 0;                                       // (ungranted ones take none)
            a.cache_len_out[b] = on ? r.len + r.n : r.len;
        }
        block_scan(x, sum, s_warp);
    }
    if (threadIdx.x == 0) {
        const int n0 = max(0, min(*a.free_count, a.free_capacity));
        *a.free_count_out = n0 + min(sum[2], a.free_capacity - n0) - sum[1];
    }
}

// ---- radar_cache_store and radar_cache_load -----------------------------------------------------------------------------
// A lane takes 16 channels of a token's K and V: a warp one KV head of 32 / (d / 16) consecutive tokens.  Each lane looks up for itself
// where its token lies (the token's lanes share the loads), and nothing passes between lanes.
template <int D>
struct Lanes {
    static constexpr int kGroups = D / 16, kTokens = 32 / kGroups;       // lanes of a token, and tokens of a warp
};

struct StoreParams {
    radar_cache_store_args a;
    int64_t page_bytes;
    int64_t warps;                   // of one KV head
    int shift;
    int* status;
};

// Rows are read and written once.  A lane's 32 bytes go in one access of 256 bits: in two of 128 bits each takes half of every
// sector that the warp touches.  Rows that are only 16-byte aligned take the two.
__device__ __forceinline__ bool wide(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; }
__device__ __forceinline__ void load_row32(const void* p, uint4& a, uint4& b) {
    if (wide(p)) {
        asm volatile("ld.global.cs.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "l"(p));
    } else {
        a = __ldcs(reinterpret_cast<const uint4*>(p));
        b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
    }
}
__device__ __forceinline__ void store_row32(void* p, const uint4& a, const uint4& b) {
    if (wide(p)) {
        asm volatile("st.global.cs.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                     :: "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w), "l"(p) : "memory");
    } else {
        __stcs(reinterpret_cast<uint4*>(p), a);
        __stcs(reinterpret_cast<uint4*>(p) + 1, b);
    }
}

// 16 channels as they are loaded
template <typename T>
struct Group {
    uint4 w[sizeof(T)];                                                  // two of bf16, four of fp32
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); i += 2) load_row32(p + i * 16 / (int)sizeof(T), w[i], w[i + 1]);
    }
    __device__ __forceinline__ uint32_t word(int i) const { return (&w[i >> 2].x)[i & 3]; }
    __device__ __forceinline__ float value(int c) const {
        if (sizeof(T) == 4) return __uint_as_float(word(c));
        return __uint_as_float((c & 1) ? word(c >> 1) & 0xffff0000u : word(c >> 1) << 16);
    }
    // the largest magnitude, its bits as those of a float32: an infinity or a NaN is the largest
    __device__ __forceinline__ uint32_t top() const {
        if (sizeof(T) == 4) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) m = max(m, word(i) & 0x7fffffffu);
            return m;
        }
        uint32_t m = word(0) & 0x7fff7fffu;                              // two bf16 side by side
#pragma unroll
        for (int i = 1; i < 7; i += 2) m = __vimax3_u16x2(m, word(i) & 0x7fff7fffu, word(i + 1) & 0x7fff7fffu);
        m = __vmaxu2(m, word(7) & 0x7fff7fffu);
        return max(m << 16, m & 0xffff0000u);
    }
};

// A group's codes (two words) and scale byte.  Ties go to even, so x / s has to come out exact where it lies in the middle between
// two codes; y = 1 / s rounded is off by up to 2^-24 of itself.
// fp32: the quotient rounded to fp32, by one step of Markstein's correction (P. Markstein, "Computation of elementary functions
// on the IBM RISC System/6000 processor", 1990): with q = x y, the remainder x - q s is exact in a fused multiply-add and
// q + (x - q s) y rounds to the quotient.
// bf16: with integers V < 2^8 and 8 <= S < 16, x / s is V 2^k / S, and (for |x / s| >= 1 / 4, so 2^k >= 2^-7) off the nearest
// middle by nothing or by 2^-7 / 30 at least.  x y + 384, rounded once, is a multiple of 2^-15, off by 2^-16 + 8 2^-24: what lies in a
// middle comes out there, what does not stays on its side.  That takes half the instructions, which bound this kernel.
// Adding 1.5 2^23 + 8 rounds it to an integer (to even), whose low bits are the code; |x / s| is below 7.5, as s is at least 16 / 17
// of max / 7, but for scales at the end of their range and for values that are no numbers, which take the other branch.
__device__ __forceinline__ int scale_number(float top) {                 // not yet within 0 .. 255
    const uint32_t bits = __float_as_uint(__fdiv_rn(top, 7.f));
    return (int)((bits + 0x7FFFFu + ((bits >> 20) & 1u)) >> 20) - 107 * 8;
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float((byte + 107 * 8) << 20); }

// two fp32 operations an instruction
__device__ __forceinline__ uint64_t both(float2 a) { return (uint64_t)__float_as_uint(a.y) << 32 | __float_as_uint(a.x); }
__device__ __forceinline__ float2 parts(uint64_t a) { return make_float2(__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)(a >> 32))); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(both(a)), "l"(both(b)), "l"(both(c)));
    return parts(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(both(a)), "l"(both(b)));
    return parts(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(both(a)), "l"(both(b)));
    return parts(r);
}

template <typename T>
__device__ __forceinline__ uint2 quantise(const Group<T>& x, uint32_t& scale, bool& nan) {
    const int number = scale_number(__uint_as_float(x.top()));
    uint32_t w[2] = {0, 0};
    if (number <= 255) {
        scale = (uint32_t)max(0, number);
        const float s = scale_value(scale), y = __frcp_rn(s);
        const float2 y2 = make_float2(y, y), s2 = make_float2(-s, -s);
        constexpr float kRound = 12582912.f + 8.f, kCoarse = sizeof(T) == 2 ? 384.f : 0.f;
        const float2 coarse = make_float2(kCoarse, kCoarse), round = make_float2(kRound - kCoarse, kRound - kCoarse);
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float2 v = make_float2(x.value(i), x.value(i + 1));
            float2 q;
            if (sizeof(T) == 4) {
                q = mul2(v, y2);
                q = fma2(fma2(q, s2, v), y2, q);
            } else {
                q = fma2(v, y2, coarse);
            }
            const float2 t = add2(q, round);
            // even channels' codes lie in the low half word, odd ones' in the high one
            w[i >> 3] += __byte_perm(__float_as_uint(t.x), __float_as_uint(t.y), 0x5410) << (2 * (i & 7));
        }
    } else {                                                             // saturated, infinite or NaN
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x.value(i)));        // (of the numbers among them)
        scale = (uint32_t)max(0, min(scale_number(top), 255));
        const float s = scale_value(scale);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float v = x.value(i), q = v != v ? 0.f : fminf(fmaxf(rintf(__fdiv_rn(v, s)), -8.f), 7.f);
            nan |= v != v;
            const int c = i & 7, nibble = (c >> 1) + 4 * (c & 1);
            w[i >> 3] |= (uint32_t)((int)q + 8) << (4 * nibble);
        }
    }
    return make_uint2(w[0], w[1]);
}

// What bounds it: memory where there is much to store (8 KV heads of 128 channels, 32 layers, 2048 tokens of bf16: 53 us, 6.5 TB/s;
// fp32 90 us, 6.8 TB/s), else a lookup, a load and a launch behind one another.  bf16: 32 registers a thread for 64 warps an SM (with 48 warps
// 66 us; two or four tokens a lane in flight took 60 to 108).  fp32 has twice the bytes in flight a lane, and small calls took 3.6 us
// instead of 3.2 when held to as few registers.
template <typename T, int D>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 8 : 4) cache_store_kernel(const StoreParams P) {
    chain_wait();
    using L = Lanes<D>;
    const radar_cache_store_args& a = P.a;
    const int lane = threadIdx.x & 31, g = lane % L::kGroups, l = blockIdx.y;
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), warp = item / a.Hkv;
    if (warp >= P.warps) return;
    const int h = (int)(item - warp * a.Hkv);
    const int64_t i = warp * L::kTokens + lane / L::kGroups;
    if (i >= a.n_tokens) return;
    const int64_t slot = a.slots[i], row = a.src_row != nullptr ? (int64_t)a.src_row[i] : i;
    if (slot < 0) return;
    const int64_t page = P.shift >= 0 ? slot >> P.shift : slot / a.page_size;
    if (page >= a.n_pages || row < 0 || row >= a.n_rows) {
        set_status(P.status, RADAR_ERR_INVALID_ARG);
        return;
    }
    const int in_page = (int)(slot - page * a.page_size), r = in_page & 15;
    unsigned char* block = reinterpret_cast<unsigned char*>(a.pages) + l * a.page_layer_stride + page * P.page_bytes +
                           ((int64_t)h * (a.page_size / kBlock) + (in_page >> 4)) * Layout<D>::kBytes;
    const int64_t from = l * a.row_layer_stride + row * a.row_stride + h * D + g * 16;
    Group<T> x[2];
    x[0].load(reinterpret_cast<const T*>(a.K) + from);
    x[1].load(reinterpret_cast<const T*>(a.V) + from);
    bool nan = false;
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        uint32_t scale;
        const uint2 codes = quantise(x[v], scale, nan);
        *reinterpret_cast<uint2*>(block + (v ? v_codes_at<D>(r, g) : k_codes_at<D>(r, g))) = codes;
        block[v ? v_scale_at<D>(r, g) : k_scale_at<D>(r, g)] = (unsigned char)scale;
    }
    if (nan) set_status(P.status, RADAR_ERR_NUMERIC);
}

struct LoadParams {
    radar_cache_load_args a;
    int64_t page_bytes;
    int64_t warps;                   // of one KV head
    int shift;
    int* status;
};

__device__ __forceinline__ void store_group(float* p, const uint32_t (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
        store_row32(p + 8 * i, make_uint4(v[4 * i] << 16, v[4 * i] & 0xffff0000u, v[4 * i + 1] << 16, v[4 * i + 1] & 0xffff0000u),
                    make_uint4(v[4 * i + 2] << 16, v[4 * i + 2] & 0xffff0000u, v[4 * i + 3] << 16, v[4 * i + 3] & 0xffff0000u));
}
__device__ __forceinline__ void store_group(__nv_bfloat16* p, const uint32_t (&v)[8]) {
    store_row32(p, make_uint4(v[0], v[1], v[2], v[3]), make_uint4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void decode_group(uint2 w, uint32_t byte, uint32_t (&v)[8]) {
    const uint32_t s = scale_pair(byte | byte << 16), off = offset_pair(s);
    v[0] = decode<0>(w.x, s, off); v[1] = decode<1>(w.x, s, off); v[2] = decode<2>(w.x, s, off); v[3] = decode<3>(w.x, s, off);
    v[4] = decode<0>(w.y, s, off); v[5] = decode<1>(w.y, s, off); v[6] = decode<2>(w.y, s, off); v[7] = decode<3>(w.y, s, off);
}

// What bounds it: memory (the sizes above: bf16 55 us, 6.2 TB/s; fp32 95 us, 6.4 TB/s).
template <typename T, int D>
__global__ void __launch_bounds__(256) cache_load_kernel(const LoadParams P) {
    chain_wait();
    using L = Lanes<D>;
    const radar_cache_load_args& a = P.a;
    const int lane = threadIdx.x & 31, g = lane % L::kGroups, l = blockIdx.y;
    const int64_t item = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), warp = item / a.Hkv;
    if (warp >= P.warps) return;
    const int h = (int)(item - warp * a.Hkv);
    const int64_t i = warp * L::kTokens + lane / L::kGroups;
    const int n = a.start[a.B];
    if (i >= n) return;
    if (i >= a.n_rows) {
        set_status(P.status, RADAR_ERR_INVALID_ARG);
        return;
    }
    const int b = owner(a.start, 0, a.B, (int)i);
    const int64_t at = (int64_t)a.first[b] + (i - a.start[b]);
    const int index = P.shift >= 0 ? (int)(at >> P.shift) : (int)(at / a.page_size);
    const bool in_table = at >= 0 && at < (int64_t)a.max_pages * a.page_size;
    const int page = in_table ? a.block_table[(int64_t)b * a.max_pages + index] : -1;
    if (page < 0 || page >= a.n_pages) {
        set_status(P.status, RADAR_ERR_INVALID_ARG);
        return;
    }
    const int in_page = (int)(at - (int64_t)index * a.page_size), r = in_page & 15;
    const unsigned char* block = reinterpret_cast<const unsigned char*>(a.pages) + l * a.page_layer_stride + page * P.page_bytes +
                                 ((int64_t)h * (a.page_size / kBlock) + (in_page >> 4)) * Layout<D>::kBytes;
    const uint2 k = *reinterpret_cast<const uint2*>(block + k_codes_at<D>(r, g)), v = *reinterpret_cast<const uint2*>(block + v_codes_at<D>(r, g));
    const uint32_t k_scale = block[k_scale_at<D>(r, g)], v_scale = block[v_scale_at<D>(r, g)];
    const int64_t to = l * a.row_layer_stride + (i * a.Hkv + h) * D + g * 16;
    uint32_t out[8];
    decode_group(k, k_scale, out);
    store_group(reinterpret_cast<T*>(a.K) + to, out);
    decode_group(v, v_scale, out);
    store_group(reinterpret_cast<T*>(a.V) + to, out);
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
    auto overlap = [](const void* p, const void* q, size_t n) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(p), y = reinterpret_cast<uintptr_t>(q);
        return x < y + n && y < x + n;
    };
    const size_t lens = (size_t)a->B * sizeof(int32_t);
    const bool in_place = overlap(a->cache_len, a->cache_len_out, lens) || overlap(a->free_count, a->free_count_out, sizeof(int32_t)) ||
                          overlap(a->new_len, a->cache_len_out, lens);
    int64_t blocks = std::min<int64_t>(ctx->sm_count, (a->slot_capacity + kExtendThreads - 1) / kExtendThreads);
    if (blocks < 1 || (in_place && a->slot_capacity <= kAloneSlots)) blocks = 1;
    const bool runs = a->slot_capacity >= blocks * kExtendThreads * kSlotRuns;
    const int64_t work = std::max<int64_t>(a->B, a->slot_capacity);
    const int threads = blocks > 1 ? kExtendThreads : (int)std::min<int64_t>(kExtendThreads, (work + 31) / 32 * 32);
    P.lengths_here = blocks == 1 || !in_place;
    auto* const kernel = runs ? cache_extend_kernel<kSlotRuns> : cache_extend_kernel<1>;
    RADAR_CUDA_CHECK(radar_opt_in_smem(ctx, RADAR_SMEM_CACHE_EXTEND + runs, kernel, smem));
    {
        radar_launch_scope scope(ctx, RADAR_K_CACHE_EXTEND, stream);
        RADAR_CUDA_CHECK(launch_chained(kernel, dim3((unsigned)blocks), dim3((unsigned)threads), smem, stream, P));
    }
    if (!P.lengths_here) {
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
    const int tokens = 32 / (a->d / 16);
    P.warps = (a->n_tokens + tokens - 1) / tokens;
    const int64_t blocks = (P.warps * a->Hkv + 7) / 8;
    if (blocks > INT32_MAX || a->n_rows > INT32_MAX) return RADAR_ERR_UNSUPPORTED;
    return by_type(a->dtype, a->d, [&](auto t, auto d) -> int {
        constexpr int D = decltype(d)::value;
        radar_launch_scope scope(ctx, RADAR_K_CACHE_STORE, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_store_kernel<decltype(t), D>, dim3((unsigned)blocks, (unsigned)a->n_layers), dim3(256), 0, stream, P));
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
    const int tokens = 32 / (a->d / 16);
    P.warps = (a->n_rows + 1 + tokens - 1) / tokens;             // (one token more: it sees rows that do not fit)
    const int64_t blocks = (P.warps * a->Hkv + 7) / 8;
    if (blocks > INT32_MAX) return RADAR_ERR_UNSUPPORTED;
    return by_type(a->dtype, a->d, [&](auto t, auto d) -> int {
        constexpr int D = decltype(d)::value;
        radar_launch_scope scope(ctx, RADAR_K_CACHE_LOAD, stream);
        RADAR_CUDA_CHECK(launch_chained(cache_load_kernel<decltype(t), D>, dim3((unsigned)blocks, (unsigned)a->n_layers), dim3(256), 0, stream, P));
        return RADAR_OK;
    });
}
