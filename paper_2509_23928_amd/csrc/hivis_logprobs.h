// Log probabilities of given tokens, entropy and the most probable tokens of rows of logits.
//   y = x / T;  log p(t) = y_t - log sum exp y;  H = log sum exp y - sum p y.
// All of it relative to the row's maximum: log p(t) = (x_t - max) / T - log z, z = sum e, H = log z - sum e (x - max) / T / z, e = exp((x - max) / T).
//
// One pass over the logits, bound by reading them.  A row is cut into segments, one workgroup each, so that few rows still fill the chip; a segment goes by in
// chunks of 4096 logits, 16 to a thread, that stay in registers: their maximum, then the exponentials relative to the running one.  The most probable
// tokens of a chunk: no lane but the k with the largest own maxima can hold one of a wavefront's k largest, so the k-th of those maxima (and the k-th best so
// far) is a bound that few logits pass; those go to a list in LDS and are ranked by counting.  The workgroup that finishes a row's last segment merges.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hivis {

constexpr int LOGPROBS_MAX_TOP = 32, LOGPROBS_NT = 256, LOGPROBS_PER = 16, LOGPROBS_CHUNK = LOGPROBS_NT * LOGPROBS_PER, LOGPROBS_WGS = 1024;
constexpr int LOGPROBS_LIST = 4 * LOGPROBS_MAX_TOP * LOGPROBS_PER + LOGPROBS_MAX_TOP;       // a chunk's list at most: 16 of each of k lanes of four wavefronts, and the best so far
constexpr int LOGPROBS_STATS = 4;                            // words of a segment's partial before its keys: maximum, z, s, whether it has a NaN

struct LogprobsArgs {
    const void* x; long long ld; int rows, vocab; float inv_temp;
    const int* tokens; int n_tokens; float *logprob, *entropy;
    int top; int* top_ids; float* top_logprobs;
    int chunks, segs; int* cnt; uint32_t* part;              // chunks of a segment; segments of a row, arrivals per row (zero between launches), partials [row][seg][STATS + 2 top]
};

// order of the alternatives as one number: larger logits first, then lower ids; 0 is below all
typedef unsigned long long lp_key;
__device__ inline lp_key lp_key_of(float x, unsigned i) {
    const unsigned u = __float_as_uint(x + 0.f);             // (-0 as 0)
    return (lp_key)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | ~i;
}
__device__ inline float lp_value(lp_key key) {
    const unsigned k = (unsigned)(key >> 32);
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// sums of exponentials relative to m: z = sum e, s = sum e (x - m) / T
struct LpStats {
    float m, z, s;
    __device__ void add(const LpStats& o, float inv_temp) {
        const float to = fmaxf(m, o.m);
        if (to == -INFINITY) return;
        const float da = (m - to) * inv_temp, db = (o.m - to) * inv_temp, fa = m == -INFINITY ? 0.f : __expf(da), fb = o.m == -INFINITY ? 0.f : __expf(db);
        s = (fa > 0.f ? fa * (s + z * da) : 0.f) + (fb > 0.f ? fb * (o.s + o.z * db) : 0.f);
        z = fa * z + fb * o.z;
        m = to;
    }
};

template <int CTRL> __device__ inline float lp_dpp(float x) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false)); }
// over the 64 lanes, the same in all of them
__device__ inline float lp_max(float x) {
    x = fmaxf(x, lp_dpp<0xB1>(x)); x = fmaxf(x, lp_dpp<0x4E>(x)); x = fmaxf(x, lp_dpp<0x141>(x)); x = fmaxf(x, lp_dpp<0x140>(x));      // within rows of 16
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float lp_sum(float x) {
    x += lp_dpp<0xB1>(x); x += lp_dpp<0x4E>(x); x += lp_dpp<0x141>(x); x += lp_dpp<0x140>(x);
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

struct LpShared {
    lp_key list[LOGPROBS_LIST]; lp_key best[LOGPROBS_MAX_TOP]; lp_key lanes[LOGPROBS_NT];
    LpStats wave[4]; int n, nan, last;
};

// Puts the k largest of list[0 .. n) in order into best (all distinct but the zeros).  n: known to all threads.
__device__ inline void lp_rank(LpShared& sh, int n, int k) {
    for (int i = threadIdx.x; i < n; i += LOGPROBS_NT) {
        const lp_key mine = sh.list[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += sh.list[j] > mine;
        if (above < k && mine) sh.best[above] = mine;
    }
}

// Keys of one per lane (0: none) of which a wavefront wants the k largest: the smallest of those, 0 if there are fewer
__device__ inline lp_key lp_bound(LpShared& sh, lp_key mine, int k) {
    lp_key* const w = sh.lanes + (threadIdx.x & ~63u);
    w[threadIdx.x & 63] = mine;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    int above = 0;
    for (int j = 0; j < 64; ++j) above += w[j] > mine;
    const unsigned long long at = __ballot(above == k - 1 && mine != 0);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return at ? w[__builtin_ctzll(at)] : 0;
}

template <typename T> struct LpLoad;
template <> struct LpLoad<float> {
    static constexpr int V = 4;
    static __device__ void get(const float* p, float (&x)[4]) { struct { float v[4]; } t; __builtin_memcpy(&t, p, 16); for (int i = 0; i < 4; ++i) x[i] = t.v[i]; }
};
template <> struct LpLoad<__bf16> {
    static constexpr int V = 8;
    static __device__ void get(const __bf16* p, float (&x)[8]) {
        struct { unsigned v[4]; } t; __builtin_memcpy(&t, p, 16);
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(t.v[i] << 16); x[2 * i + 1] = __uint_as_float(t.v[i] & 0xffff0000u); }
    }
};

template <typename T, bool TOP>
__global__ __launch_bounds__(LOGPROBS_NT) void logprobs_kernel(LogprobsArgs a) {
    constexpr int V = LpLoad<T>::V, N = LOGPROBS_PER / V;
    __shared__ LpShared sh;
    const int seg = blockIdx.x, row = blockIdx.y, t = threadIdx.x, lane = t & 63, wave = t >> 6, k = TOP ? a.top : 0;
    const T* x = (const T*)a.x + (long long)row * a.ld;
    const float nothing = __uint_as_float(0x7fc00000u);
    LpStats st = {-INFINITY, 0.f, 0.f};                      // of this thread
    bool nan = false;
    if (TOP) { if (t < LOGPROBS_MAX_TOP) sh.best[t] = 0; if (t == 0) { sh.n = 0; sh.nan = 0; } __syncthreads(); }
    else { if (t == 0) sh.nan = 0; __syncthreads(); }
    const int first = seg * a.chunks, stop = min(first + a.chunks, (a.vocab + LOGPROBS_CHUNK - 1) / LOGPROBS_CHUNK);
    for (int c = first; c < stop; ++c) {
        const int at = c * LOGPROBS_CHUNK + t * V;           // this thread's: V in a row, LOGPROBS_NT V apart
        float v[LOGPROBS_PER];
        if ((c + 1) * LOGPROBS_CHUNK <= a.vocab) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                float y[V];
                LpLoad<T>::get(x + at + n * LOGPROBS_NT * V, y);
#pragma unroll
                for (int i = 0; i < V; ++i) v[n * V + i] = y[i];
            }
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < V; ++i) { const int id = at + n * LOGPROBS_NT * V + i; v[n * V + i] = id < a.vocab ? (float)x[id] : -INFINITY; }
        }
        float m = v[0];
#pragma unroll
        for (int i = 1; i < LOGPROBS_PER; ++i) m = fmaxf(m, v[i]);
        // relative to the larger of the running maximum and the chunk's; a thread's own, so that no lane waits for another
        const float to = fmaxf(st.m, m);
        if (to > -INFINITY && to < INFINITY) {
            const float d = (st.m - to) * a.inv_temp, f = st.m == -INFINITY ? 0.f : __expf(d);
            float z = f * st.z, s = f > 0.f ? f * (st.s + st.z * d) : 0.f;
#pragma unroll
            for (int i = 0; i < LOGPROBS_PER; ++i) {
                const float y = fmaxf((v[i] - to) * a.inv_temp, -200.f), e = __expf(y);      // (exp(-200) is 0; -inf would make 0 times infinity)
                nan |= v[i] != v[i];
                z += e; s = __builtin_fmaf(e, y, s);
            }
            st = {to, z, s};
        } else {
#pragma unroll
            for (int i = 0; i < LOGPROBS_PER; ++i) nan |= v[i] != v[i];
            st.m = to;
        }
        if constexpr (TOP) {
            // the largest key of this thread; a chunk without one above the k-th best so far changes nothing
            lp_key own = 0;
#pragma unroll
            for (int i = 0; i < LOGPROBS_PER; ++i) {
                const int id = at + (i / V) * LOGPROBS_NT * V + i % V;
                const lp_key key = id < a.vocab ? lp_key_of(v[i], id) : 0;
                own = key > own ? key : own;
            }
            const lp_key least = sh.best[k - 1];
            if (__any(own > least)) {
                lp_key bound = lp_bound(sh, own, k);
                bound = bound > least ? bound : least + 1;
                if (own >= bound) {
#pragma unroll
                    for (int i = 0; i < LOGPROBS_PER; ++i) {
                        const int id = at + (i / V) * LOGPROBS_NT * V + i % V;
                        const lp_key key = id < a.vocab ? lp_key_of(v[i], id) : 0;
                        if (key >= bound) sh.list[atomicAdd(&sh.n, 1)] = key;
                    }
                }
            }
            __syncthreads();
            const int n = sh.n;
            if (n) {
                if (t < k && sh.best[t]) sh.list[atomicAdd(&sh.n, 1)] = sh.best[t];
                __syncthreads();
                const int all = sh.n;
                lp_rank(sh, all, k);
                __syncthreads();
                if (t == 0) sh.n = 0;
            }
            __syncthreads();
        }
    }
    // ---- the segment's sums
    if (__any(nan) && lane == 0) sh.nan = 1;
    const float m = lp_max(st.m);
    if (m > -INFINITY && m < INFINITY) {
        const float d = (st.m - m) * a.inv_temp, f = st.m == -INFINITY ? 0.f : __expf(d);
        st.s = f > 0.f ? f * (st.s + st.z * d) : 0.f; st.z *= f;
    }
    const LpStats w = {m, lp_sum(st.z), lp_sum(st.s)};
    if (lane == 0) sh.wave[wave] = w;
    __syncthreads();
    LpStats sum = sh.wave[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) sum.add(sh.wave[i], a.inv_temp);
    if (a.segs > 1) {
        const int words = LOGPROBS_STATS + 2 * k;
        uint32_t* part = a.part + ((size_t)row * a.segs + seg) * words;
        auto put = [](uint32_t* p, uint32_t v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
        auto get = [](const uint32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
        if (t == 0) { put(part, __float_as_uint(sum.m)); put(part + 1, __float_as_uint(sum.z)); put(part + 2, __float_as_uint(sum.s)); put(part + 3, sh.nan); }
        if (TOP && t < k) { put(part + LOGPROBS_STATS + 2 * t, (uint32_t)sh.best[t]); put(part + LOGPROBS_STATS + 2 * t + 1, (uint32_t)(sh.best[t] >> 32)); }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // acknowledged before the count that shows them
        __syncthreads();
        if (t == 0) sh.last = __hip_atomic_fetch_add(&a.cnt[row], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.segs - 1;
        __syncthreads();
        if (!sh.last) return;
        if (t == 0) __hip_atomic_store(&a.cnt[row], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        part = a.part + (size_t)row * a.segs * words;
        // sums: segments in turn over the threads, then over the threads, in a fixed order
        LpStats mine = {-INFINITY, 0.f, 0.f};
        bool bad = false;
        for (int i = t; i < a.segs; i += LOGPROBS_NT) {
            const uint32_t* p = part + (size_t)i * words;
            const LpStats o = {__uint_as_float(get(p)), __uint_as_float(get(p + 1)), __uint_as_float(get(p + 2))};
            bad |= get(p + 3) != 0 || o.m == INFINITY;
            mine.add(o, a.inv_temp);
        }
        if (TOP && t == 0) sh.n = 0;
        __syncthreads();
        if (__any(bad) && lane == 0) sh.nan = 1;
        for (int d = 1; d < 64; d <<= 1) {
            const LpStats o = {__shfl_xor(mine.m, d), __shfl_xor(mine.z, d), __shfl_xor(mine.s, d)};
            // both partners of a pair add in the same order
            LpStats lo = lane & d ? o : mine; const LpStats hi = lane & d ? mine : o;
            lo.add(hi, a.inv_temp);
            mine = lo;
        }
        if (lane == 0) sh.wave[wave] = mine;
        __syncthreads();
        sum = sh.wave[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) sum.add(sh.wave[i], a.inv_temp);
        if constexpr (TOP) {
            // the keys: rounds of one per thread, each with the bound of its wavefronts
            const int all = a.segs * k;
            for (int i0 = 0; i0 < all; i0 += LOGPROBS_NT) {
                const int i = i0 + t;
                lp_key key = 0;
                if (i < all) { const uint32_t* p = part + (size_t)(i / k) * words + LOGPROBS_STATS + 2 * (i % k); key = get(p) | (lp_key)get(p + 1) << 32; }
                const lp_key least = i0 ? sh.best[k - 1] : 0;
                lp_key bound = lp_bound(sh, key, k);
                bound = bound > least ? bound : least + 1;
                if (key >= bound && key) sh.list[atomicAdd(&sh.n, 1)] = key;
                __syncthreads();
                if (i0 && t < k && sh.best[t]) sh.list[atomicAdd(&sh.n, 1)] = sh.best[t];
                __syncthreads();
                const int n = sh.n;
                lp_rank(sh, n, k);
                __syncthreads();
                if (t == 0) sh.n = 0;
                __syncthreads();
            }
        }
    }
    const bool good = !sh.nan && sum.m > -INFINITY && sum.m < INFINITY;
    const float logz = logf(sum.z);
    if (t == 0 && a.entropy) a.entropy[row] = good ? logz - sum.s / sum.z : nothing;
    for (int j = t; j < a.n_tokens; j += LOGPROBS_NT) {
        const int id = a.tokens[(long long)row * a.n_tokens + j];
        a.logprob[(long long)row * a.n_tokens + j] = good && id >= 0 && id < a.vocab ? ((float)x[id] - sum.m) * a.inv_temp - logz : nothing;
    }
    if (TOP && t < k) {
        a.top_ids[(long long)row * k + t] = good ? (int)~(unsigned)sh.best[t] : -1;
        a.top_logprobs[(long long)row * k + t] = good ? (lp_value(sh.best[t]) - sum.m) * a.inv_temp - logz : nothing;
    }
}

}  // namespace hivis
