// Log probabilities of given tokens, entropy and the most probable tokens of rows of logits.
//   y = x / T;  log p(t) = y_t - log sum exp y;  H = log sum exp y - sum p y.
// All of it relative to the row's maximum: log p(t) = (x_t - max) / T - log z, z = sum e, H = log z - sum e (x - max) / T / z, e = exp((x - max) / T).
//
// One pass over the logits, bound by reading them.  A row is cut into segments, one workgroup each, so that few rows still fill the chip; a segment goes by in
// chunks of 16 logits per thread: their maximum, then the exponentials relative to the thread's running one.
// The most probable tokens: only the k threads of a wavefront with the largest own maxima can hold one of its k largest, so the k-th of those maxima is a bound
// that a few dozen of a segment's logits pass.  The threads with a maximum above it are listed, and what they had read (a few hundred pieces of 16 bytes, still in
// a cache) is read again by all threads at once for the logits themselves, which are ranked by counting.  (Selecting chunk by chunk, in registers, cost more
// than the pass: 128 rows of 152064, top 20, 41 us, and 51 with a barrier per chunk.)  Where too many are equal to the bound (a row that is mostly one value):
// k rounds of maxima, each thread with its own next one.  The workgroup that finishes a row's last segment merges.
#pragma once
#include "hivis_logprobs_args.h"

namespace hivis {

constexpr int LOGPROBS_NT = 256, LOGPROBS_PER = 16, LOGPROBS_CHUNK = LOGPROBS_NT * LOGPROBS_PER, LOGPROBS_WGS = 1024;
constexpr int LOGPROBS_LIST = 512;                           // keys ranked together, at most
constexpr int LOGPROBS_AHEAD = 4;                            // keys of the segments that a thread of the merging workgroup takes at a time
constexpr int LOGPROBS_STATS = 4;                            // words of a segment's partial before its keys: maximum, z, s, whether it has a NaN

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
    alignas(16) lp_key list[LOGPROBS_LIST + LOGPROBS_MAX_TOP + 8];         // (beside the best so far, with the padding of lp_rank)
    lp_key best[LOGPROBS_MAX_TOP]; alignas(16) lp_key lanes[LOGPROBS_NT];
    int who[LOGPROBS_NT], n, n_who, nan, last;
    LpStats wave[4]; lp_key bound[4];
};

// Puts the k largest of list[0 .. n) in order into best (all distinct but zeros, which are left out).  All threads, in step before and after.
__device__ inline void lp_rank(LpShared& sh, int n, int k) {
    if (threadIdx.x < 8) sh.list[n + threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += LOGPROBS_NT) {
        const lp_key mine = sh.list[i];
        int above = 0;
        for (int j = 0; j < n; j += 8) {
            lp_key o[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) o[u] = sh.list[j + u];
#pragma unroll
            for (int u = 0; u < 8; ++u) above += o[u] > mine;
        }
        if (above < k && mine) sh.best[above] = mine;
    }
    __syncthreads();
}

// The k-th largest of one number per lane (k <= 64): values, or keys (0: the lane has none; 0 if there are fewer than k)
template <typename X>
__device__ inline X lp_bound(X* w, X mine, int k, int lane) {
    w[lane] = mine;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // (a wavefront's LDS accesses are in order)
    int above = 0;
#pragma unroll 2
    for (int j = 0; j < 64; j += 8) {
        X o[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) o[u] = w[j + u];
#pragma unroll
        for (int u = 0; u < 8; ++u) above += o[u] > mine || (o[u] == mine && j + u < lane);
    }
    const unsigned long long at = __ballot(above == k - 1);
    return at ? w[__builtin_ctzll(at)] : (X)0;                // (none: a NaN among them, and the row has no result anyway)
}
// the largest key of the workgroup, the same for all threads
__device__ inline lp_key lp_largest(LpShared& sh, lp_key x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const lp_key o = __shfl_xor(x, d); x = o > x ? o : x; }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.bound[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) x = sh.bound[w] > x ? sh.bound[w] : x;
    return x;
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
__global__ __launch_bounds__(LOGPROBS_NT, 8) void logprobs_kernel(LogprobsArgs a) {
    constexpr int V = LpLoad<T>::V, PER = LOGPROBS_PER, N = PER / V, CHUNK = LOGPROBS_CHUNK;
    __shared__ LpShared sh;
    const int seg = blockIdx.x, row = blockIdx.y, t = threadIdx.x, lane = t & 63, wave = t >> 6, k = TOP ? a.top : 0;
    const T* x = (const T*)a.x + (long long)row * a.ld;
    const float nothing = __uint_as_float(0x7fc00000u);
    LpStats st = {-INFINITY, 0.f, 0.f};                      // of this thread; its largest logit is st.m
    bool nan = false;
    if (t == 0) { sh.nan = 0; sh.n = 0; sh.n_who = 0; }
    if (TOP && t < LOGPROBS_MAX_TOP) sh.best[t] = 0;
    // this thread's given token (those beyond the threads: at the end)
    int given = -1;
    float given_x = 0.f;
    if (t < a.n_tokens) { given = a.tokens[(long long)row * a.n_tokens + t]; if (given >= 0 && given < a.vocab) given_x = (float)x[given]; else given = -1; }
    __syncthreads();
    const int first = seg * a.chunks, stop = min(first + a.chunks, (a.vocab - 1) / CHUNK + 1);
    for (int c = first; c < stop; ++c) {
        const int at = c * CHUNK + t * V;                    // V logits in a row per thread, LOGPROBS_NT V apart
        float v[PER];
        if (c < a.vocab / CHUNK) {
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
        for (int i = 1; i < PER; ++i) m = fmaxf(m, v[i]);
        // relative to the larger of the running maximum and the chunk's; a thread's own, so that no lane waits for another
        const float to = fmaxf(st.m, m);
        if (to > -INFINITY && to < INFINITY) {
            const float d = (st.m - to) * a.inv_temp, f = st.m == -INFINITY ? 0.f : __expf(d);
            float z = f * st.z, s = f > 0.f ? f * (st.s + st.z * d) : 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const float y = fmaxf((v[i] - to) * a.inv_temp, -200.f), e = __expf(y);      // (exp(-200) is 0; -inf would make 0 times infinity)
                nan |= v[i] != v[i];
                z += e; s = __builtin_fmaf(e, y, s);
            }
            st = {to, z, s};
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) nan |= v[i] != v[i];
            st.m = to;
        }
    }
    if constexpr (TOP) {
        // bound: the best of the wavefronts' own
        const float own = st.m, mine = lp_bound((float*)(sh.lanes + 64 * wave), own, k, lane);
        if (lane == 0) sh.wave[wave].m = mine;
        __syncthreads();
        float bound = fmaxf(fmaxf(sh.wave[0].m, sh.wave[1].m), fmaxf(sh.wave[2].m, sh.wave[3].m));
        float* const tops = (float*)sh.lanes;
        auto enlist = [&] { if (own >= bound) { const int at = atomicAdd(&sh.n_who, 1); sh.who[at] = t; tops[at] = own; } };
        enlist();
        __syncthreads();
        int listed = sh.n_who;
        const int pieces = (stop - first) * N;
        // The k-th of the threads listed is the k-th of all: where that spares more than two pieces per thread (128 rows of 152064, top 20: 34.3 -> 30.4 us; 48 rows, whose
        // segments are shorter, 22.6 -> 24.1, and with top 5 24.1 -> 24.7)
        if ((listed - k) * pieces > 2 * LOGPROBS_NT) {
            if (t < listed) {
                const float x = tops[t];
                int above = 0;
#pragma unroll 8
                for (int j = 0; j < listed; ++j) above += tops[j] > x || (tops[j] == x && j < t);
                if (above == k - 1) sh.wave[0].m = x;
            }
            __syncthreads();
            if (t == 0) sh.n_who = 0;
            bound = sh.wave[0].m;
            __syncthreads();
            enlist();
            __syncthreads();
            listed = sh.n_who;
        }
        const int all = listed * pieces;
        // (a piece may come out of its wavefront's turn, so the order of the list varies; ranks do not)
        if (bound > -INFINITY)
            for (int p = t; p < all; p += LOGPROBS_NT) {
                const int q = p / pieces, r = p - q * pieces, id0 = (first + r / N) * CHUNK + (r % N) * LOGPROBS_NT * V + sh.who[q] * V;
                float y[V];
                if (id0 + V <= a.vocab) LpLoad<T>::get(x + id0, y);
                else {
#pragma unroll
                    for (int i = 0; i < V; ++i) y[i] = id0 + i < a.vocab ? (float)x[id0 + i] : -INFINITY;
                }
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (y[i] >= bound) { const int at = atomicAdd(&sh.n, 1); if (at < LOGPROBS_LIST) sh.list[at] = lp_key_of(y[i], id0 + i); }
            }
        __syncthreads();
        const int n = sh.n;
        if (bound > -INFINITY && n <= LOGPROBS_LIST) lp_rank(sh, n, k);
        else {                                               // k rounds: the largest of all threads' next ones, whose thread then looks for its next
            lp_key next = ~0ull, last;
            bool look = true;
            for (int j = 0; j < k; ++j) {
                if (look) {
                    last = next; next = 0;
                    for (int p = 0; p < pieces; ++p) {
                        const int id0 = (first + p / N) * CHUNK + (p % N) * LOGPROBS_NT * V + t * V;
#pragma unroll
                        for (int i = 0; i < V; ++i)
                            if (id0 + i < a.vocab) { const lp_key key = lp_key_of((float)x[id0 + i], id0 + i); if (key < last && key > next) next = key; }
                    }
                }
                const lp_key top = lp_largest(sh, next);
                if (t == 0) sh.best[j] = top;
                look = next == top;
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
        // everything is requested at once; sums: segments in turn over the threads, then over the threads, in a fixed order
        const int all = a.segs * k;
        auto take = [&](int i) {
            lp_key key = 0;
            if (i < all) { const uint32_t* p = part + (size_t)(i / k) * words + LOGPROBS_STATS + 2 * (i % k); key = get(p) | (lp_key)get(p + 1) << 32; }
            return key;
        };
        lp_key keys[LOGPROBS_AHEAD];
        if constexpr (TOP) {
#pragma unroll
            for (int u = 0; u < LOGPROBS_AHEAD; ++u) keys[u] = take(t + u * LOGPROBS_NT);
        }
        LpStats mine = {-INFINITY, 0.f, 0.f};
        bool bad = false;
        for (int i = t; i < a.segs; i += LOGPROBS_NT) {
            const uint32_t* p = part + (size_t)i * words;
            const LpStats o = {__uint_as_float(get(p)), __uint_as_float(get(p + 1)), __uint_as_float(get(p + 2))};
            bad |= get(p + 3) != 0 || o.m == INFINITY;
            mine.add(o, a.inv_temp);
        }
        if (__any(bad) && lane == 0) sh.nan = 1;
        for (int d = 1; d < 64 && d < a.segs; d <<= 1) {
            const LpStats o = {__shfl_xor(mine.m, d), __shfl_xor(mine.z, d), __shfl_xor(mine.s, d)};
            // both partners of a pair add in the same order
            LpStats lo = lane & d ? o : mine;
            const LpStats hi = lane & d ? mine : o;
            lo.add(hi, a.inv_temp);
            mine = lo;
        }
        if (lane == 0) sh.wave[wave] = mine;
        if (TOP && t < LOGPROBS_MAX_TOP) sh.best[t] = 0;
        __syncthreads();
        sum = sh.wave[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) sum.add(sh.wave[i], a.inv_temp);
        if constexpr (TOP) {
            for (int i0 = 0; i0 < all; i0 += LOGPROBS_AHEAD * LOGPROBS_NT) {
                if (i0) {
#pragma unroll
                    for (int u = 0; u < LOGPROBS_AHEAD; ++u) keys[u] = take(i0 + t + u * LOGPROBS_NT);
                }
                // as above, by whole keys: at most four of each of k threads of a wavefront pass the best bound
                const lp_key least = i0 ? sh.best[k - 1] : 0;
                lp_key bound = least;
                if (all > 64) {
                    lp_key own = keys[0];
#pragma unroll
                    for (int u = 1; u < LOGPROBS_AHEAD; ++u) own = keys[u] > own ? keys[u] : own;
                    const lp_key b = lp_bound(sh.lanes + 64 * wave, own, k, lane);
                    if (lane == 0) sh.bound[wave] = b;
                    __syncthreads();
#pragma unroll
                    for (int w = 0; w < 4; ++w) bound = sh.bound[w] > bound ? sh.bound[w] : bound;
                }
                if (t == 0) sh.n = 0;
                __syncthreads();
#pragma unroll
                for (int u = 0; u < LOGPROBS_AHEAD; ++u) if (keys[u] && keys[u] >= bound) sh.list[atomicAdd(&sh.n, 1)] = keys[u];
                if (i0 && t < k && sh.best[t]) sh.list[atomicAdd(&sh.n, 1)] = sh.best[t];
                __syncthreads();
                lp_rank(sh, sh.n, k);
            }
        }
    }
    const bool good = !sh.nan && sum.m > -INFINITY && sum.m < INFINITY;
    const float logz = logf(sum.z);
    if (t == 0 && a.entropy) a.entropy[row] = good ? logz - sum.s / sum.z : nothing;
    for (int j = t; j < a.n_tokens; j += LOGPROBS_NT) {
        if (j != t) { given = a.tokens[(long long)row * a.n_tokens + j]; if (given >= 0 && given < a.vocab) given_x = (float)x[given]; else given = -1; }
        a.logprob[(long long)row * a.n_tokens + j] = good && given >= 0 ? (given_x - sum.m) * a.inv_temp - logz : nothing;
    }
    if (TOP && t < k) {
        a.top_ids[(long long)row * k + t] = good ? (int)~(unsigned)sh.best[t] : -1;
        a.top_logprobs[(long long)row * k + t] = good ? (lp_value(sh.best[t]) - sum.m) * a.inv_temp - logz : nothing;
    }
}

}  // namespace hivis
