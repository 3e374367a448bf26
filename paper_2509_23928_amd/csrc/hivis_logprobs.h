// Log probabilities of given tokens, entropy and the most probable tokens of rows of logits.
//   y = x / T;  log p(t) = y_t - log sum exp y;  H = log sum exp y - sum p y.
// All of it relative to the row's maximum: log p(t) = (x_t - max) / T - log z, z = sum e, H = log z - sum e (x - max) / T / z, e = exp((x - max) / T).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hivis {

constexpr int LOGPROBS_MAX_TOP = 32;

struct LogprobsArgs {
    const void* x; long long ld; int rows, vocab; float inv_temp;
    const int* tokens; int n_tokens; float *logprob, *entropy;
    int top; int* top_ids; float* top_logprobs;
};

// order of the alternatives as one number: larger logits first, then lower indices
__device__ inline unsigned long long logprob_key(float x, unsigned i) {
    const unsigned u = __float_as_uint(x + 0.f);            // (-0 as 0)
    const unsigned k = u & 0x80000000u ? ~u : u | 0x80000000u;
    return (unsigned long long)k << 32 | ~i;
}
__device__ inline float logprob_value(unsigned long long key) {
    const unsigned k = (unsigned)(key >> 32);
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

template <typename T>
__global__ __launch_bounds__(1024) void logprobs_kernel(LogprobsArgs a) {
    __shared__ float fm[16], fz[16], fs[16];
    __shared__ unsigned long long fk[16];
    const int row = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const T* x = (const T*)a.x + (long long)row * a.ld;
    float m = -INFINITY;
    bool nan = false;
    for (int i = t; i < a.vocab; i += 1024) { const float v = (float)x[i]; m = fmaxf(m, v); nan |= v != v; }
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (__any(nan)) m = __uint_as_float(0x7fc00000u);
    if (lane == 0) fm[wave] = m;
    __syncthreads();
    m = -INFINITY;
    for (int w = 0; w < 16; ++w) m = fm[w] != fm[w] || m != m ? __uint_as_float(0x7fc00000u) : fmaxf(m, fm[w]);
    const bool good = m > -INFINITY && m < INFINITY;
    float z = 0.f, s = 0.f;
    if (good)
        for (int i = t; i < a.vocab; i += 1024) {
            const float y = ((float)x[i] - m) * a.inv_temp, e = __expf(y);
            z += e;
            if (e > 0.f) s += e * y;                        // (a logit of -inf adds nothing)
        }
#pragma unroll
    for (int d = 32; d; d >>= 1) { z += __shfl_xor(z, d); s += __shfl_xor(s, d); }
    if (lane == 0) { fz[wave] = z; fs[wave] = s; }
    __syncthreads();
    z = s = 0.f;
    for (int w = 0; w < 16; ++w) { z += fz[w]; s += fs[w]; }
    const float logz = logf(z), none = __uint_as_float(0x7fc00000u);
    if (t == 0 && a.entropy) a.entropy[row] = good ? logz - s / z : none;
    for (int j = t; j < a.n_tokens; j += 1024) {
        const int id = a.tokens[(long long)row * a.n_tokens + j];
        a.logprob[(long long)row * a.n_tokens + j] = good && id >= 0 && id < a.vocab ? ((float)x[id] - m) * a.inv_temp - logz : none;
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
        unsigned long long best = 0;
        if (good)
            for (int i = t; i < a.vocab; i += 1024) { const unsigned long long key = logprob_key((float)x[i], i); if (key < last && key > best) best = key; }
#pragma unroll
        for (int d = 32; d; d >>= 1) { const unsigned long long o = __shfl_xor(best, d); best = best > o ? best : o; }
        if (lane == 0) fk[wave] = best;
        __syncthreads();
        for (int w = 0; w < 16; ++w) best = best > fk[w] ? best : fk[w];
        __syncthreads();
        last = best;
        if (t == 0) {
            a.top_ids[(long long)row * a.top + k] = good ? (int)~(unsigned)best : -1;
            a.top_logprobs[(long long)row * a.top + k] = good ? (logprob_value(best) - m) * a.inv_temp - logz : none;
        }
    }
}

}  // namespace hivis
