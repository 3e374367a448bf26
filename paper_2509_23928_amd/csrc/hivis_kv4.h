// Kernels of the paged cache in 4 bits: tables and slots (plan), rows into the cache (append) and back (read), attention over it.
//
// Format (include/hivis.h states it for callers).  A code is e2m1: sign, two exponent bits, one mantissa bit; 32 consecutive dims of a row share a
// power-of-two scale, one byte b = 2^(b - 127).  A scaled value x / 2^e is exact in fp32, so rounding to a code has one right answer, and every held
// value (two significant bits) is exact in bf16, the operand type of the matrix products: the cache itself adds no rounding.
// A block holds block_tokens rows of every key head; per head one run of memory: key codes [T][HD/2] | value codes [T][HD/2] |
// key scales [T][HD/32] | value scales [T][HD/32].
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hivis {

typedef __bf16 kv4_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 kv4_bf16x8 __attribute__((ext_vector_type(8)));
typedef float kv4_f32x4 __attribute__((ext_vector_type(4)));
typedef short kv4_s16x4 __attribute__((ext_vector_type(4)));

// What the kernels know of a cache
struct Kv4Dims { int heads, hd, block, shift, n_blocks; };       // block = 1 << shift rows

__host__ __device__ inline int kv4_chunk(int hd, int block) { return block * (hd + hd / 16); }      // bytes of one head in one block

// Scale byte of a group whose largest magnitude has the bits `a` (sign cleared): the smallest power of two at which no value is cut by more than
// half a step (a <= 7 scale; the largest code stands for 6 and its step is 2), between 2^-100 (products of two held values stay normal numbers) and
// 2^125 (a held value stays finite).  NaN and infinities: 255.
__host__ __device__ inline int kv4_scale_byte(unsigned a) {
    if (a >= 0x7f800000u) return 255;
    const int e = (int)(a >> 23) - 2 + ((a & 0x7fffffu) > 0x600000u);
    return e < 27 ? 27 : e > 252 ? 252 : e;
}

// ---- plan ------------------------------------------------------------------------------------------------------------------------------
// One workgroup; sequences in rounds of its 1024 threads.  Three sums over the sequences in order (rows, blocks given back from the last sequence on,
// blocks taken) decide everything, so the result does not depend on timing.  Latency bound: the sums, then one pass over the slots.
constexpr int PLAN_NT = 1024;

struct PlanArgs {
    int n, max_blocks, shift, n_blocks, max_rows;
    const int *keep, *add; int *held, *table, *free_list, *row_start, *slots, *positions, *status;
};

// inclusive sum over the workgroup's threads (64-bit: adds of many sequences pass 32 bits)
__device__ inline long long plan_scan(long long x, long long* part, long long* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const long long y = __shfl_up(x, d); if (lane >= d) x += y; }
    if (lane == 63) part[wave] = x;
    __syncthreads();
    long long before = 0, all = 0;
    for (int w = 0; w < PLAN_NT / 64; ++w) { if (w < wave) before += part[w]; all += part[w]; }
    __syncthreads();
    *total = all;
    return x + before;
}

// what sequence s asks for: status 2 if it cannot be meant (lengths below zero, more rows kept than its blocks hold, longer than its table row)
__device__ inline int plan_need(const PlanArgs& a, int s, int& keep, int& add, int& held) {
    keep = a.keep[s]; add = a.add[s]; held = a.held[s];
    const long long end = (long long)keep + add, room = (long long)held << a.shift;
    if (keep < 0 || add < 0 || held < 0 || held > a.max_blocks || keep > room || end > ((long long)a.max_blocks << a.shift)) return -1;
    return (int)((end + (1 << a.shift) - 1) >> a.shift);
}

__global__ __launch_bounds__(PLAN_NT) void kv4_plan_kernel(PlanArgs a) {
    __shared__ long long part[PLAN_NT / 64];
    const int t = threadIdx.x;
    // a list whose count is no count of blocks gives nothing
    int count = a.free_list[0];
    if (count < 0 || count > a.n_blocks) count = 0;
    __syncthreads();
    // ---- rows in order: who has room among the slots; blocks given back
    long long rows = 0, total;
    for (int s0 = 0; s0 < a.n; s0 += PLAN_NT) {
        const int s = s0 + t;
        int keep = 0, add = 0, held = 0, need = -1;
        if (s < a.n) need = plan_need(a, s, keep, add, held);
        const long long upto = rows + plan_scan(need >= 0 ? add : 0, part, &total);
        rows += total;
        if (s < a.n) a.status[s] = need < 0 ? 2 : upto > a.max_rows ? 3 : 0;
    }
    __syncthreads();
    for (int s0 = (a.n - 1) / PLAN_NT * PLAN_NT; s0 >= 0; s0 -= PLAN_NT) {       // the last sequence first
        const int s = s0 + PLAN_NT - 1 - t;
        int keep, add, held = 0, need = 0;
        bool give = false;
        if (s < a.n && a.status[s] == 0) { need = plan_need(a, s, keep, add, held); give = need < held; }
        const int n = give ? held - need : 0;
        int at = count + (int)(plan_scan(n, part, &total) - n);
        count = (int)min((long long)a.n_blocks, count + total);
        if (give) {
            int* row = a.table + (size_t)s * a.max_blocks;
            for (int j = held - 1; j >= need; --j, ++at) {
                if (at < a.n_blocks) a.free_list[1 + at] = row[j];               // (more blocks than there are: the tables were not this pool's)
                row[j] = -1;
            }
            a.held[s] = need;
        }
    }
    __threadfence_block();
    __syncthreads();
    // ---- blocks taken from the top of the list, in order of the sequences; row starts
    long long want = 0, start = 0;
    int left = count;
    for (int s0 = 0; s0 < a.n; s0 += PLAN_NT) {
        const int s = s0 + t;
        int keep = 0, add = 0, held = 0, need = 0, n = 0;
        bool ok = s < a.n && a.status[s] == 0;
        if (ok) { need = plan_need(a, s, keep, add, held); n = max(need - held, 0); }
        const long long upto = want + plan_scan(n, part, &total);
        want += total;
        if (ok && n > 0) {
            if (upto > count) { ok = false; a.status[s] = 1; }
            else {
                int* row = a.table + (size_t)s * a.max_blocks;
                const int top = count - (int)(upto - n);                         // list entry 1 + (top - 1) is the next one
                for (int j = 0; j < n; ++j) row[held + j] = a.free_list[top - j];
                a.held[s] = need;
            }
        }
        (void)plan_scan(ok ? n : 0, part, &total);
        left -= (int)total;
        const int mine = ok ? add : 0;
        const long long end = start + plan_scan(mine, part, &total);
        start += total;
        if (s < a.n) a.row_start[s] = (int)(end - mine);
    }
    if (t == 0) { a.row_start[a.n] = (int)start; a.free_list[0] = left; }
    __threadfence_block();
    __syncthreads();
    // ---- slots and positions of the rows; -1 behind the last
    for (int r = t; r < a.max_rows; r += PLAN_NT) {
        int slot = -1, pos = -1;
        if (r < (int)start) {
            int lo = 0, hi = a.n - 1;                                            // the last sequence that starts at or before r
            while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (a.row_start[mid] <= r) lo = mid; else hi = mid - 1; }
            pos = a.keep[lo] + r - a.row_start[lo];
            slot = (a.table[(size_t)lo * a.max_blocks + (pos >> a.shift)] << a.shift) + (pos & ((1 << a.shift) - 1));
        }
        a.slots[r] = slot;
        if (a.positions) a.positions[r] = pos;
    }
}

// ---- append and read ----------------------------------------------------------------------------------------------------------------------
// Rows as callers hold them: T (float, __bf16, or Kv4Halves: a high and a low IEEE half per value, all high halves of a row first), row r of head h at
// r * row + h * head (elements; Kv4Halves: values).
struct Kv4Halves {};
struct RowsArgs {
    Kv4Dims d; const void *k, *v; long long row, head; int n; const int* slots; uint8_t* pool;
    // rows of several sequences at equal distance instead (slots from the plan all the same): row r is row first[s] + r % m of sequence r / m, sequences `seq` elements apart
    const int* first; int m, offset; long long seq;
};

template <typename T> __device__ inline void kv4_load8(const T* p, float (&x)[8]);
template <> __device__ inline void kv4_load8<float>(const float* p, float (&x)[8]) {
    const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <> __device__ inline void kv4_load8<__bf16>(const __bf16* p, float (&x)[8]) {
    const uint4 a = *(const uint4*)p;
    const unsigned u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
}

// place of one group of eight dims: its code word and (for the group's first eight) scale byte
struct Kv4Place { uint8_t *code, *scale; };
__device__ inline Kv4Place kv4_place(const Kv4Dims& d, uint8_t* pool, int slot, int h, int kv, int piece) {
    const int r = slot & (d.block - 1);
    uint8_t* c = pool + ((size_t)(slot >> d.shift) * d.heads + h) * kv4_chunk(d.hd, d.block);
    return {c + (size_t)kv * d.block * (d.hd / 2) + r * (d.hd / 2) + piece * 4, c + (size_t)d.block * d.hd + (size_t)kv * d.block * (d.hd / 32) + r * (d.hd / 32) + piece / 4};
}

// A lane per eight dims: 16 or 32 bytes in, one word of codes out; four lanes agree on the group's scale.  Bound by the rows it reads.
// (Magnitudes are compared as integers: a NaN is then the largest, which fmax would drop.)
template <typename T>
__global__ __launch_bounds__(256) void kv4_append_kernel(RowsArgs a) {
    const int pieces = a.d.hd / 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, all = (long long)a.n * a.d.heads * 2 * pieces;
    if (i >= all) return;                                   // (whole groups of four lanes: all is a multiple of 8)
    const int piece = (int)(i % pieces), kv = (int)(i / pieces) & 1;
    const long long rh = i / (2 * pieces);
    const int h = (int)(rh % a.d.heads), r = (int)(rh / a.d.heads);
    const int slot = a.slots[r];
    if (slot < 0 || (slot >> a.d.shift) >= a.d.n_blocks) return;
    long long at = (long long)r * a.row;
    if (a.first) at = (long long)(r / a.m) * a.seq + ((long long)a.first[r / a.m] + a.offset + r % a.m) * a.row;
    at += (long long)h * a.head;
    float x[8];
    if constexpr (sizeof(T) == 1) {
        const _Float16* p = (const _Float16*)(kv ? a.v : a.k) + 2 * at + piece * 8;
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        const h8 hi = *(const h8*)p, lo = *(const h8*)(p + a.d.hd);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)hi[e] + (float)lo[e];
    } else kv4_load8<T>((const T*)(kv ? a.v : a.k) + at + piece * 8, x);
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
    m = max(m, (unsigned)__shfl_xor((int)m, 1)); m = max(m, (unsigned)__shfl_xor((int)m, 2));
    const int b = kv4_scale_byte(m);
    const float scale = __uint_as_float((unsigned)(b == 255 ? 127 : b) << 23);
    unsigned code = 0;
    if (b != 255) {
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0], x[1], scale, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2], x[3], scale, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4], x[5], scale, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6], x[7], scale, 3);
    }
    const Kv4Place p = kv4_place(a.d, a.pool, slot, h, kv, piece);
    *(unsigned*)p.code = code;
    if ((piece & 3) == 0) *p.scale = (uint8_t)b;
}

// the value of code c (four bits) at a scale
__device__ inline float kv4_value(unsigned c, float scale) {
    const unsigned m = c & 7;
    const float x = m < 2 ? 0.5f * m : __uint_as_float(((126 + (m >> 1)) << 23) | (m & 1) << 22);
    return ((c & 8) ? -x : x) * scale;
}

template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(RowsArgs a) {
    const int pieces = a.d.hd / 8;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x, all = (long long)a.n * a.d.heads * 2 * pieces;
    if (i >= all) return;
    const int piece = (int)(i % pieces), kv = (int)(i / pieces) & 1;
    const long long rh = i / (2 * pieces);
    const int h = (int)(rh % a.d.heads), r = (int)(rh / a.d.heads);
    const int slot = a.slots[r];
    if (slot < 0 || (slot >> a.d.shift) >= a.d.n_blocks) return;
    const Kv4Place p = kv4_place(a.d, a.pool, slot, h, kv, piece);
    const unsigned code = *(const unsigned*)p.code, b = *p.scale;
    const float scale = b == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float(b << 23);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = kv4_value(code >> (4 * e), scale);
    T* o = (T*)(kv ? a.v : a.k) + (long long)r * a.row + (long long)h * a.head + piece * 8;
    if constexpr (sizeof(T) == 4) { *(float4*)o = make_float4(x[0], x[1], x[2], x[3]); *(float4*)(o + 4) = make_float4(x[4], x[5], x[6], x[7]); }
    else {
        unsigned u[4];                                      // (exact: two significant bits)
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(x[2 * e]) >> 16 | (__float_as_uint(x[2 * e + 1]) & 0xffff0000u);
        *(uint4*)o = make_uint4(u[0], u[1], u[2], u[3]);
    }
}

// ---- attention ------------------------------------------------------------------------------------------------------------------------------
struct Kv4AttnArgs {
    Kv4Dims d; int group, n_seqs, n_rows, max_blocks, tiles; // group: query heads per key head; tiles: row tiles per sequence in the grid
    float scale2;                                            // softmax scale times log2 e
    const uint8_t* pool; const int *table, *row_start, *kv_len;
    const void* q; long long ldq; const unsigned long long* mask; void* out; long long ldo;
    // rows of the context's passes instead of row_start: m rows of every sequence, row r of sequence s at s * qrows + r in q and s * m + r in out, lengths kv_len[seq0 + s] + len_add
    int m, qrows, seq0, len_add;
};

// A work item is one key head of one sequence and 16 (row, query head) pairs of it, row by row; four wavefronts take 32-key tiles in turn, each with its
// own running maximum and sum, and merge at the end.
//   S^T[key][pair] = K Q^T: mfma 16x16x32 with 16 keys as rows.  Lane (n, g) reads a quarter g of key n's codes: one wide load, one scale; products
//     may take the dims in any order as long as both operands do, so step j multiplies dims g HD/4 + 8j ...
//   O^T[dim][pair] += V^T P^T: a lane holds the weights of keys 4g.. of both halves as they come out of S^T; V^T comes from a row-major bf16 tile
//     in LDS through the transposing read.
// fp32 queries and weights are split into three bf16 parts (24 bits: exact), so that an fp32 result has fp32 rounding; bf16 queries are one part, their
// weights are rounded to bf16 (off by at most 2^-8 each, as the result is).
template <int HD> struct Kv4Tile { static constexpr int VSTRIDE = HD * 2 + 32, BYTES = 32 * VSTRIDE; };

__device__ inline float kv4_xmax(float x) {                  // over the four lanes that share a pair
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float kv4_xsum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// eight codes (one word) as bf16
__device__ inline kv4_bf16x8 kv4_expand(unsigned w, float scale) {
    const kv4_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const kv4_bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return kv4_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// NP bf16 parts of eight fp32 values, each part what the ones before leave
template <int NP>
__device__ inline void kv4_parts(const float (&x)[8], kv4_bf16x8 (&p)[NP]) {
    float rest[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) rest[e] = x[e];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { p[k][e] = (__bf16)rest[e]; rest[e] -= (float)p[k][e]; }
    }
}

template <typename T, int HD>
__global__ __launch_bounds__(256) void kv4_attend_kernel(Kv4AttnArgs a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1, STEPS = HD / 32, NB = HD / 16, VSTRIDE = Kv4Tile<HD>::VSTRIDE, NW = 4;
    constexpr int MSTRIDE = HD + 2;                          // a pair's partial: HD sums, maximum, denominator
    constexpr int VB = NW * Kv4Tile<HD>::BYTES, MB = NW * 16 * MSTRIDE * 4;
    __shared__ __align__(16) char lds[VB > MB ? VB : MB];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const int h = blockIdx.x % a.d.heads, ti = blockIdx.x / a.d.heads % a.tiles, s = blockIdx.x / a.d.heads / a.tiles;
    int row0, orow0, rows, len;
    if (a.row_start) { row0 = orow0 = a.row_start[s]; rows = a.row_start[s + 1] - row0; len = a.kv_len[s]; }
    else { row0 = s * a.qrows; orow0 = s * a.m; rows = a.m; len = a.kv_len[a.seq0 + s] + a.len_add; }
    len = min(len, a.max_blocks << a.d.shift);
    if (row0 < 0 || rows < 0 || rows > a.n_rows - orow0) return;      // (no rows of this call)
    const int pairs = rows * a.group, p0 = ti * 16;
    if (p0 >= pairs) return;
    // this lane's pair (lanes behind the last repeat it) and the keys it sees: those below `below`, and from `below` on the bits of its mask
    const int pair = min(p0 + n16, pairs - 1), prow = pair / a.group, ph = h * a.group + pair % a.group;
    const int below = a.mask ? len - rows : len - rows + prow + 1;
    const unsigned long long bits = a.mask ? a.mask[orow0 + prow] : 0;
    const int limit = a.mask ? len : len - rows + min(p0 + 15, pairs - 1) / a.group + 1;       // no pair of the item sees a key from here on

    kv4_bf16x8 qf[STEPS][NP];
    {
        const T* q = (const T*)a.q + (long long)(row0 + prow) * a.ldq + (long long)ph * HD + g * (HD / 4);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) { float x[8]; kv4_load8<T>(q + 8 * j, x); kv4_parts<NP>(x, qf[j]); }
    }
    kv4_f32x4 o[NB];
#pragma unroll
    for (int t = 0; t < NB; ++t) o[t] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    char* const vt = lds + wave * Kv4Tile<HD>::BYTES;
    const int chunk = kv4_chunk(HD, a.d.block), mask_b = a.d.block - 1;
    for (int k0 = 32 * wave; k0 < limit; k0 += 32 * NW) {
        float sc[2][4];
        unsigned bad_k = 0, bad_v[HD / 32];                  // keys (bits 0..31) whose scale says NaN
#pragma unroll
        for (int t = 0; t < HD / 32; ++t) bad_v[t] = 0;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int key = k0 + 16 * half;
            // the half tile's block; one outside the pool: its keys are left out
            const int e = key < len ? __builtin_amdgcn_readfirstlane(a.table[(size_t)(a.row_start ? s : a.seq0 + s) * a.max_blocks + (key >> a.d.shift)]) : -1;
            const bool there = e >= 0 && e < a.d.n_blocks;
            const uint8_t* c = a.pool + ((size_t)(there ? e : 0) * a.d.heads + h) * chunk;
            const int r = (key & mask_b) + n16;
            const bool in = there && key + n16 < len;        // rows behind the last hold anything
            unsigned kw[STEPS], vw[STEPS];
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                kw[j] = ((const unsigned*)(c + r * (HD / 2) + g * (HD / 8)))[j];
                vw[j] = ((const unsigned*)(c + a.d.block * (HD / 2) + r * (HD / 2) + g * (HD / 8)))[j];
            }
            unsigned kb = c[a.d.block * HD + r * (HD / 32) + g * (HD / 4) / 32], vb = c[a.d.block * (HD + HD / 32) + r * (HD / 32) + g * (HD / 4) / 32];
            // a scale that says NaN is taken out of the products, where it would reach rows that do not see the key, and put back below
            const unsigned long long nk = __ballot(in && kb == 255), nv = __ballot(in && vb == 255);
            if (nk | nv) {
                bad_k |= (unsigned)((nk | nk >> 16 | nk >> 32 | nk >> 48) & 0xffff) << (16 * half);
#pragma unroll
                for (int t = 0; t < HD / 32; ++t) {          // group t of 32 dims: lanes g = 4 t 32 / HD ..
                    unsigned long long w = 0;
#pragma unroll
                    for (int u = 0; u < 128 / HD; ++u) w |= nv >> (16 * (t * (128 / HD) + u));
                    bad_v[t] |= (unsigned)(w & 0xffff) << (16 * half);
                }
            }
            if (!in || kb == 255) kb = 127;
            if (!in || vb == 255) vb = 127;
            const float ks = __uint_as_float(kb << 23), vs = __uint_as_float(vb << 23);
            kv4_f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                const kv4_bf16x8 kf = kv4_expand(kw[j], ks);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[j][p], x, 0, 0, 0);
                *(kv4_bf16x8*)(vt + (16 * half + n16) * VSTRIDE + (g * (HD / 4) + 8 * j) * 2) = kv4_expand(vw[j], vs);
            }
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const int kk = key + 4 * g + r4, nw = kk - below;
                const bool see = there && kk < len && (nw < 0 || (a.mask && nw < 64 && (bits >> nw & 1)));
                float y = x[r4];
                if (bad_k >> (16 * half + 4 * g + r4) & 1) y = __uint_as_float(0x7fc00000u);
                sc[half][r4] = see ? y * a.scale2 : -INFINITY;
            }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) mx = fmaxf(mx, sc[i >> 2][i & 3]);
        const float mn = fmaxf(m, kv4_xmax(mx)), ref = mn == -INFINITY ? 0.f : mn;
        const float f = __builtin_amdgcn_exp2f(m - ref);
        m = mn;
        l *= f;
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) { p[i] = __builtin_amdgcn_exp2f(sc[i >> 2][i & 3] - ref); l += p[i]; }
        kv4_bf16x8 pf[NP];
        kv4_parts<NP>(p, pf);
#pragma unroll
        for (int t = 0; t < NB; ++t) {
            o[t] *= f;
            typedef __attribute__((address_space(3))) kv4_s16x4* lds_p;
            const char* src = vt + (4 * g + n16 / 4) * VSTRIDE + (16 * t + 4 * (n16 & 3)) * 2;
            union { kv4_s16x4 s[2]; kv4_bf16x8 b; } vf;
            vf.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(src));
            vf.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(src + 16 * VSTRIDE));
#pragma unroll
            for (int q = NP - 1; q >= 0; --q) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf.b, pf[q], o[t], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < HD / 32; ++t)
            for (unsigned w = bad_v[t]; w; w &= w - 1) {      // values that are NaN, for the pairs that see them
                const int kk = k0 + __builtin_ctz(w), nw = kk - below;
                if (nw < 0 || (a.mask && nw < 64 && (bits >> nw & 1))) { o[2 * t] += __uint_as_float(0x7fc00000u); o[2 * t + 1] += __uint_as_float(0x7fc00000u); }
            }
    }
    l = kv4_xsum(l);
    __syncthreads();
    float* const mrg = (float*)lds;
    {
        float* dst = mrg + (wave * 16 + n16) * MSTRIDE;
#pragma unroll
        for (int t = 0; t < NB; ++t)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) dst[16 * t + 4 * g + r4] = o[t][r4];
        if (g == 0) { dst[HD] = m; dst[HD + 1] = l; }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * HD; i += 256) {
        const int pr = i / HD, c = i % HD;
        if (p0 + pr >= pairs) break;
        float mx = -INFINITY, den = 0.f, num = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) mx = fmaxf(mx, mrg[(w * 16 + pr) * MSTRIDE + HD]);
        if (mx == -INFINITY) mx = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float* src = mrg + (w * 16 + pr) * MSTRIDE;
            const float f = __builtin_amdgcn_exp2f(src[HD] - mx);
            den += src[HD + 1] * f; num += src[c] * f;
        }
        const int row = (p0 + pr) / a.group, hq = h * a.group + (p0 + pr) % a.group;
        const float y = den == 0.f ? 0.f : num / den;        // a row that sees nothing: zero
        ((T*)a.out)[(long long)(orow0 + row) * a.ldo + (long long)hq * HD + c] = (T)y;
    }
}

}  // namespace hivis
