// Kernels of the paged cache in 4 bits: tables and slots (plan), rows into the cache (append) and back (read), attention over it.
//
// Format (include/hivis.h states it for callers).  A code is e2m1: sign, two exponent bits, one mantissa bit; 32 consecutive dims of a row share a
// power-of-two scale, one byte b = 2^(b - 127).  A scaled value x / 2^e is exact in fp32, so rounding to a code has one right answer, and every held
// value (two significant bits) is exact in bf16, the operand type of the matrix products: the cache itself adds no rounding.
// A block holds block_tokens rows of every key head; per head one run of memory: key codes [T][HD/2] | value codes [T][HD/2] |
// key scales [T][HD/32] | value scales [T][HD/32].
#pragma once
#include "hivis_kv4_args.h"

namespace hivis {

typedef __bf16 kv4_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 kv4_bf16x8 __attribute__((ext_vector_type(8)));
typedef float kv4_f32x4 __attribute__((ext_vector_type(4)));
typedef float kv4_f32x16 __attribute__((ext_vector_type(16)));
typedef short kv4_s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned kv4_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned kv4_u32x2 __attribute__((ext_vector_type(2)));

// Scale byte of a group whose largest magnitude has the bits `a` (sign cleared): the smallest power of two at which no value is cut by more than
// half a step (a <= 7 scale; the largest code stands for 6 and its step is 2), between 2^-100 (products of two held values stay normal numbers) and
// 2^125 (a held value stays finite).  NaN and infinities: 255.
__host__ __device__ inline int kv4_scale_byte(unsigned a) {
    if (a >= 0x7f800000u) return 255;
    const int e = (int)(a >> 23) - 2 + ((a & 0x7fffffu) > 0x600000u);
    return e < 27 ? 27 : e > 252 ? 252 : e;
}

// ---- plan ------------------------------------------------------------------------------------------------------------------------------
// Three sums over the sequences in order (rows, blocks given back from the last sequence on, blocks taken) decide everything, so the result does not depend on
// timing.  Latency bound: one workgroup, a wavefront for every 64 sequences up to sixteen (and rounds of 1024 beyond), sums in registers, one batch of requests
// per step; blocks are moved by all threads, a block each.  The slots of many rows are a launch of their own, over the chip (plan_fused).
constexpr int PLAN_MAX = 1024;                               // threads at most

struct PlanShared { long long part[PLAN_MAX / 64]; int from[PLAN_MAX], base[PLAN_MAX], s[PLAN_MAX]; };

// inclusive sum over the workgroup's threads (64-bit: adds of many sequences pass 32 bits)
__device__ inline long long plan_scan(long long x, long long* part, long long* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const long long y = __shfl_up(x, d); if (lane >= d) x += y; }
    if (waves == 1) { *total = __shfl(x, 63); return x; }
    if (lane == 63) part[wave] = x;
    __syncthreads();
    long long before = 0, all = 0;
    for (int w = 0; w < waves; ++w) { if (w < wave) before += part[w]; all += part[w]; }
    __syncthreads();
    *total = all;
    return x + before;
}

// what sequence s asks for, in blocks; -1 if it cannot be meant (lengths below zero, more rows kept than its blocks hold, longer than its table row)
__device__ inline int plan_need(const PlanArgs& a, int keep, int add, int held) {
    const long long end = (long long)keep + add, room = (long long)held << a.shift;
    if (keep < 0 || add < 0 || held < 0 || held > a.max_blocks || keep > room || end > ((long long)a.max_blocks << a.shift)) return -1;
    return (int)((end + (1 << a.shift) - 1) >> a.shift);
}

// Blocks of the round's sequences, a thread each: `n` of this thread's sequence s (upto: with those of the threads before it, all in total), from its block `from` on.
// f(sequence, block index, position among the round's blocks)
template <typename F>
__device__ inline void plan_blocks(PlanShared& sh, int s, int n, int from, long long upto, long long total, F f) {
    sh.s[threadIdx.x] = s; sh.from[threadIdx.x] = from; sh.base[threadIdx.x] = (int)upto;
    __syncthreads();
    for (long long i = threadIdx.x; i < total; i += blockDim.x) {
        int lo = 0, hi = blockDim.x - 1;                     // the first thread whose blocks end behind i
        while (lo < hi) { const int mid = (lo + hi) >> 1; if (sh.base[mid] > i) hi = mid; else lo = mid + 1; }
        const int before = lo ? sh.base[lo - 1] : 0;
        f(sh.s[lo], sh.from[lo] + (int)i - before, (int)i);
    }
    __syncthreads();
}

__device__ inline void plan_fill(const PlanArgs& a, int r, int total) {
    int slot = -1, pos = -1;
    if (r < total) {
        int lo = 0, hi = a.n - 1;                            // the last sequence that starts at or before r
        while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (a.row_start[mid] <= r) lo = mid; else hi = mid - 1; }
        pos = (a.keep ? a.keep[lo] : 0) + r - a.row_start[lo];
        slot = (a.table[(size_t)lo * a.max_blocks + (pos >> a.shift)] << a.shift) + (pos & ((1 << a.shift) - 1));
    }
    a.slots[r] = slot;
    if (a.positions) a.positions[r] = pos;
}

__global__ __launch_bounds__(PLAN_MAX) void kv4_plan_kernel(PlanArgs a) {
    __shared__ PlanShared sh;
    const int t = threadIdx.x, threads = blockDim.x, rounds = (a.n + threads - 1) / threads;
    // a list whose count is no count of blocks gives nothing
    int count = a.free_list[0];
    if (count < 0 || count > a.n_blocks) count = 0;
    // One round: everything stays in registers.  More: what a sequence asks for is read again for every sum (held changes only where blocks are given back).
    int keep = 0, add = 0, held = 0, need = -1, status = 0;
    auto load = [&](int s) { keep = add = held = 0; need = -1; if (s < a.n) { keep = a.keep ? a.keep[s] : 0; add = a.add ? a.add[s] : a.add_each; held = a.held[s]; need = plan_need(a, keep, add, held); } };
    long long rows = 0, total;
    // ---- rows in order: who has room among the slots
    for (int r = 0; r < rounds; ++r) {
        const int s = r * threads + t;
        load(s);
        const long long upto = rows + plan_scan(need >= 0 ? add : 0, sh.part, &total);
        rows += total;
        status = need < 0 ? 2 : upto > a.max_rows ? 3 : 0;
        if (s < a.n && rounds > 1) a.status[s] = status;
    }
    // ---- blocks given back, the last sequence's last block first
    __syncthreads();
    for (int r = rounds - 1; r >= 0; --r) {
        const int s = r * threads + t;
        if (rounds > 1) { load(s); status = s < a.n ? a.status[s] : 2; }
        const int n = status == 0 && need >= 0 ? max(held - need, 0) : 0;
        const long long upto = plan_scan(n, sh.part, &total);
        if (total) {
            const long long all = total;
            plan_blocks(sh, s, n, need, upto, total, [&](int seq, int j, int i) {
                const long long at = count + (all - 1 - i);              // (more blocks than there are: the tables were not this pool's)
                int* b = a.table + (size_t)seq * a.max_blocks + j;
                if (at < a.n_blocks) a.free_list[1 + at] = *b;
                *b = -1;
            });
            if (n) { held = need; a.held[s] = need; }
            count = (int)min((long long)a.n_blocks, count + total);
        }
    }
    __threadfence_block();
    __syncthreads();
    // ---- blocks taken from the top of the list, in order of the sequences; row starts
    long long want = 0, start = 0;
    int left = count;
    for (int r = 0; r < rounds; ++r) {
        const int s = r * threads + t;
        if (rounds > 1) { load(s); status = s < a.n ? a.status[s] : 2; }
        const int n = status == 0 && need >= 0 ? max(need - held, 0) : 0;
        const long long upto = want + plan_scan(n, sh.part, &total);
        if (n > 0 && upto > count) status = 1;
        // those before the first that is refused are served, so what is taken is a run from the top
        const int mine = status == 0 ? n : 0;
        long long taken = total;
        if (want + total > count) (void)plan_scan(mine, sh.part, &taken);
        if (taken) {
            const int top = count - (int)want;               // list entry `top` is the next one
            plan_blocks(sh, s, mine, held, taken == total ? upto - want : min(upto - want, taken), taken, [&](int seq, int j, int i) { a.table[(size_t)seq * a.max_blocks + j] = a.free_list[top - i]; });
            if (mine) a.held[s] = need;
        }
        want += total;
        left -= (int)taken;
        const int lines = status == 0 && s < a.n ? add : 0;
        const long long end = start + plan_scan(lines, sh.part, &total);
        start += total;
        if (s < a.n) { a.row_start[s] = (int)(end - lines); a.status[s] = status; }
    }
    if (t == 0) { a.row_start[a.n] = (int)start; a.free_list[0] = left; }
    if (!a.fill) return;
    __threadfence_block();
    __syncthreads();
    for (int r = t; r < a.max_rows; r += threads) plan_fill(a, r, (int)start);
}

__global__ __launch_bounds__(256) void kv4_plan_slots_kernel(PlanArgs a) {
    const int r = blockIdx.x * 256 + threadIdx.x;
    if (r < a.max_rows) plan_fill(a, r, a.row_start[a.n]);
}

// ---- append and read ----------------------------------------------------------------------------------------------------------------------
// Rows as callers hold them: T (float, __bf16, or Kv4Halves: a high and a low IEEE half per value, all high halves of a row first), row r of head h at
// r * row + h * head (elements; Kv4Halves: values).
struct Kv4Halves {};
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

// Grid of append and read: lanes over a row's keys, then its values, eight dims each (x), and RPT rows per thread (y, in rounds of the grid): no quotients, the slots in
// scalar registers, RPT requests under way.
struct Kv4Lane { int kv, h, piece; long long at; bool in; };         // at: of its eight dims in a row (values)
__device__ inline Kv4Lane kv4_lane(const RowsArgs& a) {
    const int i = blockIdx.x * 256 + threadIdx.x, sh = a.d.hd == 128 ? 4 : 3, half = a.d.heads << sh;
    Kv4Lane l;
    l.in = i < 2 * half;
    l.kv = i >= half;
    l.h = (i - l.kv * half) >> sh; l.piece = i & ((1 << sh) - 1);
    l.at = (long long)l.h * a.head + l.piece * 8;
    return l;
}
// places of those dims in a slot's block: code word, and scale byte of the group that they belong to
struct Kv4Place { uint8_t *code, *scale; };
__device__ inline Kv4Place kv4_place(const Kv4Dims& d, uint8_t* pool, int slot, const Kv4Lane& l) {
    const int r = slot & (d.block - 1);
    uint8_t* c = pool + ((size_t)(slot >> d.shift) * d.heads + l.h) * kv4_chunk(d.hd, d.block);
    return {c + (l.kv * d.block + r) * (d.hd / 2) + l.piece * 4, c + d.block * d.hd + (l.kv * d.block + r) * (d.hd / 32) + l.piece / 4};
}
__device__ inline int kv4_slot(const RowsArgs& a, int r) {           // -1: the row is left out
    const int slot = r < a.n ? a.slots[r] : -1;
    return slot >= 0 && (slot >> a.d.shift) < a.d.n_blocks ? slot : -1;
}

// A lane per eight dims: 16 or 32 bytes in, one word of codes out; four lanes agree on the group's scale.  Bound by the rows it reads.
// (Magnitudes are compared as integers: a NaN is then the largest, which fmax would drop.)
template <typename T, int RPT>
__global__ __launch_bounds__(256) void kv4_append_kernel(RowsArgs a) {
    const Kv4Lane l = kv4_lane(a);
    if (!l.in) return;                                       // (whole groups of four lanes)
    const char* const base = (const char*)(l.kv ? a.v : a.k);
    for (int r0 = blockIdx.y * RPT; r0 < a.n; r0 += gridDim.y * RPT) {
        float x[RPT][8];
        int slot[RPT];
#pragma unroll
        for (int u = 0; u < RPT; ++u) slot[u] = kv4_slot(a, r0 + u);
#pragma unroll
        for (int u = 0; u < RPT; ++u) {
            const int r = min(r0 + u, a.n - 1);              // (a row that is left out is read, not written)
            long long at = (long long)r * a.row;
            if (a.first) at = (long long)(r / a.m) * a.seq + ((long long)a.first[r / a.m] + a.offset + r % a.m) * a.row;
            at += l.at;
            if constexpr (sizeof(T) == 1) {
                typedef _Float16 h8 __attribute__((ext_vector_type(8)));
                const _Float16* p = (const _Float16*)base + 2 * (at - l.piece * 8) + l.piece * 8;
                const h8 hi = *(const h8*)p, lo = *(const h8*)(p + a.d.hd);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[u][e] = (float)hi[e] + (float)lo[e];
            } else kv4_load8<T>((const T*)base + at, x[u]);
        }
#pragma unroll
        for (int u = 0; u < RPT; ++u) {
            unsigned m = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[u][e]) & 0x7fffffffu);
            m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, false)); m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, false));
            const int b = kv4_scale_byte(m);
            const float scale = __uint_as_float((unsigned)(b == 255 ? 127 : b) << 23);
            unsigned code = 0;
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[u][0], x[u][1], scale, 0);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[u][2], x[u][3], scale, 1);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[u][4], x[u][5], scale, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[u][6], x[u][7], scale, 3);
            if (slot[u] < 0) continue;
            const Kv4Place p = kv4_place(a.d, a.pool, slot[u], l);
            *(unsigned*)p.code = b == 255 ? 0 : code;
            if ((l.piece & 3) == 0) *p.scale = (uint8_t)b;
        }
    }
}

// the value of code c (four bits) at a scale
__device__ inline float kv4_value(unsigned c, float scale) {
    const unsigned m = c & 7;
    const float x = m < 2 ? 0.5f * m : __uint_as_float(((126 + (m >> 1)) << 23) | (m & 1) << 22);
    return ((c & 8) ? -x : x) * scale;
}

template <typename T, int RPT>
__global__ __launch_bounds__(256) void kv4_read_kernel(RowsArgs a) {
    const Kv4Lane l = kv4_lane(a);
    if (!l.in) return;
    for (int r0 = blockIdx.y * RPT; r0 < a.n; r0 += gridDim.y * RPT) {
        unsigned code[RPT], b[RPT];
        int slot[RPT];
#pragma unroll
        for (int u = 0; u < RPT; ++u) slot[u] = kv4_slot(a, r0 + u);
#pragma unroll
        for (int u = 0; u < RPT; ++u) {
            const Kv4Place p = kv4_place(a.d, a.pool, max(slot[u], 0), l);
            code[u] = *(const unsigned*)p.code; b[u] = *p.scale;
        }
#pragma unroll
        for (int u = 0; u < RPT; ++u) {
            if (slot[u] < 0) continue;
            const float scale = b[u] == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float(b[u] << 23);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = kv4_value(code[u] >> (4 * e), scale);
            T* o = (T*)(l.kv ? a.v : a.k) + (long long)(r0 + u) * a.row + l.at;
            if constexpr (sizeof(T) == 4) { *(float4*)o = make_float4(x[0], x[1], x[2], x[3]); *(float4*)(o + 4) = make_float4(x[4], x[5], x[6], x[7]); }
            else {
                unsigned w[4];                               // (exact: two significant bits)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(x[2 * e]) >> 16 | (__float_as_uint(x[2 * e + 1]) & 0xffff0000u);
                *(uint4*)o = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
}

// Rows of sequence 0 from positions len + path[j] to len + j, j = 1 .. *n, in the pools of all layers (blockIdx.x) for each key head (blockIdx.y): all are read before any is
// written, for one row's place can be another's origin.
__global__ __launch_bounds__(256) void kv4_move_kernel(Kv4Dims d, uint8_t* mem, long long pool, const int* table, const int* len, const int* n, const int* path) {
    extern __shared__ uint16_t kv4_moved[];                  // [row][codes of the key, of the value, their scales], two bytes each
    const int units = (d.hd + d.hd / 16) / 2, rows = n[0];
    uint8_t* const base = mem + blockIdx.x * pool;
    auto at = [&](int pos, int u) -> uint16_t* {
        uint8_t* c = base + ((size_t)table[pos >> d.shift] * d.heads + blockIdx.y) * kv4_chunk(d.hd, d.block);
        const int r = pos & (d.block - 1), code = d.hd / 4, scale = d.hd / 64;
        if (u < 2 * code) return (uint16_t*)(c + ((u >= code) * d.block + r) * (d.hd / 2)) + u % code;
        u -= 2 * code;
        return (uint16_t*)(c + d.block * d.hd + ((u >= scale) * d.block + r) * (d.hd / 32)) + u % scale;
    };
    for (int i = threadIdx.x; i < rows * units; i += 256) kv4_moved[i] = *at(len[0] + path[1 + i / units], i % units);
    __syncthreads();
    for (int i = threadIdx.x; i < rows * units; i += 256) *at(len[0] + 1 + i / units, i % units) = kv4_moved[i];
}

// ---- attention ------------------------------------------------------------------------------------------------------------------------------
// The kernels multiply alike.  A tile of 16 (row, query head) pairs of one key head, row by row, is the N dimension of
//   S^T[key][pair] = K Q^T          mfma 16x16x32, 16 keys as rows
//   O^T[dim][pair] += V^T P^T       a lane's weights of keys 4g .. 4g+3 of two 16-key halves are its operand as they come out of S^T (contractions take any
//                                   order that both operands share); V^T comes from row-major bf16 in LDS through the transposing read.
// fp32 queries and weights are split into three bf16 parts (24 bits: exact), so that an fp32 result has fp32 rounding; bf16 queries are one part, their
// weights are rounded to bf16 (off by at most 2^-8 each, as the result is).
// Weights are 2^(s - ref); ref follows a pair's largest score s only when that outgrows it by 2^8, so most tiles need no maximum over lanes and no
// rescaling; sums and maxima are fp32.
constexpr float KV4_REF0 = -3.0e38f;                         // ref before the first key (finite: a difference of two infinities would be no number)
constexpr float KV4_SLACK = 8.f;
constexpr int KV4_UNIT = 128;                                // keys of a unit of work: four wavefronts, 32 each
constexpr int KV4_ITEM_COST = 2;                             // what opening and closing an item costs, in units

// LDS rows: the transposing read of four rows, and eight lanes' 16-byte accesses, meet all banks
template <int HD> constexpr int kv4_vstride() { return HD * 2 + 32; }
template <int HD> constexpr int kv4_vstride32() { return HD * 2 + 64; }
template <int HD> constexpr int kv4_kstride() { return HD * 2 + 16; }

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
// orders LDS accesses only (__syncthreads waits for all requests to memory as well)
__device__ inline void kv4_lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
__device__ inline float kv4_nan() { return __uint_as_float(0x7fc00000u); }

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
        for (int e = 0; e < 8; ++e) { p[k][e] = (__bf16)rest[e]; if (k + 1 < NP) rest[e] -= (float)p[k][e]; }
    }
}

// four keys of one dim of two 16-key halves, from row-major bf16 rows (row 0 of the tile at `tile`)
template <int HD>
__device__ inline kv4_bf16x8 kv4_vfrag(const char* tile, int t, int lane) {
    typedef __attribute__((address_space(3))) kv4_s16x4* lds_p;
    const char* src = tile + (4 * (lane >> 4) + (lane & 15) / 4) * kv4_vstride<HD>() + (16 * t + 4 * (lane & 3)) * 2;
    union { kv4_s16x4 s[2]; kv4_bf16x8 b; } f;
    f.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)src);
    f.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(src + 16 * kv4_vstride<HD>()));
    return f.b;
}

// The rows of sequence s: where they start in q and out, how many, how many cached rows
struct Kv4Seq { int q0, o0, rows, pairs, len; };            // pairs: of the rows that the launch is sized for
__device__ inline Kv4Seq kv4_seq(const Kv4AttnArgs& a, int s) {
    Kv4Seq x;
    if (a.row_start) { x.q0 = x.o0 = a.row_start[s]; x.rows = a.row_start[s + 1] - x.q0; x.len = a.kv_len[s]; }
    else { x.q0 = s * a.qrows; x.o0 = s * a.m; x.rows = a.m; x.len = a.kv_len[a.seq0 + s] + a.len_add; }
    x.len = max(0, min(x.len, a.max_blocks << a.d.shift));
    if (x.o0 < 0 || x.rows < 0 || x.rows > a.n_rows - x.o0) x.rows = 0;      // (no rows of this call)
    x.pairs = min(x.rows, a.max_rows) * a.group;
    return x;
}

// What a lane's pair sees: the keys below `below`, and of the 64 from there on those of `bits`
struct Kv4Sight {
    int below; unsigned long long bits;
    __device__ unsigned long long of(int k0) const {         // of the 64 keys from k0 on, a bit each
        const int n = below - k0;
        return (n >= 64 ? ~0ull : (1ull << max(n, 0)) - 1) | (n >= 0 ? n < 64 ? bits << n : 0 : n > -64 ? bits >> -n : 0);
    }
};

// Queries of 16 pairs from pair p0 on (lanes behind the last repeat it), eight values of each in the order of dims that `dim` gives for lane quarter g and
// step j: as they lie in memory, and as operand parts
template <typename T> struct Kv4Raw { kv4_u32x4 x[sizeof(T) / 2]; };
template <typename T, int HD, typename Dim>
__device__ inline void kv4_queries(const Kv4AttnArgs& a, const Kv4Seq& s, int h, int p0, int n16, int g, Dim dim, Kv4Raw<T> (&raw)[HD / 32], Kv4Sight& see) {
    const int pair = min(p0 + n16, s.pairs - 1), row = a.group == 1 ? pair : pair / a.group, hq = h * a.group + pair - row * a.group;
    see.below = s.len - s.rows + (a.mask ? 0 : row + 1);
    see.bits = a.mask ? a.mask[s.o0 + row] : 0;
    const T* q = (const T*)a.q + (long long)(s.q0 + row) * a.ldq + (long long)hq * HD;
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) raw[j] = *(const Kv4Raw<T>*)(q + dim(g, j));
}
template <typename T, int NP>
__device__ inline void kv4_query_part(bool negate, const Kv4Raw<T>& raw, kv4_bf16x8 (&f)[NP]) {
    if constexpr (sizeof(T) == 2) {
        kv4_u32x4 x = raw.x[0];
        if (negate) x ^= 0x80008000u;
        f[0] = __builtin_bit_cast(kv4_bf16x8, x);
    } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[e] = __uint_as_float(raw.x[e >> 2][e & 3]); if (negate) x[e] = -x[e]; }
        kv4_parts<NP>(x, f);
    }
}

// One tile of pairs against NH halves of 16 keys, scores x (bit 16 c + 4 g + r of a lane's word: x[c][r]).
// The keys that a pair does not see weigh nothing (a scale of zero is a tiny one in scale2, so that no product of zero and infinity comes up).
template <int NH>
__device__ inline void kv4_hide(kv4_f32x4 (&x)[NH], unsigned long long vis, int g) {
    vis >>= 4 * g;
    const unsigned on[2] = {(unsigned)vis, (unsigned)(vis >> 32)};
#pragma unroll
    for (int i = 0; i < 4 * NH; ++i)                         // (an all-ones or all-zeros word selects)
        x[i >> 2][i & 3] = ((int)(on[i >> 3] << (31 - 16 * (i >> 2 & 1) - (i & 3))) >> 31) ? x[i >> 2][i & 3] : -INFINITY;
}
template <int NH>
__device__ inline float kv4_top(const kv4_f32x4 (&x)[NH]) {
    float mx = x[0][0];
#pragma unroll
    for (int i = 1; i < 4 * NH; ++i) mx = fmaxf(mx, x[i >> 2][i & 3]);
    return mx;
}
// A weight's exponent is s - ref in one rounding, with s the exact product of a score and the scale, but ref a rounded one: beyond 2^24 the two are so far apart that
// the weight of the largest score itself may be infinite or nothing.  There (`far`, of any lane) s is rounded first, as ref was.
__device__ inline bool kv4_far(float ref) { return __any(fabsf(ref) > 0x1p24f && ref != KV4_REF0); }
__device__ inline float kv4_rounded(float x, float scale2, float ref) {
#pragma clang fp contract(off)
    const float s = x * scale2;
    return s - ref;
}
// ref follows a largest score of mx; what was added up so far follows it
template <int NB>
__device__ inline void kv4_follow(float mx, kv4_f32x4 (&o)[NB], float& ref, float& l, bool& far) {
    const float to = fmaxf(ref, kv4_xmax(mx)), f = __builtin_amdgcn_exp2f(ref - to);
    ref = to; far = kv4_far(to);
    l *= f;
#pragma unroll
    for (int t = 0; t < NB; ++t) o[t] *= f;
}
// scores to weights in operand parts, and their sum
template <int NH, int NP>
__device__ inline void kv4_weights(kv4_f32x4 (&x)[NH], float scale2, float ref, bool far, float& l, kv4_bf16x8 (&pf)[NH / 2][NP]) {
    float p[4 * NH], s[4];
    if (far) {
#pragma unroll
        for (int i = 0; i < 4 * NH; ++i) x[i >> 2][i & 3] = kv4_rounded(x[i >> 2][i & 3], scale2, ref);
        scale2 = 1.f; ref = 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4 * NH; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i >> 2][i & 3], scale2, -ref));
#pragma unroll
    for (int i = 0; i < 4; ++i) { s[i] = p[i] + p[i + 4]; if (NH == 4) s[i] += p[(i + 8) % (4 * NH)] + p[(i + 12) % (4 * NH)]; }
    l += (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int k = 0; k < NH / 2; ++k) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = p[8 * k + i];
        kv4_parts<NP>(e, pf[k]);
    }
}
// Scales that say NaN never enter the products, where they would reach pairs that do not see the key: a pair that sees one notes which dims of its result are no
// numbers (a bit per 32; a key's scale: all), and they are set at the end.
template <int NB>
__device__ inline void kv4_poison(unsigned no_number, kv4_f32x4 (&o)[NB]) {
#pragma unroll
    for (int t = 0; t < NB; ++t) if (no_number >> (t / 2) & 1) o[t] = kv4_f32x4{kv4_nan(), kv4_nan(), kv4_nan(), kv4_nan()};
}

// result of pair pr (of the sequence), dims c .. c + 3
template <typename T, int HD>
__device__ inline void kv4_store4(const Kv4AttnArgs& a, const Kv4Seq& s, int h, int pr, int c, const kv4_f32x4& x) {
    const int row = pr / a.group, hq = h * a.group + pr - row * a.group;
    T* o = (T*)a.out + (long long)(s.o0 + row) * a.ldo + (long long)hq * HD + c;
    if constexpr (sizeof(T) == 4) *(kv4_f32x4*)o = x;
    else { typedef __bf16 b4 __attribute__((ext_vector_type(4))); *(b4*)o = b4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]}; }
}
// Partial results of a workgroup for workgroups of other chiplets: written through, read past the own L2 (agent scope), 16 or 8 bytes at a time
constexpr int KV4_AGENT = 16;                                // cache policy of buffer accesses: agent scope
struct Kv4Partials {
    __amdgpu_buffer_rsrc_t r;
    __device__ Kv4Partials(float* p, unsigned bytes) : r(__builtin_amdgcn_make_buffer_rsrc(p, 0, bytes, 0x00020000)) {}
    __device__ void put4(unsigned at, const kv4_f32x4& x) const { __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(kv4_u32x4, x), r, at * 4, 0, KV4_AGENT); }
    __device__ void put2(unsigned at, float x, float y) const { __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(kv4_u32x2, make_float2(x, y)), r, at * 4, 0, KV4_AGENT); }
    __device__ kv4_f32x4 get4(unsigned at) const { return __builtin_bit_cast(kv4_f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at * 4, 0, KV4_AGENT)); }
    __device__ float2 get2(unsigned at) const { return __builtin_bit_cast(float2, __builtin_amdgcn_raw_buffer_load_b64(r, at * 4, 0, KV4_AGENT)); }
};

// ---- few rows: bound by the cache's bytes, or by latency ----
// An item is 16 pairs of one key head of one sequence (32 pairs: 61 rows of 28 heads over 3075 rows 26 -> 49 us, and slower in 31 of 32 other shapes), a unit KV4_UNIT
// keys of an item; the units of all items in a row are dealt to the workgroups in equal runs, so lengths as different as they come leave no workgroup idle
// (one workgroup per item and split of a fixed length: 54 us for 48 conversations of 30 to 16000 rows, and 41 with the best length, where most of a grid sized for
// the longest had nothing to do).  An item that lies in several runs is merged by the workgroup that finishes last.
// (Eight wavefronts per workgroup and units of 256 keys: one token over 650 rows 8.1 -> 9.5 us, the 48 conversations 33.7 -> 40.6.)
// The four wavefronts take tiles of 32 keys in turn, each with its own ref and sum.  A lane reads a quarter of a key's codes with one wide load and one scale byte,
// and the next tile's while it multiplies this one; quarters are contiguous, so step j of the products takes dims g HD/4 + 8j of quarter g, and the keys
// go from registers to the matrix cores.  Values go through the wavefront's own LDS tile (no barrier).

// Where the units of the sequences lie in the row of all (fewer than 2^31): 64 sequences at a time, one per lane.  What is the same for all lanes goes to scalar registers.
__device__ inline int kv4_scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
// a / b, both the same for all lanes (below 2^22 by a reciprocal, whose quotient is off by one at most: a division by a run-time value is forty dependent instructions)
__device__ inline int kv4_div(int a, int b) {
    if (a >= 1 << 22) return kv4_scalar(a / b);
    int q = kv4_scalar((int)((float)a * __builtin_amdgcn_rcpf((float)b)));
    const int r = a - q * b;
    return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}
struct Kv4Units {
    const Kv4AttnArgs& a; int lane, from, before, mine, upto, here;          // sequences from .. from + 63: units before them, of this lane's, up to and with it, of all 64
    Kv4Seq seq;                                              // this lane's
    __device__ Kv4Units(const Kv4AttnArgs& a_, int lane_) : a(a_), lane(lane_), from(0), before(0) { load(); }
    __device__ void load() {
        seq = kv4_seq(a, min(from + lane, a.n_seqs - 1));
        mine = from + lane < a.n_seqs ? (seq.pairs + 15) / 16 * a.d.heads * (blocks(seq.len) + KV4_ITEM_COST) : 0;
        int x = mine;                                        // sums over the lanes below, within rows of 16, then across them
        x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false); x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false); x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false); x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
        upto = x;
        here = __builtin_amdgcn_readlane(upto, 63);
    }
    __device__ void next() { before += here; from += 64; load(); }
    __device__ static int blocks(int len) { return max(1, (len + KV4_UNIT - 1) / KV4_UNIT); }      // (len: at most 2^31 - 256)
    __device__ int total() {                                 // of all sequences; stands at the last 64 of them afterwards
        while (from + 64 < a.n_seqs) next();
        return before + here;
    }
    __device__ int find(int pos, int& base, Kv4Seq& s) {     // the sequence of unit pos (< total()), and its first unit
        if (pos < before) { from = 0; before = 0; load(); }
        while (pos >= before + here) next();
        const int i = __builtin_ctzll(__ballot(pos < before + upto));
        base = before + __builtin_amdgcn_readlane(upto - mine, i);
        s.q0 = __builtin_amdgcn_readlane(seq.q0, i); s.o0 = __builtin_amdgcn_readlane(seq.o0, i); s.rows = __builtin_amdgcn_readlane(seq.rows, i);
        s.pairs = __builtin_amdgcn_readlane(seq.pairs, i); s.len = __builtin_amdgcn_readlane(seq.len, i);
        return from + i;
    }
};

// Workgroups per CU that the kernel is compiled for, with all registers that it wants (with one more per CU it spilled: 37 -> 47 us).  A launch has as many.
template <typename T, int HD> constexpr int kv4_stream_per_cu() { return HD == 128 ? sizeof(T) == 4 ? 2 : 3 : sizeof(T) == 4 ? 3 : 4; }
template <typename T, int HD>
__global__ __launch_bounds__(256, (kv4_stream_per_cu<T, HD>())) void kv4_stream_kernel(Kv4AttnArgs a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1, STEPS = HD / 32, NB = HD / 16, VSTRIDE = kv4_vstride<HD>(), NW = 4;
    constexpr int MSTRIDE = HD + 4;                          // a pair's results in LDS: HD sums, ref, denominator
    constexpr int VB = NW * 32 * VSTRIDE, MB = NW * 16 * MSTRIDE * 4, PLACE = 16 * (HD + 2);
    __shared__ __align__(16) char lds[VB > MB ? VB : MB];
    __shared__ int last;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Kv4Units units(a, threadIdx.x & 63);
    const int total = units.total(), per = kv4_div(total + (int)gridDim.x - 1, gridDim.x);
    const int bytes = kv4_chunk(HD, a.d.block);
    char* const vt = lds + wave * 32 * VSTRIDE;
    float* const mrg = (float*)lds;
    const int stop = (int)min((long long)total, (blockIdx.x + 1ll) * per);
    int pos = (int)min((long long)total, (long long)blockIdx.x * per);
    if (pos >= stop) return;
    // Partials: two places per workgroup, [0] for an item that began before its run, [1] for an item that goes on behind it; a place: [pair][HD] sums, [pair] ref and denominator
    const Kv4Partials ws(a.ws, gridDim.x * (2u * PLACE * 4));
    auto place = [&](int wg, bool begins_there) { return (2u * wg + begins_there) * PLACE; };

    // ---- an item's part in this run: what it is, and the first requests to memory
    struct Item { Kv4Seq s; int seq, ti, h, nb, first, units, begins; } it;
    struct Tile { unsigned k[2][STEPS], v[2][STEPS], kb[2], vb[2]; int e[2]; } now;
    Kv4Raw<T> raw[STEPS];
    Kv4Sight see;
    int k0, end, all, e0, e1, at;
    const int* row;
    auto entries = [&](int from, int lane) {                 // this wavefront's blocks, 64 tiles ahead: entry i of lane i
        const int key = from + 32 * NW * lane;
        e0 = key < end ? row[key >> a.d.shift] : -1;
        e1 = key + 16 < end ? row[(key + 16) >> a.d.shift] : -1;
    };
    auto fetch = [&](Tile& t, int key, int i, unsigned at_code, unsigned at_scale) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int e = __builtin_amdgcn_readlane(half ? e1 : e0, i);
            t.e[half] = e;
            const uint8_t* c = a.pool + ((size_t)(e >= 0 && e < a.d.n_blocks ? e : 0) * a.d.heads + it.h) * bytes;    // (no block: any one's memory, left out below)
            const int r = (key + 16 * half) & (a.d.block - 1);
            const uint8_t *kp = c + r * (HD / 2) + at_code, *vp = c + (a.d.block + r) * (HD / 2) + at_code;       // (scalar base, lane's offset)
            if constexpr (HD == 128) {
                const uint4 x = *(const uint4*)kp, y = *(const uint4*)vp;
                t.k[half][0] = x.x; t.k[half][1] = x.y; t.k[half][2] = x.z; t.k[half][3] = x.w;
                t.v[half][0] = y.x; t.v[half][1] = y.y; t.v[half][2] = y.z; t.v[half][3] = y.w;
            } else {
                const uint2 x = *(const uint2*)kp, y = *(const uint2*)vp;
                t.k[half][0] = x.x; t.k[half][1] = x.y; t.v[half][0] = y.x; t.v[half][1] = y.y;
            }
            t.kb[half] = (c + a.d.block * HD + r * (HD / 32))[at_scale];
            t.vb[half] = (c + a.d.block * HD + (a.d.block + r) * (HD / 32))[at_scale];
        }
    };
    // opens the item at pos (which moves behind its units here); an item of which only its cost without keys lies here has units = 0
    auto open = [&](int lane) {
        const int n16 = lane & 15, g = lane >> 4;
        int base;
        it.seq = units.find(pos, base, it.s);
        it.nb = Kv4Units::blocks(it.s.len);
        const int cost = it.nb + KV4_ITEM_COST, at_item = kv4_div(pos - base, cost), from = pos - base - at_item * cost;
        it.ti = a.tiles > 1 ? kv4_div(at_item, a.d.heads) : 0; it.h = at_item - it.ti * a.d.heads;
        const int n = min(cost - from, stop - pos);
        it.first = max(0, from - KV4_ITEM_COST); it.units = max(0, from + n - KV4_ITEM_COST) - it.first;
        it.begins = pos - from + KV4_ITEM_COST;
        pos += n;
        const int p0 = it.ti * 16;
        // keys of the item: no pair of it sees one from `limit` on, all see those below `all`
        const int limit = a.mask ? it.s.len : it.s.len - it.s.rows + min(p0 + 15, it.s.pairs - 1) / a.group + 1;
        all = it.s.len - it.s.rows + (a.mask ? 0 : p0 / a.group + 1);
        end = (int)min((long long)limit, (long long)(it.first + it.units) * KV4_UNIT);
        row = a.table + (size_t)(a.row_start ? it.seq : a.seq0 + it.seq) * a.max_blocks;
        k0 = it.first * KV4_UNIT + 32 * wave;
        at = 0;
        if (it.units == 0) { end = k0; return; }
        entries(k0, lane);
        kv4_queries<T, HD>(a, it.s, it.h, p0, n16, g, [](int g_, int j) { return g_ * (HD / 4) + 8 * j; }, raw, see);
        if (k0 < end) fetch(now, k0, 0, n16 * (HD / 2) + g * (HD / 8), n16 * (HD / 32) + g * (HD / 4) / 32);
    };
    open(threadIdx.x & 63);
    int due[2] = {-1, -1}; Item due_it[2];       // items to report as arrived: one that began before, one that goes on
    for (bool more = true; more;) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                            // (what follows from it is not kept across items: 80 registers)
    const int lane = tid & 63, n16 = lane & 15, g = lane >> 4;
    kv4_f32x4 o[NB];
    float ref = KV4_REF0, l = 0.f;
    bool far = false;
    unsigned no_number = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) o[b] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
    if (it.units) {
    kv4_bf16x8 qf[STEPS][NP];
#pragma unroll
    for (int j = 0; j < STEPS; ++j) kv4_query_part<T, NP>(a.negate, raw[j], qf[j]);
    for (; k0 < end; k0 += 32 * NW) {                        // (below 2^31: end is, and a step is short of the next block's last row)
        Tile t = now;
        if (++at == 64) { entries(k0 + 32 * NW, lane); at = 0; }
        if (k0 + 32 * NW < end) fetch(now, k0 + 32 * NW, at, n16 * (HD / 2) + g * (HD / 8), n16 * (HD / 32) + g * (HD / 4) / 32);
        // rows that are not held, and scales that say NaN, stay out of the products
        bool plain = k0 + 32 <= all;
        const bool there0 = t.e[0] >= 0 && t.e[0] < a.d.n_blocks, there1 = t.e[1] >= 0 && t.e[1] < a.d.n_blocks;
        const bool odd = t.kb[0] == 255 || t.vb[0] == 255 || t.kb[1] == 255 || t.vb[1] == 255;
        unsigned held = ~0u;                                 // keys that are held
        if (!plain || !there0 || !there1 || __any(odd)) {
            plain = false;
            held = (there0 ? 0xffffu : 0) | (there1 ? 0xffff0000u : 0);
            if (k0 + 32 > it.s.len) held &= (1u << (it.s.len - k0)) - 1;               // (k0 < end <= len)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const bool in = held >> (16 * half + n16) & 1;
                unsigned long long nk = __ballot(in && t.kb[half] == 255), nv = __ballot(in && t.vb[half] == 255);
                if (nk | nv)
                    for (int i = 0; i < 64; ++i) {           // lane i: key i % 16, quarter i / 16
                        const unsigned dims = nk >> i & 1 ? 15u : nv >> i & 1 ? 1u << ((i >> 4) * (HD / 4) / 32) : 0u;
                        if (dims)
                            if (see.of(k0 + 16 * half + (i & 15)) & 1) no_number |= dims;
                    }
                if (!in || t.kb[half] == 255) t.kb[half] = 127;
                if (!in || t.vb[half] == 255) t.vb[half] = 127;
            }
        }
        kv4_f32x4 x[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const float ks = __uint_as_float(t.kb[half] << 23), vs = __uint_as_float(t.vb[half] << 23);
#pragma unroll
            for (int j = 0; j < STEPS; ++j) *(kv4_bf16x8*)(vt + (16 * half + n16) * VSTRIDE + (g * (HD / 4) + 8 * j) * 2) = kv4_expand(t.v[half][j], vs);
            x[half] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                const kv4_bf16x8 kf = kv4_expand(t.k[half][j], ks);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
                    x[half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[j][p], x[half], 0, 0, 0);
            }
        }
        kv4_bf16x8 pf[1][NP];
        if (!plain) kv4_hide(x, see.of(k0) & held, g);
        const float mx = kv4_top(x) * a.scale2;
        if (__any(mx > ref + KV4_SLACK)) kv4_follow(mx, o, ref, l, far);
        kv4_weights<2, NP>(x, a.scale2, ref, far, l, pf);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const kv4_bf16x8 vf = kv4_vfrag<HD>(vt, b, lane);
#pragma unroll
            for (int p = NP - 1; p >= 0; --p)
                o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[0][p], o[b], 0, 0, 0);
        }
    }
    }
    const Item done = it;
    more = pos < stop;
    if (more) open(lane);                                    // (its requests travel while this one's results are put together)
    if (done.units == 0) continue;
    // ---- the wavefronts' results, 16 pairs at a time
    asm volatile("" : "+v"(tid));
    const int n16_ = tid & 15, g_ = tid >> 4 & 3, p0 = done.ti * 16, count = min(16, done.s.pairs - p0);
    const bool whole = done.units == done.nb, begins_here = done.first == 0;
    const unsigned part = place(blockIdx.x, begins_here);
    l = kv4_xsum(l);
    kv4_poison<NB>(no_number, o);
    kv4_lds_barrier();
    float* dst = mrg + (wave * 16 + n16_) * MSTRIDE;
#pragma unroll
    for (int b = 0; b < NB; ++b) *(kv4_f32x4*)(dst + 16 * b + 4 * g_) = o[b];
    if (g_ == 0) *(float2*)(dst + HD) = make_float2(ref, l);
    kv4_lds_barrier();
    for (int i = tid; i < 16 * HD / 4; i += 256) {
        const int pr = i / (HD / 4), c = 4 * (i % (HD / 4));
        if (pr >= count) break;
        float mx = KV4_REF0, den = 0.f;
        kv4_f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) mx = fmaxf(mx, mrg[(w * 16 + pr) * MSTRIDE + HD]);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float* src = mrg + (w * 16 + pr) * MSTRIDE;
            const float2 st = *(const float2*)(src + HD);
            const float f = __builtin_amdgcn_exp2f(st.x - mx);
            den += st.y * f; sum += *(const kv4_f32x4*)(src + c) * f;
        }
        if (whole) kv4_store4<T, HD>(a, done.s, done.h, p0 + pr, c, sum * (den == 0.f ? 0.f : 1.f / den));    // (a row that sees nothing: zeros)
        else {
            ws.put4(part + pr * HD + c, sum);
            if (c == 0) ws.put2(part + 16 * HD + 2 * pr, mx, den);
        }
    }
    kv4_lds_barrier();                                       // (the next item's values go where these results were)
    if (!whole) { if (begins_here) { due_it[1] = done; due[1] = 0; } else { due_it[0] = done; due[0] = 0; } }
    }
    // ---- arrivals, all at the end of the run: the partials are acknowledged before the count that shows them
    if (due[0] < 0 && due[1] < 0) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    for (int w = 0; w < 2; ++w) {
    if (due[w] < 0) continue;
    const int tid = threadIdx.x;
    const Item x = due_it[w];
    const Kv4Seq s = x.s;
    const int h = x.h, p0 = x.ti * 16, count = min(16, s.pairs - p0);
    // (counted where the item begins: one at most begins in a run and goes on behind it)
    const int w0 = kv4_div(x.begins, per), parts = kv4_div(x.begins + x.nb - 1, per) - w0 + 1;
    if (tid == 0) last = __hip_atomic_fetch_add(&a.cnt[w0], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
    __syncthreads();
    const bool mine = last;
    __syncthreads();
    if (!mine) continue;
    if (tid == 0) __hip_atomic_store(&a.cnt[w0], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // Merge, in the order of the keys (the same whoever merges): a thread takes four dims of a pair and eight partials at a time, all requested at once with their
    // refs and denominators; where there are fewer pairs than threads for them, several threads share the partials and add up in LDS.
    int sh_pr = 0;                                           // pairs padded to a power of two
    while ((1 << sh_pr) < count) ++sh_pr;
    const int elems = HD / 4 << sh_pr, groups = max(1, 256 / elems);
    for (int e = tid; e < max(256, elems); e += 256) {
        const int el = e & (elems - 1), grp = elems < 256 ? e / elems : 0, pr = min(el / (HD / 4), count - 1), c = 4 * (el % (HD / 4));
        float mx = KV4_REF0, den = 0.f;
        kv4_f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int q0 = grp; q0 < parts; q0 += 8 * groups) {
            kv4_f32x4 v[8];
            float2 st[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int q = min(q0 + u * groups, parts - 1);
                const unsigned from = place(w0 + q, q == 0);
                v[u] = ws.get4(from + pr * HD + c); st[u] = ws.get2(from + 16 * HD + 2 * pr);
            }
            float to = mx;
#pragma unroll
            for (int u = 0; u < 8; ++u) { if (q0 + u * groups >= parts) st[u] = make_float2(KV4_REF0, 0.f); to = fmaxf(to, st[u].x); }
            const float f = __builtin_amdgcn_exp2f(mx - to);
            den *= f; sum *= f; mx = to;
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (q0 + u * groups < parts) { const float w = __builtin_amdgcn_exp2f(st[u].x - to); den += st[u].y * w; sum += v[u] * w; }
        }
        if (groups > 1) {
            float* at = mrg + e * 6;                         // (256 of them)
            at[0] = mx; at[1] = den;
#pragma unroll
            for (int i = 0; i < 4; ++i) at[2 + i] = sum[i];
            __syncthreads();
            if (grp == 0) {
                for (int u = 1; u < groups; ++u) {
                    const float* o = mrg + (u * elems + el) * 6;
                    const float to = fmaxf(mx, o[0]), f = __builtin_amdgcn_exp2f(mx - to), w = __builtin_amdgcn_exp2f(o[0] - to);
                    den = den * f + o[1] * w; mx = to;
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = sum[i] * f + o[2 + i] * w;
                }
            }
        }
        if (grp == 0 && el / (HD / 4) < count) kv4_store4<T, HD>(a, s, h, p0 + pr, c, sum * (den == 0.f ? 0.f : 1.f / den));
    }
    __syncthreads();
    }
}

// ---- many rows (prompts): bound by the matrix cores and the vector work of the softmax ----
// A workgroup is one key head of one sequence and 64 pairs, 16 per wavefront; the cache is expanded to bf16 once per workgroup, 64 keys at a time, into two
// LDS buffers in turn (one barrier per tile).  A thread expands a quarter of one key and of one value: one wide load and one scale each, requested
// a tile ahead.
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void kv4_rows_kernel(Kv4AttnArgs a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1, STEPS = HD / 32, NB = HD / 16, KT = 64, VSTRIDE = kv4_vstride<HD>(), KSTRIDE = kv4_kstride<HD>();
    constexpr int BUF = KT * (VSTRIDE + KSTRIDE), NG = HD / 32;
    extern __shared__ __align__(16) char kv4_lds[];
    // Bits of a tile's keys: [0] any of the others; [1] not held; [2] the key's scale says NaN; [3 ..] those of the values' groups.  Three tiles in turn: written
    // before a tile's barrier, read behind it, cleared behind the next one.
    unsigned long long (*const odd)[3 + NG] = (unsigned long long (*)[3 + NG])(kv4_lds + 2 * BUF);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    // The last rows of every sequence, which see most, first (by row tile alone, what starts last may be long: four prompts of 641 to 3008 rows 199 us instead of 175);
    // sequences in turn, or each would always meet the same shader engine of a chiplet (405 us)
    const int sh = blockIdx.x;
    if (sh >= a.n_seqs * a.d.heads) return;
    const int h = sh % a.d.heads, seq = (int)((sh / a.d.heads + blockIdx.y) % a.n_seqs);
    const Kv4Seq s = kv4_seq(a, seq);
    const int pairs = s.pairs, ti = (pairs + 63) / 64 - 1 - (int)blockIdx.y, p0 = ti * 64, w0 = p0 + wave * 16;
    if (ti < 0) return;
    const int limit = a.mask ? s.len : s.len - s.rows + min(p0 + 63, pairs - 1) / a.group + 1;
    const int mine = w0 >= pairs ? 0 : a.mask ? s.len : s.len - s.rows + min(w0 + 15, pairs - 1) / a.group + 1;       // of this wavefront
    const int all = s.len - s.rows + (a.mask ? 0 : w0 / a.group + 1);
    const int* row = a.table + (size_t)(a.row_start ? seq : a.seq0 + seq) * a.max_blocks;
    const int bytes = kv4_chunk(HD, a.d.block);
    if (threadIdx.x < 3 * (3 + NG)) ((unsigned long long*)odd)[threadIdx.x] = 0;
    __syncthreads();

    const int kr = threadIdx.x >> 2, kq = threadIdx.x & 3;   // this thread's key of a tile and quarter
    unsigned kc[STEPS], vc[STEPS], kb, vb;
    bool in;
    auto entry = [&](int k0) { return k0 + kr < s.len ? row[(k0 + kr) >> a.d.shift] : -1; };
    int next = entry(0);                                     // block of the tile that is fetched next, a tile ahead of it
    auto fetch = [&](int k0) {
        const int key = k0 + kr, e = next;
        next = entry(k0 + KT);
        in = e >= 0 && e < a.d.n_blocks;
        const uint8_t* c = a.pool + ((size_t)(in ? e : 0) * a.d.heads + h) * bytes;
        const int r = key & (a.d.block - 1);
        const uint8_t *kp = c + r * (HD / 2) + kq * (HD / 8), *vp = kp + a.d.block * (HD / 2), *sp = c + a.d.block * HD + r * (HD / 32) + kq * (HD / 4) / 32;
        if constexpr (HD == 128) {
            const uint4 x = *(const uint4*)kp, y = *(const uint4*)vp;
            kc[0] = x.x; kc[1] = x.y; kc[2] = x.z; kc[3] = x.w; vc[0] = y.x; vc[1] = y.y; vc[2] = y.z; vc[3] = y.w;
        } else {
            const uint2 x = *(const uint2*)kp, y = *(const uint2*)vp;
            kc[0] = x.x; kc[1] = x.y; vc[0] = y.x; vc[1] = y.y;
        }
        kb = sp[0]; vb = sp[a.d.block * (HD / 32)];
    };
    fetch(0);
    kv4_bf16x8 qf[STEPS][NP];
    Kv4Sight see;
    {
        Kv4Raw<T> raw[STEPS];
        kv4_queries<T, HD>(a, s, h, min(w0, pairs - 1), n16, g, [](int g_, int j) { return 32 * j + 8 * g_; }, raw, see);
    #pragma unroll
    for (int j = 0; j < STEPS; ++j) kv4_query_part<T, NP>(a.negate, raw[j], qf[j]);
    }
    kv4_f32x4 o[NB];
    float ref = KV4_REF0, l = 0.f;
    bool far = false;
    unsigned no_number = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) o[b] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
    int buf = 0, turn = 0;
    for (int k0 = 0; k0 < limit; k0 += KT, buf ^= 1, turn = turn == 2 ? 0 : turn + 1) {
        char* const kt = kv4_lds + buf * BUF; char* const vt = kt + KT * KSTRIDE;
        if (!in || kb == 255 || vb == 255) {
            const unsigned long long bit = 1ull << kr;
            atomicOr(&odd[turn][0], bit);
            atomicOr(&odd[turn][!in ? 1 : kb == 255 ? 2 : 3 + kq * (HD / 4) / 32], bit);
            if (in && kb == 255 && vb == 255) atomicOr(&odd[turn][3 + kq * (HD / 4) / 32], bit);
        }
        const float ks = __uint_as_float((in && kb != 255 ? kb : 127u) << 23), vs = __uint_as_float((in && vb != 255 ? vb : 127u) << 23);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            *(kv4_bf16x8*)(kt + kr * KSTRIDE + (kq * (HD / 4) + 8 * j) * 2) = kv4_expand(kc[j], ks);
            *(kv4_bf16x8*)(vt + kr * VSTRIDE + (kq * (HD / 4) + 8 * j) * 2) = kv4_expand(vc[j], vs);
        }
        __syncthreads();
        if (k0 + KT < limit) fetch(k0 + KT);
        if (threadIdx.x < 3 + NG) odd[turn == 0 ? 2 : turn - 1][threadIdx.x] = 0;
        if (k0 >= mine) continue;
        kv4_f32x4 x[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            x[c] = kv4_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < STEPS; ++j) {
                const kv4_bf16x8 kf = *(const kv4_bf16x8*)(kt + (16 * c + n16) * KSTRIDE + (32 * j + 8 * g) * 2);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
                    x[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[j][p], x[c], 0, 0, 0);
            }
        }
        const bool any = odd[turn][0] != 0, plain = k0 + KT <= all && !any;
        unsigned long long gone = 0;
        if (any) {
            gone = odd[turn][1];
            for (int b = 0; b <= NG; ++b)
                for (unsigned long long w = odd[turn][2 + b]; w; w &= w - 1) {
                    if (see.of(k0 + __builtin_ctzll(w)) & 1) no_number |= b ? 1u << (b - 1) : 15u;
                }
        }
        kv4_bf16x8 pf[2][NP];
        if (!plain) kv4_hide(x, see.of(k0) & ~gone, g);
        const float mx = kv4_top(x) * a.scale2;
        if (__any(mx > ref + KV4_SLACK)) kv4_follow(mx, o, ref, l, far);
        kv4_weights<4, NP>(x, a.scale2, ref, far, l, pf);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const kv4_bf16x8 vf = kv4_vfrag<HD>(vt + 32 * k * VSTRIDE, b, lane);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)
                    o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[k][p], o[b], 0, 0, 0);
            }
    }
    const float den = kv4_xsum(l), inv = den == 0.f ? 0.f : 1.f / den;    // a row that sees nothing: zeros
    kv4_poison<NB>(no_number, o);
    const int pr = w0 + n16;
    if (pr < pairs) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
            kv4_store4<T, HD>(a, s, h, pr, 16 * b + 4 * g, o[b] * inv);
    }
}

// ---- more rows than fill the chip ----
// As above with products of 32 x 32: 32 pairs per wavefront, 128 per workgroup, for half the reads of LDS per product.  Half as many instructions of the matrix cores leave
// more room for vector work beside them (per SIMD, 128 multiply-adds beside the products of two wavefronts: 842 cycles with 16 x 16, 723 with 32 x 32).  Four
// prompts of 641 to 3008 rows, 32 heads: 160 us, 0.82 PFLOP/s (tiles of 16 x 16, two per wavefront: 175; scores a tile ahead of the weights 173; two workgroups' work
// in one, keys shared: 223; 32 keys per tile and three wavefronts per SIMD: 177; 64 pairs per wavefront: registers spill).
// A lane has one pair and, of every eight keys, the four of its half.  Keys of KS at a time go through the softmax (32 where the operand parts of 64 would not
// fit the registers).  What GROUP products read from LDS is requested a group ahead (left to the compiler, each read stood before its product: 168 -> 160 us).
template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void kv4_rows32_kernel(Kv4AttnArgs a) {
    constexpr int NP = sizeof(T) == 4 ? 3 : 1, KS = sizeof(T) == 4 ? 32 : 64, STEPS = HD / 16, NB = HD / 32, KT = 64, VSTRIDE = kv4_vstride32<HD>(), KSTRIDE = kv4_kstride<HD>();
    constexpr int BUF = KT * (VSTRIDE + KSTRIDE), NG = HD / 32, NC = HD / 32, GROUP = NP == 1 ? 4 : 2;
    extern __shared__ __align__(16) char kv4_lds[];
    // Bits of a tile's keys as above
    unsigned long long (*const odd)[3 + NG] = (unsigned long long (*)[3 + NG])(kv4_lds + 2 * BUF);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n32 = lane & 31, hh = lane >> 5;
    const int sh = blockIdx.x;
    if (sh >= a.n_seqs * a.d.heads) return;
    const int h = sh % a.d.heads, seq = (int)((sh / a.d.heads + blockIdx.y) % a.n_seqs);
    const Kv4Seq s = kv4_seq(a, seq);
    const int pairs = s.pairs, ti = (pairs + 127) / 128 - 1 - (int)blockIdx.y, p0 = ti * 128, w0 = p0 + wave * 32;
    if (ti < 0) return;
    const int limit = a.mask ? s.len : s.len - s.rows + min(p0 + 127, pairs - 1) / a.group + 1;
    const int mine = w0 >= pairs ? 0 : a.mask ? s.len : s.len - s.rows + min(w0 + 31, pairs - 1) / a.group + 1;       // of this wavefront
    const int all = s.len - s.rows + (a.mask ? 0 : w0 / a.group + 1);
    const int* row = a.table + (size_t)(a.row_start ? seq : a.seq0 + seq) * a.max_blocks;
    const int bytes = kv4_chunk(HD, a.d.block);
    if (threadIdx.x < 3 * (3 + NG)) ((unsigned long long*)odd)[threadIdx.x] = 0;
    __syncthreads();

    // a wavefront's 16 keys lie in one block: the address is the same for all lanes but for an offset
    const int kr = threadIdx.x >> 2, kq = threadIdx.x & 3;   // this thread's key of a tile and quarter
    const unsigned at_code = (lane >> 2) * (HD / 2) + kq * (HD / 8), at_scale = (lane >> 2) * (HD / 32) + kq * (HD / 4) / 32;
    struct Part { unsigned c[NC], b; } kp, vp;               // a quarter of a key and of a value: codes, scale
    bool in;
    auto entry = [&](int k0) { const int key = k0 + 16 * wave; return key < s.len ? row[key >> a.d.shift] : -1; };
    int next = entry(0);                                     // block of the tile that is fetched next, a tile ahead of it
    auto get = [&](Part& t, const uint8_t* c, int r) {
        const uint8_t* p = c + r * (HD / 2) + at_code;
        if constexpr (HD == 128) { const uint4 x = *(const uint4*)p; t.c[0] = x.x; t.c[1] = x.y; t.c[2] = x.z; t.c[3] = x.w; }
        else { const uint2 x = *(const uint2*)p; t.c[0] = x.x; t.c[1] = x.y; }
        t.b = (c + a.d.block * HD + r * (HD / 32))[at_scale];
    };
    auto fetch = [&](int k0) {
        const int e = kv4_scalar(next), r = (k0 + 16 * wave) & (a.d.block - 1);
        next = entry(k0 + KT);
        in = e >= 0 && e < a.d.n_blocks;
        const uint8_t* c = a.pool + ((size_t)(in ? e : 0) * a.d.heads + h) * bytes;
        get(kp, c, r);
        get(vp, c, a.d.block + r);
    };
    // Values lie in LDS in pieces of eight dims, of every four pieces in an order of the key's: rows 16 banks apart, so neither writes nor reads of four keys meet
    int to_v[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) to_v[j] = kr * VSTRIDE + (((kq * NC + j) ^ (kr & 3)) * 16);
    const int from_v = (4 * hh + (lane & 15) / 4) * VSTRIDE + (((lane >> 4 & 1) * 2 + (lane & 3) / 2) ^ ((lane & 15) / 4)) * 16 + (lane & 1) * 8;
    fetch(0);
    kv4_bf16x8 qf[STEPS][NP];
    Kv4Sight see;
    {
        const int pair = min(w0 + n32, pairs - 1), i = a.group == 1 ? pair : pair / a.group, hq = h * a.group + pair - i * a.group;
        see.below = s.len - s.rows + (a.mask ? 0 : i + 1);
        see.bits = a.mask ? a.mask[s.o0 + i] : 0;
        const T* q = (const T*)a.q + (long long)(s.q0 + i) * a.ldq + (long long)hq * HD + 8 * hh;
        Kv4Raw<T> raw[1][STEPS];
#pragma unroll
        for (int j = 0; j < STEPS; ++j) raw[0][j] = *(const Kv4Raw<T>*)(q + 16 * j);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) kv4_query_part<T, NP>(a.negate, raw[0][j], qf[j]);
    }
    kv4_f32x16 o[NB];
    float ref = KV4_REF0, l = 0.f;
    bool far = false;
    unsigned no_number = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    auto noted = [&](unsigned long long w, unsigned dims, int k0) {
        for (; w; w &= w - 1) if (see.of(k0 + __builtin_ctzll(w)) & 1) no_number |= dims;
    };
    int buf = 0, turn = 0;
    for (int k0 = 0; k0 < limit; k0 += KT, buf ^= BUF, turn = turn == 2 ? 0 : turn + 1) {
        unsigned long long* const w = odd[turn];
        char* const kt = kv4_lds + buf; char* const vt = kt + KT * KSTRIDE;
        {                                                    // rows that are not held and scales that say NaN stay out of the products
            const bool held = in && k0 + kr < s.len;
            if (!held || kp.b == 255 || vp.b == 255) {
                const unsigned long long bit = 1ull << kr;
                atomicOr(&w[0], bit);
                if (!held || kp.b == 255) atomicOr(&w[held ? 2 : 1], bit);
                if (held && vp.b == 255) atomicOr(&w[3 + kq * (HD / 4) / 32], bit);
            }
            const float ks = __uint_as_float((held && kp.b != 255 ? kp.b : 127u) << 23), vs = __uint_as_float((held && vp.b != 255 ? vp.b : 127u) << 23);
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                *(kv4_bf16x8*)(kt + kr * KSTRIDE + (kq * NC + j) * 16) = kv4_expand(kp.c[j], ks);
                *(kv4_bf16x8*)(vt + to_v[j]) = kv4_expand(vp.c[j], vs);
            }
        }
        __syncthreads();
        if (k0 + KT < limit) fetch(k0 + KT);
        if (threadIdx.x < 3 + NG) odd[turn == 0 ? 2 : turn - 1][threadIdx.x] = 0;
        if (k0 >= mine) continue;
        const unsigned long long any = w[0];                 // (asked for before the keys, looked at behind their products)
        unsigned long long vis = 0;
        bool plain = k0 + KT <= all;
#pragma unroll
        for (int part = 0; part < KT / KS; ++part) {
            kv4_f32x16 x[KS / 32];
            kv4_bf16x8 f[2][GROUP], vf[2][GROUP];
#pragma unroll
            for (int c = 0; c < KS / 32; ++c)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[c][i] = 0.f;
            auto keys = [&](int first, kv4_bf16x8 (&to)[GROUP]) {
#pragma unroll
                for (int i = first; i < first + GROUP; ++i)
                    to[i - first] = *(const kv4_bf16x8*)(kt + (part * KS + 32 * (i % (KS / 32)) + n32) * KSTRIDE + (16 * (i / (KS / 32)) + 8 * hh) * 2);
            };
            auto values = [&](int first, kv4_bf16x8 (&to)[GROUP]) {
#pragma unroll
                for (int i = first; i < first + GROUP; ++i) {
                    typedef __attribute__((address_space(3))) kv4_s16x4* lds_p;
                    const char* src = vt + from_v + (part * KS + 16 * (i / NB)) * VSTRIDE + 64 * (i % NB);
                    union { kv4_s16x4 s[2]; kv4_bf16x8 f; } v;
                    v.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)src);
                    v.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_p)(src + 8 * VSTRIDE));
                    to[i - first] = v.f;
                }
            };
            keys(0, f[0]);
#pragma unroll
            for (int i = 0; i < KS / 32 * STEPS; i += GROUP) {
                if (i + GROUP < KS / 32 * STEPS) keys(i + GROUP, f[i / GROUP + 1 & 1]); else values(0, vf[0]);
#pragma unroll
                for (int u = 0; u < GROUP; ++u)
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        x[(i + u) % (KS / 32)] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i / GROUP & 1][u], qf[(i + u) / (KS / 32)][p], x[(i + u) % (KS / 32)], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (part == 0 && (any || !plain)) {
                unsigned long long gone = 0;
                if (any) {
                    gone = w[1]; noted(w[2], 15u, k0);
                    for (int b = 0; b < NG; ++b) noted(w[3 + b], 1u << b, k0);
                }
                plain = false;
                vis = (see.of(k0) & ~gone) >> 4 * hh;
            }
            if (!plain)
#pragma unroll
                for (int c = 0; c < KS / 32; ++c) {
                    const unsigned on = (unsigned)(vis >> (part * KS + 32 * c));
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[c][i] = ((int)(on << (31 - 8 * (i / 4) - (i & 3))) >> 31) ? x[c][i] : -INFINITY;
                }
            float mx = x[0][0];
#pragma unroll
            for (int i = 1; i < KS / 2; ++i) mx = fmaxf(mx, x[i / 16][i & 15]);
            mx *= a.scale2;
            if (__any(mx > ref + KV4_SLACK)) {
                const auto other = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                const float up = fmaxf(ref, fmaxf(__uint_as_float(other[0]), __uint_as_float(other[1]))), f = __builtin_amdgcn_exp2f(ref - up);
                ref = up; far = kv4_far(up);
                l *= f;
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[b][i] *= f;
            }
            float sum[4] = {0.f, 0.f, 0.f, 0.f}, scale2 = a.scale2, from = ref;
            if (far) {
#pragma unroll
                for (int i = 0; i < KS / 2; ++i) x[i / 16][i & 15] = kv4_rounded(x[i / 16][i & 15], scale2, ref);
                scale2 = 1.f; from = 0.f;
            }
            kv4_bf16x8 pf[KS / 16][NP];
#pragma unroll
            for (int k = 0; k < KS / 16; ++k) {
                float e[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) { e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[k / 2][8 * (k & 1) + i], scale2, -from)); sum[i & 3] += e[i]; }
                kv4_parts<NP>(e, pf[k]);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
            for (int i = 0; i < KS / 16 * NB; i += GROUP) {
                if (i + GROUP < KS / 16 * NB) values(i + GROUP, vf[i / GROUP + 1 & 1]);
#pragma unroll
                for (int u = 0; u < GROUP; ++u)
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p)
                        o[(i + u) % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i / GROUP & 1][u], pf[(i + u) / NB][p], o[(i + u) % NB], 0, 0, 0);
            }
        }
    }
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    const float den = __uint_as_float(both[0]) + __uint_as_float(both[1]), inv = den == 0.f ? 0.f : 1.f / den;       // a row that sees nothing: zeros
    if (w0 + n32 < pairs) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const kv4_f32x4 x = no_number >> b & 1 ? kv4_f32x4{kv4_nan(), kv4_nan(), kv4_nan(), kv4_nan()} : kv4_f32x4{o[b][4 * q], o[b][4 * q + 1], o[b][4 * q + 2], o[b][4 * q + 3]} * inv;
                kv4_store4<T, HD>(a, s, h, w0 + n32, 32 * b + 8 * q + 4 * hh, x);
            }
    }
}

}  // namespace hivis
