// Host side of the operators that work on callers' tensors: the paged cache in 4 bits and the log probabilities.  The C ABI is declared and documented in include/hivis.h.
#include "hivis.h"
#include "hivis_kv4.h"
#include "hivis_logprobs.h"
#include "hivis_ops.h"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <string>

using namespace hivis;

namespace hivis {

int op_fail(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap; va_start(ap, fmt); vsnprintf(buf, sizeof buf, fmt, ap); va_end(ap);
    set_thread_error(buf);
    return code;
}

}  // namespace hivis

namespace {

#define OP_TRY(expr)                                                                                              \
    do {                                                                                                          \
        hipError_t e_ = (expr);                                                                                   \
        if (e_ != hipSuccess) return op_fail(HIVIS_EHIP, "%s failed: %s", #expr, hipGetErrorString(e_));          \
    } while (0)
#define CHECK(cond, ...) do { if (!(cond)) return op_fail(HIVIS_EINVAL, __VA_ARGS__); } while (0)

// Memory of the current device: the kernels run there, and a host address or another device's would fault.
int check_device(const void* p, const char* what, int dev) {
    hipPointerAttribute_t at{};
    const hipError_t e = hipPointerGetAttributes(&at, p);
    if (e != hipSuccess) { (void)hipGetLastError(); return op_fail(HIVIS_EINVAL, "%s is not device memory", what); }
    if (at.type != hipMemoryTypeDevice && at.type != hipMemoryTypeManaged) return op_fail(HIVIS_EINVAL, "%s is not device memory", what);
    if (at.device != dev) return op_fail(HIVIS_EINVAL, "%s is on device %d, the current device is %d", what, at.device, dev);
    return HIVIS_OK;
}
struct Named { const void* p; const char* name; };
int check_devices(std::initializer_list<Named> list) {
    int dev = 0;
    OP_TRY(hipGetDevice(&dev));
    for (const Named& n : list)
        if (n.p) if (int rc = check_device(n.p, n.name, dev)) return rc;
    return HIVIS_OK;
}
bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int check_shape(const hivis_kv4_shape* s, Kv4Dims* d) {
    CHECK(s, "null shape");
    CHECK(s->head_dim == 64 || s->head_dim == 128, "head_dim %d not in {64,128}", s->head_dim);
    CHECK(s->n_kv_heads >= 1 && s->n_kv_heads <= 65535, "n_kv_heads %d outside [1,65535]", s->n_kv_heads);
    CHECK(s->block_tokens >= 16 && s->block_tokens <= 256 && !(s->block_tokens & (s->block_tokens - 1)), "block_tokens %d not in {16,32,64,128,256}", s->block_tokens);
    CHECK(s->n_blocks >= 1 && (long long)s->n_blocks * s->block_tokens <= 0x7fffffffLL, "n_blocks %d: the slots of a pool must be in 1..2^31-1", s->n_blocks);
    *d = Kv4Dims{s->n_kv_heads, s->head_dim, s->block_tokens, __builtin_ctz(s->block_tokens), s->n_blocks};
    return HIVIS_OK;
}

int check_rows(const void* k, const void* v, int dtype, const Kv4Dims& d, long long row, long long head, int n) {
    CHECK(dtype == HIVIS_F32 || dtype == HIVIS_BF16, "dtype %d unknown", dtype);
    CHECK(n >= 0 && n <= 1 << 30 && (long long)n * d.heads <= 0x7fffffffLL, "n_rows %d (2^30 at most) x n_kv_heads %d", n, d.heads);
    CHECK(row % 8 == 0 && head % 8 == 0, "row and head strides must be multiples of 8 values (%lld, %lld)", row, head);
    CHECK(row >= 0 && head >= d.hd, "strides %lld, %lld: rows of a head are head_dim values side by side", row, head);
    CHECK(aligned(k, 16) && aligned(v, 16), "rows must start at multiples of 16 bytes");
    return HIVIS_OK;
}

}  // namespace

namespace hivis {

// Slots beyond PLAN_FUSED rows are filled by a launch of their own
constexpr int PLAN_FUSED = 4096;
int kv4_plan_launch(hipStream_t st, PlanArgs a) {
    a.fill = a.max_rows <= PLAN_FUSED;
    // a thread per sequence, or for four of the blocks that the rows can take; a wavefront alone needs no barriers (48 sequences of 6 rows: 7.4 us, 9.9 in 14 wavefronts; 400 of up
    // to 700 rows: 23 us in 7, 17 in 16)
    const long long blocks = std::min<long long>(a.n_blocks, a.n + ((long long)a.max_rows >> a.shift));
    const int threads = (int)std::min<long long>(PLAN_MAX, std::max<long long>(a.n, blocks / 4)), waves = std::max((threads + 63) / 64, a.fill ? std::min(a.max_rows / 256, PLAN_MAX / 64) : 1);
    hipLaunchKernelGGL(kv4_plan_kernel, dim3(1), dim3(64 * waves), 0, st, a);
    if (!a.fill) hipLaunchKernelGGL(kv4_plan_slots_kernel, dim3((unsigned)(((long long)a.max_rows + 255) / 256)), dim3(256), 0, st, a);
    OP_TRY(hipGetLastError());
    return HIVIS_OK;
}

// Four rows per thread where that leaves two workgroups to a CU, one where there are fewer (32 rows of 40 heads: latency)
static bool rows_by_four(const RowsArgs& a, dim3* grid) {
    const unsigned x = (unsigned)((2LL * a.d.heads * (a.d.hd / 8) + 255) / 256);
    const bool four = (long long)x * (a.n / 4) >= 512;
    *grid = dim3(x, (unsigned)std::min(65535, four ? (a.n + 3) / 4 : a.n));
    return four;
}

int kv4_append_launch(hipStream_t st, int type, const RowsArgs& a) {
    if (a.n == 0) return HIVIS_OK;
    dim3 grid;
    const bool four = rows_by_four(a, &grid);
#define KV4_APPEND(T_) do { if (four) hipLaunchKernelGGL((kv4_append_kernel<T_, 4>), grid, dim3(256), 0, st, a); else hipLaunchKernelGGL((kv4_append_kernel<T_, 1>), grid, dim3(256), 0, st, a); } while (0)
    if (type == KV4_ROWS_F32) KV4_APPEND(float);
    else if (type == KV4_ROWS_BF16) KV4_APPEND(__bf16);
    else KV4_APPEND(Kv4Halves);
#undef KV4_APPEND
    OP_TRY(hipGetLastError());
    return HIVIS_OK;
}

int kv4_read_launch(hipStream_t st, int type, const RowsArgs& a) {
    if (a.n == 0) return HIVIS_OK;
    dim3 grid;
    const bool four = rows_by_four(a, &grid);
#define KV4_READ(T_) do { if (four) hipLaunchKernelGGL((kv4_read_kernel<T_, 4>), grid, dim3(256), 0, st, a); else hipLaunchKernelGGL((kv4_read_kernel<T_, 1>), grid, dim3(256), 0, st, a); } while (0)
    if (type == KV4_ROWS_F32) KV4_READ(float);
    else KV4_READ(__bf16);
#undef KV4_READ
    OP_TRY(hipGetLastError());
    return HIVIS_OK;
}

// How a call is cut: kernel, pairs per workgroup in sixty-fours (0: the stream kernel; 1: rows; 2: rows32), row tiles of a sequence at most, workgroups.
// The kernel is the one with the shortest estimate, in us; all from calls of 1 to 256 key heads, 1 to 3000 rows, 64 to 6000 cached rows:
//   stream: 8 us to open, merge and close (5.5 where no item is cut), and its 128-key units (16 pairs; two for each item) at the rate that a full chip reached;
//   rows:   5.5 us, and the longer of its 64-key tiles one after the other (few workgroups: their latency) and all steps of 64 pairs x 64 keys at the full rate.
// 61 rows of 28 heads over 3000 rows: stream 26 us, rows 112; 128 rows of 32 heads over 628: 16 and 21; 256 rows of 32 heads over themselves: 14, 11 and 12 (rows32);
// 1024 rows of 32 heads: 57, 31 and 34; 2000 rows x 4 of 32 heads: rows 253, rows32 183 (fp32 383 and 344; heads of 64 dims 120 and 100).
struct Kv4Plan { int rt, tiles, wgs; long long items; };
static Kv4Plan kv4_plan_attend(const Kv4Dims& d, bool f32, int group, int n_seqs, int max_rows, int max_len) {
    const long long pairs = (long long)max_rows * group, sh = (long long)n_seqs * d.heads;
    const int form = (d.hd == 128 ? 0 : 1) + (f32 ? 2 : 0);
    static const double unit_rate[4] = {350, 600, 260, 400}, tile_us[2][4] = {{1.5, 0.9, 2.5, 1.45}, {1.7, 1.15, 3.3, 2.05}}, step_rate[2][4] = {{255, 560, 172, 335}, {365, 670, 192, 345}};
    const double keys = std::max(1.0, max_len - 0.5 * max_rows);         // that a row sees on average
    Kv4Plan p{};
    p.tiles = (int)((pairs + 15) / 16);
    p.items = sh * p.tiles;
    p.wgs = (int)std::min<double>(256 * (f32 ? d.hd == 128 ? kv4_stream_per_cu<float, 128>() : kv4_stream_per_cu<float, 64>() : d.hd == 128 ? kv4_stream_per_cu<__bf16, 128>() : kv4_stream_per_cu<__bf16, 64>()),
                                  (double)p.items * (std::max(1, (int)(((long long)max_len + KV4_UNIT - 1) / KV4_UNIT)) + KV4_ITEM_COST));
    double best = (max_len > KV4_UNIT ? 8.0 : 5.5) + p.items * (keys / KV4_UNIT + 0.5 + KV4_ITEM_COST) / unit_rate[form];
    for (int rt = 1; rt <= 2; ++rt) {
        const long long tiles = (pairs + 64 * rt - 1) / (64 * rt);
        const double us = 5.5 + std::max((max_len + 63) / 64 * tile_us[rt - 1][form], sh * tiles * rt * (keys / 64 + 0.5) / step_rate[rt - 1][form]);
        if (us < best) { best = us; p.rt = rt; p.tiles = (int)tiles; }
    }
    return p;
}
// A workspace: counters, of the same number in every call (what one call leaves there is zero for the next, of whatever size), then partials
constexpr int WS_COUNTERS = 1024 * sizeof(int);
static long long kv4_space(const Kv4Plan& p, int hd) { return p.rt ? 16 : WS_COUNTERS + 2LL * p.wgs * 16 * (hd + 2) * 4; }

int kv4_attend_launch(hipStream_t st, int dtype, Kv4AttnArgs a, int max_rows, int max_len, void* ws) {
    const bool f32 = dtype == HIVIS_F32;
    const Kv4Plan p = kv4_plan_attend(a.d, f32, a.group, a.n_seqs, max_rows, max_len);
    const long long sh = ((long long)a.n_seqs * a.d.heads + 7) / 8 * 8;
    a.tiles = p.tiles; a.max_rows = max_rows; a.cnt = (int*)ws; a.ws = (float*)((char*)ws + WS_COUNTERS);
#define KV4_ROWS_(KERNEL_, VSTRIDE_, HD_)                                                                                                      \
    do {                                                                                                                                       \
        constexpr int lds_ = 2 * 64 * (VSTRIDE_ + kv4_kstride<HD_>()) + 3 * (3 + HD_ / 32) * 8;                                                \
        OP_TRY(hipFuncSetAttribute((const void*)KERNEL_, hipFuncAttributeMaxDynamicSharedMemorySize, lds_));                                   \
        hipLaunchKernelGGL(KERNEL_, dim3((unsigned)sh, p.tiles), dim3(256), lds_, st, a);                                                      \
    } while (0)
#define KV4_FORMS(T_, HD_)                                                                                      \
    if (p.rt == 0) hipLaunchKernelGGL((kv4_stream_kernel<T_, HD_>), dim3(p.wgs), dim3(256), 0, st, a);            \
    else if (p.rt == 1) KV4_ROWS_((kv4_rows_kernel<T_, HD_>), kv4_vstride<HD_>(), HD_);                         \
    else KV4_ROWS_((kv4_rows32_kernel<T_, HD_>), kv4_vstride32<HD_>(), HD_);
    if (f32) { if (a.d.hd == 128) { KV4_FORMS(float, 128) } else { KV4_FORMS(float, 64) } }
    else { if (a.d.hd == 128) { KV4_FORMS(__bf16, 128) } else { KV4_FORMS(__bf16, 64) } }
#undef KV4_FORMS
#undef KV4_ROWS_
    OP_TRY(hipGetLastError());
    return HIVIS_OK;
}

long long kv4_attend_space(const Kv4Dims& d, int dtype, int n_q_heads, int n_seqs, int max_rows, int max_len) {
    return kv4_space(kv4_plan_attend(d, dtype == HIVIS_F32, n_q_heads / d.heads, n_seqs, max_rows, max_len), d.hd);
}

// Segments of a row: enough workgroups for four to a CU, of at least one chunk
static void logprobs_cut(int rows, int vocab, int* chunks, int* segs) {
    const int all = (vocab - 1) / LOGPROBS_CHUNK + 1, want = std::max(1, std::min(all, LOGPROBS_WGS / std::max(rows, 1)));
    *chunks = (all + want - 1) / want;
    *segs = (all + *chunks - 1) / *chunks;
}
static_assert(LOGPROBS_WGS / 2 <= WS_COUNTERS / (int)sizeof(int), "rows in more than one segment");

long long kv4_stream_space(int hd) { return WS_COUNTERS + 2LL * 1024 * 16 * (hd + 2) * 4; }

int kv4_move_launch(hipStream_t st, const Kv4Dims& d, uint8_t* mem, long long pool, int layers, const int* table, const int* len, const int* n, const int* path, int depth) {
    hipLaunchKernelGGL(kv4_move_kernel, dim3(layers, d.heads), dim3(256), depth * (d.hd + d.hd / 16), st, d, mem, pool, table, len, n, path);
    OP_TRY(hipGetLastError());
    return HIVIS_OK;
}

// ---- log probabilities ----
int logprobs_launch(hipStream_t st, int dtype, LogprobsArgs a, void* ws) {
    if (a.rows == 0) return HIVIS_OK;
    logprobs_cut(a.rows, a.vocab, &a.chunks, &a.segs);
    a.cnt = (int*)ws; a.part = (uint32_t*)((char*)ws + WS_COUNTERS);
#define LOGPROBS_(T_, TOP_) hipLaunchKernelGGL((logprobs_kernel<T_, TOP_>), dim3(a.segs, a.rows), dim3(LOGPROBS_NT), 0, st, a)
    if (dtype == HIVIS_F32) { if (a.top) LOGPROBS_(float, true); else LOGPROBS_(float, false); }
    else { if (a.top) LOGPROBS_(__bf16, true); else LOGPROBS_(__bf16, false); }
#undef LOGPROBS_
    OP_TRY(hipGetLastError());
    return HIVIS_OK;
}

long long logprobs_space(int rows, int vocab, int top) {
    int chunks, segs;
    logprobs_cut(rows, vocab, &chunks, &segs);
    return segs > 1 ? WS_COUNTERS + (long long)rows * segs * (LOGPROBS_STATS + 2 * top) * 4 : 16;
}

}  // namespace hivis

extern "C" {

int64_t hivis_kv4_pool_bytes(const hivis_kv4_shape* shape) {
    Kv4Dims d;
    if (int rc = check_shape(shape, &d)) return rc;
    return (int64_t)d.n_blocks * d.heads * kv4_chunk(d.hd, d.block);
}

int hivis_kv4_plan(void* hip_stream, int32_t n_seqs, int32_t max_blocks, int32_t block_tokens, int32_t n_blocks, const int32_t* keep, const int32_t* add, int32_t* held,
                   int32_t* table, int32_t* free_list, int32_t* row_start, int32_t* slots, int32_t* positions, int32_t max_rows, int32_t* status) {
    hivis_kv4_shape shape{1, 64, block_tokens, n_blocks};
    Kv4Dims d;
    if (int rc = check_shape(&shape, &d)) return rc;
    CHECK(n_seqs >= 1, "n_seqs %d", n_seqs);
    CHECK(max_blocks >= 1 && (long long)max_blocks * block_tokens <= 0x7fffffffLL, "max_blocks %d: a sequence's positions must be in 0..2^31-1", max_blocks);
    CHECK((long long)n_seqs * max_blocks <= 0x7fffffffLL, "n_seqs %d x max_blocks %d: a table has fewer than 2^31 entries", n_seqs, max_blocks);
    CHECK(max_rows >= 0, "max_rows %d", max_rows);
    CHECK(keep && add && held && table && free_list && row_start && status && (slots || max_rows == 0), "null argument");
    if (int rc = check_devices({{keep, "keep"}, {add, "add"}, {held, "held"}, {table, "table"}, {free_list, "free_list"}, {row_start, "row_start"}, {slots, "slots"},
                                {positions, "positions"}, {status, "status"}})) return rc;
    return kv4_plan_launch((hipStream_t)hip_stream, PlanArgs{n_seqs, max_blocks, d.shift, n_blocks, max_rows, keep, add, held, table, free_list, row_start, slots, positions, status, 0, false});
}

int hivis_kv4_append(void* hip_stream, const hivis_kv4_shape* shape, int32_t dtype, const void* k, const void* v, int64_t row_stride, int64_t head_stride, int32_t n_rows,
                     const int32_t* slots, void* pool) {
    RowsArgs a{};
    if (int rc = check_shape(shape, &a.d)) return rc;
    CHECK(n_rows == 0 || (k && v && slots && pool), "null argument");
    if (int rc = check_rows(k, v, dtype, a.d, row_stride, head_stride, n_rows)) return rc;
    CHECK(aligned(pool, 16), "the pool must start at a multiple of 16 bytes");
    if (int rc = check_devices({{k, "k"}, {v, "v"}, {slots, "slots"}, {pool, "pool"}})) return rc;
    a.k = k; a.v = v; a.row = row_stride; a.head = head_stride; a.n = n_rows; a.slots = slots; a.pool = (uint8_t*)pool;
    return kv4_append_launch((hipStream_t)hip_stream, dtype == HIVIS_F32 ? KV4_ROWS_F32 : KV4_ROWS_BF16, a);
}

int hivis_kv4_read(void* hip_stream, const hivis_kv4_shape* shape, int32_t dtype, const void* pool, int32_t n_rows, const int32_t* slots, void* k, void* v, int64_t row_stride,
                   int64_t head_stride) {
    RowsArgs a{};
    if (int rc = check_shape(shape, &a.d)) return rc;
    CHECK(n_rows == 0 || (k && v && slots && pool), "null argument");
    if (int rc = check_rows(k, v, dtype, a.d, row_stride, head_stride, n_rows)) return rc;
    CHECK(aligned(pool, 16), "the pool must start at a multiple of 16 bytes");
    if (int rc = check_devices({{k, "k"}, {v, "v"}, {slots, "slots"}, {pool, "pool"}})) return rc;
    a.k = k; a.v = v; a.row = row_stride; a.head = head_stride; a.n = n_rows; a.slots = slots; a.pool = (uint8_t*)const_cast<void*>(pool);
    return kv4_read_launch((hipStream_t)hip_stream, dtype == HIVIS_F32 ? KV4_ROWS_F32 : KV4_ROWS_BF16, a);
}

static int check_attention(const hivis_kv4_attention* a, Kv4Dims* d) {
    CHECK(a, "null argument");
    if (int rc = check_shape(&a->cache, d)) return rc;
    CHECK(a->dtype == HIVIS_F32 || a->dtype == HIVIS_BF16, "dtype %d unknown", a->dtype);
    CHECK(a->n_q_heads >= 1 && a->n_q_heads % d->heads == 0, "n_q_heads %d is no multiple of n_kv_heads %d", a->n_q_heads, d->heads);
    CHECK(a->n_seqs >= 0 && a->max_rows >= 0 && a->max_len >= 0, "n_seqs %d, max_rows %d, max_len %d", a->n_seqs, a->max_rows, a->max_len);
    // a launch has at most 2^31 - 1 heads of sequences with their row tiles (of 16 pairs at least), 65535 of those for one head
    const long long tiles = ((long long)a->max_rows * (a->n_q_heads / d->heads) + 15) / 16;
    CHECK(tiles <= 65535 && ((long long)a->n_seqs * d->heads + 7) * std::max(tiles, 1LL) <= 0x7fffffffLL, "n_seqs %d, n_kv_heads %d, max_rows %d, n_q_heads %d: more than a launch takes",
          a->n_seqs, d->heads, a->max_rows, a->n_q_heads);
    return HIVIS_OK;
}

int64_t hivis_kv4_attend_bytes(const hivis_kv4_attention* a) {
    Kv4Dims d;
    if (int rc = check_attention(a, &d)) return rc;
    return kv4_attend_space(d, a->dtype, a->n_q_heads, a->n_seqs, a->max_rows, a->max_len);
}

int hivis_kv4_attend(void* hip_stream, const hivis_kv4_attention* a) {
    Kv4AttnArgs k{};
    if (int rc = check_attention(a, &k.d)) return rc;
    CHECK(a->n_rows >= 0 && (long long)a->n_rows * a->n_q_heads <= 0x7fffffffLL, "n_rows %d x n_q_heads %d", a->n_rows, a->n_q_heads);
    if (a->n_seqs == 0 || a->max_rows == 0 || a->n_rows == 0) return HIVIS_OK;
    CHECK(a->max_blocks >= 1 && (long long)a->max_blocks * k.d.block <= 0x7fffffffLL - 255, "max_blocks %d: a sequence's positions must be below 2^31 - 256", a->max_blocks);
    CHECK((double)a->n_seqs * k.d.heads * (((long long)a->max_rows * (a->n_q_heads / k.d.heads) + 15) / 16) * ((long long)a->max_blocks * k.d.block / KV4_UNIT + 1 + KV4_ITEM_COST) < 2147483648.0,
          "n_seqs %d, max_blocks %d, max_rows %d: more than a launch takes", a->n_seqs, a->max_blocks, a->max_rows);
    CHECK(!a->mask || a->max_rows <= 64, "max_rows %d: a mask has bits for 64 rows", a->max_rows);
    CHECK(std::isfinite(a->scale), "scale is not finite");
    const int align = a->dtype == HIVIS_F32 ? 4 : 8;
    const long long width = (long long)a->n_q_heads * k.d.hd;
    CHECK(a->q_stride % align == 0 && a->q_stride >= 0 && a->out_stride >= width && a->out_stride % align == 0,
          "row strides %lld, %lld: multiples of %d values, of the output not below n_q_heads * head_dim", (long long)a->q_stride, (long long)a->out_stride, align);
    CHECK(a->pool && a->table && a->row_start && a->kv_len && a->q && a->out && a->workspace, "null argument");
    CHECK(aligned(a->pool, 16) && aligned(a->q, 16) && aligned(a->out, 16) && aligned(a->workspace, 16), "pool, q, out and workspace must start at multiples of 16 bytes");
    const long long need = kv4_attend_space(k.d, a->dtype, a->n_q_heads, a->n_seqs, a->max_rows, a->max_len);
    CHECK(a->workspace_bytes >= need, "workspace of %lld bytes, %lld needed", (long long)a->workspace_bytes, need);
    if (int rc = check_devices({{a->pool, "pool"}, {a->table, "table"}, {a->row_start, "row_start"}, {a->kv_len, "kv_len"}, {a->q, "q"}, {a->mask, "mask"}, {a->out, "out"},
                                {a->workspace, "workspace"}})) return rc;
    k.group = a->n_q_heads / k.d.heads; k.n_seqs = a->n_seqs; k.n_rows = a->n_rows; k.max_blocks = a->max_blocks; k.scale2 = std::max((float)(std::fabs(a->scale) * 1.4426950408889634), FLT_MIN); k.negate = a->scale < 0;
    k.pool = (const uint8_t*)a->pool; k.table = a->table; k.row_start = a->row_start; k.kv_len = a->kv_len; k.q = a->q; k.ldq = a->q_stride;
    k.mask = (const unsigned long long*)a->mask; k.out = a->out; k.ldo = a->out_stride;
    return kv4_attend_launch((hipStream_t)hip_stream, a->dtype, k, a->max_rows, a->max_len, a->workspace);
}

static int check_logprobs(int32_t n_rows, int32_t vocab, int32_t top_k) {
    CHECK(n_rows >= 0 && n_rows <= 65535, "n_rows %d outside [0,65535]", n_rows);
    CHECK(vocab >= 1 && vocab <= 0x7fffffff - LOGPROBS_CHUNK, "vocab %d", vocab);
    CHECK(top_k >= 0 && top_k <= LOGPROBS_MAX_TOP && top_k <= vocab, "top_k %d outside [0,%d] or above vocab %d", top_k, LOGPROBS_MAX_TOP, vocab);
    return HIVIS_OK;
}

int64_t hivis_logprobs_bytes(int32_t n_rows, int32_t vocab, int32_t top_k) {
    if (int rc = check_logprobs(n_rows, vocab, top_k)) return rc;
    return logprobs_space(n_rows, vocab, top_k);
}

int hivis_logprobs(void* hip_stream, int32_t dtype, const void* logits, int64_t row_stride, int32_t n_rows, int32_t vocab, float temperature, const int32_t* tokens, int32_t n_tokens,
                   float* logprob, float* entropy, int32_t top_k, int32_t* top_ids, float* top_logprobs, void* workspace, int64_t workspace_bytes) {
    if (int rc = check_logprobs(n_rows, vocab, top_k)) return rc;
    CHECK(dtype == HIVIS_F32 || dtype == HIVIS_BF16, "dtype %d unknown", dtype);
    CHECK(row_stride >= vocab, "row_stride %lld below vocab %d", (long long)row_stride, vocab);
    const float inv = 1.f / temperature;
    CHECK(temperature > 0.f && inv > 0.f && std::isfinite(inv), "temperature %g: it and its reciprocal must be positive and finite", (double)temperature);
    CHECK(n_tokens >= 0 && (n_tokens == 0 || (tokens && logprob)) && (top_k == 0 || (top_ids && top_logprobs)), "null argument");
    if (n_rows == 0) return HIVIS_OK;
    CHECK(logits && workspace, "null argument");
    CHECK(aligned(logits, dtype == HIVIS_F32 ? 4 : 2) && aligned(workspace, 16), "logits must start at a multiple of their size, the workspace at one of 16 bytes");
    const long long need = logprobs_space(n_rows, vocab, top_k);
    CHECK(workspace_bytes >= need, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, need);
    if (int rc = check_devices({{logits, "logits"}, {n_tokens ? tokens : nullptr, "tokens"}, {n_tokens ? logprob : nullptr, "logprob"}, {entropy, "entropy"}, {top_k ? top_ids : nullptr, "top_ids"},
                                {top_k ? top_logprobs : nullptr, "top_logprobs"}, {workspace, "workspace"}})) return rc;
    return logprobs_launch((hipStream_t)hip_stream, dtype,
                           LogprobsArgs{logits, row_stride, n_rows, vocab, inv, tokens, n_tokens, logprob, entropy, top_k, top_ids, top_logprobs, 0, 0, nullptr, nullptr}, workspace);
}

}  // extern "C"
