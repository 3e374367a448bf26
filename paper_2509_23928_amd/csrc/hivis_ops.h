// What the contexts (hivis.hip) use of the operators (hivis_ops.hip): launches without the checks of callers' arguments.
#pragma once
#include "hivis_kv4_args.h"
#include "hivis_logprobs_args.h"

namespace hivis {

enum { KV4_ROWS_F32 = 0, KV4_ROWS_BF16 = 1, KV4_ROWS_HALVES = 2 };

void set_thread_error(const char* message);                  // what hivis_last_error(NULL) returns on this thread
int op_fail(int code, const char* fmt, ...);

int kv4_plan_launch(hipStream_t st, PlanArgs a);
int kv4_append_launch(hipStream_t st, int type, const RowsArgs& a);
int kv4_read_launch(hipStream_t st, int type, const RowsArgs& a);
int kv4_attend_launch(hipStream_t st, int dtype, Kv4AttnArgs a, int max_rows, int max_len, void* ws);
long long kv4_attend_space(const Kv4Dims& d, int dtype, int n_q_heads, int n_seqs, int max_rows, int max_len);
long long kv4_stream_space(int hd);                         // of any attention call with this head_dim
// Rows of sequence 0 at positions len + path[j] to len + j (j = 1 .. *n), all layers (pools `pool` bytes apart)
int kv4_move_launch(hipStream_t st, const Kv4Dims& d, uint8_t* mem, long long pool, int layers, const int* table, const int* len, const int* n, const int* path, int depth);
int logprobs_launch(hipStream_t st, int dtype, LogprobsArgs a, void* ws);
long long logprobs_space(int rows, int vocab, int top);

}  // namespace hivis
