// Arguments of the log-probability kernel (hivis_logprobs.h), for its launches.
#pragma once
#include <stdint.h>

namespace hivis {

constexpr int LOGPROBS_MAX_TOP = 32;

struct LogprobsArgs {
    const void* x; long long ld; int rows, vocab; float inv_temp;
    const int* tokens; int n_tokens; float *logprob, *entropy;
    int top; int* top_ids; float* top_logprobs;
    int chunks, segs; int* cnt; uint32_t* part;              // chunks of a segment; segments of a row, arrivals per row (zero between launches), partials [row][seg][STATS + 2 top]
};

}  // namespace hivis
