// Arguments of the kernels of the paged cache in 4 bits (hivis_kv4.h), for their launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace hivis {

// What the kernels know of a cache
struct Kv4Dims { int heads, hd, block, shift, n_blocks; };       // block = 1 << shift rows

__host__ __device__ inline int kv4_chunk(int hd, int block) { return block * (hd + hd / 16); }      // bytes of one head in one block

struct PlanArgs {
    int n, max_blocks, shift, n_blocks, max_rows;
    const int *keep, *add; int *held, *table, *free_list, *row_start, *slots, *positions, *status;
    int add_each;                                            // no keep: 0; no add: this for every sequence
    bool fill;                                               // slots and positions in the same launch
};

// Rows as their owners hold them, for append and read: row r of head h at r * row + h * head (values)
struct RowsArgs {
    Kv4Dims d; const void *k, *v; long long row, head; int n; const int* slots; uint8_t* pool;
    // rows of several sequences at equal distance instead (slots from the plan all the same): row r is row first[s] + r % m of sequence r / m, sequences `seq` elements apart
    const int* first; int m, offset; long long seq;
};

struct Kv4AttnArgs {
    Kv4Dims d; int group, n_seqs, n_rows, max_rows, max_blocks, tiles; // group: query heads per key head; tiles: row tiles per sequence in the grid
    float scale2;                                            // |softmax scale| times log2 e, not below the smallest normal number (infinity times zero has no value); negative ones negate the queries
    bool negate;
    const uint8_t* pool; const int *table, *row_start, *kv_len;
    const void* q; long long ldq; const unsigned long long* mask; void* out; long long ldo;
    // rows of the context's passes instead of row_start: m rows of every sequence, row r of sequence s at s * qrows + r in q and s * m + r in out, lengths kv_len[seq0 + s] + len_add
    int m, qrows, seq0, len_add;
    float* ws; int* cnt;                                     // kv4_stream_kernel: partials; arrivals at the item that goes on behind a workgroup's run (zero between launches)
};

}  // namespace hivis
