// twk_cache_internal.h -- argument blocks and launchers of the operators around the pass: norms
// with rotation, the 4-bit pages and the attention over them (host-side declarations only).
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

#include "twinkv.h"

namespace twk {

// The current device's facts (set up on first use), or why there are none.
twinkv_status device_facts(int* sms);
twinkv_status cuda_result(cudaError_t e);

struct RopeArgs {
    const void *q, *k;             // [tokens][heads][d], strides in elements
    int64_t q_token, q_head, k_token, k_head;
    void *out_q, *out_k;
    int64_t oq_token, oq_head, ok_token, ok_head;
    const void *wq, *wk;           // [d] or null
    const float* cos_sin;          // [rows][d]: d / 2 cosines, d / 2 sines
    const int* positions;          // [tokens]
    int* out_status;               // [tokens] or null
    int tokens, heads_q, heads_k, d, rows;
    float eps;
};
cudaError_t launch_rope(const RopeArgs& a, bool f32, int sms, cudaStream_t st);

// Pages of units: entry j of a unit's row of `table` is the page with its slots
// [64 j, 64 j + 64).
struct Pages {
    uint8_t* base;
    int n_pages;
    const int* table;      // [units][max_pages]
    int max_pages;
};

// The kept rows of each unit in order: index [units][N] (null: all rows), lens, statuses.
struct IndexArgs {
    const uint8_t* mask;       // [units][N] or null
    const int* limit;          // [units] rows that count, or null (N)
    int units, N, limit_most;  // limit beyond limit_most (or below 0): a data error
    const int* src_table;      // pages the rows come from, or null
    int src_max_pages;
    const int* dst_table;      // pages they go to
    int dst_max_pages, n_pages;
    int* index;
    int* out_lens;
    int* out_status;           // or null
};
cudaError_t launch_index(const IndexArgs& a, cudaStream_t st);

struct PackArgs {
    const void *keys, *values;   // [units][N][d]
    int units, N;
    const int* index;            // [units][N] or null
    const int* lens;             // [units] slots to fill
    Pages to;
    int* out_status;             // written by the index; or null
};
cudaError_t launch_pack(const PackArgs& a, int d, bool f32, cudaStream_t st);

struct AppendArgs {
    const void *keys, *values;   // [B][n][H][d], strides in elements
    int64_t k_batch, k_token, k_head, v_batch, v_token, v_head;
    int B, H, n;
    const int* positions;        // [B][n]
    Pages to;
    const int* lens;             // [B * H]
    int* out_lens;               // may be lens
    int* out_status;             // or null
};
cudaError_t launch_append(const AppendArgs& a, int d, bool f32, cudaStream_t st);

struct CompactArgs {
    Pages from, to;
    int units, N;                // N: row stride of index
    const int* index;            // [units][N] or null
    const int* lens;             // [units] slots to fill
};
cudaError_t launch_compact(const CompactArgs& a, int d, cudaStream_t st);

struct ReadArgs {
    Pages from;
    const int* lens;             // [units]
    int units, rows;
    int last;                    // the last `rows` slots instead of the first
    uint16_t *out_keys, *out_values;   // [units][rows][d] bf16
    int* out_positions;          // [units][rows] or null
    int* out_status;             // [units] or null
};
cudaError_t launch_read(const ReadArgs& a, int d, cudaStream_t st);

struct AttendArgs {
    const uint16_t* q;           // [B][n][Hq][d], strides in elements
    int64_t q_batch, q_token, q_head;
    int B, H, G, n;              // G: query heads per KV head
    int d;
    float scale;
    int window, n_sink;          // window 0: none
    Pages from;
    const int* lens;             // [B * H]
    uint16_t* out;               // [B][n][H * G][d]
    float* out_lse;              // [B][n][H * G] or null
    int* out_status;             // [B * H] or null
    void* ws;
};
// The grid has a block per SM, and at most this many (a GB300's), so that the workspace's size does
// not depend on the device.
constexpr int kAttendBlocks = 152;
size_t attend_workspace(int units, int rows, int n, int d);
cudaError_t launch_attend(const AttendArgs& a, int sms, cudaStream_t st);

}  // namespace twk
