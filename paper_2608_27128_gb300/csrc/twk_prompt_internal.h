// twk_prompt_internal.h -- argument blocks and launchers of the operators that make a retained set:
// attention over prompts, its weights per key, and the eviction by accumulated weight (host-side
// declarations only).
#pragma once
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "twinkv.h"
#include "twk_cache_internal.h"

namespace twk {

struct PromptArgs {
    const uint16_t *q, *k, *v;     // [tokens][Hq][d], [keys][H][d], strides in elements
    twinkv_prompt s;
    twinkv_sequences seqs;
    int G;                         // query heads per KV head
    int tile_tokens;               // 128 / G: tokens of a tile of query rows
    int snap;                      // how the work is cut, see twk_prompt.cuh
    float scale;
    int window, n_sink;            // window 0: none
    int* out_status;               // [B] or null
    // attention
    uint16_t* out;                 // [tokens][Hq][d]
    float* out_lse;                // [tokens][Hq] or null
    // weights
    const float* lse;              // [tokens][Hq]
    int last;                      // tokens of a sequence that count, 0: all
    const float* score;            // [H][keys] or null
    float* out_score;
    void* ws;
};

// What a kernel with bounded waits needs: the device's error word and the limit of a wait.
struct WaitFacts {
    int* err;
    unsigned long long timeout_ns;
};
twinkv_status wait_facts(WaitFacts* w);

// A tensor map over bf16 rows [rows][heads][d] (strides in elements): boxes of 64 elements x box_heads x
// box_rows, 128-byte swizzle, zeros beyond the ends.
bool encode_rows(CUtensorMap* map, const void* base, int d, int heads, int rows, int64_t head,
                 int64_t row, int box_heads, int box_rows);

size_t prompt_attend_workspace(const twinkv_prompt& s);
cudaError_t launch_prompt_attend(const PromptArgs& a, int sms, const WaitFacts& w, cudaStream_t st);
size_t prompt_weights_workspace(const twinkv_prompt& s);
cudaError_t launch_prompt_weights(const PromptArgs& a, int sms, const WaitFacts& w, cudaStream_t st);

struct CacheWeightsArgs {
    AttendArgs a;                  // as for the attention; its outputs are not used, but the statuses
    const float* lse;              // [B][n][H * G]
    const float* score;            // [B * H][N]
    float* out_score;
    int N;
};
cudaError_t launch_cache_weights(const CacheWeightsArgs& a, int sms, cudaStream_t st);

// The first slots that windows show, see twk_attend.cu: seen [units][1 + n].
cudaError_t launch_windows(const AttendArgs& a, int units, int* seen, cudaStream_t st);

struct WeightPolicyArgs {
    const float* score;            // [units][N]
    int units, N;
    const int* lens;               // [units] or null
    const int* budget;             // [units]
    int n_sink, n_recent;
    uint8_t* out_mask;             // [units][N]
    float* out_score;              // [units][N] or null
    int* out_status;               // [units] or null
};
cudaError_t launch_weight_policy(const WeightPolicyArgs& a, cudaStream_t st);

}  // namespace twk
