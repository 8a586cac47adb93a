// twk_weight_policy.cu -- eviction by accumulated attention weight.
//
// Per unit, of the positions below its length: the budget's worth by (protected first, score
// descending, position ascending).  A score becomes a 32-bit key that ascends where scores descend:
//     protected: 0;   NaN: 2^32 - 1;   others: the order of floats as integers, inverted
// and the K smallest keys are kept, equal keys in position order.
//
// One 1024-thread block per unit:
//   1. a radix select, 12 bits at a time from the top, finds the cut: the key c and how many items
//      equal to c are still to be kept (stopping early when every item with the prefix is kept);
//   2. one ordered pass writes the mask and, where asked for, the kept scores one after another.
// A thread takes eight consecutive positions; units of up to 8192 are read once and stay in
// registers.
#include "twk_internal.h"
#include "twk_prompt_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

constexpr int kThreads = 1024;
constexpr int kVec = 8;       // consecutive positions of a thread and step
constexpr int kDigit = 12;
constexpr int kBins = 1 << kDigit;

struct Shared {
    int hist[kBins];
    int wsum[32];
    int sel_digit, sel_before, sel_count;
};

__device__ __forceinline__ uint32_t key_of(float x)
{
    if (x != x) return 0xffffffffu;
    const uint32_t u = __float_as_uint(x + 0.0f);      // -0 as 0
    return ~(u >> 31 ? ~u : u | 0x80000000u);
}

// Exclusive block prefix of v; every thread also gets the total.
__device__ __forceinline__ int block_scan(Shared& s, int v, int& total)
{
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) s.wsum[wid] = x;
    __syncthreads();
    const int t = s.wsum[lane];
    total = __reduce_add_sync(0xFFFFFFFFu, t);
    const int before = __reduce_add_sync(0xFFFFFFFFu, lane < wid ? t : 0);
    __syncthreads();
    return before + x - v;
}

__global__ void __launch_bounds__(kThreads, 1)
    weight_policy_kernel(const __grid_constant__ WeightPolicyArgs a)
{
    wait_for_previous();
    __shared__ Shared s;
    const int u = blockIdx.x;
    const float* score = a.score + static_cast<int64_t>(u) * a.N;
    uint8_t* mask = a.out_mask + static_cast<int64_t>(u) * a.N;
    float* kept = a.out_score ? a.out_score + static_cast<int64_t>(u) * a.N : nullptr;
    int len = a.lens ? a.lens[u] : a.N, K = a.budget[u];
    const bool bad = K < 0 || K > a.N || len < 0 || len > a.N;
    if (threadIdx.x == 0 && a.out_status)
        a.out_status[u] = bad ? TWINKV_ERR_INVALID_ARG : TWINKV_OK;
    if (bad) len = K = 0;
    K = min(K, len);
    const bool all = K == len;
    for (int i = len + threadIdx.x; i < a.N; i += kThreads) mask[i] = 0;
    if (kept)
        for (int i = K + threadIdx.x; i < a.N; i += kThreads) kept[i] = 0.0f;
    if (all || K == 0) {
        for (int i = threadIdx.x; i < len; i += kThreads) {
            mask[i] = all ? 1 : 0;
            if (kept && all) kept[i] = score[i];
        }
        return;
    }
    constexpr int kStep = kThreads * kVec;
    const bool once = len <= kStep;
    const int mine = threadIdx.x * kVec;
    float x[kVec];
    uint32_t key[kVec];
    auto load = [&](int p0) {
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            x[j] = p0 + j < len ? score[p0 + j] : 0.0f;
            const bool prot = p0 + j < a.n_sink || p0 + j >= len - a.n_recent;
            key[j] = prot ? 0u : key_of(x[j]);
        }
    };
    if (once) load(mine);

    // 1. the cut: `prefix` is its key >> top
    uint32_t prefix = 0;
    int top = 32, need = K;
    bool whole = false;
    while (top > 0 && !whole) {
        const int shift = max(top - kDigit, 0), bins = 1 << (top - shift);
        for (int d = threadIdx.x; d < bins; d += kThreads) s.hist[d] = 0;
        __syncthreads();
        for (int c0 = 0; c0 < len; c0 += kStep) {
            if (!once) load(c0 + mine);
#pragma unroll
            for (int j = 0; j < kVec; ++j)
                if (c0 + mine + j < len &&
                    (top == 32 || static_cast<uint32_t>(key[j] >> (top & 31)) == prefix))
                    atomicAdd(&s.hist[(key[j] >> shift) & (bins - 1)], 1);
        }
        __syncthreads();
        constexpr int kPer = kBins / kThreads;
        int h[kPer], sum = 0, total;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int d = threadIdx.x * kPer + j;
            h[j] = d < bins ? s.hist[d] : 0;
            sum += h[j];
        }
        int run = block_scan(s, sum, total);
        if (run < need && need <= run + sum) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                if (run < need && need <= run + h[j]) {
                    s.sel_digit = threadIdx.x * kPer + j;
                    s.sel_before = run;
                    s.sel_count = h[j];
                }
                run += h[j];
            }
        }
        __syncthreads();
        need -= s.sel_before;
        prefix = prefix << (top - shift) | static_cast<uint32_t>(s.sel_digit);
        whole = s.sel_count == need;
        top = shift;   // the barriers of the next pass come before sel_* is written again
    }

    // 2. keep the keys below the cut and the first `need` equal to it
    int seen_eq = 0, seen_kept = 0;
    for (int c0 = 0; c0 < len; c0 += kStep) {
        if (!once) load(c0 + mine);
        int eq = 0;
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            eq += c0 + mine + j < len && !whole && (key[j] >> top) == prefix ? 1 : 0;
        int total = 0, at = 0;
        if (!whole) at = seen_eq + block_scan(s, eq, total);   // alike in the whole block
        seen_eq += total;
        uint32_t keep = 0;
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const uint32_t km = key[j] >> top;
            const bool same = km == prefix;
            const bool in = c0 + mine + j < len;
            if (in && (km < prefix || (same && (whole || at < need)))) keep |= 1u << j;
            at += in && same ? 1 : 0;
        }
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            if (c0 + mine + j < len) mask[c0 + mine + j] = keep >> j & 1u;
        if (kept) {
            int to = seen_kept + block_scan(s, __popc(keep), total);
            seen_kept += total;
#pragma unroll
            for (int j = 0; j < kVec; ++j)
                if (keep >> j & 1u) kept[to++] = x[j];
        }
    }
}

}  // namespace

cudaError_t launch_weight_policy(const WeightPolicyArgs& a, cudaStream_t st)
{
    weight_policy_kernel<<<a.units, kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace twk
