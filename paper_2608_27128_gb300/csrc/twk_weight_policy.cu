// twk_weight_policy.cu -- eviction by accumulated attention weight.
//
// Per unit, of the positions below its length: the budget's worth by (protected first, score
// descending, position ascending).  A score becomes a 32-bit key that ascends where scores descend:
//     protected: 0;   NaN: 2^32 - 1;   others: the order of floats as integers, inverted
// and the K smallest keys are kept, equal keys in position order.
//
// One block per unit:
//   1. a radix select, 11 bits at a time from the top, finds the cut: the key c and how many items
//      equal to c are still to be kept (stopping early when every item with the prefix is kept);
//   2. one ordered pass writes the mask and, where asked for, the kept scores one after another.
// Positions go to the threads four at a time, in turn: loads and stores are contiguous over a warp, and
// the order within a step is (round, thread, position).  A unit's keys stay in shared memory (V to a
// thread) up to 32768 positions; longer units are read again in every pass.
//
// Bound by latency: barriers and shared-memory atomics of the passes.  So a block is no larger than
// its unit needs, and several share an SM.  Measured in a graph: 8 units of 4096 positions 5.6 us, 288 of
// 16384 18, 512 of 1040 to 4160 with the kept scores 17, 32 of 65536 46.  (Keys in registers, one block an
// SM: 25 us for the second.)
#include <atomic>

#include "twk_internal.h"
#include "twk_prompt_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

constexpr int kDigit = 11;
constexpr int kBins = 1 << kDigit;

template <int V>
struct Shared {
    int4 hist[kBins / 4];
    int round[V / 4][32];      // counts of a round's warps, then what is before them
    int wsum[32];
    int sel_digit, sel_before, sel_count, total;
};

__device__ __forceinline__ uint32_t key_of(float x)
{
    if (x != x) return 0xffffffffu;
    const uint32_t u = __float_as_uint(x + 0.0f);      // -0 as 0
    return ~(u >> 31 ? ~u : u | 0x80000000u);
}

__device__ __forceinline__ int warp_scan(int x)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// Per round (of the step's V / 4) the positions before the thread's that are marked in `bits`, four to a
// round, and the step's total.
template <int V>
__device__ __forceinline__ int prefix(Shared<V>& s, uint32_t bits, int (&before)[V / 4])
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
    for (int r = 0; r < V / 4; r += 4) {
        // four rounds' counts at a time, at most 128 a warp each, in the bytes of a word
        uint32_t n = 0;
#pragma unroll
        for (int k = 0; k < 4 && r + k < V / 4; ++k)
            n |= static_cast<uint32_t>(__popc(bits >> (4 * (r + k)) & 15u)) << (8 * k);
        const uint32_t scan = static_cast<uint32_t>(warp_scan(static_cast<int>(n)));
#pragma unroll
        for (int k = 0; k < 4 && r + k < V / 4; ++k) {
            before[r + k] = static_cast<int>((scan - n) >> (8 * k) & 255u);
            if (lane == 31) s.round[r + k][warp] = static_cast<int>(scan >> (8 * k) & 255u);
        }
    }
    __syncthreads();
    if (warp == 0) {
        int sum = 0;
#pragma unroll
        for (int r = 0; r < V / 4; ++r) {
            const int n = lane < warps ? s.round[r][lane] : 0, scan = warp_scan(n);
            s.round[r][lane] = sum + scan - n;
            sum += __shfl_sync(0xffffffffu, scan, 31);
        }
        if (lane == 0) s.total = sum;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < V / 4; ++r) before[r] += s.round[r][warp];
    return s.total;
}

template <int V, int kThreads>
__global__ void __launch_bounds__(kThreads)
    weight_policy_kernel(const __grid_constant__ WeightPolicyArgs a)
{
    static_assert(V == 8 || V == 16 || V == 32, "a thread's marks are bits of a word");
    wait_for_previous();
    __shared__ Shared<V> s;
    const int u = blockIdx.x, threads = blockDim.x;
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
    for (int i = len + threadIdx.x; i < a.N; i += threads) mask[i] = 0;
    if (kept)
        for (int i = K + threadIdx.x; i < a.N; i += threads) kept[i] = 0.0f;
    if (all || K == 0) {
        for (int i = threadIdx.x; i < len; i += threads) {
            mask[i] = all ? 1 : 0;
            if (kept && all) kept[i] = score[i];
        }
        return;
    }
    const bool wide = (reinterpret_cast<uintptr_t>(score) & 15) == 0;
    const bool wide_mask = (reinterpret_cast<uintptr_t>(mask) & 3) == 0;
    const int step = threads * V;
    const bool once = len <= step;
    const int last = len - a.n_recent;      // first recent position
    extern __shared__ uint4 keys[];          // round r of the thread's: [r threads + thread]
    auto place = [&](int p0, int r) { return p0 + (r * threads + static_cast<int>(threadIdx.x)) * 4; };
    auto load = [&](int p0) {
#pragma unroll 2
        for (int r = 0; r < V / 4; ++r) {
            const int p = place(p0, r);
            float x[4] = {};
            if (wide && p + 4 <= len) {
                const float4 v = *reinterpret_cast<const float4*>(score + p);
                x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (p + j < len) x[j] = score[p + j];
            }
            uint32_t k[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                k[j] = p + j < a.n_sink || p + j >= last ? 0u : key_of(x[j]);
            keys[r * threads + threadIdx.x] = make_uint4(k[0], k[1], k[2], k[3]);
        }
    };
    if (once) load(0);

    // 1. the cut: `prefix_` is its key >> top
    uint32_t cut = 0;
    int top = 32, need = K;
    bool whole = false;
    while (top > 0 && !whole) {
        const int shift = max(top - kDigit, 0), bins = 1 << (top - shift);
        int* hist = reinterpret_cast<int*>(s.hist);
        for (int d = threadIdx.x; d < bins / 4; d += threads) s.hist[d] = int4{};
        __syncthreads();
        for (int p0 = 0; p0 < len; p0 += step) {
            if (!once) load(p0);
#pragma unroll 2
            for (int r = 0; r < V / 4; ++r) {
                const uint4 v = keys[r * threads + threadIdx.x];
                const uint32_t k[4] = {v.x, v.y, v.z, v.w};
                const int p = place(p0, r);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (p + j < len && (top == 32 || k[j] >> (top & 31) == cut))
                        atomicAdd(&hist[(k[j] >> shift) & (bins - 1)], 1);
            }
        }
        __syncthreads();
        // the bin that holds the need-th key: a thread adds up some of them
        const int per = (bins / 4 + threads - 1) / threads, d0 = threadIdx.x * per;
        int sum = 0;
        for (int d = d0; d < min(d0 + per, bins / 4); ++d) {
            const int4 n = s.hist[d];
            sum += (n.x + n.y) + (n.z + n.w);
        }
        const int scan = warp_scan(sum);
        if ((threadIdx.x & 31) == 31) s.wsum[threadIdx.x >> 5] = scan;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        const int others = lane < static_cast<int>(threadIdx.x >> 5) ? s.wsum[lane] : 0;
        int run = __reduce_add_sync(0xffffffffu, others) + scan - sum;
        if (run < need && need <= run + sum)
            for (int d = 4 * d0; d < min(4 * (d0 + per), bins); ++d) {
                const int n = hist[d];
                if (run < need && need <= run + n) {
                    s.sel_digit = d;
                    s.sel_before = run;
                    s.sel_count = n;
                }
                run += n;
            }
        __syncthreads();
        need -= s.sel_before;
        cut = cut << (top - shift) | static_cast<uint32_t>(s.sel_digit);
        whole = s.sel_count == need;
        top = shift;   // the barriers of the next pass come before sel_* is written again
    }

    // 2. keep the keys below the cut and the first `need` equal to it
    int seen_eq = 0, seen_kept = 0;
    for (int p0 = 0; p0 < len; p0 += step) {
        if (!once) load(p0);
        uint32_t below = 0, same = 0;
#pragma unroll
        for (int r = 0; r < V / 4; ++r) {
            const uint4 v = keys[r * threads + threadIdx.x];
            const uint32_t k[4] = {v.x >> top, v.y >> top, v.z >> top, v.w >> top};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool in = place(p0, r) + j < len;
                below |= in && k[j] < cut ? 1u << (4 * r + j) : 0u;
                same |= in && k[j] == cut ? 1u << (4 * r + j) : 0u;
            }
        }
        uint32_t keep = below | same;
        int before[V / 4];
        if (!whole) {            // alike in the whole block
            const int total = prefix<V>(s, same, before);
            keep = below;
#pragma unroll
            for (int r = 0; r < V / 4; ++r) {
                int at = seen_eq + before[r];
#pragma unroll
                for (int i = 4 * r; i < 4 * r + 4; ++i) {
                    if (same >> i & 1u && at < need) keep |= 1u << i;
                    at += same >> i & 1u;
                }
            }
            seen_eq += total;
        }
#pragma unroll
        for (int r = 0; r < V / 4; ++r) {
            const int p = place(p0, r);
            const uint32_t bits = keep >> (4 * r) & 15u;
            const uint32_t bytes = bits * 0x00204081u & 0x01010101u;
            if (wide_mask && p + 4 <= len) {
                *reinterpret_cast<uint32_t*>(mask + p) = bytes;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (p + j < len) mask[p + j] = bits >> j & 1u;
            }
        }
        if (kept) {
            __syncthreads();     // the counts of `same` have been read
            const int total = prefix<V>(s, keep, before);
#pragma unroll
            for (int r = 0; r < V / 4; ++r) {
                int to = seen_kept + before[r];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (keep >> (4 * r + j) & 1u) kept[to++] = score[place(p0, r) + j];
            }
            seen_kept += total;
        }
        if (!once) __syncthreads();
    }
}

template <int V, int kThreads>
cudaError_t launch(const WeightPolicyArgs& a, cudaStream_t st)
{
    const int threads = std::min(kThreads, ((a.N + V - 1) / V + 31) / 32 * 32);
    const int bytes = threads * V * 4;
    if constexpr (V * kThreads * 4 > 40000) {
        static std::atomic<bool> allowed[64];     // by device
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev >= 64 || !allowed[dev].load(std::memory_order_relaxed)) {
            e = cudaFuncSetAttribute(weight_policy_kernel<V, kThreads>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, V * kThreads * 4);
            if (e != cudaSuccess) return e;
            if (dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
        }
    }
    weight_policy_kernel<V, kThreads><<<a.units, threads, bytes, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_weight_policy(const WeightPolicyArgs& a, cudaStream_t st)
{
    // 8 to a thread, 768 threads at most (512 units of 1040 to 4160 positions: 16.6 us, with 16 to a thread
    // 19.2); more to a thread where a block would fill half an SM (288 units of 8192 positions: 11.3 us
    // with 16, 13.8 with 8; of 16384: 18.4 with 32, 20.4 with 16)
    return a.N <= 6144    ? launch<8, 768>(a, st)
           : a.N <= 8192  ? launch<16, 512>(a, st)
           : a.N <= 16384 ? launch<32, 512>(a, st)
                          : launch<32, 1024>(a, st);
}

}  // namespace twk
