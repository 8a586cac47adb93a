// twk_weight_policy.cu -- eviction by accumulated attention weight.
//
// Per unit, of the positions below its length: the budget's worth by (protected first, score
// descending, position ascending).  A score becomes a 32-bit key that ascends where scores descend: the order
// of floats as integers, inverted, NaN the last; keys below that of +inf are free, and 0 stands for
// what is protected, 2^32 - 1 for no position.  The K smallest keys are kept, equal ones in position order.
//
// One block per unit:
//   1. the keys' least and greatest;
//   2. a radix select, 11 bits at a time of what is between them, finds the cut: the key c and how many keys
//      equal to c are still to be kept.  It stops early when every key with the prefix is kept, and where
//      at most kFew have it, which are then compared with one another;
//   3. one ordered pass writes the mask and, where asked for, the kept scores one after another.
// Digits of the keys' own range instead of the type's: weights fill few of the 2048 bins that the type has
// at the top (some 40), so that atomics on one of them wait for each other, and two more digits follow
// (288 units of 16384: 18.2 -> 13.7 us).
// Positions go to the threads four at a time, in turn: loads and stores are contiguous over a warp, and
// the order within a step is (round, thread, position).  A unit's keys stay in shared memory (V to a
// thread) up to 32768 positions; longer units are read again in every pass.
//
// Bound by latency: barriers and shared-memory atomics of the passes.  So a block is no larger than
// its unit needs, and several share an SM.  Measured in a graph: 8 units of 4096 positions 5.6 us, 288 of
// 16384 13.7 (of 20000 to 24000 cycles 6000 to 10000 go to loads, 6000 to two digits, 3000 to their cuts),
// 512 of 1040 to 4160 with the kept scores 12.7, 32 of 65536 38.7.  (Keys in registers, one block an SM:
// 25 us for the second.)
#include <atomic>

#include "twk_internal.h"
#include "twk_prompt_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

constexpr int kDigit = 11;
constexpr int kBins = 1 << kDigit;
constexpr int kFew = 128;

template <int V>
struct Shared {
    int4 hist[kBins / 4];
    int round[V / 4][32];      // counts of a round's warps, then what is before them
    int wsum[32];
    uint32_t low[32], high[32], few[kFew];
    uint32_t sel_key;
    int sel_digit, sel_before, sel_count, found, total;
};

constexpr uint32_t kNone = 0xffffffffu;

__device__ __forceinline__ uint32_t key_of(float x)
{
    if (x != x) return 0xff800001u;
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

template <int V, int kThreads, int kBlocks>
__global__ void __launch_bounds__(kThreads, kBlocks)
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
    // protected: [0, sinks) and [recent, len)
    const int sinks = min(a.n_sink, len), recent = max(len - a.n_recent, sinks);
    const int others = K - (sinks + len - recent);      // to keep beside them
    extern __shared__ uint4 keys[];          // round r of the thread's: [r threads + thread]
    auto place = [&](int p0, int r) { return p0 + (r * threads + static_cast<int>(threadIdx.x)) * 4; };
    uint32_t low = 0xffffffffu, high = 0;
    auto load = [&](int p0) {
#pragma unroll 4
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
            for (int j = 0; j < 4; ++j) k[j] = key_of(x[j]);
            if (p >= sinks && p + 4 <= recent) {
                low = min(min(low, min(k[0], k[1])), min(k[2], k[3]));
                high = max(max(high, max(k[0], k[1])), max(k[2], k[3]));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (p + j >= sinks && p + j < recent) low = min(low, k[j]), high = max(high, k[j]);
                    else k[j] = p + j < len ? 0u : kNone;
                }
            }
            keys[r * threads + threadIdx.x] = make_uint4(k[0], k[1], k[2], k[3]);
        }
    };
    auto each = [&](auto&& f) {
        for (int p0 = 0; p0 < len; p0 += step) {
            if (!once) load(p0);
            const int rounds = min(V / 4, (len - p0 + 4 * threads - 1) / (4 * threads));
#pragma unroll 2
            for (int r = 0; r < rounds; ++r) {
                const uint4 v = keys[r * threads + threadIdx.x];
                f(v.x), f(v.y), f(v.z), f(v.w);
            }
        }
    };

    // The keys below `base` are kept, and `need` of the `count` others below base + span (which is no more
    // than 2^32 - 1, so that neither 0 nor kNone is among them): all of them where `whole`.
    uint32_t base = 0, span = 1;
    int need = others, count = recent - sinks;
    bool whole = false;
    if (others > 0) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = threads >> 5;
        int* hist = reinterpret_cast<int*>(s.hist);
        auto clear = [&] {
            for (int d = threadIdx.x; d < kBins / 4; d += threads) s.hist[d] = int4{};
        };
        for (int p0 = 0; p0 < len; p0 += step) load(p0);
        clear();
        low = __reduce_min_sync(0xffffffffu, low);
        high = __reduce_max_sync(0xffffffffu, high);
        if (lane == 0) s.low[warp] = low, s.high[warp] = high;
        if (threadIdx.x == 0) s.found = 0;
        __syncthreads();
        base = __reduce_min_sync(0xffffffffu, lane < warps ? s.low[lane] : 0xffffffffu);
        high = __reduce_max_sync(0xffffffffu, lane < warps ? s.high[lane] : 0u);
        int bits = 32 - __clz(static_cast<int>(high - base));
        if (bits < 32) {
            span = 1u << bits;
            base = min(base, kNone - span);
        } else {                 // with what is protected, as keys of 0
            span = kNone;
            base = 0;
            need = K;
            count = len;
        }
        for (bool first = true; bits > 0 && !whole && count > kFew; first = false) {
            if (!first) {
                clear();
                __syncthreads();
            }
            const int shift = max(bits - kDigit, 0);
            each([&](uint32_t k) {
                const uint32_t at = k - base;
                if (at < span) atomicAdd(&hist[at >> shift & (kBins - 1)], 1);
            });
            __syncthreads();
            // the bin that holds the need-th key: a thread adds up some of them
            const int per = (kBins / 4 + threads - 1) / threads, d0 = threadIdx.x * per;
            int sum = 0;
            for (int d = d0; d < min(d0 + per, kBins / 4); ++d) {
                const int4 n = s.hist[d];
                sum += (n.x + n.y) + (n.z + n.w);
            }
            const int scan = warp_scan(sum);
            if (lane == 31) s.wsum[warp] = scan;
            __syncthreads();
            int run = __reduce_add_sync(0xffffffffu, lane < warp ? s.wsum[lane] : 0) + scan - sum;
            if (run < need && need <= run + sum)
                for (int d = 4 * d0; d < min(4 * (d0 + per), kBins); ++d) {
                    const int n = hist[d];
                    if (run < need && need <= run + n) {
                        s.sel_digit = d;
                        s.sel_before = run;
                        s.sel_count = n;
                    }
                    run += n;
                }
            __syncthreads();      // and those of the next pass come before sel_* is written again
            need -= s.sel_before;
            count = s.sel_count;
            base += static_cast<uint32_t>(s.sel_digit) << shift;
            bits = shift;
            span = 1u << bits;
            whole = count == need;
        }
        if (bits > 0 && !whole) {
            // few: the one with less than `need` before it, and enough with those like it
            each([&](uint32_t k) {
                if (k - base < span) s.few[atomicAdd(&s.found, 1) & (kFew - 1)] = k;
            });
            __syncthreads();
            for (int i = threadIdx.x; i < count; i += threads) {
                const uint32_t k = s.few[i];
                int before = 0, like = 0;
#pragma unroll 8
                for (int j = 0; j < count; ++j) {
                    before += s.few[j] < k;
                    like += s.few[j] == k;
                }
                if (before < need && need <= before + like) {      // those alike write the same
                    s.sel_key = k;
                    s.sel_before = before;
                    s.sel_count = like;
                }
            }
            __syncthreads();
            base = s.sel_key;
            need -= s.sel_before;
            whole = s.sel_count == need;
            span = 1;
        }
    }

    // 3. keep what is protected, the keys below the cut and the first `need` equal to it
    int seen_eq = 0, seen_kept = 0;
    for (int p0 = 0; p0 < len; p0 += step) {
        if (!once && others > 0) load(p0);
        const uint32_t end = base + span;
        if (whole && !kept) {
#pragma unroll 4
            for (int r = 0; r < V / 4; ++r) {
                const int p = place(p0, r);
                if (p >= len) break;
                const uint4 v = keys[r * threads + threadIdx.x];
                if (wide_mask && p + 4 <= len) {
                    *reinterpret_cast<uint32_t*>(mask + p) =
                        (v.x < end ? 1u : 0u) | (v.y < end ? 1u << 8 : 0u) |
                        (v.z < end ? 1u << 16 : 0u) | (v.w < end ? 1u << 24 : 0u);
                } else {
                    const uint32_t k[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (p + j < len) mask[p + j] = k[j] < end;
                }
            }
            continue;
        }
        uint32_t below = 0, same = 0;
#pragma unroll
        for (int r = 0; r < V / 4; ++r) {
            const int p = place(p0, r);
            if (others > 0) {
                const uint4 v = keys[r * threads + threadIdx.x];
                const uint32_t k[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    below |= k[j] < base ? 1u << (4 * r + j) : 0u;
                    same |= k[j] - base < span ? 1u << (4 * r + j) : 0u;
                }
            } else {                     // the first K that are protected
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = p + j < sinks ? p + j : p + j >= recent ? sinks + p + j - recent : K;
                    below |= p + j < len && n < K ? 1u << (4 * r + j) : 0u;
                }
            }
        }
        uint32_t keep = below | same;
        int before[V / 4];
        if (others > 0 && !whole) {            // alike in the whole block
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

template <int V, int kThreads, int kBlocks>
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
            e = cudaFuncSetAttribute(weight_policy_kernel<V, kThreads, kBlocks>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, V * kThreads * 4);
            if (e != cudaSuccess) return e;
            if (dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
        }
    }
    weight_policy_kernel<V, kThreads, kBlocks><<<a.units, threads, bytes, st>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_weight_policy(const WeightPolicyArgs& a, cudaStream_t st)
{
    // as few positions to a thread as leave room for several blocks on an SM: 512 units of 1040 to 4160 take
    // 12.7 us with 16, 16.8 with 8 in 768 threads; 288 of 16384 13.7 with 32, 14.9 with 16 in 1024
    return a.N <= 4096    ? launch<8, 512, 3>(a, st)
           : a.N <= 8192  ? launch<16, 512, 3>(a, st)
           : a.N <= 16384 ? launch<32, 512, 2>(a, st)
                          : launch<32, 1024, 1>(a, st);
}

}  // namespace twk
