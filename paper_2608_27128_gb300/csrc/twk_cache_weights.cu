// twk_cache_weights.cu -- what the newest tokens' attention pays to each slot of the pages.
//
//     A(j) = score(j) + sum over tokens i that see j, and query heads of the KV head:
//            exp(scale q_i . k_j - lse_i)
//
// One thread per slot: right for every case, and the measure for what follows.
#include "twk_cache.cuh"
#include "twk_prompt_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

template <int D>
__global__ void __launch_bounds__(64)
    cache_weights_kernel(const __grid_constant__ CacheWeightsArgs p, const int* seen)
{
    using P = PageLayout<D>;
    const AttendArgs& a = p.a;
    wait_for_previous();
    const int unit = blockIdx.y, page = blockIdx.x, slot = page * kPage + threadIdx.x;
    const int len = a.lens[unit];
    const bool bad = len < 0 || len > static_cast<int64_t>(a.from.max_pages) * kPage;
    const bool large = !bad && len > p.N;
    const int* table = a.from.table + static_cast<int64_t>(unit) * a.from.max_pages;
    if (page == 0 && a.out_status) {
        bool wrong = false;
        if (!bad)
            for (int j = threadIdx.x; j * kPage < len; j += 64)
                wrong |= static_cast<unsigned>(table[j]) >= static_cast<unsigned>(a.from.n_pages);
        wrong = __syncthreads_or(wrong);
        if (threadIdx.x == 0)
            a.out_status[unit] = large ? TWINKV_ERR_TOO_LARGE
                                       : bad || wrong ? TWINKV_ERR_INVALID_ARG : TWINKV_OK;
    }
    if (bad || large || slot >= len) return;
    const int id = table[page];
    const int64_t at = static_cast<int64_t>(unit) * p.N + slot;
    float sum = p.score[at];
    if (static_cast<unsigned>(id) < static_cast<unsigned>(a.from.n_pages)) {
        const uint8_t* base = a.from.base + static_cast<int64_t>(id) * P::kBytes;
        const int b = unit / a.H, h = unit % a.H;
        const int* see = seen ? seen + static_cast<int64_t>(unit) * (1 + a.n) : nullptr;
        for (int i = 0; i < a.n; ++i) {
            if (slot > len - a.n + i || (see && slot < see[1 + i] && slot >= see[0])) continue;
            for (int g = 0; g < a.G; ++g) {
                const int head = h * a.G + g;
                const uint16_t* q = a.q + b * a.q_batch + i * a.q_token + head * a.q_head;
                float x = 0.0f;
                for (int G = 0; G < P::kGroups; ++G) {
                    const uint32_t m = *reinterpret_cast<const uint32_t*>(
                        base + P::kKeyGroups + (threadIdx.x * P::kGroups + G) * 4);
                    const float zero = bf16_hi(m) + 128.0f;
                    float y = 0.0f;
                    for (int e = 0; e < 64; ++e) {
                        const int at_e = 64 * G + e;
                        const uint32_t w = *reinterpret_cast<const uint32_t*>(
                            base + P::key_word(threadIdx.x, at_e / 8));
                        const int nibble = 4 * (e % 2) + e % 8 / 2;
                        y = fmaf(bf16_lo(q[at_e]), (w >> (4 * nibble) & 15u) + zero, y);
                    }
                    x = fmaf(bf16_lo(m), y, x);
                }
                sum += expf(x * a.scale -
                            p.lse[(static_cast<int64_t>(b) * a.n + i) * (a.H * a.G) + head]);
            }
        }
    }
    p.out_score[at] = sum;
}

}  // namespace

cudaError_t launch_cache_weights(const CacheWeightsArgs& p, int sms, cudaStream_t st)
{
    const int units = p.a.B * p.a.H;
    int* seen = nullptr;
    if (p.a.window > 0) {
        seen = static_cast<int*>(p.a.ws);
        const cudaError_t e = launch_windows(p.a, units, seen, st);
        if (e != cudaSuccess) return e;
    }
    const dim3 grid((p.N + kPage - 1) / kPage, units);
    if (p.a.d == 128) cache_weights_kernel<128><<<grid, 64, 0, st>>>(p, seen);
    else cache_weights_kernel<64><<<grid, 64, 0, st>>>(p, seen);
    return cudaGetLastError();
}

}  // namespace twk
