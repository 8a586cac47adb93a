// twk_prompt.cu -- attention over prompts.
//
// Per token at position p = m - n + i of its sequence and query head:
//     o = sum_j exp(scale q . k_j - lse) v_j,   lse = log sum_j exp(scale q . k_j)
// over the keys j <= p and, with a window W, of those p - j < W or j < n_sink.
//
// One warp per token and query head, over the keys one by one: right for every case, and the measure for
// what follows.
#include "twk_cache.cuh"
#include "twk_prompt.cuh"
#include "twk_ptx.cuh"

namespace twk {
namespace {

template <int D>
__global__ void __launch_bounds__(128) prompt_attend_kernel(const __grid_constant__ PromptArgs a)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    if (blockIdx.x == 0 && a.out_status)
        for (int b = threadIdx.x; b < a.s.B; b += 128)
            a.out_status[b] = sequence_of(a, b).ok ? TWINKV_OK : TWINKV_ERR_INVALID_ARG;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + warp;
    const int t = static_cast<int>(item / a.s.Hq), head = static_cast<int>(item % a.s.Hq);
    if (t >= a.s.tokens) return;
    Sequence s{};
    int b = 0;
    for (; b < a.s.B; ++b) {
        s = sequence_of(a, b);
        if (s.ok && t >= s.t0 && t - s.t0 < s.n) break;
    }
    if (b == a.s.B) return;
    constexpr int V = D / 32;
    float q[V], o[V] = {};
    const uint16_t* src = a.q + t * a.s.q_token + head * a.s.q_head + V * lane;
#pragma unroll
    for (int v = 0; v < V; ++v) q[v] = bf16_lo(src[v]);
    const int p = s.m - s.n + t - s.t0, h = head / a.G;
    float top = -INFINITY, sum = 0.0f;
    for (int j = 0; j <= p; ++j) {
        if (a.window > 0 && p - j >= a.window && j >= a.n_sink) continue;
        const int64_t row = s.j0 + j;
        const uint16_t* k = a.k + row * a.s.k_token + h * a.s.k_head + V * lane;
        const uint16_t* w = a.v + row * a.s.v_token + h * a.s.v_head + V * lane;
        float x = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) x = fmaf(q[v], bf16_lo(k[v]), x);
#pragma unroll
        for (int i = 16; i > 0; i /= 2) x += __shfl_xor_sync(0xffffffffu, x, i);
        x *= a.scale;
        const float most = fmaxf(top, x), f = expf(top - most), y = expf(x - most);
        sum = fmaf(sum, f, y);
#pragma unroll
        for (int v = 0; v < V; ++v) o[v] = fmaf(o[v], f, y * bf16_lo(w[v]));
        top = most;
    }
    const int64_t at = static_cast<int64_t>(t) * a.s.Hq + head;
#pragma unroll
    for (int v = 0; v < V; v += 2)
        *reinterpret_cast<uint32_t*>(a.out + at * D + V * lane + v) =
            sum > 0.0f ? bf16_pair(o[v] / sum, o[v + 1] / sum) : 0u;
    if (a.out_lse && lane == 0) a.out_lse[at] = sum > 0.0f ? top + logf(sum) : -INFINITY;
}

}  // namespace

cudaError_t launch_prompt_attend(const PromptArgs& a, int sms, cudaStream_t st)
{
    const int64_t items = static_cast<int64_t>(a.s.tokens) * a.s.Hq;
    const unsigned grid = static_cast<unsigned>((items + 3) / 4);
    if (a.s.d == 128) prompt_attend_kernel<128><<<grid, 128, 0, st>>>(a);
    else prompt_attend_kernel<64><<<grid, 128, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace twk
