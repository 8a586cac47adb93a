// twk_cache_weights.cu -- what the newest tokens' attention pays to each slot of the pages (layout:
// twk_cache.cuh).
//
//     A(j) = score(j) + sum over tokens i that see j, and query heads of the KV head:
//            exp(scale q_i . k_j - lse_i)
//
// Bound by the bytes of the keys: 72 a slot (d = 128) and 8 of sums, against 128 multiplications per query
// row.  As in the attention over pages, codes enter mma.sync as f16 bit patterns as they are (a code c
// is the number c 2^-24, or 16 c one place up), 16 slots to the left operand, up to 8 query rows to
// the other one; the zeros are the accumulators' start, a scale is one multiplication per group.  With
// c = scale log2(e), a weight is 2^(c q . k - log2(e) lse).
//
// A block of four warps takes some pages of one unit, a warp a page at a time.  Its lanes load their operands
// straight from the page (512 contiguous bytes an instruction): nothing is shared between lanes, and
// enough warps are on an SM to keep loads on their way.  The query rows, scaled to f16 by a power of two
// each, are laid out once per block in shared memory, 64 rows at a time; a slot's sum is the same lanes',
// in the order of the rows, whatever the grid.
#include <algorithm>

#include "twk_cache.cuh"
#include "twk_internal.h"
#include "twk_prompt_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

constexpr int kWarps = 4;
constexpr int kParts = 8;         // of 8 rows, in shared memory at a time
constexpr int kAhead = 2, kMostPages = 8;
static_assert(kMostPages + kAhead <= 32);

struct Params {
    CacheWeightsArgs p;
    int rows;                     // G n, query rows of a unit
    int pages;                    // of a warp
    float c;                      // scale * log2(e)
    const int* seen;              // [units][1 + n], see twk_attend.cu, or null
};

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t f16_pair(float x, float y)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    return r;
}

__device__ __forceinline__ float exp2_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// What a lane keeps of a part's 8 rows: the operand's registers of column g, and of the rows 2 t and
// 2 t + 1 (the accumulator's columns) the sums of q, the factor of a score, and log2(e) lse.
template <int G>
struct Rows {
    uint32_t q[G][8];
    float sum[G][2], up[2], log[2];
    static constexpr int kWords = 10 * G + 4;
};

template <int D>
__global__ void __launch_bounds__(32 * kWarps, 4) cache_weights_kernel(const __grid_constant__ Params x)
{
    using P = PageLayout<D>;
    constexpr int G = P::kGroups;
    using R = Rows<G>;
    __shared__ uint32_t s_rows[kParts][R::kWords][32];
    const AttendArgs& a = x.p.a;
    wait_for_previous();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, t = lane % 4;
    const int unit = blockIdx.y, b = unit / a.H, h = unit - b * a.H;
    const int len = a.lens[unit];
    const bool bad = len < 0 || len > static_cast<int64_t>(a.from.max_pages) * kPage;
    const bool large = !bad && len > x.p.N;
    const int* table = a.from.table + static_cast<int64_t>(unit) * a.from.max_pages;
    if (blockIdx.x == 0 && a.out_status) {
        bool wrong = false;
        if (!bad)
            for (int j = threadIdx.x; j * kPage < len; j += 32 * kWarps)
                wrong |= static_cast<unsigned>(table[j]) >= static_cast<unsigned>(a.from.n_pages);
        wrong = __syncthreads_or(wrong);
        if (threadIdx.x == 0)
            a.out_status[unit] = large ? TWINKV_ERR_TOO_LARGE
                                       : bad || wrong ? TWINKV_ERR_INVALID_ARG : TWINKV_OK;
    }
    const int first_page = blockIdx.x * kWarps * x.pages;
    if (bad || large || first_page * kPage >= len) return;
    const int* seen = x.seen ? x.seen + static_cast<int64_t>(unit) * (1 + a.n) : nullptr;
    const int sinks = seen ? seen[0] : 0;
    // the warp's page numbers, one to a lane; its pages' keys are on their way to L2 kAhead pages before they
    // are wanted, the first ones while the query rows are laid out
    const int my_page = first_page + lane * kWarps + warp;
    const int my_id = lane < x.pages && my_page * kPage < len ? table[my_page] : -1;
    auto ahead = [&](int i) {
        const int id = __shfl_sync(0xffffffffu, my_id, i & 31);
        if (lane == 0 && i < x.pages &&
            static_cast<unsigned>(id) < static_cast<unsigned>(a.from.n_pages))
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(
                             a.from.base + static_cast<int64_t>(id) * P::kBytes),
                         "r"(P::kValCodes)
                         : "memory");
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) ahead(i);
    const float* from = x.p.score;
    for (int r0 = 0; r0 < x.rows; r0 += 8 * kParts, from = x.p.out_score) {
        // ---- the query rows
        if (r0 > 0) __syncthreads();
        const int parts = min((x.rows - r0 + 7) / 8, kParts);
        for (int part = warp; part < parts; part += kWarps) {
            const int row = r0 + 8 * part + g;
            const bool held = row < x.rows;
            const int token = row / a.G, head = h * a.G + row - token * a.G;
            uint32_t w[G][8], most = 0;
#pragma unroll
            for (int k = 0; k < G; ++k) {
                uint4 v0 = {}, v1 = {};
                if (held) {
                    const uint16_t* q = a.q + b * a.q_batch + token * a.q_token + head * a.q_head +
                                        64 * k + 16 * t;
                    v0 = *reinterpret_cast<const uint4*>(q);
                    v1 = *reinterpret_cast<const uint4*>(q + 8);
                }
                w[k][0] = v0.x, w[k][1] = v0.y, w[k][2] = v0.z, w[k][3] = v0.w;
                w[k][4] = v1.x, w[k][5] = v1.y, w[k][6] = v1.z, w[k][7] = v1.w;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    most = max(most, max(w[k][i] & 0x7fffu, w[k][i] >> 16 & 0x7fffu));
            }
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            // the row's largest value goes to [2^14, 2^15): values down to 2^-27 of it stay exact; rows of
            // exponents outside [-100, 100] are scaled as those
            const int exponent = min(max(static_cast<int>(most >> 7) - 127, -100), 100);
            const float up = __uint_as_float(static_cast<uint32_t>(127 + 14 - exponent) << 23);
            // a score's sums are of 2^(14 - exponent - 24) q c
            const float down = __uint_as_float(static_cast<uint32_t>(127 + 10 + exponent) << 23);
            const float log =
                held ? -1.4426950408889634f *
                           x.p.lse[(static_cast<int64_t>(b) * a.n + token) * (a.H * a.G) + head]
                     : -INFINITY;
            uint32_t* out = &s_rows[part][0][lane];
#pragma unroll
            for (int k = 0; k < G; ++k) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    // the odd pairs of a word's codes enter times 16
                    const float y = bf16_lo(w[k][i]) * up, z = bf16_hi(w[k][i]) * up;
                    const float f = i % 2 ? 0.0625f : 1.0f;
                    out[32 * (8 * k + i)] = f16_pair(y * f, z * f);
                    s += y + z;
                }
                s += __shfl_xor_sync(0xffffffffu, s, 1);
                s += __shfl_xor_sync(0xffffffffu, s, 2);
                s *= 0x1p-24f;
#pragma unroll
                for (int e = 0; e < 2; ++e)       // lane 4 r has row r's
                    out[32 * (8 * G + 2 * k + e)] =
                        __float_as_uint(__shfl_sync(0xffffffffu, s, 4 * (2 * t + e)));
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                out[32 * (10 * G + e)] =
                    __float_as_uint(__shfl_sync(0xffffffffu, down, 4 * (2 * t + e)) * x.c);
                out[32 * (10 * G + 2 + e)] =
                    __float_as_uint(__shfl_sync(0xffffffffu, log, 4 * (2 * t + e)));
            }
        }
        __syncthreads();

        // ---- pages
        for (int i = 0; i < x.pages; ++i) {
            const int page = first_page + i * kWarps + warp, base = page * kPage;
            if (base >= len) break;
            const int id = __shfl_sync(0xffffffffu, my_id, i);
            ahead(i + kAhead);
            const bool gone = static_cast<unsigned>(id) >= static_cast<unsigned>(a.from.n_pages);
            const uint8_t* src = a.from.base + static_cast<int64_t>(gone ? 0 : id) * P::kBytes;
            // slots 16 m + g and 16 m + 8 + g of tile m
            uint32_t code[4][2][2 * G], group[4][2][G];
            float sum[4][2];
            const int64_t at = static_cast<int64_t>(unit) * x.p.N + base;
            // slots of no token's window keep their sums
            const bool none = gone || (seen && base + kPage <= seen[1] && base >= sinks);
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int slot = 16 * m + 8 * k + g;
                    if (!none) {
                        if constexpr (D == 128) {
                            const uint4 v =
                                *reinterpret_cast<const uint4*>(src + slot * P::kRow + 16 * t);
                            code[m][k][0] = v.x, code[m][k][1] = v.y;
                            code[m][k][2] = v.z, code[m][k][3] = v.w;
                            const uint2 w = *reinterpret_cast<const uint2*>(src + P::kKeyGroups +
                                                                            slot * 8);
                            group[m][k][0] = w.x, group[m][k][1] = w.y;
                        } else {
                            const uint2 v =
                                *reinterpret_cast<const uint2*>(src + slot * P::kRow + 8 * t);
                            code[m][k][0] = v.x, code[m][k][1] = v.y;
                            group[m][k][0] = *reinterpret_cast<const uint32_t*>(
                                src + P::kKeyGroups + slot * 4);
                        }
                    }
                    sum[m][k] = 0.0f;
                }
            // the lane writes slots 16 t + 8 k + g
            float before[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int slot = 16 * t + 8 * k + g;
                before[k] = base + slot < len ? from[at + slot] : 0.0f;
            }
            for (int part = 0; part < parts && !none; ++part) {
                R r;
                const uint32_t* in = &s_rows[part][0][lane];
#pragma unroll
                for (int k = 0; k < G; ++k) {
#pragma unroll
                    for (int y = 0; y < 8; ++y) r.q[k][y] = in[32 * (8 * k + y)];
                    r.sum[k][0] = __uint_as_float(in[32 * (8 * G + 2 * k)]);
                    r.sum[k][1] = __uint_as_float(in[32 * (8 * G + 2 * k + 1)]);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    r.up[e] = __uint_as_float(in[32 * (10 * G + e)]);
                    r.log[e] = __uint_as_float(in[32 * (10 * G + 2 + e)]);
                }
                // the rows' tokens: which slots they see
                const int row = r0 + 8 * part;
                const int first_token = row / a.G, last_token = min((row + 7) / a.G, a.n - 1);
                const bool full = base + kPage <= len - a.n + first_token + 1 &&
                                  (!seen || base >= seen[1 + last_token] || base + kPage <= sinks);
                int limit[2] = {INT_MAX, INT_MAX}, low[2] = {};
                if (!full) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int token = min((row + 2 * t + e) / a.G, a.n - 1);
                        limit[e] = len - a.n + token + 1;
                        low[e] = seen ? seen[1 + token] : 0;
                    }
                }
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    float s[2][2];               // of slot k, row e
#pragma unroll
                    for (int y = 0; y < G; ++y) {
                        float acc[4];            // -z Q at first
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                acc[2 * k + e] = fmaf(bf16_hi(group[m][k][y]), r.sum[y][e],
                                                      128.0f * r.sum[y][e]);
#pragma unroll
                        for (int w = 0; w < 2; ++w)
#pragma unroll
                            for (int z = 0; z < 2; ++z) {
                                const uint32_t u = code[m][0][2 * y + w] >> (8 * z);
                                const uint32_t v = code[m][1][2 * y + w] >> (8 * z);
                                mma_f16(acc, u & 0x000f000fu, v & 0x000f000fu, u & 0x00f000f0u,
                                        v & 0x00f000f0u, r.q[y][4 * w + 2 * z],
                                        r.q[y][4 * w + 2 * z + 1]);
                            }
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float f = bf16_lo(group[m][k][y]);
                                s[k][e] = y == 0 ? acc[2 * k + e] * f
                                                 : fmaf(acc[2 * k + e], f, s[k][e]);
                            }
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float w = exp2_approx(fmaf(s[k][e], r.up[e], r.log[e]));
                            if (!full) {
                                const int slot = base + 16 * m + 8 * k + g;
                                const bool see = slot < min(limit[e], len) &&
                                                 (slot >= low[e] || slot < sinks);
                                w = see ? w : 0.0f;
                            }
                            sum[m][k] += w;
                        }
                }
            }
            // the rows of the other lanes
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    sum[m][k] += __shfl_xor_sync(0xffffffffu, sum[m][k], 1);
                    sum[m][k] += __shfl_xor_sync(0xffffffffu, sum[m][k], 2);
                }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float add = t == 0 ? sum[0][k] : t == 1 ? sum[1][k] : t == 2 ? sum[2][k]
                                                                                  : sum[3][k];
                const int slot = 16 * t + 8 * k + g;
                if (base + slot < len) x.p.out_score[at + slot] = before[k] + add;
            }
        }
    }
}

template <int D>
cudaError_t launch(const Params& x, int units, int sms, cudaStream_t st)
{
    // as few pages to a warp as leave the SMs four blocks each to do: a block's start (lengths, query
    // rows) is then seldom waited for
    Params y = x;
    const int most = (x.p.N + kPage - 1) / kPage;
    const int64_t all = static_cast<int64_t>(units) * most;
    y.pages = static_cast<int>(std::min<int64_t>(kMostPages, std::max<int64_t>(1, all / (kWarps * 4 * sms))));
    const dim3 grid((most + kWarps * y.pages - 1) / (kWarps * y.pages), units);
    if (x.seen) return launch_dependent(cache_weights_kernel<D>, grid, 32 * kWarps, 0, st, y);
    cache_weights_kernel<D><<<grid, 32 * kWarps, 0, st>>>(y);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache_weights(const CacheWeightsArgs& p, int sms, cudaStream_t st)
{
    const int units = p.a.B * p.a.H;
    Params x{};
    x.p = p;
    x.rows = p.a.G * p.a.n;
    x.c = p.a.scale * 1.4426950408889634f;
    if (p.a.window > 0) {
        int* seen = static_cast<int*>(p.a.ws);
        const cudaError_t e = launch_windows(p.a, units, seen, st);
        if (e != cudaSuccess) return e;
        x.seen = seen;
    }
    return p.a.d == 128 ? launch<128>(x, units, sms, st) : launch<64>(x, units, sms, st);
}

}  // namespace twk
