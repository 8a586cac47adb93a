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
// Up to 8 rows: a persistent kernel whose warps divide the pages of all units evenly, with the query rows in
// registers and the pages' keys on their way in rings.  More: a block of four warps to some pages of a
// unit, its query rows laid out once in shared memory, up to 64 at a time.  A slot's sum is the same
// lanes', in the order of the rows, whatever the grid.
//
// Measured (us in a graph; share of the measured copy rate by the bytes above):
//   32 x 8 units of 4k to 16k slots, 4 rows, d = 128   42.6   74 %;  d = 64, 16384 slots 45.1   60 %
//   8 units of 131009 slots, 4 rows                    23.5   53 %
//   16 x 8 units of 16384 slots, 8 rows 35.4   70 %;  16 rows 61, 41 %: blocks that start anew for some pages
//                                                each, with one page on its way
//   8 units of 2048 slots, 4 rows                       5.4
// A block of warps for each unit's pages instead of the persistent kernel: 58 us for the first, whatever its
// pages' prefetching (loads wait behind the start of each block).
#include <algorithm>
#include <atomic>

#include "twk_cache.cuh"
#include "twk_internal.h"
#include "twk_prompt_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

constexpr int kWarps = 4;
constexpr int kHalf = kPage / 2;
constexpr int kParts = 8;         // of 4 or 8 rows, in shared memory at a time
constexpr int kAhead = 1, kMostPages = 8;
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

// What a lane keeps of a part's 4 E rows, which are the other operand's columns: column 2 t + e is row E t + e
// (with four rows every second column is none).  The operand's registers of column g; and of the lane's
// E rows the sums of q, the factor of a score, and -log2(e) lse.
template <int G, int E>
struct Rows {
    uint32_t q[G][8];
    float sum[G][E], up[E], log[E];
    static constexpr int kWords = (8 + E) * G + 2 * E, kQuads = (kWords + 3) / 4;
};

// A lane's words of a part: rows r0 .. r0 + 4 E - 1 of a unit (sequence b, KV head h), in the order of Rows.
template <int D, int E>
__device__ __forceinline__ void rows_of(const Params& x, int b, int h, int r0,
                                        uint32_t (&out)[4 * Rows<D / 64, E>::kQuads])
{
    constexpr int G = D / 64;
    const AttendArgs& a = x.p.a;
    const int lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const int row = r0 + (E == 1 ? g / 2 : g);
    const bool held = row < x.rows && (E == 2 || g % 2 == 0);
    const int token = row / a.G, head = h * a.G + row - token * a.G;
    uint32_t w[G][8], most = 0;
#pragma unroll
    for (int k = 0; k < G; ++k) {
        uint4 v0 = {}, v1 = {};
        if (held) {
            const uint16_t* q =
                a.q + b * a.q_batch + token * a.q_token + head * a.q_head + 64 * k + 16 * t;
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
    const float log = held ? -1.4426950408889634f *
                                 x.p.lse[(static_cast<int64_t>(b) * a.n + token) * (a.H * a.G) + head]
                           : -INFINITY;
#pragma unroll
    for (int k = 0; k < G; ++k) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // the odd pairs of a word's codes enter times 16
            const float y = bf16_lo(w[k][i]) * up, z = bf16_hi(w[k][i]) * up;
            const float f = i % 2 ? 0.0625f : 1.0f;
            out[8 * k + i] = f16_pair(y * f, z * f);
            s += y + z;
        }
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        s += __shfl_xor_sync(0xffffffffu, s, 2);
        s *= 0x1p-24f;
#pragma unroll
        for (int e = 0; e < E; ++e)       // lanes 4 c have column c's
            out[8 * G + E * k + e] = __float_as_uint(__shfl_sync(0xffffffffu, s, 4 * (2 * t + e)));
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        out[(8 + E) * G + e] =
            __float_as_uint(__shfl_sync(0xffffffffu, down, 4 * (2 * t + e)) * x.c);
        out[(8 + E) * G + E + e] =
            __float_as_uint(__shfl_sync(0xffffffffu, log, 4 * (2 * t + e)));
    }
}

// Adds a part's weights of 32 slots from `base` on, 16 m + g and 16 m + 8 + g of them the lane's, to sum[m].
// kFull: all its rows see every slot; else row e sees those below limit[e] that are not below low[e], or
// below `sinks`.
template <int D, int E, bool kFull>
__device__ __forceinline__ void add_weights(const uint32_t (&code)[2][2][D / 32],
                                            const uint32_t (&group)[2][2][D / 64],
                                            const uint32_t* in, int base, const int (&limit)[E],
                                            const int (&low)[E], int sinks, float (&sum)[2][2])
{
    constexpr int G = D / 64;
    const int g = threadIdx.x % 32 / 4;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        float s[2][E];               // of slot k, row e
#pragma unroll
        for (int y = 0; y < G; ++y) {
            float acc[4] = {};       // -z Q at first
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    acc[2 * k + e] = (bf16_hi(group[m][k][y]) + 128.0f) *
                                     __uint_as_float(in[8 * G + E * y + e]);
#pragma unroll
            for (int w = 0; w < 2; ++w)
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const uint32_t u = code[m][0][2 * y + w] >> (8 * z);
                    const uint32_t v = code[m][1][2 * y + w] >> (8 * z);
                    const int at = 8 * y + 4 * w + 2 * z;
                    mma_f16(acc, u & 0x000f000fu, v & 0x000f000fu, u & 0x00f000f0u, v & 0x00f000f0u,
                            in[at], in[at + 1]);
                }
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float f = bf16_lo(group[m][k][y]);
                    s[k][e] = y == 0 ? acc[2 * k + e] * f : fmaf(acc[2 * k + e], f, s[k][e]);
                }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float w = exp2_approx(fmaf(s[k][e], __uint_as_float(in[(8 + E) * G + e]),
                                           __uint_as_float(in[(8 + E) * G + E + e])));
                if constexpr (!kFull) {
                    const int slot = base + 16 * m + 8 * k + g;
                    const bool see = slot < limit[e] && (slot >= low[e] || slot < sinks);
                    w = see ? w : 0.0f;
                }
                sum[m][k] += w;
            }
    }
}

// The sums of all rows of slot 16 (t / 2) + 8 (t % 2) + g: tile m's of slots k go to the lanes t = 2 m + k.
__device__ __forceinline__ float own_sum(const float (&sum)[2][2])
{
    const bool high = threadIdx.x & 2, odd = threadIdx.x & 1;
    float half[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        half[k] = (high ? sum[1][k] : sum[0][k]) +
                  __shfl_xor_sync(0xffffffffu, high ? sum[0][k] : sum[1][k], 2);
    return (odd ? half[1] : half[0]) +
           __shfl_xor_sync(0xffffffffu, odd ? half[0] : half[1], 1);
}

// More than 8 rows: a block of four warps takes some pages of one unit.
template <int D>
__global__ void __launch_bounds__(32 * kWarps, 4) cache_weights_kernel(const __grid_constant__ Params x)
{
    using P = PageLayout<D>;
    constexpr int G = P::kGroups, E = 2;
    using R = Rows<G, E>;
    constexpr int kRows = 4 * E;
    __shared__ uint4 s_rows[kParts][R::kQuads][32];
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
    for (int r0 = 0; r0 < x.rows; r0 += kRows * kParts, from = x.p.out_score) {
        // ---- the query rows
        if (r0 > 0) __syncthreads();
        const int parts = min((x.rows - r0 + kRows - 1) / kRows, kParts);
        for (int part = warp; part < parts; part += kWarps) {
            uint32_t out[4 * R::kQuads] = {};
            rows_of<D, E>(x, b, h, r0 + kRows * part, out);
#pragma unroll
            for (int i = 0; i < R::kQuads; ++i)
                s_rows[part][i][lane] =
                    make_uint4(out[4 * i], out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]);
        }
        __syncthreads();

        // ---- pages
        // half a page at a time: the operands of a whole one leave room for few warps
        for (int i = 0; i < 2 * x.pages; ++i) {
            const int page = first_page + i / 2 * kWarps + warp, in_page = i % 2 * kHalf;
            const int base = page * kPage + in_page;
            if (base >= len) break;
            const int id = __shfl_sync(0xffffffffu, my_id, i / 2);
            if (in_page == 0) ahead(i / 2 + kAhead);
            const int64_t at = static_cast<int64_t>(unit) * x.p.N + base;
            // the lane writes slot 16 (t / 2) + 8 (t % 2) + g
            const int own = 8 * t + g;
            const float before = base + own < len ? from[at + own] : 0.0f;
            // slots of no token's window, or of a page outside the pool, keep their sums
            if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.from.n_pages) ||
                (seen && base + kHalf <= seen[1] && base >= sinks)) {
                if (base + own < len) x.p.out_score[at + own] = before;
                continue;
            }
            const uint8_t* src = a.from.base + static_cast<int64_t>(id) * P::kBytes;
            // slots 16 m + g and 16 m + 8 + g of the half's tile m
            uint32_t code[2][2][2 * G], group[2][2][G];
            float sum[2][2];
            const uint8_t* src_code = src + (in_page + g) * P::kRow + 8 * G * t;
            const uint8_t* src_group = src + P::kKeyGroups + (in_page + g) * 4 * G;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int slot = 16 * m + 8 * k;
                    if constexpr (D == 128) {
                        const uint4 v = *reinterpret_cast<const uint4*>(src_code + slot * P::kRow);
                        code[m][k][0] = v.x, code[m][k][1] = v.y;
                        code[m][k][2] = v.z, code[m][k][3] = v.w;
                        const uint2 w = *reinterpret_cast<const uint2*>(src_group + slot * 8);
                        group[m][k][0] = w.x, group[m][k][1] = w.y;
                    } else {
                        const uint2 v = *reinterpret_cast<const uint2*>(src_code + slot * P::kRow);
                        code[m][k][0] = v.x, code[m][k][1] = v.y;
                        group[m][k][0] = *reinterpret_cast<const uint32_t*>(src_group + slot * 4);
                    }
                    sum[m][k] = 0.0f;
                }
            for (int part = 0; part < parts; ++part) {
                // operands are made anew for every part: kept over parts they would not fit the registers
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int y = 0; y < 2 * G; ++y) asm volatile("" : "+r"(code[m][k][y]));
                uint32_t in[4 * R::kQuads];
#pragma unroll
                for (int y = 0; y < R::kQuads; ++y) {
                    const uint4 v = s_rows[part][y][lane];
                    in[4 * y] = v.x, in[4 * y + 1] = v.y, in[4 * y + 2] = v.z, in[4 * y + 3] = v.w;
                }
                const int row = r0 + kRows * part;
                const int first_token = row / a.G, last_token = min((row + kRows - 1) / a.G, a.n - 1);
                int limit[E] = {}, low[E] = {};
                if (base + kHalf <= len - a.n + first_token + 1 &&
                    (!seen || base >= seen[1 + last_token] || base + kHalf <= sinks)) {
                    add_weights<D, E, true>(code, group, in, base, limit, low, sinks, sum);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int token = min((row + E * t + e) / a.G, a.n - 1);
                        limit[e] = min(len - a.n + token + 1, len);
                        low[e] = seen ? seen[1 + token] : 0;
                    }
                    add_weights<D, E, false>(code, group, in, base, limit, low, sinks, sum);
                }
            }
            const float add = own_sum(sum);
            if (base + own < len) x.p.out_score[at + own] = before + add;
        }
    }
}

template <int D>
cudaError_t launch_many(const Params& x, int units, int sms, cudaStream_t st)
{
    // as few pages to a warp as leave the SMs four blocks each to do: a block's start (lengths, query
    // rows) is then seldom waited for
    Params y = x;
    const int most = (x.p.N + kPage - 1) / kPage;
    const int64_t all = static_cast<int64_t>(units) * most;
    y.pages = static_cast<int>(
        std::min<int64_t>(kMostPages, std::max<int64_t>(1, all / (kWarps * 4 * sms))));
    const dim3 grid((most + kWarps * y.pages - 1) / (kWarps * y.pages), units);
    if (x.seen) return launch_dependent(cache_weights_kernel<D>, grid, 32 * kWarps, 0, st, y);
    cache_weights_kernel<D><<<grid, 32 * kWarps, 0, st>>>(y);
    return cudaGetLastError();
}

// ---- up to 8 rows

// Persistent: the pages of all units in one sequence are divided evenly among the warps of the grid.  A warp
// keeps its unit's query rows in registers and has its pages' keys copied into its own ring in shared
// memory, two pages ahead (cp.async, 16 bytes a lane).
constexpr int kFewWarps = 16;

template <int D>
struct Few {
    static constexpr int kKeys = PageLayout<D>::kValCodes;            // bytes of a page's keys
    static constexpr int kStages = 221184 / (kFewWarps * kKeys);
    static constexpr int kRings = kFewWarps * kStages * kKeys;
    static constexpr int kMostChunks = 2048;                          // of 32 units
    static_assert(kKeys % 16 == 0 && kStages >= 3);
    static_assert(kRings + (kMostChunks + 1) * 4 <= 232448, "shared memory per block");
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// pages of a unit: 0 where its length is an error
__device__ __forceinline__ int pages_of(const Params& x, int unit, int& len)
{
    len = x.p.a.lens[unit];
    if (len < 0 || len > static_cast<int64_t>(x.p.a.from.max_pages) * kPage || len > x.p.N) len = 0;
    return (len + kPage - 1) / kPage;
}

template <int D, int E>
__global__ void __launch_bounds__(32 * kFewWarps, 1)
    cache_weights_few_kernel(const __grid_constant__ Params x, int units)
{
    using P = PageLayout<D>;
    using F = Few<D>;
    constexpr int G = P::kGroups;
    extern __shared__ __align__(128) uint8_t smem[];
    int* sums = reinterpret_cast<int*>(smem + F::kRings);
    const AttendArgs& a = x.p.a;
    wait_for_previous();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, t = lane % 4;
    const int chunks = (units + 31) / 32;

    // pages before each 32 units: a single chunk is summed by every warp for itself
    int total = 0, none = 0;
    if (chunks == 1) {
        total = __reduce_add_sync(0xffffffffu, lane < units ? pages_of(x, lane, none) : 0);
    } else {
        for (int c = warp; c < chunks; c += kFewWarps) {
            const int u = 32 * c + lane;
            const int n = __reduce_add_sync(0xffffffffu, u < units ? pages_of(x, u, none) : 0);
            if (lane == 0) sums[c] = n;
        }
        __syncthreads();
        if (warp == 0) {
            for (int c0 = 0; c0 < chunks; c0 += 32) {
                const int n = c0 + lane < chunks ? sums[c0 + lane] : 0;
                int scan = n;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) {
                    const int y = __shfl_up_sync(0xffffffffu, scan, o);
                    if (lane >= o) scan += y;
                }
                if (c0 + lane < chunks) sums[c0 + lane] = total + scan - n;
                total += __shfl_sync(0xffffffffu, scan, 31);
            }
            if (lane == 0) sums[chunks] = total;
        }
        __syncthreads();
        total = sums[chunks];
    }
    // neighbours in the sequence of pages go to different SMs, a warp's own pages to it
    const unsigned workers = gridDim.x * kFewWarps, worker = warp * gridDim.x + blockIdx.x;
    const unsigned each = static_cast<unsigned>(total) / workers, over = total % workers;
    const int begin = static_cast<int>(each * worker + static_cast<uint64_t>(over) * worker / workers);
    int todo = static_cast<int>(each * (worker + 1) +
                                static_cast<uint64_t>(over) * (worker + 1) / workers) - begin;

    if (a.out_status)
        for (int u = worker; u < units; u += workers) {
            const int len = a.lens[u];
            const bool bad = len < 0 || len > static_cast<int64_t>(a.from.max_pages) * kPage;
            const int* table = a.from.table + static_cast<int64_t>(u) * a.from.max_pages;
            bool wrong = bad;
            for (int j = lane; !bad && j * kPage < len; j += 32)
                wrong |= static_cast<unsigned>(table[j]) >= static_cast<unsigned>(a.from.n_pages);
            wrong = __any_sync(0xffffffffu, wrong);
            if (lane == 0)
                a.out_status[u] = !bad && len > x.p.N ? TWINKV_ERR_TOO_LARGE
                                  : wrong             ? TWINKV_ERR_INVALID_ARG
                                                      : TWINKV_OK;
        }
    if (todo == 0) return;

    // the span's first page
    struct Place {
        int unit, j, pages, len;
    };
    Place at{};
    {
        int lo = 0, before = 0;
        if (chunks > 1) {
            for (int hi = chunks - 1; lo < hi;) {
                const int mid = (lo + hi + 1) / 2;
                if (sums[mid] <= begin) lo = mid;
                else hi = mid - 1;
            }
            before = sums[lo];
        }
        const int u = 32 * lo + lane, n = u < units ? pages_of(x, u, none) : 0;
        int scan = n;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int y = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += y;
        }
        const int rest = begin - before;
        const int l = __ffs(__ballot_sync(0xffffffffu, scan > rest)) - 1;
        at.unit = 32 * lo + l;
        at.j = rest - (__shfl_sync(0xffffffffu, scan, l) - __shfl_sync(0xffffffffu, n, l));
        at.pages = pages_of(x, at.unit, at.len);
    }
    auto advance = [&](Place& f) {           // only where a page is left
        if (++f.j < f.pages) return;
        f.j = 0;
        do f.pages = pages_of(x, ++f.unit, f.len);
        while (f.pages == 0);
    };
    // slots of no token's window, or of a page outside the pool, keep their sums
    auto unseen = [&](const Place& f, int id) {
        if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.from.n_pages)) return true;
        if (!x.seen) return false;
        const int* seen = x.seen + static_cast<int64_t>(f.unit) * (1 + a.n);
        return f.j * kPage + kPage <= seen[1] && f.j * kPage >= seen[0];
    };
    auto number = [&](const Place& f) {
        return a.from.table[static_cast<int64_t>(f.unit) * a.from.max_pages + f.j];
    };

    // ---- copies run kStages pages ahead
    const uint32_t ring = smem_u32(smem + warp * F::kStages * F::kKeys);
    Place ahead = at;
    int ahead_todo = todo;
    uint32_t skip = 0;                       // stages without keys
    auto copy = [&](int stage) {
        skip &= ~(1u << stage);
        if (ahead_todo > 0) {
            const int id = number(ahead);
            if (unseen(ahead, id)) {
                skip |= 1u << stage;
            } else {
                const uint8_t* src = a.from.base + static_cast<int64_t>(id) * P::kBytes;
                const uint32_t dst = ring + stage * F::kKeys;
#pragma unroll
                for (int i = 0; i < (F::kKeys + 511) / 512; ++i)
                    if (F::kKeys % 512 == 0 || 512 * i + 16 * lane < F::kKeys)
                        cp_async16(dst + 512 * i + 16 * lane, src + 512 * i + 16 * lane);
            }
            if (--ahead_todo > 0) advance(ahead);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < F::kStages; ++s) copy(s);

    // ---- pages
    uint32_t rows[4 * Rows<G, E>::kQuads] = {};
    int unit = -1;
    const int own = 8 * t + g;               // and 32 more: the slots that the lane writes
    for (int stage = 0; todo > 0; --todo) {
        const int64_t out = static_cast<int64_t>(at.unit) * x.p.N + at.j * kPage;
        float before[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int slot = at.j * kPage + 32 * h + own;
            before[h] = slot < at.len ? x.p.score[out + 32 * h + own] : 0.0f;
        }
        if (at.unit != unit) {
            unit = at.unit;
            rows_of<D, E>(x, unit / a.H, unit % a.H, 0, rows);
        }
        const int* seen = x.seen ? x.seen + static_cast<int64_t>(unit) * (1 + a.n) : nullptr;
        const int sinks = seen ? seen[0] : 0;
        asm volatile("cp.async.wait_group %0;" ::"n"(F::kStages - 1) : "memory");
        __syncwarp();
        const bool dark = skip >> stage & 1u;
        const uint8_t* src = smem + (warp * F::kStages + stage) * F::kKeys;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int base = at.j * kPage + 32 * h;
            float add = 0.0f;
            if (!dark && base < at.len) {
                uint32_t code[2][2][2 * G], group[2][2][G];
                float sum[2][2] = {};
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int slot = 32 * h + 16 * m + 8 * k + g;
                        if constexpr (D == 128) {
                            const uint4 v =
                                *reinterpret_cast<const uint4*>(src + slot * P::kRow + 16 * t);
                            code[m][k][0] = v.x, code[m][k][1] = v.y;
                            code[m][k][2] = v.z, code[m][k][3] = v.w;
                            const uint2 w =
                                *reinterpret_cast<const uint2*>(src + P::kKeyGroups + slot * 8);
                            group[m][k][0] = w.x, group[m][k][1] = w.y;
                        } else {
                            const uint2 v =
                                *reinterpret_cast<const uint2*>(src + slot * P::kRow + 8 * t);
                            code[m][k][0] = v.x, code[m][k][1] = v.y;
                            group[m][k][0] = *reinterpret_cast<const uint32_t*>(
                                src + P::kKeyGroups + slot * 4);
                        }
                    }
                int limit[E] = {}, low[E] = {};
                // every row: the first token sees least at the end, the last at the window's begin
                if (base + 32 <= at.len - a.n + 1 &&
                    (!seen || base >= seen[a.n] || base + 32 <= sinks)) {
                    add_weights<D, E, true>(code, group, rows, base, limit, low, sinks, sum);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const int token = min((E * t + e) / a.G, a.n - 1);
                        limit[e] = min(at.len - a.n + token + 1, at.len);
                        low[e] = seen ? seen[1 + token] : 0;
                    }
                    add_weights<D, E, false>(code, group, rows, base, limit, low, sinks, sum);
                }
                add = own_sum(sum);
            }
            if (base + own < at.len) x.p.out_score[out + 32 * h + own] = before[h] + add;
        }
        __syncwarp();
        copy(stage);
        if (++stage == F::kStages) stage = 0;
        if (todo > 1) advance(at);
    }
}

template <int D, int E>
cudaError_t launch_few(const Params& x, int units, int sms, cudaStream_t st)
{
    using F = Few<D>;
    constexpr int kMost = F::kRings + (F::kMostChunks + 1) * 4;
    static std::atomic<bool> allowed[64];     // by device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(cache_weights_few_kernel<D, E>,
                                 cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
    }
    const int bytes = F::kRings + ((units + 31) / 32 + 1) * 4;
    if (x.seen)
        return launch_dependent(cache_weights_few_kernel<D, E>, dim3(sms), 32 * kFewWarps, bytes, st,
                                x, units);
    cache_weights_few_kernel<D, E><<<sms, 32 * kFewWarps, bytes, st>>>(x, units);
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
    if (x.rows <= 4)
        return p.a.d == 128 ? launch_few<128, 1>(x, units, sms, st)
                            : launch_few<64, 1>(x, units, sms, st);
    if (x.rows <= 8)
        return p.a.d == 128 ? launch_few<128, 2>(x, units, sms, st)
                            : launch_few<64, 2>(x, units, sms, st);
    return p.a.d == 128 ? launch_many<128>(x, units, sms, st) : launch_many<64>(x, units, sms, st);
}

}  // namespace twk
