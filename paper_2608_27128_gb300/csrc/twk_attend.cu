// twk_attend.cu -- attention of the newest tokens over a cache held in 4 bits
// (layout: twk_cache.cuh).
//
// Per unit (sequence b, KV head h), query token i of n and query head of the group:
//     p_j = softmax over the slots j that i sees of scale * q . k_j,     o = sum_j p_j v_j,
// k_j = s (c - z) per group of 64 dimensions, v_j likewise.  Token i is the one in slot len - n + i;
// it sees the slots up to its own and, with a window, of those only the ones whose position is
// within the window of its own or below n_sink.  A query that sees nothing gives 0.
//
// Bound by memory: 144 bytes a slot (d = 128) against 512 operations per query row, and a unit has
// G n rows, 4 to 16 as a rule.  So what a slot costs in instructions counts, and the design is for
// few of them:
//   - Codes enter the tensor cores as the bf16 numbers 128 + c (exact), three instructions for two
//     pairs; nothing is subtracted or scaled per element.  With Q_G the sum of q over a group,
//         q . k = sum_G s_G (sum q (128 + c) - (128 + z_G) Q_G):
//     the second term is the accumulator's start value, the scale one multiplication per group.
//     For values the scale goes into the probabilities, P s rounded to bf16 (2^-9 relative, as
//     large as the output's own rounding, and independent from slot to slot), and the zeros into
//     one more product with the same rounded numbers, so that no rounding error is multiplied by 128.
//   - mma.sync m16n8k16 with the cache as the 16-row operand (slots for keys, dimensions for values)
//     and up to 8 query rows as the other one: 18 multiplications for 16 slots at d = 128.  With
//     tcgen05 the cache would have to be written to shared memory again as bf16, four times its
//     bytes, for a 128-row operand; here codes go from the page to registers to the multiplication.
//   - A warp works alone: it takes pages in order, keeps the running maxima, sums and outputs of its
//     rows in registers, and has its pages' bytes copied into its own ring in shared memory (cp.async,
//     16 bytes a lane), two pages ahead.  No block barrier after the start.
//
// The pages of all units in one sequence are divided evenly among all warps of the grid, whatever
// the units' lengths: a warp's span may begin and end inside a unit.  A unit that lies in
// one span is written at once; of the others each warp writes its part (maximum, sum, unnormalised
// output), and merge_kernel joins them in the order of the slots.
#include <algorithm>
#include <climits>

#include "twk_cache.cuh"
#include "twk_cache_internal.h"
#include "twk_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

template <int D, int NT>
struct Config {
    // NT: groups of 8 query rows.  A warp's registers: 32 NT (d = 128) of output, 16 NT of queries,
    // 32 NT of scores and probabilities.
    static constexpr int kWarps = NT == 1 ? 12 : 8;
    static constexpr int kHalf = PageLayout<D>::kValCodes;        // bytes of a page's keys
    static constexpr int kStages = (NT == 1 ? 2 : 3) * (128 / D); // pages of a warp's ring
    static constexpr int kRing = 2 * kHalf * kStages;
    static_assert(PageLayout<D>::kPos == 2 * kHalf, "values take as many bytes as keys");
    static_assert(kHalf % 16 == 0);
};

struct AttendParams {
    AttendArgs a;
    int units, parts;        // parts: row parts (8 NT rows) of a unit
    int rows;                // G n
    int chunks;              // of 32 (unit, part) pairs
    float c;                 // scale * log2(e)
    const int* seen;         // [units][1 + n]: slots below n_sink, window's first slot per token
    float* part;             // [2 warps of the grid][8 NT D + 16 NT]
    int2* spans;             // [units * parts]: first part, last warp
};

// What a query row part of a unit visits: the pages of the sinks, then those of the window.
struct Visit {
    int len, sink_pages, skip, count;    // page j of the visit is page j, or j + skip past the sinks
};

__device__ __forceinline__ Visit visit_of(const AttendParams& p, int unit)
{
    Visit v;
    int len = p.a.lens[unit];
    if (len < 0 || len > static_cast<int64_t>(p.a.from.max_pages) * kPage) len = 0;
    const int pages = (len + kPage - 1) / kPage;
    v.len = len;
    v.sink_pages = 0;
    v.skip = 0;
    if (p.seen) {
        const int* s = p.seen + static_cast<int64_t>(unit) * (1 + p.a.n);
        const int sink = (s[0] + kPage - 1) / kPage, first = s[1] / kPage;
        if (first > sink) {
            v.sink_pages = sink;
            v.skip = first - sink;
        }
    }
    v.count = pages - v.skip;
    return v;
}

// floats of a part: outputs, maxima, sums
template <int D, int NT>
constexpr int kPartSize = 8 * NT * D + 16 * NT;

// row of out and out_lse
__device__ __forceinline__ int64_t out_row(const AttendParams& p, int unit, int row)
{
    const int b = unit / p.a.H, h = unit % p.a.H;
    return (static_cast<int64_t>(b) * p.a.n + row / p.a.G) * (p.a.H * p.a.G) + h * p.a.G +
           row % p.a.G;
}

// log of the softmax's denominator
__device__ __forceinline__ float log_sum(const AttendParams& p, float top, float sum)
{
    return sum > 0.0f ? top * p.a.scale + logf(sum) : -INFINITY;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit()
{
    asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int kPending>
__device__ __forceinline__ void cp_async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 8 x 8 block of 16-bit numbers, thread (g, t) holding row g, columns 2 t and 2 t + 1: transposed
__device__ __forceinline__ uint32_t transpose16(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

__device__ __forceinline__ float exp2_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

__device__ __forceinline__ uint4 lds128(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t at)
{
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at));
    return v;
}

// The G words (or halves) that a lane wants of one slot.
template <int D>
__device__ __forceinline__ void load_groups(uint32_t at, uint32_t (&w)[D / 64])
{
    if constexpr (D == 128) {
        const uint2 v = lds64(at);
        w[0] = v.x;
        w[1] = v.y;
    } else {
        w[0] = lds32(at);
    }
}
template <int D>
__device__ __forceinline__ void load_scales(uint32_t at, float (&s)[D / 64])
{
    if constexpr (D == 128) {
        const uint32_t v = lds32(at);
        s[0] = bf16_lo(v);
        s[1] = bf16_hi(v);
    } else {
        s[0] = bf16_lo(lds16(at));
    }
}

// The warp's place in the sequence of all pages: (unit, part) pair and page of its visit.
struct Place {
    int pair, j;
    Visit v;
};

template <int D, int NT>
__global__ void __launch_bounds__(32 * Config<D, NT>::kWarps, 1)
    attend_kernel(const __grid_constant__ AttendParams p)
{
    using P = PageLayout<D>;
    using C = Config<D, NT>;
    constexpr int G = P::kGroups, M = D / 16;
    constexpr int kRows = 8 * NT;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int s_pair[C::kWarps], s_slot[C::kWarps];
    __shared__ bool s_begins[C::kWarps], s_ends[C::kWarps];
    int* chunk_pages = reinterpret_cast<int*>(smem + C::kWarps * C::kRing);
    wait_for_previous();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, t = lane % 4;
    const int pairs = p.units * p.parts;

    // pages before each chunk of 32 pairs
    for (int c = warp; c < p.chunks; c += C::kWarps) {
        const int pair = 32 * c + lane;
        int n = pair < pairs ? visit_of(p, pair / p.parts).count : 0;
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) chunk_pages[c] = n;
    }
    __syncthreads();
    if (warp == 0) {
        int before = 0;
        for (int c0 = 0; c0 < p.chunks; c0 += 32) {
            const int n = c0 + lane < p.chunks ? chunk_pages[c0 + lane] : 0;
            int scan = n;
#pragma unroll
            for (int m = 1; m < 32; m *= 2) {
                const int y = __shfl_up_sync(0xffffffffu, scan, m);
                if (lane >= m) scan += y;
            }
            if (c0 + lane < p.chunks) chunk_pages[c0 + lane] = before + scan - n;
            before += __shfl_sync(0xffffffffu, scan, 31);
        }
        if (lane == 0) chunk_pages[p.chunks] = before;
    }
    __syncthreads();
    const int64_t total = chunk_pages[p.chunks];
    // Blocks, and warps within a block, that have a page each, as even as can be; the spans of a
    // block's warps follow one another.
    const int64_t blocks = min(total, static_cast<int64_t>(gridDim.x));
    const int64_t workers = min(total, static_cast<int64_t>(gridDim.x) * C::kWarps);
    if (blockIdx.x >= blocks) return;
    const int64_t index = workers * blockIdx.x / blocks + warp;
    const bool has_span = index < workers * (blockIdx.x + 1) / blocks;
    const int worker = blockIdx.x * C::kWarps + warp;
    const int64_t begin = has_span ? total * index / workers : 0;
    int todo = has_span ? static_cast<int>(total * (index + 1) / workers - begin) : 0;

    // the span's first page
    Place at = {};
    if (has_span) {
        int lo = 0, hi = p.chunks - 1;       // last chunk that starts at or before `begin`
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (chunk_pages[mid] <= begin) lo = mid;
            else hi = mid - 1;
        }
        const int pair = 32 * lo + lane;
        const int n = pair < pairs ? visit_of(p, pair / p.parts).count : 0;
        int scan = n;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            const int y = __shfl_up_sync(0xffffffffu, scan, m);
            if (lane >= m) scan += y;
        }
        const int rest = static_cast<int>(begin - chunk_pages[lo]);
        const unsigned past = __ballot_sync(0xffffffffu, scan > rest);
        const int l = __ffs(past) - 1;
        at.pair = 32 * lo + l;
        at.j = rest - (__shfl_sync(0xffffffffu, scan, l) - __shfl_sync(0xffffffffu, n, l));
        at.v = visit_of(p, at.pair / p.parts);
    }

    // ---- copies: the page `ahead` is one past those in the ring; its number is already loaded
    Place ahead = at;
    int ahead_todo = todo;
    auto next_id = [&]() -> int {
        if (ahead_todo == 0) return -1;
        --ahead_todo;
        while (ahead.j >= ahead.v.count) {
            ++ahead.pair;
            ahead.v = visit_of(p, ahead.pair / p.parts);
            ahead.j = 0;
        }
        const int page = ahead.j + (ahead.j < ahead.v.sink_pages ? 0 : ahead.v.skip);
        ++ahead.j;
        return p.a.from.table[static_cast<int64_t>(ahead.pair / p.parts) * p.a.from.max_pages +
                              page];
    };
    const uint32_t ring = smem_u32(smem + warp * C::kRing);
    auto copy_half = [&](int id, int stage, int half) {
        if (static_cast<unsigned>(id) < static_cast<unsigned>(p.a.from.n_pages)) {
            const uint8_t* src =
                p.a.from.base + static_cast<int64_t>(id) * P::kBytes + half * C::kHalf;
            const uint32_t dst = ring + (2 * stage + half) * C::kHalf;
#pragma unroll
            for (int i = 0; i < (C::kHalf + 511) / 512; ++i)
                if (C::kHalf % 512 == 0 || 512 * i + 16 * lane < C::kHalf)
                    cp_async16(dst + 512 * i + 16 * lane, src + 512 * i + 16 * lane);
        }
        cp_async_commit();
    };
    uint32_t absent = 0;       // stages whose page number is outside the pool
    int id = next_id();
#pragma unroll
    for (int s = 0; s < C::kStages; ++s) {
        copy_half(id, s, 0);
        copy_half(id, s, 1);
        if (static_cast<unsigned>(id) >= static_cast<unsigned>(p.a.from.n_pages)) absent |= 1u << s;
        id = next_id();
    }

    // ---- state of the unit's rows: thread (g, t) has the columns 2 t and 2 t + 1 of every 8 rows
    uint32_t q[NT][G][8];
    float qsum[NT][G][2];
    float o[NT][M][4], zero_part[NT][G][4], top[NT][2], sum[NT][2];
    int limit[NT][2], from[NT][2];    // row sees slots < limit that are >= from or < sinks
    int sinks = 0, all_limit = 0, all_from = 0;
    int seg_begin = 0;
    bool first_seg = true;

    auto start_unit = [&]() {
        const int unit = at.pair / p.parts, r0 = at.pair % p.parts * kRows;
        const int b = unit / p.a.H, h = unit % p.a.H;
        seg_begin = at.j;
        const int* seen =
            p.seen ? p.seen + static_cast<int64_t>(unit) * (1 + p.a.n) : nullptr;
        sinks = seen ? seen[0] : 0;
        all_limit = INT_MAX;
        all_from = 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = r0 + 8 * nt + g;
            const uint16_t* src = nullptr;
            if (r < p.rows)
                src = p.a.q + b * p.a.q_batch + r / p.a.G * p.a.q_token +
                      (h * p.a.G + r % p.a.G) * p.a.q_head;
#pragma unroll
            for (int G_ = 0; G_ < G; ++G_) {
                uint4 v0 = {}, v1 = {};
                if (src) {
                    v0 = *reinterpret_cast<const uint4*>(src + 64 * G_ + 16 * t);
                    v1 = *reinterpret_cast<const uint4*>(src + 64 * G_ + 16 * t + 8);
                }
                const uint32_t w[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    q[nt][G_][i] = w[i];
                    s += bf16_lo(w[i]) + bf16_hi(w[i]);
                }
                s += __shfl_xor_sync(0xffffffffu, s, 1);
                s += __shfl_xor_sync(0xffffffffu, s, 2);
                qsum[nt][G_][0] = __shfl_sync(0xffffffffu, s, 8 * t);
                qsum[nt][G_][1] = __shfl_sync(0xffffffffu, s, 8 * t + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) zero_part[nt][G_][i] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = r0 + 8 * nt + 2 * t + e, token = row / p.a.G;
                limit[nt][e] = row < p.rows ? at.v.len - p.a.n + token + 1 : INT_MAX;
                from[nt][e] = row < p.rows && seen ? seen[1 + token] : 0;
                top[nt][e] = -INFINITY;
                sum[nt][e] = 0.0f;
            }
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[nt][m][i] = 0.0f;
        }
        // every row of the part: the first token sees least at the end, the last at the window's
        // begin
        const int first_token = r0 / p.a.G, last_token = (min(r0 + kRows, p.rows) - 1) / p.a.G;
        all_limit = at.v.len - p.a.n + first_token + 1;
        all_from = seen ? seen[1 + last_token] : 0;
    };

    // the sums of the lanes that share a row; the zeros' part joins the output
    auto close_rows = [&]() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float s = sum[nt][e];
                s += __shfl_xor_sync(0xffffffffu, s, 4);
                s += __shfl_xor_sync(0xffffffffu, s, 8);
                s += __shfl_xor_sync(0xffffffffu, s, 16);
                sum[nt][e] = s;
            }
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][m][e] += zero_part[nt][m / 4][e % 2];
        }
    };
    // rows as maxima, sums and outputs [kRows][D], [kRows], [kRows]
    auto put_part = [&](float* part) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    part[(8 * nt + 2 * t + e % 2) * D + 16 * m + 8 * (e / 2) + g] = o[nt][m][e];
            if (g == 0) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    part[kRows * D + 8 * nt + 2 * t + e] = top[nt][e];
                    part[kRows * D + kRows + 8 * nt + 2 * t + e] = sum[nt][e];
                }
            }
        }
    };
    // a unit that ends inside the span: written at once if it began there
    auto finish_unit = [&]() {
        close_rows();
        if (seg_begin > 0) {
            put_part(p.part + static_cast<int64_t>(2 * worker) * kPartSize<D, NT>);
            if (lane == 0) p.spans[at.pair].y = worker;
            return;
        }
        if (lane == 0) p.spans[at.pair] = make_int2(0, -1);
        const int r0 = at.pair % p.parts * kRows;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float inv[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) inv[e] = sum[nt][e] > 0.0f ? 1.0f / sum[nt][e] : 0.0f;
            const int row = r0 + 8 * nt + g;
            uint16_t* out = p.a.out + out_row(p, at.pair / p.parts, row) * D;
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const uint32_t w =
                        transpose16(bf16_pair(o[nt][m][e] * inv[0], o[nt][m][e + 1] * inv[1]));
                    if (row < p.rows)
                        *reinterpret_cast<uint32_t*>(out + 16 * m + 4 * e + 2 * t) = w;
                }
            if (p.a.out_lse && g == 0) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = r0 + 8 * nt + 2 * t + e;
                    if (r < p.rows)
                        p.a.out_lse[out_row(p, at.pair / p.parts, r)] =
                            log_sum(p, top[nt][e], sum[nt][e]);
                }
            }
        }
    };

    if (todo > 0) start_unit();
    for (int stage = 0; todo > 0;) {
        const int page = at.j + (at.j < at.v.sink_pages ? 0 : at.v.skip);
        const int base = page * kPage;
        const bool gone = absent >> stage & 1;
        const bool full = !gone && base + kPage <= all_limit &&
                          (base >= all_from || base + kPage <= sinks);
        const uint32_t keys = ring + 2 * stage * C::kHalf, values = keys + C::kHalf;
        const bool id_ok = static_cast<unsigned>(id) < static_cast<unsigned>(p.a.from.n_pages);

        // ---- scores of 64 slots
        cp_async_wait<2 * C::kStages - 1>();
        __syncwarp();
        float s[NT][4][4];
#pragma unroll
        for (int tile = 0; tile < 4; ++tile) {
            const int lo = 16 * tile + g;
            uint32_t a0[4 * G / 2], a1[4 * G / 2];    // words of slots lo and lo + 8
            if constexpr (D == 128) {
                const uint4 u = lds128(keys + lo * P::kRow + 16 * t);
                const uint4 w = lds128(keys + (lo + 8) * P::kRow + 16 * t);
                a0[0] = u.x, a0[1] = u.y, a0[2] = u.z, a0[3] = u.w;
                a1[0] = w.x, a1[1] = w.y, a1[2] = w.z, a1[3] = w.w;
            } else {
                const uint2 u = lds64(keys + lo * P::kRow + 8 * t);
                const uint2 w = lds64(keys + (lo + 8) * P::kRow + 8 * t);
                a0[0] = u.x, a0[1] = u.y;
                a1[0] = w.x, a1[1] = w.y;
            }
            uint32_t k0[G], k1[G];
            load_groups<D>(keys + P::kKeyGroups + lo * 4 * G, k0);
            load_groups<D>(keys + P::kKeyGroups + (lo + 8) * 4 * G, k1);
#pragma unroll
            for (int G_ = 0; G_ < G; ++G_) {
                float acc[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        acc[nt][e] = bf16_hi(k0[G_]) * qsum[nt][G_][e];
                        acc[nt][2 + e] = bf16_hi(k1[G_]) * qsum[nt][G_][e];
                    }
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const uint32_t u = a0[2 * G_ + w], v = a1[2 * G_ + w];
                        const uint32_t r0 = code_pair(u, 2 * x), r1 = code_pair(v, 2 * x);
                        const uint32_t r2 = code_pair(u, 2 * x + 1), r3 = code_pair(v, 2 * x + 1);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            mma_bf16(acc[nt], r0, r1, r2, r3, q[nt][G_][4 * w + 2 * x],
                                     q[nt][G_][4 * w + 2 * x + 1]);
                    }
                const float s0 = bf16_lo(k0[G_]), s1 = bf16_lo(k1[G_]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float f = e < 2 ? s0 : s1;
                        s[nt][tile][e] = G_ == 0 ? acc[nt][e] * f
                                                 : fmaf(acc[nt][e], f, s[nt][tile][e]);
                    }
            }
        }
        __syncwarp();
        copy_half(id, stage, 0);
        if (!full) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int tile = 0; tile < 4; ++tile)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int slot = base + 16 * tile + 8 * (e / 2) + g;
                        const bool see = !gone && slot < min(limit[nt][e % 2], at.v.len) &&
                                         (slot >= from[nt][e % 2] || slot < sinks);
                        if (!see) s[nt][tile][e] = -INFINITY;
                    }
        }

        // ---- running maxima; probabilities
        bool grown = false;
        float shift[NT][2], shrink[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float m = fmaxf(s[nt][0][e], s[nt][0][2 + e]);
#pragma unroll
                for (int tile = 1; tile < 4; ++tile)
                    m = fmaxf(m, fmaxf(s[nt][tile][e], s[nt][tile][2 + e]));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                m = fmaxf(m, top[nt][e]);
                grown |= m > top[nt][e];
                // a row that has seen nothing yet keeps -inf, and its probabilities are 0
                shift[nt][e] = m == -INFINITY ? 0.0f : m * p.c;
                shrink[nt][e] = top[nt][e] == -INFINITY ? 0.0f
                                                        : exp2_approx((top[nt][e] - m) * p.c);
                top[nt][e] = m;
            }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2; ++e) sum[nt][e] *= shrink[nt][e];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int m = 0; m < M; ++m) o[nt][m][i] *= shrink[nt][i % 2];
#pragma unroll
                    for (int G_ = 0; G_ < G; ++G_) zero_part[nt][G_][i] *= shrink[nt][i % 2];
                }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int tile = 0; tile < 4; ++tile)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = exp2_approx(fmaf(s[nt][tile][e], p.c, -shift[nt][e % 2]));
                    s[nt][tile][e] = x;
                    sum[nt][e % 2] += x;
                }

        // ---- values
        cp_async_wait<2 * C::kStages - 1>();
        __syncwarp();
        uint32_t prob[NT][4][G][2];      // P s, bf16, slots in the order of the value codes
#pragma unroll
        for (int tile = 0; tile < 4; ++tile) {
            float v0[G], v1[G];
            load_scales<D>(values + P::kValScales - P::kValCodes + (16 * tile + g) * 2 * G, v0);
            load_scales<D>(values + P::kValScales - P::kValCodes + (16 * tile + 8 + g) * 2 * G, v1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int G_ = 0; G_ < G; ++G_) {
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[e] = s[nt][tile][e] * (e < 2 ? v0[G_] : v1[G_]);
                        // what an unseen slot holds may be anything
                        if (!full && s[nt][tile][e] == 0.0f) x[e] = 0.0f;
                    }
                    prob[nt][tile][G_][0] = transpose16(bf16_pair(x[0], x[1]));
                    prob[nt][tile][G_][1] = transpose16(bf16_pair(x[2], x[3]));
                }
        }
#pragma unroll
        for (int G_ = 0; G_ < G; ++G_)
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                uint4 z = lds128(values + P::kValZeros - P::kValCodes + G_ * 2 * kPage + 32 * t +
                                 16 * a);
                if (!full) {     // likewise, where it would not be a number
                    z.x = (z.x & 0x000f000fu) | 0xc300c300u;
                    z.y = (z.y & 0x000f000fu) | 0xc300c300u;
                    z.z = (z.z & 0x000f000fu) | 0xc300c300u;
                    z.w = (z.w & 0x000f000fu) | 0xc300c300u;
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma_bf16(zero_part[nt][G_], z.x, z.x, z.y, z.y, prob[nt][2 * a][G_][0],
                             prob[nt][2 * a][G_][1]);
                    mma_bf16(zero_part[nt][G_], z.z, z.z, z.w, z.w, prob[nt][2 * a + 1][G_][0],
                             prob[nt][2 * a + 1][G_][1]);
                }
            }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const uint4 w = lds128(values + ((m * 8 + g) * 4 + t) * 16);
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const uint32_t lo = a ? w.y : w.x, hi = a ? w.w : w.z;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint32_t r0 = code_pair(lo, 2 * c), r1 = code_pair(hi, 2 * c);
                    const uint32_t r2 = code_pair(lo, 2 * c + 1), r3 = code_pair(hi, 2 * c + 1);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        mma_bf16(o[nt][m], r0, r1, r2, r3, prob[nt][2 * a + c][m / 4][0],
                                 prob[nt][2 * a + c][m / 4][1]);
                }
            }
        }
        __syncwarp();
        copy_half(id, stage, 1);
        absent = (absent & ~(1u << stage)) | (id_ok ? 0u : 1u << stage);
        id = next_id();

        // ---- the next page
        stage = stage + 1 == C::kStages ? 0 : stage + 1;
        ++at.j;
        --todo;
        if (todo > 0 && at.j == at.v.count) {
            finish_unit();
            first_seg = false;
            do {
                ++at.pair;
                at.v = visit_of(p, at.pair / p.parts);
            } while (at.v.count == 0);
            at.j = 0;
            start_unit();
        }
    }

    // ---- the spans' last units: the warps of the block that end in the same one join their parts
    cp_async_wait<0>();
    __syncwarp();
    if (has_span) {
        close_rows();
        put_part(reinterpret_cast<float*>(smem + warp * C::kRing));
    }
    if (lane == 0) {
        s_pair[warp] = has_span ? at.pair : -1;
        s_slot[warp] = 2 * worker + (first_seg ? 0 : 1);
        s_begins[warp] = seg_begin == 0;
        s_ends[warp] = at.j == at.v.count;
    }
    __syncthreads();
    for (int w0 = 0, w1; w0 < C::kWarps && s_pair[w0] >= 0; w0 = w1) {
        const int pair = s_pair[w0], unit = pair / p.parts, r0 = pair % p.parts * kRows;
        for (w1 = w0 + 1; w1 < C::kWarps && s_pair[w1] == pair; ++w1) {}
        const bool begins = s_begins[w0], ends = s_ends[w1 - 1], whole = begins && ends;
        float* part = p.part + static_cast<int64_t>(s_slot[w0]) * kPartSize<D, NT>;
        for (int i = threadIdx.x; i < kRows * D / 4; i += 32 * C::kWarps) {
            const int r = 4 * i / D, x = 4 * i % D;
            float m = -INFINITY, l = 0.0f;
            float4 acc = {};
            for (int w = w0; w < w1; ++w)
                m = fmaxf(m, reinterpret_cast<const float*>(smem + w * C::kRing)[kRows * D + r]);
            for (int w = w0; w < w1 && m > -INFINITY; ++w) {
                const float* from_warp = reinterpret_cast<const float*>(smem + w * C::kRing);
                const float f = exp2_approx((from_warp[kRows * D + r] - m) * p.c);
                const float4 y = *reinterpret_cast<const float4*>(from_warp + 4 * i);
                l = fmaf(from_warp[kRows * D + kRows + r], f, l);
                acc.x = fmaf(y.x, f, acc.x);
                acc.y = fmaf(y.y, f, acc.y);
                acc.z = fmaf(y.z, f, acc.z);
                acc.w = fmaf(y.w, f, acc.w);
            }
            if (!whole) {
                *reinterpret_cast<float4*>(part + 4 * i) = acc;
                if (x == 0) {
                    part[kRows * D + r] = m;
                    part[kRows * D + kRows + r] = l;
                }
            } else if (r0 + r < p.rows) {
                const int64_t row = out_row(p, unit, r0 + r);
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
                *reinterpret_cast<uint2*>(p.a.out + row * D + x) = make_uint2(
                    bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
                if (p.a.out_lse && x == 0) p.a.out_lse[row] = log_sum(p, m, l);
            }
        }
        if (threadIdx.x == 0) {
            if (whole) p.spans[pair] = make_int2(0, -1);
            if (!whole && begins) p.spans[pair].x = s_slot[w0];
            if (!whole && ends) p.spans[pair].y = blockIdx.x * C::kWarps + w1 - 1;
        }
        // merge_kernel looks at the unit's last worker, whose part is in the run's first one's
        if (!whole && ends && w1 - w0 > 1)
            for (int r = threadIdx.x; r < 2 * kRows; r += 32 * C::kWarps)
                p.part[static_cast<int64_t>(s_slot[w1 - 1]) * kPartSize<D, NT> + kRows * D + r] =
                    r < kRows ? -INFINITY : 0.0f;
    }
}

// One block per (unit, part) pair and row: joins the parts of a unit that several blocks took, in
// the order of its slots, and writes the rows of units without slots.  Its parts are those of the
// warp it begins in, of the first warp of every block after that, and of the warp it ends in.  The
// warps take them in turn, their sums are added in order.  The first block of a unit also checks
// its length and page numbers.
constexpr int kMergeWarps = 4;

template <int D, int NT>
__global__ void __launch_bounds__(32 * kMergeWarps)
    merge_kernel(const __grid_constant__ AttendParams p)
{
    constexpr int kRows = 8 * NT, kWarps = Config<D, NT>::kWarps, kVec = D / 32;
    __shared__ float s_acc[kMergeWarps][D];
    __shared__ float s_top[kMergeWarps], s_sum[kMergeWarps];
    wait_for_previous();
    const int pair = blockIdx.x, unit = pair / p.parts, r = blockIdx.y;
    const int row = pair % p.parts * kRows + r, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    if (pair % p.parts == 0 && r == 0 && p.a.out_status) {
        const int len = p.a.lens[unit];
        bool bad = len < 0 || len > static_cast<int64_t>(p.a.from.max_pages) * kPage;
        if (!bad)
            for (int j = threadIdx.x; j * kPage < len; j += 32 * kMergeWarps)
                bad |= static_cast<unsigned>(
                           p.a.from.table[static_cast<int64_t>(unit) * p.a.from.max_pages + j]) >=
                       static_cast<unsigned>(p.a.from.n_pages);
        bad = __syncthreads_or(bad);
        if (threadIdx.x == 0) p.a.out_status[unit] = bad ? TWINKV_ERR_INVALID_ARG : TWINKV_OK;
    }
    if (row >= p.rows) return;
    int n = 0;
    int2 span = make_int2(0, 0);
    if (visit_of(p, unit).count > 0) {
        span = p.spans[pair];
        if (span.y < 0) return;       // written already
        n = span.y / kWarps - span.x / 2 / kWarps + 1;
    }
    const bool own_end = n > 0 && span.y % kWarps != 0 && span.y != span.x / 2;
    const int parts = n + own_end;
    auto part = [&](int i) {
        const int slot = i == 0  ? span.x
                         : i < n ? 2 * kWarps * (span.x / 2 / kWarps + i)
                                 : 2 * span.y;
        return p.part + static_cast<int64_t>(slot) * kPartSize<D, NT>;
    };
    float top = -INFINITY;
    for (int i = threadIdx.x; i < parts; i += 32 * kMergeWarps)
        top = fmaxf(top, part(i)[kRows * D + r]);
#pragma unroll
    for (int m = 1; m < 32; m *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kMergeWarps; ++w) top = fmaxf(top, s_top[w]);
    float sum = 0.0f, acc[kVec] = {};
    if (top > -INFINITY) {
#pragma unroll 4
        for (int i = warp; i < parts; i += kMergeWarps) {
            const float* x = part(i);
            const float m = x[kRows * D + r];
            if (m == -INFINITY) continue;     // an empty part has no outputs
            const float f = exp2_approx((m - top) * p.c);
            sum = fmaf(x[kRows * D + kRows + r], f, sum);
            float y[kVec];
            if constexpr (D == 128) {
                const float4 v = *reinterpret_cast<const float4*>(x + r * D + 4 * lane);
                y[0] = v.x, y[1] = v.y, y[2] = v.z, y[3] = v.w;
            } else {
                const float2 v = *reinterpret_cast<const float2*>(x + r * D + 2 * lane);
                y[0] = v.x, y[1] = v.y;
            }
#pragma unroll
            for (int k = 0; k < kVec; ++k) acc[k] = fmaf(y[k], f, acc[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < kVec; ++k) s_acc[warp][kVec * lane + k] = acc[k];
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    if (threadIdx.x < D / 2) {
        float a = 0.0f, b = 0.0f;
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kMergeWarps; ++w) {
            a += s_acc[w][2 * threadIdx.x];
            b += s_acc[w][2 * threadIdx.x + 1];
            sum += s_sum[w];
        }
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        const int64_t at = out_row(p, unit, row);
        reinterpret_cast<uint32_t*>(p.a.out + at * D)[threadIdx.x] = bf16_pair(a * inv, b * inv);
        if (p.a.out_lse && threadIdx.x == 0) p.a.out_lse[at] = log_sum(p, top, sum);
    }
}

// ---------------------------------------------------------------- windows

// Positions ascend over a unit's slots, so what a window shows is a run of slots.  A warp per unit
// and search, 32 probes at a time: the number of slots below n_sink, and per token the first slot
// inside its window.
template <int D>
__global__ void __launch_bounds__(128) window_kernel(const AttendArgs a, int units, int* seen)
{
    using P = PageLayout<D>;
    wait_for_previous();
    const int w = (blockIdx.x * blockDim.x + threadIdx.x) / 32, lane = threadIdx.x % 32;
    const int unit = w / (1 + a.n), which = w % (1 + a.n) - 1;
    if (unit >= units) return;
    int len = a.lens[unit];
    if (len < 0 || len > static_cast<int64_t>(a.from.max_pages) * kPage) len = 0;
    const int* table = a.from.table + static_cast<int64_t>(unit) * a.from.max_pages;
    auto position = [&](int slot) -> int64_t {
        const int id = table[slot / kPage];
        if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.from.n_pages)) return 0;
        return reinterpret_cast<const int*>(a.from.base + static_cast<int64_t>(id) * P::kBytes +
                                            P::kPos)[slot % kPage];
    };
    int64_t wanted = a.n_sink;       // the first slot whose position is not below this
    int hi = len;
    if (which >= 0) {
        const int own = len - a.n + which;
        if (own < 0) {
            if (lane == 0) seen[static_cast<int64_t>(unit) * (1 + a.n) + 1 + which] = 0;
            return;
        }
        wanted = position(own) - a.window + 1;
        hi = own;                    // its own slot is inside
    }
    int lo = 0;                      // the answer is in [lo, hi]
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32;
        const int slot = lo + (lane + 1) * step - 1;
        const unsigned below = __ballot_sync(0xffffffffu, slot < hi && position(slot) < wanted);
        const int n = __popc(below);
        lo += n * step;
        hi = min(hi, lo + step - 1);
        lo = min(lo, hi);
    }
    if (lane == 0) seen[static_cast<int64_t>(unit) * (1 + a.n) + 1 + which] = lo;
}

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

int part_rows(int rows) { return rows <= 8 ? 8 : 16; }

template <int D, int NT>
cudaError_t launch(AttendParams& p, int sms, cudaStream_t st)
{
    using C = Config<D, NT>;
    const size_t smem = static_cast<size_t>(C::kWarps) * C::kRing + (p.chunks + 1) * 4;
    cudaError_t e = cudaFuncSetAttribute(attend_kernel<D, NT>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    const dim3 grid(std::min(sms, kAttendBlocks));
    if (p.seen) {
        const int warps = p.units * (1 + p.a.n);
        window_kernel<D><<<(warps + 3) / 4, 128, 0, st>>>(p.a, p.units,
                                                          const_cast<int*>(p.seen));
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        e = launch_dependent(attend_kernel<D, NT>, grid, 32 * C::kWarps, smem, st, p);
    } else {
        attend_kernel<D, NT><<<grid, 32 * C::kWarps, smem, st>>>(p);
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) return e;
    return launch_dependent(merge_kernel<D, NT>,
                            dim3(p.units * p.parts, std::min(p.rows, 8 * NT)), 32 * kMergeWarps, 0,
                            st, p);
}

}  // namespace

// spans, then windows, then parts
size_t attend_workspace(int units, int rows, int n, int d)
{
    const int pr = part_rows(rows), parts = (rows + pr - 1) / pr;
    const int warps = kAttendBlocks * (pr == 8 ? Config<128, 1>::kWarps : Config<128, 2>::kWarps);
    static_assert(Config<64, 1>::kWarps == Config<128, 1>::kWarps &&
                  Config<64, 2>::kWarps == Config<128, 2>::kWarps);
    return up256(static_cast<size_t>(units) * parts * sizeof(int2)) +
           up256(static_cast<size_t>(units) * (1 + n) * 4) +
           up256(static_cast<size_t>(2) * warps * (pr * d + 2 * pr) * 4);
}

cudaError_t launch_attend(const AttendArgs& a, int sms, cudaStream_t st)
{
    AttendParams p;
    p.a = a;
    p.units = a.B * a.H;
    p.rows = a.G * a.n;
    const int pr = part_rows(p.rows);
    p.parts = (p.rows + pr - 1) / pr;
    p.chunks = (p.units * p.parts + 31) / 32;
    p.c = a.scale * 1.4426950408889634f;
    uint8_t* ws = static_cast<uint8_t*>(a.ws);
    p.spans = reinterpret_cast<int2*>(ws);
    ws += up256(static_cast<size_t>(p.units) * p.parts * sizeof(int2));
    p.seen = a.window > 0 ? reinterpret_cast<const int*>(ws) : nullptr;
    ws += up256(static_cast<size_t>(p.units) * (1 + a.n) * 4);
    p.part = reinterpret_cast<float*>(ws);
    if (a.d == 128) return pr == 8 ? launch<128, 1>(p, sms, st) : launch<128, 2>(p, sms, st);
    return pr == 8 ? launch<64, 1>(p, sms, st) : launch<64, 2>(p, sms, st);
}

}  // namespace twk
