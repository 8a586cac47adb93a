// twk_attend.cu -- attention of the newest tokens over a cache held in 4 bits
// (layout: twk_cache.cuh).
//
// Per unit (sequence b, KV head h), query token i of n and query head of the group:
//     p_j = softmax over the slots j that i sees of scale * q . k_j,     o = sum_j p_j v_j,
// k_j = s (c - z) per group of 64 dimensions, v_j likewise.  Token i is the one in slot len - n + i;
// it sees the slots up to its own and, with a window, of those only the ones whose position is
// within the window of its own or below n_sink.  A query that sees nothing gives 0.
//
// Bound by memory where it is large: 144 bytes a slot (d = 128) against 512 operations per query row,
// and a unit has G n rows, 4 to 16 as a rule.  So what a slot costs in instructions counts, and the
// design is for few of them:
//   - Codes enter the tensor cores as f16 bit patterns as they are: a code c in the last bits of a
//     half is the number c 2^-24, and 16 c one place up, so that a word of 8 codes gives 4 operand
//     registers in 5 instructions; what meets the second kind is divided by 16.  Nothing is
//     subtracted or scaled per element.
//   - Keys: with Q_G the sum of q over a group, q . k = sum_G s_G (sum q c - z_G Q_G): the second term
//     is the accumulator's start value, the scale one multiplication per group.  Queries are scaled
//     by a power of two per row, which leaves them exact down to 2^-27 of the row's largest.
//   - Values: a probability is multiplied by its slot's scale and rounded to f16, in units that follow
//     the largest scale seen: to 11 bits, or by up to 2^-28 of that scale where the product is below
//     2^-17 of it (bf16 needs no units, but has 8 bits, and its codes, as 128 + c, take 7 instructions
//     a word: error against 64 bits 0.0021, 0.0017 now, which is the output's rounding).  The zeros go
//     into one more product with the same rounded numbers.
//   - mma.sync m16n8k16 with the cache as the 16-row operand (slots for keys, dimensions for values)
//     and up to 8 query rows as the other one: 18 multiplications for 16 slots at d = 128.  With
//     tcgen05 the cache would have to be written to shared memory again as 16-bit numbers, four
//     times its bytes, for a 128-row operand of which 4 to 16 rows are wanted; here codes go from
//     the page to registers to the multiplication.
//   - With 16 rows the operands change sides: the rows are the 16-row operand, and the same registers
//     of codes two 8-column ones.  As many multiplications, but a lane then has 2 rows and 16 slots of
//     each instead of 4 rows and 8: maxima take 4 shuffles instead of 12, probabilities are the next
//     operand as they are (32 transpositions a page less), zeros take half the products, and neighbours
//     are computed in pairs (f32x2): 86.1 us where 90.3 (16 x 8 units of 16384 slots, 16 rows).
//   - A warp works alone: it takes pages in order, keeps the running maxima, sums and outputs of its
//     rows in registers, and has its pages' bytes copied into its own ring in shared memory (cp.async,
//     16 bytes a lane), two pages ahead.  No block barrier between the first page and the last.
//
// The pages of all units in one sequence are divided evenly among all warps of the grid, whatever
// the units' lengths: a warp's span may begin and end inside a unit.  A unit that lies in one span, or
// in a block's, is written by the block; of the others each block writes its part (maxima, sums,
// unnormalised outputs), and merge_kernel joins them in the order of the slots.  Nothing depends on
// which warp comes first: results are the same from call to call.
//
// Measured (us a call in a graph, over caches taken in turn; share of the measured copy rate):
//   32 x 8 units of 4k to 16k slots, 4 rows, d = 128     71.7   79 %
//   32 x 8 units of 8192, 16384, 32768 slots, the same   57.4, 100.4, 188.3   78, 89, 95 %
//   8 units of 131009 slots, 4 rows, d = 128             32.8   68 %
//   16 x 8 units of 16384 slots, 8 rows, d = 128         58.9   76 %; 16 rows 83.6, 53 %
//   32 x 8 units of 16384 slots, 4 rows, d = 64          60.3   74 %
//   32 x 8 units of 8192 slots, 16 rows, d = 64          57.8   39 %
// By the differences of the second line loads run at 6.9 TB/s, and about 15 us go into the launches,
// the lengths, the first pages' latency, the last warps and the merge.  With 16 rows two warps on a
// quarter of the SM bound it, which do not cover each other's latencies: at d = 128 their registers fill
// it, at d = 64 (186 registers) more warps gained 4 % at best (Config).
// Tried, in us of a call on the first where not said (then 75 to 85): one bulk copy per half page and a barrier 92 where
// cp.async took 82; 16 warps with 3 half pages each instead of 12 with 4: 88 against 85; shifts on the
// multiplier pipe 88 against 82; e4m3 codes with q in two parts, which mma.sync runs no faster than
// f16 here: 90 against 82, and twice the time with more rows; one kernel in which the block that
// arrives last joins the parts: 80 against 75, and 14.4 against 12.4 for 8 units of 2048 slots (three
// device-wide fences cost more than the second launch).
#include <algorithm>
#include <atomic>
#include <climits>

#include "twk_cache.cuh"
#include "twk_cache_internal.h"
#include "twk_internal.h"
#include "twk_prompt_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

// R: query rows of a part (4, 8 or 16).  Up to 8 are columns: column 2 t is row t, and column 2 t + 1 row
// t + 4, so that with 4 rows a lane has one of them and no idle second.
template <int D, int R>
struct Config {
    static constexpr bool kLeft = R == 16;       // rows are the left operand's
    static constexpr int E = R == 4 ? 1 : 2;     // rows of a lane
    // as many as their registers let be, equally many on each quarter of the SM (12 instead of 8 for
    // 16 rows at d = 64: 60.9 against 63.6 us for 256 units of 8192 slots, but 28.8 against 28.0 for
    // 128 units with a window of 4096, and 20.6 against 18.5 for 32 units of 8192)
    static constexpr int kWarps = R == 16 ? 8 : D == 128 ? 12 : 16;
    static constexpr int kHalf = PageLayout<D>::kValCodes;        // bytes of a page's keys
    static constexpr int kStages = 221184 / (2 * kHalf * kWarps); // pages of a warp's ring
    static constexpr int kRing = 2 * kHalf * kStages;
    static_assert(PageLayout<D>::kPos == 2 * kHalf, "values take as many bytes as keys");
    static_assert(kHalf % 16 == 0 && kStages >= 2);
};

// x / d and x % d for x and d below 2^16: with m = ceil(2^32 / d), x m / 2^32 is above x / d by less
// than x / 2^32 < 1 / d.  (d = 1 has no such m.)  A unit's change has some 25 of them, and a kernel's code is
// read anew with every launch: 64 x 8 units of 100 slots, 56 rows, 40.7 -> 36.9 us; 8 units of 131009
// slots, 36.8 -> 36.3.
struct Divisor {
    unsigned d, m, one;
    explicit Divisor(unsigned by = 1)
        : d(by), m(by > 1 ? 0xffffffffu / by + 1 : 0), one(by > 1 ? 0 : ~0u)
    {
    }
};
__device__ __forceinline__ int operator/(int x, const Divisor& by)
{
    return __umulhi(x, by.m) + (x & by.one);
}
__device__ __forceinline__ int operator%(int x, const Divisor& by)
{
    return x - x / by * static_cast<int>(by.d);
}

struct AttendParams {
    AttendArgs a;
    int units;
    Divisor parts, G, H;     // parts: of R rows, of a unit
    int rows;                // G n
    int chunks;              // of 32 (unit, part) pairs
    float c;                 // scale * log2(e)
    const int* seen;         // [units][1 + n]: slots below n_sink, window's first slot per token
    float* part;             // [warps of the grid + its blocks][kPartSize]
    int2* split;             // [blocks of the grid]: pair that begins in the block and ends in another
                             // one, or -1; whether one that began in another one ends in it
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
template <int D, int R>
constexpr int kPartSize = R * (D + 2);

// Parts of units that began before a warp's span and end in it are in the warp's slot; the block's first
// is its head.  The block's tail: the part of a unit that begins in it and ends in another block.
template <int D, int R>
__device__ __forceinline__ int head_slot(int block)
{
    return block * Config<D, R>::kWarps;
}
template <int D, int R>
__device__ __forceinline__ int tail_slot(int block)
{
    return kAttendBlocks * Config<D, R>::kWarps + block;
}

// row of out and out_lse
__device__ __forceinline__ int64_t out_row(const AttendParams& p, int unit, int row)
{
    const int b = unit / p.H, h = unit % p.H;
    return (static_cast<int64_t>(b) * p.a.n + row / p.G) * (p.H.d * p.G.d) + h * p.G.d +
           row % p.G;
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

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// x and y as f16, x in the low half
__device__ __forceinline__ uint32_t f16_pair(float x, float y)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
    return r;
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

// (x a + c, y b + d), (x + a, y + b) and (x a, y b) in one instruction each
__device__ __forceinline__ void fma_two(float& x, float& y, float a, float b, float c, float d)
{
    asm("{.reg .b64 v, m, c;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 m, {%2, %3};\n\t"
        "mov.b64 c, {%4, %5};\n\tfma.rn.f32x2 v, v, m, c;\n\tmov.b64 {%0, %1}, v;}"
        : "+f"(x), "+f"(y)
        : "f"(a), "f"(b), "f"(c), "f"(d));
}
__device__ __forceinline__ void add_two(float& x, float& y, float a, float b)
{
    asm("{.reg .b64 v, m;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 m, {%2, %3};\n\t"
        "add.rn.f32x2 v, v, m;\n\tmov.b64 {%0, %1}, v;}"
        : "+f"(x), "+f"(y)
        : "f"(a), "f"(b));
}
__device__ __forceinline__ void mul_two(float& x, float& y, float a, float b)
{
    asm("{.reg .b64 v, m;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 m, {%2, %3};\n\t"
        "mul.rn.f32x2 v, v, m;\n\tmov.b64 {%0, %1}, v;}"
        : "+f"(x), "+f"(y)
        : "f"(a), "f"(b));
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
// 2^e, 0 for e < -126
__device__ __forceinline__ float power_of_two(int e)
{
    return __uint_as_float(static_cast<uint32_t>(max(e + 127, 0)) << 23);
}

// The warp's place in the sequence of all pages: (unit, part) pair and page of its visit.
struct Place {
    int pair, j;
    Visit v;
};

template <int D, int R>
__global__ void __launch_bounds__(32 * Config<D, R>::kWarps, 1)
    attend_kernel(const __grid_constant__ AttendParams p)
{
    using P = PageLayout<D>;
    using C = Config<D, R>;
    constexpr int G = P::kGroups, M = D / 16, E = C::E;
    constexpr int kRows = R, kTiles = 2, kDims = 2;
    constexpr bool kLeft = C::kLeft;
    constexpr int kScores = kLeft ? 16 : 8;          // of a lane, row and page
    constexpr int kWritten = -2;
    constexpr int kOut = kLeft ? 2 * M : M;          // accumulators of outputs
    extern __shared__ __align__(128) uint8_t smem[];   // rows of a copy on whole lines of 128 bytes
    __shared__ int s_pair[C::kWarps], s_rest[C::kWarps], s_head[C::kWarps];
    __shared__ bool s_begins[C::kWarps];
    int* chunk_pages = reinterpret_cast<int*>(smem + C::kWarps * C::kRing);
    wait_for_previous();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, t = lane % 4;
    const int pairs = p.units * static_cast<int>(p.parts.d);

    // Pages before each chunk of 32 pairs: a single chunk is summed by every warp for itself, without a
    // barrier, more by the block (up to eight so by every warp: the same lines read by 1824 warps,
    // 4.6 us where the block takes 1.6).
    unsigned total;
    if (p.chunks == 1) {
        total = __reduce_add_sync(0xffffffffu,
                                  lane < pairs ? visit_of(p, lane / p.parts).count : 0);
    } else {
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
        total = chunk_pages[p.chunks];
    }
    // Blocks, and warps within a block, that have a page each, as even as can be; the spans of a
    // block's warps follow one another.
    const unsigned blocks = min(total, gridDim.x), workers = min(total, gridDim.x * C::kWarps);
    if (blockIdx.x >= blocks) {
        if (threadIdx.x == 0) p.split[blockIdx.x] = make_int2(-1, 0);
        return;
    }
    const unsigned index = workers * blockIdx.x / blocks + warp;
    const bool has_span = index < workers * (blockIdx.x + 1) / blocks;
    const int worker = blockIdx.x * C::kWarps + warp;
    // total i / workers, in 32 bits (64-bit divisions here cost 1.1 us of 36 for 8 units of 131009 slots)
    const unsigned each = total / workers, over = total % workers;
    const int begin = has_span ? each * index + over * index / workers : 0;
    int todo = has_span ? each * (index + 1) + over * (index + 1) / workers - begin : 0;

    // the span's first page
    Place at = {};
    if (has_span) {
        int lo = 0, before = 0;              // last chunk that starts at or before `begin`
        if (p.chunks > 1) {
            for (int hi = p.chunks - 1; lo < hi;) {
                const int mid = (lo + hi + 1) / 2;
                if (chunk_pages[mid] <= begin) lo = mid;
                else hi = mid - 1;
            }
            before = chunk_pages[lo];
        }
        const int pair = 32 * lo + lane;
        const int n = pair < pairs ? visit_of(p, pair / p.parts).count : 0;
        int scan = n;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            const int y = __shfl_up_sync(0xffffffffu, scan, m);
            if (lane >= m) scan += y;
        }
        const int rest = begin - before;
        const unsigned past = __ballot_sync(0xffffffffu, scan > rest);
        const int l = __ffs(past) - 1;
        at.pair = 32 * lo + l;
        at.j = rest - (__shfl_sync(0xffffffffu, scan, l) - __shfl_sync(0xffffffffu, n, l));
        at.v = visit_of(p, at.pair / p.parts);
    }

    // ---- copies: the page `ahead` is one past those in the ring; its number is already loaded
    Place ahead = at;
    int ahead_todo = todo;
    const int* ahead_row = p.a.from.table +
                           static_cast<int64_t>(at.pair / p.parts) * p.a.from.max_pages;
    auto next_id = [&]() -> int {
        if (ahead_todo == 0) return -1;
        --ahead_todo;
        if (ahead.j >= ahead.v.count) {
            do {
                ++ahead.pair;
                ahead.v = visit_of(p, ahead.pair / p.parts);
            } while (ahead.v.count == 0);
            ahead.j = 0;
            ahead_row = p.a.from.table +
                        static_cast<int64_t>(ahead.pair / p.parts) * p.a.from.max_pages;
        }
        const int page = ahead.j + (ahead.j < ahead.v.sink_pages ? 0 : ahead.v.skip);
        ++ahead.j;
        return ahead_row[page];
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

    // ---- state of the unit's rows; a lane has the rows row_of(e), of them the slots slot_of(i) of a
    // page, and of accumulators the elements element(e, k)
    auto row_of = [&](int e) { return kLeft ? g + 8 * e : t + 4 * e; };
    auto slot_of = [&](int i) { return kLeft ? 8 * (i / 2) + 2 * t + i % 2 : 8 * i + g; };
    auto element = [](int e, int k) { return kLeft ? 2 * e + k : 2 * k + e; };
    uint32_t q[kLeft ? 2 : 1][G][8];
    float qsum[G][E], unit_of[E];     // sums of q, and what a score's unit is, see below
    float o[kOut][4], zero_part[G][4], top[E], sum[E];
    float value_up[G];                // probabilities' scale, see below
    int value_e[G];
    uint32_t value_limit;
    int limit[E], from[E];            // row sees slots < limit that are >= from or < sinks
    int sinks = 0, all_limit = 0, all_from = 0;
    int seg_begin = 0;
    if (lane == 0) s_head[warp] = -1;    // the pair that began before the span and ends inside it

    auto start_unit = [&]() {
        const int unit = at.pair / p.parts, r0 = at.pair % p.parts * kRows;
        const int b = unit / p.H, h = unit % p.H;
        seg_begin = at.j;
        const int* seen =
            p.seen ? p.seen + static_cast<int64_t>(unit) * (1 + p.a.n) : nullptr;
        sinks = seen ? seen[0] : 0;
        // Queries as f16: a row is scaled by a power of two, 2^k, so that its largest value is in
        // [2^14, 2^15); values down to 2^-27 of it stay exact.  Its scores are sums of 2^(k - 24) q c.
#pragma unroll
        for (int half = 0; half < (kLeft ? 2 : 1); ++half) {
            const int in_part = kLeft ? g + 8 * half : g / 2 + g % 2 * 4, r = r0 + in_part;
            const uint16_t* src = nullptr;
            if (r < p.rows && in_part < R)
                src = p.a.q + b * p.a.q_batch + r / p.G * p.a.q_token +
                      (h * static_cast<int>(p.G.d) + r % p.G) * p.a.q_head;
            uint32_t w[G][8];
            uint32_t most = 0;
#pragma unroll
            for (int G_ = 0; G_ < G; ++G_) {
                uint4 v0 = {}, v1 = {};
                if (src) {
                    v0 = *reinterpret_cast<const uint4*>(src + 64 * G_ + 16 * t);
                    v1 = *reinterpret_cast<const uint4*>(src + 64 * G_ + 16 * t + 8);
                }
                w[G_][0] = v0.x, w[G_][1] = v0.y, w[G_][2] = v0.z, w[G_][3] = v0.w;
                w[G_][4] = v1.x, w[G_][5] = v1.y, w[G_][6] = v1.z, w[G_][7] = v1.w;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    most = max(most, max(w[G_][i] & 0x7fffu, w[G_][i] >> 16 & 0x7fffu));
            }
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            // rows of exponents outside [-100, 100] are scaled as those
            const int exponent = min(max(static_cast<int>(most >> 7) - 127, -100), 100);
            const float up = __uint_as_float(static_cast<uint32_t>(127 + 14 - exponent) << 23);
            const float down = __uint_as_float(static_cast<uint32_t>(127 + 10 + exponent) << 23);
#pragma unroll
            for (int G_ = 0; G_ < G; ++G_) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    // the odd pairs of a word's codes enter times 16
                    const float x = bf16_lo(w[G_][i]) * up, y = bf16_hi(w[G_][i]) * up;
                    const float f = i % 2 ? 0.0625f : 1.0f;
                    q[half][G_][i] = f16_pair(x * f, y * f);
                    s += x + y;
                }
                s += __shfl_xor_sync(0xffffffffu, s, 1);
                s += __shfl_xor_sync(0xffffffffu, s, 2);
                if constexpr (kLeft) {
                    qsum[G_][half] = s * 0x1p-24f;
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        qsum[G_][e] = __shfl_sync(0xffffffffu, s, 8 * t + 4 * e) * 0x1p-24f;
                }
            }
            if constexpr (kLeft) {
                unit_of[half] = down;
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    unit_of[e] = __shfl_sync(0xffffffffu, down, 8 * t + 4 * e);
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int row = r0 + row_of(e), token = row / p.G;
            limit[e] = row < p.rows ? at.v.len - p.a.n + token + 1 : INT_MAX;
            from[e] = row < p.rows && seen ? seen[1 + token] : 0;
            top[e] = -INFINITY;
            sum[e] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int m = 0; m < kOut; ++m) o[m][i] = 0.0f;
#pragma unroll
            for (int G_ = 0; G_ < G; ++G_) zero_part[G_][i] = 0.0f;
        }
        value_limit = 0;
#pragma unroll
        for (int G_ = 0; G_ < G; ++G_) {
            value_up[G_] = 0.0f;
            value_e[G_] = 0;
        }
        // every row of the part: the first token sees least at the end, the last at the window's
        // begin
        const int first_token = r0 / p.G, last_token = (min(r0 + kRows, p.rows) - 1) / p.G;
        all_limit = at.v.len - p.a.n + first_token + 1;
        all_from = seen ? seen[1 + last_token] : 0;
    };

    // the sums of the lanes that share a row; the zeros' part joins the output
    auto close_rows = [&]() {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float s = sum[e];
#pragma unroll
            for (int i = kLeft ? 1 : 4; i < (kLeft ? 4 : 32); i *= 2)
                s += __shfl_xor_sync(0xffffffffu, s, i);
            sum[e] = s;
            top[e] *= unit_of[e];
        }
#pragma unroll
        for (int m = 0; m < kOut; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int G_ = m / (kOut / G);
                o[m][i] = (o[m][i] - zero_part[G_][kLeft ? i : i % 2]) * 0x1p17f *
                          power_of_two(value_e[G_]);
            }
    };
    // rows as outputs [kRows][D], then maxima and sums [kRows]
    auto put_part = [&](float* part) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int r = row_of(e);
#pragma unroll
            for (int m = 0; m < kOut; ++m) {
                if constexpr (kLeft) {
                    *reinterpret_cast<float2*>(part + r * D + 8 * m + 2 * t) =
                        make_float2(o[m][2 * e], o[m][2 * e + 1]);
                } else {
                    part[r * D + 16 * m + g] = o[m][e];
                    part[r * D + 16 * m + 8 + g] = o[m][2 + e];
                }
            }
            if ((kLeft ? t : g) == 0) {
                part[kRows * D + r] = top[e];
                part[kRows * D + kRows + r] = sum[e];
            }
        }
    };
    // a unit that ends inside the span: written at once if it began there
    auto finish_unit = [&]() {
        close_rows();
        if (seg_begin > 0) {
            put_part(p.part + static_cast<int64_t>(worker) * kPartSize<D, R>);
            if (lane == 0) s_head[warp] = at.pair;
            return;
        }
        const int r0 = at.pair % p.parts * kRows, unit = at.pair / p.parts;
        float inv[2] = {};
#pragma unroll
        for (int e = 0; e < E; ++e) inv[e] = sum[e] > 0.0f ? 1.0f / sum[e] : 0.0f;
        if constexpr (kLeft) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int row = r0 + row_of(e);
                if (row >= p.rows) continue;
                uint16_t* out = p.a.out + out_row(p, unit, row) * D;
#pragma unroll
                for (int m = 0; m < kOut; ++m)
                    *reinterpret_cast<uint32_t*>(out + 8 * m + 2 * t) =
                        bf16_pair(o[m][2 * e] * inv[e], o[m][2 * e + 1] * inv[e]);
            }
        } else {
            const int row = r0 + g / 2 + g % 2 * 4;     // of column g
            uint16_t* out = p.a.out + out_row(p, unit, row) * D;
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const uint32_t w =
                        transpose16(bf16_pair(o[m][e] * inv[0], o[m][e + 1] * inv[1]));
                    if (row < p.rows)
                        *reinterpret_cast<uint32_t*>(out + 16 * m + 4 * e + 2 * t) = w;
                }
        }
        if (p.a.out_lse && (kLeft ? t : g) == 0) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int r = r0 + row_of(e);
                if (r < p.rows) p.a.out_lse[out_row(p, unit, r)] = log_sum(p, top[e], sum[e]);
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
        float s[E][kScores];
#pragma unroll
        for (int t0 = 0; t0 < 4; t0 += kTiles) {   // tiles side by side: the multiplications' latency
            uint32_t a0[kTiles][2 * G], a1[kTiles][2 * G];    // words of slots lo and lo + 8
            constexpr int kMine = kTiles * kScores / 4;
            uint32_t k[kMine][G];              // scales and zeros of the lane's slots
#pragma unroll
            for (int i = 0; i < kTiles; ++i) {
                const int lo = 16 * (t0 + i) + g;
                if constexpr (D == 128) {
                    const uint4 u = lds128(keys + lo * P::kRow + 16 * t);
                    const uint4 w = lds128(keys + (lo + 8) * P::kRow + 16 * t);
                    a0[i][0] = u.x, a0[i][1] = u.y, a0[i][2] = u.z, a0[i][3] = u.w;
                    a1[i][0] = w.x, a1[i][1] = w.y, a1[i][2] = w.z, a1[i][3] = w.w;
                } else {
                    const uint2 u = lds64(keys + lo * P::kRow + 8 * t);
                    const uint2 w = lds64(keys + (lo + 8) * P::kRow + 8 * t);
                    a0[i][0] = u.x, a0[i][1] = u.y;
                    a1[i][0] = w.x, a1[i][1] = w.y;
                }
#pragma unroll
                for (int l = i * kMine / kTiles; l < (i + 1) * kMine / kTiles; l += kLeft ? 2 : 1) {
                    const int slot = slot_of(t0 * (kScores / 4) + l);
                    const uint32_t at_k = keys + P::kKeyGroups + slot * 4 * G;
                    if constexpr (kLeft && D == 128) {
                        const uint4 u = lds128(at_k);
                        k[l][0] = u.x, k[l][1] = u.y, k[l + 1][0] = u.z, k[l + 1][1] = u.w;
                    } else if constexpr (kLeft) {
                        const uint2 u = lds64(at_k);
                        k[l][0] = u.x, k[l + 1][0] = u.y;
                    } else {
                        load_groups<D>(at_k, k[l]);
                    }
                }
            }
#pragma unroll
            for (int G_ = 0; G_ < G; ++G_) {
                // slots lo and lo + 8 of a tile are two accumulators' columns, or one's rows
                constexpr int kAcc = kLeft ? 2 : 1;
                float acc[kTiles][kAcc][4] = {};       // -z Q at first
                // accumulator's element of the lane's slot i of a tile
                auto of = [&](int tile, int i, int e) -> float& {
                    return kLeft ? acc[tile][i / 2][2 * e + i % 2] : acc[tile][0][2 * i + e];
                };
#pragma unroll
                for (int i = 0; i < kMine; i += kLeft ? 2 : 1)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        const float Q = qsum[G_][e];
                        float& x = of(i / (kScores / 4), i % (kScores / 4), e);
                        if constexpr (kLeft) {
                            float y0 = bf16_hi(k[i][G_]), y1 = bf16_hi(k[i + 1][G_]);
                            fma_two(y0, y1, Q, Q, 128.0f * Q, 128.0f * Q);
                            x = y0;
                            of(i / (kScores / 4), i % (kScores / 4) + 1, e) = y1;
                        } else {
                            x = fmaf(bf16_hi(k[i][G_]), Q, 128.0f * Q);
                        }
                    }
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int i = 0; i < kTiles; ++i) {
                            const uint32_t u = a0[i][2 * G_ + w] >> (8 * x);
                            const uint32_t v = a1[i][2 * G_ + w] >> (8 * x);
                            const int y = 4 * w + 2 * x;
                            if constexpr (kLeft) {
                                mma_f16(acc[i][0], q[0][G_][y], q[1][G_][y], q[0][G_][y + 1],
                                        q[1][G_][y + 1], u & 0x000f000fu, u & 0x00f000f0u);
                                mma_f16(acc[i][1], q[0][G_][y], q[1][G_][y], q[0][G_][y + 1],
                                        q[1][G_][y + 1], v & 0x000f000fu, v & 0x00f000f0u);
                            } else {
                                mma_f16(acc[i][0], u & 0x000f000fu, v & 0x000f000fu,
                                        u & 0x00f000f0u, v & 0x00f000f0u, q[0][G_][y],
                                        q[0][G_][y + 1]);
                            }
                        }
#pragma unroll
                for (int i = 0; i < kMine; i += kLeft ? 2 : 1)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        float& y = s[e][t0 * (kScores / 4) + i];
                        if constexpr (kLeft) {
                            float x0 = of(i / (kScores / 4), i % (kScores / 4), e);
                            float x1 = of(i / (kScores / 4), i % (kScores / 4) + 1, e);
                            float& z = s[e][t0 * (kScores / 4) + i + 1];
                            if (G_ == 0) mul_two(x0, x1, bf16_lo(k[i][G_]), bf16_lo(k[i + 1][G_]));
                            else fma_two(x0, x1, bf16_lo(k[i][G_]), bf16_lo(k[i + 1][G_]), y, z);
                            y = x0, z = x1;
                        } else {
                            const float x = of(i / (kScores / 4), i % (kScores / 4), e);
                            y = G_ == 0 ? x * bf16_lo(k[i][G_]) : fmaf(x, bf16_lo(k[i][G_]), y);
                        }
                    }
            }
        }
        __syncwarp();
        copy_half(id, stage, 0);
        if (!full) {
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int i = 0; i < kScores; ++i) {
                    const int slot = base + slot_of(i);
                    const bool see = !gone && slot < min(limit[e], at.v.len) &&
                                     (slot >= from[e] || slot < sinks);
                    if (!see) s[e][i] = -INFINITY;
                }
        }

        // ---- running maxima; probabilities
        bool grown = false;
        float shrink[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float(&y)[kScores] = s[e];
            // not 0, which times an unseen slot's -inf is no number
            const float last = top[e], c = fmaxf(p.c * unit_of[e], 0x1p-126f);
            float m = last;
#pragma unroll
            for (int i = 0; i < kScores; i += 2) m = fmaxf(m, fmaxf(y[i], y[i + 1]));
#pragma unroll
            for (int i = kLeft ? 1 : 4; i < (kLeft ? 4 : 32); i *= 2)
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, i));
            grown |= m > last;
            // a row that has seen nothing yet keeps -inf, and its probabilities are 0
            const float high = m == -INFINITY ? 0.0f : m;
            const float f = last == -INFINITY ? 0.0f : exp2_approx((last - m) * c);
            shrink[e] = f;
            top[e] = m;
            float l = 0.0f, l2 = 0.0f;
#pragma unroll
            for (int i = 0; i < kScores; i += 2) {
                // the difference first: one of products is off by 2^-24 of the scores' size
                if constexpr (kLeft) {
                    add_two(y[i], y[i + 1], -high, -high);
                    mul_two(y[i], y[i + 1], c, c);
                } else {
                    y[i] = (y[i] - high) * c;
                    y[i + 1] = (y[i + 1] - high) * c;
                }
                y[i] = exp2_approx(y[i]);
                y[i + 1] = exp2_approx(y[i + 1]);
                if constexpr (kLeft) add_two(l, l2, y[i], y[i + 1]);
                else l += y[i], l += y[i + 1];
            }
            sum[e] = fmaf(sum[e], f, l + l2);
        }
        if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
#pragma unroll
                for (int m = 0; m < kOut; ++m) {
                    if constexpr (kLeft) {
                        mul_two(o[m][2 * e], o[m][2 * e + 1], shrink[e], shrink[e]);
                    } else {
                        o[m][e] *= shrink[e];
                        o[m][2 + e] *= shrink[e];
                    }
                }
#pragma unroll
                for (int G_ = 0; G_ < G; ++G_)
#pragma unroll
                    for (int k = 0; k < 2; ++k) zero_part[G_][element(e, k)] *= shrink[e];
            }
        }

        // ---- values
        cp_async_wait<2 * C::kStages - 1>();
        __syncwarp();
        // The slots' scales, bf16 (those of two groups in one word); slots never written count as 0.
        uint32_t scales[kScores];
        uint32_t most = 0;
#pragma unroll
        for (int tile = 0; tile < 4; ++tile)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int at_tile = (2 * tile + i) * (kScores / 8), slot = slot_of(at_tile);
                const uint32_t at_scale = values + P::kValScales - P::kValCodes + slot * 2 * G;
                uint32_t w, w2 = 0;
                if constexpr (kLeft && D == 128) {
                    const uint2 u = lds64(at_scale);
                    w = u.x, w2 = u.y;
                } else if constexpr (kLeft) {
                    w = lds32(at_scale);
                    w2 = w >> 16, w &= 0xffffu;
                } else if constexpr (D == 128) {
                    w = lds32(at_scale);
                } else {
                    w = lds16(at_scale);
                }
                if (!full && (gone || base + slot >= at.v.len)) w = 0;
                scales[at_tile] = w;
                most = __vmaxu2(most, w);
                if constexpr (kLeft) {
                    if (!full && (gone || base + slot + 1 >= at.v.len)) w2 = 0;
                    scales[at_tile + 1] = w2;
                    most = __vmaxu2(most, w2);
                }
            }
        // Probabilities times scales enter as f16, in units of 2^(e - 7), 2^e the power of two below
        // the largest scale seen.  There is room for scales up to 2^(e + 8); a larger one makes
        // the unit its own.
        if (__any_sync(0xffffffffu, __vmaxu2(most, value_limit) != value_limit)) {
            uint32_t limits = 0;
#pragma unroll
            for (int G_ = 0; G_ < G; ++G_) {
                const uint32_t b = __reduce_max_sync(0xffffffffu, most >> (16 * G_) & 0xffffu);
                const uint32_t old = value_limit >> (16 * G_) & 0xffffu;
                uint32_t now = old;
                if (b > old) {
                    const int e = max(static_cast<int>(b >> 7) - 127, -110);
                    const float f = old == 0 ? 1.0f : power_of_two(value_e[G_] - e);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
#pragma unroll
                        for (int m = 0; m < kOut / G; ++m) o[kOut / G * G_ + m][i] *= f;
                        zero_part[G_][i] *= f;
                    }
                    value_e[G_] = e;
                    value_up[G_] = power_of_two(7 - e);
                    now = static_cast<uint32_t>(min(e + 127 + 8, 255)) << 7;
                }
                limits |= now << (16 * G_);
            }
            value_limit = limits;
        }
        uint32_t prob[4][G][kLeft ? 4 : 2];      // f16, slots in the order of the value codes
#pragma unroll
        for (int tile = 0; tile < 4; ++tile)
#pragma unroll
            for (int half = 0; half < 2; ++half)       // of the tile's slots
#pragma unroll
                for (int G_ = 0; G_ < G; ++G_) {
                    // the odd pairs of a word's codes enter times 16
                    const float up = half ? value_up[G_] * 0.0625f : value_up[G_];
                    const int i = (2 * tile + half) * (kScores / 8);
                    auto scale = [&](int j) {
                        return (G_ ? bf16_hi(scales[j]) : bf16_lo(scales[j])) * up;
                    };
                    if constexpr (kLeft) {
                        float f0 = G_ ? bf16_hi(scales[i]) : bf16_lo(scales[i]);
                        float f1 = G_ ? bf16_hi(scales[i + 1]) : bf16_lo(scales[i + 1]);
                        mul_two(f0, f1, up, up);
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            float x0 = s[e][i], x1 = s[e][i + 1];
                            mul_two(x0, x1, f0, f1);
                            prob[tile][G_][2 * half + e] = f16_pair(x0, x1);
                        }
                    } else {
                        const float f = scale(i);
                        float x[2] = {};        // rows t and t + 4
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] = s[e][i] * f;
                        prob[tile][G_][half] = transpose16(f16_pair(x[0], x[1]));
                    }
                }
#pragma unroll
        for (int G_ = 0; G_ < G; ++G_)
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                // the last bits of -(128 + z) are z
                const uint4 z = lds128(values + P::kValZeros - P::kValCodes + G_ * 2 * kPage +
                                       32 * t + 16 * a);
                const uint32_t zeros[2][2] = {{z.x & 0x000f000fu, z.y << 4 & 0x00f000f0u},
                                              {z.z & 0x000f000fu, z.w << 4 & 0x00f000f0u}};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint32_t(&pr)[kLeft ? 4 : 2] = prob[2 * a + c][G_];
                    if constexpr (kLeft)
                        mma_f16(zero_part[G_], pr[0], pr[1], pr[2], pr[3], zeros[c][0], zeros[c][1]);
                    else
                        mma_f16(zero_part[G_], zeros[c][0], zeros[c][0], zeros[c][1], zeros[c][1],
                                pr[0], pr[1]);
                }
            }
#pragma unroll
        for (int m0 = 0; m0 < M; m0 += kDims) {
            uint4 w[kDims];
#pragma unroll
            for (int i = 0; i < kDims; ++i)
                w[i] = lds128(values + (((m0 + i) * 8 + g) * 4 + t) * 16);
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < kDims; ++i) {
                        const int m = m0 + i;
                        const uint32_t u = (a ? w[i].y : w[i].x) >> (8 * c);
                        const uint32_t v = (a ? w[i].w : w[i].z) >> (8 * c);
                        const uint32_t(&pr)[kLeft ? 4 : 2] = prob[2 * a + c][m / 4];
                        if constexpr (kLeft) {
                            mma_f16(o[2 * m], pr[0], pr[1], pr[2], pr[3], u & 0x000f000fu,
                                    u & 0x00f000f0u);
                            mma_f16(o[2 * m + 1], pr[0], pr[1], pr[2], pr[3], v & 0x000f000fu,
                                    v & 0x00f000f0u);
                        } else {
                            mma_f16(o[m], u & 0x000f000fu, v & 0x000f000fu, u & 0x00f000f0u,
                                    v & 0x00f000f0u, pr[0], pr[1]);
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
        if (at.j == at.v.count && (todo > 0 || seg_begin == 0)) {
            finish_unit();
            if (todo == 0) break;
            do {
                ++at.pair;
                at.v = visit_of(p, at.pair / p.parts);
            } while (at.v.count == 0);
            at.j = 0;
            start_unit();
        }
    }

    // ---- the spans' last units, if not written: the warps of the block that end in the same one join
    // their parts
    cp_async_wait<0>();
    __syncwarp();
    const bool written = at.j == at.v.count && seg_begin == 0;
    if (has_span && !written) {
        close_rows();
        put_part(reinterpret_cast<float*>(smem + warp * C::kRing));
    }
    if (lane == 0) {
        s_pair[warp] = !has_span ? -1 : written ? kWritten : at.pair;
        s_rest[warp] = at.v.count - at.j;
        s_begins[warp] = seg_begin == 0;
    }
    __syncthreads();
    // a warp per run of such warps and row; the next warp may have the rest of the unit as its head
    for (int w0 = 0, w1, turn = warp; w0 < C::kWarps && s_pair[w0] != -1; w0 = w1) {
        const int pair = s_pair[w0], unit = pair / p.parts, r0 = pair % p.parts * kRows;
        for (w1 = w0 + 1; w1 < C::kWarps && s_pair[w1] == pair; ++w1) {}
        const bool with_head = w1 < C::kWarps && s_head[w1] == pair;
        const bool begins = s_begins[w0], ends = with_head || s_rest[w1 - 1] == 0;
        const float* rest = p.part + static_cast<int64_t>(worker - warp + w1) * kPartSize<D, R>;
        for (int r = turn % C::kWarps; r < kRows && pair != kWritten; r += C::kWarps) {
            constexpr int kVec = D / 32;
            float m = -INFINITY, l = 0.0f, acc[kVec] = {};
            float m_rest = -INFINITY, l_rest = 0.0f, rest_acc[kVec] = {};
            if (with_head) {
                m = m_rest = rest[kRows * D + r];
                l_rest = rest[kRows * D + kRows + r];
#pragma unroll
                for (int v = 0; v < kVec; v += 2) {
                    const float2 y =
                        *reinterpret_cast<const float2*>(rest + r * D + 32 * v + 2 * lane);
                    rest_acc[v] = y.x;
                    rest_acc[v + 1] = y.y;
                }
            }
            for (int w = w0; w < w1; ++w)
                m = fmaxf(m, reinterpret_cast<const float*>(smem + w * C::kRing)[kRows * D + r]);
            for (int w = w0; w < w1 && m > -INFINITY; ++w) {
                const float* from_warp = reinterpret_cast<const float*>(smem + w * C::kRing);
                const float f = exp2_approx((from_warp[kRows * D + r] - m) * p.c);
                l = fmaf(from_warp[kRows * D + kRows + r], f, l);
#pragma unroll
                for (int v = 0; v < kVec; v += 2) {
                    const float2 y = *reinterpret_cast<const float2*>(from_warp + r * D + 32 * v +
                                                                      2 * lane);
                    acc[v] = fmaf(y.x, f, acc[v]);
                    acc[v + 1] = fmaf(y.y, f, acc[v + 1]);
                }
            }
            if (with_head && m > -INFINITY) {
                const float f = exp2_approx((m_rest - m) * p.c);
                l = fmaf(l_rest, f, l);
#pragma unroll
                for (int v = 0; v < kVec; ++v) acc[v] = fmaf(rest_acc[v], f, acc[v]);
            }
            if (!begins || !ends) {
                float* part = p.part + static_cast<int64_t>(begins ? tail_slot<D, R>(blockIdx.x)
                                                                   : head_slot<D, R>(blockIdx.x)) *
                                           kPartSize<D, R>;
#pragma unroll
                for (int v = 0; v < kVec; v += 2)
                    *reinterpret_cast<float2*>(part + r * D + 32 * v + 2 * lane) =
                        make_float2(acc[v], acc[v + 1]);
                if (lane == 0) {
                    part[kRows * D + r] = m;
                    part[kRows * D + kRows + r] = l;
                }
            } else if (r0 + r < p.rows) {
                const int64_t row = out_row(p, unit, r0 + r);
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
                for (int v = 0; v < kVec; v += 2)
                    *reinterpret_cast<uint32_t*>(p.a.out + row * D + 32 * v + 2 * lane) =
                        bf16_pair(acc[v] * inv, acc[v + 1] * inv);
                if (p.a.out_lse && lane == 0) p.a.out_lse[row] = log_sum(p, m, l);
            }
        }
        turn += pair != kWritten ? kRows : 0;
        if (threadIdx.x == 0) {
            if (w0 == 0) p.split[blockIdx.x].y = begins ? s_head[0] >= 0 : ends;
            if (w1 == C::kWarps || s_pair[w1] < 0)
                p.split[blockIdx.x].x = begins && !ends ? pair : -1;
        }
    }
}

// Joins the parts of a unit that several blocks took, in the order of its slots: a block per block that
// such a unit begins in and row.  Its parts are that block's tail and the heads of the blocks after it, up
// to the one it ends in.  Bound by latency: every warp reads five parts at once, maxima, sums and
// outputs, and joins them as it would pages; the warps' results are joined in order.  (With four, the 19
// or 20 parts of each of 8 units took a second round: 27.9 us where 26.9, 65536 slots.  Blocks for
// every pair and row, most of which find nothing to do: 37 us for 2048 pairs of 16 rows.)  The
// blocks past the rows are the units': each checks the length and page numbers of one, and writes
// the rows of one without slots.
constexpr int kMergeWarps = 4, kMergeParts = 5;

template <int D, int R>
__global__ void __launch_bounds__(32 * kMergeWarps)
    merge_kernel(const __grid_constant__ AttendParams p, int rows)
{
    constexpr int kRows = R, kVec = D / 32;
    __shared__ float s_acc[kMergeWarps][D];
    __shared__ float s_top[kMergeWarps], s_sum[kMergeWarps];
    wait_for_previous();
    if (static_cast<int>(blockIdx.y) >= rows) {
        const int unit = (blockIdx.y - rows) * gridDim.x + blockIdx.x;
        if (unit >= p.units) return;
        const int len = p.a.lens[unit];
        bool bad = len < 0 || len > static_cast<int64_t>(p.a.from.max_pages) * kPage;
        if (bad || len == 0)
            for (int i = threadIdx.x; i < p.rows * (D / 2); i += 32 * kMergeWarps) {
                const int64_t at = out_row(p, unit, i / (D / 2));
                reinterpret_cast<uint32_t*>(p.a.out + at * D)[i % (D / 2)] = 0;
                if (p.a.out_lse && i % (D / 2) == 0) p.a.out_lse[at] = -INFINITY;
            }
        if (!p.a.out_status) return;
        if (!bad)
            for (int j = threadIdx.x; j * kPage < len; j += 32 * kMergeWarps)
                bad |= static_cast<unsigned>(
                           p.a.from.table[static_cast<int64_t>(unit) * p.a.from.max_pages + j]) >=
                       static_cast<unsigned>(p.a.from.n_pages);
        bad = __syncthreads_or(bad);
        if (threadIdx.x == 0) p.a.out_status[unit] = bad ? TWINKV_ERR_INVALID_ARG : TWINKV_OK;
        return;
    }
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int parts = 1;                     // up to the first block after this one that a unit ends in
    bool open = true;
#pragma unroll
    for (int i = 0; i < (kAttendBlocks + 31) / 32; ++i) {
        const int b = 32 * i + lane;
        const bool ends = b > blockIdx.x && b < gridDim.x && p.split[b].y;
        const unsigned at = __ballot_sync(0xffffffffu, ends);
        if (open && at) parts = 32 * i + __ffs(at) - blockIdx.x;
        open &= at == 0;
    }
    const int pair = p.split[blockIdx.x].x;
    const int unit = pair / p.parts, r = blockIdx.y, row = pair % p.parts * kRows + r;
    if (pair < 0 || row >= p.rows) return;
    float top = -INFINITY, sum = 0.0f, acc[kVec] = {};
    for (int i0 = warp; i0 < parts; i0 += kMergeWarps * kMergeParts) {
        float m[kMergeParts], l[kMergeParts], y[kMergeParts][kVec];
#pragma unroll
        for (int k = 0; k < kMergeParts; ++k) {
            const int i = i0 + k * kMergeWarps;
            m[k] = -INFINITY;
            if (i >= parts) continue;
            const int slot = i == 0 ? tail_slot<D, R>(blockIdx.x) : head_slot<D, R>(blockIdx.x + i);
            const float* x = p.part + static_cast<int64_t>(slot) * kPartSize<D, R>;
            m[k] = x[kRows * D + r];
            l[k] = x[kRows * D + kRows + r];
            if constexpr (D == 128) {
                const float4 v = *reinterpret_cast<const float4*>(x + r * D + 4 * lane);
                y[k][0] = v.x, y[k][1] = v.y, y[k][2] = v.z, y[k][3] = v.w;
            } else {
                const float2 v = *reinterpret_cast<const float2*>(x + r * D + 2 * lane);
                y[k][0] = v.x, y[k][1] = v.y;
            }
        }
        float most = top;
#pragma unroll
        for (int k = 0; k < kMergeParts; ++k) most = fmaxf(most, m[k]);
        if (top > -INFINITY) {
            const float f = exp2_approx((top - most) * p.c);
            sum *= f;
#pragma unroll
            for (int v = 0; v < kVec; ++v) acc[v] *= f;
        }
        top = most;
#pragma unroll
        for (int k = 0; k < kMergeParts; ++k) {
            if (m[k] == -INFINITY) continue;       // an empty part has no outputs
            const float f = exp2_approx((m[k] - top) * p.c);
            sum = fmaf(l[k], f, sum);
#pragma unroll
            for (int v = 0; v < kVec; ++v) acc[v] = fmaf(y[k][v], f, acc[v]);
        }
    }
#pragma unroll
    for (int v = 0; v < kVec; ++v) s_acc[warp][kVec * lane + v] = acc[v];
    if (lane == 0) {
        s_top[warp] = top;
        s_sum[warp] = sum;
    }
    __syncthreads();
    if (threadIdx.x < D / 2) {
        top = s_top[0];
#pragma unroll
        for (int w = 1; w < kMergeWarps; ++w) top = fmaxf(top, s_top[w]);
        float a = 0.0f, b = 0.0f;
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kMergeWarps; ++w) {
            if (s_top[w] == -INFINITY) continue;
            const float f = exp2_approx((s_top[w] - top) * p.c);
            sum = fmaf(s_sum[w], f, sum);
            a = fmaf(s_acc[w][2 * threadIdx.x], f, a);
            b = fmaf(s_acc[w][2 * threadIdx.x + 1], f, b);
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
    // Slots of a page outside the pool are unseen and have no position: with that of the last slot before
    // them that has one, positions ascend all the same.
    auto position = [&](int slot) -> int64_t {
        int page = slot / kPage, at = slot % kPage, id = table[page];
        while (static_cast<unsigned>(id) >= static_cast<unsigned>(a.from.n_pages)) {
            if (page == 0) return -1;
            id = table[--page];
            at = kPage - 1;
        }
        return reinterpret_cast<const int*>(a.from.base + static_cast<int64_t>(id) * P::kBytes +
                                            P::kPos)[at];
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

}  // namespace

cudaError_t launch_windows(const AttendArgs& a, int units, int* seen, cudaStream_t st)
{
    const int warps = units * (1 + a.n);
    if (a.d == 128) window_kernel<128><<<(warps + 3) / 4, 128, 0, st>>>(a, units, seen);
    else window_kernel<64><<<(warps + 3) / 4, 128, 0, st>>>(a, units, seen);
    return cudaGetLastError();
}

namespace {

size_t up256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

int part_rows(int rows) { return rows <= 8 ? 8 : 16; }

template <int D, int R>
cudaError_t launch(AttendParams& p, int sms, cudaStream_t st)
{
    using C = Config<D, R>;
    constexpr int kRings = C::kWarps * C::kRing, kMostChunks = 2048;
    static std::atomic<bool> allowed[64];     // by device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(attend_kernel<D, R>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kRings + (kMostChunks + 1) * 4);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
    }
    const size_t smem = kRings + (p.chunks + 1) * 4;
    const dim3 grid(std::min(sms, kAttendBlocks));
    if (p.seen) {
        if ((e = launch_windows(p.a, p.units, const_cast<int*>(p.seen), st)) != cudaSuccess)
            return e;
        e = launch_dependent(attend_kernel<D, R>, grid, 32 * C::kWarps, smem, st, p);
    } else {
        attend_kernel<D, R><<<grid, 32 * C::kWarps, smem, st>>>(p);
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) return e;
    const int rows = std::min(p.rows, R);
    return launch_dependent(merge_kernel<D, R>,
                            dim3(grid.x, rows + (p.units + grid.x - 1) / grid.x), 32 * kMergeWarps,
                            0, st, p, rows);
}

}  // namespace

// A part for each warp and block of the largest grid; as many warps as any of the kernels of 8 rows, or of
// 16, has.
template <int R>
constexpr size_t kParts =
    kAttendBlocks * (1 + std::max(std::max(Config<64, R>::kWarps, Config<128, R>::kWarps),
                                  R == 8 ? std::max(Config<64, 4>::kWarps, Config<128, 4>::kWarps)
                                         : 0));

// blocks' split units, then windows, then parts
size_t attend_workspace(int units, int rows, int n, int d)
{
    const int pr = part_rows(rows);
    return up256(kAttendBlocks * sizeof(int2)) +
           up256(static_cast<size_t>(units) * (1 + n) * 4) +
           up256((pr == 8 ? kParts<8> : kParts<16>) * (pr * d + 2 * pr) * 4);
}

cudaError_t launch_attend(const AttendArgs& a, int sms, cudaStream_t st)
{
    AttendParams p;
    p.a = a;
    p.units = a.B * a.H;
    p.rows = a.G * a.n;
    const int pr = part_rows(p.rows);
    const int parts = (p.rows + pr - 1) / pr;
    p.parts = Divisor(parts);
    p.G = Divisor(a.G);
    p.H = Divisor(a.H);
    p.chunks = (p.units * parts + 31) / 32;
    p.c = a.scale * 1.4426950408889634f;
    uint8_t* ws = static_cast<uint8_t*>(a.ws);
    p.split = reinterpret_cast<int2*>(ws);
    ws += up256(kAttendBlocks * sizeof(int2));
    p.seen = a.window > 0 ? reinterpret_cast<const int*>(ws) : nullptr;
    ws += up256(static_cast<size_t>(p.units) * (1 + a.n) * 4);
    p.part = reinterpret_cast<float*>(ws);
    if (a.d == 128)
        return p.rows <= 4   ? launch<128, 4>(p, sms, st)
               : p.rows <= 8 ? launch<128, 8>(p, sms, st)
                             : launch<128, 16>(p, sms, st);
    return p.rows <= 4   ? launch<64, 4>(p, sms, st)
           : p.rows <= 8 ? launch<64, 8>(p, sms, st)
                         : launch<64, 16>(p, sms, st);
}

}  // namespace twk
