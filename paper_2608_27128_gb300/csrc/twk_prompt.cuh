// twk_prompt.cuh -- what the kernels over packed prompts share: the sequences, the keys that tokens
// see, in tiles, and the even division of a call's work among the blocks of a grid.
#pragma once
#include <cstdint>

#include "twk_internal.h"
#include "twk_prompt_internal.h"
#include "twk_ptx.cuh"

namespace twk {

constexpr int kTileKeys = 128;      // keys of a tile
constexpr int kTileRows = 128;      // query rows of a tile: (token, head) pairs, the heads side by side
constexpr int kPromptBlocks = 152;  // of the largest grid: workspaces do not depend on the device

struct Sequence {
    int t0, n;       // first row of q, tokens
    int j0, m;       // first row of k, keys
    bool ok;         // false: a data error, n = m = 0
};

__device__ __forceinline__ void rows_of(const int* offsets, const int* lens, int b, int rows,
                                        int& first, int& count, bool& ok)
{
    first = offsets ? offsets[b] : 0;
    const int end = offsets ? offsets[b + 1] : rows;
    ok = ok && first >= 0 && first <= end && end <= rows;
    count = end - first;
    if (lens) {
        const int n = lens[b];
        ok = ok && n >= 0 && n <= count;
        count = n;
    }
}

__device__ __forceinline__ Sequence sequence_of(const PromptArgs& a, int b)
{
    Sequence q;
    q.ok = true;
    rows_of(a.seqs.offsets, a.seqs.lens, b, a.s.tokens, q.t0, q.n, q.ok);
    // without offsets of their own the keys are as the tokens: also their number, where lens gives that
    rows_of(a.seqs.k_offsets ? a.seqs.k_offsets : a.seqs.offsets,
            a.seqs.k_lens ? a.seqs.k_lens : a.seqs.k_offsets ? nullptr : a.seqs.lens, b, a.s.keys, q.j0,
            q.m, q.ok);
    if (!q.ok) q.n = q.m = 0;
    return q;
}

// The key tiles that some tokens at positions [first, last] see, in order: the first `sinks`, then
// those from `from` on: tile i is i where i < sinks, from + i - sinks else.
struct KeyTiles {
    int sinks, from, count;
    __device__ __forceinline__ int tile(int i) const { return i < sinks ? i : from + i - sinks; }
};

__device__ __forceinline__ KeyTiles key_tiles(const PromptArgs& a, int first, int last)
{
    KeyTiles t{};
    if (last < 0) return t;
    first = max(first, 0);
    const int end = last / kTileKeys + 1;
    if (a.window > 0) {
        t.from = max(first - a.window + 1, 0) / kTileKeys;
        t.sinks = min((min(a.n_sink, last + 1) + kTileKeys - 1) / kTileKeys, t.from);
    }
    t.count = t.sinks + end - t.from;
    return t;
}

// ---- small things

__device__ __forceinline__ float exp2_approx(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// the lowest n bits (none for n <= 0, all for n >= 32)
__device__ __forceinline__ uint32_t bits_below(int n)
{
    return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u;
}
__device__ __forceinline__ float as_f(uint32_t x) { return __uint_as_float(x); }

// Orders every later use of x after the preceding tcgen05.wait::ld.
__device__ __forceinline__ void reg_fence(uint32_t (&x)[32])
{
#pragma unroll
    for (int i = 0; i < 32; i += 8)
        asm volatile(""
                     : "+r"(x[i]), "+r"(x[i + 1]), "+r"(x[i + 2]), "+r"(x[i + 3]), "+r"(x[i + 4]),
                       "+r"(x[i + 5]), "+r"(x[i + 6]), "+r"(x[i + 7]));
}

// Every lane waits (each needs the acquire), the warp agrees on the verdict.
__device__ __forceinline__ bool all_wait(uint64_t* bar, uint32_t parity, const WaitCtl& w, int where)
{
    if (__all_sync(0xffffffffu, mbar_try_wait(smem_u32(bar), parity))) return true;
    const bool ok = mbar_wait(bar, parity, w, where);
    return __all_sync(0xffffffffu, ok);
}

__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity, uint64_t limit_ns)
{
    const uint64_t limit = limit_ns > kDrainFloorNs ? limit_ns : kDrainFloorNs;
    const uint32_t a = smem_u32(bar);
    const uint64_t t0 = globaltimer_ns();
    while (!mbar_try_wait_sleep(a, parity, 1000000u))
        if (globaltimer_ns() - t0 > limit) return;
}

// A ring's slot and the parity of its phase.
template <int kN>
struct Ring {
    uint32_t slot = 0, phase = 0;
    __device__ __forceinline__ void next()
    {
        if (++slot == kN) {
            slot = 0;
            phase ^= 1u;
        }
    }
};

// ---- work among blocks
//
// A call's items (of a sequence and KV head) follow one another, each as long as W::length says: its tiles,
// and up to kSnap more for what it takes beside them, at least 1.  All units are cut into even spans, one for
// each block.  An item that spans share is done in parts, which a second kernel joins in order: what is cut
// where depends on the sizes alone.  A cut within a.snap units of an item's end moves there, since a part
// costs about as much as so many units (and a cut that stays inside an item is at one of its tiles).

constexpr int kSnap = 3;            // least a.snap
constexpr int kChunks = 256;        // groups of sequences with their sums in shared memory

// x / y, both above 0
__device__ __forceinline__ long long quotient(long long x, long long y)
{
    if (((x | y) >> 31) == 0) return static_cast<unsigned>(x) / static_cast<unsigned>(y);
    return x / y;
}

__device__ __forceinline__ long long shfl64(long long x, int lane)
{
    return __shfl_sync(0xffffffffu, x, lane);
}

__device__ __forceinline__ long long inclusive_scan(long long x)
{
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (threadIdx.x % 32 >= o) x += y;
    }
    return x;
}

// The sequence of a lane, its items of a head and their units.
struct LaneUnits {
    Sequence s;
    int items;
    long long units;
};

// The lanes' sequences b0 + lane (0 items from B on), by a converged warp.
template <class W>
__device__ __forceinline__ LaneUnits lane_units(const PromptArgs& a, int b0)
{
    const int lane = threadIdx.x % 32;
    LaneUnits u{};
    if (b0 + lane < a.s.B) u.s = sequence_of(a, b0 + lane);
    u.items = W::items(a, u.s);
    if (u.items <= 4)
        for (int i = 0; i < u.items; ++i) u.units += W::length(a, u.s, i);
    // the long ones by all lanes
    for (unsigned big = __ballot_sync(0xffffffffu, u.items > 4); big; big &= big - 1) {
        const int l = __ffs(big) - 1, items = __shfl_sync(0xffffffffu, u.items, l);
        Sequence t;
        t.t0 = t.j0 = 0;
        t.ok = true;
        t.n = __shfl_sync(0xffffffffu, u.s.n, l);
        t.m = __shfl_sync(0xffffffffu, u.s.m, l);
        long long all = 0;
        for (int i = lane; i < items; i += 32) all += W::length(a, t, i);
#pragma unroll
        for (int o = 16; o > 0; o /= 2) all += __shfl_xor_sync(0xffffffffu, all, o);
        if (lane == l) u.units = all;
    }
    return u;
}

__device__ __forceinline__ int chunk_size(int B)
{
    return (B + 32 * kChunks - 1) / (32 * kChunks) * 32;
}

// More than 32 sequences: units (of all heads) before each chunk, by all warps of the block, to
// sums[kChunks + 1] in shared memory, and all items in sums[kChunks + 1].  Ends with a barrier.
template <class W>
__device__ __forceinline__ void sum_chunks(const PromptArgs& a, long long* sums)
{
    const int lane = threadIdx.x % 32, size = chunk_size(a.s.B);
    const int chunks = (a.s.B + size - 1) / size;
    long long* counts = sums + kChunks + 1;
    for (int c = threadIdx.x / 32; c < chunks; c += blockDim.x / 32) {
        long long units = 0, items = 0;
        for (int b = c * size; b < min((c + 1) * size, a.s.B); b += 32) {
            const LaneUnits u = lane_units<W>(a, b);
            units += u.units;
            items += u.items;
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            units += __shfl_xor_sync(0xffffffffu, units, o);
            items += __shfl_xor_sync(0xffffffffu, items, o);
        }
        if (lane == 0) {
            sums[c] = units * a.s.H;
            counts[c] = items * a.s.H;
        }
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        long long before = 0, items = 0;
        for (int c0 = 0; c0 < chunks; c0 += 32) {
            const long long n = c0 + lane < chunks ? sums[c0 + lane] : 0;
            items += c0 + lane < chunks ? counts[c0 + lane] : 0;
            const long long scan = inclusive_scan(n);
            if (c0 + lane < chunks) sums[c0 + lane] = before + scan - n;
            before += shfl64(scan, 31);
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) items += __shfl_xor_sync(0xffffffffu, items, o);
        if (lane == 0) {
            sums[chunks] = before;
            counts[0] = items;
        }
    }
    __syncthreads();
}
constexpr int kSumsBytes = (2 * kChunks + 1) * 8;

// A block's walk over the items of its span: next() gives one part after another.
// ONE: with a start of its own for one sequence.
template <class W, bool ONE = true>
struct Walk {
    int b = 0, head = 0, item = 0, length = 0;   // where it is; length of the item
    int items = 0;                               // of the sequence and head
    int off = 0, take = 0;                       // the part: its first unit and units
    Sequence s{};
    long long begin = 0, end = 0;                // the item's first unit; where the span ends, before it snaps
    long long each = 0;                          // units of a block, and how many blocks have one more
    unsigned over = 0;
    int blocks = 0;
    bool more = false;                           // the part at hand is one

    // By one converged warp; sums as sum_chunks left them, not looked at for up to 32 sequences.
    __device__ __forceinline__ void start(const PromptArgs& a, const long long* sums)
    {
        const int lane = threadIdx.x % 32;
        if constexpr (ONE) {
            if (a.s.B == 1 && start_one(a)) return;
        }
        long long units, count;
        LaneUnits u{};
        if (a.s.B <= 32) {
            u = lane_units<W>(a, 0);
            units = u.units;
            count = u.items;
#pragma unroll
            for (int o = 16; o > 0; o /= 2) {
                units += __shfl_xor_sync(0xffffffffu, units, o);
                count += __shfl_xor_sync(0xffffffffu, count, o);
            }
            units *= a.s.H;
            count *= a.s.H;
        } else {
            const int size = chunk_size(a.s.B);
            units = sums[(a.s.B + size - 1) / size];
            count = sums[kChunks + 1];
        }
        if (units == 0) return;
        // at least four units to a block, or half an item where those are short
        long long want = units / 4 > 2 * count ? units / 4 : 2 * count;
        if (want > units) want = units;          // every span has units
        blocks = static_cast<int>(want < gridDim.x ? want : gridDim.x);
        if (static_cast<int>(blockIdx.x) >= blocks) return;
        each = quotient(units, blocks);
        over = static_cast<unsigned>(units - each * blocks);
        const long long g = cut(blockIdx.x);
        if (g >= units) return;
        end = cut(blockIdx.x + 1);

        // the sequence, then the head, then the item with unit g
        long long rest = g;
        int b0 = 0;
        if (a.s.B > 32) {
            const int size = chunk_size(a.s.B);
            int lo = 0;
            for (int hi = (a.s.B + size - 1) / size - 1; lo < hi;) {
                const int mid = (lo + hi + 1) / 2;
                if (sums[mid] <= g) lo = mid;
                else hi = mid - 1;
            }
            rest -= sums[lo];
            b0 = lo * size;
            u = lane_units<W>(a, b0);
        }
        long long per_head = 0;
        for (;;) {
            const long long scan = inclusive_scan(u.units * a.s.H);
            const unsigned past = __ballot_sync(0xffffffffu, scan > rest);
            if (past) {
                const int l = __ffs(past) - 1;
                per_head = shfl64(u.units, l);
                rest -= shfl64(scan, l) - per_head * a.s.H;
                b = b0 + l;
                items = __shfl_sync(0xffffffffu, u.items, l);
                s.t0 = __shfl_sync(0xffffffffu, u.s.t0, l);
                s.n = __shfl_sync(0xffffffffu, u.s.n, l);
                s.j0 = __shfl_sync(0xffffffffu, u.s.j0, l);
                s.m = __shfl_sync(0xffffffffu, u.s.m, l);
                s.ok = true;
                break;
            }
            rest -= shfl64(scan, 31);
            b0 += 32;
            if (b0 >= a.s.B) return;
            u = lane_units<W>(a, b0);
        }
        head = static_cast<int>(quotient(rest, per_head));
        rest -= per_head * head;
        for (int i = 0;; i += 32) {
            if (i >= items) return;
            const long long mine = i + lane < items ? W::length(a, s, i + lane) : 0;
            const long long scan = inclusive_scan(mine);
            const unsigned past = __ballot_sync(0xffffffffu, scan > rest);
            if (past) {
                const int l = __ffs(past) - 1;
                length = static_cast<int>(shfl64(mine, l));
                off = static_cast<int>(rest - (shfl64(scan, l) - length));
                item = i + l;
                break;
            }
            rest -= shfl64(scan, 31);
        }
        begin = g - off;
        more = true;
        if (off <= a.snap) off = 0;
        else if (length - off <= a.snap) advance(a);
        part(a);
    }

    // The part after this one, by any one lane.
    __device__ __forceinline__ void next(const PromptArgs& a)
    {
        if (off + take < length) more = false;
        else advance(a);
        part(a);
    }

    // What to add to x so that it is, modulo the length of a span, the part's place in its span.
    __device__ __forceinline__ int turn(int x) const
    {
        const long long d = begin + off - cut(blockIdx.x) - x;
        const int r = static_cast<int>(d % each);
        return r < 0 ? r + static_cast<int>(each) : r;
    }

    // Blocks that share the item, this one being the first.
    __device__ __forceinline__ int parts(const PromptArgs& a) const
    {
        int n = 1;
        while (cut(blockIdx.x + n) + a.snap < begin + length) ++n;
        return n;
    }

private:
    // The same for one sequence whose units are counted in 32 bits: a third of the instructions, which are
    // read anew with every launch (4500 cycles before the first item, now 3500).  False where they are
    // not.
    __device__ __forceinline__ bool start_one(const PromptArgs& a)
    {
        const int lane = threadIdx.x % 32;
        s = sequence_of(a, 0);
        items = W::items(a, s);
        if (items > 8192 || max(s.n, s.m) > 1 << 19 || a.s.H > 1024) return false;
        unsigned mine = 0;          // at most 256 items of 2^19 + kSnap units
        for (int i = lane; i < items; i += 32) mine += W::length(a, s, i);
        if (__any_sync(0xffffffffu, mine > (1u << 30) / 32 / static_cast<unsigned>(a.s.H)))
            return false;
        const unsigned per_head = __reduce_add_sync(0xffffffffu, mine);
        if (per_head == 0) return true;
        const unsigned units = per_head * a.s.H, count = items * a.s.H;
        blocks = static_cast<int>(min(min(max(units / 4, 2 * count), units), gridDim.x));
        if (static_cast<int>(blockIdx.x) >= blocks) return true;
        each = units / blocks;
        over = units % blocks;
        const unsigned g = static_cast<unsigned>(cut(blockIdx.x));
        end = cut(blockIdx.x + 1);
        head = static_cast<int>(g / per_head);
        unsigned rest = g - head * per_head;
        for (int i = 0;; i += 32) {
            const unsigned n = i + lane < items ? W::length(a, s, i + lane) : 0;
            unsigned scan = n;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const unsigned y = __shfl_up_sync(0xffffffffu, scan, o);
                if (lane >= o) scan += y;
            }
            const unsigned past = __ballot_sync(0xffffffffu, scan > rest);
            if (past) {
                const int l = __ffs(past) - 1;
                length = __shfl_sync(0xffffffffu, n, l);
                off = static_cast<int>(rest) - (__shfl_sync(0xffffffffu, scan, l) - length);
                item = i + l;
                break;
            }
            rest -= __shfl_sync(0xffffffffu, scan, 31);
        }
        begin = static_cast<long long>(g) - off;
        more = true;
        if (off <= a.snap) off = 0;
        else if (length - off <= a.snap) advance(a);
        part(a);
        return true;
    }

    // where the span of block c begins, before it snaps
    __device__ __forceinline__ long long cut(unsigned c) const
    {
        return each * c + over * c / static_cast<unsigned>(blocks);
    }
    __device__ __forceinline__ void advance(const PromptArgs& a)
    {
        begin += length;
        off = 0;
        if (++item == items) {
            item = 0;
            if (++head == a.s.H) {
                head = 0;
                do {
                    if (++b == a.s.B) {
                        more = false;
                        return;
                    }
                    s = sequence_of(a, b);
                    items = W::items(a, s);
                } while (items == 0);
            }
        }
        length = W::length(a, s, item);
    }
    // how far the span takes the item
    __device__ __forceinline__ void part(const PromptArgs& a)
    {
        if (!more) return;
        take = length - off;
        if (end < begin + length) {
            if (end - begin <= a.snap) more = false;
            else if (begin + length - end > a.snap) take = static_cast<int>(end - begin) - off;
        }
    }
};

}  // namespace twk
