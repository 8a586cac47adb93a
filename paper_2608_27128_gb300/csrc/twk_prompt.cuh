// twk_prompt.cuh -- what the kernels over packed prompts share: the sequences, the keys that tokens
// see, in tiles, and the even division of a call's work among the blocks of a grid.
#pragma once
#include <cstdint>

#include "twk_prompt_internal.h"

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
    const bool own = a.seqs.k_offsets || !a.seqs.offsets;
    rows_of(own ? a.seqs.k_offsets : a.seqs.offsets,
            a.seqs.k_lens ? a.seqs.k_lens : own ? nullptr : a.seqs.lens, b, a.s.keys, q.j0, q.m,
            q.ok);
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

// ---- work among blocks
//
// A call's items (of a sequence and KV head) follow one another, each as long as W::length says (1
// or more units), and all units are cut into equal spans, one for each block.  An item that spans share
// is done in parts, which a second kernel joins in order: what is cut where depends on the sizes alone.
// A cut within kSnap units of an item's end moves there, since a part costs about as much as so many
// units.

constexpr int kSnap = 3;
constexpr int kChunks = 256;        // groups of sequences with their sums in shared memory

// lengths of the sequence's items of one head, added up by a warp
template <class W>
__device__ __forceinline__ long long warp_length(const PromptArgs& a, const Sequence& s, int items)
{
    int sum = 0;                    // at most 2^18 items a lane, of 2^17 + 2 units: in 64 bits below
    long long all = 0;
    for (int i = threadIdx.x % 32; i < items; i += 32) {
        sum += W::length(a, s, i);
        if (sum > (1 << 29)) all += sum, sum = 0;
    }
    all += sum;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) all += __shfl_xor_sync(0xffffffffu, all, o);
    return all;
}

// The lanes' sequences b0 + lane below `end`: units of all their heads (0 where there is none), and items.
template <class W>
__device__ __forceinline__ long long lane_units(const PromptArgs& a, int b, int end, long long& items_all)
{
    Sequence s{};
    if (b < end) s = sequence_of(a, b);
    const int items = W::items(a, s);
    long long units = 0;
    if (items <= 8)
        for (int i = 0; i < items; ++i) units += W::length(a, s, i);
    for (unsigned big = __ballot_sync(0xffffffffu, items > 8); big; big &= big - 1) {
        const int l = __ffs(big) - 1;
        Sequence t;
        t.t0 = __shfl_sync(0xffffffffu, s.t0, l);
        t.n = __shfl_sync(0xffffffffu, s.n, l);
        t.j0 = __shfl_sync(0xffffffffu, s.j0, l);
        t.m = __shfl_sync(0xffffffffu, s.m, l);
        t.ok = true;
        const long long x = warp_length<W>(a, t, __shfl_sync(0xffffffffu, items, l));
        if (threadIdx.x % 32 == l) units = x;
    }
    items_all = static_cast<long long>(items) * a.s.H;
    return units * a.s.H;
}

__device__ __forceinline__ int chunk_size(int B) { return (B + 32 * kChunks - 1) / (32 * kChunks) * 32; }

struct Totals {
    long long units, items;
};

// Units before each chunk, by all warps of the block, to sums[kChunks + 1] in shared memory, and the totals.
// Ends with a barrier.
template <class W>
__device__ __forceinline__ Totals sum_chunks(const PromptArgs& a, long long* sums, long long* counts)
{
    const int lane = threadIdx.x % 32, size = chunk_size(a.s.B);
    const int chunks = (a.s.B + size - 1) / size;
    for (int c = threadIdx.x / 32; c < chunks; c += blockDim.x / 32) {
        long long units = 0, items = 0;
        for (int b = c * size; b < min((c + 1) * size, a.s.B); b += 32) {
            long long n;
            units += lane_units<W>(a, b + lane, a.s.B, n);
            items += n;
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) {
            units += __shfl_xor_sync(0xffffffffu, units, o);
            items += __shfl_xor_sync(0xffffffffu, items, o);
        }
        if (lane == 0) {
            sums[c] = units;
            counts[c] = items;
        }
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        long long before = 0, items = 0;
        for (int c0 = 0; c0 < chunks; c0 += 32) {
            const long long n = c0 + lane < chunks ? sums[c0 + lane] : 0;
            items += c0 + lane < chunks ? counts[c0 + lane] : 0;
            long long scan = n;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const long long y = __shfl_up_sync(0xffffffffu, scan, o);
                if (lane >= o) scan += y;
            }
            __syncwarp();
            if (c0 + lane < chunks) sums[c0 + lane] = before + scan - n;
            before += __shfl_sync(0xffffffffu, scan, 31);
        }
#pragma unroll
        for (int o = 16; o > 0; o /= 2) items += __shfl_xor_sync(0xffffffffu, items, o);
        if (lane == 0) {
            sums[chunks] = before;
            counts[0] = items;
        }
    }
    __syncthreads();
    return {sums[chunks], counts[0]};
}

// Blocks that get a span: no more than there are items where those are short, and at least four
// units to a block where they are long.
__device__ __forceinline__ int span_blocks(const Totals& t)
{
    long long n = t.units / 4 > t.items ? t.units / 4 : t.items;
    return static_cast<int>(n < gridDim.x ? n : gridDim.x);
}

// A place in the sequence of all units.
struct Place {
    int b, head, item, length;      // length: of the item
    int items;                      // of the sequence and head
    int off;                        // unit of the item
    Sequence s;
};

// The place of unit g < total, by one warp.
template <class W>
__device__ __forceinline__ Place locate(const PromptArgs& a, const long long* sums, long long g)
{
    const int lane = threadIdx.x % 32, size = chunk_size(a.s.B);
    int lo = 0;
    for (int hi = (a.s.B + size - 1) / size - 1; lo < hi;) {
        const int mid = (lo + hi + 1) / 2;
        if (sums[mid] <= g) lo = mid;
        else hi = mid - 1;
    }
    long long rest = g - sums[lo];
    Place p{};
    long long units = 0;
    for (int b = lo * size; b < a.s.B; b += 32) {
        long long n, mine = lane_units<W>(a, b + lane, a.s.B, n), scan = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const long long y = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += y;
        }
        const unsigned past = __ballot_sync(0xffffffffu, scan > rest);
        if (past) {
            const int l = __ffs(past) - 1;
            units = __shfl_sync(0xffffffffu, mine, l);
            rest -= __shfl_sync(0xffffffffu, scan, l) - units;
            p.b = b + l;
            break;
        }
        rest -= __shfl_sync(0xffffffffu, scan, 31);
    }
    p.s = sequence_of(a, p.b);
    p.items = W::items(a, p.s);
    units /= a.s.H;
    if (units > 0) {
        p.head = static_cast<int>(rest / units);
        rest -= units * p.head;
    }
    for (int i = 0; i < p.items; i += 32) {
        const int mine = i + lane < p.items ? W::length(a, p.s, i + lane) : 0;
        int scan = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int y = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += y;
        }
        const unsigned past = __ballot_sync(0xffffffffu, scan > rest);
        if (past) {
            const int l = __ffs(past) - 1;
            p.length = __shfl_sync(0xffffffffu, mine, l);
            p.off = static_cast<int>(rest - (__shfl_sync(0xffffffffu, scan, l) - p.length));
            p.item = i + l;
            break;
        }
        rest -= __shfl_sync(0xffffffffu, scan, 31);
    }
    return p;
}

// The next item; false past the last one.
template <class W>
__device__ __forceinline__ bool next_item(const PromptArgs& a, Place& p)
{
    p.off = 0;
    if (++p.item == p.items) {
        p.item = 0;
        if (++p.head == a.s.H) {
            p.head = 0;
            do {
                if (++p.b == a.s.B) return false;
                p.s = sequence_of(a, p.b);
                p.items = W::items(a, p.s);
            } while (p.items == 0);
        }
    }
    p.length = W::length(a, p.s, p.item);
    return true;
}

// Where the span of block c begins, and its place; the end of a block's span is the next one's begin.
__device__ __forceinline__ long long raw_cut(long long units, int blocks, int c)
{
    return units / blocks * c + units % blocks * c / blocks;
}

template <class W>
__device__ __forceinline__ long long cut(const PromptArgs& a, const long long* sums, long long units,
                                         int blocks, int c, Place& p)
{
    const long long g = raw_cut(units, blocks, c);
    if (g >= units) return units;
    p = locate<W>(a, sums, g);
    if (p.off <= kSnap) {
        const int off = p.off;
        p.off = 0;
        return g - off;
    }
    if (p.length - p.off <= kSnap) {
        const int more = p.length - p.off;
        next_item<W>(a, p);
        return g + more;
    }
    return g;
}

// Blocks that share the item, from the one that has its unit `off` (the item begins at unit `begin`) on.
__device__ __forceinline__ int parts_of(long long units, int blocks, int c, long long begin, int length)
{
    int parts = 1;
    while (c + parts < blocks && raw_cut(units, blocks, c + parts) + kSnap < begin + length) ++parts;
    return parts;
}

}  // namespace twk
