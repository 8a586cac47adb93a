// twk_cache.cu -- writing, moving and reading the pages of a cache held in 4 bits
// (layout and rounding: twk_cache.cuh).
//
//   index_kernel    the kept rows of every unit in order, from a mask
//   pack_kernel     kept rows of a dense cache -> codes -> pages
//   append_kernel   the rows of new tokens -> codes -> the slots after a unit's last
//   compact_kernel  kept slots of pages -> other pages, codes as they are
//   read_kernel     pages -> bf16 rows
//
// All are bound by memory, or by latency where the call is small.  Keys are stored slot by slot.
// Values are stored for the attention kernel with eight slots of one dimension to a word, while
// rounding, moving and reading want eight dimensions of one slot: the word held by both sides is
// an 8 x 8 block of codes, transposed in registers in 32 instructions (transpose8).
#include "twk_cache.cuh"
#include "twk_cache_internal.h"
#include "twk_internal.h"
#include "twk_ptx.cuh"

namespace twk {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kInvalid = TWINKV_ERR_INVALID_ARG;
constexpr int kTooLarge = TWINKV_ERR_TOO_LARGE;

// out[i] nibble n = in[n] nibble i
__device__ __forceinline__ void transpose8(uint32_t (&r)[8])
{
    uint32_t a[8], b[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = __byte_perm(r[i], r[i + 4], 0x5410);
        a[i + 4] = __byte_perm(r[i], r[i + 4], 0x7632);
    }
#pragma unroll
    for (int i = 0; i < 8; i += 4)
#pragma unroll
        for (int j = i; j < i + 2; ++j) {
            b[j] = __byte_perm(a[j], a[j + 2], 0x6240);
            b[j + 2] = __byte_perm(a[j], a[j + 2], 0x7351);
        }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        r[i] = (b[i] & 0x0f0f0f0fu) | ((b[i + 1] << 4) & 0xf0f0f0f0u);
        r[i + 1] = ((b[i] >> 4) & 0x0f0f0f0fu) | (b[i + 1] & 0xf0f0f0f0u);
    }
}

// A slot's words of eight value codes (dimensions 8 j .. 8 j + 7, in the key words' order of
// nibbles) are kept in shared memory at slot * kSlotWords + j, the stride odd against bank
// conflicts.
template <int D>
constexpr int kSlotWords = D / 8 + 1;

// One block of transpose8: the values of dimensions [8 j, 8 j + 8) at the eight slots with the
// given t and a (slot = 32 a + 16 c + 8 k + 2 t + b).
struct Block8 {
    int j, t, a;
    // consecutive blocks are the 16 words of a page's row (m, g), then the next m
    __device__ explicit Block8(int i) : j(i / 16 * 2 + i / 2 % 2), t(i / 4 % 4), a(i % 2) {}
    __device__ int slot(int n) const
    {
        return 32 * a + n / 2 % 2 * 16 + n % 2 * 8 + 2 * t + n / 4;
    }
    // word of the page's value codes with dimension 8 j + g
    __device__ int word(int g) const
    {
        return ((j / 2 * 8 + g) * 4 + t) * 4 + j % 2 * 2 + a;
    }
    // nibble of a slot's word that holds dimension 8 j + g
    __device__ static constexpr int nibble(int g) { return g / 2 + 4 * (g % 2); }
};

// ---------------------------------------------------------------- index

constexpr int kVecChunk = kThreads;       // 16-byte vectors of a block

// Vector v of a unit's mask: the bytes at positions [16 v - mis, +16) of the row, those outside
// [0, limit) zero.  Rows start at any address: mis makes the vectors' addresses multiples of 16.
__device__ __forceinline__ uint4 mask_vector(const uint8_t* row, int mis, int64_t v, int limit)
{
    const int64_t p = 16 * v - mis;
    if (p >= 0 && p + 16 <= limit) return *reinterpret_cast<const uint4*>(row + p);
    uint32_t w[4] = {};
    for (int i = 0; i < 16; ++i)
        if (p + i >= 0 && p + i < limit)
            w[i / 4] |= static_cast<uint32_t>(row[p + i]) << (8 * (i % 4));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ int mask_count(const uint4& v)
{
    return __popc((v.x & 0x01010101u) | (v.y & 0x01010101u) << 1 | (v.z & 0x01010101u) << 2 |
                  (v.w & 0x01010101u) << 3);
}

// A block per 4096 positions of a unit.  Each counts what lies before its own positions by itself
// (masks are small against the rows: at 131072 positions a unit's blocks read 2 MB of L2 where
// its rows are 32 MB), so that one launch does it; the unit's last block, which thus sees the
// whole mask, also checks it, the length and the page numbers.
__global__ void __launch_bounds__(kThreads) index_kernel(const IndexArgs a)
{
    __shared__ int s_sum[kWarps], s_bad[kWarps], s_scan[kWarps];
    __shared__ uint16_t s_place[16 * kVecChunk];
    wait_for_previous();
    const int u = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int limit = a.limit ? a.limit[u] : a.N;
    int status = 0;
    if (limit < 0 || limit > a.limit_most) {
        status = kInvalid;
        limit = 0;
    }
    const uint8_t* row = a.mask ? a.mask + static_cast<int64_t>(u) * a.N : nullptr;
    const int mis = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15);
    const int64_t vectors = row ? (static_cast<int64_t>(limit) + mis + 15) / 16 : 0;
    const int64_t v0 = static_cast<int64_t>(blockIdx.x) * kVecChunk;
    const int last = vectors > 0 ? static_cast<int>((vectors - 1) / kVecChunk) : 0;
    if (static_cast<int>(blockIdx.x) > last) return;
    int total = limit;
    bool bad = false;
    if (row) {
        int before = 0;
#pragma unroll 4
        for (int64_t v = threadIdx.x; v < v0; v += kThreads) {
            const uint4 x = mask_vector(row, mis, v, limit);
            before += mask_count(x);
            bad |= ((x.x | x.y | x.z | x.w) & 0xfefefefeu) != 0;
        }
        const int64_t v = v0 + threadIdx.x;
        const uint4 x = v < vectors ? mask_vector(row, mis, v, limit) : make_uint4(0, 0, 0, 0);
        bad |= ((x.x | x.y | x.z | x.w) & 0xfefefefeu) != 0;
        const int own = mask_count(x);
        int scan = own;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            const int y = __shfl_up_sync(0xffffffffu, scan, m);
            if (lane >= m) scan += y;
        }
        before = __reduce_add_sync(0xffffffffu, before);
        bad = __any_sync(0xffffffffu, bad);
        if (lane == 31) s_scan[warp] = scan;
        if (lane == 0) {
            s_sum[warp] = before;
            s_bad[warp] = bad;
        }
        __syncthreads();
        int base = 0;
        total = 0;
        bad = false;
        for (int i = 0; i < kWarps; ++i) {
            base += s_sum[i];
            total += s_sum[i] + s_scan[i];
            bad |= s_bad[i] != 0;
        }
        // in shared memory by rank, then out in order
        int rank = scan - own, here = 0;
        for (int i = 0; i < kWarps; ++i) {
            rank += i < warp ? s_scan[i] : 0;
            here += s_scan[i];
        }
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (w[i / 4] >> (8 * (i % 4)) & 1)
                s_place[rank++] = static_cast<uint16_t>(16 * threadIdx.x + i);
        __syncthreads();
        int* out = a.index + static_cast<int64_t>(u) * a.N + base;
        const int p0 = static_cast<int>(16 * v0 - mis);
        for (int i = threadIdx.x; i < here; i += kThreads) out[i] = p0 + s_place[i];
    }
    if (static_cast<int>(blockIdx.x) != last) return;
    if (bad) status = kInvalid;
    if (status == 0 && total > static_cast<int64_t>(a.dst_max_pages) * kPage) status = kTooLarge;
    if (status) total = 0;
    bool off = false;
    for (int j = threadIdx.x; j < (total + kPage - 1) / kPage; j += kThreads)
        off |= static_cast<unsigned>(a.dst_table[static_cast<int64_t>(u) * a.dst_max_pages + j]) >=
               static_cast<unsigned>(a.n_pages);
    if (a.src_table && total)
        for (int j = threadIdx.x; j < (limit + kPage - 1) / kPage; j += kThreads)
            off |= static_cast<unsigned>(
                       a.src_table[static_cast<int64_t>(u) * a.src_max_pages + j]) >=
                   static_cast<unsigned>(a.n_pages);
    if (__syncthreads_or(off)) {
        status = kInvalid;
        total = 0;
    }
    if (threadIdx.x == 0) {
        a.out_lens[u] = total;
        if (a.out_status) a.out_status[u] = status;
    }
}

// ---------------------------------------------------------------- pages in shared memory

// The page is put together in shared memory and leaves in 16-byte stores.
template <int D>
struct PageImage {
    alignas(16) uint8_t bytes[PageLayout<D>::kBytes];
    uint32_t slots[kPage * kSlotWords<D>];   // value codes by slot
};

// a lane's share of a key row: the codes of chunks j and j + 4, and the group's scale and zero
template <int D>
__device__ __forceinline__ void put_key(uint8_t* page, int slot, int j, const uint32_t (&w)[2],
                                        float scale, int zero)
{
    using P = PageLayout<D>;
    *reinterpret_cast<uint32_t*>(page + P::key_word(slot, j)) = w[0];
    *reinterpret_cast<uint32_t*>(page + P::key_word(slot, j + 4)) = w[1];
    if (j % 8 == 0)
        *reinterpret_cast<uint32_t*>(page + P::kKeyGroups + (slot * P::kGroups + j / 8) * 4) =
            (__float_as_uint(scale) >> 16) | (0xc3000000u + (static_cast<uint32_t>(zero) << 16));
}

// the same of a value row, its codes as words of the slot
template <int D>
__device__ __forceinline__ void put_value(uint8_t* page, uint32_t* slot_words, int slot, int j,
                                          const uint32_t (&w)[2], float scale, int zero)
{
    using P = PageLayout<D>;
    slot_words[j] = w[0];
    slot_words[j + 4] = w[1];
    if (j % 8 == 0) {
        reinterpret_cast<uint16_t*>(page + P::kValScales)[slot * P::kGroups + j / 8] =
            static_cast<uint16_t>(__float_as_uint(scale) >> 16);
        reinterpret_cast<uint16_t*>(page + P::kValZeros)[P::val_zero(j / 8, slot)] =
            static_cast<uint16_t>(0xc300 + zero);
    }
}

// the value codes of the page from the slots' words
template <int D, int kBlock>
__device__ __forceinline__ void slots_to_page(PageImage<D>& im)
{
    uint32_t* codes = reinterpret_cast<uint32_t*>(im.bytes + PageLayout<D>::kValCodes);
    for (int i = threadIdx.x; i < D; i += kBlock) {
        const Block8 b(i);
        uint32_t r[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) r[n] = im.slots[b.slot(n) * kSlotWords<D> + b.j];
        transpose8(r);
#pragma unroll
        for (int g = 0; g < 8; ++g) codes[b.word(g)] = r[Block8::nibble(g)];
    }
}

template <int D, int kBlock>
__device__ __forceinline__ void store_page(const PageImage<D>& im, uint8_t* page)
{
    constexpr int kVec = PageLayout<D>::kBytes / 16;
#pragma unroll
    for (int i = threadIdx.x; i < kVec; i += kBlock)
        reinterpret_cast<uint4*>(page)[i] = reinterpret_cast<const uint4*>(im.bytes)[i];
}

// A lane's 16 values of a row, as bf16 pairs (float32 ones rounded): the 8 from `p` on and the 8 that
// lie 32 values further, so that four lanes read whole 64-byte pieces of a group.
template <typename T>
struct Values16;

template <>
struct Values16<uint16_t> {
    uint4 v[2] = {};
    __device__ void load(const uint16_t* p)
    {
        v[0] = __ldg(reinterpret_cast<const uint4*>(p));
        v[1] = __ldg(reinterpret_cast<const uint4*>(p + 32));
    }
    __device__ void get(uint32_t (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            x[4 * i] = v[i].x, x[4 * i + 1] = v[i].y, x[4 * i + 2] = v[i].z, x[4 * i + 3] = v[i].w;
    }
};

template <>
struct Values16<float> {
    float4 v[4] = {};
    __device__ void load(const float* p)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = __ldg(reinterpret_cast<const float4*>(p + i / 2 * 32) + i % 2);
    }
    __device__ void get(uint32_t (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_pair(v[i].x, v[i].y);
            x[2 * i + 1] = bf16_pair(v[i].z, v[i].w);
        }
    }
};

// Lane l of a row has the groups of 8 values (chunks) first() and first() + 4.
__device__ __forceinline__ int first_chunk(int l) { return l / 4 * 8 + l % 4; }

// ---------------------------------------------------------------- pack

// A block per page to fill.  D / 16 lanes hold a row, 16 values each; a thread loads all of its
// rows before it rounds the first, and five blocks of an SM do so in turn (two of float32 rows at
// d = 128, which are twice as large).
template <typename T, int D>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 4 && D == 128 ? 2 : 5)
    pack_kernel(const PackArgs a)
{
    using P = PageLayout<D>;
    constexpr int kLanes = D / 16, kStep = kThreads / kLanes, kSteps = kPage / kStep;
    __shared__ PageImage<D> im;
    wait_for_previous();
    const int u = blockIdx.y, first = blockIdx.x * kPage;
    const int count = min(kPage, a.lens[u] - first);
    if (count <= 0) return;
    const int j = first_chunk(threadIdx.x % kLanes), s0 = threadIdx.x / kLanes;
    const T* keys = static_cast<const T*>(a.keys) + static_cast<int64_t>(u) * a.N * D + 8 * j;
    const T* values = static_cast<const T*>(a.values) + static_cast<int64_t>(u) * a.N * D + 8 * j;
    const int* index = a.index ? a.index + static_cast<int64_t>(u) * a.N + first : nullptr;
    const int page = a.to.table[static_cast<int64_t>(u) * a.to.max_pages + blockIdx.x];
    // slots past the last row read that of slot 0 and become zeros
    int row[kSteps];
    Values16<T> k[kSteps], v[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int s = s0 + i * kStep < count ? s0 + i * kStep : 0;
        row[i] = index ? index[s] : first + s;
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) k[i].load(keys + static_cast<int64_t>(row[i]) * D);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) v[i].load(values + static_cast<int64_t>(row[i]) * D);
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
        if (s0 + i * kStep >= count) {
            row[i] = -1;
            k[i] = v[i] = Values16<T>{};
        }
    bool beyond = false;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int s = s0 + i * kStep;
        uint32_t x[8], w[2];
        float scale;
        int zero;
        k[i].get(x);
        beyond |= quantize16(x, w, &scale, &zero);
        put_key<D>(im.bytes, s, j, w, scale, zero);
        if (j == 0) reinterpret_cast<int*>(im.bytes + P::kPos)[s] = row[i];
        v[i].get(x);
        beyond |= quantize16(x, w, &scale, &zero);
        put_value<D>(im.bytes, im.slots + s * kSlotWords<D>, s, j, w, scale, zero);
    }
    if (beyond && a.out_status) a.out_status[u] = kInvalid;     // the index kernel has written it
    __syncthreads();
    slots_to_page<D, kThreads>(im);
    __syncthreads();
    store_page<D, kThreads>(im, a.to.base + static_cast<int64_t>(page) * P::kBytes);
}

// ---------------------------------------------------------------- append

constexpr int kAppendMost = kPage;   // new rows of a unit: they reach two pages at most

// A block per unit.  Rows are rounded side by side; the value codes, whose words hold eight
// slots, are then written word by word, each by one thread, which keeps the other slots' codes.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) append_kernel(const AppendArgs a)
{
    using P = PageLayout<D>;
    constexpr int kLanes = D / 16;
    __shared__ uint32_t slots[kAppendMost * kSlotWords<D>];
    const int u = blockIdx.x, b = u / a.H, h = u % a.H;
    const int len = a.lens[u];
    const int* table = a.to.table + static_cast<int64_t>(u) * a.to.max_pages;
    int status = len < 0 ? kInvalid
                 : static_cast<int64_t>(len) + a.n > static_cast<int64_t>(a.to.max_pages) * kPage
                     ? kTooLarge
                     : 0;
    uint8_t* page[2] = {};
    const int p0 = len / kPage;
    if (status == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (len + a.n > (p0 + i) * kPage) {
                const int id = table[p0 + i];
                if (static_cast<unsigned>(id) >= static_cast<unsigned>(a.to.n_pages))
                    status = kInvalid;
                else
                    page[i] = a.to.base + static_cast<int64_t>(id) * P::kBytes;
            }
    }
    __syncthreads();                 // out_lens may be lens
    if (threadIdx.x == 0) {
        a.out_lens[u] = status ? len : len + a.n;
        if (a.out_status) a.out_status[u] = status;
    }
    if (status) return;
    const int at = len % kPage;      // the first new row's slot of page[0]
    bool beyond = false;
    for (int i0 = 0; i0 < a.n; i0 += kThreads / kLanes) {
        const int i = i0 + threadIdx.x / kLanes, j = first_chunk(threadIdx.x % kLanes);
        const bool on = i < a.n;
        Values16<T> k, v;
        if (on) {
            k.load(static_cast<const T*>(a.keys) + b * a.k_batch + i * a.k_token + h * a.k_head +
                   8 * j);
            v.load(static_cast<const T*>(a.values) + b * a.v_batch + i * a.v_token +
                   h * a.v_head + 8 * j);
        }
        uint8_t* to = page[(at + i) / kPage ? 1 : 0];
        const int s = (at + i) % kPage;
        uint32_t x[8], w[2];
        float scale;
        int zero;
        k.get(x);
        beyond |= quantize16(x, w, &scale, &zero);
        if (on) {
            put_key<D>(to, s, j, w, scale, zero);
            if (j == 0)
                reinterpret_cast<int*>(to + P::kPos)[s] =
                    a.positions[static_cast<int64_t>(b) * a.n + i];
        }
        v.get(x);
        beyond |= quantize16(x, w, &scale, &zero);
        if (on) put_value<D>(to, slots + i * kSlotWords<D>, s, j, w, scale, zero);
    }
    __syncthreads();
    if (beyond && a.out_status) a.out_status[u] = kInvalid;     // the first thread has written it
    const int blocks = at + a.n > kPage ? 2 * D : D;
    for (int i = threadIdx.x; i < blocks; i += kThreads) {
        const Block8 blk(i % D);
        const int base = (i / D) * kPage - at;   // the page's first slot, counted in new rows
        uint32_t r[8], fresh = 0;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const int row = base + blk.slot(n);
            r[n] = 0;
            if (row >= 0 && row < a.n) {
                r[n] = slots[row * kSlotWords<D> + blk.j];
                fresh |= 15u << (4 * n);
            }
        }
        if (!fresh) continue;
        transpose8(r);
        uint32_t* codes = reinterpret_cast<uint32_t*>(page[i / D] + P::kValCodes);
#pragma unroll
        for (int g = 0; g < 8; ++g) {
            uint32_t* w = codes + blk.word(g);
            *w = (*w & ~fresh) | r[Block8::nibble(g)];
        }
    }
}

// ---------------------------------------------------------------- compact

// A block per page to fill.  Its slots come from a run of source pages in ascending order (two
// or three where half of the slots are kept).  Of each source page the kept slots are a 64-bit
// mask: D threads turn the page's value codes to slot order and put down the words of those in the
// mask, each behind as many as the mask has before it.  Blocks of 128 threads, so that many are at
// different steps on an SM.
constexpr int kCompactThreads = 128;

template <int D>
__global__ void __launch_bounds__(kCompactThreads) compact_kernel(const CompactArgs a)
{
    using P = PageLayout<D>;
    constexpr int kVecs = P::kRow / 16, kPagesAtOnce = kCompactThreads / D;
    static_assert(kPagesAtOnce >= 1 && kCompactThreads >= kPage * P::kGroups);
    __shared__ PageImage<D> im;
    __shared__ const uint8_t* s_from[kPage];     // page of each slot, and the slot in it
    __shared__ uint8_t s_slot[kPage];
    __shared__ const uint8_t* s_run_page[kPage]; // the run's pages, which of their slots are kept,
    __shared__ uint32_t s_run_mask[kPage][2];    // and the first slot that they go to
    __shared__ int s_run_first[kPage];
    __shared__ unsigned s_changes[2];
    wait_for_previous();
    const int u = blockIdx.y, first = blockIdx.x * kPage;
    const int count = min(kPage, a.lens[u] - first);
    if (count <= 0) return;
    const int* table = a.from.table + static_cast<int64_t>(u) * a.from.max_pages;
    const int* index = a.index ? a.index + static_cast<int64_t>(u) * a.N + first : nullptr;
    const int to = a.to.table[static_cast<int64_t>(u) * a.to.max_pages + blockIdx.x];
    int src = -1;
    const uint8_t* page = nullptr;
    bool change = false;
    if (threadIdx.x < kPage) {
        const int s = threadIdx.x;
        s_run_mask[s][0] = s_run_mask[s][1] = 0;
        if (s < count) {
            src = index ? index[s] : first + s;
            const int before = s == 0 ? -1 : index ? index[s - 1] : first + s - 1;
            change = s == 0 || before / kPage != src / kPage;
            page = a.from.base + static_cast<int64_t>(table[src / kPage]) * P::kBytes;
        }
        s_from[s] = page;
        s_slot[s] = static_cast<uint8_t>(src & (kPage - 1));
        const unsigned changes = __ballot_sync(0xffffffffu, change);
        if (s % 32 == 0) s_changes[s / 32] = changes;
    }
    if (count < kPage)
        for (int i = threadIdx.x; i < kPage * kSlotWords<D>; i += kCompactThreads) im.slots[i] = 0;
    __syncthreads();
    const int runs = __popc(s_changes[0]) + __popc(s_changes[1]);
    if (threadIdx.x < count) {
        const int s = threadIdx.x;
        const int run = (s < 32 ? 0 : __popc(s_changes[0])) +
                        __popc(s_changes[s / 32] & (0xffffffffu >> (31 - s % 32))) - 1;
        if (change) {
            s_run_page[run] = page;
            s_run_first[run] = s;
        }
        atomicOr(&s_run_mask[run][src / 32 % 2], 1u << (src % 32));
    }
    // what is stored by slot
    constexpr int kCopies = kPage * kVecs / kCompactThreads;
    uint4 copy[kCopies];
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
        const int at = threadIdx.x + i * kCompactThreads, s = at / kVecs;
        copy[i] = make_uint4(0, 0, 0, 0);
        if (s < count)
            copy[i] = *reinterpret_cast<const uint4*>(s_from[s] + s_slot[s] * P::kRow +
                                                      at % kVecs * 16);
    }
    uint32_t kg = 0xc3000000u;
    uint16_t vs = 0, vz = 0xc300;
    int pos = -1;
    const int gs = threadIdx.x / P::kGroups, G = threadIdx.x % P::kGroups;
    if (gs < count) {
        const uint8_t* p = s_from[gs];
        const int from = s_slot[gs];
        kg = reinterpret_cast<const uint32_t*>(p + P::kKeyGroups)[from * P::kGroups + G];
        vs = reinterpret_cast<const uint16_t*>(p + P::kValScales)[from * P::kGroups + G];
        vz = reinterpret_cast<const uint16_t*>(p + P::kValZeros)[P::val_zero(G, from)];
        if (G == 0) pos = reinterpret_cast<const int*>(p + P::kPos)[from];
    }
    __syncthreads();
    // value codes, by source page: the next one's are loaded while one is turned
    const Block8 blk(threadIdx.x % D);
    uint32_t ahead[8] = {};
    auto load = [&](int run) {
        const uint32_t* codes = reinterpret_cast<const uint32_t*>(s_run_page[run] + P::kValCodes);
#pragma unroll
        for (int g = 0; g < 8; ++g) ahead[Block8::nibble(g)] = codes[blk.word(g)];
    };
    int run = threadIdx.x / D;
    if (run < runs) load(run);
    for (; run < runs; run += kPagesAtOnce) {
        uint32_t r[8];
#pragma unroll
        for (int n = 0; n < 8; ++n) r[n] = ahead[n];
        if (run + kPagesAtOnce < runs) load(run + kPagesAtOnce);
        const uint32_t low = s_run_mask[run][0], mask = blk.a ? s_run_mask[run][1] : low;
        const int at = s_run_first[run] + (blk.a ? __popc(low) : 0);
        transpose8(r);                       // r[n]: the word of slot(n)
#pragma unroll
        for (int n = 0; n < 4; ++n) {        // slots b and b + 1 of the half page
            const int b = n / 2 * 16 + n % 2 * 8 + 2 * blk.t;
            const uint32_t rest = mask >> b;
            uint32_t* dst = im.slots + (at + __popc(mask & ~(~0u << b))) * kSlotWords<D> + blk.j;
            if (rest & 1) *dst = r[n];
            if (rest & 2) dst[(rest & 1) * kSlotWords<D>] = r[n + 4];
        }
    }
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
        const int at = threadIdx.x + i * kCompactThreads;
        *reinterpret_cast<uint4*>(im.bytes + at / kVecs * P::kRow + at % kVecs * 16) = copy[i];
    }
    if (gs < kPage) {
        reinterpret_cast<uint32_t*>(im.bytes + P::kKeyGroups)[gs * P::kGroups + G] = kg;
        reinterpret_cast<uint16_t*>(im.bytes + P::kValScales)[gs * P::kGroups + G] = vs;
        reinterpret_cast<uint16_t*>(im.bytes + P::kValZeros)[P::val_zero(G, gs)] = vz;
        if (G == 0) reinterpret_cast<int*>(im.bytes + P::kPos)[gs] = pos;
    }
    __syncthreads();
    slots_to_page<D, kCompactThreads>(im);
    __syncthreads();
    store_page<D, kCompactThreads>(im, a.to.base + static_cast<int64_t>(to) * P::kBytes);
}

// ---------------------------------------------------------------- read

// Eight codes as bf16 values s (c - z), one 16-byte store.  The product of the bf16 s and an
// integer below 16 is exact in float32 and rounded once.
__device__ __forceinline__ uint4 decode8(uint32_t word, float scale, float neg_zero)
{
    uint32_t o[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t c = code_pair(word, p);
        o[p] = bf16_pair((bf16_lo(c) + neg_zero) * scale, (bf16_hi(c) + neg_zero) * scale);
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

// A block per page that the rows touch.
template <int D>
__global__ void __launch_bounds__(kThreads) read_kernel(const ReadArgs a)
{
    using P = PageLayout<D>;
    constexpr int kLanes = D / 8;
    __shared__ uint32_t slots[kPage * kSlotWords<D>];
    const int u = blockIdx.y;
    int len = a.lens[u], status = 0;
    if (len < 0 || len > static_cast<int64_t>(a.from.max_pages) * kPage) {
        len = 0;
        status = kInvalid;
    }
    const int first = a.last ? max(0, len - a.rows) : 0;
    const int64_t end = static_cast<int64_t>(first) + a.rows;         // past the last row's slot
    const int* table = a.from.table + static_cast<int64_t>(u) * a.from.max_pages;
    if (blockIdx.x == 0 && a.out_status) {
        bool off = false;
        for (int p = first / kPage + threadIdx.x; p * kPage < min(static_cast<int64_t>(len), end);
             p += kThreads)
            off |= static_cast<unsigned>(table[p]) >= static_cast<unsigned>(a.from.n_pages);
        off = __syncthreads_or(off);
        if (threadIdx.x == 0) a.out_status[u] = off ? kInvalid : status;
    }
    const int64_t base = (static_cast<int64_t>(first / kPage) + blockIdx.x) * kPage;
    if (base >= end) return;
    const uint8_t* page = nullptr;
    if (base < len) {
        const int id = table[base / kPage];
        if (static_cast<unsigned>(id) < static_cast<unsigned>(a.from.n_pages))
            page = a.from.base + static_cast<int64_t>(id) * P::kBytes;
    }
    // everything is loaded before anything is used
    constexpr int kItems = kPage * kLanes / kThreads;
    const int j = threadIdx.x % kLanes, s0 = threadIdx.x / kLanes;
    const Block8 blk(threadIdx.x % D);
    uint32_t r[8], kw[kItems] = {}, kg[kItems] = {};
    uint16_t vs[kItems] = {}, vz[kItems] = {};
    int pos = -1;
    const bool turns = page && threadIdx.x < D;
    if (turns) {
        const uint32_t* codes = reinterpret_cast<const uint32_t*>(page + P::kValCodes);
#pragma unroll
        for (int g = 0; g < 8; ++g) r[Block8::nibble(g)] = codes[blk.word(g)];
    }
    if (page) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int s = s0 + i * (kThreads / kLanes), x = s * P::kGroups + j / 8;
            kw[i] = *reinterpret_cast<const uint32_t*>(page + P::key_word(s, j));
            kg[i] = reinterpret_cast<const uint32_t*>(page + P::kKeyGroups)[x];
            vs[i] = reinterpret_cast<const uint16_t*>(page + P::kValScales)[x];
            vz[i] = reinterpret_cast<const uint16_t*>(page + P::kValZeros)[P::val_zero(j / 8, s)];
        }
        if (threadIdx.x < kPage) pos = reinterpret_cast<const int*>(page + P::kPos)[threadIdx.x];
    }
    if (turns) {
        transpose8(r);
#pragma unroll
        for (int n = 0; n < 8; ++n) slots[blk.slot(n) * kSlotWords<D> + blk.j] = r[n];
    }
    if (threadIdx.x < kPage && a.out_positions) {
        const int64_t slot = base + threadIdx.x, row = slot - first;
        if (row >= 0 && row < a.rows)
            a.out_positions[static_cast<int64_t>(u) * a.rows + row] =
                page && slot < len ? pos : -1;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int s = s0 + i * (kThreads / kLanes);
        const int64_t slot = base + s, row = slot - first;
        if (row < 0 || row >= a.rows) continue;
        uint4 k = {}, v = {};
        if (page && slot < len) {
            k = decode8(kw[i], bf16_lo(kg[i]), bf16_hi(kg[i]));
            v = decode8(slots[s * kSlotWords<D> + j], bf16_lo(vs[i]), bf16_lo(vz[i]));
        }
        const int64_t at = (static_cast<int64_t>(u) * a.rows + row) * D + 8 * j;
        *reinterpret_cast<uint4*>(a.out_keys + at) = k;
        *reinterpret_cast<uint4*>(a.out_values + at) = v;
    }
}

unsigned pages_of(int64_t slots) { return static_cast<unsigned>((slots + kPage - 1) / kPage); }

}  // namespace

cudaError_t launch_index(const IndexArgs& a, cudaStream_t st)
{
    const int64_t vectors = a.mask ? (static_cast<int64_t>(a.N) + 30) / 16 : 1;
    const dim3 grid(static_cast<unsigned>((vectors + kVecChunk - 1) / kVecChunk), a.units);
    index_kernel<<<grid, kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_pack(const PackArgs& a, int d, bool f32, cudaStream_t st)
{
    const dim3 grid(std::min<unsigned>(a.to.max_pages, pages_of(a.N)), a.units);
    if (d == 128)
        return f32 ? launch_dependent(pack_kernel<float, 128>, grid, kThreads, 0, st, a)
                   : launch_dependent(pack_kernel<uint16_t, 128>, grid, kThreads, 0, st, a);
    return f32 ? launch_dependent(pack_kernel<float, 64>, grid, kThreads, 0, st, a)
               : launch_dependent(pack_kernel<uint16_t, 64>, grid, kThreads, 0, st, a);
}

cudaError_t launch_append(const AppendArgs& a, int d, bool f32, cudaStream_t st)
{
    const unsigned grid = static_cast<unsigned>(a.B) * a.H;
    if (d == 128) {
        if (f32) append_kernel<float, 128><<<grid, kThreads, 0, st>>>(a);
        else append_kernel<uint16_t, 128><<<grid, kThreads, 0, st>>>(a);
    } else {
        if (f32) append_kernel<float, 64><<<grid, kThreads, 0, st>>>(a);
        else append_kernel<uint16_t, 64><<<grid, kThreads, 0, st>>>(a);
    }
    return cudaGetLastError();
}

cudaError_t launch_compact(const CompactArgs& a, int d, cudaStream_t st)
{
    const dim3 grid(std::min<unsigned>(a.to.max_pages, pages_of(a.N)), a.units);
    return d == 128 ? launch_dependent(compact_kernel<128>, grid, kCompactThreads, 0, st, a)
                    : launch_dependent(compact_kernel<64>, grid, kCompactThreads, 0, st, a);
}

cudaError_t launch_read(const ReadArgs& a, int d, cudaStream_t st)
{
    // the last rows need not start with a page
    const dim3 grid(pages_of(a.rows) + (a.last ? 1 : 0), a.units);
    if (d == 128) read_kernel<128><<<grid, kThreads, 0, st>>>(a);
    else read_kernel<64><<<grid, kThreads, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace twk
