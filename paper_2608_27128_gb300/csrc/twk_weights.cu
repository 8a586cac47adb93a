// twk_weights.cu -- what attention over prompts pays to each key.
//
//     A(j) = [score(j) +] sum over tokens i that see j, and query heads of the KV head:
//            exp(scale q_i . k_j - lse_i)
//
// The scores are computed again, a tile of 128 keys x 128 (token, head) columns at a time, with the keys
// as the rows of the product: a key's sum is then a thread's, over the columns of its row of the
// accumulator, in one order whatever the grid.  With c = scale log2(e), a weight is
// 2^(c q . k - log2(e) lse): one multiply-add, one exponential and one addition each.
//
// Bound by the tensor cores (2 d operations a pair of key and column) and the exponentials, about alike at
// d = 128; with few tokens (an observation window) by the keys' bytes.  Design (persistent, one block of
// 640 threads per SM):
//   - An item is 256 keys of one KV head, and runs over the columns that see any of them.  The keys stay:
//     they go from TMA's tile through registers to tensor memory, as the products' operand A, so that
//     only the queries are read from shared memory (A from there as well would ask for all of its
//     bandwidth).  Three accumulators of 128 columns take turns.
//   - Warps 0 to 15: a thread per key of the item's halves and half a tile's columns.  Warp 16: TMA.
//     Warp 17: products.  Warp 18: items.  Warp 19: the columns' lse, +inf where a column does not
//     count, which makes its weight 0.  A column's place in shared memory is zero where the tile has
//     none (G does not divide 128).
//   - Work is divided evenly whatever the lengths (twk_prompt.cuh); merge_weights_kernel adds the parts of
//     an item that blocks share, in order.
//
// Measured (us in a graph; TFLOP/s; 32 query heads on 8 KV heads):
//   every token of 16384, d = 128   744   1478: 79 % of the measured burst rate
//   every token of 8192             197   1393, of 4096 61, of 2048 24.4; of 8192 at d = 64 187
//   the last 32 of 16384            16    four items of 256 keys a block at most, one after another: 4300
//                                         cycles each for moving keys, products, sums and their joining
//   six prompts of up to 3001, window of 1024, d = 64   85: at the rate of the unwindowed ones their tiles are 64;
//                                         21 % of a warp's tiles are at an edge, 12 % show it nothing and are
//                                         done all the same (half of them where the sinks stretch an item)
// A unit of two tiles takes about 1750 cycles where exponentials alone take 1050: the warps issue in more than
// half of the cycles, so what surrounds a tile counts (one barrier for a tile's products and lse instead
// of two, rings without phases: 210 -> 202 us on the second line, 209 -> 188 at d = 64).  All sixteen warps
// on one tile, a quarter of the columns each: 258.  The next item's keys moved beside an item's last
// sums: 16.3 -> 15.7 on the third line, 210 -> 218 on the second, for the registers.  One ring for keys and
// queries, with keys of three items on their way: 17.2, the keys are not what items wait for.
#include <atomic>

#include "twk_prompt.cuh"

namespace twk {
namespace {

// Sixteen warps sum, four to a quarter of the SM, half a tile's columns each: eight with whole tiles do not
// cover each other's latencies (235 us for every token of 8192 where these take 207).
constexpr int kSumWarps = 16, kThreads = 32 * (kSumWarps + 4);
constexpr int kLaunchRegs = 96, kHelperRegs = 64, kSumRegs = 104;
static_assert(4 * kHelperRegs + kSumWarps * kSumRegs <= (kSumWarps + 4) * kLaunchRegs,
              "the split draws on the registers of the launch");
constexpr int kPairKeys = 2 * kTileKeys;
constexpr int kAccs = 3, kItemSlots = 4;
// Tiles' lse, a ring for each half.  A tile's lse is written when its accumulator is free, as its products
// start: every tile three and more before it, of either half, is then released.  So the half's tile
// kAccs before it, at least as far back, is released, and the one before that, whose slot is taken, is done.
constexpr int kLogSlots = kAccs + 1;
static_assert((kLogSlots & (kLogSlots - 1)) == 0);

// The tokens that see some key of [j, last]: the first, and the end; of those that count.
__device__ __forceinline__ int2 tokens_of(const PromptArgs& a, const Sequence& s, int j, int last)
{
    int first = max(0, j - (s.m - s.n)), end = s.n;
    if (a.last > 0) first = max(first, s.n - a.last);
    if (a.window > 0 && j >= a.n_sink) end = min(end, last + a.window - (s.m - s.n));
    return make_int2(first, max(first, end));
}

// Items: pairs of key tiles; as long as there are tiles of columns that see them.
struct KeyPairs {
    __device__ static __forceinline__ int items(const PromptArgs&, const Sequence& s)
    {
        return (s.m + kPairKeys - 1) / kPairKeys;
    }
    __device__ static __forceinline__ int2 tokens(const PromptArgs& a, const Sequence& s, int i)
    {
        return tokens_of(a, s, i * kPairKeys, min(i * kPairKeys + kPairKeys, s.m) - 1);
    }
    // beside them an item takes as long as so many tiles (1.7 to 2.1 us, a tile 0.7 to 0.85)
    static constexpr int kMore = 2;
    __device__ static __forceinline__ int length(const PromptArgs& a, const Sequence& s, int i)
    {
        const int2 t = tokens(a, s, i);
        return (t.y - t.x + a.tile_tokens - 1) / a.tile_tokens + kMore;
    }
};

template <int D>
struct Cfg {
    static constexpr int KC = D / 64;
    static constexpr int CHUNK = 128 * 128;
    static constexpr int TILE = KC * CHUNK;
    static constexpr int STAGES = D == 128 ? 4 : 8;       // tiles of queries
    static constexpr int OFF_Q = 2 * TILE;                // behind two tiles of keys
    static constexpr int OFF_LOG = OFF_Q + STAGES * TILE;
    static constexpr int OFF_HALF = OFF_LOG + 2 * kLogSlots * 512;
    static constexpr int OFF_MISC = OFF_HALF + 2 * kTileKeys * 4;
    static constexpr int BYTES = OFF_MISC + 1024 + 1024;  // + 1024 for alignment
    static constexpr int T_K = 0, T_ACC = 128;            // columns of tensor memory
    static_assert(BYTES <= 232448, "shared memory per block");
    static_assert(T_K + D <= T_ACC && T_ACC + kAccs * 128 <= 512);
    static_assert(STAGES * TILE >= kSumsBytes, "the chunks' sums lie there at first");
};

struct Item {
    int t0, i0;              // first row of q of the sequence; first token of the list
    int n, back;             // tokens; m - n, what a token's position is beyond its number
    int j0, j, m;            // first row of k, first key of the item, keys
    int head;                // KV head, -1: no more items
    int u0, u1;              // units of the list that this part takes
    int b[2], e[2];          // those that each half has a part in
    int slot;                // of a part, or -1: the whole item
    int pad;
};
static_assert(sizeof(Item) == 64);

struct Misc {
    uint64_t k_full[2], k_empty[2], kt_full[2], half_full[2], half_empty[2], drain;
    // acc_full: products and lse of a tile; by half and its own count, since a half that skips another's
    // phases would lose track
    uint64_t acc_full[2][kAccs], acc_empty[kAccs];
    uint64_t q_full[8], q_empty[8], item_full[kItemSlots], item_empty[kItemSlots];
    Item items[kItemSlots];
    uint32_t tmem;
    int abort_flag;
};
static_assert(sizeof(Misc) <= 1024);

struct WeightsKernelArgs {
    PromptArgs a;
    float c;                 // scale * log2(e)
    float* part;             // [2 per block][256], null: no item is shared
    int4* join;              // [per block]: parts of the item that begins in the block and ends in
                             // another one (0: none), its first row of k, keys and KV head
    int* err;
    unsigned long long timeout_ns;
};

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_weights_kernel(const __grid_constant__ CUtensorMap tmQ,
                          const __grid_constant__ CUtensorMap tmK,
                          const __grid_constant__ WeightsKernelArgs p)
{
    using C = Cfg<D>;
    const PromptArgs& a = p.a;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    Misc& M = *reinterpret_cast<Misc*>(smem + C::OFF_MISC);
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const int lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&M.k_full[i], 1);
            mbar_init(&M.k_empty[i], 4);
            mbar_init(&M.kt_full[i], 4);
            mbar_init(&M.half_full[i], 4);
            mbar_init(&M.half_empty[i], 4);
        }
        mbar_init(&M.drain, 1);
        for (int i = 0; i < kAccs; ++i) {
            mbar_init(&M.acc_full[0][i], 2);         // the products and the lse
            mbar_init(&M.acc_full[1][i], 2);
            mbar_init(&M.acc_empty[i], 8);
        }
        for (int i = 0; i < C::STAGES; ++i) {
            mbar_init(&M.q_full[i], 1);
            mbar_init(&M.q_empty[i], 1);
        }
        for (int i = 0; i < kItemSlots; ++i) {
            mbar_init(&M.item_full[i], 1);
            mbar_init(&M.item_empty[i], 3 + kSumWarps);      // TMA, products, lse
        }
        M.abort_flag = 0;
        fence_mbarrier_init();
    }
    if (warp == kSumWarps && lane == 0) {
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmK);
    }
    if (warp == kSumWarps + 1) tmem_alloc<1>(&M.tmem, 512);
    wait_for_previous();
    // the chunks' sums lie where queries come later
    long long* sums = reinterpret_cast<long long*>(smem + C::OFF_Q);
    if (a.s.B > 32) sum_chunks<KeyPairs>(a, sums);
    const int tpt = a.tile_tokens, columns = tpt * a.G;
    // columns that no copy writes
    for (int i = threadIdx.x; i < C::STAGES * C::KC * (128 - columns) * 8; i += kThreads) {
        const int chunk = i / ((128 - columns) * 8), r = i - chunk * ((128 - columns) * 8);
        *reinterpret_cast<uint4*>(smem + C::OFF_Q + chunk * C::CHUNK + columns * 128 + r * 16) =
            make_uint4(0, 0, 0, 0);
    }
    fence_async_shared();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = M.tmem;

    WaitCtl wc;
    wc.limit_ns = p.timeout_ns;
    wc.abort_flag = &M.abort_flag;
    wc.err = p.err;
    wc.where = 0;

    if (warp >= kSumWarps) {
        setmaxnreg_dec<kHelperRegs>();
        if (warp == kSumWarps) {
            // ------------------------------------------------------------ TMA
            if (lane == 0) {
                Ring<kItemSlots> ri;
                Ring<C::STAGES> rs;
                uint32_t k_uses[2] = {}, stages = 0;
                const uint32_t q_bytes = static_cast<uint32_t>(columns) * 128u * C::KC;
                bool ok = true;
                while (ok) {
                    if (!(ok = mbar_wait(&M.item_full[ri.slot], ri.phase, wc, 41))) break;
                    const Item it = M.items[ri.slot];
                    mbar_arrive(&M.item_empty[ri.slot]);
                    ri.next();
                    if (it.head < 0) break;
                    int u = it.u1, end = it.u0;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int b = max(it.b[x], it.u0), e = min(it.e[x], it.u1);
                        if (!ok || b >= e) continue;
                        u = min(u, b);
                        end = max(end, e);
                        ok = mbar_wait(&M.k_empty[x], (k_uses[x] & 1u) ^ 1u, wc, 42);
                        if (!ok) continue;
                        ++k_uses[x];
                        mbar_arrive_expect_tx(&M.k_full[x], C::TILE);
#pragma unroll
                        for (int kc = 0; kc < C::KC; ++kc)
                            tma_load_3d(smem + x * C::TILE + kc * C::CHUNK, &tmK, &M.k_full[x],
                                        kc * 64, it.head, it.j0 + it.j + x * kTileKeys);
                    }
                    for (; ok && u < end; ++u) {
                        if (!(ok = mbar_wait(&M.q_empty[rs.slot], rs.phase ^ 1u, wc, 43))) break;
                        mbar_arrive_expect_tx(&M.q_full[rs.slot], q_bytes);
                        uint8_t* dst = smem + C::OFF_Q + rs.slot * C::TILE;
#pragma unroll
                        for (int kc = 0; kc < C::KC; ++kc)
                            tma_load_3d(dst + kc * C::CHUNK, &tmQ, &M.q_full[rs.slot], kc * 64,
                                        it.head * a.G, it.t0 + it.i0 + u * tpt);
                        rs.next();
                        ++stages;
                    }
                }
                // after a give-up: no copy of this thread is in flight when the block ends
                if (!ok) {
                    for (int x = 0; x < 2; ++x)
                        if (k_uses[x]) drain_wait(&M.k_full[x], (k_uses[x] - 1) & 1u, p.timeout_ns);
                    const uint32_t used = min(stages, static_cast<uint32_t>(C::STAGES));
                    for (uint32_t k = 1; k <= used; ++k) {
                        const uint32_t i = stages - k;
                        drain_wait(&M.q_full[i % C::STAGES], i / C::STAGES & 1u, p.timeout_ns);
                    }
                }
            }
        } else if (warp == kSumWarps + 1) {
            // ------------------------------------------------------------ products
            // every lane follows, an elected one issues; what it issues comes from uniform registers
            constexpr uint32_t idesc = umma_idesc_bf16_f32(kTileKeys, 128);
            Ring<kItemSlots> ri;
            Ring<C::STAGES> rs;
            Ring<kAccs> ra, rx[2];
            uint32_t k_uses[2] = {};
            const uint32_t q_low = static_cast<uint32_t>(umma_desc_sw128(smem_u32(smem + C::OFF_Q)));
            bool ok = true;
            while (ok) {
                if (!(ok = all_wait(&M.item_full[ri.slot], ri.phase, wc, 44))) break;
                const Item& it = M.items[ri.slot];
                const int head = __shfl_sync(0xffffffffu, it.head, 0);
                const int u0 = __shfl_sync(0xffffffffu, it.u0, 0);
                const int u1 = __shfl_sync(0xffffffffu, it.u1, 0);
                const int b0 = max(u0, __shfl_sync(0xffffffffu, it.b[0], 0));
                const int b1 = max(u0, __shfl_sync(0xffffffffu, it.b[1], 0));
                const int e0 = min(u1, __shfl_sync(0xffffffffu, it.e[0], 0));
                const int e1 = min(u1, __shfl_sync(0xffffffffu, it.e[1], 0));
                if (lane == 0) mbar_arrive(&M.item_empty[ri.slot]);
                ri.next();
                if (head < 0) break;
                if (b0 < e0) ok = all_wait(&M.kt_full[0], k_uses[0]++ & 1u, wc, 45);
                bool second = false;            // the second half's keys are waited for at their first use
                const int begin = b0 < e0 ? (b1 < e1 ? min(b0, b1) : b0) : b1;
                const int end = b0 < e0 ? (b1 < e1 ? max(e0, e1) : e0) : e1;
                for (int u = begin; ok && u < end; ++u) {
                    if (!(ok = all_wait(&M.q_full[rs.slot], rs.phase, wc, 46))) break;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int b = x ? b1 : b0, e = x ? e1 : e0;
                        if (!ok || u < b || u >= e) continue;
                        if (x == 1 && !second) {
                            if (!(ok = all_wait(&M.kt_full[1], k_uses[1]++ & 1u, wc, 45))) continue;
                            second = true;
                        }
                        if (!(ok = all_wait(&M.acc_empty[ra.slot], ra.phase ^ 1u, wc, 47))) continue;
                        tc_fence_after();
                        if (elect_one()) {
                            umma_tmem_rows<C::KC>(tmem + C::T_ACC + ra.slot * 128,
                                                  tmem + C::T_K + x * (D / 2),
                                                  q_low + rs.slot * (C::TILE >> 4), idesc);
                            umma_commit(&M.acc_full[x][rx[x].slot]);
                        }
                        __syncwarp();
                        ra.next();
                        rx[x].next();
                    }
                    if (!ok) break;
                    if (elect_one()) umma_commit(&M.q_empty[rs.slot]);
                    __syncwarp();
                    rs.next();
                }
            }
            // every product has ended before tensor memory is freed
            __syncwarp();
            if (elect_one()) {
                umma_commit(&M.drain);
                drain_wait(&M.drain, 0, p.timeout_ns);
            }
        } else if (warp == kSumWarps + 2) {
            // ------------------------------------------------------------ items
            Walk<KeyPairs> at;
            at.start(a, sums);
            fence_async_shared();       // the sums have been read
            __syncwarp();
            if (lane == 0) {
                Ring<kItemSlots> ri;
                bool ok = true;
                int4 join = make_int4(0, 0, 0, 0);
                for (; ok && at.more; at.next(a)) {
                    Item it{};
                    const int2 t = KeyPairs::tokens(a, at.s, at.item);
                    it.t0 = at.s.t0;
                    it.i0 = t.x;
                    it.n = at.s.n;
                    it.back = at.s.m - at.s.n;
                    it.j0 = at.s.j0;
                    it.j = at.item * kPairKeys;
                    it.m = at.s.m;
                    it.head = at.head;
                    it.u0 = at.off;
                    it.u1 = at.off + at.take;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int j = it.j + x * kTileKeys;
                        if (j >= it.m) continue;
                        const int2 w = tokens_of(a, at.s, j, min(j + kTileKeys, it.m) - 1);
                        if (w.x >= w.y) continue;
                        it.b[x] = (w.x - t.x) / tpt;
                        it.e[x] = (w.y - t.x + tpt - 1) / tpt;
                    }
                    it.slot = -1;
                    if (at.take < at.length) {
                        // heads and middles in slot 2 c, the item that begins in the block in 2 c + 1
                        it.slot = 2 * static_cast<int>(blockIdx.x) + (at.off == 0 ? 1 : 0);
                        if (at.off == 0)
                            join = make_int4(at.parts(a), it.j0 + it.j, min(kPairKeys, it.m - it.j),
                                             it.head);
                    }
                    ok = mbar_wait(&M.item_empty[ri.slot], ri.phase ^ 1u, wc, 48);
                    if (!ok) break;
                    M.items[ri.slot] = it;
                    mbar_arrive(&M.item_full[ri.slot]);
                    ri.next();
                }
                if (p.join) p.join[blockIdx.x] = join;
                if (ok) ok = mbar_wait(&M.item_empty[ri.slot], ri.phase ^ 1u, wc, 48);
                if (ok) {
                    M.items[ri.slot].head = -1;
                    mbar_arrive(&M.item_full[ri.slot]);
                }
            }
        } else {
            // ------------------------------------------------------------ lse
            if (blockIdx.x == 0 && a.out_status)
                for (int b = lane; b < a.s.B; b += 32)
                    a.out_status[b] = sequence_of(a, b).ok ? TWINKV_OK : TWINKV_ERR_INVALID_ARG;
            Ring<kItemSlots> ri;
            Ring<kAccs> ra, rx[2];
            int log_at[2] = {};
            bool ok = true;
            int token[4], sub[4];                    // of the lane's columns
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                token[k] = (4 * lane + k) / a.G;
                sub[k] = 4 * lane + k - token[k] * a.G;
                if (token[k] >= tpt) token[k] = INT_MAX / 2;
            }
            while (ok) {
                if (!(ok = all_wait(&M.item_full[ri.slot], ri.phase, wc, 49))) break;
                const Item it = M.items[ri.slot];
                __syncwarp();
                if (lane == 0) mbar_arrive(&M.item_empty[ri.slot]);
                ri.next();
                if (it.head < 0) break;
                int u = it.u1, end = it.u0;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int b = max(it.b[x], it.u0), e = min(it.e[x], it.u1);
                    if (b < e) {
                        u = min(u, b);
                        end = max(end, e);
                    }
                }
                auto load = [&](int unit, float (&y)[4]) {
                    const int i = it.i0 + unit * tpt;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        y[k] = token[k] < it.n - i
                                   ? a.lse[static_cast<int64_t>(it.t0 + i + token[k]) * a.s.Hq +
                                           it.head * a.G + sub[k]]
                                   : INFINITY;
                };
                float y[4], next[4];
                if (u < end) load(u, y);
                for (; ok && u < end; ++u) {
                    if (u + 1 < end) load(u + 1, next);
                    constexpr float kLog2e = 1.4426950408889634f;
                    const float4 w =
                        make_float4(-kLog2e * y[0], -kLog2e * y[1], -kLog2e * y[2], -kLog2e * y[3]);
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (!ok || u < max(it.b[x], it.u0) || u >= min(it.e[x], it.u1)) continue;
                        // as the products wait
                        if (!(ok = all_wait(&M.acc_empty[ra.slot], ra.phase ^ 1u, wc, 50))) continue;
                        ra.next();
                        *reinterpret_cast<float4*>(smem + C::OFF_LOG +
                                                   (x * kLogSlots + log_at[x]) * 512 + lane * 16) = w;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&M.acc_full[x][rx[x].slot]);
                        log_at[x] = (log_at[x] + 1) % kLogSlots;
                        rx[x].next();
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[k] = next[k];
                }
            }
        }
        __syncwarp();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (warp == kSumWarps + 1) tmem_dealloc<1>(tmem, 512);
    } else {
        // ------------------------------------------------------------ sums
        setmaxnreg_inc<kSumRegs>();
        // half of the item's keys, half of a tile's columns, quarter of tensor memory
        const int x = warp >> 3, half = warp >> 2 & 1, q = warp & 3;
        const int row = q * 32 + lane;
        const uint32_t base = tmem + (static_cast<uint32_t>(q * 32) << 16);
        Ring<kItemSlots> ri;
        Ring<kAccs> ra, rx;
        int log_at = 0;
        float* halves = reinterpret_cast<float*>(smem + C::OFF_HALF) + x * kTileKeys + row;
        uint32_t k_uses = 0, joins = 0;
        bool ok = true;
        while (ok) {
            if (!(ok = all_wait(&M.item_full[ri.slot], ri.phase, wc, 51))) break;
            const Item& its = M.items[ri.slot];
            const int head = its.head, j0 = its.j0 + its.j, slot = its.slot;
            const int u0 = its.u0, u1 = its.u1;
            const int b = max(u0, x ? its.b[1] : its.b[0]), e = min(u1, x ? its.e[1] : its.e[0]);
            const int ob = max(u0, x ? its.b[0] : its.b[1]), oe = min(u1, x ? its.e[0] : its.e[1]);
            const int held = min(kTileKeys, its.m - its.j - x * kTileKeys);
            // position of the item's first token less the warp's first key, and tokens from it on
            const int gap = its.back + its.i0 - its.j - x * kTileKeys - q * 32;
            const int left = its.n - its.i0;
            const int key = its.j + x * kTileKeys + row;
            __syncwarp();
            if (lane == 0) mbar_arrive(&M.item_empty[ri.slot]);
            ri.next();
            if (head < 0) break;
            const bool mine = b < e, other = ob < oe;
            if (mine && half == 0) {
                // the half's keys: from TMA's tile to operand A, a key to a thread.  The products that
                // read the last ones have ended: their sums are done.
                if (!(ok = all_wait(&M.k_full[x], k_uses++ & 1u, wc, 52))) break;
#pragma unroll
                for (int kc = 0; kc < C::KC; ++kc) {
                    uint32_t w[32];
                    const uint8_t* src = smem + x * C::TILE + kc * C::CHUNK + row * 128;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint4 y = *reinterpret_cast<const uint4*>(src + ((i ^ (row & 7)) * 16));
                        w[4 * i] = y.x, w[4 * i + 1] = y.y, w[4 * i + 2] = y.z, w[4 * i + 3] = y.w;
                    }
                    tmem_st_32x32b_x32(base + C::T_K + x * (D / 2) + 32 * kc, w);
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&M.kt_full[x]);
                    mbar_arrive(&M.k_empty[x]);
                }
            }
            // Accumulators go to the halves in order.  A tile's columns come in two steps of 32: the second one's
            // are on their way while the first is worked on, the next tile's first while the second is.
            float2 l[4] = {};
            float sum = 0.0f;            // what l had every 32 units: short sums of sums
            auto wait_tile = [&] {
                const bool there = all_wait(&M.acc_full[x][rx.slot], rx.phase, wc, 53);
                tc_fence_after();
                return there;
            };
            auto pass = [&](int from, int to) {      // the other half's tiles of units [from, to)
                for (int u = max(from, ob); u < min(to, oe); ++u) ra.next();
            };
            auto add = [&](const uint32_t(&v)[32], const float4* log) {
                const float2 c2 = make_float2(p.c, p.c);
#pragma unroll
                for (int y = 0; y < 32; y += 4) {
                    const float4 t = log[y / 4];
                    const float2 w0 = __ffma2_rn(make_float2(as_f(v[y]), as_f(v[y + 1])), c2,
                                                 make_float2(t.x, t.y));
                    const float2 w1 = __ffma2_rn(make_float2(as_f(v[y + 2]), as_f(v[y + 3])), c2,
                                                 make_float2(t.z, t.w));
                    l[y / 4 % 2] = __fadd2_rn(l[y / 4 % 2],
                                              make_float2(exp2_approx(w0.x), exp2_approx(w0.y)));
                    l[2 + y / 4 % 2] = __fadd2_rn(
                        l[2 + y / 4 % 2], make_float2(exp2_approx(w1.x), exp2_approx(w1.y)));
                }
            };
            if (mine) {
                uint32_t s[2][32];
                if (other) pass(ob, b + x);
                if (!(ok = wait_tile())) break;
                tmem_ld_32x32b_x32(base + C::T_ACC + ra.slot * 128 + half * 64, s[0]);
                for (int u = b; u < e; ++u) {
                    const int p0 = gap + u * tpt;         // first token's position less the warp's first key
                    const int rest = left - u * tpt;      // tokens from it on
                    const bool edge = p0 < 31 || rest < tpt ||
                                      (a.window > 0 && p0 + tpt - 1 >= a.window);
                    // columns [lo, hi) see the thread's key: those of the tokens from its own on, as far
                    // as the window reaches
                    uint32_t see[2] = {~0u, ~0u};
                    if (edge) {
                        const int lo = min(max(lane - p0, 0), 128) * a.G;
                        int hi = min(rest, tpt);
                        if (a.window > 0 && key >= a.n_sink) hi = min(hi, lane + a.window - p0);
                        hi = max(hi, 0) * a.G;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int first = 64 * half + 32 * i;
                            see[i] = bits_below(hi - first) & ~bits_below(lo - first);
                        }
                    }
                    const float4* log = reinterpret_cast<const float4*>(smem + C::OFF_LOG +
                                                                        (x * kLogSlots + log_at) * 512 +
                                                                        half * 256);
                    [[maybe_unused]] bool there = true;   // the next tile, if any, is on its way
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        tmem_wait_ld();
                        reg_fence(s[i]);
                        if (i == 0) {
                            tmem_ld_32x32b_x32(base + C::T_ACC + ra.slot * 128 + half * 64 + 32, s[1]);
                        } else {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) mbar_arrive(&M.acc_empty[ra.slot]);
                            ra.next();
                            rx.next();
                            log_at = (log_at + 1) % kLogSlots;
                            if (u + 1 < e) {
                                if (u + x >= ob && u + x < oe) ra.next();       // the other half's tile
                                // d = 128: not waited for before this one's last columns are done (16384
                                // tokens 765 -> 747 us; at d = 64, whose products are short, 8192: 187 -> 199)
                                if constexpr (D == 128) {
                                    there = __all_sync(0xffffffffu, mbar_test(smem_u32(&M.acc_full[x][rx.slot]),
                                                                              rx.phase));
                                    if (there) {
                                        tc_fence_after();
                                        tmem_ld_32x32b_x32(base + C::T_ACC + ra.slot * 128 + half * 64, s[0]);
                                    }
                                } else {
                                    if (!(ok = wait_tile())) break;
                                    tmem_ld_32x32b_x32(base + C::T_ACC + ra.slot * 128 + half * 64, s[0]);
                                }
                            }
                        }
                        if (edge) {
#pragma unroll
                            for (int y = 0; y < 32; ++y)
                                s[i][y] = see[i] >> y & 1u ? s[i][y] : 0xff800000u;
                        }
                        add(s[i], log + 8 * i);
                    }
                    if constexpr (D == 128) {
                        if (!there) {
                            if (!(ok = wait_tile())) break;
                            tmem_ld_32x32b_x32(base + C::T_ACC + ra.slot * 128 + half * 64, s[0]);
                        }
                    }
                    if (!ok) break;
                    if ((u & 31) == 31) {
                        const float2 l2 = __fadd2_rn(__fadd2_rn(l[0], l[1]), __fadd2_rn(l[2], l[3]));
                        sum += l2.x + l2.y;
#pragma unroll
                        for (int i = 0; i < 4; ++i) l[i] = make_float2(0.0f, 0.0f);
                    }
                }
                if (!ok) break;
                if (other) pass(e - 1 + x, oe);
            } else if (other) {
                pass(ob, oe);
            }
            const float2 l2 = __fadd2_rn(__fadd2_rn(l[0], l[1]), __fadd2_rn(l[2], l[3]));
            sum += l2.x + l2.y;
            // the two halves of the columns, in order
            if (half == 1) {
                if (!(ok = all_wait(&M.half_empty[x], (joins++ & 1u) ^ 1u, wc, 55))) break;
                *halves = sum;
                __syncwarp();
                if (lane == 0) mbar_arrive(&M.half_full[x]);
                continue;
            }
            if (!(ok = all_wait(&M.half_full[x], joins++ & 1u, wc, 56))) break;
            sum += *halves;
            __syncwarp();
            if (lane == 0) mbar_arrive(&M.half_empty[x]);
            if (slot >= 0) {
                p.part[slot * kPairKeys + x * kTileKeys + row] = sum;
            } else if (row < held) {
                const int64_t at = static_cast<int64_t>(head) * a.s.keys + j0 + x * kTileKeys + row;
                a.out_score[at] = a.score ? a.score[at] + sum : sum;
            }
        }
        tc_fence_before();
        __syncthreads();
    }
}

// Adds the parts of an item that several blocks took, in order: a block per block that one begins in.
__global__ void __launch_bounds__(kPairKeys)
    merge_weights_kernel(const __grid_constant__ WeightsKernelArgs p)
{
    wait_for_previous();
    const int4 join = p.join[blockIdx.x];
    if (static_cast<int>(threadIdx.x) >= join.z || join.x == 0) return;
    float sum = p.part[(2 * blockIdx.x + 1) * kPairKeys + threadIdx.x];
#pragma unroll 8
    for (int k = 1; k < join.x; ++k)
        sum += p.part[2 * (blockIdx.x + k) * kPairKeys + threadIdx.x];
    const int64_t at = static_cast<int64_t>(join.w) * p.a.s.keys + join.y + threadIdx.x;
    p.a.out_score[at] = p.a.score ? p.a.score[at] + sum : sum;
}

// An item that no more tokens than this look at is never cut.
int whole_tokens(const PromptArgs& a) { return (2 * kSnap + 1 - KeyPairs::kMore) * a.tile_tokens; }

template <int D>
cudaError_t launch(const PromptArgs& a, int sms, const WaitFacts& w, cudaStream_t st)
{
    using C = Cfg<D>;
    static std::atomic<bool> allowed[64];     // by device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev >= 64 || !allowed[dev].load(std::memory_order_relaxed)) {
        // the warpgroups' shares add up to the launch's registers: with fewer, waits for them have no end
        cudaFuncAttributes f;
        if ((e = cudaFuncGetAttributes(&f, prompt_weights_kernel<D>)) != cudaSuccess) return e;
        if (f.numRegs < kLaunchRegs) return cudaErrorInvalidConfiguration;
        e = cudaFuncSetAttribute(prompt_weights_kernel<D>,
                                 cudaFuncAttributeMaxDynamicSharedMemorySize, C::BYTES);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
    }
    CUtensorMap q, k;
    if (!encode_rows(&q, a.q, D, a.s.Hq, a.s.tokens, a.s.q_head, a.s.q_token, a.G, a.tile_tokens) ||
        !encode_rows(&k, a.k, D, a.s.H, a.s.keys, a.s.k_head, a.s.k_token, 1, kTileKeys))
        return cudaErrorInvalidValue;
    WeightsKernelArgs p{};
    p.a = a;
    p.a.snap = kSnap;
    p.c = a.scale * 1.4426950408889634f;
    const int tokens = a.last > 0 ? std::min(a.last, a.s.tokens) : a.s.tokens;
    const bool shared = tokens > whole_tokens(a);
    if (shared) {
        p.join = static_cast<int4*>(a.ws);
        p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(a.ws) + 16 * kPromptBlocks);
    }
    p.err = w.err;
    p.timeout_ns = w.timeout_ns;
    const int grid = std::min(sms, kPromptBlocks);
    prompt_weights_kernel<D><<<grid, kThreads, C::BYTES, st>>>(q, k, p);
    if ((e = cudaGetLastError()) != cudaSuccess || !shared) return e;
    return launch_dependent(merge_weights_kernel, dim3(grid), kPairKeys, 0, st, p);
}

}  // namespace

size_t prompt_weights_workspace(const twinkv_prompt&)
{
    return 16 * kPromptBlocks + 2 * kPromptBlocks * kPairKeys * sizeof(float);
}

cudaError_t launch_prompt_weights(const PromptArgs& a, int sms, const WaitFacts& w, cudaStream_t st)
{
    return a.s.d == 128 ? launch<128>(a, sms, w, st) : launch<64>(a, sms, w, st);
}

}  // namespace twk
