// twk_prompt.cu -- attention over prompts.
//
// Per token at position p = m - n + i of its sequence and query head:
//     o = sum_j exp(x_j - lse) v_j,   x_j = scale q . k_j,   lse = log sum_j exp(x_j)
// over the keys j <= p and, with a window W, of those p - j < W or j < n_sink.
//
// One pass over the keys, a tile of 128 at a time, with a running maximum and sum per row: with
// c = scale log2(e) and t the row's top, about the largest c q . k so far,
//     p_j = 2^(c q . k_j - t),   l = sum p_j,   O = sum p_j v_j,   o = O / l,   lse = ln2 t + ln l.
// The top is the maximum of the row's first tile, and follows later ones only where a tile's sum of
// probabilities shows that it is far behind them (2^15: floats and bf16 do not notice such factors, and
// the sum of 128 probabilities stays below it else): the tile's maximum is found, O scaled in tensor
// memory and the tile done again, a rare event.  So a tile costs no maximum (a fifth of the softmax's
// instructions at d = 64).
//
// t is rounded, by 2^-24 of itself: a factor that the row's probabilities have in common, and that its sum and lse
// take out again, as long as it is about 1.  A row's top is kept as the q . k that it comes from, and where one
// of a warp's is beyond 2^12 in units of log 2 (kLarge) the difference is taken first, p_j = 2^(c (q . k_j - top)),
// which is right for scores of any size; every tile then has its maximum found.
//
// Bound by the tensor cores at d = 128: 4 d operations for each pair of a row and a key, of which a prompt of
// n tokens has n^2 / 2 per head; an exponential for each (4 cycles a warp) takes half their time there, and
// as long at d = 64.  There no pipe is above 41 % and an instruction issues in 39 % of the cycles: latency bounds
// it, two softmax warps to a quarter of the SM, each in a chain of load, exponentials, store and wait.  Design
// (persistent, one block of 384 threads per SM):
//   - An item is 256 query rows of one KV head: (token, head) pairs, the heads of a token side by side,
//     so that every head of the group reads the same keys, and short sequences fill a tile.  Two
//     tiles of 128 rows take turns: one's softmax runs beside the other's products.
//   - S = Q K^T by tcgen05.mma from shared memory, both K-major; P (bf16, in tensor memory) times V, whose
//     rows run along the keys: operand A from tensor memory, B as TMA left it.
//   - Warps 0 to 3 and 4 to 7: softmax, a thread per row.  Warp 8: TMA (queries once per item, then keys
//     and values in one ring).  Warp 9 issues the products, warp 11 those with V at d = 64 (Cfg).  Warp 10
//     hands out items.
//   - Work is divided evenly whatever the lengths (twk_prompt.cuh): a block's span may begin and end inside
//     an item, whose parts (unnormalised O, top, l in float32) merge_kernel joins in order.
//
// Measured (us in a graph; TFLOP/s; 32 query heads on 8 KV heads), before and after what is named:
//   16384 tokens, d = 128   1370   1605: 85 % of the measured burst rate, 95 % of the sustained (1474 us
//                           from call to call, under the power limit)
//   4096 tokens, d = 128     116   1180; 2048: 44.5 us, 1024: 21; 101: 9.0, most of it the start and the end
//   256 tokens over 65536    185   1483, items cut into 5 parts (199 us from call to call)
//   16384 tokens, d = 64     862   1275; 12 packed prompts of 752 to 3001 tokens 246, 858
//   descriptors in uniform registers: 2095 -> 1451 on the first line
//   cutting by tiles and what an item takes beside them, instead of by tiles: 305 -> 255 on the last
//   tops kept as q . k, for scores of any size: 1404 -> 1379 on the first, 843 -> 861 and 252 -> 246 on the last
#include <atomic>

#include "twk_cache.cuh"
#include "twk_internal.h"
#include "twk_prompt.cuh"
#include "twk_ptx.cuh"

namespace twk {
namespace {

constexpr int kThreads = 384;
constexpr int kLaunchRegs = 168, kHelperRegs = 88, kSoftmaxRegs = 208;
static_assert(4 * kHelperRegs + 8 * kSoftmaxRegs <= 12 * kLaunchRegs,
              "the split draws on the registers of the launch");
constexpr int kPairRows = 2 * kTileRows;
constexpr float kFar = 0x1p15f;          // sum of a tile's probabilities from which the top follows
constexpr float kLarge = 0x1p12f;        // |c top| up to which c top enters rounded

// Items of attention: pairs of row tiles; as long as their list of key tiles.
struct RowPairs {
    __device__ static __forceinline__ int items(const PromptArgs& a, const Sequence& s)
    {
        const int tokens = 2 * a.tile_tokens;
        return (s.n + tokens - 1) / tokens;
    }
    __device__ static __forceinline__ KeyTiles tiles(const PromptArgs& a, const Sequence& s, int i)
    {
        const int tokens = 2 * a.tile_tokens, first = s.m - s.n + i * tokens;
        return key_tiles(a, first, min(first + tokens, s.m) - 1);
    }
    // beside them an item takes as long as so many tiles (its start, masks and rows: 2.3 to 3 us, a tile 0.9 at
    // d = 64; 1.4 and 1.5 at d = 128)
    __device__ __host__ static constexpr int more(int d) { return d == 64 ? 3 : 1; }
    __device__ static __forceinline__ int length(const PromptArgs& a, const Sequence& s, int i)
    {
        return tiles(a, s, i).count + more(a.s.d);
    }
};

template <int D>
struct Cfg {
    static constexpr int KC = D / 64;                     // chunks of 128 bytes of a row
    static constexpr int CHUNK = kTileRows * 128;
    static constexpr int Q_BYTES = KC * CHUNK;            // a tile of queries
    static constexpr int STAGE = KC * CHUNK;              // a tile of keys or values
    static constexpr int STAGES = D == 128 ? 4 : 8;
    static constexpr int OFF_KV = 2 * Q_BYTES;
    static constexpr int OFF_OUT = OFF_KV + STAGES * STAGE;     // a warp's rows, 128 bytes of each
    static constexpr int OFF_MISC = OFF_OUT + 8 * 32 * 128;
    static constexpr int BYTES = OFF_MISC + 1024 + 1024;  // + 1024 for alignment
    // Columns of tensor memory, of tile 0.  At d = 128 the probabilities take the scores' place, and the next
    // scores come after their products.  At d = 64 there is room beside them: the next scores come as soon
    // as the softmax has the last ones in registers, and are there when it is done.  Scores and outputs are
    // then issued by a warp each: what a warp does around its products takes longer than they do
    // (16384 tokens, one warp and one place: 1075 us; two warps and places: 899).
    static constexpr bool EARLY = D == 64;
    static constexpr int T_S = 0, T_P = EARLY ? 256 : 0, P_STRIDE = EARLY ? 64 : kTileKeys;
    static constexpr int T_O = EARLY ? 384 : 256;
    static_assert(T_O + 2 * D <= 512);
    static_assert(STAGES % 2 == 0, "keys in even stages, values in odd ones");
    static_assert(BYTES <= 232448, "shared memory per block");
    static_assert(STAGES * STAGE >= kSumsBytes, "the chunks' sums lie there at first");
};

constexpr int kItemSlots = 4;

// What the roles have to know of an item's part.
struct Item {
    int t0, tokens;          // first row of q, tokens from there to the sequence's end (for both tiles)
    int pos;                 // position of the first token
    int j0, m, head;         // keys; KV head, -1: no more items
    int s0, s1;              // units of the list that this part takes
    int count[2];            // length of each tile's list
    int sinks, from;         // see KeyTiles
    int slot;                // part's slot, or -1: the whole item
    int pad[3];
};
static_assert(sizeof(Item) == 64);

struct Misc {
    uint64_t q_full[2], q_empty[2], s_full[2], s_free[2], p_full[2], o_full[2], drain[2];
    uint64_t kv_full[8], kv_empty[8], item_full[kItemSlots], item_empty[kItemSlots];
    Item items[kItemSlots];
    uint32_t tmem;
    int abort_flag;
};
static_assert(sizeof(Misc) <= 1024);

struct AttendKernelArgs {
    PromptArgs a;
    float c;                 // scale * log2(e)
    float* part;             // [2 per block] parts, null: no item is shared
    int4* join;              // [per block]: parts of the item that begins in the block and ends in
                             // another one (0: none), its t0, tokens and KV head
    int* err;
    unsigned long long timeout_ns;
};

// A part: outputs [D / 4][256 rows][4], tops [256], sums [256].
template <int D>
constexpr int kPartFloats = kPairRows * (D + 2);

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// c (x - y) of two tops (-inf: none yet), with their products rounded as they enter the probabilities.
__device__ __forceinline__ float top_gap(float x, float y, float c)
{
    const float u = __fmul_rn(x, c), v = __fmul_rn(y, c);
    return fabsf(u) <= kLarge && fabsf(v) <= kLarge ? u - v : (x - y) * c;
}

// The logarithm of a row's denominator.
__device__ __forceinline__ float log_sum(float top, float sum, float c, float scale)
{
    if (!(sum > 0.0f)) return -INFINITY;
    const float t = __fmul_rn(top, c);
    return fabsf(t) <= kLarge ? fmaf(t, 0.6931471805599453f, logf(sum)) : fmaf(top, scale, logf(sum));
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_attend_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                         const __grid_constant__ CUtensorMap tmV,
                         const __grid_constant__ AttendKernelArgs p)
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
            mbar_init(&M.q_full[i], 1);
            mbar_init(&M.q_empty[i], 1);
            mbar_init(&M.s_full[i], 1);
            mbar_init(&M.s_free[i], 4);
            mbar_init(&M.p_full[i], 4);
            mbar_init(&M.drain[i], 1);
            mbar_init(&M.o_full[i], 1);
        }
        for (int i = 0; i < C::STAGES; ++i) {
            mbar_init(&M.kv_full[i], 1);
            mbar_init(&M.kv_empty[i], 1);
        }
        for (int i = 0; i < kItemSlots; ++i) {
            mbar_init(&M.item_full[i], 1);
            mbar_init(&M.item_empty[i], C::EARLY ? 11 : 10);      // TMA, products, eight of softmax
        }
        M.abort_flag = 0;
        fence_mbarrier_init();
    }
    if (warp == 8 && lane == 0) {
        prefetch_tensormap(&tmQ);
        prefetch_tensormap(&tmK);
        prefetch_tensormap(&tmV);
    }
    if (warp == 9) tmem_alloc<1>(&M.tmem, 512);
    wait_for_previous();
    // the chunks' sums lie where keys and values come later
    long long* sums = reinterpret_cast<long long*>(smem + C::OFF_KV);
    if (a.s.B > 32) sum_chunks<RowPairs>(a, sums);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = M.tmem;

    WaitCtl wc;
    wc.limit_ns = p.timeout_ns;
    wc.abort_flag = &M.abort_flag;
    wc.err = p.err;
    wc.where = 0;
    const int tpt = a.tile_tokens;

    if (warp >= 8) {
        setmaxnreg_dec<kHelperRegs>();
        if (warp == 8) {
            // ------------------------------------------------------------ TMA
            if (lane == 0) {
                Ring<kItemSlots> ri;
                Ring<C::STAGES> rs;
                uint32_t q_uses[2] = {}, stages = 0;
                const uint32_t q_bytes = static_cast<uint32_t>(tpt * a.G) * 128u * C::KC;
                bool ok = true;
                auto load = [&](const CUtensorMap* map, const Item& it, int tile) {
                    if (!(ok = mbar_wait(&M.kv_empty[rs.slot], rs.phase ^ 1u, wc, 21))) return;
                    mbar_arrive_expect_tx(&M.kv_full[rs.slot], C::STAGE);
                    uint8_t* dst = smem + C::OFF_KV + rs.slot * C::STAGE;
#pragma unroll
                    for (int kc = 0; kc < C::KC; ++kc)
                        tma_load_3d(dst + kc * C::CHUNK, map, &M.kv_full[rs.slot], kc * 64, it.head,
                                    it.j0 + tile * kTileKeys);
                    rs.next();
                    ++stages;
                };
                for (;;) {
                    if (!(ok = mbar_wait(&M.item_full[ri.slot], ri.phase, wc, 22))) break;
                    const Item it = M.items[ri.slot];
                    mbar_arrive(&M.item_empty[ri.slot]);
                    ri.next();
                    if (it.head < 0) break;
                    const KeyTiles kt{it.sinks, it.from, 0};
                    // the queries of a tile that has products, then the first keys
                    for (int x = 0; x < 2 && ok; ++x) {
                        if (min(it.s1, it.count[x]) <= it.s0) continue;
                        ok = mbar_wait(&M.q_empty[x], (q_uses[x] & 1u) ^ 1u, wc, 23);
                        if (!ok) break;
                        ++q_uses[x];
                        mbar_arrive_expect_tx(&M.q_full[x], q_bytes);
#pragma unroll
                        for (int kc = 0; kc < C::KC; ++kc)
                            tma_load_3d(smem + x * C::Q_BYTES + kc * C::CHUNK, &tmQ, &M.q_full[x],
                                        kc * 64, it.head * a.G, it.t0 + x * tpt);
                    }
                    const int n = min(it.s1, max(it.count[0], it.count[1]));
                    for (int j = it.s0; j < n && ok; ++j) {
                        load(&tmK, it, kt.tile(j));
                        if (ok) load(&tmV, it, kt.tile(j));
                    }
                    if (!ok) break;
                }
                // after a give-up: no copy of this thread is in flight when the block ends
                if (!ok) {
                    for (int x = 0; x < 2; ++x)
                        if (q_uses[x]) drain_wait(&M.q_full[x], (q_uses[x] - 1) & 1u, p.timeout_ns);
                    const uint32_t used = min(stages, static_cast<uint32_t>(C::STAGES));
                    for (uint32_t k = 1; k <= used; ++k) {
                        const uint32_t i = stages - k;
                        drain_wait(&M.kv_full[i % C::STAGES], i / C::STAGES & 1u, p.timeout_ns);
                    }
                }
            }
        } else if (warp == 9 || (C::EARLY && warp == 11)) {
            // ------------------------------------------------------------ products
            // Every lane follows, an elected one issues.  What the descriptors and the loops depend on comes
            // from shuffles and votes, so that the compiler knows it to be the same in all lanes and keeps it
            // in uniform registers: an instruction took 80 cycles to issue where it did not.
            constexpr uint32_t id_s = umma_idesc_bf16_f32(kTileRows, kTileKeys);
            constexpr uint32_t id_o = umma_idesc_bf16_f32(kTileRows, D) | kIdescBRows;
            Ring<kItemSlots> ri;
            const uint32_t q_low = static_cast<uint32_t>(umma_desc_sw128(smem_u32(smem)));
            const uint32_t k_low = static_cast<uint32_t>(umma_desc_sw128(smem_u32(smem + C::OFF_KV)));
            const uint32_t v_low =
                static_cast<uint32_t>(umma_desc_sw128_rows(smem_u32(smem + C::OFF_KV), C::CHUNK));
            auto scores = [&](int x, uint32_t stage) {
                umma_rows<C::KC>(tmem + C::T_S + x * kTileKeys, q_low + x * (C::Q_BYTES >> 4),
                                 k_low + stage * (C::STAGE >> 4), id_s);
                umma_commit(&M.s_full[x]);
            };
            auto outputs = [&](int x, uint32_t stage, uint32_t add) {
                umma_tmem_128(tmem + C::T_O + x * D, tmem + C::T_P + x * C::P_STRIDE,
                              v_low + stage * (C::STAGE >> 4), id_o, add);
            };
            bool ok = true;
            // an item with products: its list's units [s0, all), of which tile x takes those below n[x]
            struct Part {
                int s0, n[2], all, last;        // last: the last tile that has any
                int m;
                KeyTiles kt;
            };
            auto fetch = [&](Part& f) {         // all = s0: there are no more
                for (;;) {
                    f.s0 = f.all = 0;
                    if (!(ok = all_wait(&M.item_full[ri.slot], ri.phase, wc, 24))) return;
                    const Item& it = M.items[ri.slot];
                    const int head = __shfl_sync(0xffffffffu, it.head, 0);
                    const int s1 = __shfl_sync(0xffffffffu, it.s1, 0);
                    f.s0 = __shfl_sync(0xffffffffu, it.s0, 0);
                    f.n[0] = min(s1, __shfl_sync(0xffffffffu, it.count[0], 0));
                    f.n[1] = min(s1, __shfl_sync(0xffffffffu, it.count[1], 0));
                    f.kt = KeyTiles{__shfl_sync(0xffffffffu, it.sinks, 0),
                                    __shfl_sync(0xffffffffu, it.from, 0), 0};
                    f.m = __shfl_sync(0xffffffffu, it.m, 0);
                    if (lane == 0) mbar_arrive(&M.item_empty[ri.slot]);
                    ri.next();
                    f.last = f.n[1] > f.s0 ? 1 : 0;
                    f.all = head < 0 ? f.s0 : max(f.s0, max(f.n[0], f.n[1]));
                    if (head < 0 || f.all > f.s0) return;
                }
            };
            // where the sequence ends inside the tile its probabilities are 0 from there on, and so are the
            // values, whatever lies behind it
            auto end_values = [&](int held, uint32_t stage) {
                if (held >= kTileKeys) return;
                uint8_t* v = smem + C::OFF_KV + stage * C::STAGE;
                for (int y = held * 128 + lane * 16; y < C::CHUNK; y += 512)
#pragma unroll
                    for (int kc = 0; kc < C::KC; ++kc)
                        *reinterpret_cast<uint4*>(v + kc * C::CHUNK + y) = make_uint4(0, 0, 0, 0);
                fence_async_shared();
                __syncwarp();
            };
            Part f;
            if constexpr (C::EARLY) {
                Ring<C::STAGES / 2> rs;          // even stages for scores, odd ones for outputs
                uint32_t uses[2] = {}, q_uses[2] = {};
                if (warp == 9) {
                    for (fetch(f); ok && f.all > f.s0; fetch(f)) {
                        for (int j = f.s0; ok && j < f.all; ++j) {
                            const uint32_t stage = 2 * rs.slot;
                            if (!(ok = all_wait(&M.kv_full[stage], rs.phase, wc, 25))) break;
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                if (!ok || j >= f.n[x]) continue;
                                if (j == f.s0) ok = all_wait(&M.q_full[x], q_uses[x]++ & 1u, wc, 26);
                                if (ok) ok = all_wait(&M.s_free[x], (uses[x]++ & 1u) ^ 1u, wc, 37);
                                if (!ok) continue;
                                tc_fence_after();
                                if (elect_one()) {
                                    scores(x, stage);
                                    if (j + 1 == f.n[x]) umma_commit(&M.q_empty[x]);
                                    if (x == f.last) umma_commit(&M.kv_empty[stage]);
                                }
                                __syncwarp();
                            }
                            // the second tile's last unit may be past the first's, not the other way round
                            rs.next();
                        }
                        if (!ok) break;
                    }
                } else {
                    for (fetch(f); ok && f.all > f.s0; fetch(f)) {
                        for (int j = f.s0; ok && j < f.all; ++j) {
                            const uint32_t stage = 2 * rs.slot + 1;
                            if (!(ok = all_wait(&M.kv_full[stage], rs.phase, wc, 27))) break;
                            end_values(f.m - f.kt.tile(j) * kTileKeys, stage);
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                if (!ok || j >= f.n[x]) continue;
                                if (!(ok = all_wait(&M.p_full[x], uses[x]++ & 1u, wc, 29))) continue;
                                tc_fence_after();
                                if (elect_one()) {
                                    outputs(x, stage, j != f.s0);
                                    umma_commit(&M.o_full[x]);
                                    if (x == f.last) umma_commit(&M.kv_empty[stage]);
                                }
                                __syncwarp();
                            }
                            rs.next();
                        }
                        if (!ok) break;
                    }
                }
            } else {
                Ring<C::STAGES> rs;
                uint32_t q_uses[2] = {}, p_uses[2] = {};
                // the scores of the item's first unit by tile x
                auto first_scores = [&](const Part& f, int x) {
                    if (!ok || f.n[x] <= f.s0) return;
                    ok = all_wait(&M.kv_full[rs.slot], rs.phase, wc, 25) &&
                         all_wait(&M.q_full[x], q_uses[x]++ & 1u, wc, 26);
                    if (!ok) return;
                    tc_fence_after();
                    if (elect_one()) {
                        scores(x, rs.slot);
                        if (f.s0 + 1 == f.n[x]) umma_commit(&M.q_empty[x]);
                        if (x == f.last) umma_commit(&M.kv_empty[rs.slot]);
                    }
                };
                Part g;
                fetch(f);
                if (ok && f.all > f.s0) {
                    first_scores(f, 0);
                    first_scores(f, 1);
                    rs.next();
                }
                while (ok && f.all > f.s0) {
                    for (int j = f.s0; j < f.all; ++j) {
                        const Ring<C::STAGES> rv = rs;
                        rs.next();
                        const bool end = j + 1 == f.all;
                        if (!(ok = all_wait(&M.kv_full[rv.slot], rv.phase, wc, 27))) break;
                        if (!end && !(ok = all_wait(&M.kv_full[rs.slot], rs.phase, wc, 30))) break;
                        end_values(f.m - f.kt.tile(j) * kTileKeys, rv.slot);
                        if (end) {
                            fetch(g);
                            if (!ok) break;
                        }
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            if (ok && j < f.n[x]) {
                                ok = all_wait(&M.p_full[x], p_uses[x]++ & 1u, wc, 29);
                                if (ok) tc_fence_after();
                                if (ok && elect_one()) {
                                    outputs(x, rv.slot, j != f.s0);
                                    if (j + 1 < f.n[x]) {
                                        scores(x, rs.slot);
                                        if (j + 2 == f.n[x]) umma_commit(&M.q_empty[x]);
                                    } else {
                                        umma_commit(&M.o_full[x]);
                                    }
                                    if (x == f.last) {
                                        umma_commit(&M.kv_empty[rv.slot]);
                                        if (!end) umma_commit(&M.kv_empty[rs.slot]);
                                    }
                                }
                                __syncwarp();
                            }
                            // the next item's first scores, while the softmax of this one's last unit runs
                            if (end && g.all > g.s0) first_scores(g, x);
                        }
                        if (!ok) break;
                        if (!end || g.all > g.s0) rs.next();
                    }
                    f = g;
                }
            }
            // every product has ended before tensor memory is freed
            __syncwarp();
            if (elect_one()) {
                umma_commit(&M.drain[warp == 9 ? 0 : 1]);
                drain_wait(&M.drain[warp == 9 ? 0 : 1], 0, p.timeout_ns);
            }
        } else if (warp == 10) {
            // ------------------------------------------------------------ items
            // d = 64 ran 12 % slower with the code of a second start in the kernel (16384 tokens: 938 us, not
            // 844); why is not known: code, registers or their scheduling
            Walk<RowPairs, D == 128> at;
            at.start(a, sums);
            fence_async_shared();       // the sums have been read
            __syncwarp();
            if (lane == 0) {
                Ring<kItemSlots> ri;
                bool ok = true;
                int4 join = make_int4(0, 0, 0, 0);
                for (; ok && at.more; at.next(a)) {
                    Item it{};
                    const int i0 = at.item * 2 * tpt;
                    it.t0 = at.s.t0 + i0;
                    it.tokens = at.s.n - i0;
                    it.pos = at.s.m - at.s.n + i0;
                    it.j0 = at.s.j0;
                    it.m = at.s.m;
                    it.head = at.head;
                    it.s0 = at.off;
                    it.s1 = at.off + at.take;
                    const KeyTiles kt = RowPairs::tiles(a, at.s, at.item);
                    it.sinks = kt.sinks;
                    it.from = kt.from;
                    for (int x = 0; x < 2; ++x) {
                        // the same list, as far as the tile's last token sees
                        const int last = min(it.pos + (x + 1) * tpt, it.m) - 1;
                        const bool any = it.tokens > x * tpt && last >= 0;
                        it.count[x] = any ? kt.sinks + last / kTileKeys + 1 - kt.from : 0;
                    }
                    it.slot = -1;
                    if (at.take < at.length) {
                        // heads and middles in slot 2 c, the item that begins in the block in 2 c + 1
                        it.slot = 2 * static_cast<int>(blockIdx.x) + (at.off == 0 ? 1 : 0);
                        if (at.off == 0) join = make_int4(at.parts(a), it.t0, it.tokens, it.head);
                        // Items longer than a span: those of a head read the same keys at the same time, or
                        // L2 would not hold them until the next one does (256 tokens over 65536: 198 ->
                        // 185 us; at d = 64 packed prompts lose what it gains there).  What one visits after t units of
                        // the span is, in tiles, t modulo the span's length: a part begins inside and ends
                        // with what is before.  Its list is then tiles [first + r, end), [first, first + r).
                        if constexpr (D == 128) {
                            const int tiles = min(it.s1, min(it.count[0], it.count[1]));
                            if (at.length > at.each && it.s0 >= kt.sinks &&
                                tiles == min(it.s1, max(it.count[0], it.count[1]))) {
                                const int shift = kt.from - kt.sinks;
                                const int first = it.s0 + shift, end = tiles + shift;
                                const int r = at.turn(first);
                                if (r < end - first) {
                                    it.s0 = first + r;
                                    it.s1 = it.count[0] = it.count[1] = end + r;
                                    it.sinks = end;
                                    it.from = first;
                                }
                            }
                        }
                    }
                    ok = mbar_wait(&M.item_empty[ri.slot], ri.phase ^ 1u, wc, 31);
                    if (!ok) break;
                    M.items[ri.slot] = it;
                    mbar_arrive(&M.item_full[ri.slot]);
                    ri.next();
                }
                if (p.join) p.join[blockIdx.x] = join;
                if (ok) ok = mbar_wait(&M.item_empty[ri.slot], ri.phase ^ 1u, wc, 31);
                if (ok) {
                    M.items[ri.slot].head = -1;
                    mbar_arrive(&M.item_full[ri.slot]);
                }
            }
            __syncwarp();
            if (blockIdx.x == 0 && a.out_status)
                for (int b = lane; b < a.s.B; b += 32)
                    a.out_status[b] = sequence_of(a, b).ok ? TWINKV_OK : TWINKV_ERR_INVALID_ARG;
        }
        __syncwarp();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
        if (warp == 9) tmem_dealloc<1>(tmem, 512);
    } else {
        // ------------------------------------------------------------ softmax
        setmaxnreg_inc<kSoftmaxRegs>();
        const int x = warp >> 2, q = warp & 3;
        const int row = q * 32 + lane;
        const uint32_t base = tmem + (static_cast<uint32_t>(q * 32) << 16);
        const uint32_t t_s = base + C::T_S + x * kTileKeys, t_o = base + C::T_O + x * D;
        const uint32_t t_p = base + C::T_P + x * C::P_STRIDE;
        const int token = row / a.G, sub = row - token * a.G;        // of the tile
        const int first_token = q * 32 / a.G, last_token = (q * 32 + 31) / a.G;
        Ring<kItemSlots> ri;
        uint32_t s_uses = 0, o_uses = 0;
        bool ok = true;
        while (ok) {
            if (!(ok = all_wait(&M.item_full[ri.slot], ri.phase, wc, 34))) break;
            const Item it = M.items[ri.slot];
            __syncwarp();
            if (lane == 0) mbar_arrive(&M.item_empty[ri.slot]);
            ri.next();
            if (it.head < 0) break;
            const KeyTiles kt{it.sinks, it.from, 0};
            const int n = min(it.s1, x ? it.count[1] : it.count[0]);
            const int p0 = it.pos + x * tpt;                         // position of the tile's first token
            const int pos = p0 + token;
            const int low = a.window > 0 ? pos - a.window + 1 : INT_MIN;
            // rows of no token hold anything
            const bool sees = token < tpt && x * tpt + token < it.tokens && pos >= 0;
            float top = -INFINITY, sum = 0.0f;
            bool large = false;                                      // one of the warp's tops is
            for (int j = it.s0; j < n; ++j) {
                const int k0 = kt.tile(j) * kTileKeys;
                if (!(ok = all_wait(&M.s_full[x], s_uses++ & 1u, wc, 35))) break;
                tc_fence_after();
                uint32_t s[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) tmem_ld_32x32b_x32(t_s + 32 * i, s[i]);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 4; ++i) reg_fence(s[i]);
                if constexpr (C::EARLY) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&M.s_free[x]);
                }
                const bool edge = k0 + kTileKeys - 1 > p0 + first_token ||
                                  (a.window > 0 && k0 < p0 + last_token - a.window + 1 &&
                                   k0 + kTileKeys > a.n_sink);
                if (edge) {
                    const int hi = pos - k0, lo = low - k0, sinks = a.n_sink - k0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t see = bits_below(hi + 1 - 32 * i);
                        if (a.window > 0)
                            see &= ~bits_below(lo - 32 * i) | bits_below(sinks - 32 * i);
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            s[i][e] = see >> e & 1u ? s[i][e] : 0xff800000u;
                    }
                }
                // With the top so far; again with the true one where a row has none, or its sum shows that
                // the scores have left it far behind.
                bool exact = large || __any_sync(0xffffffffu, sees && top == -INFINITY);
                // the products with the tile's last probabilities, whose place the next ones take
                if (C::EARLY && j > it.s0) {
                    if (!(ok = all_wait(&M.o_full[x], o_uses++ & 1u, wc, 36))) break;
                    tc_fence_after();
                }
                for (;;) {
                    if (exact) {
                        float m[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            m[i] = as_f(s[i][0]);
#pragma unroll
                            for (int e = 1; e < 31; e += 2)
                                m[i] = max3(m[i], as_f(s[i][e]), as_f(s[i][e + 1]));
                            m[i] = fmaxf(m[i], as_f(s[i][31]));
                        }
                        const float most = fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
                        const bool rise = most > top;
                        const float f = rise ? exp2_approx(top_gap(top, most, p.c)) : 1.0f;    // top -inf: 0
                        if (rise) top = most;
                        if (j > it.s0 && __any_sync(0xffffffffu, rise)) {
                            sum *= f;
#pragma unroll
                            for (int i = 0; i < D / 32; ++i) {
                                uint32_t o[32];
                                tmem_ld_32x32b_x32(t_o + 32 * i, o);
                                tmem_wait_ld();
                                reg_fence(o);
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(as_f(o[e]) * f);
                                tmem_st_32x32b_x32(t_o + 32 * i, o);
                            }
                        }
                        large = __any_sync(0xffffffffu, sees && top > -INFINITY &&
                                                            fabsf(top * p.c) > kLarge);
                        if (large) {             // the tile is not done again: s may change
                            const float y = top == -INFINITY ? 0.0f : -top;
#pragma unroll
                            for (int i = 0; i < 4; ++i)
#pragma unroll
                                for (int e = 0; e < 32; e += 2) {
                                    const float2 z = __fadd2_rn(
                                        make_float2(as_f(s[i][e]), as_f(s[i][e + 1])), make_float2(y, y));
                                    s[i][e] = __float_as_uint(z.x);
                                    s[i][e + 1] = __float_as_uint(z.y);
                                }
                        }
                    }
                    const float t = large || top == -INFINITY ? 0.0f : __fmul_rn(top, p.c);
                    const float2 c2 = make_float2(p.c, p.c), t2 = make_float2(-t, -t);
                    float2 l[4] = {};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t w[32];
#pragma unroll
                        for (int e = 0; e < 64; e += 2) {
                            const int i = 2 * h + e / 32;
                            const float2 y = __ffma2_rn(
                                make_float2(as_f(s[i][e % 32]), as_f(s[i][e % 32 + 1])), c2, t2);
                            const float u = exp2_approx(y.x), v = exp2_approx(y.y);
                            l[e / 2 % 4] = __fadd2_rn(l[e / 2 % 4], make_float2(u, v));
                            w[e / 2] = bf16_pair(u, v);
                        }
                        tmem_st_32x32b_x32(t_p + 32 * h, w);
                    }
                    const float2 l2 = __fadd2_rn(__fadd2_rn(l[0], l[1]), __fadd2_rn(l[2], l[3]));
                    const float add = l2.x + l2.y;
                    if (exact || !__any_sync(0xffffffffu, sees && add > kFar)) {
                        sum += add;
                        break;
                    }
                    exact = true;
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&M.p_full[x]);
            }
            if (!ok) break;
            // ---- the item's rows: outputs, or a part
            const bool any = n > it.s0;
            if (any) {
                if (!(ok = all_wait(&M.o_full[x], o_uses++ & 1u, wc, 36))) break;
                tc_fence_after();
            }
            const bool held = token < tpt && x * tpt + token < it.tokens;
            const int64_t at_row = static_cast<int64_t>(it.t0 + x * tpt + token) * a.s.Hq +
                                   it.head * a.G + sub;
            if (it.slot < 0) {
                const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;      // O is 0 where sum is
                // through shared memory, 128 bytes of every row at a time, so that eight lanes write a
                // row's (a row to a lane: 6700 cycles for 256 rows of 128, now 2000)
                uint8_t* mine = smem + C::OFF_OUT + warp * 32 * 128;
                const int to = held ? (x * tpt + token) * a.s.Hq + sub : -1;
                uint16_t* out = a.out + (static_cast<int64_t>(it.t0) * a.s.Hq + it.head * a.G) * D;
#pragma unroll
                for (int h = 0; h < C::KC; ++h) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t o[32] = {};
                        if (any) {
                            tmem_ld_32x32b_x32(t_o + 64 * h + 32 * i, o);
                            tmem_wait_ld();
                            reg_fence(o);
                        }
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint4 w;
                            w.x = bf16_pair(as_f(o[e]) * inv, as_f(o[e + 1]) * inv);
                            w.y = bf16_pair(as_f(o[e + 2]) * inv, as_f(o[e + 3]) * inv);
                            w.z = bf16_pair(as_f(o[e + 4]) * inv, as_f(o[e + 5]) * inv);
                            w.w = bf16_pair(as_f(o[e + 6]) * inv, as_f(o[e + 7]) * inv);
                            *reinterpret_cast<uint4*>(mine + lane * 128 +
                                                      ((4 * i + e / 8) ^ (lane & 7)) * 16) = w;
                        }
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int r = 4 * i + lane / 8;
                        const uint4 w = *reinterpret_cast<const uint4*>(
                            mine + r * 128 + ((lane & 7) ^ (r & 7)) * 16);
                        const int at_r = __shfl_sync(0xffffffffu, to, r);
                        if (at_r >= 0)
                            *reinterpret_cast<uint4*>(out + static_cast<int64_t>(at_r) * D + 64 * h +
                                                      8 * (lane & 7)) = w;
                    }
                    __syncwarp();
                }
                if (held && a.out_lse)
                    a.out_lse[at_row] = log_sum(top, sum, p.c, a.scale);
            } else {
                float* part = p.part + static_cast<int64_t>(it.slot) * kPartFloats<D>;
                const int r = x * kTileRows + row;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    uint32_t o[32] = {};
                    if (any) {
                        tmem_ld_32x32b_x32(t_o + 32 * i, o);
                        tmem_wait_ld();
                        reg_fence(o);
                    }
                    if (!any) continue;
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        *reinterpret_cast<uint4*>(part + ((8 * i + e / 4) * kPairRows + r) * 4) =
                            make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                }
                part[kPairRows * D + r] = sum > 0.0f ? top : -INFINITY;
                part[kPairRows * (D + 1) + r] = sum;
            }
            tc_fence_before();
        }
        tc_fence_before();
        __syncthreads();
    }
}

// Joins the parts of an item that several blocks took, in order: a block per block that such an item
// begins in and 32 rows of it, a warp for every eighth group of four values.  Rows leave through shared
// memory, whole ones side by side (4096 tokens, 40 MB of parts: 7 us beside the rest, with 8 bytes of 32 rows
// in a store 11).
constexpr int kMergeWarps = 8;

template <int D>
__global__ void __launch_bounds__(32 * kMergeWarps)
    merge_kernel(const __grid_constant__ AttendKernelArgs p)
{
    constexpr int kVec = D / 4 / kMergeWarps;
    __shared__ __align__(16) uint8_t rows[32][2 * D + 16];
    wait_for_previous();
    const PromptArgs& a = p.a;
    const int4 join = p.join[blockIdx.x];
    if (join.x == 0) return;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int r = blockIdx.y * 32 + lane;
    const int x = r / kTileRows, row = r % kTileRows, tpt = a.tile_tokens;
    const int token = row / a.G;
    const bool held = token < tpt && x * tpt + token < join.z;
    float top = -INFINITY, sum = 0.0f, acc[kVec][4] = {};
    constexpr int kAhead = 4;
    for (int k0 = 0; held && k0 < join.x; k0 += kAhead) {
        float m[kAhead], l[kAhead];
        float4 y[kAhead][kVec];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            m[k] = -INFINITY;
            l[k] = 0.0f;
            if (k0 + k >= join.x) continue;
            const int slot = 2 * (blockIdx.x + k0 + k) + (k0 + k == 0 ? 1 : 0);
            const float* part = p.part + static_cast<int64_t>(slot) * kPartFloats<D>;
            m[k] = part[kPairRows * D + r];
            l[k] = part[kPairRows * (D + 1) + r];
#pragma unroll
            for (int v = 0; v < kVec; ++v)
                y[k][v] = *reinterpret_cast<const float4*>(
                    part + ((warp + kMergeWarps * v) * kPairRows + r) * 4);
        }
        float most = top;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) most = fmaxf(most, m[k]);
        if (most == -INFINITY) continue;
        const float f = exp2_approx(top_gap(top, most, p.c));
        sum *= f;
#pragma unroll
        for (int v = 0; v < kVec; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[v][e] *= f;
        top = most;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (m[k] == -INFINITY) continue;          // what it holds is no number
            const float w = exp2_approx(top_gap(m[k], top, p.c));
            sum = fmaf(l[k], w, sum);
#pragma unroll
            for (int v = 0; v < kVec; ++v) {
                acc[v][0] = fmaf(y[k][v].x, w, acc[v][0]);
                acc[v][1] = fmaf(y[k][v].y, w, acc[v][1]);
                acc[v][2] = fmaf(y[k][v].z, w, acc[v][2]);
                acc[v][3] = fmaf(y[k][v].w, w, acc[v][3]);
            }
        }
    }
    const int64_t first = static_cast<int64_t>(join.y) * a.s.Hq + join.w * a.G;
    const int at = held ? (x * tpt + token) * a.s.Hq + row - token * a.G : -1;
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int v = 0; v < kVec; ++v)
        *reinterpret_cast<uint2*>(rows[lane] + 8 * (warp + kMergeWarps * v)) =
            make_uint2(bf16_pair(acc[v][0] * inv, acc[v][1] * inv),
                       bf16_pair(acc[v][2] * inv, acc[v][3] * inv));
    if (warp == 0 && held && a.out_lse)
        a.out_lse[first + at] = log_sum(top, sum, p.c, a.scale);
    __syncthreads();
    constexpr int kRowLanes = D / 8;
#pragma unroll
    for (int i = 0; i < 32 * kRowLanes; i += 32 * kMergeWarps) {
        const int n = (i + static_cast<int>(threadIdx.x)) / kRowLanes, e = threadIdx.x % kRowLanes;
        const int to = __shfl_sync(0xffffffffu, at, n);
        if (to >= 0)
            *reinterpret_cast<uint4*>(a.out + (first + to) * D + 8 * e) =
                *reinterpret_cast<const uint4*>(rows[n] + 16 * e);
    }
}

// Where no item is longer than 13 units none is cut: the longest takes no longer than shares and a second
// kernel (d = 128: 512 tokens 15.8 -> 13.7 us, 1024 24.7 -> 21.0, 1500 35.3 -> 29.0; d = 64: 1024 19.4 -> 16.2).
// The lengths being on the device, all rows of k decide: a batch of short prompts gets the second kernel.
constexpr int kSnapFew = 6;
constexpr int whole_keys(int d) { return (2 * kSnapFew + 1 - RowPairs::more(d)) * kTileKeys; }

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
        if ((e = cudaFuncGetAttributes(&f, prompt_attend_kernel<D>)) != cudaSuccess) return e;
        if (f.numRegs < kLaunchRegs) return cudaErrorInvalidConfiguration;
        e = cudaFuncSetAttribute(prompt_attend_kernel<D>,
                                 cudaFuncAttributeMaxDynamicSharedMemorySize, C::BYTES);
        if (e != cudaSuccess) return e;
        if (dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
    }
    CUtensorMap q, k, v;
    const int tpt = a.tile_tokens;
    if (!encode_rows(&q, a.q, D, a.s.Hq, a.s.tokens, a.s.q_head, a.s.q_token, a.G, tpt) ||
        !encode_rows(&k, a.k, D, a.s.H, a.s.keys, a.s.k_head, a.s.k_token, 1, kTileKeys) ||
        !encode_rows(&v, a.v, D, a.s.H, a.s.keys, a.s.v_head, a.s.v_token, 1, kTileKeys))
        return cudaErrorInvalidValue;
    AttendKernelArgs p{};
    const bool shared = a.s.keys > whole_keys(D);
    p.a = a;
    p.a.snap = shared ? kSnap : kSnapFew;
    p.c = a.scale * 1.4426950408889634f;
    if (shared) {
        p.join = static_cast<int4*>(a.ws);
        p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(a.ws) + 16 * kPromptBlocks);
    }
    p.err = w.err;
    p.timeout_ns = w.timeout_ns;
    const int grid = std::min(sms, kPromptBlocks);
    prompt_attend_kernel<D><<<grid, kThreads, C::BYTES, st>>>(q, k, v, p);
    if ((e = cudaGetLastError()) != cudaSuccess || !shared) return e;
    return launch_dependent(merge_kernel<D>, dim3(grid, kPairRows / 32), 32 * kMergeWarps, 0, st, p);
}

}  // namespace

size_t prompt_attend_workspace(const twinkv_prompt& s)
{
    if (s.keys <= whole_keys(s.d)) return 256;
    return 16 * kPromptBlocks +
           2 * kPromptBlocks * static_cast<size_t>(kPairRows) * (s.d + 2) * sizeof(float);
}

cudaError_t launch_prompt_attend(const PromptArgs& a, int sms, const WaitFacts& w, cudaStream_t st)
{
    return a.s.d == 128 ? launch<128>(a, sms, w, st) : launch<64>(a, sms, w, st);
}

}  // namespace twk
