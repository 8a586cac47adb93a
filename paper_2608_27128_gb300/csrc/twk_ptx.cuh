// twk_ptx.cuh -- inline-PTX building blocks for sm_103a: mbarriers with bounded waits,
// TMA (cp.async.bulk / cp.async.bulk.tensor), and the tcgen05 tensor-core path
// (TMEM alloc/ld, UMMA shared-memory and instruction descriptors, mma, commit).
#pragma once
#include <cstdint>
#include <cuda.h>

namespace twk {

// Device error word layout (int32[4], lives in the library's device memory):
//   [0] first sticky status (TWINKV_ERR_TIMEOUT), [1] where it happened,
//   [2] block index, [3] reserved.
enum : int { kErrTimeout = 5 };

__device__ __forceinline__ uint32_t smem_u32(const void* p)
{
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// True in one lane of a converged warp, always the same one.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(p));
    return p != 0;
}

__device__ __forceinline__ uint64_t globaltimer_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// ---------------------------------------------------------------- mbarrier

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count)
                 : "memory");
}

__device__ __forceinline__ void fence_mbarrier_init()
{
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}

__device__ __forceinline__ void mbar_arrive(uint64_t* bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ void mbar_arrive_expect_tx(uint64_t* bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)),
                 "r"(bytes)
                 : "memory");
}

// The same shared-memory address in CTA `rank` of the cluster (a shared::cluster address).
__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// Every thread of every CTA of the cluster arrives, then waits for the others.
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Arrival on a barrier of a CTA of the cluster, named by its shared::cluster address.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar)
                 : "memory");
}

__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Whether the barrier's phase is complete, without waiting.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Whether both barriers' phases are complete (1 or 0), without waiting.
__device__ __forceinline__ uint32_t mbar_test2(uint32_t bar0, uint32_t parity0, uint32_t bar1,
                                               uint32_t parity1)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 q, [%3], %4;\n\t"
        "and.pred p, p, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar0), "r"(parity0), "r"(bar1), "r"(parity1)
        : "memory");
    return ok;
}

// The same, but the thread may stay suspended for up to `hint_ns` while the phase is
// incomplete (it resumes as soon as the phase completes): a waiting warp then takes
// no issue slots from the warps that share its sub-partition.
__device__ __forceinline__ bool mbar_try_wait_sleep(uint32_t bar, uint32_t parity,
                                                    uint32_t hint_ns)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(hint_ns)
        : "memory");
    return ok != 0;
}

// Everything a bounded wait needs: the time limit, the block's abort flag (shared
// memory) and the device error word.
struct WaitCtl {
    uint64_t limit_ns;
    volatile int* abort_flag;
    int* err;
    int where;
};

__device__ __forceinline__ void record_timeout(const WaitCtl& w, int where)
{
    if (atomicCAS(w.err, 0, kErrTimeout) == 0) {
        w.err[1] = where;
        w.err[2] = static_cast<int>(blockIdx.x);
    }
    *w.abort_flag = 1;
}

// Wait for the phase of `bar` with parity `parity` to complete.  Gives up (returns
// false) when the block's abort flag is raised or after w.limit_ns; a give-up records
// TWINKV_ERR_TIMEOUT in the error word and raises the abort flag for the whole block.
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity, const WaitCtl& w,
                                          int where)
{
    const uint32_t a = smem_u32(bar);
    if (mbar_try_wait(a, parity)) return true;
    const uint64_t t0 = globaltimer_ns();
    for (;;) {
        // suspended for up to ~1 ms per attempt, woken when the phase completes
        if (mbar_try_wait_sleep(a, parity, 1000000u)) return true;
        if (*w.abort_flag) return false;
        if (globaltimer_ns() - t0 > w.limit_ns) {
            record_timeout(w, where);
            return false;
        }
    }
}

// ---------------------------------------------------------------- TMA

// 2-D tiled tensor load into this CTA's shared memory, completion (tx bytes) signalled on
// `bar`, a shared::cluster address of a barrier in either CTA of the pair.
__device__ __forceinline__ void tma_load_2d_pair(void* dst, const CUtensorMap* map, uint32_t bar,
                                                 int x, int y)
{
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
        : "memory");
}

// 3-D tiled tensor load into this CTA's shared memory, completion signalled on its barrier.
__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, uint64_t* bar, int x,
                                            int y, int z)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
        : "memory");
}

// Plain bulk copy global -> shared (16-byte aligned addresses, size multiple of 16).
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes,
                                          uint64_t* bar)
{
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
            "r"(smem_u32(dst)),
        "l"(src), "r"(bytes), "r"(smem_u32(bar))
        : "memory");
}

__device__ __forceinline__ void prefetch_tensormap(const CUtensorMap* map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}

// ---------------------------------------------------------------- dependent launches

// Waits until the kernel before this one on its stream has ended and its writes are visible
// (at once where the launch was not a programmatic dependent), and lets the next kernel's
// blocks be set up as soon as every block of this one has started.
__device__ __forceinline__ void wait_for_previous()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ---------------------------------------------------------------- registers
// Every warp of a warpgroup gives up or takes registers (kRegs per thread afterwards).

template <int kRegs>
__device__ __forceinline__ void setmaxnreg_dec()
{
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs));
}

template <int kRegs>
__device__ __forceinline__ void setmaxnreg_inc()
{
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs));
}

// ---------------------------------------------------------------- tcgen05
// kGroup = 2 forms act on a pair of CTAs (ranks 2k and 2k + 1 of a cluster): both CTAs
// allocate and free, one thread of the even CTA issues the MMAs and commits.

template <int kGroup>
__device__ __forceinline__ void tmem_alloc(uint32_t* slot, uint32_t ncols)
{
    asm volatile("tcgen05.alloc.cta_group::%2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(slot)),
                 "r"(ncols), "n"(kGroup)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::%0.sync.aligned;" ::"n"(kGroup)
                 : "memory");
}

template <int kGroup>
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols)
{
    asm volatile("tcgen05.dealloc.cta_group::%2.sync.aligned.b32 %0, %1;" ::"r"(taddr),
                 "r"(ncols), "n"(kGroup)
                 : "memory");
}

__device__ __forceinline__ void tc_fence_before()
{
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}

__device__ __forceinline__ void tc_fence_after()
{
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// D[tmem] (+)= A[smem] * B[smem]^T over a CTA pair, one instruction of shape M x N x 16,
// bf16 -> f32: each CTA holds half of A's rows, half of B's rows (the N side) and its own
// A rows' accumulators; the descriptors' offsets are the same in both CTAs.
__device__ __forceinline__ void umma_bf16_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc,
                                               uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Arrive, in both CTAs of the pair, on the barrier at this offset once every tcgen05
// operation this thread issued so far has completed.
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64"
        " [%0], %1;" ::"r"(smem_u32(bar)),
        "h"(static_cast<uint16_t>(3))
        : "memory");
}

// The same on this CTA's barrier only.
__device__ __forceinline__ void umma_commit_own(uint64_t* bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
            smem_u32(bar))
        : "memory");
}

// The forms of one CTA, for operands as umma_desc_sw128 and umma_desc_sw128_rows describe them (low words
// of the descriptors, the high word being kDescHigh): D[tmem] (+)= A B, bf16 -> f32, in steps of 16 along
// K.  The steps' descriptors are made inside: as C++ values the compiler keeps them all in registers.
// The high word: stride byte offset >> 4 of 1024 B from bit 0, version 1 at bit 14, layout type 2 at bit 29.
constexpr uint32_t kDescHigh = 1024u >> 4 | 1u << 14 | 2u << 29;

// A and B K-major in shared memory, K = 64 kChunks: rows of 64 values, chunks of 64 of them 16 KB apart.
template <int kChunks>
__device__ __forceinline__ void umma_rows(uint32_t d_tmem, uint32_t a_low, uint32_t b_low,
                                          uint32_t idesc)
{
#define TWK_STEP(offset, sum)                                                              \
    "add.u32 a, %1, " #offset ";\n\tadd.u32 b, %2, " #offset ";\n\t"                       \
    "mov.b64 x, {a, h};\n\tmov.b64 y, {b, h};\n\t"                                        \
    "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, " #sum ";\n\t"
#define TWK_BEGIN(high)                                                                    \
    "{\n\t.reg .pred p, q;\n\t.reg .b32 a, b, h;\n\t.reg .b64 x, y;\n\t"                   \
    "mov.b32 h, %" #high ";\n\tsetp.ne.b32 p, h, 0;\n\t"
    if constexpr (kChunks == 2)
        asm volatile(TWK_BEGIN(4) "setp.eq.b32 q, h, 0;\n\t" TWK_STEP(0, q) TWK_STEP(2, p)
                         TWK_STEP(4, p) TWK_STEP(6, p) TWK_STEP(1024, p) TWK_STEP(1026, p)
                             TWK_STEP(1028, p) TWK_STEP(1030, p) "}" ::"r"(d_tmem),
                     "r"(a_low), "r"(b_low), "r"(idesc), "n"(kDescHigh)
                     : "memory");
    else
        asm volatile(TWK_BEGIN(4) "setp.eq.b32 q, h, 0;\n\t" TWK_STEP(0, q) TWK_STEP(2, p)
                         TWK_STEP(4, p) TWK_STEP(6, p) "}" ::"r"(d_tmem),
                     "r"(a_low), "r"(b_low), "r"(idesc), "n"(kDescHigh)
                     : "memory");
#undef TWK_STEP
}

// A [128][128] in tensor memory (a 32-bit column holds two neighbours along K), B's rows along K; the
// first step adds to D where `add`.
__device__ __forceinline__ void umma_tmem_128(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_low,
                                              uint32_t idesc, uint32_t add)
{
#define TWK_STEP(i, column, offset, sum)                                                   \
    "add.u32 a, %1, " #column ";\n\tadd.u32 b, %2, " #offset ";\n\tmov.b64 y, {b, h};\n\t" \
    "tcgen05.mma.cta_group::1.kind::f16 [%0], [a], y, %3, " #sum ";\n\t"
    asm volatile(TWK_BEGIN(5) "setp.ne.b32 q, %4, 0;\n\t" TWK_STEP(0, 0, 0, q) TWK_STEP(1, 8, 128, p)
                     TWK_STEP(2, 16, 256, p) TWK_STEP(3, 24, 384, p) TWK_STEP(4, 32, 512, p)
                         TWK_STEP(5, 40, 640, p) TWK_STEP(6, 48, 768, p)
                             TWK_STEP(7, 56, 896, p) "}" ::"r"(d_tmem),
                 "r"(a_tmem), "r"(b_low), "r"(idesc), "r"(add), "n"(kDescHigh)
                 : "memory");
#undef TWK_STEP
}

// A [128][64 kChunks] in tensor memory, B K-major in shared memory as in umma_rows.
template <int kChunks>
__device__ __forceinline__ void umma_tmem_rows(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_low,
                                               uint32_t idesc)
{
#define TWK_STEP(column, offset, sum)                                                      \
    "add.u32 a, %1, " #column ";\n\tadd.u32 b, %2, " #offset ";\n\tmov.b64 y, {b, h};\n\t" \
    "tcgen05.mma.cta_group::1.kind::f16 [%0], [a], y, %3, " #sum ";\n\t"
    if constexpr (kChunks == 2)
        asm volatile(TWK_BEGIN(4) "setp.eq.b32 q, h, 0;\n\t" TWK_STEP(0, 0, q) TWK_STEP(8, 2, p)
                         TWK_STEP(16, 4, p) TWK_STEP(24, 6, p) TWK_STEP(32, 1024, p)
                             TWK_STEP(40, 1026, p) TWK_STEP(48, 1028, p)
                                 TWK_STEP(56, 1030, p) "}" ::"r"(d_tmem),
                     "r"(a_tmem), "r"(b_low), "r"(idesc), "n"(kDescHigh)
                     : "memory");
    else
        asm volatile(TWK_BEGIN(4) "setp.eq.b32 q, h, 0;\n\t" TWK_STEP(0, 0, q) TWK_STEP(8, 2, p)
                         TWK_STEP(16, 4, p) TWK_STEP(24, 6, p) "}" ::"r"(d_tmem),
                     "r"(a_tmem), "r"(b_low), "r"(idesc), "n"(kDescHigh)
                     : "memory");
#undef TWK_STEP
#undef TWK_BEGIN
}

// Arrive on the barrier once every tcgen05 operation this thread issued so far has completed.
__device__ __forceinline__ void umma_commit(uint64_t* bar)
{
    asm volatile(
        "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
            smem_u32(bar))
        : "memory");
}

__device__ __forceinline__ void tmem_wait_st()
{
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Generic accesses to shared memory before this come before the asynchronous proxy's (TMA, MMA)
// that follow.
__device__ __forceinline__ void fence_async_shared()
{
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

__device__ __forceinline__ void tmem_wait_ld()
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// 32 lanes x 32 consecutive 32-bit columns: thread t of the warp gets lane (base + t),
// columns [col, col + 32) in r[0..31].
__device__ __forceinline__ void tmem_ld_32x32b_x32(uint32_t taddr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
          "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(taddr)
        : "memory");
}

// The same store: thread t of the warp writes its lane's 32 columns.
__device__ __forceinline__ void tmem_st_32x32b_x32(uint32_t taddr, const uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
        "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}

// UMMA shared-memory descriptor for a K-major operand laid out by TMA with 128-byte
// swizzling: rows of 128 bytes (64 bf16 along K), 8-row groups 1024 bytes apart.
// Fields: start address >> 4 [0,14); leading byte offset >> 4 [16,30) (not used by
// swizzled K-major layouts, set to 1); stride byte offset >> 4 [32,46) = 1024 B;
// descriptor version 1 at bit 46; base offset 0 (tiles are 1024-byte aligned);
// layout type [61,64) = 2 (128-byte swizzle).
__device__ __forceinline__ uint64_t umma_desc_sw128(uint32_t saddr)
{
    uint64_t d = 0;
    d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(1u) << 16;
    d |= static_cast<uint64_t>(kDescHigh) << 32;
    return d;
}

// The same for an operand whose rows run along K, 64 of its M or N values to a row of 128 bytes:
// the leading byte offset is what the next 64 values are apart, the stride byte offset (1024 B) what
// the next 8 rows are.
__device__ __forceinline__ uint64_t umma_desc_sw128_rows(uint32_t saddr, uint32_t next64)
{
    return (umma_desc_sw128(saddr) & ~0xffff0000ull) | static_cast<uint64_t>(next64 >> 4) << 16;
}
constexpr uint32_t kIdescBRows = 1u << 16;   // of the instruction: B is such an operand

// Instruction descriptor, kind::f16: f32 accumulator [4,6)=1, A and B bf16 [7,10)=1 and
// [10,13)=1, both K-major (bits 15, 16 clear), N >> 3 at [17,23), M >> 4 at [24,29).
__host__ __device__ constexpr uint32_t umma_idesc_bf16_f32(int M, int N)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(N >> 3) << 17) |
           (static_cast<uint32_t>(M >> 4) << 24);
}

}  // namespace twk
