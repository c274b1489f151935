// PTX wrappers and small helpers shared by the tensor-core translation units (tcgen05, TMA, mbarriers).
// Everything sits in an anonymous namespace: each translation unit that includes this file gets its own copy,
// including its own device status word for waits that ran out.
#pragma once
#include <cuda.h>
#include "qnn_internal.cuh"

namespace qnn {
namespace {

constexpr int BM = 128;              // rows of A per tile (UMMA M)
constexpr int BKB = 128;             // bytes of K per pipeline stage = one 128-byte swizzle row
constexpr uint32_t WAIT_LIMIT = 1u << 22;
constexpr int SMEM_LIMIT = 232448;   // 227 KB of dynamic shared memory per CTA

__device__ int g_tc_status = 0;      // 0 = fine; otherwise the code of the first wait that ran out (per translation unit)

// ---- PTX wrappers -----------------------------------------------------------

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded wait.  Returns false when the block is aborting (this wait ran out, or another one did).
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, int code,
                                          const uint32_t limit = WAIT_LIMIT)
{
    for (uint32_t it = 0; it < limit; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if (it > 4096) __nanosleep(64);
        if ((it & 63) == 63 && *abort_flag) return false;
    }
    *abort_flag = 1;
    atomicCAS(&g_tc_status, 0, code);
    return false;
}


// bulk tensor stores (shared -> global); rows / columns past the tensor's extents are clipped by the hardware
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, int32_t x, int32_t y, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                 ::"l"(map), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t src)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// waits until the shared-memory side of all but the N most recent store groups has been read
template <int N>
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// CTAS = 1: a CTA works alone.  CTAS = 2: two CTAs of a cluster share 256 x BN tiles (cta_group::2); the same
// warp of both CTAs allocates / frees.
template <int CTAS>
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t ncols)
{
    if (CTAS == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(ncols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(ncols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <int CTAS>
__device__ __forceinline__ void tmem_dealloc(uint32_t taddr, uint32_t ncols)
{
    if (CTAS == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
__device__ __forceinline__ uint32_t cluster_ctarank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// shared::cluster address of the same shared-memory location in CTA `rank` of this cluster
__device__ __forceinline__ uint32_t map_to_cta(uint32_t saddr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
    return r;
}
// (release at CTA scope, the default: a cluster-scope release makes the arriving thread wait until its earlier global
// stores are visible cluster-wide -- measured 2500 clk per tile in the pair's epilogue -- and nothing the peer reads
// depends on them: the barrier only hands tensor-memory columns back)
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// After a wait that ran out: time for copies and products still in flight to land before shared and tensor memory go away.
__device__ __forceinline__ void let_flights_land()
{
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
}
// A CTA that gave up must not end while others of its cluster may still store into its shared memory.  It stays until every
// thread of theirs has ended or given up too (a cluster barrier waits for threads that have not exited, and for no others), and
// then for what those sent last.  For all warps that are left in the CTA, each past its wait for the barrier's phase before.
__device__ __forceinline__ void stay_for_cluster()
{
    cluster_sync_all();
    let_flights_land();
}
__device__ __forceinline__ void umma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
// this warp's 32 lanes x 8 columns, all set to `val`
__device__ __forceinline__ void tmem_st8(uint32_t taddr, uint32_t val)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %1, %1, %1, %1, %1, %1, %1};" ::"r"(taddr), "r"(val) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory matrix descriptor of a K-major tile whose rows are KB = 128 (or 64) bytes, swizzled over 128 (64)
// bytes -- the layout a TMA box of KB bytes x rows produces: 8-row groups are 8*KB bytes apart.
template <int KB>
__device__ __forceinline__ uint64_t make_kmajor_desc(uint32_t saddr)
{
    uint64_t d = 0;
    d |= (uint64_t)((saddr & 0x3ffffu) >> 4);          // start address, 16-byte units
    d |= (uint64_t)1 << 16;                            // leading-dimension offset (unused with swizzle) = 1
    d |= (uint64_t)((8 * KB) >> 4) << 32;              // stride between 8-row groups
    d |= (uint64_t)1 << 46;                            // descriptor version of this architecture
    d |= (uint64_t)(KB == 128 ? 2 : 4) << 61;          // 128-byte / 64-byte swizzle
    return d;
}

// One pipeline stage of the MMA warp as ONE instruction stream: poll the NEXT stage's full barrier, issue the
// four K steps of this stage (+32 bytes of K = +2 in the descriptors' address field), commit them to this
// stage's empty barrier, and only then read the poll's result -- the poll's latency hides behind the issue.
// Returns non-zero when the next stage has already landed.
template <int FORM>
__device__ __forceinline__ uint32_t umma_stage(uint32_t next_full_bar, uint32_t next_parity, uint32_t d_tmem, uint32_t a_lo,
                                               uint32_t b_lo, uint32_t desc_hi, uint32_t idesc, uint32_t accumulate_first,
                                               uint32_t sf, uint32_t empty_bar)
{
    uint32_t ready;
    if (FORM == QNN_FORM_FP4) {
        asm volatile(
            "{\n"
            ".reg .pred P, Q, T;\n"
            ".reg .b64 a0, a1, a2, a3, b0, b1, b2, b3;\n"
            ".reg .b32 t1, t2, t3, u1, u2, u3;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 Q, [%1], %2;\n"
            "setp.ne.b32 P, %7, 0;\n"
            "setp.eq.b32 T, 0, 0;\n"
            "add.u32 t1, %4, 2;\n add.u32 t2, %4, 4;\n add.u32 t3, %4, 6;\n"
            "add.u32 u1, %5, 2;\n add.u32 u2, %5, 4;\n add.u32 u3, %5, 6;\n"
            "mov.b64 a0, {%4, %10};\n mov.b64 a1, {t1, %10};\n mov.b64 a2, {t2, %10};\n mov.b64 a3, {t3, %10};\n"
            "mov.b64 b0, {%5, %10};\n mov.b64 b1, {u1, %10};\n mov.b64 b2, {u2, %10};\n mov.b64 b3, {u3, %10};\n"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%3], a0, b0, %6, [%8], [%8], P;\n"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%3], a1, b1, %6, [%8], [%8], T;\n"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%3], a2, b2, %6, [%8], [%8], T;\n"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%3], a3, b3, %6, [%8], [%8], T;\n"
            "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%9];\n"
            "selp.u32 %0, 1, 0, Q;\n"
            "}\n"
            : "=r"(ready)
            : "r"(next_full_bar), "r"(next_parity), "r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate_first),
              "r"(sf), "r"(empty_bar), "r"(desc_hi)
            : "memory");
    } else {
        asm volatile(
            "{\n"
            ".reg .pred P, Q, T;\n"
            ".reg .b64 a0, a1, a2, a3, b0, b1, b2, b3;\n"
            ".reg .b32 t1, t2, t3, u1, u2, u3;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 Q, [%1], %2;\n"
            "setp.ne.b32 P, %7, 0;\n"
            "setp.eq.b32 T, 0, 0;\n"
            "add.u32 t1, %4, 2;\n add.u32 t2, %4, 4;\n add.u32 t3, %4, 6;\n"
            "add.u32 u1, %5, 2;\n add.u32 u2, %5, 4;\n add.u32 u3, %5, 6;\n"
            "mov.b64 a0, {%4, %10};\n mov.b64 a1, {t1, %10};\n mov.b64 a2, {t2, %10};\n mov.b64 a3, {t3, %10};\n"
            "mov.b64 b0, {%5, %10};\n mov.b64 b1, {u1, %10};\n mov.b64 b2, {u2, %10};\n mov.b64 b3, {u3, %10};\n"
            "tcgen05.mma.cta_group::1.kind::i8 [%3], a0, b0, %6, P;\n"
            "tcgen05.mma.cta_group::1.kind::i8 [%3], a1, b1, %6, T;\n"
            "tcgen05.mma.cta_group::1.kind::i8 [%3], a2, b2, %6, T;\n"
            "tcgen05.mma.cta_group::1.kind::i8 [%3], a3, b3, %6, T;\n"
            "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%9];\n"
            "selp.u32 %0, 1, 0, Q;\n"
            "}\n"
            : "=r"(ready)
            : "r"(next_full_bar), "r"(next_parity), "r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate_first),
              "r"(sf), "r"(empty_bar), "r"(desc_hi)
            : "memory");
    }
    return ready;
}

// The same stage for a CTA pair (issued by the leader CTA): one instruction multiplies the 256 x BN tile of both
// CTAs; the commit arrives on this stage's empty barrier of BOTH CTAs.
template <int FORM>
__device__ __forceinline__ uint32_t umma_stage_pair(uint32_t next_full_bar, uint32_t next_parity, uint32_t d_tmem, uint32_t a_lo,
                                                    uint32_t b_lo, uint32_t desc_hi, uint32_t idesc, uint32_t accumulate_first,
                                                    uint32_t sf, uint32_t empty_bar)
{
    uint32_t ready;
    if (FORM == QNN_FORM_FP4) {
        asm volatile(
            "{\n"
            ".reg .pred P, Q, T;\n"
            ".reg .b64 a0, a1, a2, a3, b0, b1, b2, b3;\n"
            ".reg .b32 t1, t2, t3, u1, u2, u3;\n"
            ".reg .b16 both;\n"
            "mov.b16 both, 3;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 Q, [%1], %2;\n"
            "setp.ne.b32 P, %7, 0;\n"
            "setp.eq.b32 T, 0, 0;\n"
            "add.u32 t1, %4, 2;\n add.u32 t2, %4, 4;\n add.u32 t3, %4, 6;\n"
            "add.u32 u1, %5, 2;\n add.u32 u2, %5, 4;\n add.u32 u3, %5, 6;\n"
            "mov.b64 a0, {%4, %10};\n mov.b64 a1, {t1, %10};\n mov.b64 a2, {t2, %10};\n mov.b64 a3, {t3, %10};\n"
            "mov.b64 b0, {%5, %10};\n mov.b64 b1, {u1, %10};\n mov.b64 b2, {u2, %10};\n mov.b64 b3, {u3, %10};\n"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%3], a0, b0, %6, [%8], [%8], P;\n"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%3], a1, b1, %6, [%8], [%8], T;\n"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%3], a2, b2, %6, [%8], [%8], T;\n"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%3], a3, b3, %6, [%8], [%8], T;\n"
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%9], both;\n"
            "selp.u32 %0, 1, 0, Q;\n"
            "}\n"
            : "=r"(ready)
            : "r"(next_full_bar), "r"(next_parity), "r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate_first),
              "r"(sf), "r"(empty_bar), "r"(desc_hi)
            : "memory");
    } else {
        asm volatile(
            "{\n"
            ".reg .pred P, Q, T;\n"
            ".reg .b64 a0, a1, a2, a3, b0, b1, b2, b3;\n"
            ".reg .b32 t1, t2, t3, u1, u2, u3;\n"
            ".reg .b16 both;\n"
            "mov.b16 both, 3;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 Q, [%1], %2;\n"
            "setp.ne.b32 P, %7, 0;\n"
            "setp.eq.b32 T, 0, 0;\n"
            "add.u32 t1, %4, 2;\n add.u32 t2, %4, 4;\n add.u32 t3, %4, 6;\n"
            "add.u32 u1, %5, 2;\n add.u32 u2, %5, 4;\n add.u32 u3, %5, 6;\n"
            "mov.b64 a0, {%4, %10};\n mov.b64 a1, {t1, %10};\n mov.b64 a2, {t2, %10};\n mov.b64 a3, {t3, %10};\n"
            "mov.b64 b0, {%5, %10};\n mov.b64 b1, {u1, %10};\n mov.b64 b2, {u2, %10};\n mov.b64 b3, {u3, %10};\n"
            "tcgen05.mma.cta_group::2.kind::i8 [%3], a0, b0, %6, P;\n"
            "tcgen05.mma.cta_group::2.kind::i8 [%3], a1, b1, %6, T;\n"
            "tcgen05.mma.cta_group::2.kind::i8 [%3], a2, b2, %6, T;\n"
            "tcgen05.mma.cta_group::2.kind::i8 [%3], a3, b3, %6, T;\n"
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%9], both;\n"
            "selp.u32 %0, 1, 0, Q;\n"
            "}\n"
            : "=r"(ready)
            : "r"(next_full_bar), "r"(next_parity), "r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate_first),
              "r"(sf), "r"(empty_bar), "r"(desc_hi)
            : "memory");
    }
    return ready;
}
// accumulator-complete signal to both CTAs of a pair
__device__ __forceinline__ void umma_commit_pair(uint32_t bar)
{
    asm volatile(
        "{\n.reg .b16 both;\nmov.b16 both, 3;\n"
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], both;\n}\n"
        ::"r"(bar) : "memory");
}

// TMA stage of one CTA of a pair: the loads land in this CTA's shared memory and report their bytes to the
// LEADER's full barrier (`leader_full_bar`, a shared::cluster address); only the leader announces the bytes
// (those of both CTAs).  No load is multicast.
__device__ __forceinline__ uint32_t tma_stage_2d_pair(uint32_t next_empty_bar, uint32_t next_parity, uint32_t leader_full_bar,
                                                      uint32_t tx_bytes_both, uint32_t is_leader, uint32_t dst_a,
                                                      const CUtensorMap *map_a, int32_t ax, int32_t ay, uint32_t dst_b,
                                                      const CUtensorMap *map_b, int32_t bx, int32_t by)
{
    uint32_t ready;
    asm volatile(
        "{\n"
        ".reg .pred Q, L;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 Q, [%1], %2;\n"
        "setp.ne.b32 L, %13, 0;\n"
        "@L mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%3], %4;\n"
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%5], [%6, {%7, %8}], [%3];\n"
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%9], [%10, {%11, %12}], [%3];\n"
        "selp.u32 %0, 1, 0, Q;\n"
        "}\n"
        : "=r"(ready)
        : "r"(next_empty_bar), "r"(next_parity), "r"(leader_full_bar), "r"(tx_bytes_both), "r"(dst_a), "l"(map_a), "r"(ax),
          "r"(ay), "r"(dst_b), "l"(map_b), "r"(bx), "r"(by), "r"(is_leader)
        : "memory");
    return ready;
}

// One pipeline stage of the TMA warp the same way: poll the NEXT stage's empty barrier first, announce this
// stage's bytes, issue its two loads, then read the poll's result.
__device__ __forceinline__ uint32_t tma_stage_2d(uint32_t next_empty_bar, uint32_t next_parity, uint32_t full_bar, uint32_t tx_bytes,
                                                 uint32_t dst_a, const CUtensorMap *map_a, int32_t ax, int32_t ay,
                                                 uint32_t dst_b, const CUtensorMap *map_b, int32_t bx, int32_t by)
{
    uint32_t ready;
    asm volatile(
        "{\n"
        ".reg .pred Q;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 Q, [%1], %2;\n"
        "mbarrier.arrive.expect_tx.shared::cta.b64 _, [%3], %4;\n"
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%5], [%6, {%7, %8}], [%3];\n"
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%9], [%10, {%11, %12}], [%3];\n"
        "selp.u32 %0, 1, 0, Q;\n"
        "}\n"
        : "=r"(ready)
        : "r"(next_empty_bar), "r"(next_parity), "r"(full_bar), "r"(tx_bytes), "r"(dst_a), "l"(map_a), "r"(ax), "r"(ay),
          "r"(dst_b), "l"(map_b), "r"(bx), "r"(by)
        : "memory");
    return ready;
}
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void *sym = nullptr;
        cudaDriverEntryPointQueryResult qr;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &qr) == cudaSuccess &&
            qr == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(sym);
    }
    return fn;
}

// Reads and clears this translation unit's status word (0 = no wait ran out).
inline cudaError_t status_read_clear(int *code)
{
    *code = 0;
    cudaError_t e = cudaMemcpyFromSymbol(code, g_tc_status, sizeof(int));
    if (e != cudaSuccess) return e;
    if (*code != 0) {
        const int zero = 0;
        e = cudaMemcpyToSymbol(g_tc_status, &zero, sizeof(int));
    }
    return e;
}

}  // namespace
}  // namespace qnn
