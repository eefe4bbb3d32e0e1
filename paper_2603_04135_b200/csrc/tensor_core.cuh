// Building blocks of the tensor-core kernels: bounded mbarrier waits, shared-memory matrix descriptors, tiled TMA
// loads, tensor-memory reads (shared by the fused LM-head and the 8-bit product; not part of the ABI).
#pragma once
#include <cuda.h>

#include "common.cuh"

namespace dppo {

__device__ __forceinline__ uint32_t lm_smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ unsigned long long lm_global_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

__device__ __forceinline__ bool lm_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

// Bounded wait; also leaves when another role has raised the abort flag.  The clock and the flag are looked at once
// per sixteen tries (a try already suspends the thread for a short, hardware-chosen time), not per try.
__device__ __forceinline__ bool lm_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns) {
    if (lm_try(bar, parity)) return true;
    const unsigned long long t0 = lm_global_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 16; ++i)
            if (lm_try(bar, parity)) return true;
        if (*abort_flag) return false;
        if (lm_global_ns() - t0 > limit_ns) { *abort_flag = 1; return false; }
    }
}

// Bounded wait that ignores the abort flag (used on the way out).
__device__ __forceinline__ bool lm_wait_plain(uint32_t bar, uint32_t parity, unsigned long long limit_ns) {
    if (lm_try(bar, parity)) return true;
    const unsigned long long t0 = lm_global_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 16; ++i)
            if (lm_try(bar, parity)) return true;
        if (lm_global_ns() - t0 > limit_ns) return false;
    }
}

__device__ __forceinline__ void lm_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}

// Shared-memory descriptor of a K-major operand tile (descriptor version 1 = sm_100, layout type 2 = SWIZZLE_128B;
// addresses and offsets in 16-byte units): rows of 128 bytes of K, in 1024-byte swizzle atoms of 8 rows, exactly as a
// 128B-swizzled TMA box with a 128-byte inner extent lands them; 8-row groups are 1024 bytes apart (stride offset), the
// leading offset is unused.  The next 32 bytes of K (one instruction's share) are 32 bytes further along the row.
__device__ __forceinline__ uint64_t lm_smem_desc_k(uint32_t smem_addr) {
    return (uint64_t)((smem_addr >> 4) & 0x3FFF) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

// L2 eviction policy of an operand's loads: a tile that other CTAs (or later waves) will ask for again is kept
// (evict_last), one that is streamed through once makes room first (evict_first).
enum { kHintNone = 0, kHintEvictFirst = 1, kHintEvictLast = 2 };
__device__ __forceinline__ uint64_t lm_l2_policy(int hint) {
    uint64_t pol = 0;
    if (hint == kHintEvictFirst) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    else if (hint == kHintEvictLast) asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}

// One tiled TMA load (x = innermost coordinate, 16-byte aligned by construction: multiples of 64 elements).
// pol = 0: no hint.
__device__ __forceinline__ void lm_tma_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, uint64_t pol) {
    if (pol)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4}], [%2], %5;"
                     :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "l"(pol) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
// The same from a CTA of a pair: the barrier may be the peer's (the pair's leader collects both CTAs' bytes).
__device__ __forceinline__ void lm_tma_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, uint64_t pol) {
    if (pol)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4}], [%2], %5;"
                     :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "l"(pol) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                     :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}

// Instructions marked .aligned want the warp's lanes together.  After code that some lanes leave early (rows or channels past
// the end), or that one lane runs alone, only a __syncwarp() promises that: callers of these helpers see to it.

// 32 consecutive f32 columns of this thread's TMEM lane (its tile row) into registers.
__device__ __forceinline__ void lm_tmem_load32(uint32_t (&v)[32], uint32_t taddr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
                   "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
                   "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

// Address of the pair leader's copy of a barrier, from either CTA of a pair.
constexpr uint32_t kPeerMask = 0xFEFFFFFFu;                  // shared::cluster address of the pair's leader (rank bit cleared)

__device__ __forceinline__ void lm_cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled_fn() {
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = (EncodeTiledFn)p;
    }
    return fn;
}

}  // namespace dppo
