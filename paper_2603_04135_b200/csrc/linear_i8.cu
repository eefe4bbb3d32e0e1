// Matrix product in 8-bit integers with one scale per token and one per output channel, on the 5th-generation tensor
// cores: out[t, n] = (sx[t] sw[n]) sum_k x[t, k] w[n, k], the sum an exact int32 (tcgen05.mma kind::i8); and the
// quantisation of rows that makes its operands.
//
// The weights take the M side of the tensor-core tile (TMEM lanes = output channels), the tokens its N side (TMEM
// columns): a tile of 128 channels then fits any number of tokens from 16 up without wasted columns, and the epilogue,
// whose thread holds one channel, writes 32 consecutive channels of a token per warp instruction whatever the row
// pitch of the output (64 or 128 contiguous bytes, no alignment asked for).
//
// Two kernels:
//   many tokens (tensor-core bound): persistent CTA pairs (cta_group::2), 256 channels x 256 tokens per tile, 128-byte K
//     slabs through a TMA ring of 224 KB, two TMEM accumulators so that the epilogue of a tile runs under the next one's
//     products; tiles are handed out so that the CTAs running together share their weights and their tokens in L2
//   few tokens (bound by reading the weights): a CTA per 128 channels, 16 to 128 tokens, and the contraction split over
//     the CTAs of a cluster when there are too few tiles to keep all SMs reading; the int32 partial sums are joined
//     through distributed shared memory (exact, so the split changes no result)
// Every wait is bounded; on a time-out the CTA reports DPPO_STATUS_TIMEOUT, leaves its loops, lets copies and products in
// flight finish (bounded), frees its tensor memory and returns.
#include <type_traits>

#include "common.cuh"
#include "grpo_loss.cuh"
#include "tensor_core.cuh"

namespace dppo {
namespace i8 {

constexpr int kBK = 128;                  // K slab: 128 codes = one 128-byte swizzle row
constexpr int kTileM = 128;               // channels per CTA
constexpr int kTileN = 256;               // most tokens per tile of the pair kernel
constexpr int kMaxStages = 12;
constexpr int kBytesA = kTileM * kBK;                        // 16 KB
constexpr int kThreads = 320;              // producer warp, MMA warp, 8 epilogue warps (two per TMEM lane quarter)
constexpr int kTokenGroup = 16;           // token tiles swept together (4096 tokens: 10 MB of codes at K = 2560)
constexpr int kRingBytes = 7 * (kBytesA + kTileN / 2 * kBK);   // pair kernel: 7 stages of the largest tile, more of smaller ones
constexpr size_t kDynSmem2 = (size_t)kRingBytes + 1024;
static_assert(kDynSmem2 + 512 <= 232448, "the ring must fit one CTA's shared memory");

struct Args {
    const float* x_scale;
    const float* w_scale;
    void* out;
    const int32_t* n_rows_dev;
    int32_t* status;
    long long M_max, out_stride;
    int N, n_ksteps, out_bf16;
    int tile_n;                           // pair kernel: tokens per tile, a multiple of 32 up to 256
    unsigned long long wait_limit_ns;
    int test_extra_tx;
};

// Instruction descriptor of kind::i8: D = s32, A = B = s8, both K-major.
__host__ __device__ constexpr uint32_t idesc(int m, int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ long long true_rows(const Args& a) {
    return a.n_rows_dev ? min((long long)max(*a.n_rows_dev, 0), a.M_max) : a.M_max;
}

// One output: the scales are multiplied first, each step rounded to f32, then to the output's type.
__device__ __forceinline__ float value_of(int32_t acc, float sx, float sw) { return __fmul_rn(__int2float_rn(acc), __fmul_rn(sx, sw)); }
template <bool kBf16> __device__ __forceinline__ void store(const Args& a, long long t, int n, float v) {
    if constexpr (kBf16) reinterpret_cast<__nv_bfloat16*>(a.out)[t * a.out_stride + n] = __float2bfloat16_rn(v);
    else reinterpret_cast<float*>(a.out)[t * a.out_stride + n] = v;
}
// kCount consecutive tokens t0 .. of this lane's channel (sx: lane i holds token t0 + i's scale).  All values first, then all
// stores: with a test per output the shuffles and stores of a warp wait for each other (the product of 2,048 x 2,560 x 40,000
// bf16: 168 us instead of 146; of 1,003 x 2,563 x 5,003: 22.6 instead of 18.3).
template <bool kBf16, int kCount>
__device__ __forceinline__ void store_column(const Args& a, long long t0, long long T, int ch, const uint32_t (&v)[32], float sx, float sw) {
    typedef typename std::conditional<kBf16, __nv_bfloat16, float>::type Out;
    const int nt = (int)min((long long)kCount, T - t0);
    Out x[kCount];
#pragma unroll
    for (int i = 0; i < kCount; i += 2) {
        const float x0 = value_of((int32_t)v[i], __shfl_sync(0xffffffffu, sx, i), sw);
        const float x1 = value_of((int32_t)v[i + 1], __shfl_sync(0xffffffffu, sx, i + 1), sw);
        if constexpr (kBf16) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(x0, x1);
            x[i] = b.x; x[i + 1] = b.y;
        } else {
            x[i] = x0; x[i + 1] = x1;
        }
    }
    if (ch < a.N) {
        Out* p = reinterpret_cast<Out*>(a.out) + t0 * a.out_stride + ch;
        if (nt == kCount) {
#pragma unroll
            for (int i = 0; i < kCount; ++i, p += a.out_stride) *p = x[i];
        } else {
#pragma unroll
            for (int i = 0; i < kCount; ++i, p += a.out_stride)
                if (i < nt) *p = x[i];
        }
    }
}

// ---- many tokens: CTA pairs ---------------------------------------------------------------------------
struct Shared2 {
    unsigned long long full[kMaxStages];
    unsigned long long empty[kMaxStages];
    unsigned long long acc_full[2];
    unsigned long long acc_empty[2];      // the leader's copy counts 16 arrivals: 8 epilogue warps x 2 CTAs
    unsigned long long drain;             // products in flight on an early way out
    uint32_t tmem_base;
    int abort;
};

// Tile j of this pair: token tiles are taken kTokenGroup at a time; within a group the token tiles of one channel tile
// follow each other, so that every weight is fetched once per group and the group's codes stay in L2.
__device__ __forceinline__ bool tile_of(uint32_t j, int n_m2, int n_tok, int& m2, int& n) {
    const long long id = (long long)(blockIdx.x >> 1) + (long long)j * (gridDim.x >> 1);
    if (id >= (long long)n_m2 * n_tok) return false;
    const long long per = (long long)kTokenGroup * n_m2;
    const int g = (int)(id / per), local = (int)(id - (long long)g * per);
    const int n0 = g * kTokenGroup, width = min(kTokenGroup, n_tok - n0);
    m2 = local / width;
    n = n0 + local - m2 * width;
    return true;
}

template <bool kBf16>
__global__ void __launch_bounds__(kThreads, 1)
linear_i8_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const Args a) {
    extern __shared__ unsigned char i8_raw[];
    __shared__ Shared2 sh;
    const uint32_t tiles = (lm_smem_u32(i8_raw) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint32_t rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const bool leader = rank == 0;
    volatile int* abort_flag = &sh.abort;
    const int n_m2 = (a.N + 2 * kTileM - 1) / (2 * kTileM);
    // a stage: 128 codes of K of this CTA's 128 channels and of its half of the token tile
    const uint32_t stage_bytes = (uint32_t)(kBytesA + a.tile_n / 2 * kBK);
    const uint32_t stages = min((uint32_t)kMaxStages, (uint32_t)kRingBytes / stage_bytes);

    if (tid == 0) {
        sh.abort = 0;
        for (uint32_t s = 0; s < stages; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(lm_smem_u32(&sh.full[s])));
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(lm_smem_u32(&sh.empty[s])));
        }
        for (int b = 0; b < 2; ++b) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(lm_smem_u32(&sh.acc_full[b])));
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 16;" :: "r"(lm_smem_u32(&sh.acc_empty[b])));
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(lm_smem_u32(&sh.drain)));
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(lm_smem_u32(&sh.tmem_base)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    __syncwarp();
    lm_cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = sh.tmem_base;
    enter_kernel();
    const long long T = true_rows(a);
    const int n_tok = (int)((T + a.tile_n - 1) / a.tile_n);

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer (both CTAs)
        if (lane == 0) {
            uint32_t it = 0, s = 0, use = 0;
            int m2, n;
            for (uint32_t j = 0; tile_of(j, n_m2, n_tok, m2, n) && !*abort_flag; ++j) {
                const int row_w = (2 * m2 + (int)rank) * kTileM, row_x = n * a.tile_n + (int)rank * (a.tile_n / 2);
                for (int k = 0; k < a.n_ksteps; ++k, ++it, s = s + 1 == stages ? 0 : s + 1, use += s == 0 ? 1 : 0) {
                    if (use > 0 && !lm_wait(lm_smem_u32(&sh.empty[s]), (use - 1) & 1, abort_flag, a.wait_limit_ns)) break;
                    const uint32_t bar_local = lm_smem_u32(&sh.full[s]), bar = bar_local & kPeerMask;
                    const uint32_t dst = tiles + s * stage_bytes;
                    if (leader)                                        // the leader's barrier collects both CTAs' bytes
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                                     :: "r"(bar_local), "r"(2 * stage_bytes + (it == 0 ? (uint32_t)a.test_extra_tx : 0u)) : "memory");
                    lm_tma_2d_pair(dst, &map_w, bar, k * kBK, row_w, 0);
                    lm_tma_2d_pair(dst + kBytesA, &map_x, bar, k * kBK, row_x, 0);
                }
            }
            if (*abort_flag && leader) {                               // copies in flight get a bounded chance to land
                const uint32_t pending = it < stages ? it : stages;
                for (uint32_t i = 0; i < pending; ++i) {
                    const uint32_t i2 = it - 1 - i;
                    lm_wait_plain(lm_smem_u32(&sh.full[i2 % stages]), (i2 / stages) & 1, a.wait_limit_ns);
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (leader CTA only)
        if (lane == 0 && leader) {
            const uint32_t desc = idesc(2 * kTileM, a.tile_n);
            uint32_t s = 0, use = 0;
            int m2, n;
            bool ok = true;
            for (uint32_t j = 0; ok && tile_of(j, n_m2, n_tok, m2, n) && !*abort_flag; ++j) {
                const uint32_t b = j & 1, use_b = j >> 1;
                if (use_b > 0 && !lm_wait(lm_smem_u32(&sh.acc_empty[b]), (use_b - 1) & 1, abort_flag, a.wait_limit_ns)) { ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t d_tmem = tmem_base + b * kTileN;
                for (int k = 0; k < a.n_ksteps; ++k, s = s + 1 == stages ? 0 : s + 1, use += s == 0 ? 1 : 0) {
                    if (!lm_wait(lm_smem_u32(&sh.full[s]), use & 1, abort_flag, a.wait_limit_ns)) { ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t dw = lm_smem_desc_k(tiles + s * stage_bytes), dx = lm_smem_desc_k(tiles + s * stage_bytes + kBytesA);
#pragma unroll
                    for (int kk = 0; kk < kBK / 32; ++kk) {              // 32 codes of K per instruction
                        const uint32_t accumulate = (k > 0 || kk > 0) ? 1u : 0u;
                        asm volatile("{\n\t.reg .pred p;\n\t"
                                     "setp.ne.b32 p, %4, 0;\n\t"
                                     "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                                     :: "r"(d_tmem), "l"(dw + kk * 2), "l"(dx + kk * 2), "r"(desc), "r"(accumulate) : "memory");
                    }
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                                 :: "r"(lm_smem_u32(&sh.empty[s])), "h"((unsigned short)3) : "memory");
                }
                if (!ok) break;
                asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                             :: "r"(lm_smem_u32(&sh.acc_full[b])), "h"((unsigned short)3) : "memory");
            }
            if (!ok || *abort_flag) {                                  // products already issued finish before memory goes away
                asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(lm_smem_u32(&sh.drain)) : "memory");
                lm_wait_plain(lm_smem_u32(&sh.drain), 0, a.wait_limit_ns);
            }
        }
    } else {
        // ------------------------------------------------------------------ epilogue (warps 2..9, both CTAs)
        const int q = warp & 3, half = (warp - 2) >> 2;                  // TMEM lane quarter of this warp; which blocks of 32 tokens
        int m2, n;
        for (uint32_t j = 0; tile_of(j, n_m2, n_tok, m2, n); ++j) {
            const int ch = (2 * m2 + (int)rank) * kTileM + q * 32 + lane;
            const float sw = ch < a.N ? a.w_scale[ch] : 0.0f;
            const uint32_t b = j & 1, use_b = j >> 1;
            // warp-uniform outcome: the tcgen05.ld below must be executed by all 32 lanes together
            if (!__all_sync(0xffffffffu, lm_wait(lm_smem_u32(&sh.acc_full[b]), use_b & 1, abort_flag, a.wait_limit_ns))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + b * kTileN;
#pragma unroll 1
            for (int c = half; c < a.tile_n / 32; c += 2) {
                const long long t0 = (long long)n * a.tile_n + c * 32;
                if (t0 >= T) break;
                uint32_t v[32];
                lm_tmem_load32(v, taddr + (uint32_t)(c * 32));
                const float sx = t0 + lane < T ? a.x_scale[t0 + lane] : 0.0f;
                store_column<kBf16, 32>(a, t0, T, ch, v, sx, sw);
                __syncwarp();                                            // lanes without a channel went ahead; the next load wants all
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0)                                               // the leader's MMA thread waits for all 16 warps
                asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(lm_smem_u32(&sh.acc_empty[b]) & kPeerMask) : "memory");
        }
    }

    // ---- common exit: both CTAs are done with tensor memory and with each other's barriers, then free
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    __syncwarp();
    lm_cluster_sync();
    if (tid == 0 && sh.abort) set_status(a.status, DPPO_STATUS_TIMEOUT);
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"(512u) : "memory");
    }
}

// ---- few tokens: a CTA per 128 channels, K split over a cluster ---------------------------------------
// Stages for two resident CTAs per SM.
template <int kNB> __host__ __device__ constexpr int small_stages() { return kNB <= 16 ? 6 : kNB <= 32 ? 5 : kNB <= 64 ? 4 : 3; }
template <int kNB> __host__ __device__ constexpr int small_stage_bytes() { return kBytesA + kNB * kBK; }
template <int kNB> constexpr size_t small_smem() { return (size_t)small_stages<kNB>() * small_stage_bytes<kNB>() + 1024; }

struct SharedSmall {
    unsigned long long full[6];
    unsigned long long empty[6];
    unsigned long long done;
    uint32_t tmem_base;
    int abort;
};

// 16 or 32 columns of this thread's TMEM lane.
__device__ __forceinline__ void tmem_load16(uint32_t (&v)[32], uint32_t taddr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

template <int kNB, bool kBf16>
__global__ void __launch_bounds__(kThreads)
linear_i8_small_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const Args a, int n_ch, int split) {
    constexpr int kStages = small_stages<kNB>(), kStageBytes = small_stage_bytes<kNB>();
    constexpr int kCols = kNB < 32 ? 32 : kNB;
    constexpr int kChunk = kNB < 32 ? kNB : 32;
    extern __shared__ unsigned char i8_raw[];
    __shared__ SharedSmall sh;
    const uint32_t tiles = (lm_smem_u32(i8_raw) + 1023u) & ~1023u;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &sh.abort;
    const int part = (int)(blockIdx.x % (unsigned)split);                 // rank in the cluster: clusters are consecutive CTAs
    const int id = (int)(blockIdx.x / (unsigned)split);
    const int m = id % n_ch;
    const long long t_tile = (long long)(id / n_ch) * kNB;
    const int k0 = (int)((long long)a.n_ksteps * part / split), k1 = (int)((long long)a.n_ksteps * (part + 1) / split);

    if (tid == 0) {
        sh.abort = 0;
        for (int s = 0; s < kStages; ++s) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(lm_smem_u32(&sh.full[s])));
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(lm_smem_u32(&sh.empty[s])));
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" :: "r"(lm_smem_u32(&sh.done)));
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    enter_kernel();
    const long long T = true_rows(a);
    if (t_tile >= T) return;                                              // the whole cluster leaves together
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(lm_smem_u32(&sh.tmem_base)), "r"((uint32_t)kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = sh.tmem_base;

    if (warp == 0) {
        if (lane == 0) {
            int it = 0;
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it % kStages, use = it / kStages;
                if (use > 0 && !lm_wait(lm_smem_u32(&sh.empty[s]), (use - 1) & 1, abort_flag, a.wait_limit_ns)) break;
                const uint32_t bar = lm_smem_u32(&sh.full[s]), dst = tiles + s * kStageBytes;
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                             :: "r"(bar), "r"((uint32_t)kStageBytes + (it == 0 ? (uint32_t)a.test_extra_tx : 0u)) : "memory");
                lm_tma_2d(dst, &map_w, bar, k * kBK, m * kTileM, 0);
                lm_tma_2d(dst + kBytesA, &map_x, bar, k * kBK, (int)t_tile, 0);
            }
            if (*abort_flag) {
                const int pending = it < kStages ? it : kStages;
                for (int i = 0; i < pending; ++i) {
                    const int i2 = it - 1 - i;
                    lm_wait_plain(lm_smem_u32(&sh.full[i2 % kStages]), (i2 / kStages) & 1, a.wait_limit_ns);
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            int it = 0;
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it % kStages, use = it / kStages;
                if (!lm_wait(lm_smem_u32(&sh.full[s]), use & 1, abort_flag, a.wait_limit_ns)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint64_t dw = lm_smem_desc_k(tiles + s * kStageBytes), dx = lm_smem_desc_k(tiles + s * kStageBytes + kBytesA);
#pragma unroll
                for (int kk = 0; kk < kBK / 32; ++kk) {
                    const uint32_t accumulate = (it > 0 || kk > 0) ? 1u : 0u;
                    asm volatile("{\n\t.reg .pred p;\n\t"
                                 "setp.ne.b32 p, %4, 0;\n\t"
                                 "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                                 :: "r"(tmem_base), "l"(dw + kk * 2), "l"(dx + kk * 2), "r"(idesc(kTileM, kNB)), "r"(accumulate) : "memory");
                }
                asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(lm_smem_u32(&sh.empty[s])) : "memory");
            }
            // all products issued so far (on an early way out too: they finish before memory goes away)
            asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(lm_smem_u32(&sh.done)) : "memory");
            lm_wait_plain(lm_smem_u32(&sh.done), 0, a.wait_limit_ns);
        }
    }
    // epilogue warps; the int32 sums of a split contraction go through shared memory: [token][channel], in the ring,
    // which nothing reads or writes any more once `done` has completed
    const int q = warp & 3, row = q * 32 + lane;
    const int half = (warp - 2) >> 2, halves = (int)(blockDim.x - 64) >> 7;         // one or two warps per lane quarter share the tokens
    const int ch = m * kTileM + row;
    bool live = false;
    const float sw = warp >= 2 && ch < a.N ? a.w_scale[ch] : 0.0f;
    if (warp >= 2) {
        live = __all_sync(0xffffffffu, lm_wait(lm_smem_u32(&sh.done), 0, abort_flag, a.wait_limit_ns)) && !*abort_flag;
        live = __all_sync(0xffffffffu, live);
        if (live) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
            for (int c = half; c < kNB / kChunk; c += halves) {
                const long long t0 = t_tile + c * kChunk;
                if (t0 >= T) break;
                uint32_t v[32];
                if constexpr (kChunk == 16) tmem_load16(v, taddr); else lm_tmem_load32(v, taddr + (uint32_t)(c * 32));
                if (split == 1) {
                    const float sx = t0 + lane < T && lane < kChunk ? a.x_scale[t0 + lane] : 0.0f;
                    store_column<kBf16, kChunk>(a, t0, T, ch, v, sx, sw);
                    // as there; fewer tokens are one block per warp (in every warp and for all kNB: 16 tokens 5.55 -> 5.8 us)
                    if constexpr (kNB > 64) { if ((ch | 31) >= a.N) __syncwarp(); }
                } else {
#pragma unroll
                    for (int i = 0; i < kChunk; ++i)
                        asm volatile("st.shared.b32 [%0], %1;" :: "r"(tiles + (uint32_t)((c * kChunk + i) * kTileM + row) * 4u), "r"(v[i]) : "memory");
                }
            }
        }
    }
    if (split > 1) {
        __syncwarp();
        lm_cluster_sync();                                               // every CTA's sums are in its shared memory
        if (live) {
            // this CTA's share of the tokens: part, part + split, ...; a batch's loads are all under way before the first is used
            // (one token at a time, each waits out the latency of its remote reads: 128 tokens 31 us instead of 14)
            constexpr int kBatch = 4;
            const int n_tok = (int)min((long long)kNB, T - t_tile);
            const int step = halves * split;
            for (int c0 = part + half * split; c0 < n_tok; c0 += kBatch * step) {
                int32_t sum[kBatch];
                float sx[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    sum[i] = 0;
                    sx[i] = c0 + i * step < n_tok ? a.x_scale[t_tile + c0 + i * step] : 0.0f;
                }
                for (int i0 = 0; i0 < split; ++i0) {                     // every CTA starts with another one's memory
                    const int r = (part + i0) & (split - 1);
                    int32_t x[kBatch];
                    uint32_t remote;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(tiles + (uint32_t)row * 4u), "r"(r));
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) {
                        const int c = c0 + i * step;
                        x[i] = 0;
                        if (c < n_tok)
                            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(x[i]) : "r"(remote + (uint32_t)(c * kTileM) * 4u) : "memory");
                    }
#pragma unroll
                    for (int i = 0; i < kBatch; ++i) sum[i] += x[i];
                }
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (c0 + i * step < n_tok && ch < a.N)
                        store<kBf16>(a, t_tile + c0 + i * step, ch, value_of(sum[i], sx[i], sw));
            }
        }
        if ((ch | 31) >= a.N) __syncwarp();                              // lanes without a channel went ahead; no other warp parts
        lm_cluster_sync();                                               // the others have read this CTA's shared memory
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (tid == 0 && sh.abort) set_status(a.status, DPPO_STATUS_TIMEOUT);
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"((uint32_t)kCols) : "memory");
    }
}

// ---- quantisation of rows -----------------------------------------------------------------------------
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

struct QuantArgs {
    const char* x;
    int8_t* q;
    float* scale;
    const int32_t* n_rows_dev;
    long long rows_max, x_row_bytes, q_stride;
    int K;
};

__device__ __forceinline__ uint32_t code_of(float x, float s) {
    const float v = rintf(__fdiv_rn(x, s));
    return (uint32_t)(int32_t)fminf(fmaxf(v, -127.0f), 127.0f) & 0xffu;
}

// The codes of kPer values (4 per word).  x / s lies within 4e-5 of x * r, r = fl(1/s) (|x / s| <= 127.1, relative errors of r and
// of the quotient 2^-24 each), so unless x * r is that close to a tie, both round to the same integer; adding 1.5 * 2^23 rounds
// to it and leaves it in the low bits.  A vector with such a value is divided out (one in thousands).  The division alone
// held the kernel to 3.1 TB/s on 16,384 x 4,096 bf16.
// quick: s is large enough for r to be a normal number.
template <int kPer> __device__ __forceinline__ void codes_of(const float (&f)[kPer], float s, float r, bool quick, bool live, uint32_t (&w)[kPer / 4]) {
    constexpr float kMagic = 12582912.0f;
    float t[kPer], far = quick ? 0.0f : 1.0f;
    using namespace packed;
    const f32x2 r2 = pair_of(r, r), magic = pair_of(kMagic, kMagic), neg = pair_of(-1.0f, -1.0f);
#pragma unroll
    for (int j = 0; j < kPer; j += 2) {
        const f32x2 x = pair_of(f[j], f[j + 1]), n = fma2(x, r2, magic);
        float d0, d1;
        unpair(fma2(x, r2, fma2(n, neg, magic)), d0, d1);
        far = fmaxf(fmaxf(far, fabsf(d0)), fabsf(d1));
        unpair(n, t[j], t[j + 1]);
    }
#pragma unroll
    for (int j = 0; j < kPer; j += 4) {
        const uint32_t lo = __byte_perm(__float_as_uint(t[j]), __float_as_uint(t[j + 1]), 0x0040);
        const uint32_t hi = __byte_perm(__float_as_uint(t[j + 2]), __float_as_uint(t[j + 3]), 0x0040);
        w[j / 4] = __byte_perm(lo, hi, 0x5410);
    }
    if (!(far < 0.4999f)) {
#pragma unroll
        for (int j = 0; j < kPer; j += 4)
            w[j / 4] = live ? code_of(f[j], s) | code_of(f[j + 1], s) << 8 | code_of(f[j + 2], s) << 16 | code_of(f[j + 3], s) << 24 : 0u;
    }
}

// A team of kThreads per row: the maximum, then the codes.  Rows of up to kVecs vectors per thread stay in registers in between;
// longer ones are read a second time (out of L2).
template <bool kBf16, int kThreads, int kVecs>
__global__ void __launch_bounds__(kThreads < 128 ? 128 : kThreads)
quantize_rows_kernel(const QuantArgs a) {
    constexpr int kPer = Elems<kBf16>::kPerVec, kTeams = kThreads < 128 ? 128 / kThreads : 1;
    __shared__ float red[kThreads / 32];
    enter_kernel();
    const int tid = kTeams == 1 ? threadIdx.x : threadIdx.x % kThreads;
    const long long t = kTeams == 1 ? (long long)blockIdx.x : (long long)blockIdx.x * kTeams + threadIdx.x / kThreads;
    const long long T = a.n_rows_dev ? min((long long)*a.n_rows_dev, a.rows_max) : a.rows_max;
    if (t >= T) return;
    const char* row = a.x + t * a.x_row_bytes;
    const uint4* rv = reinterpret_cast<const uint4*>(row);
    int8_t* q = a.q + t * a.q_stride;
    const int nvec = a.K / kPer, tail = nvec * kPer + tid;
    uint4 v[kVecs];
    float amax = 0.0f;
    __nv_bfloat162 amax2 = __floats2bfloat162_rn(0.0f, 0.0f);
    auto look = [&](const uint4& x) {
        if constexpr (kBf16) {                                     // two magnitudes at a time (16,384 x 4,096: 45 -> 42 us)
            const uint32_t w[4] = {x.x & 0x7fff7fffu, x.y & 0x7fff7fffu, x.z & 0x7fff7fffu, x.w & 0x7fff7fffu};
            const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(w);
            amax2 = __hmax2_nan(amax2, __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
        } else {
            float f[kPer];
            Elems<kBf16>::unpack(x, f);
#pragma unroll
            for (int j = 0; j < kPer; ++j) amax = max_nan(amax, fabsf(f[j]));
        }
    };
#pragma unroll
    for (int u = 0; u < kVecs; ++u) v[u] = u * kThreads + tid < nvec ? rv[u * kThreads + tid] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int u = 0; u < kVecs; ++u) look(v[u]);
    // the rest in rounds of kVecs loads; zeros do not move a maximum of magnitudes
    auto rest = [&](auto use) {
        for (int i = kVecs * kThreads + tid; i < nvec; i += kVecs * kThreads) {
            uint4 x[kVecs];
#pragma unroll
            for (int u = 0; u < kVecs; ++u) x[u] = i + u * kThreads < nvec ? rv[i + u * kThreads] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int u = 0; u < kVecs; ++u) use(x[u], i + u * kThreads);
        }
    };
    rest([&](const uint4& x, int) { look(x); });
    const float xt = tail < a.K ? Elems<kBf16>::load1(row, tail) : 0.0f;
    if constexpr (kBf16) amax = max_nan(__low2float(amax2), __high2float(amax2));
    amax = max_nan(amax, fabsf(xt));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    if constexpr (kThreads > 32) {
        if ((tid & 31) == 0) red[tid >> 5] = amax;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) amax = max_nan(amax, red[w]);
    }
    const bool fine = amax < INFINITY;
    const float s = fine ? __fmul_rn(amax, 1.0f / 127.0f) : __int_as_float(0x7fffffff);
    if (tid == 0) a.scale[t] = s;
    const bool live = fine && s > 0.0f;
    const bool quick = s > 1e-30f;
    const float r = quick ? __fdiv_rn(1.0f, s) : 0.0f;
    auto put = [&](const uint4& x, int i) {
        float f[kPer];
        Elems<kBf16>::unpack(x, f);
        uint32_t w[kPer / 4];
        codes_of<kPer>(f, s, r, quick, live, w);
        if constexpr (kBf16) reinterpret_cast<uint2*>(q)[i] = make_uint2(w[0], w[1]);
        else reinterpret_cast<uint32_t*>(q)[i] = w[0];
    };
#pragma unroll
    for (int u = 0; u < kVecs; ++u)
        if (u * kThreads + tid < nvec) put(v[u], u * kThreads + tid);
    rest([&](const uint4& x, int i) { if (i < nvec) put(x, i); });
    if (tail < a.K) q[tail] = live ? (int8_t)code_of(xt, s) : (int8_t)0;
}

// ---- host side ---------------------------------------------------------------------------------------
// i8 [rows x K] with row pitch `ld` bytes; boxes of 128 codes x box_rows rows, 128B swizzle, zeros outside.
static int make_map(CUtensorMap* map, const void* base, long long rows, int K, long long ld, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return fail(DPPO_ERR_CUDA, "linear_i8: cuTensorMapEncodeTiled is not available from this driver");
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kBK, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(DPPO_ERR_CUDA, "linear_i8: cuTensorMapEncodeTiled failed with %d", (int)r);
    return DPPO_OK;
}

template <bool kBf16, int kThreads, int kVecs> static int launch_quantize(const QuantArgs& a, cudaStream_t s) {
    constexpr int kCta = kThreads < 128 ? 128 : kThreads, kTeams = kCta / kThreads;
    return launch_after("quantize_rows_i8 launch", quantize_rows_kernel<kBf16, kThreads, kVecs>, (a.rows_max + kTeams - 1) / kTeams, kCta, 0, s, 1, a);
}

// Which team per row, by its length in vectors: the row in registers where that takes no more than eight loads a thread, small
// teams where the rows are many (the reduction and the launch of each CTA count), large ones where they are few and a row's
// latency counts.  bf16: 16,000 x 1,024 14 us with warps, 19 with 128 threads of one load, 26 of four; 64 x 4,096 2.3 with 512
// threads, 3.1 with 128, 16,000 of them 81 and 41; 1,000 x 16,384 18 with 512, 22 with 128.  f32, whose loads bring half the
// work, in eight: 16,000 x 4,096 48 us (6.8 TB/s), 65 in four with a second read; 16,000 x 8,192 93 with 256 threads, 135 with
// 128 of four.  Longer rows are read twice whatever the team (1,000 x 28,672 bf16: 28 us in rounds of two, 31 of four).
template <bool kBf16> static int run_quantize(const QuantArgs& a, cudaStream_t s) {
    const int nvec = a.K / Elems<kBf16>::kPerVec;
    const long long M = a.rows_max, sms = sm_count();
    if (nvec <= 64 && M >= 4 * sms) return launch_quantize<kBf16, 32, 4>(a, s);
    if (nvec <= 128 && M >= 13 * sms) return launch_quantize<kBf16, 32, 4>(a, s);
    if (nvec <= 128) return launch_quantize<kBf16, 128, 1>(a, s);
    if constexpr (kBf16) {
        if (nvec <= 256) return launch_quantize<kBf16, 128, 2>(a, s);
        if (nvec <= 512) return M <= 2 * sms ? launch_quantize<kBf16, 512, 1>(a, s) : launch_quantize<kBf16, 128, 4>(a, s);
        if (nvec <= 1024) return M <= 4 * sms ? launch_quantize<kBf16, 512, 2>(a, s) : launch_quantize<kBf16, 256, 4>(a, s);
        if (nvec <= 2048) return M <= 8 * sms ? launch_quantize<kBf16, 512, 4>(a, s) : launch_quantize<kBf16, 256, 4>(a, s);
        return launch_quantize<kBf16, 512, 2>(a, s);
    } else {
        if (nvec <= 256) return M >= 13 * sms ? launch_quantize<kBf16, 32, 8>(a, s) : launch_quantize<kBf16, 128, 2>(a, s);
        if (nvec <= 512) return launch_quantize<kBf16, 128, 4>(a, s);
        if (nvec <= 1024) return M <= 2 * sms ? launch_quantize<kBf16, 512, 2>(a, s) : launch_quantize<kBf16, 128, 8>(a, s);
        if (nvec <= 2048) return launch_quantize<kBf16, 256, 8>(a, s);
        return launch_quantize<kBf16, 512, 8>(a, s);
    }
}

// Raises a kernel's shared-memory limit once per device.
template <class Kernel> static int raise_smem(Kernel kernel, size_t bytes, bool (&done)[64]) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); dev = -1; }
    if (dev >= 0 && done[dev]) return DPPO_OK;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(e, "linear_i8: shared memory attribute"); }
    if (dev >= 0) done[dev] = true;
    return DPPO_OK;
}

// ---- which kernel, which tile ----
// Both kernels' times in microseconds, fitted to 420 random shapes of 1 to 3,000 tokens, N = 100 to 160,000 and K = 64 to
// 17,000: over those the choice costs 0.5 % against the faster kernel of each, 40 % at worst (52 tokens x 21,152 x 6,652).
//
// Pair kernel: whole waves of tiles.  A 128-code slab of a tile takes 300 ns, bound by fetching the weights' 16 KB, until the
// tensor cores take longer (256 tokens: 380); a wave ends with an epilogue.  The token tile is the one with the least time
// (1,003 x 5,003 x 2,563: 140 tiles of 160 in two waves instead of 80 of 256 in two; 19.3 -> 18.6 us).
static double pair_time(long long M, int N, int n_ksteps, int* tile) {
    const long long n_m2 = (N + 255) / 256, pairs = sm_count() / 2 > 0 ? sm_count() / 2 : 1;
    double best = 0.0;
    for (int tn = kTileN; tn >= 64; tn -= 32) {
        const long long tiles = n_m2 * ((M + tn - 1) / tn), waves = (tiles + pairs - 1) / pairs;
        const double slab = tn * 0.0015 > 0.3 ? tn * 0.0015 : 0.3;
        const double t = 2.9 + (double)waves * (n_ksteps * slab + 0.3 + 0.011 * tn);
        if (best == 0.0 || t < best) { best = t; *tile = tn; }
    }
    return best;
}
// The other, with the split of the contraction that takes least (400 random shapes: 1 % from the best on average; splitting
// until there are two CTAs per SM was 5 %: 64 x 4,096 x 4,096 in four 7.8 us, in eight 9.0).  A slab costs its latency, or,
// where two CTAs share an SM, what the SM can fetch (75 KB/us); each CTA starts and ends, later with a second one beside it;
// a join grows with the CTAs that take part and with the tokens.
static double small_time(long long M, int N, int n_ksteps, int* tokens, int* split) {
    const int nb = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128;
    const long long tiles = (long long)((N + kTileM - 1) / kTileM) * ((M + nb - 1) / nb), sms = sm_count();
    const double latency = 0.25 + 0.00075 * nb, fetch = 2 * (16384 + nb * 128) / 75e3;
    double best = 0.0;
    for (int sp = 1, i = 0; sp <= 8; sp *= 2, ++i) {
        constexpr double kJoin[4] = {0.0, 0.3, 0.4, 0.9};
        const long long ctas = tiles * sp;
        if (sp > 1 && (ctas > 2 * sms || n_ksteps < sp)) break;
        const bool two = ctas > sms;
        const double waves = ctas <= 2 * sms ? 1.0 : (double)ctas / (double)(2 * sms) + 0.4;
        const double slab = two && fetch > latency ? fetch : latency;
        const double t = waves * (((n_ksteps + sp - 1) / sp) * slab + 3.0 + 0.0075 * nb) + (two ? 1.8 : 0.0)
                       + (sp > 1 ? kJoin[i] + 0.017 * nb : 0.0);
        if (best == 0.0 || t < best) { best = t; *split = sp; }
    }
    *tokens = nb;
    return best;
}

template <bool kBf16> static int launch_pair(const CUtensorMap& mw, const CUtensorMap& mx, const Args& a, cudaStream_t s) {
    auto kernel = linear_i8_pair_kernel<kBf16>;
    static bool raised[64];
    const int rc = raise_smem(kernel, kDynSmem2, raised);
    if (rc != DPPO_OK) return rc;
    const long long work = (long long)((a.N + 255) / 256) * ((a.M_max + a.tile_n - 1) / a.tile_n), most = sm_count() / 2;
    return launch_after("linear_i8 launch", kernel, 2 * (work < most ? work : most), kThreads, kDynSmem2, s, 2, mw, mx, a);
}

template <int kNB, bool kBf16> static int launch_small(const CUtensorMap& mw, const CUtensorMap& mx, const Args& a, int split, cudaStream_t s) {
    auto kernel = linear_i8_small_kernel<kNB, kBf16>;
    static bool raised[64];
    const int rc = raise_smem(kernel, small_smem<kNB>(), raised);
    if (rc != DPPO_OK) return rc;
    const int n_ch = (a.N + kTileM - 1) / kTileM;
    const long long tiles = (long long)n_ch * ((a.M_max + kNB - 1) / kNB);
    if (tiles * split > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "linear_i8: too many tiles");
    // four more epilogue warps where they have work: they shorten a join or a wide epilogue (16 x 1,024 x 1,024: 5.3 -> 4.7 us)
    // and only cost their launch elsewhere (1 x 151,936 x 2,560: 62 -> 65)
    const int threads = split > 1 || kNB >= 64 ? kThreads : kThreads - 128;
    return launch_after("linear_i8 launch", kernel, tiles * split, threads, small_smem<kNB>(), s, split, mw, mx, a, n_ch, split);
}

template <bool kBf16> static int launch(bool pair, int nb, int split, const CUtensorMap& mw, const CUtensorMap& mx, const Args& a, cudaStream_t s) {
    if (pair) return launch_pair<kBf16>(mw, mx, a, s);
    switch (nb) {
        case 16: return launch_small<16, kBf16>(mw, mx, a, split, s);
        case 32: return launch_small<32, kBf16>(mw, mx, a, split, s);
        case 64: return launch_small<64, kBf16>(mw, mx, a, split, s);
        default: return launch_small<128, kBf16>(mw, mx, a, split, s);
    }
}

}  // namespace i8
}  // namespace dppo

extern "C" int dppo_quantize_rows_i8(const dppo_quantize_params* p, const void* x, int8_t* q, float* scale,
                                     const int32_t* n_rows_dev, int32_t* status, void* stream) {
    dppo::NvtxRange nvtx_range("dppo_quantize_rows_i8");
    using namespace dppo;
    (void)status;
    if (!p) return fail(DPPO_ERR_INVALID_ARG, "quantize_rows_i8: NULL params");
    if (p->rows_max < 0 || p->K < 1) return fail(DPPO_ERR_INVALID_ARG, "quantize_rows_i8: rows_max=%lld K=%d", (long long)p->rows_max, p->K);
    if (p->dtype != DPPO_F32 && p->dtype != DPPO_BF16) return fail(DPPO_ERR_UNSUPPORTED, "quantize_rows_i8: dtype %d", p->dtype);
    if (p->x_stride < p->K || p->q_stride < p->K)
        return fail(DPPO_ERR_BAD_SHAPE, "quantize_rows_i8: strides %lld, %lld < K %d", (long long)p->x_stride, (long long)p->q_stride, p->K);
    if (p->rows_max >= ((int64_t)1 << 31)) return fail(DPPO_ERR_BAD_SHAPE, "quantize_rows_i8: rows_max must be below 2^31");
    if (p->K > (1 << 30)) return fail(DPPO_ERR_BAD_SHAPE, "quantize_rows_i8: K=%d, the limit is 2^30", p->K);
    const long long x_row_bytes = (long long)p->x_stride * (p->dtype == DPPO_BF16 ? 2 : 4);
    if (p->rows_max == 0) return DPPO_OK;
    if (!x || !q || !scale) return fail(DPPO_ERR_INVALID_ARG, "quantize_rows_i8: NULL array");
    if (((uintptr_t)x & 15) || ((uintptr_t)q & 15) || x_row_bytes % 16 != 0 || p->q_stride % 16 != 0)
        return fail(DPPO_ERR_MISALIGNED, "quantize_rows_i8: x / q base and row strides must be multiples of 16 bytes");
    const i8::QuantArgs a = {(const char*)x, q, scale, n_rows_dev, p->rows_max, x_row_bytes, p->q_stride, p->K};
    return p->dtype == DPPO_BF16 ? i8::run_quantize<true>(a, (cudaStream_t)stream) : i8::run_quantize<false>(a, (cudaStream_t)stream);
}

extern "C" int dppo_linear_i8(const dppo_linear_i8_params* p, const int8_t* x, const float* x_scale, const int8_t* w,
                              const float* w_scale, void* out, const int32_t* n_rows_dev, int32_t* status, void* stream) {
    dppo::NvtxRange nvtx_range("dppo_linear_i8");
    using namespace dppo;
    if (!p) return fail(DPPO_ERR_INVALID_ARG, "linear_i8: NULL params");
    if (p->M_max < 0 || p->N < 1 || p->K < 1)
        return fail(DPPO_ERR_INVALID_ARG, "linear_i8: M_max=%lld N=%d K=%d", (long long)p->M_max, p->N, p->K);
    if (p->out_dtype != DPPO_F32 && p->out_dtype != DPPO_BF16) return fail(DPPO_ERR_UNSUPPORTED, "linear_i8: out_dtype %d", p->out_dtype);
    if (p->K > 131071) return fail(DPPO_ERR_BAD_SHAPE, "linear_i8: K=%d, the int32 sums are exact up to 131071", p->K);
    if (p->N > 0x7fffff00) return fail(DPPO_ERR_BAD_SHAPE, "linear_i8: N=%d", p->N);
    if (p->x_stride < p->K || p->w_stride < p->K || p->out_stride < p->N)
        return fail(DPPO_ERR_BAD_SHAPE, "linear_i8: strides %lld, %lld, %lld for K=%d N=%d", (long long)p->x_stride, (long long)p->w_stride,
                    (long long)p->out_stride, p->K, p->N);
    if (p->M_max >= ((int64_t)1 << 31) - 256) return fail(DPPO_ERR_BAD_SHAPE, "linear_i8: M_max too large");
    const int variant = p->variant >= 100 ? p->variant - 100 : p->variant;
    if (variant < 0 || variant > 2 || p->variant == 100) return fail(DPPO_ERR_INVALID_ARG, "linear_i8: variant %d", p->variant);
    if (p->M_max == 0) return DPPO_OK;
    if (!x || !x_scale || !w || !w_scale || !out) return fail(DPPO_ERR_INVALID_ARG, "linear_i8: NULL array");
    if (((uintptr_t)x & 15) || ((uintptr_t)w & 15) || p->x_stride % 16 != 0 || p->w_stride % 16 != 0)
        return fail(DPPO_ERR_MISALIGNED, "linear_i8: x / w base and row strides must be multiples of 16 bytes");
    if (p->x_stride >= (1ll << 40) || p->w_stride >= (1ll << 40)) return fail(DPPO_ERR_BAD_SHAPE, "linear_i8: strides of x and w must be below 2^40");

    i8::Args a = {};
    a.x_scale = x_scale; a.w_scale = w_scale; a.out = out; a.n_rows_dev = n_rows_dev; a.status = status;
    a.M_max = p->M_max; a.out_stride = p->out_stride;
    a.N = p->N; a.n_ksteps = (p->K + i8::kBK - 1) / i8::kBK; a.out_bf16 = p->out_dtype == DPPO_BF16;
    a.wait_limit_ns = p->variant >= 100 ? kSelfTestWaitLimitNs : kDefaultWaitLimitNs;
    a.test_extra_tx = p->variant >= 100 ? 16 : 0;
    int nb = 0, split = 1;
    const double t_pair = i8::pair_time(p->M_max, p->N, a.n_ksteps, &a.tile_n), t_small = i8::small_time(p->M_max, p->N, a.n_ksteps, &nb, &split);
    const bool pair = variant == 1 || (variant == 0 && t_pair < t_small);
    if (pair) nb = a.tile_n / 2;
    alignas(64) CUtensorMap mw, mx;
    int rc = i8::make_map(&mw, w, p->N, p->K, p->w_stride, i8::kTileM);
    if (rc == DPPO_OK) rc = i8::make_map(&mx, x, p->M_max, p->K, p->x_stride, nb);
    if (rc != DPPO_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    return a.out_bf16 ? i8::launch<true>(pair, nb, split, mw, mx, a, s) : i8::launch<false>(pair, nb, split, mw, mx, a, s);
}
