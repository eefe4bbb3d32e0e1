// Matrix product in 8-bit floating point (e4m3) with a scale for each block of 128 of the contraction, on the 5th-generation
// tensor cores: out[t, n] = sum_B sx[B, t] sw[n / 128, B] sum_{k in B} x[t, k] w[n, k]; and the quantisation that makes its
// operands (a scale per token and 128 values; per 128 x 128 of the weights).
//
// A block of 128 codes is one 128-byte swizzle row: one stage of the TMA ring, four instructions (tcgen05.mma kind::f8f6f4, f32
// accumulation) into a tensor-memory accumulator of its own.  The epilogue warps read that accumulator back while the next
// block's products run, and add it, times its scales, to f32 sums in their registers.
//
// Two kernels.
//   many tokens: persistent CTA pairs (cta_group::2), 256 tokens x up to 256 channels per tile.  The tokens take the M side (TMEM lanes): a
//     thread of the epilogue then holds 128 channels of one token, which share one weight scale, so a block's factor is ONE number per
//     thread.  That matters because shared memory is what the tensor cores read their operands from: with the channels on the
//     lanes the factors came as 16 shared-memory loads per warp and block, and the products waited for the epilogue (2,048 x 2,560
//     x 151,936: 1,260 us).  A tile's outputs leave through shared memory by tiled copies that run under the next tile's products.
//   few tokens (bound by reading the weights): a CTA per 128 channels, 16 to 128 tokens on the N side, so that few tokens waste
//     nothing; the contraction is split over the CTAs of a cluster when there are too few tiles to keep all SMs reading, and the
//     partial sums are joined in a fixed order through distributed shared memory.
// The tokens' scales of a block travel with its codes, through a ring of their own that is longer than the codes' (kSlots > stages +
// accumulators + 1): a slot is then read long before its turn comes again, with no barrier.
// Every wait is bounded; on a time-out the CTA reports DPPO_STATUS_TIMEOUT, leaves its loops, lets copies and products
// in flight finish (bounded), frees its tensor memory and returns.
#include <cuda_fp8.h>

#include <type_traits>

#include "common.cuh"
#include "grpo_loss.cuh"
#include "tensor_core.cuh"

namespace dppo {
using namespace packed;

namespace f8 {

constexpr int kBK = 128;                  // codes of a block = of a stage
constexpr int kTileM = 128;               // rows of the M side per CTA
constexpr int kTileN = 256;               // most channels per tile of the pair kernel
constexpr int kBytesA = kTileM * kBK;
constexpr int kMaxStages = 6;             // + 2 accumulators + 1 < kSlots
constexpr int kSlots = 16;                // blocks whose token scales are in shared memory
constexpr int kEpiWarps = 8;              // pair kernel: two per TMEM lane quarter, half of the tile's channels each
constexpr int kThreads = 128 + 32 * kEpiWarps;     // producer, MMA, watch and one idle warp before them
constexpr int kTokenGroup = 8;            // token tiles swept together (2,048 tokens: 5 MB of codes at K = 2,560)
constexpr int kRingBytes = 4 * (kBytesA + kTileN / 2 * kBK);
constexpr int kStageOut = 8192;           // an epilogue warp's outputs on their way: 256 bytes of each of its 32 tokens
constexpr int kSlotBytes2 = kTileM * 4;   // pair kernel: of this CTA's tokens
constexpr size_t kDynSmem2 = (size_t)kRingBytes + kEpiWarps * kStageOut + kSlots * kSlotBytes2 + 1024;

struct Args {
    const float* w_scale;
    void* out;
    const int32_t* n_rows_dev;
    int32_t* status;
    long long M_max, out_stride, ws_stride;
    int N, n_ksteps;
    int tile_n;                           // pair kernel: channels per tile, 128 or 256
    int vec_out;                          // out: base and rows on 16 bytes
    unsigned long long wait_limit_ns;
    int test_extra_tx;
};

// Instruction descriptor of kind::f8f6f4: D = f32, A = B = e4m3, both K-major.
__host__ __device__ constexpr uint32_t idesc(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

__device__ __forceinline__ long long true_rows(const Args& a) {
    return a.n_rows_dev ? min((long long)max(*a.n_rows_dev, 0), a.M_max) : a.M_max;
}
__device__ __forceinline__ void init_bar(unsigned long long* bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(lm_smem_u32(bar)), "r"(count));
}

// A warp's bounded wait: warp-uniform outcome, since what follows is executed by all 32 lanes together.
__device__ __forceinline__ bool warp_wait(unsigned long long* bar, uint32_t parity, volatile int* abort_flag, unsigned long long limit_ns) {
    if (__all_sync(0xffffffffu, lm_try(lm_smem_u32(bar), parity))) return true;
    return __all_sync(0xffffffffu, lm_wait(lm_smem_u32(bar), parity, abort_flag, limit_ns));
}

// lm_wait for two barriers, looked at together: two looks one after the other are 500 cycles while the tensor cores read shared memory.
__device__ __forceinline__ bool test_both(uint32_t bar0, uint32_t parity0, uint32_t bar1, uint32_t parity1) {
    uint32_t d0, d1;
    asm volatile("{\n\t.reg .pred p, q;\n\t"
                 "mbarrier.test_wait.parity.shared::cta.b64 p, [%2], %3;\n\t"
                 "mbarrier.test_wait.parity.shared::cta.b64 q, [%4], %5;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t"
                 "selp.u32 %1, 1, 0, q;\n\t}"
                 : "=r"(d0), "=r"(d1) : "r"(bar0), "r"(parity0), "r"(bar1), "r"(parity1) : "memory");
    return (d0 & d1) != 0;
}
__device__ __forceinline__ bool wait_both(uint32_t bar0, uint32_t parity0, uint32_t bar1, uint32_t parity1, volatile int* abort_flag,
                                          unsigned long long limit_ns) {
    if (test_both(bar0, parity0, bar1, parity1)) return true;
    const unsigned long long t0 = lm_global_ns();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 16; ++i)
            if (test_both(bar0, parity0, bar1, parity1)) return true;
        if (*abort_flag) return false;
        if (lm_global_ns() - t0 > limit_ns) { *abort_flag = 1; return false; }
    }
}

// kCount consecutive tokens t0 .. of this lane's channel.
template <bool kBf16, int kCount> __device__ __forceinline__ void store_tokens(const Args& a, long long t0, long long T, int ch, const float* acc) {
    typedef typename std::conditional<kBf16, __nv_bfloat16, float>::type Out;
    const int nt = (int)min((long long)kCount, T - t0);
    if (ch >= a.N) return;
    Out* p = reinterpret_cast<Out*>(a.out) + t0 * a.out_stride + ch;
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
        Out o;
        if constexpr (kBf16) o = __float2bfloat16_rn(acc[i]); else o = acc[i];
        if (i < nt) *p = o;
        p += a.out_stride;
    }
}

// 32 columns of this thread's TMEM lane, asked for; columns_wait waits for every load of the thread, and nothing that uses
// the registers moves ahead of it.
__device__ __forceinline__ void columns_load(uint32_t (&v)[32], uint32_t taddr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
                   "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
                   "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void columns_wait(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]),
                   "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
                   "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31]) :: "memory");
}
// Tiles at the edges, and outputs whose rows are not on 16 bytes: 64 bytes (16 f32 or 32 bf16 channels from ch on) of each of the warp's
// 32 tokens t0 + lane, through shared memory (`stage`, this warp's), where piece p of a token's 64 bytes is at 64 lane + 16 (p ^ (lane / 2 mod 4)), without bank conflicts.
template <bool kBf16> __device__ __forceinline__ void store_piece(const Args& a, long long t0, long long T, int ch, int lane, const f32x2* acc, uint32_t stage) {
    typedef typename std::conditional<kBf16, __nv_bfloat16, float>::type Out;
    constexpr int kPer = 16 / (int)sizeof(Out);
    __syncwarp();                                                        // the piece before this one has been read
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x0, x1;
            if constexpr (kBf16) {
                unpair(acc[4 * p + i], x0, x1);
                const __nv_bfloat162 h = __floats2bfloat162_rn(x0, x1);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                unpair(acc[2 * p + i / 2], x0, x1);
                w[i] = __float_as_uint(i & 1 ? x1 : x0);
            }
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                     :: "r"(stage + (uint32_t)(lane * 64 + ((p ^ (lane >> 1 & 3)) * 16))), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
    __syncwarp();
    // consecutive lanes, consecutive channels; eight loads at a time before their stores
    constexpr int kCh = 4 * kPer, kBatch = 8;
    typedef typename std::conditional<kBf16, unsigned short, float>::type Bits;
    Out* out = reinterpret_cast<Out*>(a.out) + t0 * a.out_stride + ch;
#pragma unroll 1
    for (int i0 = 0; i0 < kCh; i0 += kBatch) {
        Bits v[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int t = ((i0 + i) * 32 + lane) / kCh, c = lane % kCh;
            const uint32_t at = stage + (uint32_t)(t * 64 + (((c / kPer) ^ (t >> 1 & 3)) * 16) + c % kPer * (int)sizeof(Out));
            if constexpr (kBf16) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v[i]) : "r"(at) : "memory");
            else asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[i]) : "r"(at) : "memory");
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int t = ((i0 + i) * 32 + lane) / kCh, c = lane % kCh;
            if (t0 + t >= T || ch + c >= a.N) continue;
            if constexpr (kBf16) out[t * a.out_stride + c] = __ushort_as_bfloat16(v[i]);
            else out[t * a.out_stride + c] = v[i];
        }
    }
}

// 256 bytes of outputs (64 f32 or 128 bf16 channels) of each of the warp's 32 tokens, in two boxes of 128 bytes laid out as a
// 128B-swizzled tiled copy reads them.
template <bool kBf16> __device__ __forceinline__ void stage_boxes(int lane, const f32x2* acc, uint32_t stage) {
#pragma unroll
    for (int p = 0; p < 16; ++p) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x0, x1;
            if constexpr (kBf16) {
                unpair(acc[4 * p + i], x0, x1);
                const __nv_bfloat162 h = __floats2bfloat162_rn(x0, x1);
                w[i] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                unpair(acc[2 * p + i / 2], x0, x1);
                w[i] = __float_as_uint(i & 1 ? x1 : x0);
            }
        }
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};"
                     :: "r"(stage + (uint32_t)((p >> 3) * 4096 + lane * 128 + (((p & 7) ^ (lane & 7)) * 16))), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    }
}

// ---- many tokens: CTA pairs ---------------------------------------------------------------------------
// 2,048 x 2,560 x 151,936 into bf16: 778 us on a rested board, 2.0 PFLOP/s (930 us in a long run, under the power limit), where the products alone would
// take 464 at the rate of a plain product; into f32 995 in a long run.  What bounds it is the epilogue: each of its eight warps serves every block, one
// step after the other (barrier, tensor-memory reads, release, sums), 0.61 us for a block of 256 x 256 whose products alone take about 0.35.  With tiles
// of 128 channels a block takes 0.47 us instead of half of that, with two accumulators or with four, so it is not their number.  Sixteen epilogue
// warps, two instructions of half the channels each, and epilogue warps that look at the barriers themselves were slower (907, 880 and 976 us).
struct Shared2 {
    unsigned long long full[kMaxStages];
    unsigned long long empty[kMaxStages];
    unsigned long long acc_full[2];
    unsigned long long acc_empty[2];      // the leader's copy counts the epilogue warps of both CTAs
    unsigned long long drain;             // products in flight on an early way out
    uint32_t tmem_base;
    int abort;
};
static_assert(kDynSmem2 + sizeof(Shared2) <= 232448, "the ring must fit one CTA's shared memory");

// Tile j of this pair: token tiles are taken kTokenGroup at a time; within a group the token tiles of one channel tile
// follow each other, so that every weight is fetched once per group and the group's codes stay in L2.
__device__ __forceinline__ bool tile_of(uint32_t j, int n_ch, int n_tok, int& ch, int& tok) {
    const long long id = (long long)(blockIdx.x >> 1) + (long long)j * (gridDim.x >> 1);
    if (id >= (long long)n_ch * n_tok) return false;
    const long long per = (long long)kTokenGroup * n_ch;
    const int g = (int)(id / per), local = (int)(id - (long long)g * per);
    const int t0 = g * kTokenGroup, width = min(kTokenGroup, n_tok - t0);
    ch = local / width;
    tok = t0 + local - ch * width;
    return true;
}

template <bool kBf16>
__global__ void __launch_bounds__(kThreads, 1)
linear_f8_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_s,
                      const __grid_constant__ CUtensorMap map_out, const Args a) {
    extern __shared__ unsigned char f8_raw[];
    __shared__ Shared2 sh;
    const uint32_t tiles = (lm_smem_u32(f8_raw) + 1023u) & ~1023u, slots = tiles + (uint32_t)(kRingBytes + kEpiWarps * kStageOut);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint32_t rank;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const bool leader = rank == 0;
    volatile int* abort_flag = &sh.abort;
    const int n_ch = (a.N + a.tile_n - 1) / a.tile_n;
    // a stage: 128 codes of K of this CTA's 128 tokens and of its half of the channels
    const uint32_t stage_bytes = (uint32_t)(kBytesA + a.tile_n / 2 * kBK);
    const uint32_t stages = min((uint32_t)kMaxStages, (uint32_t)kRingBytes / stage_bytes);

    if (tid == 0) {
        sh.abort = 0;
        for (uint32_t s = 0; s < stages; ++s) { init_bar(&sh.full[s], 1); init_bar(&sh.empty[s], 1); }
        for (int b = 0; b < 2; ++b) { init_bar(&sh.acc_full[b], 1); init_bar(&sh.acc_empty[b], 2 * kEpiWarps); }
        init_bar(&sh.drain, 1);
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
    const int n_tok = (int)((T + 2 * kTileM - 1) / (2 * kTileM));

    // registers: launched with 168 a thread, 64,512 in all; 128 x 72 + 256 x 216 are as many
    if (warp < 4) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer (both CTAs)
        if (lane == 0) {
            uint32_t it = 0, s = 0, use = 0;
            int ch, tok;
            for (uint32_t j = 0; tile_of(j, n_ch, n_tok, ch, tok) && !*abort_flag; ++j) {
                const int row_x = (2 * tok + (int)rank) * kTileM, row_w = ch * a.tile_n + (int)rank * (a.tile_n / 2);
                for (int k = 0; k < a.n_ksteps; ++k, ++it, s = s + 1 == stages ? 0 : s + 1, use += s == 0 ? 1 : 0) {
                    if (use > 0 && !lm_wait(lm_smem_u32(&sh.empty[s]), (use - 1) & 1, abort_flag, a.wait_limit_ns)) break;
                    const uint32_t bar_local = lm_smem_u32(&sh.full[s]), bar = bar_local & kPeerMask;
                    const uint32_t dst = tiles + s * stage_bytes;
                    if (leader)                                        // the leader's barrier collects both CTAs' bytes
                        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                                     :: "r"(bar_local), "r"(2 * (stage_bytes + (uint32_t)kSlotBytes2) + (it == 0 ? (uint32_t)a.test_extra_tx : 0u)) : "memory");
                    lm_tma_2d_pair(dst, &map_x, bar, k * kBK, row_x, 0);
                    lm_tma_2d_pair(dst + kBytesA, &map_w, bar, k * kBK, row_w, 0);
                    lm_tma_2d_pair(slots + (it % kSlots) * kSlotBytes2, &map_s, bar, row_x, k, 0);
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
            uint32_t s = 0, use = 0, it = 0;
            int ch, tok;
            bool ok = true;
            for (uint32_t j = 0; ok && tile_of(j, n_ch, n_tok, ch, tok) && !*abort_flag; ++j) {
                for (int k = 0; k < a.n_ksteps; ++k, ++it, s = s + 1 == stages ? 0 : s + 1, use += s == 0 ? 1 : 0) {
                    const uint32_t b = it & 1, use_b = it >> 1;
                    const uint32_t full = lm_smem_u32(&sh.full[s]), empty = lm_smem_u32(&sh.acc_empty[b]);
                    // Tiles of 128 channels: the looks themselves count (705 x 7,681 x 2,000 31.0 us, 32.9 one after the other); of 256 the
                    // suspended wait is better (1,024 x 2,560 x 20,000 60.4, both polled 62.7).
                    if (a.tile_n < kTileN && use_b > 0) ok = wait_both(full, use & 1, empty, (use_b - 1) & 1, abort_flag, a.wait_limit_ns);
                    else ok = lm_wait(full, use & 1, abort_flag, a.wait_limit_ns)
                              && (use_b == 0 || lm_wait(empty, (use_b - 1) & 1, abort_flag, a.wait_limit_ns));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t d_tmem = tmem_base + b * kTileN;
                    const uint64_t dx = lm_smem_desc_k(tiles + s * stage_bytes), dw = lm_smem_desc_k(tiles + s * stage_bytes + kBytesA);
#pragma unroll
                    for (int kk = 0; kk < kBK / 32; ++kk) {              // 32 codes of K per instruction
                        asm volatile("{\n\t.reg .pred p;\n\t"
                                     "setp.ne.b32 p, %4, 0;\n\t"
                                     "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                                     :: "r"(d_tmem), "l"(dx + kk * 2), "l"(dw + kk * 2), "r"(desc), "r"(kk > 0 ? 1u : 0u) : "memory");
                    }
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                                 :: "r"(lm_smem_u32(&sh.acc_full[b])), "h"((unsigned short)3) : "memory");
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                                 :: "r"(lm_smem_u32(&sh.empty[s])), "h"((unsigned short)3) : "memory");
                }
            }
            if (!ok || *abort_flag) {                                  // products already issued finish before memory goes away
                asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(lm_smem_u32(&sh.drain)) : "memory");
                lm_wait_plain(lm_smem_u32(&sh.drain), 0, a.wait_limit_ns);
            }
        }
    } else if (warp == 2) {
        // ------------------------------------------------------------------ watch (both CTAs): hands finished accumulators on to the epilogue
        // The epilogue's warps wait at a hardware barrier, which costs a tenth of a look at an mbarrier while the tensor cores keep
        // shared memory busy (250 cycles, of 650 that a block's products take).  This warp meets them there at every accumulator, so
        // neither side is ever more than one ahead.  After a time-out it no longer looks before it goes there: the epilogue runs to
        // its end, over whatever is there.
        uint32_t it = 0;
        int ch, tok;
        for (uint32_t j = 0; tile_of(j, n_ch, n_tok, ch, tok); ++j) {
            for (int k = 0; k < a.n_ksteps; ++k, ++it) {
                if (!*abort_flag) lm_wait(lm_smem_u32(&sh.acc_full[it & 1]), (it >> 1) & 1, abort_flag, a.wait_limit_ns);
                __syncwarp();
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                asm volatile("bar.sync 1, %0;" :: "n"(32 + 32 * kEpiWarps) : "memory");
            }
        }
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ epilogue (warps 4..11, both CTAs)
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int q = warp & 3, half = (warp - 4) >> 2;                  // TMEM lane quarter of this warp; which half of the channels
        const bool wide = a.tile_n == kTileN;                            // 128 channels per warp and token, or 64
        const int blocks = wide ? 4 : 2, first = half * (a.tile_n / 2);  // blocks of 32 channels, the first of them
        const uint32_t stage = tiles + (uint32_t)kRingBytes + (uint32_t)((warp - 4) * kStageOut);
        uint32_t it = 0;
        int ch, tok;
        auto handed_on = [&]() {
            asm volatile("bar.sync 1, %0;" :: "n"(32 + 32 * kEpiWarps) : "memory");
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        };
        for (uint32_t j = 0; tile_of(j, n_ch, n_tok, ch, tok); ++j) {
            const long long t0 = (2ll * tok + (int)rank) * kTileM + q * 32;
            const int ch0 = ch * a.tile_n + first;
            // the channels' scales of 32 blocks, one per lane; 0 past the last channel
            const float* ws = a.w_scale + (ch0 < a.N ? (long long)(ch0 / kBK) * a.ws_stride : 0);
            float sw32 = ch0 < a.N && lane < a.n_ksteps ? ws[lane] : 0.0f;
            f32x2 acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = 0ull;
            const uint32_t lanes = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)first;
            const uint32_t my_slot = slots + (uint32_t)((q * 32 + lane) * 4);
            float sx;                                                    // the token's scale, asked for a block ahead
            auto ask_scale = [&](uint32_t n) { asm volatile("ld.shared.f32 %0, [%1];" : "=f"(sx) : "r"(my_slot + (n % kSlots) * kSlotBytes2) : "memory"); };
            uint32_t v[2][32];
            handed_on();
            columns_load(v[0], lanes + (it & 1) * kTileN);
            columns_load(v[1], lanes + (it & 1) * kTileN + 32u);
            ask_scale(it);
#pragma unroll 1
            for (int k = 0; k < a.n_ksteps; ++k, ++it) {
                const uint32_t b = it & 1, taddr = lanes + b * kTileN;
                if ((k & 31) == 0 && k > 0) sw32 = ch0 < a.N && k + lane < a.n_ksteps ? ws[k + lane] : 0.0f;
                const float f1 = sx * __shfl_sync(0xffffffffu, sw32, k & 31);
                const f32x2 f = pair_of(f1, f1);
                auto add = [&](int c, const uint32_t (&w)[32]) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        acc[16 * c + i] = fma2(pair_of(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])), f, acc[16 * c + i]);
                };
                // two blocks of columns under way at a time; the next accumulator's first two before this one's last sums are done
                columns_wait(v[0]);
                columns_wait(v[1]);
                if (wide) {
                    add(0, v[0]);
                    columns_load(v[0], taddr + 64u);
                    add(1, v[1]);
                    columns_load(v[1], taddr + 96u);
                    columns_wait(v[0]);
                    columns_wait(v[1]);
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                if (lane == 0)                                           // all read: the leader's MMA thread waits for every epilogue warp
                    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(lm_smem_u32(&sh.acc_empty[b]) & kPeerMask) : "memory");
                __syncwarp();
                const bool more = k + 1 < a.n_ksteps;
                if (more) {
                    handed_on();
                    ask_scale(it + 1);
                }
                const uint32_t next = lanes + ((it + 1) & 1) * kTileN;
                if (wide) add(2, v[0]); else add(0, v[0]);
                if (more) columns_load(v[0], next);
                if (wide) add(3, v[1]); else add(1, v[1]);
                if (more) columns_load(v[1], next + 32u);
            }
            // tiled copies write whole boxes, or boxes cut at the last of M_max rows: at the last channel they are cut on 16 bytes only
            if (a.vec_out && ch0 + a.tile_n / 2 <= a.N && (t0 + 32 <= T || (t0 < T && T == a.M_max))) {
                constexpr int kBox = kBf16 ? 64 : 32;                    // channels of a box
#pragma unroll
                for (int r = 0; r < (kBf16 ? 1 : 2); ++r) {
                    if (2 * r * kBox >= a.tile_n / 2) break;
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();                                        // the boxes before these have been read
                    stage_boxes<kBf16>(lane, acc + 32 * r, stage);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
#pragma unroll
                        for (int g = 2 * r; g < 2 * r + 2; ++g)
                            if (g * kBox < a.tile_n / 2)
                                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                                             :: "l"(&map_out), "r"(ch0 + g * kBox), "r"((int)t0), "r"(stage + (uint32_t)((g & 1) * 4096)) : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                }
            } else if (t0 < T) {
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (c >= blocks || ch0 + 32 * c >= a.N) break;
                    store_piece<kBf16>(a, t0, T, ch0 + 32 * c, lane, acc + 16 * c, stage);
                    if constexpr (!kBf16) store_piece<kBf16>(a, t0, T, ch0 + 32 * c + 16, lane, acc + 16 * c + 8, stage);
                }
            }
            __syncwarp();
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");      // all outputs are written
        __syncwarp();
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
// 1 x 2,560 x 151,936: 65 us, 6.0 TB/s of weights; 64 x 4,096 x 4,096 in 9.5 us, where four CTAs share a tile and a CTA's eight blocks of
// 0.4 us each, its start and the join are what takes time.
template <int kNB> struct Small {
    static constexpr int kStages = kNB <= 16 ? 6 : kNB <= 32 ? 5 : kNB <= 64 ? 4 : 6;        // two CTAs per SM, but one of 128 tokens
    static constexpr int kPerSm = kNB <= 64 ? 2 : 1;
    static constexpr int kStageBytes = kBytesA + kNB * kBK;
    static constexpr int kPitch = kNB < 32 ? 32 : kNB;                                       // TMEM columns between accumulators
    static constexpr int kBufs = 256 / kPitch > 8 ? 8 : 256 / kPitch;
    static constexpr int kHalves = kNB >= 64 ? 2 : 1;                                        // epilogue warps per lane quarter
    static constexpr int kThreads = 128 + kHalves * 128;
    static constexpr int kCols = kNB / kHalves;                                              // tokens of an epilogue warp
    static constexpr int kChunk = kCols < 32 ? kCols : 32;
    static constexpr int kSlotBytes = kNB * 4 < 128 ? 128 : kNB * 4;
    static constexpr size_t kDynSmem = (size_t)kStages * kStageBytes + kSlots * kSlotBytes + 1024;
    static_assert(kStages + kBufs + 1 < kSlots, "a slot's turn comes again too soon");
    struct Shared {
        unsigned long long full[kStages];
        unsigned long long empty[kStages];
        unsigned long long acc_full[kBufs];
        unsigned long long acc_empty[kBufs];
        unsigned long long done;
        uint32_t tmem_base;
        int abort;
    };
};

// 16 columns of this thread's TMEM lane.
__device__ __forceinline__ void tmem_load16(uint32_t (&v)[16], uint32_t taddr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

template <int kNB, bool kBf16>
__global__ void __launch_bounds__(Small<kNB>::kThreads, Small<kNB>::kPerSm)
linear_f8_small_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_s,
                       const Args a, int n_ch, int split) {
    typedef Small<kNB> S;
    extern __shared__ unsigned char f8_raw[];
    __shared__ typename S::Shared sh;
    const uint32_t tiles = (lm_smem_u32(f8_raw) + 1023u) & ~1023u, slots = tiles + (uint32_t)(S::kStages * S::kStageBytes);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &sh.abort;
    const int part = (int)(blockIdx.x % (unsigned)split);                 // rank in the cluster: clusters are consecutive CTAs
    const int id = (int)(blockIdx.x / (unsigned)split);
    const int m = id % n_ch;
    const long long t_tile = (long long)(id / n_ch) * kNB;
    const int k0 = (int)((long long)a.n_ksteps * part / split), k1 = (int)((long long)a.n_ksteps * (part + 1) / split);

    if (tid == 0) {
        sh.abort = 0;
        for (int s = 0; s < S::kStages; ++s) { init_bar(&sh.full[s], 1); init_bar(&sh.empty[s], 1); }
        for (int b = 0; b < S::kBufs; ++b) { init_bar(&sh.acc_full[b], 1); init_bar(&sh.acc_empty[b], 4 * S::kHalves); }
        init_bar(&sh.done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    enter_kernel();
    const long long T = true_rows(a);
    if (t_tile >= T) return;                                              // the whole cluster leaves together
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(lm_smem_u32(&sh.tmem_base)), "r"(256u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = sh.tmem_base;

    const int q = warp & 3, row = q * 32 + lane, half = (warp - 4) >> 2;
    const int ch = m * kTileM + row;
    float acc[S::kCols];
    bool live = false;
    if (warp == 0) {
        if (lane == 0) {
            int it = 0;
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it % S::kStages, use = it / S::kStages;
                if (use > 0 && !lm_wait(lm_smem_u32(&sh.empty[s]), (use - 1) & 1, abort_flag, a.wait_limit_ns)) break;
                const uint32_t bar = lm_smem_u32(&sh.full[s]), dst = tiles + s * S::kStageBytes;
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;"
                             :: "r"(bar), "r"((uint32_t)(S::kStageBytes + kNB * 4) + (it == 0 ? (uint32_t)a.test_extra_tx : 0u)) : "memory");
                lm_tma_2d(dst, &map_w, bar, k * kBK, m * kTileM, 0);
                lm_tma_2d(dst + kBytesA, &map_x, bar, k * kBK, (int)t_tile, 0);
                lm_tma_2d(slots + (uint32_t)(it % kSlots * S::kSlotBytes), &map_s, bar, (int)t_tile, k, 0);
            }
            if (*abort_flag) {
                const int pending = it < S::kStages ? it : S::kStages;
                for (int i = 0; i < pending; ++i) {
                    const int i2 = it - 1 - i;
                    lm_wait_plain(lm_smem_u32(&sh.full[i2 % S::kStages]), (i2 / S::kStages) & 1, a.wait_limit_ns);
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            int it = 0;
            for (int k = k0; k < k1; ++k, ++it) {
                const int s = it % S::kStages, use = it / S::kStages, b = it % S::kBufs, use_b = it / S::kBufs;
                if (use_b > 0 && !lm_wait(lm_smem_u32(&sh.acc_empty[b]), (use_b - 1) & 1, abort_flag, a.wait_limit_ns)) break;
                if (!lm_wait(lm_smem_u32(&sh.full[s]), use & 1, abort_flag, a.wait_limit_ns)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint64_t dw = lm_smem_desc_k(tiles + s * S::kStageBytes), dx = lm_smem_desc_k(tiles + s * S::kStageBytes + kBytesA);
#pragma unroll
                for (int kk = 0; kk < kBK / 32; ++kk) {
                    asm volatile("{\n\t.reg .pred p;\n\t"
                                 "setp.ne.b32 p, %4, 0;\n\t"
                                 "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
                                 :: "r"(tmem_base + (uint32_t)(b * S::kPitch)), "l"(dw + kk * 2), "l"(dx + kk * 2), "r"(idesc(kTileM, kNB)), "r"(kk > 0 ? 1u : 0u) : "memory");
                }
                asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(lm_smem_u32(&sh.acc_full[b])) : "memory");
                asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(lm_smem_u32(&sh.empty[s])) : "memory");
            }
            // all products issued so far (on an early way out too: they finish before memory goes away)
            asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(lm_smem_u32(&sh.done)) : "memory");
            lm_wait_plain(lm_smem_u32(&sh.done), 0, a.wait_limit_ns);
        }
    } else if (warp >= 4) {
#pragma unroll
        for (int i = 0; i < S::kCols; ++i) acc[i] = 0.0f;
        live = true;
        const float* ws = a.w_scale + (long long)m * a.ws_stride;
        float next_sw = k0 < k1 ? ws[k0] : 0.0f;
        uint32_t it = 0;
#pragma unroll 1
        for (int k = k0; k < k1; ++k, ++it) {
            const uint32_t b = it % S::kBufs;
            const float sw = next_sw;
            if (k + 1 < k1) next_sw = ws[k + 1];
            live = warp_wait(&sh.acc_full[b], (it / S::kBufs) & 1, abort_flag, a.wait_limit_ns);
            if (!live) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + b * S::kPitch + (uint32_t)(half * S::kCols);
            const uint32_t f = slots + it % kSlots * S::kSlotBytes + (uint32_t)(half * S::kCols * 4);
#pragma unroll
            for (int c = 0; c < S::kCols / S::kChunk; ++c) {
                uint32_t v[S::kChunk];
                if constexpr (S::kChunk == 32) lm_tmem_load32(v, taddr + (uint32_t)(c * 32)); else tmem_load16(v, taddr);
#pragma unroll
                for (int i = 0; i < S::kChunk; i += 4) {
                    float4 sx;
                    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(sx.x), "=f"(sx.y), "=f"(sx.z), "=f"(sx.w)
                                 : "r"(f + (uint32_t)(c * S::kChunk + i) * 4u) : "memory");
                    float* o = acc + c * S::kChunk + i;
                    o[0] = fmaf(__uint_as_float(v[i]), sx.x * sw, o[0]);
                    o[1] = fmaf(__uint_as_float(v[i + 1]), sx.y * sw, o[1]);
                    o[2] = fmaf(__uint_as_float(v[i + 2]), sx.z * sw, o[2]);
                    o[3] = fmaf(__uint_as_float(v[i + 3]), sx.w * sw, o[3]);
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) lm_arrive(lm_smem_u32(&sh.acc_empty[b]));
        }
        live = live && !__any_sync(0xffffffffu, *abort_flag);
        if (live) {
            if (split == 1) {
#pragma unroll
                for (int c = 0; c < S::kCols / S::kChunk; ++c) {
                    const long long t0 = t_tile + half * S::kCols + c * S::kChunk;
                    if (t0 < T) store_tokens<kBf16, S::kChunk>(a, t0, T, ch, acc + c * S::kChunk);
                }
            } else {
                // partial sums to shared memory, [token][channel], in the ring: nothing reads or writes that any more, the last
                // block's products being complete
#pragma unroll
                for (int i = 0; i < S::kCols; ++i)
                    asm volatile("st.shared.f32 [%0], %1;" :: "r"(tiles + (uint32_t)((half * S::kCols + i) * kTileM + row) * 4u), "f"(acc[i]) : "memory");
            }
        }
        __syncwarp();
    }
    if (split > 1) {
        __syncwarp();
        lm_cluster_sync();                                               // every CTA's sums are in its shared memory
        if (live) {
            // this CTA's share of the tokens: part, part + split, ...; all of a token's partial sums are under way together
            const int n_tok = (int)min((long long)kNB, T - t_tile);
            for (int c = part + half * split; c < n_tok; c += S::kHalves * split) {
                float x[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    x[r] = 0.0f;
                    if (r < split) {
                        uint32_t remote;
                        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(tiles + (uint32_t)(c * kTileM + row) * 4u), "r"(r));
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x[r]) : "r"(remote) : "memory");
                    }
                }
                const float y = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
                if (ch < a.N) {
                    if constexpr (kBf16) reinterpret_cast<__nv_bfloat16*>(a.out)[(t_tile + c) * a.out_stride + ch] = __float2bfloat16_rn(y);
                    else reinterpret_cast<float*>(a.out)[(t_tile + c) * a.out_stride + ch] = y;
                }
            }
        }
        __syncwarp();
        lm_cluster_sync();                                               // the others have read this CTA's shared memory
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (tid == 0 && sh.abort) set_status(a.status, DPPO_STATUS_TIMEOUT);
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"(256u) : "memory");
    }
}

// ---- quantisation -------------------------------------------------------------------------------------
// One read, one write: rows, 8,192 x 4,096 f32 27-33 us (6.3-5.1 TB/s), bf16 23-29 (4.3-3.5, bound by its instructions); 128 x 128, 43-51 and 29-34:
// a CTA loads a block, joins its maximum, writes and leaves, and only other CTAs' loads run under that (once per set of weights).
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

struct QuantArgs {
    const char* x;
    uint8_t* q;
    float* scale;
    const int32_t* n_rows_dev;
    long long rows_max, x_row_bytes, q_stride, scale_stride;
    int K, n_blocks;
};

// Two codes.
__device__ __forceinline__ uint32_t codes2(float a, float b) { return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3); }
// What a block's maximum makes of it: its scale, and the reciprocal's neighbours.
struct Scale {
    float s, lo, hi;
    bool fine;                            // no NaN or infinity in the block
};
__device__ __forceinline__ Scale scale_of(float amax) {
    Scale r;
    r.fine = amax < INFINITY;
    r.s = r.fine ? fmaxf(__fmul_rn(amax, 1.0f / 448.0f), 1.17549435e-38f) : __int_as_float(0x7fffffff);
    const float inv = __fdividef(1.0f, r.s);
    r.lo = inv * (1.0f - 0x1p-21f);
    r.hi = inv * (1.0f + 0x1p-21f);
    return r;
}
// The codes of kPer values, 4 per word.  The quotient x / s lies strictly between x lo and x hi (1 / s is off by 2^-22 of it at most, the
// roundings of the products by 2^-24 each), and rounding to a code is monotonous: where both ends have the same code, so has the quotient.  A
// vector where they differ (one in ten thousand) is divided out.
template <int kPer> __device__ __forceinline__ void codes_of(const float (&f)[kPer], const Scale& sc, uint32_t (&w)[kPer / 4]) {
    uint32_t diff = 0;
    const f32x2 lo = pair_of(sc.lo, sc.lo), hi = pair_of(sc.hi, sc.hi);
#pragma unroll
    for (int j = 0; j < kPer; j += 4) {
        float a0, a1, a2, a3, b0, b1, b2, b3;
        unpair(mul2(pair_of(f[j], f[j + 1]), lo), a0, a1);
        unpair(mul2(pair_of(f[j + 2], f[j + 3]), lo), a2, a3);
        unpair(mul2(pair_of(f[j], f[j + 1]), hi), b0, b1);
        unpair(mul2(pair_of(f[j + 2], f[j + 3]), hi), b2, b3);
        w[j / 4] = codes2(a0, a1) | codes2(a2, a3) << 16;
        diff |= w[j / 4] ^ (codes2(b0, b1) | codes2(b2, b3) << 16);
    }
    if (diff != 0 || !sc.fine) {
#pragma unroll
        for (int j = 0; j < kPer; j += 4)
            w[j / 4] = sc.fine ? codes2(__fdiv_rn(f[j], sc.s), __fdiv_rn(f[j + 1], sc.s)) | codes2(__fdiv_rn(f[j + 2], sc.s), __fdiv_rn(f[j + 3], sc.s)) << 16 : 0u;
    }
}
// kPer values of a row from element e0 on; 0 past its end.  Whole vectors in one load.
template <bool kBf16> __device__ __forceinline__ uint4 load_part(const char* row, int e0, int K) {
    constexpr int kPer = Elems<kBf16>::kPerVec;
    if (e0 + kPer <= K) return *reinterpret_cast<const uint4*>(row + (size_t)e0 * (16 / kPer));
    float f[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) f[j] = e0 + j < K ? Elems<kBf16>::load1(row, e0 + j) : 0.0f;
    return Elems<kBf16>::pack(f);
}
// The largest magnitude of a vector, and of several lanes' (bf16: of each half of a word, joined at the end).
template <bool kBf16> __device__ __forceinline__ uint32_t amax_join(uint32_t a, uint32_t b) {
    if constexpr (kBf16) {
        const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
        return *reinterpret_cast<const uint32_t*>(&m);
    } else {
        return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b)));
    }
}
template <bool kBf16> __device__ __forceinline__ uint32_t amax_vec(const uint4& v) {
    constexpr uint32_t kMag = kBf16 ? 0x7fff7fffu : 0x7fffffffu;
    return amax_join<kBf16>(amax_join<kBf16>(v.x & kMag, v.y & kMag), amax_join<kBf16>(v.z & kMag, v.w & kMag));
}
template <bool kBf16> __device__ __forceinline__ float amax_value(uint32_t m) {
    if constexpr (kBf16) return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    else return __uint_as_float(m);
}
template <bool kBf16> __device__ __forceinline__ void store_codes(uint8_t* row, int e0, int K, const uint4& v, const Scale& sc) {
    constexpr int kPer = Elems<kBf16>::kPerVec;
    float f[kPer];
    uint32_t w[kPer / 4];
    Elems<kBf16>::unpack(v, f);
    codes_of<kPer>(f, sc, w);
    if (e0 + kPer <= K) {
        if constexpr (kBf16) *reinterpret_cast<uint2*>(row + e0) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(row + e0) = w[0];
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (e0 + j < K) row[e0 + j] = (uint8_t)(w[j / 4] >> (8 * (j & 3)));
    }
}

// A scale per row and 128 columns: 16 lanes (bf16) or 32 (f32) hold a block, one vector each; kUnroll blocks of a row at a time.
template <bool kBf16, int kUnroll> __global__ void __launch_bounds__(128) quantize_f8_rows_kernel(const QuantArgs a, int groups) {
    constexpr int kPer = Elems<kBf16>::kPerVec, kTeam = kBK / kPer, kTeams = 128 / kTeam;
    enter_kernel();
    const long long T = a.n_rows_dev ? min((long long)*a.n_rows_dev, a.rows_max) : a.rows_max;
    const long long item = (long long)blockIdx.x * kTeams + threadIdx.x / kTeam;
    const long long t = item / groups;
    const int b0 = (int)(item - t * groups) * kUnroll, l = threadIdx.x % kTeam;
    const char* row = a.x + t * a.x_row_bytes;
    const bool whole_blocks = __all_sync(0xffffffffu, (b0 + kUnroll) * kBK <= a.K);       // one way for both teams of a warp
    if (t >= T) return;                                            // a whole team
    const unsigned team = kTeam == 32 ? 0xffffffffu : 0xffffu << (threadIdx.x & 16);
    float* scale = a.scale + (long long)b0 * a.scale_stride + t;
    uint8_t* codes = a.q + t * a.q_stride;
    auto block = [&](const uint4& v, int u, bool whole) {
        uint32_t m = amax_vec<kBf16>(v);
#pragma unroll
        for (int o = kTeam / 2; o > 0; o >>= 1) m = amax_join<kBf16>(m, __shfl_xor_sync(team, m, o));
        const Scale sc = scale_of(amax_value<kBf16>(m));
        const int e0 = (b0 + u) * kBK + l * kPer;
        if (l == 0) scale[u * a.scale_stride] = sc.s;
        if (whole || e0 < a.K) store_codes<kBf16>(codes, e0, whole ? e0 + kPer : a.K, v, sc);
    };
    uint4 v[kUnroll];
    if (whole_blocks) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) v[u] = *reinterpret_cast<const uint4*>(row + (size_t)((b0 + u) * kBK + l * kPer) * (16 / kPer));
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) block(v[u], u, true);
    } else {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int e0 = (b0 + u) * kBK + l * kPer;
            v[u] = e0 < a.K ? load_part<kBf16>(row, e0, a.K) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (b0 + u < a.n_blocks) block(v[u], u, false);
    }
}

// A scale per 128 x 128: a CTA holds the block in registers.
template <bool kBf16> __global__ void __launch_bounds__(256) quantize_f8_blocks_kernel(const QuantArgs a) {
    constexpr int kPer = Elems<kBf16>::kPerVec, kTeam = kBK / kPer, kRows = 256 / kTeam, kVecs = kBK / kRows;
    __shared__ float red[8];
    enter_kernel();
    const long long T = a.n_rows_dev ? min((long long)*a.n_rows_dev, a.rows_max) : a.rows_max;
    const long long br = blockIdx.x / (unsigned)a.n_blocks, r0 = br * kBK + threadIdx.x / kTeam;
    const int bk = (int)(blockIdx.x - br * a.n_blocks), e0 = bk * kBK + (int)(threadIdx.x % kTeam) * kPer;
    if (br * kBK >= T) return;
    uint4 v[kVecs];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const long long t = r0 + i * kRows;
        v[i] = t < T && e0 < a.K ? load_part<kBf16>(a.x + t * a.x_row_bytes, e0, a.K) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) most = amax_join<kBf16>(most, amax_vec<kBf16>(v[i]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = amax_join<kBf16>(most, __shfl_xor_sync(0xffffffffu, most, o));
    float m = amax_value<kBf16>(most);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max_nan(m, red[w]);
    const Scale sc = scale_of(m);
    if (threadIdx.x == 0) a.scale[br * a.scale_stride + bk] = sc.s;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const long long t = r0 + i * kRows;
        if (t < T && e0 < a.K) store_codes<kBf16>(a.q + t * a.q_stride, e0, a.K, v[i], sc);
    }
}

// ---- host side ---------------------------------------------------------------------------------------
template <bool kBf16, int kUnroll> static int run_quantize_rows(const QuantArgs& a, cudaStream_t s) {
    constexpr int kTeams = kBf16 ? 8 : 4;
    const int groups = (a.n_blocks + kUnroll - 1) / kUnroll;
    const long long ctas = (a.rows_max * groups + kTeams - 1) / kTeams;
    if (ctas > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "quantize_f8: too many blocks");
    return launch_after("quantize_f8 launch", quantize_f8_rows_kernel<kBf16, kUnroll>, ctas, 128, 0, s, 1, a, groups);
}
template <bool kBf16> static int run_quantize(const QuantArgs& a, int block_rows, cudaStream_t s) {
    // Few blocks: one at a time, more CTAs (64 x 4,096 bf16 1.8 us, four at a time 2.9; 2,048 x 2,560 6.5 and 5.6)
    if (block_rows == 1) return a.rows_max * a.n_blocks <= 100ll * sm_count() ? run_quantize_rows<kBf16, 1>(a, s) : run_quantize_rows<kBf16, 4>(a, s);
    const long long ctas = (a.rows_max + kBK - 1) / kBK * a.n_blocks;
    if (ctas > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "quantize_f8: too many blocks");
    return launch_after("quantize_f8 launch", quantize_f8_blocks_kernel<kBf16>, ctas, 256, 0, s, 1, a);
}

// e4m3 [rows x K] with row pitch `ld` bytes; boxes of 128 codes x box_rows rows, 128B swizzle, zeros outside.
static int make_map(CUtensorMap* map, const void* base, long long rows, int K, long long ld, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return fail(DPPO_ERR_CUDA, "linear_f8: cuTensorMapEncodeTiled is not available from this driver");
    const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {(cuuint32_t)kBK, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(DPPO_ERR_CUDA, "linear_f8: cuTensorMapEncodeTiled failed with %d", (int)r);
    return DPPO_OK;
}

// The tokens' scales, f32 [blocks x tokens] with `ld` elements between blocks: boxes of `tokens` of one block.
static int make_scale_map(CUtensorMap* map, const float* base, long long rows, int blocks, long long ld, int tokens) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return fail(DPPO_ERR_CUDA, "linear_f8: cuTensorMapEncodeTiled is not available from this driver");
    const cuuint64_t dims[2] = {(cuuint64_t)rows, (cuuint64_t)blocks};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * 4};
    const cuuint32_t box[2] = {(cuuint32_t)tokens, 1};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, const_cast<float*>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(DPPO_ERR_CUDA, "linear_f8: cuTensorMapEncodeTiled failed with %d", (int)r);
    return DPPO_OK;
}

// The outputs, boxes of 128 bytes x 32 tokens, 128B swizzle (written: nothing outside them).
static int make_out_map(CUtensorMap* map, void* base, long long rows, int N, long long ld, bool bf16) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return fail(DPPO_ERR_CUDA, "linear_f8: cuTensorMapEncodeTiled is not available from this driver");
    const cuuint64_t dims[2] = {(cuuint64_t)N, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)ld * (bf16 ? 2 : 4)};
    const cuuint32_t box[2] = {bf16 ? 64u : 32u, 32};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, base, dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(DPPO_ERR_CUDA, "linear_f8: cuTensorMapEncodeTiled failed with %d", (int)r);
    return DPPO_OK;
}

// Raises a kernel's shared-memory limit once per device.
template <class Kernel> static int raise_smem(Kernel kernel, size_t bytes, bool (&done)[64]) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); dev = -1; }
    if (dev >= 0 && done[dev]) return DPPO_OK;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(e, "linear_f8: shared memory attribute"); }
    if (dev >= 0) done[dev] = true;
    return DPPO_OK;
}

// ---- which kernel, which tile ----
// Both kernels' times in microseconds, fitted to measurements.
//
// Pair kernel: whole waves of tiles.  A block of a tile of 256 channels takes 0.61 us, of 128 channels 0.47 (its way to the epilogue and back);
// a wave ends with its outputs, which take longer where tiled copies cannot write them.
static double pair_time(long long M, int N, int n_ksteps, bool bf16, bool tiled, int* tile) {
    const long long n_tok = (M + 255) / 256, pairs = sm_count() / 2 > 0 ? sm_count() / 2 : 1;
    const double store = !tiled ? 0.027 : bf16 ? 0.010 : 0.016;
    double best = 0.0;
    for (int tn = kTileN; tn >= 128; tn /= 2) {
        const long long tiles = n_tok * ((N + tn - 1) / tn), waves = (tiles + pairs - 1) / pairs;
        const double t = 3.4 + (double)waves * (n_ksteps * (tn == 256 ? 0.61 : 0.47) + store * tn);
        if (best == 0.0 || t < best) { best = t; *tile = tn; }
    }
    return best;
}
// The other, with the split of the contraction that takes least.  A block costs its latency, or, as far as two CTAs share an SM, what the SM can
// fetch (75 KB/us); each CTA starts and ends, later with a second one beside it; a join grows with the tokens, one of eight CTAs also with how
// many of them there are.
static double small_time(long long M, int N, int n_ksteps, int* tokens, int* split) {
    const int nb = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128;
    const long long tiles = (long long)((N + kTileM - 1) / kTileM) * ((M + nb - 1) / nb), sms = sm_count();
    const double latency = 0.30 + 0.0016 * nb, fetch = 2 * (16384 + nb * 128) / 75e3;
    const int per_sm = nb <= 64 ? 2 : 1;
    double best = 0.0;
    for (int sp = 1, i = 0; sp <= 8; sp *= 2, ++i) {
        const long long ctas = tiles * sp;
        const double joins[4] = {0.0, 0.3 + 0.017 * nb, 0.4 + 0.017 * nb, 0.2 + nb * (0.002 + 0.040 * (double)ctas / (double)sms)};
        if (sp > 1 && (ctas > per_sm * sms || n_ksteps < sp)) break;
        const double shared = per_sm == 1 || ctas <= sms ? 0.0 : ctas >= 2 * sms ? 1.0 : (double)(ctas - sms) / (double)sms;
        const double waves = per_sm == 1 ? (double)((ctas + sms - 1) / sms) : ctas <= 2 * sms ? 1.0 : (double)ctas / (double)(2 * sms) + 0.4;
        const double slab = latency + (fetch > latency ? shared * (fetch - latency) : 0.0);
        const double t = waves * (((n_ksteps + sp - 1) / sp) * slab + 3.0 + 0.0075 * nb) + 1.8 * shared + joins[i];
        if (best == 0.0 || t < best) { best = t; *split = sp; }
    }
    *tokens = nb;
    return best;
}

template <bool kBf16> static int launch_pair(const CUtensorMap& mw, const CUtensorMap& mx, const CUtensorMap& ms, const CUtensorMap& mo, const Args& a, cudaStream_t s) {
    auto kernel = linear_f8_pair_kernel<kBf16>;
    static bool raised[64];
    const int rc = raise_smem(kernel, kDynSmem2, raised);
    if (rc != DPPO_OK) return rc;
    const long long work = (long long)((a.N + a.tile_n - 1) / a.tile_n) * ((a.M_max + 2 * kTileM - 1) / (2 * kTileM)), most = sm_count() / 2;
    return launch_after("linear_f8 launch", kernel, 2 * (work < most ? work : most), kThreads, kDynSmem2, s, 2, mw, mx, ms, mo, a);
}

template <int kNB, bool kBf16> static int launch_small(const CUtensorMap& mw, const CUtensorMap& mx, const CUtensorMap& ms, const Args& a, int split, cudaStream_t s) {
    auto kernel = linear_f8_small_kernel<kNB, kBf16>;
    static bool raised[64];
    const int rc = raise_smem(kernel, Small<kNB>::kDynSmem, raised);
    if (rc != DPPO_OK) return rc;
    const int n_ch = (a.N + kTileM - 1) / kTileM;
    const long long tiles = (long long)n_ch * ((a.M_max + kNB - 1) / kNB);
    if (tiles * split > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "linear_f8: too many tiles");
    return launch_after("linear_f8 launch", kernel, tiles * split, Small<kNB>::kThreads, Small<kNB>::kDynSmem, s, split, mw, mx, ms, a, n_ch, split);
}

template <bool kBf16> static int launch(bool pair, int nb, int split, const CUtensorMap& mw, const CUtensorMap& mx, const CUtensorMap& ms, const CUtensorMap& mo,
                                        const Args& a, cudaStream_t s) {
    if (pair) return launch_pair<kBf16>(mw, mx, ms, mo, a, s);
    switch (nb) {
        case 16: return launch_small<16, kBf16>(mw, mx, ms, a, split, s);
        case 32: return launch_small<32, kBf16>(mw, mx, ms, a, split, s);
        case 64: return launch_small<64, kBf16>(mw, mx, ms, a, split, s);
        default: return launch_small<128, kBf16>(mw, mx, ms, a, split, s);
    }
}

}  // namespace f8
}  // namespace dppo

extern "C" int dppo_quantize_f8(const dppo_quantize_f8_params* p, const void* x, uint8_t* q, float* scale,
                                const int32_t* n_rows_dev, int32_t* status, void* stream) {
    dppo::NvtxRange nvtx_range("dppo_quantize_f8");
    using namespace dppo;
    (void)status;
    if (!p) return fail(DPPO_ERR_INVALID_ARG, "quantize_f8: NULL params");
    if (p->rows_max < 0 || p->K < 1) return fail(DPPO_ERR_INVALID_ARG, "quantize_f8: rows_max=%lld K=%d", (long long)p->rows_max, p->K);
    if (p->dtype != DPPO_F32 && p->dtype != DPPO_BF16) return fail(DPPO_ERR_UNSUPPORTED, "quantize_f8: dtype %d", p->dtype);
    if (p->block_rows != 1 && p->block_rows != 128) return fail(DPPO_ERR_UNSUPPORTED, "quantize_f8: block_rows %d (1 or 128)", p->block_rows);
    if (p->K > (1 << 30)) return fail(DPPO_ERR_BAD_SHAPE, "quantize_f8: K=%d, the limit is 2^30", p->K);
    if (p->rows_max >= ((int64_t)1 << 31)) return fail(DPPO_ERR_BAD_SHAPE, "quantize_f8: rows_max must be below 2^31");
    const int n_blocks = (p->K + f8::kBK - 1) / f8::kBK;
    if (p->x_stride < p->K || p->q_stride < p->K || p->scale_stride < (p->block_rows == 1 ? p->rows_max : (int64_t)n_blocks))
        return fail(DPPO_ERR_BAD_SHAPE, "quantize_f8: strides %lld, %lld, %lld for %lld rows of K=%d", (long long)p->x_stride, (long long)p->q_stride,
                    (long long)p->scale_stride, (long long)p->rows_max, p->K);
    const long long x_row_bytes = (long long)p->x_stride * (p->dtype == DPPO_BF16 ? 2 : 4);
    if (p->rows_max == 0) return DPPO_OK;
    if (!x || !q || !scale) return fail(DPPO_ERR_INVALID_ARG, "quantize_f8: NULL array");
    if (((uintptr_t)x & 15) || ((uintptr_t)q & 15) || x_row_bytes % 16 != 0 || p->q_stride % 16 != 0)
        return fail(DPPO_ERR_MISALIGNED, "quantize_f8: x / q base and row strides must be multiples of 16 bytes");
    const f8::QuantArgs a = {(const char*)x, q, scale, n_rows_dev, p->rows_max, x_row_bytes, p->q_stride, p->scale_stride, p->K, n_blocks};
    return p->dtype == DPPO_BF16 ? f8::run_quantize<true>(a, p->block_rows, (cudaStream_t)stream) : f8::run_quantize<false>(a, p->block_rows, (cudaStream_t)stream);
}

extern "C" int dppo_linear_f8(const dppo_linear_f8_params* p, const uint8_t* x, const float* x_scale, const uint8_t* w,
                              const float* w_scale, void* out, const int32_t* n_rows_dev, int32_t* status, void* stream) {
    dppo::NvtxRange nvtx_range("dppo_linear_f8");
    using namespace dppo;
    if (!p) return fail(DPPO_ERR_INVALID_ARG, "linear_f8: NULL params");
    if (p->M_max < 0 || p->N < 1 || p->K < 1)
        return fail(DPPO_ERR_INVALID_ARG, "linear_f8: M_max=%lld N=%d K=%d", (long long)p->M_max, p->N, p->K);
    if (p->out_dtype != DPPO_F32 && p->out_dtype != DPPO_BF16) return fail(DPPO_ERR_UNSUPPORTED, "linear_f8: out_dtype %d", p->out_dtype);
    if (p->K > (1 << 30)) return fail(DPPO_ERR_BAD_SHAPE, "linear_f8: K=%d, the limit is 2^30", p->K);
    if (p->N > 0x7fffff00) return fail(DPPO_ERR_BAD_SHAPE, "linear_f8: N=%d", p->N);
    const int n_blocks = (p->K + f8::kBK - 1) / f8::kBK;
    if (p->x_stride < p->K || p->w_stride < p->K || p->out_stride < p->N || p->x_scale_stride < p->M_max || p->w_scale_stride < n_blocks)
        return fail(DPPO_ERR_BAD_SHAPE, "linear_f8: strides %lld, %lld, %lld, %lld, %lld for M_max=%lld N=%d K=%d", (long long)p->x_stride,
                    (long long)p->w_stride, (long long)p->out_stride, (long long)p->x_scale_stride, (long long)p->w_scale_stride, (long long)p->M_max, p->N, p->K);
    if (p->M_max >= ((int64_t)1 << 31) - 256) return fail(DPPO_ERR_BAD_SHAPE, "linear_f8: M_max too large");
    const int variant = p->variant >= 100 ? p->variant - 100 : p->variant;
    if (variant < 0 || variant > 2 || p->variant == 100) return fail(DPPO_ERR_INVALID_ARG, "linear_f8: variant %d", p->variant);
    if (p->M_max == 0) return DPPO_OK;
    if (!x || !x_scale || !w || !w_scale || !out) return fail(DPPO_ERR_INVALID_ARG, "linear_f8: NULL array");
    if (((uintptr_t)x & 15) || ((uintptr_t)w & 15) || ((uintptr_t)x_scale & 15) || p->x_stride % 16 != 0 || p->w_stride % 16 != 0 || p->x_scale_stride % 4 != 0)
        return fail(DPPO_ERR_MISALIGNED, "linear_f8: x / w / x_scale base and row strides must be multiples of 16 bytes");
    if (p->x_stride >= (1ll << 40) || p->w_stride >= (1ll << 40) || p->x_scale_stride >= (1ll << 38))
        return fail(DPPO_ERR_BAD_SHAPE, "linear_f8: strides of x, w and x_scale must be below 2^40 bytes");

    f8::Args a = {};
    a.w_scale = w_scale; a.out = out; a.n_rows_dev = n_rows_dev; a.status = status;
    a.M_max = p->M_max; a.out_stride = p->out_stride; a.ws_stride = p->w_scale_stride;
    a.N = p->N; a.n_ksteps = n_blocks;
    const bool bf16 = p->out_dtype == DPPO_BF16;
    a.wait_limit_ns = p->variant >= 100 ? kSelfTestWaitLimitNs : kDefaultWaitLimitNs;
    a.test_extra_tx = p->variant >= 100 ? 16 : 0;
    a.vec_out = ((uintptr_t)out & 15) == 0 && p->out_stride * (bf16 ? 2 : 4) % 16 == 0 && p->out_stride < (1ll << 36);
    int nb = 0, split = 1;
    const double t_pair = f8::pair_time(p->M_max, p->N, n_blocks, bf16, a.vec_out != 0, &a.tile_n);
    const double t_small = f8::small_time(p->M_max, p->N, n_blocks, &nb, &split);
    const bool pair = variant == 1 || (variant == 0 && t_pair < t_small);
    alignas(64) CUtensorMap mw, mx, ms, mo = {};
    int rc = f8::make_map(&mw, w, p->N, p->K, p->w_stride, pair ? a.tile_n / 2 : f8::kTileM);
    if (rc == DPPO_OK) rc = f8::make_map(&mx, x, p->M_max, p->K, p->x_stride, pair ? f8::kTileM : nb);
    if (rc == DPPO_OK) rc = f8::make_scale_map(&ms, x_scale, p->M_max, n_blocks, p->x_scale_stride, pair ? f8::kTileM : nb);
    if (rc == DPPO_OK && pair && a.vec_out) rc = f8::make_out_map(&mo, out, p->M_max, p->N, p->out_stride, bf16);
    if (rc != DPPO_OK) return rc;
    cudaStream_t s = (cudaStream_t)stream;
    return bf16 ? f8::launch<true>(pair, nb, split, mw, mx, ms, mo, a, s) : f8::launch<false>(pair, nb, split, mw, mx, ms, mo, a, s);
}
