// Distillation from a teacher's top log-probs: the loss of each token and its gradient with respect to the student's logits.
//
// The teacher lists K <= 128 tokens i_j of a row with log-probs; p_j = exp of those (mode NORMALIZED: over their sum), and in
// mode REST r = 1 - sum p_j is its probability of everything else.  With the student's s = softmax(z / tau) and sigma = the
// sum of s over what is not listed:
//     loss = sum_j p_j (ln p_j - ln s_{i_j}) [+ r (ln r - ln sigma)]
//     dloss/dz_v = (G s_v - sum_{j: i_j = v} p_j - [v not listed] s_v r / sigma) / tau,      G = sum_j p_j [+ r]
// sigma of a peaked student is small: as 1 - sum s_{i_j} it would have no digits left, so the listed entries are kept OUT of
// the running sum, and S = S_rest + sum_listed exp((z - m) / tau).
//
// Forward alone (distill_forward_kernel): the row streams through registers once, bound by HBM.  Which vectors hold listed entries stands
// in a bitmap in shared memory, four words per warp and round, so an ordinary round pays one 16-byte shared load and a
// test; the marked vectors are left out there, and a warp of its own (which also fetches the teacher's entries and their logits)
// adds the unlisted entries of each from the vector itself.
//
// Loss and gradient together (distill_step_kernel): one read and one write of the row.  A row's slices lie in the shared memory of the CTAs
// of a cluster; the listed entries are set to -inf there, and once the row's sums are known the exponentials leave scaled; the listed
// entries are written last.  Short rows (distill_warp_kernel) do the same in a warp's registers.
//
// Gradient alone (distill_backward_kernel): a map over the row from the forward's {m, S, G, r / sigma}; the listed entries last here too.
#include <cooperative_groups.h>

#include <type_traits>

#include "common.cuh"
#include "grpo_loss.cuh"
#include "row_sweep.cuh"

namespace dppo {
using namespace packed;
namespace cg = cooperative_groups;

namespace distill {
using namespace sweep;

constexpr int kMaxListed = 128;
constexpr int kMaxCluster = 8;
constexpr int kMaxV = 1 << 20;
constexpr double kLeastRest = 1.0 / 65536.0;       // a remainder up to this is the rounding of f32 log-probs: it counts as none
constexpr uint32_t kAll = 0xffffffffu;

struct Args {
    const char* logits;
    const int32_t* ids;
    const float* logp;
    const int32_t* n_tokens_dev;
    const float* weight;                           // gradient: dL/dloss of each row, or NULL (1)
    float *loss, *lse;
    float4* stats;
    const float4* stats_in;
    char* dlogits;
    int32_t* status;
    long long T_max, row_bytes;
    int V, k, mode, in_place;
    int chunks, chunk_vecs;                        // gradient: a row is taken in `chunks` pieces of chunk_vecs vectors
    float c;
    double inv_tau;
};

__device__ __forceinline__ long long rows_of(const Args& a) {
    return a.n_tokens_dev ? min((long long)*a.n_tokens_dev, a.T_max) : a.T_max;
}

// ---- the teacher's entries of a row, by a warp: entry i * 32 + lane in slot i of a lane ------------------
template <int kPer> struct Listed {
    int id[kPer];                                  // -1: no entry
    double p[kPer];                                // 0 where there is none; mode NORMALIZED: relative to the largest
    float top;                                     // (all lanes) that one's log-prob; 0 in the other modes
    float z[kPer];                                 // the student's logit, -inf where there is none
    bool first[kPer];                              // no earlier entry has this id
    bool bad;                                      // (all lanes) an id outside [-1, V)
};

// Asked for, and (when they are needed) looked at: ids outside [-1, V) make the row bad and count as no entry.
template <int kPer> __device__ __forceinline__ void listed_ask(const Args& a, long long t, int lane, Listed<kPer>& e, float (&lp)[kPer]) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int j = i * 32 + lane;
        e.id[i] = j < a.k ? a.ids[t * a.k + j] : -1;
        lp[i] = j < a.k ? a.logp[t * a.k + j] : -INFINITY;
    }
}
template <int kPer> __device__ __forceinline__ void listed_check(const Args& a, Listed<kPer>& e) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        bad = bad || e.id[i] < -1 || e.id[i] >= a.V;
        if (e.id[i] < 0 || e.id[i] >= a.V) e.id[i] = -1;
    }
    e.bad = __any_sync(kAll, bad);
}
template <int kPer> __device__ __forceinline__ void listed_ids(const Args& a, long long t, int lane, Listed<kPer>& e, float (&lp)[kPer]) {
    listed_ask<kPer>(a, t, lane, e, lp);
    listed_check<kPer>(a, e);
}
template <bool kBf16, int kPer> __device__ __forceinline__ void listed_logits(const char* row, Listed<kPer>& e) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) e.z[i] = e.id[i] >= 0 ? Elems<kBf16>::load1(row, e.id[i]) : -INFINITY;
}
template <int kPer> __device__ __forceinline__ void listed_probs(const Args& a, const float (&lp)[kPer], Listed<kPer>& e) {
    e.top = 0.0f;
    if (a.mode == DPPO_DISTILL_NORMALIZED) {       // lists whose probabilities are all far below 1 keep their ratios
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (e.id[i] >= 0 && lp[i] < INFINITY) top = fmaxf(top, lp[i]);
        top = warp_max_f32(top);
        if (top > -INFINITY) e.top = top;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) e.p[i] = e.id[i] >= 0 ? exp64((double)lp[i] - (double)e.top) : 0.0;
}
// Which entries are the first with their id.  together: their p, added up in the order of the entries, goes to the first.  Lists of more than 32
// walk over all of their entries, which costs more than the sweep from about 64 on (2,048 x 151,936 bf16, loss and gradient: 20 entries 243 us, 33
// 322, 64 372, 128 512; loss 112, 132, 130, 133; gradient 192, 218, 229, 336).
template <int kPer> __device__ __forceinline__ void listed_first(const Args& a, int lane, Listed<kPer>& e, bool together) {
    if constexpr (kPer == 1) {                     // mostly no id comes twice
        const unsigned peers = __match_any_sync(kAll, e.id[0]);
        e.first[0] = e.id[0] >= 0 && __ffs(peers) - 1 == lane;
        if (!__any_sync(kAll, e.id[0] >= 0 && !e.first[0])) return;
    }
    double sum[kPer];
    bool first[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) { sum[i] = 0.0; first[i] = e.id[i] >= 0; }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
#pragma unroll 1
        for (int l = 0; l < 32 && i * 32 + l < a.k; ++l) {
            const int o = __shfl_sync(kAll, e.id[i], l);
            const double po = together ? __shfl_sync(kAll, e.p[i], l) : 0.0;
#pragma unroll
            for (int n = 0; n < kPer; ++n) {
                if (o != e.id[n]) continue;
                sum[n] += po;
                if (i * 32 + l < n * 32 + lane) first[n] = false;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        e.first[i] = first[i];
        if (together) e.p[i] = sum[i];             // of an entry that is not the first: not used again
    }
}
__device__ __forceinline__ double warp_sum_f64(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
    return v;
}

// ---- the row's loss from its parts ---------------------------------------------------------------------
// What the teacher's entries alone say (in every lane): formed while the row is under way.
struct Mass {
    double P, lp, z;                               // sums of p, of p ln p and of p (z - zmax); p as in Listed
    float G, r, norm;                              // the listed p times norm are the loss's p
    float zmax;
    bool bad;                                      // a NaN or +inf among the listed logits
};
template <int kPer> __device__ __forceinline__ Mass listed_mass(const Args& a, const Listed<kPer>& e, const float (&lp)[kPer]) {
    Mass m;
    m.zmax = kLowest;
    m.P = m.lp = m.z = 0.0;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        bad = bad || !(e.z[i] < INFINITY);
        if (e.z[i] < INFINITY) m.zmax = fmaxf(m.zmax, e.z[i]);
    }
    m.bad = __any_sync(kAll, bad);
    m.zmax = warp_max_f32(m.zmax);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        m.P += e.p[i];
        if (e.p[i] != 0.0) { m.lp += e.p[i] * ((double)lp[i] - (double)e.top); m.z += e.p[i] * ((double)e.z[i] - (double)m.zmax); }
    }
    m.P = warp_sum_f64(m.P); m.lp = warp_sum_f64(m.lp); m.z = warp_sum_f64(m.z);
    const double r = a.mode == DPPO_DISTILL_REST && 1.0 - m.P > kLeastRest ? 1.0 - m.P : 0.0;
    m.r = (float)r;
    m.norm = 1.0f;
    if (a.mode == DPPO_DISTILL_NORMALIZED) {
        m.norm = m.P > 0.0 ? (float)inv64(m.P) : 0.0f;
        m.G = m.P > 0.0 ? 1.0f : (float)m.P;       // a NaN stays one
    } else {
        m.G = (float)(m.P + r);
    }
    return m;
}

// The row's sums (in every lane), in a few f32 operations: the gradient waits for nothing else.
struct RowSums {
    float M, S, Sr;                                // the largest entry; sums relative to it: all, unlisted
    float to_rest;                                 // gradient of an unlisted entry: its exponential relative to the unlisted entries' maximum times this
    bool bad, empty;
};
// rest: the row without its listed entries.  The exponentials of the listed ones go to ej.
template <int kPer> __device__ __forceinline__ RowSums row_sums(const Args& a, const Listed<kPer>& e, const Mass& m, const Part& rest, float (&ej)[kPer]) {
    RowSums s;
    s.bad = rest.bad || m.bad;
    s.M = fmaxf(rest.m, m.zmax);
    const float shrink = rest.S > 0.0f ? ex2((rest.m - s.M) * a.c) : 0.0f;
    s.Sr = rest.S * shrink;
    float Sl = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        ej[i] = e.id[i] >= 0 ? ex2((e.z[i] - s.M) * a.c) : 0.0f;
        if (e.first[i]) Sl += ej[i];
    }
    s.S = s.Sr + warp_sum(Sl);
    s.empty = !(s.S > 0.0f) && !s.bad;
    const float nan = __int_as_float(0x7fffffff);
    if (s.bad) s.S = nan;
    s.to_rest = s.bad ? nan : rest.S > 0.0f && !e.bad ? m.G * shrink / s.S - m.r / rest.S : 0.0f;
    return s;
}

// What is written of a row, by a warp.  share: r / sigma, or -log2(r / sigma - G) where that is above 16: a large share goes into the entries'
// exponents, since times an exponential that underflows relative to M it would be lost.
__device__ __forceinline__ void row_write(const Args& a, long long t, const Mass& m, const RowSums& s, const Part& rest, bool bad_id, int lane) {
    const float nan = __int_as_float(0x7fffffff);
    const bool shared = m.r > 0.0f && rest.S > 0.0f;
    // two 64-bit logarithms at once, on two lanes: of S, and of r S / (the unlisted sum relative to its own maximum, which does not underflow)
    // or of P
    const double second = shared ? (1.0 - m.P) * (double)s.S * inv64((double)rest.S) : m.P;
    const double logs = log64(lane == 0 ? (double)s.S : second);
    const double l = __shfl_sync(kAll, logs, 0), l2 = __shfl_sync(kAll, logs, 1);
    const double cross = m.lp - (m.z + m.P * ((double)m.zmax - (double)s.M)) * a.inv_tau;      // sum of p (ln p - (z - M) / tau)
    double loss = a.mode == DPPO_DISTILL_NORMALIZED ? (m.P > 0.0 ? cross * inv64(m.P) - l2 + l : m.P) : (m.P != 0.0 ? cross + m.P * l : 0.0);
    float share = 0.0f;
    if (shared) {
        const double ln_share = l2 + ((double)s.M - (double)rest.m) * a.inv_tau;
        loss += (1.0 - m.P) * ln_share;
        share = ln_share < 69.0 ? m.r * s.S / s.Sr : (float)(-1.4426950408889634 * ln_share);
        if (ln_share > 2.8 && ln_share < 69.0) {
            const double over = exp64(ln_share) - (double)m.G;
            if (over > 16.0) share = (float)(-1.4426950408889634 * log64(over));
        }
    } else if (m.r > 0.0f) {
        share = INFINITY;
        loss = INFINITY;
    }
    if (lane != 0) return;
    if (s.empty) loss = m.P > 0.0 ? INFINITY : m.P != 0.0 ? m.P : 0.0;
    if (a.loss) a.loss[t] = s.bad ? nan : bad_id ? 0.0f : (float)loss;
    if (a.lse) a.lse[t] = s.bad ? nan : s.empty ? -INFINITY : (float)((double)s.M * a.inv_tau + l);
    if (a.stats) {
        const bool zero = bad_id && !s.bad;
        a.stats[t] = s.bad ? make_float4(nan, nan, nan, nan) : make_float4(s.empty ? -INFINITY : s.M, s.S, zero ? 0.0f : m.G, zero ? 0.0f : share);
    }
    if (bad_id) set_status(a.status, DPPO_STATUS_BAD_TARGET);
}

// ---- forward: a CTA per row, or the CTAs of a cluster ---------------------------------------------------
template <int kThreads> struct FwdShared {
    Part part[kThreads / 32];
    Part row;
    unsigned tail_listed;                          // of the V % kPerVec entries behind the last vector
};

// Words of the bitmap of a part of n vectors.
template <int kThreads> __host__ __device__ constexpr int bitmap_words(int n) {
    return (n + kRound * kThreads - 1) / (kRound * kThreads) * (kRound * kThreads / 32);
}

template <bool kBf16, int kThreads, int kPer, bool kCluster>
__global__ void __launch_bounds__(kThreads + 32)
distill_forward_kernel(const Args a) {
    constexpr int kLog2 = kBf16 ? 3 : 2, kPerVec = 1 << kLog2, kWarps = kThreads / 32;
    extern __shared__ uint4 bitmap[];
    __shared__ FwdShared<kThreads> sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    wait_for_previous();
    const long long T = rows_of(a);
    unsigned rank = 0, C = 1;
    if constexpr (kCluster) { C = cg::this_cluster().num_blocks(); rank = cg::this_cluster().block_rank(); }
    const int log2C = 31 - __clz((int)C);
    const long long t = (long long)(blockIdx.x >> log2C);
    if (t >= T) return;                                            // the whole cluster leaves together
    const char* row = a.logits + t * a.row_bytes;
    const int nvec = a.V >> kLog2;
    const int v0 = (int)((long long)nvec * rank >> log2C), v1 = (int)((long long)nvec * (rank + 1) >> log2C);
    const bool last = rank == C - 1;
    const int n_rounds = (v1 - v0 + kRound * kThreads - 1) / (kRound * kThreads);

    Listed<kPer> e;
    float lp[kPer];
    uint4 q[kRound];
    auto load = [&](int it) {
        const int i = v0 + it * (kRound * kThreads) + tid;
        if (i - tid + kRound * kThreads <= v1) {
#pragma unroll
            for (int u = 0; u < kRound; ++u) q[u] = load_vec(row + (size_t)(i + u * kThreads) * 16);
        } else {                                                   // the part's last vectors
#pragma unroll
            for (int u = 0; u < kRound; ++u)
                q[u] = i + u * kThreads < v1 ? load_vec(row + (size_t)(i + u * kThreads) * 16) : masked_vec<kBf16>();
        }
    };
    for (int i = tid; i < bitmap_words<kThreads>(v1 - v0) / 4; i += kThreads + 32) bitmap[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 0) sh.tail_listed = 0;
    if (warp == kWarps) listed_ids<kPer>(a, t, lane, e, lp);
    __syncthreads();
    if (warp == kWarps) {
        uint32_t* words = reinterpret_cast<uint32_t*>(bitmap);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int v = e.id[i] >> kLog2, rel = v - v0;
            if (e.id[i] < 0) continue;
            if (v >= nvec) {
                atomicOr(&sh.tail_listed, 1u << (e.id[i] & (kPerVec - 1)));
            } else if (rel >= 0 && v < v1) {
                const int it = rel / (kRound * kThreads), u = rel / kThreads % kRound, w = rel % kThreads >> 5;
                atomicOr(&words[(it * kWarps + w) * kRound + u], 1u << (rel & 31));
            }
        }
    } else if (n_rounds > 0) {
        load(0);                                                   // under way while the bitmap is finished
    }
    __syncthreads();

    if (warp < kWarps) {
        Sum acc;
        sum_init(acc, kLowest, a.c);
        for (int it = 0; it < n_rounds; ++it) {
            if (it > 0) load(it);
            const uint4 b = bitmap[it * kWarps + warp];
            if (b.x | b.y | b.z | b.w) {
                const uint32_t w[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int u = 0; u < kRound; ++u)
                    if (w[u] >> lane & 1u) q[u] = masked_vec<kBf16>();
            }
            sum_vecs<kBf16, kRound>(acc, q, a.c);
        }
        Part p = sum_part(acc);
        if (last && (nvec << kLog2) + tid < a.V && !(sh.tail_listed >> tid & 1u)) part_one(p, Elems<kBf16>::load1(row, (nvec << kLog2) + tid), a.c);
        p = part_warp(p, a.c);
        if (lane == 0) sh.part[warp] = p;
    }
    Part hot = part_none();                                        // the unlisted entries of the marked vectors
    Mass mass = {};
    if (warp == kWarps) {
        listed_probs<kPer>(a, lp, e);
        listed_logits<kBf16, kPer>(row, e);
        int vec[kPer];
        unsigned out[kPer];
        uint4 hv[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int v = e.id[i] >> kLog2;
            vec[i] = e.id[i] >= 0 && v >= v0 && v < v1 ? v : -1;
            out[i] = 0;
            if (vec[i] >= 0) hv[i] = load_vec(row + (size_t)v * 16);
        }
        // the first entry of each marked vector takes it, without what any entry lists there
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
#pragma unroll 1
            for (int l = 0; l < 32 && i * 32 + l < a.k; ++l) {
                const int o = __shfl_sync(kAll, e.id[i], l);
#pragma unroll
                for (int n = 0; n < kPer; ++n) {
                    if (o < 0 || (o >> kLog2) != vec[n]) continue;
                    out[n] |= 1u << (o & (kPerVec - 1));
                    if (i * 32 + l < n * 32 + lane) out[n] |= 1u << 31;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (vec[i] < 0 || out[i] >> 31) continue;
            float f[kPerVec];
            Elems<kBf16>::unpack(hv[i], f);
#pragma unroll
            for (int j = 0; j < kPerVec; ++j)
                if (!(out[i] >> j & 1u)) part_one(hot, f[j], a.c);
        }
        listed_first<kPer>(a, lane, e, false);
        mass = listed_mass<kPer>(a, e, lp);
    }
    __syncthreads();
    Part rest = part_none();
    if (warp == kWarps) {
        if (lane < kWarps) {                                       // kWarps <= 16: one part per lane, then the two joined
            const Part o = sh.part[lane];
            const float M = fmaxf(o.m, hot.m);
            Part x = o;
            part_to(x, M, a.c); part_to(hot, M, a.c);
            rest = {M, x.S + hot.S, x.bad | hot.bad};
        } else {
            rest = hot;
        }
        rest = part_warp(rest, a.c);
    }
    if constexpr (kCluster) {
        cg::cluster_group cl = cg::this_cluster();
        if (warp == kWarps && lane == 0) sh.row = rest;
        cl.sync();                                                 // every CTA's part is in its shared memory
        if (rank != 0) {                                           // ... which lasts until the first CTA has read it
            let_next_start();
            cl.sync();
            return;
        }
        if (warp == kWarps) {
            rest = lane < (int)C ? cl.map_shared_rank(&sh, lane)->row : part_none();
            rest = part_warp(rest, a.c);
        }
        cl.sync();
    }
    let_next_start();
    if (warp == kWarps) {
        float ej[kPer];
        const RowSums sums = row_sums<kPer>(a, e, mass, rest, ej);
        row_write(a, t, mass, sums, rest, e.bad, lane);
    }
}

// ---- loss and gradient, a row in the shared memory of a cluster ------------------------------------------------
template <int kThreads> struct StepShared {
    Part part;                                     // of this CTA's slice, listed entries left out
    float m[kThreads / 32], s[kThreads / 32];
    float scale;                                   // of the exponentials kept in this CTA's slice
    unsigned tail_listed;
};

// The gradient of the listed entries that `here` (a predicate of the vector index) accepts, after everything else of their row.
template <bool kBf16, int kPer, class F>
__device__ __forceinline__ void write_listed(char* out, const Listed<kPer>& e, const float (&ej)[kPer], const Mass& m, const RowSums& s, float wt, F here) {
    const float inv = 1.0f / s.S;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (e.first[i] && here(e.id[i] >> (kBf16 ? 3 : 2)))
            Elems<kBf16>::store1(out, e.id[i], s.bad ? s.S : s.empty || e.bad ? 0.0f : wt * (float)((double)(ej[i] * inv) * (double)m.G - e.p[i] * (double)m.norm));
}
// p of entries listed twice, added up; listed_first has to run after the loss has been formed from the single ones.
template <int kPer> __device__ __forceinline__ void listed_sums(const Args& a, int lane, Listed<kPer>& e) { listed_first<kPer>(a, lane, e, true); }

template <bool kBf16, int kThreads, int kPer>
__global__ void __launch_bounds__(kThreads + 32)
distill_step_kernel(const Args a, int log2C, int vec_per_cta) {
    constexpr int kLog2 = kBf16 ? 3 : 2, kPerVec = 1 << kLog2, kWarps = kThreads / 32;
    extern __shared__ uint4 slice[];
    __shared__ StepShared<kThreads> sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    wait_for_previous();
    const long long T = rows_of(a);
    const int rank = blockIdx.x & ((1 << log2C) - 1);
    const long long t = (long long)(blockIdx.x >> log2C);
    if (t >= T) return;                                            // the whole cluster leaves together
    const char* row = a.logits + t * a.row_bytes;
    char* out = a.dlogits + t * a.row_bytes;
    const int nvec = a.V >> kLog2, tail0 = nvec << kLog2;
    const int v0 = rank * vec_per_cta, nv = max(0, min(vec_per_cta, nvec - v0));
    const bool last = rank == (1 << log2C) - 1;

    Listed<kPer> e;
    float lp[kPer];
    Mass mass = {};
    float wt = 0.0f;
    if (warp < kWarps) {                                           // the slice: every thread's own vectors, then everybody's
        const uint32_t dst = (uint32_t)__cvta_generic_to_shared(slice);
        for (int i = tid; i < nv; i += kThreads)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst + (uint32_t)i * 16u), "l"(row + (size_t)(v0 + i) * 16) : "memory");
        if (tid == 0) sh.tail_listed = 0;
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        listed_ids<kPer>(a, t, lane, e, lp);
        wt = (float)((a.weight ? (double)a.weight[t] : 1.0) * a.inv_tau);
        listed_logits<kBf16, kPer>(row, e);
        listed_probs<kPer>(a, lp, e);
        listed_first<kPer>(a, lane, e, false);
        mass = listed_mass<kPer>(a, e, lp);
    }
    __syncthreads();
    if (warp == kWarps) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int rel = (e.id[i] >> kLog2) - v0;
            if (e.id[i] < 0) continue;
            if ((e.id[i] >> kLog2) >= nvec) {
                if (last) atomicOr(&sh.tail_listed, 1u << (e.id[i] & (kPerVec - 1)));
            } else if (rel >= 0 && rel < nv) {
                Elems<kBf16>::store1(slice + rel, e.id[i] & (kPerVec - 1), -INFINITY);
            }
        }
    }
    __syncthreads();

    // the slice's maximum (NaN where there is one)
    float m = -INFINITY, ztail = -INFINITY;
    if (warp < kWarps) {
        if constexpr (kBf16) {
            __nv_bfloat162 x = __float2bfloat162_rn(-INFINITY);
#pragma unroll 4
            for (int i = tid; i < nv; i += kThreads) {
                const uint4 q = slice[i];
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(w);
                x = __hmax2_nan(x, __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3])));
            }
            m = max_nan(__low2float(x), __high2float(x));
        } else {
#pragma unroll 4
            for (int i = tid; i < nv; i += kThreads) {
                const uint4 q = slice[i];
                m = max_nan(m, max_nan(max_nan(__uint_as_float(q.x), __uint_as_float(q.y)), max_nan(__uint_as_float(q.z), __uint_as_float(q.w))));
            }
        }
        if (last && tail0 + tid < a.V && !(sh.tail_listed >> tid & 1u)) ztail = Elems<kBf16>::load1(row, tail0 + tid);
        m = max_nan(m, ztail);
        const bool bad = __any_sync(kAll, !(m < INFINITY));
        m = warp_max_f32(bad ? 0.0f : m);
        if (bad) m = __int_as_float(0x7fffffff);
        if (lane == 0) sh.m[warp] = m;
    }
    __syncthreads();
    m = sh.m[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) m = max_nan(m, sh.m[w]);
    const bool bad = !(m < INFINITY);
    m = bad ? 0.0f : fmaxf(m, kLowest);

    // the exponentials and their sum, in the frame of a running sum (see Sum).  Those of f32 rows take the logits' place; bf16 rows form
    // theirs again for the gradient, since 16 bits would not hold the range that a gradient of that type has
    Sum acc;
    sum_init(acc, m, a.c);
    float etail = 0.0f;
    const f32x2 c2 = pair_of(a.c, a.c), nr2 = pair_of(acc.nr, acc.nr), nm2 = pair_of(-m, -m);
    auto e2 = [&](float z0, float z1, auto is_quick) {
        float y0, y1;
        if constexpr (decltype(is_quick)::value) unpair(fma2(pair_of(z0, z1), c2, nr2), y0, y1);
        else unpair(mul2(add2(pair_of(z0, z1), nm2), c2), y0, y1);
        return pair_of(ex2(y0), ex2(y1));
    };
    if (warp < kWarps) {
        auto pass = [&](auto is_quick) {
#pragma unroll 4
            for (int i = tid; i < nv; i += kThreads) {
                const uint4 q = slice[i];
                uint32_t w[4] = {q.x, q.y, q.z, q.w};
                if constexpr (kBf16) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc.S = add2(acc.S, e2(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u), is_quick));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; j += 2) {
                        const f32x2 x = e2(__uint_as_float(w[j]), __uint_as_float(w[j + 1]), is_quick);
                        float x0, x1;
                        acc.S = add2(acc.S, x);
                        unpair(x, x0, x1);
                        w[j] = __float_as_uint(x0); w[j + 1] = __float_as_uint(x1);
                    }
                    slice[i] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            if (ztail > -INFINITY) {
                const f32x2 x = e2(ztail, -INFINITY, is_quick);
                float unused;
                acc.S = add2(acc.S, x);
                unpair(x, etail, unused);
            }
        };
        if (acc.quick) pass(std::true_type()); else pass(std::false_type());
        float s0, s1;
        unpair(acc.S, s0, s1);
        const float s = warp_sum(s0 + s1);
        if (lane == 0) sh.s[warp] = s;
    }
    __syncthreads();
    const float back = ex2(-acc.res);                              // the frame's shift, out of what was kept
    cg::cluster_group cl = cg::this_cluster();
    if (warp == kWarps) {
        const float s = warp_sum(lane < kWarps ? sh.s[lane] : 0.0f);
        Part p = {m, bad ? 0.0f : s * back, bad ? 1 : 0};
        if (!(p.S > 0.0f)) p.m = kLowest;
        if (lane == 0) sh.part = p;
        __syncwarp();
    }
    if (log2C > 0) cl.sync();                                      // every CTA's part is in its shared memory
    RowSums sums = {};
    Part p = part_none();
    float ej[kPer];
    if (warp == kWarps) {
        p = lane < (1 << log2C) ? (log2C > 0 ? *cl.map_shared_rank(&sh.part, lane) : sh.part) : part_none();
        p = part_warp(p, a.c);
        sums = row_sums<kPer>(a, e, mass, p, ej);
        // to_rest is relative to the row's unlisted maximum, what is kept to this slice's
        if (lane == 0) sh.scale = wt * sums.to_rest * (p.m > m ? ex2((m - p.m) * a.c) : 1.0f) * back;
        __syncwarp();
    }
    if (log2C > 0) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // the parts have been read
    __syncthreads();
    const float scale = sh.scale;
    if (warp < kWarps) {
        uint4* dst = reinterpret_cast<uint4*>(out) + v0;
        const f32x2 s2 = pair_of(scale, scale);
        auto put = [&](auto is_quick) {
#pragma unroll 2
            for (int i = tid; i < nv; i += kThreads) {
                float f[kPerVec];
                Elems<kBf16>::unpack(slice[i], f);
#pragma unroll
                for (int j = 0; j < kPerVec; j += 2) {
                    f32x2 x;
                    if constexpr (kBf16) x = e2(f[j], f[j + 1], is_quick); else x = pair_of(f[j], f[j + 1]);
                    unpair(mul2(x, s2), f[j], f[j + 1]);
                }
                __stcs(dst + i, Elems<kBf16>::pack(f));
            }
        };
        if (!kBf16 || acc.quick) put(std::true_type()); else put(std::false_type());
        if (last && tail0 + tid < a.V) Elems<kBf16>::store1(out, tail0 + tid, scale * etail);
    } else {
        if (rank == 0) row_write(a, t, mass, sums, p, e.bad, lane);
        __syncwarp();
        listed_sums<kPer>(a, lane, e);
    }
    __syncthreads();                                               // the listed entries' places have been written
    let_next_start();
    if (warp == kWarps) write_listed<kBf16, kPer>(out, e, ej, mass, sums, wt, [&](int v) { return v >= nvec ? last : v >= v0 && v < v0 + nv; });
    __syncwarp();
    if (log2C > 0) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- short rows: a warp per row, with or without the gradient --------------------------------------------------
// The row goes through the warp's shared memory once, where its listed entries are read and masked, and stays in registers.  (Several rows
// per warp, with their 64-bit scalars one row per lane at the end, save instructions and lose as much to their registers.)
template <bool kBf16, int kVecs, int kTeams, bool kGradient, int kPer>
__global__ void __launch_bounds__(32 * kTeams)
distill_warp_kernel(const Args a) {
    constexpr int kLog2 = kBf16 ? 3 : 2, kPerVec = 1 << kLog2;
    __shared__ uint4 rows[kTeams][kVecs * 32];
    __shared__ unsigned tails[kTeams];
    const int lane = threadIdx.x & 31, team = threadIdx.x >> 5;
    uint4* mine = rows[team];
    enter_kernel();
    const long long t = (long long)blockIdx.x * kTeams + team;
    if (t >= rows_of(a)) return;
    const char* row = a.logits + t * a.row_bytes;
    const int nvec = a.V >> kLog2, tail = (nvec << kLog2) + lane;
    uint4 q[kVecs];
#pragma unroll
    for (int u = 0; u < kVecs; ++u) q[u] = u * 32 + lane < nvec ? load_vec_rw(row + (size_t)(u * 32 + lane) * 16) : masked_vec<kBf16>();
    float zt = tail < a.V ? Elems<kBf16>::load1(row, tail) : -INFINITY;
    Listed<kPer> e;
    float lp[kPer];
    listed_ids<kPer>(a, t, lane, e, lp);
    const float wt = kGradient ? (float)((a.weight ? (double)a.weight[t] : 1.0) * a.inv_tau) : 0.0f;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) mine[u * 32 + lane] = q[u];
    if (lane == 0) tails[team] = 0;
    __syncwarp();
    listed_probs<kPer>(a, lp, e);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int v = e.id[i] >> kLog2;
        e.z[i] = e.id[i] < 0 ? -INFINITY : v >= nvec ? Elems<kBf16>::load1(row, e.id[i]) : Elems<kBf16>::load1(mine, e.id[i]);
    }
    listed_first<kPer>(a, lane, e, false);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (e.id[i] < 0) continue;
        if ((e.id[i] >> kLog2) >= nvec) atomicOr(&tails[team], 1u << (e.id[i] & (kPerVec - 1)));
        else Elems<kBf16>::store1(mine, e.id[i], -INFINITY);
    }
    __syncwarp();
    if (tails[team] >> lane & 1u) zt = -INFINITY;
#pragma unroll
    for (int u = 0; u < kVecs; ++u) q[u] = mine[u * 32 + lane];
    __nv_bfloat162 unused;
    float m = max_nan(vecs_max<kBf16, kVecs>(q, unused), zt);
    const bool bad = __any_sync(kAll, !(m < INFINITY));
    m = fmaxf(warp_max_f32(bad ? 0.0f : m), kLowest);
    Sum acc;
    sum_init(acc, m, a.c);
    f32x2 x[kVecs * kPerVec / 2];                                  // the exponentials
    float xt = 0.0f;
    {
        const f32x2 c2 = pair_of(a.c, a.c), nr2 = pair_of(acc.nr, acc.nr), nm2 = pair_of(-m, -m);
        const bool quick = acc.quick;
#pragma unroll
        for (int u = 0; u < kVecs; ++u) {
            float f[kPerVec];
            Elems<kBf16>::unpack(q[u], f);
#pragma unroll
            for (int j = 0; j < kPerVec; j += 2) {
                float y0, y1;
                unpair(quick ? fma2(pair_of(f[j], f[j + 1]), c2, nr2) : mul2(add2(pair_of(f[j], f[j + 1]), nm2), c2), y0, y1);
                x[(u * kPerVec + j) / 2] = pair_of(ex2(y0), ex2(y1));
                acc.S = add2(acc.S, x[(u * kPerVec + j) / 2]);
            }
        }
        xt = ex2(quick ? fmaf(zt, a.c, acc.nr) : (zt - m) * a.c);
    }
    const float back = ex2(-acc.res);
    float s0, s1;
    unpair(acc.S, s0, s1);
    Part p = {m, warp_sum(s0 + s1 + xt) * back, bad ? 1 : 0};
    if (!(p.S > 0.0f)) p.m = kLowest;
    float ej[kPer];
    const Mass mass = listed_mass<kPer>(a, e, lp);
    const RowSums sums = row_sums<kPer>(a, e, mass, p, ej);
    row_write(a, t, mass, sums, p, e.bad, lane);
    if constexpr (kGradient) {
        char* out = a.dlogits + t * a.row_bytes;
        const float scale = wt * sums.to_rest * back;
        const f32x2 s2 = pair_of(scale, scale);
#pragma unroll
        for (int u = 0; u < kVecs; ++u) {
            if (u * 32 + lane >= nvec) continue;
            float f[kPerVec];
#pragma unroll
            for (int j = 0; j < kPerVec; j += 2) unpair(mul2(x[(u * kPerVec + j) / 2], s2), f[j], f[j + 1]);
            __stcs(reinterpret_cast<uint4*>(out) + u * 32 + lane, Elems<kBf16>::pack(f));
        }
        if (tail < a.V) Elems<kBf16>::store1(out, tail, scale * xt);
        listed_sums<kPer>(a, lane, e);
        __syncwarp();
        write_listed<kBf16, kPer>(out, e, ej, mass, sums, wt, [](int) { return true; });
    }
}

// ---- gradient from the forward's statistics ---------------------------------------------------------------
// A warp per row (kThreads = 32, kTeams rows in a CTA), or kThreads threads per piece of a row and a warp for what is listed in it.
template <bool kBf16, int kThreads, int kTeams, int kUnroll, int kPer>
__global__ void __launch_bounds__(kThreads == 32 ? 32 * kTeams : kThreads + 32)
distill_backward_kernel(const Args a) {
    constexpr int kPerVec = Elems<kBf16>::kPerVec, kLog2 = kBf16 ? 3 : 2;
    const int team = kTeams == 1 ? 0 : threadIdx.x / kThreads;
    const int tid = kTeams == 1 ? threadIdx.x : threadIdx.x % kThreads, lane = tid & 31;
    const bool lister = kThreads == 32 || tid >= kThreads, sweeper = tid < kThreads;
    enter_kernel();
    const long long T = rows_of(a);
    const long long item = (long long)blockIdx.x * kTeams + team;
    const long long t = a.chunks == 1 ? item : item / a.chunks;
    const int chunk = a.chunks == 1 ? 0 : (int)(item - t * a.chunks);
    if (t >= T) return;                                            // a team is a warp, or the whole CTA
    const char* row = a.logits + t * a.row_bytes;
    char* out = a.dlogits + t * a.row_bytes;
    const int nvec = a.V >> kLog2, tail0 = nvec << kLog2;
    const int v0 = chunk * a.chunk_vecs, v1 = min(nvec, v0 + a.chunk_vecs);
    const bool last = chunk == a.chunks - 1;
    const float4 st = a.stats_in[t];
    const float wt = (float)((a.weight ? (double)a.weight[t] : 1.0) * a.inv_tau);

    // what is listed in this piece: its ids and logits (in place: before anything is written)
    Listed<kPer> e;
    float lp[kPer];
    bool any = false;
    auto here = [&](int i) { const int v = e.id[i] >> kLog2; return e.id[i] >= 0 && (v >= nvec ? last : v >= v0 && v < v1); };
    if (lister) {
        listed_ids<kPer>(a, t, lane, e, lp);
#pragma unroll
        for (int i = 0; i < kPer; ++i) any = any || here(i);
        any = __any_sync(kAll, any);
#pragma unroll
        for (int i = 0; i < kPer; ++i) e.z[i] = here(i) ? Elems<kBf16>::load1(row, e.id[i]) : -INFINITY;      // the other pieces' are being written
    }
    if (a.in_place) { if constexpr (kThreads == 32) __syncwarp(); else __syncthreads(); }

    const bool empty = st.x == -INFINITY;
    const float inv = st.y > 0.0f || st.y != st.y ? 1.0f / st.y : 0.0f;
    // share = inf: nothing unlisted has a probability, so nothing is multiplied by it; below 0: its exponent, which the entries' take up
    const bool far = st.w < 0.0f;
    const float coef = empty || st.w == INFINITY ? 0.0f : far ? -wt * inv : wt * (st.z - st.w) * inv;
    const bool zero = empty || coef == 0.0f;
    const f32x2 c2 = pair_of(a.c, a.c), g2 = pair_of(coef, coef);
    const float r = st.x * a.c;
    const bool quick = !far && fabsf(r) <= 1048576.0f && fabsf(st.x) <= 1e37f;     // as in the forward's sum
    const f32x2 nr2 = pair_of(-r, -r), nm2 = pair_of(-st.x, -st.x), up2 = pair_of(-st.w, -st.w);
    const float res = quick ? fmaf(st.x, a.c, -r) : 0.0f;
    const f32x2 gq2 = pair_of(coef * ex2(-res), coef * ex2(-res));
    auto put = [&](const uint4& q, int i, auto is_quick) {
        float z[kPerVec];
        Elems<kBf16>::unpack(q, z);
#pragma unroll
        for (int j = 0; j < kPerVec; j += 2) {
            float y0, y1;
            if constexpr (decltype(is_quick)::value) unpair(fma2(pair_of(z[j], z[j + 1]), c2, nr2), y0, y1);
            else if (far) unpair(fma2(add2(pair_of(z[j], z[j + 1]), nm2), c2, up2), y0, y1);
            else unpair(mul2(add2(pair_of(z[j], z[j + 1]), nm2), c2), y0, y1);
            unpair(mul2(pair_of(ex2(y0), ex2(y1)), decltype(is_quick)::value ? gq2 : g2), z[j], z[j + 1]);
        }
        __stcs(reinterpret_cast<uint4*>(out) + i, Elems<kBf16>::pack(z));
    };
    auto sweep = [&](auto is_quick) {
        for (int i = v0 + tid; i - tid < v1; i += kUnroll * kThreads) {        // all loads of a round before its stores
            uint4 q[kUnroll];
            if (i - tid + kUnroll * kThreads <= v1) {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) q[u] = load_vec_rw(row + (size_t)(i + u * kThreads) * 16);
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) put(q[u], i + u * kThreads, is_quick);
            } else {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u)
                    if (i + u * kThreads < v1) q[u] = load_vec_rw(row + (size_t)(i + u * kThreads) * 16);
#pragma unroll
                for (int u = 0; u < kUnroll; ++u)
                    if (i + u * kThreads < v1) put(q[u], i + u * kThreads, is_quick);
            }
        }
    };
    if (!sweeper) {
    } else if (zero) {
        for (int i = v0 + tid; i < v1; i += kThreads) __stcs(reinterpret_cast<uint4*>(out) + i, make_uint4(0u, 0u, 0u, 0u));
    } else if (quick) {
        sweep(std::true_type());
    } else {
        sweep(std::false_type());
    }
    if (sweeper && last && tail0 + tid < a.V) {
        const float z = Elems<kBf16>::load1(row, tail0 + tid);
        Elems<kBf16>::store1(out, tail0 + tid, zero ? 0.0f : coef * ex2(fmaf(z - st.x, a.c, far ? -st.w : 0.0f)));
    }
    double norm = 1.0;
    if (lister && any) {
        listed_probs<kPer>(a, lp, e);
        if (a.mode == DPPO_DISTILL_NORMALIZED) {
            double P = 0.0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) P += e.p[i];
            P = warp_sum_f64(P);
            norm = P > 0.0 ? inv64(P) : 0.0;
        }
        listed_first<kPer>(a, lane, e, true);
    }
    if constexpr (kThreads == 32) __syncwarp(); else __syncthreads();          // the listed entries' places have been written
    if (!lister) return;
    if (e.bad) {
        if (lane == 0 && chunk == 0) set_status(a.status, DPPO_STATUS_BAD_TARGET);
        return;                                                    // G = 0: the row is zero
    }
    if (empty || !any) return;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        if (!e.first[i] || !here(i)) continue;
        const float s = ex2((e.z[i] - st.x) * a.c) * inv;
        Elems<kBf16>::store1(out, e.id[i], wt * (float)((double)s * (double)st.z - e.p[i] * norm));
    }
}

// ---- host side -------------------------------------------------------------------------------------------
template <bool kBf16, bool kGradient, int kPer> static int run_warp(const Args& a, cudaStream_t s);

template <bool kBf16, int kThreads, int kPer, bool kCluster> static int launch_fwd(const Args& a, int C, cudaStream_t s) {
    auto kernel = distill_forward_kernel<kBf16, kThreads, kPer, kCluster>;
    const int nvec = a.V >> (kBf16 ? 3 : 2);
    const size_t smem = (size_t)bitmap_words<kThreads>((nvec + C - 1) / C) * 4;       // 32 KB at kMaxV
    if (a.T_max * C > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "distill_topk: T_max=%lld needs too large a grid", a.T_max);
    return launch_after("distill_topk launch", kernel, a.T_max * C, kThreads + 32, smem, s, kCluster ? C : 1, a);
}

// Loss alone: a warp per row up to 4 KB, else a CTA, in a cluster while the rows do not give every SM two (40 x 151,936 bf16 8.5 us).  A CTA alone has 256
// threads up to five rows per SM (400 x 151,936 bf16 29.5 us, with 128 44.6; 700 x 50,304 18.4, 20.2) and 128 beyond, where they are as fast and
// leave room for shorter ones (8,192 x 151,936 390-434 us, 6.4-5.7 TB/s: the power limit).
template <bool kBf16, int kPer> static int run_fwd(const Args& a, cudaStream_t s) {
    const int nvec = a.V >> (kBf16 ? 3 : 2);
    const long long sms = sm_count();
    int C = 1;
    if (nvec <= 256) return run_warp<kBf16, false, kPer>(a, s);
    if (nvec > 4096)
        while (C < kMaxCluster && a.T_max * C < 2 * sms) C *= 2;
    if (C > 1) return launch_fwd<kBf16, 256, kPer, true>(a, C, s);
    if (nvec > 1024 && a.T_max <= 5 * sms) return launch_fwd<kBf16, 256, kPer, false>(a, 1, s);
    return launch_fwd<kBf16, 128, kPer, false>(a, 1, s);
}

template <bool kBf16, int kVecs, bool kGradient, int kPer> static int launch_warp(const Args& a, cudaStream_t s) {
    constexpr int kTeams = 2;
    return launch_after("distill_topk launch", distill_warp_kernel<kBf16, kVecs, kTeams, kGradient, kPer>, (a.T_max + kTeams - 1) / kTeams, 32 * kTeams, 0, s, 1, a);
}
template <bool kBf16, bool kGradient, int kPer> static int run_warp(const Args& a, cudaStream_t s) {
    const int nvec = a.V >> (kBf16 ? 3 : 2);
    if (nvec <= 32) return launch_warp<kBf16, 1, kGradient, kPer>(a, s);
    if (nvec <= 64) return launch_warp<kBf16, 2, kGradient, kPer>(a, s);
    if (nvec <= 128) return launch_warp<kBf16, 4, kGradient, kPer>(a, s);
    return launch_warp<kBf16, 8, kGradient, kPer>(a, s);
}

constexpr size_t kSliceMax = 220 * 1024;
template <bool kBf16, int kThreads, int kPer> static int launch_step(const Args& a, int log2C, int vec_per_cta, cudaStream_t s) {
    auto kernel = distill_step_kernel<kBf16, kThreads, kPer>;
    static bool raised[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) { cudaGetLastError(); dev = -1; }
    if (dev < 0 || !raised[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSliceMax);
        if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(e, "distill_topk: shared memory attribute"); }
        if (dev >= 0) raised[dev] = true;
    }
    if (a.T_max << log2C > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "distill_topk: T_max=%lld needs too large a grid", a.T_max);
    return launch_after("distill_topk launch", kernel, a.T_max << log2C, kThreads + 32, (size_t)max(vec_per_cta, 1) * 16, s, 1 << log2C, a, log2C, vec_per_cta);
}
// Loss and gradient, 8,192 x 151,936 bf16 990-1,015 us (5.0 TB/s of one read and one write; as two kernels 1,160; 895-945 with the exponentials
// kept as fp16, which lost the digits of entries more than e^-10 below the largest); 20,011 x 1,021 f32 32.5 (5.1).
// The slices of a row: in one CTA up to 44 KB, in two of up to 55 KB, else in four or eight of up to 76 KB, three of which share an SM.  Few
// rows: more CTAs for each (37 x 151,936 bf16 8.7 us, 10.2 in four; 16 x 20,000 f32 5.1, 5.9 in two).
template <bool kBf16, int kPer> static int run_step(const Args& a, cudaStream_t s, bool* done) {
    const int nvec = a.V >> (kBf16 ? 3 : 2);
    *done = true;
    if (nvec <= 256) return run_warp<kBf16, true, kPer>(a, s);
    const long long bytes = (long long)nvec * 16;
    int log2C = bytes <= 44 << 10 ? 0 : bytes <= 110 << 10 ? 1 : bytes <= 304 << 10 ? 2 : 3;
    while (log2C > 0 && log2C < 3 && a.T_max << (log2C + 1) <= 2ll * sm_count()) ++log2C;
    const int vec = (nvec + (1 << log2C) - 1) >> log2C;
    if ((size_t)vec * 16 > kSliceMax) { *done = false; return DPPO_OK; }
    if (vec * 16 > (kBf16 ? 28 : 64) << 10) return launch_step<kBf16, 256, kPer>(a, log2C, vec, s);
    return launch_step<kBf16, 128, kPer>(a, log2C, vec, s);
}

template <bool kBf16, int kThreads, int kTeams, int kUnroll, int kPer> static int launch_bwd(const Args& a, cudaStream_t s) {
    const long long ctas = (a.T_max * a.chunks + kTeams - 1) / kTeams;
    if (ctas > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "distill_topk_backward: T_max=%lld needs too large a grid", a.T_max);
    return launch_after("distill_topk_backward launch", distill_backward_kernel<kBf16, kThreads, kTeams, kUnroll, kPer>, ctas, kThreads == 32 ? 32 * kTeams : kThreads + 32, 0, s, 1, a);
}

template <bool kBf16, int kPer> static int run_bwd(Args a, cudaStream_t s) {
    const int nvec = a.V >> (kBf16 ? 3 : 2);
    a.chunks = 1; a.chunk_vecs = nvec;
    if (nvec <= 320) return launch_bwd<kBf16, 32, 4, 4, kPer>(a, s);
    // Pieces long enough that the listed entries' chain of loads (id, logit) is over before the sweep is: 8,192 x 151,936 bf16 in 512
    // vectors by 128 threads 957 us, in 4,096 by 256 768; 2,003 x 50,304 f32 161 and 133.  Where there are too few of those to
    // go round, shorter ones (64 x 151,936: 9.9 us in 4,096, 8.2 in 1,024).  Rounds of four loads: eight take 1,070 and 138.
    const long long share = a.T_max * nvec / (8 * sm_count());
    const int most = share >= 4096 ? 4096 : share >= 2048 ? 2048 : 1024;
    a.chunks = (nvec + most - 1) / most;
    a.chunk_vecs = (nvec + a.chunks - 1) / a.chunks;
    if (most == 1024) return launch_bwd<kBf16, 128, 1, 4, kPer>(a, s);
    return launch_bwd<kBf16, 256, 1, 4, kPer>(a, s);
}

// Checks that both calls make; 0 or the error.
static int check(const dppo_distill_params* p, const char* what, const void* logits, const void* top_ids, const void* top_logp, const void* stats,
                 const void* dlogits) {
    if (!p) return fail(DPPO_ERR_INVALID_ARG, "%s: NULL params", what);
    if (p->T_max < 0 || p->V < 1) return fail(DPPO_ERR_INVALID_ARG, "%s: T_max=%lld V=%d", what, (long long)p->T_max, p->V);
    if (p->dtype != DPPO_F32 && p->dtype != DPPO_BF16) return fail(DPPO_ERR_UNSUPPORTED, "%s: dtype %d", what, p->dtype);
    if (p->row_stride < p->V) return fail(DPPO_ERR_BAD_SHAPE, "%s: row_stride %lld < V %d", what, (long long)p->row_stride, p->V);
    if (!(p->temperature >= 1e-6) || !(p->temperature <= 1e6)) return fail(DPPO_ERR_INVALID_ARG, "%s: temperature must be in [1e-6, 1e6]", what);
    if (p->V > kMaxV) return fail(DPPO_ERR_BAD_SHAPE, "%s: V=%d, the limit is 2^20", what, p->V);
    if (p->T_max >= ((int64_t)1 << 31)) return fail(DPPO_ERR_BAD_SHAPE, "%s: T_max must be below 2^31", what);
    if (p->top_k < 1 || p->top_k > kMaxListed) return fail(DPPO_ERR_INVALID_ARG, "%s: top_k=%d (1..%d)", what, p->top_k, kMaxListed);
    if (p->mode < DPPO_DISTILL_GIVEN || p->mode > DPPO_DISTILL_REST) return fail(DPPO_ERR_INVALID_ARG, "%s: mode %d", what, p->mode);
    const size_t esize = p->dtype == DPPO_BF16 ? 2 : 4;
    if (((uintptr_t)logits & 15) || ((uintptr_t)stats & 15) || ((uintptr_t)dlogits & 15) || ((size_t)p->row_stride * esize) % 16 != 0)
        return fail(DPPO_ERR_MISALIGNED, "%s: logits / dlogits / stats base and row stride must be multiples of 16 bytes", what);
    if (p->T_max > 0 && (!logits || !top_ids || !top_logp)) return fail(DPPO_ERR_INVALID_ARG, "%s: NULL logits, top_ids or top_logp", what);
    return DPPO_OK;
}

static Args args_of(const dppo_distill_params* p, const void* logits, const int32_t* top_ids, const float* top_logp, const int32_t* n_tokens_dev,
                    const float* weight, void* dlogits, int32_t* status) {
    Args a = {};
    a.logits = (const char*)logits; a.ids = top_ids; a.logp = top_logp; a.n_tokens_dev = n_tokens_dev; a.weight = weight;
    a.dlogits = (char*)dlogits; a.status = status;
    a.T_max = p->T_max; a.row_bytes = (long long)p->row_stride * (p->dtype == DPPO_BF16 ? 2 : 4);
    a.V = p->V; a.k = p->top_k; a.mode = p->mode; a.in_place = dlogits == logits;
    a.c = (float)(1.4426950408889634 / p->temperature); a.inv_tau = 1.0 / p->temperature;
    return a;
}

template <bool kBf16> static int run_fwd_k(const Args& a, cudaStream_t s) { return a.k <= 32 ? run_fwd<kBf16, 1>(a, s) : run_fwd<kBf16, 4>(a, s); }
// Loss and gradient in one kernel where the row fits the shared memory of eight CTAs, else one after the other.
template <bool kBf16, int kPer> static int run_both(const Args& a, cudaStream_t s) {
    bool done;
    int rc = run_step<kBf16, kPer>(a, s, &done);
    if (rc != DPPO_OK || done) return rc;
    rc = run_fwd<kBf16, kPer>(a, s);
    return rc != DPPO_OK ? rc : run_bwd<kBf16, kPer>(a, s);
}
template <bool kBf16> static int run_both_k(const Args& a, cudaStream_t s) { return a.k <= 32 ? run_both<kBf16, 1>(a, s) : run_both<kBf16, 4>(a, s); }
template <bool kBf16> static int run_bwd_k(const Args& a, cudaStream_t s) { return a.k <= 32 ? run_bwd<kBf16, 1>(a, s) : run_bwd<kBf16, 4>(a, s); }

}  // namespace distill
}  // namespace dppo

extern "C" int dppo_distill_topk(const dppo_distill_params* p, const void* logits, const int32_t* top_ids, const float* top_logp,
                                 const int32_t* n_tokens_dev, const float* weight, float* loss_out, float* lse_out, float* stats,
                                 void* dlogits, int32_t* status, void* stream) {
    dppo::NvtxRange nvtx_range("dppo_distill_topk");
    using namespace dppo;
    const int rc = distill::check(p, "distill_topk", logits, top_ids, top_logp, stats, dlogits);
    if (rc != DPPO_OK || p->T_max == 0) return rc;
    if (dlogits && !stats) return fail(DPPO_ERR_INVALID_ARG, "distill_topk: dlogits without stats");
    if (weight && !dlogits) return fail(DPPO_ERR_INVALID_ARG, "distill_topk: weight without dlogits");
    distill::Args a = distill::args_of(p, logits, top_ids, top_logp, n_tokens_dev, weight, dlogits, status);
    a.loss = loss_out; a.lse = lse_out; a.stats = (float4*)stats; a.stats_in = (const float4*)stats;
    cudaStream_t s = (cudaStream_t)stream;
    if (dlogits) return p->dtype == DPPO_BF16 ? distill::run_both_k<true>(a, s) : distill::run_both_k<false>(a, s);
    return p->dtype == DPPO_BF16 ? distill::run_fwd_k<true>(a, s) : distill::run_fwd_k<false>(a, s);
}

extern "C" int dppo_distill_topk_backward(const dppo_distill_params* p, const void* logits, const int32_t* top_ids, const float* top_logp,
                                          const int32_t* n_tokens_dev, const float* stats, const float* dloss, void* dlogits,
                                          int32_t* status, void* stream) {
    dppo::NvtxRange nvtx_range("dppo_distill_topk_backward");
    using namespace dppo;
    const int rc = distill::check(p, "distill_topk_backward", logits, top_ids, top_logp, stats, dlogits);
    if (rc != DPPO_OK || p->T_max == 0) return rc;
    if (!stats || !dlogits) return fail(DPPO_ERR_INVALID_ARG, "distill_topk_backward: NULL stats or dlogits");
    distill::Args a = distill::args_of(p, logits, top_ids, top_logp, n_tokens_dev, dloss, dlogits, status);
    a.stats_in = (const float4*)stats;
    return p->dtype == DPPO_BF16 ? distill::run_bwd_k<true>(a, (cudaStream_t)stream) : distill::run_bwd_k<false>(a, (cudaStream_t)stream);
}
