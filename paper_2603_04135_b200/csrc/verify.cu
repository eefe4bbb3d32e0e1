// Verification of drafted tokens against the target policy, from given random numbers.
//
// A sequence's drafts y_0 .. y_{n-1} are accepted one after the other while u_j q_j(y_j) < p_j(y_j) (p, q: the target's and the
// draft's probabilities; q = 1 at y_j where the drafts come without logits).  At the first rejection the next token is drawn from
// max(p - q, 0), after n acceptances from p: as the largest w_v / e_v with given exponential variates e (the first of n
// independent exponential clocks with rates w_v rings for v with probability w_v / sum w: no normalisation, no prefix sum over the row).
//
// Two kernels.  The first reduces every row of both policies to {m, S} (one read of all logits: what bounds the call); the second, a
// cluster of CTAs per sequence, finds the first rejection (a warp, 32 drafts at a time) and races over that one row.
//
// The race: an entry counts only if its p / e, by one fma and a logarithm, comes near the best lower bound among the first entries of its
// CTA, which a few dozen do; only those look at the draft's row, all at once.  f32 decides a race only where no second entry's upper bound
// reaches the winner's lower bound; otherwise the entries within reach are compared in 64 bits, ties to the lower index.
//
// What that leaves: the rows' sums S are f32 sums (about 1e-6 of them off), common to all of a race over p alone, but not to both sides of
// u q < p nor to p and q in p - q.  Decisions whose sides are closer than that may differ from the definition's; they are the same in every call.
#include <cooperative_groups.h>

#include "common.cuh"
#include "grpo_loss.cuh"
#include "row_sweep.cuh"

namespace dppo {
using namespace packed;
namespace cg = cooperative_groups;

namespace verify {
using namespace sweep;

constexpr int kMaxCluster = 8;
constexpr int kCand = 512;
constexpr uint32_t kAll = 0xffffffffu;
// Relative error of an f32 probability: 3 roundings and the constant in an exponent of up to 100, the exponential, the sum.
constexpr float kEps = 1.0f / 65536.0f;
// Where the exponent is beyond 100, down to probabilities that f32 makes 0, the error is that of this one.
constexpr float kTiny = 0x1p-96f;
// Noise between these has a reciprocal that, times kEps kTiny or a probability, is a normal f32; entries with any other are decided in 64 bits.
constexpr float kLeastNoise = 0x1p-64f, kMostNoise = 0x1p13f;

struct Args {
    const char *target, *draft;
    const int32_t *drafts, *cu;
    const float *u, *noise;
    int32_t *n_accepted, *tokens;
    float* logp;
    float2* rows;                         // {m, S}: T_max + n_seqs target rows, then T_max draft rows
    int32_t* status;
    long long T_max, target_bytes, draft_bytes, noise_stride;
    int n_seqs, V;
    float ct, cd;
    double inv_tau_t, inv_tau_d;
};

// ---- {m, S} of every row ---------------------------------------------------------------------------------
// Row `item` of the call: its address (NULL: not one of the true rows), and the factor of its exponents.
__device__ __forceinline__ const char* row_of(const Args& a, long long item, long long T, float& c) {
    const long long n_target = a.T_max + a.n_seqs;
    c = item < n_target ? a.ct : a.cd;
    if (item < n_target) return item < T + a.n_seqs ? a.target + item * a.target_bytes : nullptr;
    return item - n_target < T ? a.draft + (item - n_target) * a.draft_bytes : nullptr;
}
__device__ __forceinline__ long long true_drafts(const Args& a) { return min((long long)max(a.cu[a.n_seqs], 0), a.T_max); }
__device__ __forceinline__ float2 row_stats(const Part& p) {
    return p.bad ? make_float2(__int_as_float(0x7fffffff), __int_as_float(0x7fffffff)) : make_float2(p.m, p.S);
}

// A warp per row.
template <bool kBf16, int kTeams> __global__ void __launch_bounds__(32 * kTeams) verify_rows_warp_kernel(const Args a, long long n_rows) {
    constexpr int kLog2 = kBf16 ? 3 : 2;
    const int lane = threadIdx.x & 31;
    enter_kernel();
    const long long item = (long long)blockIdx.x * kTeams + (threadIdx.x >> 5);
    float c;
    const char* row = item < n_rows ? row_of(a, item, true_drafts(a), c) : nullptr;
    if (!row) return;
    const int nvec = a.V >> kLog2, tail = (nvec << kLog2) + lane;
    const float zt = tail < a.V ? Elems<kBf16>::load1(row, tail) : -INFINITY;
    Sum acc;
    sum_init(acc, kLowest, c);
    for (int i = lane; i - lane < nvec; i += kRound * 32) {
        uint4 q[kRound];
#pragma unroll
        for (int u = 0; u < kRound; ++u) q[u] = i + u * 32 < nvec ? load_vec(row + (size_t)(i + u * 32) * 16) : masked_vec<kBf16>();
        sum_vecs<kBf16, kRound>(acc, q, c);
    }
    Part p = sum_part(acc);
    part_one(p, zt, c);
    p = part_warp(p, c);
    if (lane == 0) a.rows[item] = row_stats(p);
}

// A CTA per row, or the CTAs of a cluster.
template <bool kBf16, int kThreads, bool kCluster> __global__ void __launch_bounds__(kThreads) verify_rows_kernel(const Args a) {
    constexpr int kLog2 = kBf16 ? 3 : 2, kWarps = kThreads / 32;
    __shared__ Part parts[kWarps];
    __shared__ Part mine;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    enter_kernel();
    unsigned rank = 0, C = 1;
    if constexpr (kCluster) { C = cg::this_cluster().num_blocks(); rank = cg::this_cluster().block_rank(); }
    const int log2C = 31 - __clz((int)C);
    const long long item = (long long)(blockIdx.x >> log2C);
    float c;
    const char* row = row_of(a, item, true_drafts(a), c);
    if (!row) return;                                              // the whole cluster leaves together
    const int nvec = a.V >> kLog2;
    const int v0 = (int)((long long)nvec * rank >> log2C), v1 = (int)((long long)nvec * (rank + 1) >> log2C);
    Sum acc;
    sum_init(acc, kLowest, c);
    for (int i = v0 + tid; i - tid < v1; i += kRound * kThreads) {
        uint4 q[kRound];
        if (i - tid + kRound * kThreads <= v1) {
#pragma unroll
            for (int u = 0; u < kRound; ++u) q[u] = load_vec(row + (size_t)(i + u * kThreads) * 16);
        } else {
#pragma unroll
            for (int u = 0; u < kRound; ++u) q[u] = i + u * kThreads < v1 ? load_vec(row + (size_t)(i + u * kThreads) * 16) : masked_vec<kBf16>();
        }
        sum_vecs<kBf16, kRound>(acc, q, c);
    }
    Part p = sum_part(acc);
    if (rank == C - 1 && (nvec << kLog2) + tid < a.V) part_one(p, Elems<kBf16>::load1(row, (nvec << kLog2) + tid), c);
    p = part_warp(p, c);
    if (lane == 0) parts[warp] = p;
    __syncthreads();
    if (warp == 0) p = part_warp(lane < kWarps ? parts[lane] : part_none(), c);
    if constexpr (kCluster) {
        cg::cluster_group cl = cg::this_cluster();
        if (tid == 0) mine = p;
        cl.sync();                                                 // every CTA's part is in its shared memory
        if (rank == 0 && warp == 0) {
            p = lane < (int)C ? *cl.map_shared_rank(&mine, lane) : part_none();
            p = part_warp(p, c);
        }
        cl.sync();                                                 // ... and has been read
    }
    if (rank == 0 && tid == 0) a.rows[item] = row_stats(p);
}

// ---- acceptance and the race -------------------------------------------------------------------------------
// Of a set of entries: the largest upper bound of w / e with its index, the second largest, the largest lower bound.
struct Race {
    float hi, second, lo;
    int at;
};
__device__ __forceinline__ Race race_join(const Race& a, const Race& b) {
    const bool first = a.hi >= b.hi;
    Race r;
    r.hi = first ? a.hi : b.hi;
    r.at = first ? a.at : b.at;
    r.second = fmaxf(first ? b.hi : a.hi, fmaxf(a.second, b.second));
    r.lo = fmaxf(a.lo, b.lo);
    return r;
}
__device__ __forceinline__ Race race_warp(Race r) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        r = race_join(r, {__shfl_xor_sync(kAll, r.hi, o), __shfl_xor_sync(kAll, r.second, o), __shfl_xor_sync(kAll, r.lo, o), __shfl_xor_sync(kAll, r.at, o)});
    return r;
}
// The winner of a comparison in 64 bits: the larger w / e, then the lower index.
struct Exact {
    double x;
    int at;
};
__device__ __forceinline__ Exact exact_join(const Exact& a, const Exact& b) { return a.x > b.x || (a.x == b.x && a.at < b.at) ? a : b; }
__device__ __forceinline__ Exact exact_warp(Exact r) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) r = exact_join(r, {__shfl_xor_sync(kAll, r.x, o), __shfl_xor_sync(kAll, r.at, o)});
    return r;
}

// What the race runs on.
struct Field {
    const char *p, *q;                    // rows of logits; q NULL: no second policy
    const float* e;
    float mp, mq, ip, iq;                 // maxima and reciprocal sums
    int drop;                             // copied drafts: this entry is out (-1: none)
};
struct PickShared {
    Race race[16];
    Exact exact[16];
    Race mine;
    Exact mine_exact;
    Field f;
    float2 sp, sq;
    long long row;                        // of the next token
    int bound, n_cand;                    // bits of the largest lower bound of the CTA's first entries; entries that come near it
    float z[kCand], e[kCand];
    int at[kCand];
    int state;                            // 0 go on, 1 the sequence has no next token, 2 nothing may be written
};

template <int kThreads> __device__ __forceinline__ Race race_cta(Race r, PickShared& sh) {
    r = race_warp(r);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.race[threadIdx.x >> 5] = r;
    __syncthreads();
    return race_warp((threadIdx.x & 31) < kThreads / 32 ? sh.race[threadIdx.x & 31] : Race{0.0f, 0.0f, 0.0f, 0x7fffffff});
}
template <int kThreads> __device__ __forceinline__ Exact exact_cta(Exact r, PickShared& sh) {
    r = exact_warp(r);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sh.exact[threadIdx.x >> 5] = r;
    __syncthreads();
    return exact_warp((threadIdx.x & 31) < kThreads / 32 ? sh.exact[threadIdx.x & 31] : Exact{0.0, 0x7fffffff});
}

// Calls f(z_p, e, index) for those entries of vectors [v0, v1), and of the row's tail, whose log2(p / e) is not below `bound` by more than a
// margin (far above the errors of its f32 estimate; p relative to its row's sum).  kUnroll vectors' loads under way together.
template <bool kBf16, int kThreads, int kUnroll, class F>
__device__ __forceinline__ void for_field(const Field& w, float ct, int v0, int v1, int tail0, int V, float bound, F f) {
    constexpr int kPer = Elems<kBf16>::kPerVec;
    constexpr float kMargin = 0.01f;
    const int tid = threadIdx.x;
    auto one = [&](float z, float e, int at) {
        float l;
        asm("lg2.approx.f32 %0, %1;" : "=f"(l) : "f"(e));
        if (fmaf(z - w.mp, ct, -l) > bound - kMargin) f(z, e, at);
    };
#pragma unroll 1
    for (int i0 = v0 + tid; i0 < v1; i0 += kUnroll * kThreads) {
        uint4 vp[kUnroll], ve[kUnroll][kPer / 4];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int i = i0 + u * kThreads;
            const bool in = i < v1;
            vp[u] = in ? load_vec(w.p + (size_t)i * 16) : masked_vec<kBf16>();
#pragma unroll
            for (int j = 0; j < kPer / 4; ++j) ve[u][j] = in ? load_vec(w.e + (size_t)i * kPer + 4 * j) : make_uint4(0x3f800000u, 0x3f800000u, 0x3f800000u, 0x3f800000u);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float zp[kPer];
            Elems<kBf16>::unpack(vp[u], zp);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const uint32_t x[4] = {ve[u][j / 4].x, ve[u][j / 4].y, ve[u][j / 4].z, ve[u][j / 4].w};
                one(zp[j], __uint_as_float(x[j & 3]), (i0 + u * kThreads) * kPer + j);
            }
        }
    }
    if (tail0 + tid < V) one(Elems<kBf16>::load1(w.p, tail0 + tid), w.e[tail0 + tid], tail0 + tid);
}
// f(z_p, z_q, e, index) for every entry of this thread's vector i, if it is one.
template <bool kBf16, class F> __device__ __forceinline__ void for_vector(const Field& w, int i, int v1, F f) {
    constexpr int kPer = Elems<kBf16>::kPerVec;
    if (i >= v1) return;
    float zp[kPer], zq[kPer];
    uint4 ve[kPer / 4];
    const uint4 vp = load_vec(w.p + (size_t)i * 16), vq = w.q ? load_vec(w.q + (size_t)i * 16) : masked_vec<kBf16>();
#pragma unroll
    for (int j = 0; j < kPer / 4; ++j) ve[j] = load_vec(w.e + (size_t)i * kPer + 4 * j);
    Elems<kBf16>::unpack(vp, zp);
    Elems<kBf16>::unpack(vq, zq);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const uint32_t x[4] = {ve[j / 4].x, ve[j / 4].y, ve[j / 4].z, ve[j / 4].w};
        f(zp[j], zq[j], __uint_as_float(x[j & 3]), i * kPer + j);
    }
}

// CTAs per SM that the registers leave room for: of 256 threads four (128 x 151,936 bf16 111 us; with 76 registers, three, 122), of 512 threads two for
// f32 (clusters of four do not come out even on 148 SMs: 37 x 32,003 48.7 us, with one 56), one for bf16, whose loads want registers (16 sequences of
// 4 drafts x 151,936 30.4 us, with two 33.1).
template <bool kBf16, int kThreads, bool kCluster> __global__ void __launch_bounds__(kThreads, kThreads == 256 ? 4 : kBf16 ? 1 : 2) verify_pick_kernel(const Args a) {
    constexpr int kLog2 = kBf16 ? 3 : 2;
    __shared__ PickShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    enter_kernel();
    unsigned rank = 0, C = 1;
    if constexpr (kCluster) { C = cg::this_cluster().num_blocks(); rank = cg::this_cluster().block_rank(); }
    const int log2C = 31 - __clz((int)C);
    const int b = (int)(blockIdx.x >> log2C);

    const int nvec = a.V >> kLog2;
    const int v0 = (int)((long long)nvec * rank >> log2C), v1 = (int)((long long)nvec * (rank + 1) >> log2C);
    // the noise does not depend on where the sequence stops: on its way to L2 while that is found
    {
        const char* e = reinterpret_cast<const char*>(a.noise + (size_t)b * a.noise_stride);
        const long long lo = (long long)v0 << kLog2 << 2, hi = (long long)v1 << kLog2 << 2;
        for (long long at = lo + 128ll * tid; at < hi; at += 128ll * kThreads) asm volatile("prefetch.global.L2 [%0];" :: "l"(e + at));
    }

    // ---- the first rejection, by one warp of every CTA; the first CTA writes
    if (warp == 0) {
        const long long T = true_drafts(a);
        const int c0 = a.cu[b], c1 = a.cu[b + 1], n = c1 - c0;
        const bool fine = c0 >= 0 && c1 >= c0 && c1 <= T && a.cu[a.n_seqs] <= a.T_max;
        int n_acc = 0, state = fine ? 0 : 2;
        float2 sp = make_float2(0.0f, 0.0f), sq = sp;
        const long long base = (long long)c0 + b;
        bool bad_id = false, dropped = false;
        for (int j0 = 0; state == 0; j0 += 32) {                   // position n is the row after the last draft
            const int j = j0 + lane;
            bool accept = false, bad = false;
            int y = -1;
            float lp = 0.0f;
            float2 s = make_float2(kLowest, 0.0f), d = s;
            if (j <= n) {
                s = a.rows[base + j];
                bad = s.x != s.x;
            }
            if (j < n) {
                y = a.drafts[c0 + j];
                if (a.draft) { d = a.rows[a.T_max + a.n_seqs + c0 + j]; bad = bad || d.x != d.x; }
                if (y < 0 || y >= a.V) {
                    y = -1;
                } else if (!bad && s.y > 0.0f) {
                    const float zp = Elems<kBf16>::load1(a.target + (base + j) * a.target_bytes, y);
                    const double l = ((double)zp - (double)s.x) * a.inv_tau_t - log64((double)s.y);
                    double x = l;                                  // of p / q
                    if (a.draft) {
                        const float zq = Elems<kBf16>::load1(a.draft + (c0 + j) * a.draft_bytes, y);
                        if (zq > -INFINITY && d.y > 0.0f) x = l - (((double)zq - (double)d.x) * a.inv_tau_d - log64((double)d.y));
                        else x = l > -INFINITY ? INFINITY : l;
                    }
                    const float u = a.u[c0 + j];                   // 0: whatever is possible, also where exp64 returns 0
                    accept = l > -INFINITY && (x >= 700.0 || u == 0.0f || (double)u < exp64(x));
                    lp = (float)l;
                }
            }
            const unsigned stop = ~__ballot_sync(kAll, accept);
            const int first = stop ? __ffs(stop) - 1 : 32;
            if (rank == 0 && lane < first) { a.tokens[base + j] = y; a.logp[base + j] = lp; }
            if (first < 32) {
                n_acc = j0 + first;
                sp = make_float2(__shfl_sync(kAll, s.x, first), __shfl_sync(kAll, s.y, first));
                sq = make_float2(__shfl_sync(kAll, d.x, first), __shfl_sync(kAll, d.y, first));
                y = __shfl_sync(kAll, y, first);
                bad_id = n_acc < n && y < 0;
                dropped = n_acc < n && !a.draft;
                if (__shfl_sync(kAll, bad, first) || !(sp.y > 0.0f)) state = 1;
                if (lane == 0) {
                    sh.f.p = a.target + (base + n_acc) * a.target_bytes;
                    sh.f.q = n_acc < n && a.draft && sq.y > 0.0f ? a.draft + (c0 + n_acc) * a.draft_bytes : nullptr;
                    sh.f.e = a.noise + (size_t)b * a.noise_stride;
                    sh.f.mp = sp.x; sh.f.mq = sq.x;
                    sh.f.ip = 1.0f / sp.y; sh.f.iq = 1.0f / sq.y;
                    sh.f.drop = dropped ? y : -1;
                }
                break;
            }
        }
        if (rank == 0) {
            if (state == 2) {
                if (lane == 0) { a.n_accepted[b] = 0; set_status(a.status, DPPO_STATUS_BAD_SEGMENTS); }
            } else {
                for (int j = n_acc + 1 + lane; j <= n; j += 32) { a.tokens[base + j] = -1; a.logp[base + j] = 0.0f; }
                if (lane == 0) {
                    a.n_accepted[b] = n_acc;
                    if (bad_id) set_status(a.status, DPPO_STATUS_BAD_TARGET);
                    if (state == 1) {                              // an invalid row, or one that its mask leaves empty
                        a.tokens[base + n_acc] = -1;
                        a.logp[base + n_acc] = sp.y == 0.0f && sq.x == sq.x ? -INFINITY : __int_as_float(0x7fffffff);
                    }
                }
            }
        }
        if (lane == 0) { sh.sp = sp; sh.sq = sq; sh.row = base + n_acc; sh.state = state; }
    }
    __syncthreads();
    if (sh.state != 0) return;                                     // the same in every CTA of the cluster

    // ---- the race
    Field f = sh.f;
    const int tail0 = rank == C - 1 ? nvec << kLog2 : a.V;
    int won = -1;
    const double ln_sum = log64((double)sh.sp.y);
#pragma unroll 1
    for (int pass = 0; pass < 2 && won < 0; ++pass) {
        Race r = {0.0f, 0.0f, 0.0f, 0x7fffffff};
        float z_best = 0.0f;
        auto bounds = [&](float zp, float zq, float e, int at, float& hi, float& lo) {
            const float p = ex2((zp - f.mp) * a.ct) * f.ip;
            float w = p, t = p + kTiny;
            if (f.q) {
                const float q = ex2((zq - f.mq) * a.cd) * f.iq;
                w = p - q; t += q;
            }
            if (at == f.drop) w = t = 0.0f;
            const bool sure = e >= kLeastNoise && e <= kMostNoise;
            const float inv = __fdividef(1.0f, e);
            hi = sure ? fmaf(t, kEps, w) * inv : INFINITY;
            lo = sure ? fmaf(t, -kEps, w) * inv : 0.0f;
        };
        auto enter = [&](float zp, float zq, float e, int at) {
            float hi, lo;
            bounds(zp, zq, e, at, hi, lo);
            if (hi > r.hi) { r.second = r.hi; r.hi = hi; r.at = at; z_best = zp; }
            else if (hi > r.second) r.second = hi;
            if (lo > r.lo) r.lo = lo;
        };
        auto draft_at = [&](int at) { return f.q ? Elems<kBf16>::load1(f.q, at) : -INFINITY; };
        auto log_bound = [&](float lo) { return lo > 0.0f ? __log2f(lo) + __log2f(sh.sp.y) : -INFINITY; };
        if (tid == 0) { sh.bound = 0; sh.n_cand = 0; }
        __syncthreads();
        for_vector<kBf16>(f, v0 + tid, v1, enter);                 // every thread's first vector
        if (__any_sync(kAll, r.lo > 0.0f)) {                       // positive floats order as integers do
            const float best = warp_max_f32(r.lo);
            if (lane == 0) atomicMax(&sh.bound, __float_as_int(best));
        }
        __syncthreads();
        for_field<kBf16, kThreads, 2>(f, a.ct, v0 + kThreads, v1, tail0, a.V, log_bound(__int_as_float(sh.bound)), [&](float zp, float e, int at) {
            const int slot = atomicAdd(&sh.n_cand, 1);
            if (slot < kCand) { sh.z[slot] = zp; sh.e[slot] = e; sh.at[slot] = at; }
            else enter(zp, draft_at(at), e, at);                   // more than there is room for
        });
        __syncthreads();
        for (int i = tid; i < min(sh.n_cand, kCand); i += kThreads) enter(sh.z[i], draft_at(sh.at[i]), sh.e[i], sh.at[i]);
        const float z_mine = z_best;
        const int at_mine = r.at;
        r = race_cta<kThreads>(r, sh);
        if constexpr (kCluster) {
            cg::cluster_group cl = cg::this_cluster();
            if (tid == 0) sh.mine = r;
            cl.sync();
            r = race_warp(lane < (int)C ? *cl.map_shared_rank(&sh.mine, lane) : Race{0.0f, 0.0f, 0.0f, 0x7fffffff});
            cl.sync();
        }
        if (r.lo > 0.0f && r.second < r.lo && r.hi < INFINITY) {
            won = r.at;
            if (at_mine == won) {                                  // one thread of the cluster
                a.tokens[sh.row] = won;
                a.logp[sh.row] = (float)(((double)z_mine - (double)sh.sp.x) * a.inv_tau_t - ln_sum);
            }
            return;
        }
        if (r.hi > 0.0f) {                                         // in 64 bits, over the entries within reach (r.lo is finite)
            const double ip = 1.0 / (double)sh.sp.y, iq = f.q ? 1.0 / (double)sh.sq.y : 0.0;
            Exact x = {0.0, 0x7fffffff};
            const float bound = log_bound(r.lo);
            for_field<kBf16, kThreads, 1>(f, a.ct, v0, v1, tail0, a.V, bound, [&](float zp, float e, int at) {
                float hi, lo;
                const float zq = draft_at(at);
                bounds(zp, zq, e, at, hi, lo);
                if (!(hi >= r.lo) || !(hi > 0.0f) || !(zp > -INFINITY) || at == f.drop) return;
                double w = exp64(((double)zp - (double)f.mp) * a.inv_tau_t) * ip;
                if (zq > -INFINITY) w -= exp64(((double)zq - (double)f.mq) * a.inv_tau_d) * iq;
                if (w > 0.0) x = exact_join({w / (double)e, at}, x);
            });
            x = exact_cta<kThreads>(x, sh);
            if constexpr (kCluster) {
                cg::cluster_group cl = cg::this_cluster();
                if (tid == 0) sh.mine_exact = x;
                cl.sync();
                x = exact_warp(lane < (int)C ? *cl.map_shared_rank(&sh.mine_exact, lane) : Exact{0.0, 0x7fffffff});
                cl.sync();
            }
            if (x.x > 0.0) won = x.at;
        }
        f.q = nullptr; f.drop = -1;                                // p <= q everywhere: the target itself
    }
    if (rank == 0 && tid == 0) {
        if (won < 0 || won >= a.V) {                               // no entry with a positive, valid noise
            a.tokens[sh.row] = -1; a.logp[sh.row] = __int_as_float(0x7fffffff);
        } else {
            a.tokens[sh.row] = won;
            a.logp[sh.row] = (float)(((double)Elems<kBf16>::load1(f.p, won) - (double)sh.sp.x) * a.inv_tau_t - ln_sum);
        }
    }
}

// ---- host side -------------------------------------------------------------------------------------------
template <bool kBf16> static int run(const Args& a, cudaStream_t s) {
    const int nvec = a.V >> (kBf16 ? 3 : 2);
    const long long sms = sm_count(), rows = a.T_max + a.n_seqs + (a.draft ? a.T_max : 0);
    // Rows: a warp each up to 4 KB; a CTA each where they fill the SMs twice (1,414 x 151,936 bf16: 256 threads 71 us, 128 80; 4,096 x 8,003 f32
    // 512 threads 36.6, 256 37.2, 128 41.4); else a cluster (9 x 151,936: eight CTAs of 256 threads 5.0 us, four 5.9, one of 512 8.1).
    int rc, C = 1;
    if (nvec > 4096)
        while (C < kMaxCluster && rows * C < 2 * sms) C *= 2;
    if (rows * C > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "verify_drafts: %lld rows need too large a grid", rows);
    if (nvec <= 256) rc = launch_after("verify_drafts launch", verify_rows_warp_kernel<kBf16, 4>, (rows + 3) / 4, 128, 0, s, 1, a, rows);
    else if (C > 1) rc = launch_after("verify_drafts launch", verify_rows_kernel<kBf16, 256, true>, rows * C, 256, 0, s, C, a);
    else if (nvec <= 1024) rc = launch_after("verify_drafts launch", verify_rows_kernel<kBf16, 128, false>, rows, 128, 0, s, 1, a);
    else rc = launch_after("verify_drafts launch", verify_rows_kernel<kBf16, 256, false>, rows, 256, 0, s, 1, a);
    if (rc != DPPO_OK) return rc;
    // The race: four CTAs per sequence, of 512 threads where each has an SM to itself (37 x 32,003 f32 47.9 us with the rows; eight 56.5, two 49.5;
    // 128 x 151,936 bf16 109 with 256 threads, 139 with 512); eight for a few sequences (1: 16.3, four 19.0, sixteen 17.6), fewer for many.
    C = nvec <= 512 || a.n_seqs > 4 * sms ? 1 : a.n_seqs > 2 * sms ? 2 : 16ll * a.n_seqs > sms ? 4 : 8;
    const long long ctas = (long long)a.n_seqs * C;
    if (ctas > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "verify_drafts: too many sequences");
    if (C == 1) return launch_after("verify_drafts launch", verify_pick_kernel<kBf16, 256, false>, ctas, 256, 0, s, 1, a);
    if (ctas <= sms) return launch_after("verify_drafts launch", verify_pick_kernel<kBf16, 512, true>, ctas, 512, 0, s, C, a);
    return launch_after("verify_drafts launch", verify_pick_kernel<kBf16, 256, true>, ctas, 256, 0, s, C, a);
}

}  // namespace verify
}  // namespace dppo

extern "C" size_t dppo_verify_drafts_workspace_bytes(const dppo_verify_params* p) {
    if (!p || p->T_max < 0 || p->n_seqs < 0) return 0;
    return (size_t)(2 * p->T_max + p->n_seqs) * sizeof(float2);
}

extern "C" int dppo_verify_drafts(const dppo_verify_params* p, const void* target_logits, const void* draft_logits, const int32_t* drafts,
                                  const int32_t* cu_drafts, const float* uniforms, const float* noise, int32_t* n_accepted, int32_t* tokens_out,
                                  float* logp_out, void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
    dppo::NvtxRange nvtx_range("dppo_verify_drafts");
    using namespace dppo;
    if (!p) return fail(DPPO_ERR_INVALID_ARG, "verify_drafts: NULL params");
    if (p->T_max < 0 || p->n_seqs < 0 || p->V < 1)
        return fail(DPPO_ERR_INVALID_ARG, "verify_drafts: T_max=%lld n_seqs=%d V=%d", (long long)p->T_max, p->n_seqs, p->V);
    if (p->dtype != DPPO_F32 && p->dtype != DPPO_BF16) return fail(DPPO_ERR_UNSUPPORTED, "verify_drafts: dtype %d", p->dtype);
    if (!(p->temperature >= 1e-6) || !(p->temperature <= 1e6) || (draft_logits && (!(p->draft_temperature >= 1e-6) || !(p->draft_temperature <= 1e6))))
        return fail(DPPO_ERR_INVALID_ARG, "verify_drafts: temperatures must be in [1e-6, 1e6]");
    if (p->V > (1 << 30)) return fail(DPPO_ERR_BAD_SHAPE, "verify_drafts: V=%d, the limit is 2^30", p->V);
    if (2 * p->T_max + p->n_seqs >= ((int64_t)1 << 31)) return fail(DPPO_ERR_BAD_SHAPE, "verify_drafts: 2 T_max + n_seqs must be below 2^31");
    if (p->target_stride < p->V || (draft_logits && p->draft_stride < p->V) || p->noise_stride < p->V)
        return fail(DPPO_ERR_BAD_SHAPE, "verify_drafts: strides %lld, %lld, %lld < V %d", (long long)p->target_stride, (long long)p->draft_stride,
                    (long long)p->noise_stride, p->V);
    if (p->n_seqs == 0) return DPPO_OK;
    if (!target_logits || !cu_drafts || !noise || !n_accepted || !tokens_out || !logp_out || (p->T_max > 0 && (!drafts || !uniforms)))
        return fail(DPPO_ERR_INVALID_ARG, "verify_drafts: NULL array");
    const size_t esize = p->dtype == DPPO_BF16 ? 2 : 4;
    if (((uintptr_t)target_logits & 15) || ((uintptr_t)draft_logits & 15) || ((uintptr_t)noise & 15) || (p->target_stride * esize) % 16 != 0 ||
        (draft_logits && (p->draft_stride * esize) % 16 != 0) || p->noise_stride % 4 != 0 || ((uintptr_t)workspace & 15))
        return fail(DPPO_ERR_MISALIGNED, "verify_drafts: logits, noise and workspace bases and row strides must be multiples of 16 bytes");
    const size_t need = dppo_verify_drafts_workspace_bytes(p);
    if (!workspace || workspace_bytes < need) return fail(DPPO_ERR_WORKSPACE_TOO_SMALL, "verify_drafts: workspace of %zu bytes, %zu needed", workspace_bytes, need);
    verify::Args a = {};
    a.target = (const char*)target_logits; a.draft = (const char*)draft_logits; a.drafts = drafts; a.cu = cu_drafts; a.u = uniforms; a.noise = noise;
    a.n_accepted = n_accepted; a.tokens = tokens_out; a.logp = logp_out; a.rows = (float2*)workspace; a.status = status;
    a.T_max = p->T_max; a.target_bytes = (long long)(p->target_stride * esize); a.draft_bytes = (long long)(p->draft_stride * esize);
    a.noise_stride = p->noise_stride;
    a.n_seqs = p->n_seqs; a.V = p->V;
    a.inv_tau_t = 1.0 / p->temperature; a.ct = (float)(1.4426950408889634 / p->temperature);
    if (draft_logits) { a.inv_tau_d = 1.0 / p->draft_temperature; a.cd = (float)(1.4426950408889634 / p->draft_temperature); }
    return p->dtype == DPPO_BF16 ? verify::run<true>(a, (cudaStream_t)stream) : verify::run<false>(a, (cudaStream_t)stream);
}
