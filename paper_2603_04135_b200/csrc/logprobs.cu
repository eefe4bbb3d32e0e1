// Log-probs of given tokens with entropy and top alternatives, and their gradient with respect to the logits.
//
// Forward.  Per row: m = max z, S = sum e_v and Q = sum e_v y_v with y_v = (z_v - m) c, e_v = 2^y_v, c = log2(e)/tau;
// then l = ln S, lse = m/tau + l, logp = (z_y - m)/tau - l and entropy = l - ln2 Q/S (both terms are >= 0: nothing
// cancels on a peaked row).  One pass: every thread keeps an ONLINE (m, S, Q) over the 16-byte vectors it sees; a larger
// maximum M moves them by D = (m - M) c: S' = S 2^D, Q' = (Q + D S) 2^D.
//
// The alternatives need no second pass.  A thread's running maximum is known anyway at the end of the row, and the
// k-th largest of the threads' maxima, thr, is a lower bound of the k-th largest entry (k threads have an entry that
// large): a thread whose maximum is below thr holds none of the top k.  Each thread also leaves the maximum of every round of
// its sweep (4 vectors) in shared memory, so about k such groups of vectors are read again (a few KB of the row), entries
// >= thr become candidates, and a candidate's rank is the number of candidates ahead of it in the order (value
// descending, index ascending).  Too many candidates (ties) are met by rules that need no more memory: see collect_ties.
//
// A row is worked on by a TEAM: a warp (short rows), a CTA, or a cluster of CTAs that split the row and join through
// distributed shared memory (few rows: a decode batch).
//
// Backward.  dz_v = ([v = y] a - p_v (a + b (ln p_v + H))) / tau, with p_v recomputed from the row's (m, l, H).  No
// reduction: a streaming map, one read and one write per element.
#include <cooperative_groups.h>

#include <type_traits>

#include "common.cuh"
#include "grpo_loss.cuh"

namespace dppo {
using namespace packed;
namespace cg = cooperative_groups;

namespace logprob {

constexpr int kMaxTop = 32;
constexpr int kMaxCluster = 8;
constexpr int kCand = 512;                // candidate buffer of a CTA-sized team
constexpr int kCandWarp = 256;            // and of a warp-sized one
constexpr float kLowest = -3.402823466e38f;
constexpr float kFar = -2000.0f;          // exponents are held at or above this (2^-2000 is 0): 0 * (-inf) never arises

struct Args {
    const char* logits;
    const int32_t* target;
    const int32_t* n_tokens_dev;
    float *logp, *entropy, *lse;
    int32_t* top_ids;
    float* top_logp;
    float4* stats;
    int32_t* status;
    long long T_max, row_bytes;
    int V, k;
    float c, inv_tau;
};

// What a thread (then a warp, a CTA, a cluster) has seen of a row.  m = the largest entry (kLowest if there is none but
// -inf; then S = 0); bad: a NaN or +inf was among them.
struct Part {
    float m, S, Q;
    int bad;
};

__device__ __forceinline__ void rescale(Part& p, float M, float c) {
    const float D = fmaxf((p.m - M) * c, kFar), f = ex2(D);
    p.Q = fmaf(D, p.S, p.Q) * f;
    p.S *= f;
    p.m = M;
}
// The parts of a warp's lanes as one, in every lane: the maximum first, one rescale per lane, then the sums.
__device__ __forceinline__ float warp_max_f32(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ Part warp_join(Part p, float c) {
    rescale(p, warp_max_f32(p.m), c);
    p.S = warp_sum(p.S); p.Q = warp_sum(p.Q);
    p.bad = __any_sync(0xffffffffu, p.bad);
    return p;
}

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Largest entry of a vector (NaN if there is one).
template <bool kBf16> __device__ __forceinline__ float vec_max(const uint4& q) {
    if constexpr (kBf16) {
        __nv_bfloat162 a = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&q.x), *reinterpret_cast<const __nv_bfloat162*>(&q.y));
        a = __hmax2_nan(a, __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&q.z), *reinterpret_cast<const __nv_bfloat162*>(&q.w)));
        return max_nan(__low2float(a), __high2float(a));
    } else {
        return max_nan(max_nan(__uint_as_float(q.x), __uint_as_float(q.y)), max_nan(__uint_as_float(q.z), __uint_as_float(q.w)));
    }
}

__device__ __forceinline__ uint4 load_vec(const void* p) {
    uint4 q;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p));
    return q;
}

// The backward may write where it reads (in place): not the read-only path.
__device__ __forceinline__ uint4 load_vec_rw(const void* p) {
    uint4 q;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p) : "memory");
    return q;
}

// Running sums of a thread: pairs, so that the packed f32x2 instructions take two elements at a time.
//
// What bounds a long sweep is the 1000 W limit (at 6 TB/s of bf16 logits the clock falls from 1.9 to 1.6 GHz), so what
// counts is how little is done per element.  On ordinary rows ("quick") the exponent is one fma, y' = z c - r with
// r = fl(m c); all sums of the thread then carry the same shift res = m c - r (exact in f32), which comes out when m grows
// and at the end of the row.  bf16 entries so low that their exponential is 0 are lifted to m + kFar / c by a packed
// maximum, two per instruction.  Rows of other magnitudes (|m c| > 2^20: masks of the type's lowest value with
// nothing above, logits of 10^6) take the differences z - m first, so they keep them.
struct Acc {
    f32x2 S, Q;
    float m, nr, res;                     // maximum; -r and m c - r (0 unless quick)
    uint32_t m2, low2;                    // bf16 pairs: the maximum, and what lower entries are lifted to
    int quick, bad;
};
// The least bf16 value that is not below x (a NaN or a value beyond the type: no matter, its row is NaN or x is not exceeded).
__device__ __forceinline__ __nv_bfloat16 bf16_up(float x) {
    const uint32_t b = __float_as_uint(x);
    return __ushort_as_bfloat16((unsigned short)((b + ((int32_t)b < 0 ? 0u : 0xffffu)) >> 16));
}
__device__ __forceinline__ uint32_t bf16_pair(__nv_bfloat16 x) {
    const __nv_bfloat162 p = __halves2bfloat162(x, x);
    return *reinterpret_cast<const uint32_t*>(&p);
}
// The frame of maximum m.
__device__ __forceinline__ void acc_frame(Acc& a, float m, float c) {
    const float r = m * c;
    a.quick = fabsf(r) <= 1048576.0f && fabsf(m) <= 1e37f;
    a.m = m; a.nr = -r;
    a.res = a.quick ? fmaf(m, c, -r) : 0.0f;
    a.m2 = bf16_pair(__float2bfloat16_rn(m));                      // exact where the entries are bf16
    a.low2 = bf16_pair(__float2bfloat16_rd(m + kFar / c));
}
__device__ __forceinline__ void acc_init(Acc& a, float m, float c) {
    a.S = a.Q = pair_of(0.0f, 0.0f); a.bad = 0;
    acc_frame(a, m, c);
}
__device__ __forceinline__ Part acc_part(const Acc& a) {
    float s0, s1, q0, q1;
    unpair(a.S, s0, s1); unpair(a.Q, q0, q1);
    const float S = s0 + s1, f = ex2(-a.res);
    return {a.m, S * f, fmaf(-a.res, S, q0 + q1) * f, a.bad};
}
__device__ __forceinline__ void acc_grow(Acc& a, float vmax, float c) {
    if (!(vmax < INFINITY)) { a.bad = 1; return; }                 // NaN or +inf: the row's results are NaN
    const float x = (a.m - vmax) * c, res = a.res;
    acc_frame(a, vmax, c);
    const float D = fmaxf(x + (a.res - res), kFar), f = ex2(D);
    a.Q = mul2(fma2(pair_of(D, D), a.S, a.Q), pair_of(f, f));
    a.S = mul2(a.S, pair_of(f, f));
}
// The lanes of a warp together, so that they keep one maximum: a larger one then turns up a few times per row, not in nearly
// every round in some lane (a thread's r-th round holds its largest entry so far with probability 1 / r), and lanes that have
// seen nothing but masked entries have a frame all the same.
__device__ __forceinline__ void acc_grow_warp(Acc& a, float vmax, float c) {
    if (!(vmax < INFINITY)) { a.bad = 1; vmax = -INFINITY; }
    const float m = warp_max_f32(vmax);
    if (m > a.m) acc_grow(a, m, c);
}
__device__ __forceinline__ void acc_add(Acc& a, f32x2 y) {
    float y0, y1;
    unpair(y, y0, y1);
    const f32x2 e = pair_of(ex2(y0), ex2(y1));
    a.S = add2(a.S, e);
    a.Q = fma2(e, y, a.Q);
}
__device__ __forceinline__ void acc_add_far(Acc& a, f32x2 y) {     // y may be -inf
    float y0, y1;
    unpair(y, y0, y1);
    acc_add(a, pair_of(fmaxf(y0, kFar), fmaxf(y1, kFar)));
}
__device__ __forceinline__ void acc_pair_slow(Acc& a, float z0, float z1, float c) {
    acc_add_far(a, mul2(add2(pair_of(z0, z1), pair_of(-a.m, -a.m)), pair_of(c, c)));
}
// kN vectors in the frame of a maximum that none of them exceeds.  some: one of them is above -inf.
template <bool kBf16, int kN> __device__ __forceinline__ void acc_sum(Acc& a, const uint4 (&q)[kN], float c, bool some) {
    if (a.quick) {                                                 // one test per kN vectors: what follows is a straight line
        const f32x2 c2 = pair_of(c, c), nr2 = pair_of(a.nr, a.nr);
#pragma unroll
        for (int u = 0; u < kN; ++u) {
            const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
            if constexpr (kBf16) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __nv_bfloat162 z = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]), *reinterpret_cast<const __nv_bfloat162*>(&a.low2));
                    const uint32_t b = *reinterpret_cast<const uint32_t*>(&z);
                    acc_add(a, fma2(pair_of(__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)), c2, nr2));
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; i += 2) acc_add_far(a, fma2(pair_of(__uint_as_float(w[i]), __uint_as_float(w[i + 1])), c2, nr2));
            }
        }
    } else if (some) {
#pragma unroll 1
        for (int u = 0; u < kN; ++u) {
            uint4 v = q[0];                                        // selects: q stays in registers
#pragma unroll
            for (int j = 1; j < kN; ++j) v = u == j ? q[j] : v;
            float f[Elems<kBf16>::kPerVec];
            Elems<kBf16>::unpack(v, f);
#pragma unroll
            for (int i = 0; i < Elems<kBf16>::kPerVec; i += 2) acc_pair_slow(a, f[i], f[i + 1], c);
        }
    }
}
// kN vectors, by a whole warp; a larger maximum (or a NaN) is rare after the first few of a row.  Returns their largest entry
// as bf16, rounded up (NaN where there is one); own: the thread's largest so far.
template <bool kBf16, int kN> __device__ __forceinline__ __nv_bfloat16 acc_vecs(Acc& a, const uint4 (&q)[kN], float c, float& own) {
    __nv_bfloat16 top;
    float vmax;
    if constexpr (kBf16) {
        __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&q[0].x);
#pragma unroll
        for (int u = 0; u < kN; ++u) {
            const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
            for (int i = u == 0 ? 1 : 0; i < 4; ++i) x = __hmax2_nan(x, *reinterpret_cast<const __nv_bfloat162*>(&w[i]));
        }
        top = __hmax_nan(__low2bfloat16(x), __high2bfloat16(x));
        vmax = __bfloat162float(top);
        if (__any_sync(0xffffffffu, !__hble2(x, *reinterpret_cast<const __nv_bfloat162*>(&a.m2)))) acc_grow_warp(a, vmax, c);
    } else {
        vmax = vec_max<false>(q[0]);
#pragma unroll
        for (int u = 1; u < kN; ++u) vmax = max_nan(vmax, vec_max<false>(q[u]));
        top = bf16_up(vmax);
        if (__any_sync(0xffffffffu, !(vmax <= a.m))) acc_grow_warp(a, vmax, c);
    }
    own = fmaxf(own, vmax);
    acc_sum<kBf16, kN>(a, q, c, vmax > -INFINITY);
    return top;
}

// One entry (-inf: nothing).
__device__ __forceinline__ void acc_one(Acc& a, float z, float c) {
    if (!(z <= a.m)) acc_grow(a, z, c);
    const f32x2 z2 = pair_of(z, -INFINITY), c2 = pair_of(c, c);
    acc_add_far(a, a.quick ? fma2(z2, c2, pair_of(a.nr, a.nr)) : mul2(add2(z2, pair_of(-a.m, -a.m)), c2));
}

// Order of f32 values as unsigned numbers (-0 counts as +0; no NaN gets here).
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.0f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// An entry as one number: larger = ahead in the order (value descending, index ascending).
typedef unsigned long long Entry;
__device__ __forceinline__ Entry entry_of(float z, int idx) { return (Entry)key_of(z) << 32 | (uint32_t)~idx; }
__device__ __forceinline__ float entry_value(Entry e) { return value_of((uint32_t)(e >> 32)); }
__device__ __forceinline__ int entry_index(Entry e) { return (int)~(uint32_t)e; }

// What a CTA or a warp needs to select the alternatives.
template <int kThreads, int kCap> struct TeamShared {
    Entry cand[kCap];
    Entry list[kMaxTop];                   // the team's own sorted list (joined over a cluster)
    int n_cand, n_list;
    int red[kThreads / 32];
};
// A CTA that sweeps its part of a row in rounds of kRound vectors per thread.  best: the largest entry of each thread's
// vectors of a round (of 2^shift rounds), as bf16 rounded up.
constexpr int kRound = 4;
constexpr int kSlots = 32;
constexpr int kMaxGroups = 256;
template <int kThreads> struct CtaShared : TeamShared<kThreads, kCand> {
    Part part[kThreads / 32];
    Part row;
    float tmax[kThreads];
    __nv_bfloat16 best[kSlots][kThreads];
    float thr;
    int n_group;
    int group[kMaxGroups];                 // slot * kThreads + thread
};

template <int kThreads> __device__ __forceinline__ void team_sync() {
    if constexpr (kThreads == 32) __syncwarp(); else __syncthreads();
}

// A lower bound, as a key, of the k-th largest (1-based) of 32 * kPer keys (kPer per lane) that at least k of them reach:
// found bit by bit below the bits that all keys share, by counting; exact to kBits bits of the key (bf16 values have no
// more than 16, for f32 a slightly low bound costs a few more candidates).
template <int kPer, int kBits> __device__ __forceinline__ uint32_t kth_largest(const uint32_t (&own)[kPer], int k) {
    uint32_t hi = own[0], lo = own[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) { hi = max(hi, own[i]); lo = min(lo, own[i]); }
    hi = __reduce_max_sync(0xffffffffu, hi); lo = __reduce_min_sync(0xffffffffu, lo);
    int bit = 31 - __clz(hi ^ lo);                                 // -1: all keys alike
    uint32_t r = bit < 0 ? hi : hi & ~((2u << bit) - 1u);
    // two bits a step: the three counts are under way together
#pragma unroll 1
    for (bit -= 1; bit + 1 >= 32 - kBits; bit -= 2) {
        const uint32_t unit = bit >= 0 ? 1u << bit : 0u;           // bit < 0: the last step has one bit left
        const uint32_t t1 = r + unit, t2 = r + (bit >= 0 ? unit << 1 : 1u), t3 = t2 + unit;
        int c1 = 0, c2 = 0, c3 = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            c1 += own[i] >= t1 ? 1 : 0; c2 += own[i] >= t2 ? 1 : 0; c3 += own[i] >= t3 ? 1 : 0;
        }
        c1 = __reduce_add_sync(0xffffffffu, c1); c2 = __reduce_add_sync(0xffffffffu, c2); c3 = __reduce_add_sync(0xffffffffu, c3);
        if (c3 >= k) { r = t3; c1 = c3; }
        else if (c2 >= k) { r = t2; c1 = c2; }
        else if (c1 >= k) r = t1;
        if (c1 == k) break;                                        // exactly the k largest reach r
    }
    return r;
}

// The k-th largest of the lanes' values, at least kLowest: for a small k by taking the largest away k times (those that are
// equal go together), else out of the sorted values (a bitonic network over the lanes, 15 exchanges).
__device__ __forceinline__ float kth_of_lanes(float v, int k, int lane) {
    if (k <= 6) {
        float m = kLowest;
#pragma unroll 1
        for (int have = 0; have < k;) {
            m = warp_max_f32(v);
            if (!(m > kLowest)) return kLowest;
            have += __popc(__ballot_sync(0xffffffffu, v == m));
            v = v == m ? -INFINITY : v;
        }
        return m;
    }
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
        for (int step = size >> 1; step > 0; step >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, v, step);
            const bool larger = ((lane & step) == 0) == ((lane & size) == 0);     // descending overall
            v = larger ? fmaxf(v, o) : fminf(v, o);
        }
    }
    return fmaxf(__shfl_sync(0xffffffffu, v, k - 1), kLowest);
}

// The list of the top k of n entries in shared memory, by the threads tid = 0 .. stride - 1: an entry's place is the number
// of entries ahead of it.
__device__ __forceinline__ void rank_entries(const Entry* cand, int n, int k, Entry* list, int tid, int stride) {
    for (int i = tid; i < n; i += stride) {
        const Entry e = cand[i];
        int ahead = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) ahead += cand[j] > e ? 1 : 0;
        if (ahead < k) list[ahead] = e;
    }
}

// Entries of the row part [v0, v1) (in vectors) + tail [tail0, V) as a team sees them.
struct Span {
    const char* row;
    int v0, v1, tail0, tail1;
};

// Calls f(value, index) for every entry of the part that this thread owns in the sweep's own layout.
template <bool kBf16, int kThreads, class F> __device__ __forceinline__ void for_own(const Span& sp, int tid, F f) {
    constexpr int kPer = Elems<kBf16>::kPerVec;
    for (int i = sp.v0 + tid; i < sp.v1; i += kThreads) {
        float z[kPer];
        Elems<kBf16>::unpack(load_vec(sp.row + (size_t)i * 16), z);
#pragma unroll
        for (int j = 0; j < kPer; ++j) f(z[j], i * kPer + j);
    }
    if (sp.tail0 + tid < sp.tail1) f(Elems<kBf16>::load1(sp.row, sp.tail0 + tid), sp.tail0 + tid);
}

template <int kThreads, int kCap> __device__ __forceinline__ int team_count(TeamShared<kThreads, kCap>& sh, int cnt, int tid) {
    cnt = __reduce_add_sync(0xffffffffu, cnt);
    if constexpr (kThreads == 32) return cnt;
    __syncthreads();                                               // red[] may still be read from the last call
    if ((tid & 31) == 0) sh.red[tid >> 5] = cnt;
    __syncthreads();
    int s = 0;
    for (int w = 0; w < kThreads / 32; ++w) s += sh.red[w];
    return s;
}

// Too many entries at or above thr for the buffer: mostly ties, with fewer than kCap ABOVE it.  Where that fails too, thr is
// raised to the k-th largest entry itself (bit by bit, a counting sweep per bit): at most k - 1 are above that.  The entries
// above and the first k at thr, in index order, are then the candidates.  Leaves their number in sh.n_cand.
template <bool kBf16, int kThreads, int kCap>
__device__ __noinline__ void collect_ties(TeamShared<kThreads, kCap>& sh, const Span& sp, int k, float thr, int tid) {
    constexpr int kPer = Elems<kBf16>::kPerVec;
    const int lane = tid & 31, warp = tid >> 5;
    auto count_above = [&](float t) {
        int cnt = 0;
        for_own<kBf16, kThreads>(sp, tid, [&](float z, int) { cnt += z > t ? 1 : 0; });
        return team_count(sh, cnt, tid);
    };
    if (count_above(thr) > kCap - kMaxTop) {
        uint32_t r = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t t = r | (1u << bit);
            int cnt = 0;
            for_own<kBf16, kThreads>(sp, tid, [&](float z, int) { cnt += z > -INFINITY && key_of(z) >= t ? 1 : 0; });
            if (team_count(sh, cnt, tid) >= k) r = t;
        }
        thr = fmaxf(value_of(r), kLowest);
    }
    team_sync<kThreads>();
    if (tid == 0) sh.n_cand = 0;
    team_sync<kThreads>();
    for_own<kBf16, kThreads>(sp, tid, [&](float z, int idx) {
        if (z > thr) {
            const int at = atomicAdd(&sh.n_cand, 1);
            sh.cand[at] = entry_of(z, idx);                        // at most kCap - kMaxTop of them
        }
    });
    team_sync<kThreads>();
    const int n = sh.n_cand;
    team_sync<kThreads>();
    if (warp == 0) {
        int have = 0;
        auto take = [&](bool hit, int idx) {
            const uint32_t b = __ballot_sync(0xffffffffu, hit);
            const int at = have + __popc(b & ((1u << lane) - 1u));
            if (hit && at < k) sh.cand[n + at] = entry_of(thr, idx);
            have += __popc(b);
        };
        for (int i = sp.v0 * kPer; i < sp.v1 * kPer && have < k; i += 32) {
            const int idx = i + lane;
            take(idx < sp.v1 * kPer && Elems<kBf16>::load1(sp.row, idx) == thr, idx);
        }
        if (have < k) take(sp.tail0 + lane < sp.tail1 && Elems<kBf16>::load1(sp.row, sp.tail0 + lane) == thr, sp.tail0 + lane);
        if (lane == 0) sh.n_cand = n + (have < k ? have : k);
    }
    team_sync<kThreads>();
}

// The k-th largest of the threads' maxima, by one warp (fewer than k threads hold anything: every entry above -inf is a
// candidate).
template <bool kBf16, int kThreads> __device__ __forceinline__ float cta_threshold(const float* tmax, int k, int lane) {
    uint32_t own[kThreads / 32];
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) own[i] = key_of(tmax[i * 32 + lane]);
    return fmaxf(value_of(kth_largest<kThreads / 32, kBf16 ? 16 : 20>(own, k)), kLowest);
}

// The CTA's top k of its part, sorted, into sh.list / n_list.  sh.thr, sh.best and sh.tmax are set, n_group = n_cand = 0.
// About k of the (thread, round) groups can hold a candidate: their vectors are read again, a vector per thread (a whole hot
// thread's vectors, as a first version did, were 16 % of a row at k = 20, out of DRAM by then: 525 us for 8,192 rows).
template <bool kBf16, int kThreads>
__device__ __forceinline__ void select_top(CtaShared<kThreads>& sh, const Span& sp, int k, int n_slots, int shift, int tid) {
    constexpr int kPer = Elems<kBf16>::kPerVec;
    const float thr = sh.thr;
    if (sh.tmax[tid] >= thr) {
        uint32_t hits = 0;                                         // the loads before the first atomic
#pragma unroll 4
        for (int s = 0; s < n_slots; ++s) hits |= __bfloat162float(sh.best[s][tid]) >= thr ? 1u << s : 0u;
        int at = atomicAdd(&sh.n_group, __popc(hits));
        for (; hits != 0; hits &= hits - 1, ++at)
            if (at < kMaxGroups) sh.group[at] = (__ffs(hits) - 1) * kThreads + tid;
    }
    __syncthreads();
    auto offer = [&](float z, int idx) {
        if (z >= thr) {
            const int at = atomicAdd(&sh.n_cand, 1);
            if (at < kCand) sh.cand[at] = entry_of(z, idx);
        }
    };
    const int n_group = sh.n_group, log2_vecs = 2 + shift;         // kRound << shift vectors per group
    static_assert(kRound == 4, "log2_vecs");
    if (n_group <= kMaxGroups) {
        for (int i = tid; i < n_group << log2_vecs; i += kThreads) {
            const int g = sh.group[i >> log2_vecs], slot = g / kThreads, thread = g - slot * kThreads;
            const int v = sp.v0 + ((slot << log2_vecs) + (i & ((1 << log2_vecs) - 1))) * kThreads + thread;
            if (v >= sp.v1) continue;
            const uint4 q = load_vec(sp.row + (size_t)v * 16);
            float z[kPer];
            Elems<kBf16>::unpack(q, z);
            int cnt = 0;
#pragma unroll
            for (int j = 0; j < kPer; ++j) cnt += z[j] >= thr ? 1 : 0;
            if (cnt == 0) continue;
            int at = atomicAdd(&sh.n_cand, cnt);                   // one per vector
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (z[j] >= thr) {
                    if (at < kCand) sh.cand[at] = entry_of(z[j], v * kPer + j);
                    ++at;
                }
        }
        if (sp.tail0 + tid < sp.tail1) offer(Elems<kBf16>::load1(sp.row, sp.tail0 + tid), sp.tail0 + tid);
    }
    __syncthreads();
    if (n_group > kMaxGroups || sh.n_cand > kCand) collect_ties<kBf16, kThreads, kCand>(sh, sp, k, thr, tid);
    const int n = sh.n_cand;
    rank_entries(sh.cand, n, k, sh.list, tid, kThreads);
    if (tid == 0) sh.n_list = n < k ? n : k;
    __syncthreads();
}

// The outputs of a row from its sums.
struct RowOut {
    float l, H;
};
__device__ __forceinline__ bool is_empty(const Part& r) { return r.S == 0.0f && !r.bad; }
__device__ __forceinline__ RowOut row_out(const Args& a, const Part& r) {
    const float nan = __int_as_float(0x7fffffff);
    if (r.bad) return {nan, nan};
    if (is_empty(r)) return {0.0f, 0.0f};
    const float l = logf(r.S);
    return {l, fmaxf(l - r.Q / r.S * 0.6931471805599453f, 0.0f)};
}
__device__ __forceinline__ void write_scalars(const Args& a, long long t, const Part& r, const RowOut& o, float zy, int y_state) {
    const bool empty = is_empty(r);                                // a bad row's l is NaN, and so is what is formed with it
    if (a.lse) a.lse[t] = empty ? -INFINITY : r.bad ? o.l : fmaf(r.m, a.inv_tau, o.l);
    if (a.entropy) a.entropy[t] = o.H;
    if (a.stats) a.stats[t] = make_float4(r.bad ? o.l : empty ? -INFINITY : r.m, o.l, o.H, 0.0f);
    if (y_state != 0) set_status(a.status, y_state);
    if (a.logp) a.logp[t] = y_state != 0 ? 0.0f : r.bad ? o.l : empty ? -INFINITY : fmaf(zy - r.m, a.inv_tau, -o.l);
}
__device__ __forceinline__ void write_top(const Args& a, long long t, int j, float m, float l, int bad, const Entry* list, int n_list) {
    const bool have = !bad && j < n_list;
    const Entry e = have ? list[j] : 0;
    a.top_ids[t * a.k + j] = have ? entry_index(e) : -1;
    a.top_logp[t * a.k + j] = have ? fmaf(entry_value(e) - m, a.inv_tau, -l) : bad ? l : -INFINITY;
}

// Short rows: a warp per row at a time.  Rows of up to 32 kVecs vectors are held in registers (kVecs vectors per lane), so the
// maximum is known before the exponentials and the candidates are picked out of the registers; longer ones (kVecs = 0) are
// swept in rounds, as a CTA does it, without a CTA's five barriers per row.
// What such a row costs is instructions (871 per row of 1,021 f32 in a form that treated candidates and outputs entry by
// entry: 26 us for 20,011 rows), so: the vectors that hold a candidate (a few of the row's) go through shared memory, one lane
// per entry; a warp takes several consecutive rows, and the scalar outputs of all of them are formed in one pass, a lane
// per row.
constexpr int kMaxRun = 8;
constexpr int kWarpCtas = 7;               // resident CTAs (of four warps) per SM
constexpr int kHotVecs = 64;
template <bool kSweep> struct WarpShared;
template <> struct WarpShared<false> {
    TeamShared<32, kCandWarp> team;
    uint4 hot[kHotVecs];
    int hot_vec[kHotVecs];
    Entry list[kMaxRun][kMaxTop];
};
template <> struct WarpShared<true> {
    TeamShared<32, kCandWarp> team;
    __nv_bfloat16 best[kSlots][32];
    int group[kMaxGroups];                 // slot * 32 + lane
    Entry list[kMaxRun][kMaxTop];
};

template <bool kBf16, int kVecs, int kTeams>
__global__ void __launch_bounds__(32 * kTeams, kWarpCtas)                 // 28 warps per SM: 32 spill, 24 leave latencies uncovered
token_logprobs_warp_kernel(const Args a, int run) {
    constexpr int kPer = Elems<kBf16>::kPerVec, kLog2Per = kBf16 ? 3 : 2;
    constexpr uint32_t kNone = kBf16 ? 0xff80ff80u : 0xff800000u;  // -inf
    __shared__ WarpShared<kVecs == 0> shared[kTeams];
    const int lane = threadIdx.x & 31;
    auto& ws = shared[threadIdx.x >> 5];
    enter_kernel();
    const long long T = a.n_tokens_dev ? min((long long)*a.n_tokens_dev, a.T_max) : a.T_max;
    const long long t0 = ((long long)blockIdx.x * kTeams + (threadIdx.x >> 5)) * run;
    if (t0 >= T) return;
    const int n_rows = (int)min((long long)run, T - t0);
    const int nvec = a.V >> kLog2Per, tail = (nvec << kLog2Per) + lane;
    const int n_rounds = (nvec + kRound * 32 - 1) / (kRound * 32);
    int shift = 0;
    while (n_rounds > kSlots << shift) ++shift;

    // lane r: the given token of row t0 + r, and (below) the row's sums
    float zy = 0.0f;
    int y_state = 0, my_list = 0;
    Part mine = {kLowest, 0.0f, 0.0f, 0};
    if (lane < n_rows && a.target) {
        const int y = a.target[t0 + lane];
        if (y < 0 || y >= a.V) y_state = DPPO_STATUS_BAD_TARGET;
        else zy = Elems<kBf16>::load1(a.logits + (t0 + lane) * a.row_bytes, y);
    }
#pragma unroll 1
    for (int r = 0; r < n_rows; ++r) {
        const char* row = a.logits + (t0 + r) * a.row_bytes;
        const float zt = tail < a.V ? Elems<kBf16>::load1(row, tail) : -INFINITY;
        uint4 q[kVecs > 0 ? kVecs : kRound];
        float vm[kVecs > 0 ? kVecs : 1];                           // the vectors' maxima
        float mx;                                                  // the lane's
        Part p;
        if constexpr (kVecs > 0) {
#pragma unroll
            for (int u = 0; u < kVecs; ++u) {
                q[u] = make_uint4(kNone, kNone, kNone, kNone);
                if (u * 32 + lane < nvec) q[u] = load_vec(row + (size_t)(u * 32 + lane) * 16);
            }
            mx = zt;
#pragma unroll
            for (int u = 0; u < kVecs; ++u) { vm[u] = vec_max<kBf16>(q[u]); mx = max_nan(mx, vm[u]); }
            p.bad = __any_sync(0xffffffffu, !(mx < INFINITY));
            p.m = fmaxf(warp_max_f32(mx), kLowest);
            Acc acc;
            acc_init(acc, p.m, a.c);
            acc_sum<kBf16, kVecs>(acc, q, a.c, mx > -INFINITY);
            Part own = acc_part(acc);
            if (zt > -INFINITY) {
                const float y = fmaxf((zt - p.m) * a.c, kFar), e = ex2(y);
                own.S += e; own.Q = fmaf(e, y, own.Q);
            }
            p.S = warp_sum(own.S); p.Q = warp_sum(own.Q);
        } else {
            Acc acc;
            acc_init(acc, kLowest, a.c);
            mx = zt;
#pragma unroll 1
            for (int it = 0; it < n_rounds; ++it) {
                const int i = it * (kRound * 32) + lane;
                if ((it + 1) * (kRound * 32) <= nvec) {
#pragma unroll
                    for (int u = 0; u < kRound; ++u) q[u] = load_vec(row + (size_t)(i + u * 32) * 16);
                } else {                                           // the row's last vectors
#pragma unroll
                    for (int u = 0; u < kRound; ++u)
                        q[u] = i + u * 32 < nvec ? load_vec(row + (size_t)(i + u * 32) * 16) : make_uint4(kNone, kNone, kNone, kNone);
                }
                __nv_bfloat16 top = acc_vecs<kBf16, kRound>(acc, q, a.c, mx);
                if (a.k > 0) {
                    __nv_bfloat16* best = &ws.best[it >> shift][lane];
                    if (it & ((1 << shift) - 1)) top = __hmax(top, *best);
                    *best = top;
                }
            }
            acc_one(acc, zt, a.c);
            p = warp_join(acc_part(acc), a.c);
        }

        int n = 0;
        if (a.k > 0 && !p.bad) {
            const float thr = kth_of_lanes(mx, a.k, lane);
            const uint32_t below = (1u << lane) - 1u;
            auto offer = [&](float z, int idx) {                   // by all lanes together
                const uint32_t b = __ballot_sync(0xffffffffu, z >= thr);
                const int at = n + __popc(b & below);
                if (z >= thr && at < kCandWarp) ws.team.cand[at] = entry_of(z, idx);
                n += __popc(b);
            };
            if constexpr (kVecs > 0) {
                int n_hot = 0;
#pragma unroll
                for (int u = 0; u < kVecs; ++u) {
                    const uint32_t b = __ballot_sync(0xffffffffu, vm[u] >= thr);
                    if (b == 0) continue;
                    const int at = n_hot + __popc(b & below);
                    if (vm[u] >= thr && at < kHotVecs) { ws.hot[at] = q[u]; ws.hot_vec[at] = u * 32 + lane; }
                    n_hot += __popc(b);
                }
                __syncwarp();
                n = n_hot > kHotVecs ? kCandWarp + 1 : 0;
                for (int i = 0; i < n_hot * kPer && n <= kCandWarp; i += 32) {     // a lane per entry
                    const int e = i + lane, h = e >> kLog2Per, j = e & (kPer - 1);
                    const bool in = e < n_hot * kPer;
                    offer(in ? Elems<kBf16>::load1(&ws.hot[h], j) : -INFINITY, in ? ws.hot_vec[h] * kPer + j : 0);
                }
            } else {
                const int n_slots = (n_rounds + (1 << shift) - 1) >> shift, log2_vecs = 2 + shift;
                int n_group = 0;
                for (int s = 0; s < n_slots; ++s) {
                    const bool hit = __bfloat162float(ws.best[s][lane]) >= thr;
                    const uint32_t b = __ballot_sync(0xffffffffu, hit);
                    const int at = n_group + __popc(b & below);
                    if (hit && at < kMaxGroups) ws.group[at] = s * 32 + lane;
                    n_group += __popc(b);
                }
                __syncwarp();
                n = n_group > kMaxGroups ? kCandWarp + 1 : 0;
                for (int i0 = 0; i0 < n_group << log2_vecs && n <= kCandWarp; i0 += 32) {      // a lane per vector
                    const int i = i0 + lane;
                    uint4 v = make_uint4(kNone, kNone, kNone, kNone);
                    int at = 0;
                    if (i < n_group << log2_vecs) {
                        const int g = ws.group[i >> log2_vecs];
                        at = (((g >> 5) << log2_vecs) + (i & ((1 << log2_vecs) - 1))) * 32 + (g & 31);
                        if (at < nvec) v = load_vec(row + (size_t)at * 16);
                    }
                    float z[kPer];
                    Elems<kBf16>::unpack(v, z);
#pragma unroll
                    for (int j = 0; j < kPer; ++j)
                        if (__any_sync(0xffffffffu, z[j] >= thr)) offer(z[j], at * kPer + j);
                }
            }
            if (__any_sync(0xffffffffu, zt >= thr)) offer(zt, tail);
            __syncwarp();
            if (n > kCandWarp) {                                   // ties
                const Span sp = {row, 0, nvec, nvec << kLog2Per, a.V};
                collect_ties<kBf16, 32, kCandWarp>(ws.team, sp, a.k, thr, lane);
                n = ws.team.n_cand;
            }
            rank_entries(ws.team.cand, n, a.k, ws.list[r], lane, 32);
            n = min(n, a.k);
            __syncwarp();
        }
        if (lane == r) { mine = p; my_list = n; }
    }

    const RowOut o = row_out(a, mine);
    if (lane < n_rows) write_scalars(a, t0 + lane, mine, o, zy, y_state);
    for (int r = 0; r < n_rows; ++r) {
        const float m = __shfl_sync(0xffffffffu, mine.m, r), l = __shfl_sync(0xffffffffu, o.l, r);
        const int bad = __shfl_sync(0xffffffffu, mine.bad, r), n = __shfl_sync(0xffffffffu, my_list, r);
        if (lane < a.k) write_top(a, t0 + r, lane, m, l, bad, ws.list[r], n);
    }
}

// A CTA per row; kCluster: the CTAs of a cluster split it (blockIdx.x / cluster size = row).
template <bool kBf16, int kThreads, bool kCluster>
__global__ void __launch_bounds__(kThreads)
token_logprobs_kernel(const Args a) {
    constexpr int kLog2Per = kBf16 ? 3 : 2;
    __shared__ CtaShared<kThreads> sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    wait_for_previous();
    const long long T = a.n_tokens_dev ? min((long long)*a.n_tokens_dev, a.T_max) : a.T_max;
    unsigned rank = 0, C = 1;
    if constexpr (kCluster) { C = cg::this_cluster().num_blocks(); rank = cg::this_cluster().block_rank(); }
    const int log2C = 31 - __clz((int)C);                          // C = 1, 2, 4 or 8
    const long long t = (long long)(blockIdx.x >> log2C);
    if (t >= T) return;                                            // the whole cluster leaves together

    const char* row = a.logits + t * a.row_bytes;
    const int nvec = a.V >> kLog2Per;
    Span sp;
    sp.row = row;
    sp.v0 = (int)((long long)nvec * rank >> log2C);
    sp.v1 = (int)((long long)nvec * (rank + 1) >> log2C);
    sp.tail0 = rank == C - 1 ? nvec << kLog2Per : a.V;
    sp.tail1 = a.V;

    // the given token: asked for while the row streams
    float zy = 0.0f;
    int y_state = 0;
    if (rank == 0 && tid == 0 && a.target) {
        const int y = a.target[t];
        if (y < 0 || y >= a.V) y_state = DPPO_STATUS_BAD_TARGET;
        else zy = Elems<kBf16>::load1(row, y);
    }

    Acc acc;
    acc_init(acc, kLowest, a.c);
    float own = -INFINITY;                                         // the thread's largest entry
    constexpr uint32_t kNone = kBf16 ? 0xff80ff80u : 0xff800000u;  // -inf
    const int n_rounds = (sp.v1 - sp.v0 + kRound * kThreads - 1) / (kRound * kThreads);
    int shift = 0;
    while (n_rounds > kSlots << shift) ++shift;
    for (int it = 0; it < n_rounds; ++it) {
        const int i = sp.v0 + it * (kRound * kThreads) + tid;
        uint4 q[kRound];
        if (i - tid + kRound * kThreads <= sp.v1) {
#pragma unroll
            for (int u = 0; u < kRound; ++u) q[u] = load_vec(row + (size_t)(i + u * kThreads) * 16);
        } else {                                                   // the part's last vectors
#pragma unroll
            for (int u = 0; u < kRound; ++u)
                q[u] = i + u * kThreads < sp.v1 ? load_vec(row + (size_t)(i + u * kThreads) * 16) : make_uint4(kNone, kNone, kNone, kNone);
        }
        __nv_bfloat16 top = acc_vecs<kBf16, kRound>(acc, q, a.c, own);
        if (a.k > 0) {
            __nv_bfloat16* best = &sh.best[it >> shift][tid];
            if (it & ((1 << shift) - 1)) top = __hmax(top, *best);
            *best = top;
        }
    }
    if (sp.tail0 + tid < sp.tail1) {
        const float z = Elems<kBf16>::load1(row, sp.tail0 + tid);
        acc_one(acc, z, a.c);
        own = fmaxf(own, z);
    }
    if (a.k > 0) sh.tmax[tid] = own;
    Part p = warp_join(acc_part(acc), a.c);
    if (lane == 0) sh.part[warp] = p;
    __syncthreads();
    if (warp == 0) {                                               // two warps at a time: the row's sums, the threshold
        p = warp_join(lane < kThreads / 32 ? sh.part[lane] : Part{kLowest, 0.0f, 0.0f, 0}, a.c);
        if (lane == 0) { sh.row = p; sh.n_group = 0; sh.n_cand = 0; }
    } else if (warp == 1 && a.k > 0) {
        const float thr = cta_threshold<kBf16, kThreads>(sh.tmax, a.k, lane);
        if (lane == 0) sh.thr = thr;
    }
    __syncthreads();
    if (a.k > 0 && !sh.row.bad) select_top<kBf16, kThreads>(sh, sp, a.k, (n_rounds + (1 << shift) - 1) >> shift, shift, tid);

    if constexpr (kCluster) {
        cg::cluster_group cl = cg::this_cluster();
        if (a.k > 0 && tid < kMaxTop && (sh.row.bad || tid >= sh.n_list)) sh.list[tid] = 0;      // 0 past the end of the list
        cl.sync();                                                 // every CTA's part and list are in its shared memory
        if (rank != 0) {                                           // ... which lasts until the first CTA has read it
            let_next_start();
            cl.sync();
            return;
        }
        // the sorted lists side by side (a thread holds its entry too), and the sums: one round of remote reads
        constexpr int kMine = kMaxCluster * kMaxTop / kThreads > 0 ? kMaxCluster * kMaxTop / kThreads : 1;
        Entry mine[kMine];
        if (a.k > 0) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const int at = i * kThreads + tid;
                mine[i] = 0;
                if (at < (int)C * kMaxTop) mine[i] = cl.map_shared_rank(&sh, at / kMaxTop)->list[at % kMaxTop];
            }
        }
        if (warp == 0) {
            Part o = {kLowest, 0.0f, 0.0f, 0};
            if (lane < (int)C) o = cl.map_shared_rank(&sh, lane)->row;
            o = warp_join(o, a.c);
            if (lane == 0) sh.part[0] = o;
        }
        if (a.k > 0) {
#pragma unroll
            for (int i = 0; i < kMine; ++i)
                if (i * kThreads + tid < kMaxCluster * kMaxTop) sh.cand[i * kThreads + tid] = mine[i];
        }
        cl.barrier_arrive();                                       // the others may go
        __syncthreads();
        if (tid == 0) { sh.row = sh.part[0]; sh.n_list = 0; }
        __syncthreads();
        if (a.k > 0) {
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
                const Entry e = mine[i];
                if (e == 0) continue;
                // entries ahead: by bisection of every list, its own included (all lists a step at a time)
                int n[kMaxCluster], ahead = 0;
#pragma unroll
                for (int c = 0; c < kMaxCluster; ++c) n[c] = c * kMaxTop;
#pragma unroll
                for (int step = kMaxTop / 2; step > 0; step >>= 1)
#pragma unroll
                    for (int c = 0; c < kMaxCluster; ++c) n[c] += sh.cand[n[c] + step - 1] > e ? step : 0;
#pragma unroll
                for (int c = 0; c < kMaxCluster; ++c) ahead += n[c] - c * kMaxTop + (sh.cand[n[c]] > e ? 1 : 0);
                if (ahead < a.k) { sh.list[ahead] = e; atomicMax(&sh.n_list, ahead + 1); }
            }
            __syncthreads();
        }
        cl.barrier_wait();
    }

    let_next_start();
    if (warp < 2) {                                                // k <= 32: a warp for the scalars, one for the alternatives
        const Part r = sh.row;
        const RowOut o = row_out(a, r);
        if (tid == 0) write_scalars(a, t, r, o, zy, y_state);
        if (warp == 1 && lane < a.k) write_top(a, t, lane, r.m, o.l, r.bad, sh.list, sh.n_list);
    }
}

// ---- backward -----------------------------------------------------------------------------------------
struct BwdArgs {
    const char* logits;
    char* dlogits;
    const int32_t* target;
    const int32_t* n_tokens_dev;
    const float4* stats;
    const float *dlogp, *dentropy;
    int32_t* status;
    long long T_max, row_bytes;
    int V, chunks, chunk_vecs;           // a row is taken in `chunks` pieces of chunk_vecs vectors
    float c, inv_tau;
};

// dz = -p (A + X x), x = z - m, p = 2^(x c - l log2(e)), A = (a + b (H - l)) / tau, X = b / tau^2.
struct BwdRow {
    float nm, l2n, nA, nX;               // -m, -l log2(e), -A, -X
    float far;                           // x is held at or above this: p is 0 there
    uint32_t low2;                       // bf16 pair: m + far, rounded down
};

__device__ __forceinline__ f32x2 bwd_pair(float z0, float z1, const BwdRow& r, float c, bool lift) {
    f32x2 x = add2(pair_of(z0, z1), pair_of(r.nm, r.nm));
    if (lift) {
        float x0, x1;
        unpair(x, x0, x1);
        x = pair_of(fmaxf(x0, r.far), fmaxf(x1, r.far));
    }
    float y0, y1;
    unpair(fma2(x, pair_of(c, c), pair_of(r.l2n, r.l2n)), y0, y1);
    return mul2(pair_of(ex2(y0), ex2(y1)), fma2(x, pair_of(r.nX, r.nX), pair_of(r.nA, r.nA)));
}

template <bool kBf16, int kThreads, int kTeams, int kUnroll>
__global__ void __launch_bounds__(kThreads * kTeams)
token_logprobs_bwd_kernel(const BwdArgs a) {
    constexpr int kPer = Elems<kBf16>::kPerVec, kLog2Per = kBf16 ? 3 : 2;
    const int team = kTeams == 1 ? 0 : threadIdx.x / kThreads;
    const int tid = kTeams == 1 ? threadIdx.x : threadIdx.x % kThreads;
    enter_kernel();
    const long long T = a.n_tokens_dev ? min((long long)*a.n_tokens_dev, a.T_max) : a.T_max;
    const long long item = (long long)blockIdx.x * kTeams + team;
    const long long t = a.chunks == 1 ? item : item / a.chunks;
    const int chunk = a.chunks == 1 ? 0 : (int)(item - t * a.chunks);
    if (t >= T) return;

    const float4 st = a.stats[t];
    const int y = a.target ? a.target[t] : 0;
    const float da = a.dlogp ? a.dlogp[t] : 0.0f, db = a.dentropy ? a.dentropy[t] : 0.0f;
    const bool bad_y = a.target && (y < 0 || y >= a.V);
    const bool zero = bad_y || st.x == -INFINITY;
    if (bad_y && tid == 0 && chunk == 0) set_status(a.status, DPPO_STATUS_BAD_TARGET);
    BwdRow r;
    r.nm = -st.x; r.l2n = -st.y * 1.4426950408889634f;
    const float ga = da * a.inv_tau, gb = db * a.inv_tau;
    r.nA = -fmaf(gb, st.z - st.y, ga);
    r.nX = -gb * a.inv_tau;
    r.far = kFar / a.c;
    r.low2 = bf16_pair(__float2bfloat16_rd(st.x + r.far));
    // bf16 entries are lifted by a packed maximum before they are unpacked, where m + far lies well below m (the forward's quick
    // frame: |far / m| >= 2^-9.1).  Of a maximum further from zero, far rounds away, low2 would be m itself and every entry, masked
    // ones too, would count as the maximum: there (and for f32) the differences come first and are held at far.
    const bool lift = !kBf16 || !(fabsf(st.x * a.c) <= 1048576.0f && fabsf(st.x) <= 1e37f);

    const char* row = a.logits + t * a.row_bytes;
    char* out = a.dlogits + t * a.row_bytes;
    const int nvec = a.V >> kLog2Per, tail0 = nvec << kLog2Per;
    const int v0 = chunk * a.chunk_vecs, v1 = min(nvec, v0 + a.chunk_vecs);
    // the given token's element is formed apart and stored by the thread that stores its vector, after that
    const int vy = y >> kLog2Per;
    const bool mine = a.dlogp && !zero && (y < tail0 ? vy >= v0 && vy < v1 && (vy - v0) % kThreads == tid
                                                     : chunk == a.chunks - 1 && y - tail0 == tid);
    const float zy = mine ? Elems<kBf16>::load1(row, y) : 0.0f;

    auto put = [&](uint4 q, int i, auto lift_f32) {
        if constexpr (kBf16 && !decltype(lift_f32)::value) {
            uint32_t* w[4] = {&q.x, &q.y, &q.z, &q.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 h = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(w[j]), *reinterpret_cast<const __nv_bfloat162*>(&r.low2));
                *w[j] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
        float z[kPer];
        Elems<kBf16>::unpack(q, z);
#pragma unroll
        for (int j = 0; j < kPer; j += 2) unpair(bwd_pair(z[j], z[j + 1], r, a.c, decltype(lift_f32)::value), z[j], z[j + 1]);
        __stcs(reinterpret_cast<uint4*>(out) + i, Elems<kBf16>::pack(z));
    };
    auto sweep = [&](auto lift_f32) {
        for (int i = v0 + tid; i - tid < v1; i += kUnroll * kThreads) {        // all loads of a round before its stores
            uint4 q[kUnroll];
            if (i - tid + kUnroll * kThreads <= v1) {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) q[u] = load_vec_rw(row + (size_t)(i + u * kThreads) * 16);
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) put(q[u], i + u * kThreads, lift_f32);
            } else {
#pragma unroll
                for (int u = 0; u < kUnroll; ++u)
                    if (i + u * kThreads < v1) q[u] = load_vec_rw(row + (size_t)(i + u * kThreads) * 16);
#pragma unroll
                for (int u = 0; u < kUnroll; ++u)
                    if (i + u * kThreads < v1) put(q[u], i + u * kThreads, lift_f32);
            }
        }
    };
    if (zero) {
        for (int i = v0 + tid; i < v1; i += kThreads) __stcs(reinterpret_cast<uint4*>(out) + i, make_uint4(0u, 0u, 0u, 0u));
    } else if (lift) {
        sweep(std::true_type());
    } else {
        sweep(std::false_type());
    }
    float g, unused;
    if (chunk == a.chunks - 1 && tail0 + tid < a.V) {
        unpair(bwd_pair(Elems<kBf16>::load1(row, tail0 + tid), 0.0f, r, a.c, true), g, unused);
        Elems<kBf16>::store1(out, tail0 + tid, zero ? 0.0f : g);
    }
    if (mine) {
        unpair(bwd_pair(zy, 0.0f, r, a.c, true), g, unused);
        Elems<kBf16>::store1(out, y, g + ga);
    }
}

// ---- host side ---------------------------------------------------------------------------------------
template <bool kBf16, int kThreads, bool kCluster>
static int launch_fwd(const Args& a, int C, cudaStream_t s) {
    auto kernel = token_logprobs_kernel<kBf16, kThreads, kCluster>;
    if (!kCluster) {
        return launch_after("token_logprobs launch", kernel, a.T_max, kThreads, 0, s, 1, a);
    }
    if (a.T_max * C > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "token_logprobs: T_max=%lld needs too large a grid", a.T_max);
    return launch_after("token_logprobs launch", kernel, a.T_max * C, kThreads, 0, s, C, a);
}

template <bool kBf16, int kVecs> static int launch_warp(const Args& a, cudaStream_t s) {
    constexpr int kTeams = 4;
    // Rows per warp: one where they are fewer than two waves of warps, else what takes the fewest rows one after the other, in
    // whole waves (20,011 x 1,021 f32: 5 rows a warp, one wave, 22 us; 4 rows, 1.2 waves, 27; 5,000: 1 row 8.0, 2 rows 9.3).
    const long long wave = (long long)kWarpCtas * kTeams * sm_count();
    int run = 1;
    if (a.T_max > 2 * wave) {
        long long best = 0;
        for (int r = 1; r <= kMaxRun; ++r) {
            const long long rows = ((a.T_max + r - 1) / r + wave - 1) / wave * r;
            if (best == 0 || rows <= best) { best = rows; run = r; }
        }
    }
    const long long warps = (a.T_max + run - 1) / run;
    return launch_after("token_logprobs launch", token_logprobs_warp_kernel<kBf16, kVecs, kTeams>, (warps + kTeams - 1) / kTeams, 32 * kTeams,
                        0, s, 1, a, run);
}

// The launch shape of the CTA and cluster kernels: CTAs per row and threads per CTA.  `n` below is the CTAs that the fullest SM
// gets; 2, 5 and 10 CTAs of 512, 256 and 128 threads fit on one (48 registers a thread).
struct Shape { int C, threads; };

static Shape row_shape(long long T, int nvec, bool alternatives) {
    const long long sms = sm_count();
    auto per_sm = [&](long long ctas) { return (ctas + sms - 1) / sms; };
    if (nvec <= 512) return {1, 128};
    // Rows over 80 KB (64 KB for a few without alternatives) are split over a cluster where they do not fill the SMs evenly.
    // The time in us: the rows' share that the fullest SM reads, at 30 KB/us (12 % slower when a single CTA has the SM), and
    // the join, which costs more with alternatives.  (48 rows of 256,000 f32: 12.2 in eight CTAs, 17.7 in four; 90: 20.4 in
    // four; 300: 50.7 in two, 65.9 in one; 444 are even: one.  Over 260 random shapes of 1 to 12,000 rows of 1,200 to 260,000
    // entries this rule and the one for warps take a shape 0.6 % from the best of all, 16 % at worst.)
    const bool very_long = nvec >= (alternatives ? 30000 : 12000);
    int C = 1;
    if (nvec > 5120 || (nvec > 4096 && !alternatives && 8 * T <= sms)) {
        constexpr float kJoin[4] = {0.f, 0.5f, 1.0f, 0.5f}, kJoinAlternatives[4] = {0.f, 1.4f, 1.6f, 1.5f};
        float best = 0;
        for (int i = 0; i < 4; ++i) {
            const long long n = per_sm(T << i);
            // A cluster's CTAs start together, so close to full SMs the last clusters wait (183 x 160,597 f32: 34 us in four CTAs,
            // 29 in two), and three CTAs per SM crowd each other in the selection (48 x 151,936 bf16 out of L2, 8 alternatives:
            // 10.2 us in eight CTAs, 9.4 in four).
            const int quarters = i < 3 ? 21 - i : very_long || !alternatives ? 16 : 8;       // of an SM's count of CTAs
            if (i > 0 && 4 * (T << i) > quarters * sms) break;
            const float t = (float)n / (float)(1 << i) * (n == 1 ? 1.12f : 1.f) * (float)nvec * (16.f / 30e3f)
                          + (alternatives ? kJoinAlternatives[i] : kJoin[i]);
            if (i == 0 || t < best) { best = t; C = 1 << i; }
        }
    }
    const long long n = per_sm(T * C);
    if (C == 8) return {C, very_long && 4 * T * C <= 7 * sms ? 512 : 256};
    if (C == 4) return {C, n <= 2 && (very_long || !alternatives) ? 512 : 256};
    if (C == 2) return {C, n <= 2 ? 512 : 256};
    // One CTA per row: the largest that leave every SM's rows resident at once (1,000 x 151,936 f32: 96 us with 128 threads, 106
    // with 256; 296: 30.6 with 512, 40.3 with 256); in many waves the smallest (8,192 x 151,936 bf16: 416 against 449).
    // Shorter rows give a large CTA too little to do for its reductions (148 x 16,384 bf16 with alternatives: 256 threads).
    if (nvec <= 1024) return {1, n <= 3 ? 256 : 128};
    if (nvec <= 2048) return {1, n <= 2 && !alternatives ? 512 : n <= 4 ? 256 : 128};
    return {1, n <= 2 ? 512 : n <= 5 ? 256 : n <= 10 || n >= 24 ? 128 : 256};
}

template <bool kBf16> static int run_fwd(const Args& a, int variant, cudaStream_t s) {
    const int nvec = a.V >> (kBf16 ? 3 : 2);
    int C = 1, threads = 256;
    if (variant == 0) {
        // Rows of up to 4 KB: a warp each (20,011 x 1,021 f32: 22 us, a CTA each 68).  Up to 20 KB where there are enough of them
        // to fill the SMs with warps (20,000 x 2,048 f32, 8 alternatives: 41 us against 66; 1,000 of them: 8.1 against 6.1;
        // 20,000 x 5,120: 83 against 96, 2,000 of them 15.6 against 14.4; 20,000 x 6,144: no gain either way), without
        // alternatives up to 12 KB (20,000 x 2,800: 46 against 52; 6,000 x 4,096: 23 against 20).
        const long long sms = sm_count();
        if (nvec <= 256 || (nvec <= 768 && a.T_max >= 13 * sms) || (nvec <= 1280 && a.k > 0 && a.T_max >= 20 * sms)) {
            threads = 32;
        } else {
            const Shape sh = row_shape(a.T_max, nvec, a.k > 0);
            C = sh.C; threads = sh.threads;
        }
    } else if (variant == 32) {
        threads = 32;
    } else {
        C = variant / 10000; threads = variant % 10000;
    }
    if (threads == 32 && C == 1) {
        if (nvec <= 32) return launch_warp<kBf16, 1>(a, s);
        if (nvec <= 64) return launch_warp<kBf16, 2>(a, s);
        if (nvec <= 128) return launch_warp<kBf16, 4>(a, s);
        if (nvec <= 256) return launch_warp<kBf16, 8>(a, s);
        return launch_warp<kBf16, 0>(a, s);
    }
    if (C == 1 && threads == 128) return launch_fwd<kBf16, 128, false>(a, 1, s);
    if (C == 1 && threads == 256) return launch_fwd<kBf16, 256, false>(a, 1, s);
    if (C == 1 && threads == 512) return launch_fwd<kBf16, 512, false>(a, 1, s);
    if (C == 2 || C == 4 || C == 8) {
        if (threads == 128) return launch_fwd<kBf16, 128, true>(a, C, s);
        if (threads == 256) return launch_fwd<kBf16, 256, true>(a, C, s);
        if (threads == 512) return launch_fwd<kBf16, 512, true>(a, C, s);
    }
    return fail(DPPO_ERR_UNSUPPORTED, "token_logprobs: variant %d", variant);
}

template <bool kBf16, int kThreads, int kTeams, int kUnroll> static int launch_bwd(const BwdArgs& a, cudaStream_t s) {
    const long long ctas = (a.T_max * a.chunks + kTeams - 1) / kTeams;
    if (ctas > 0x7fffffffll) return fail(DPPO_ERR_BAD_SHAPE, "token_logprobs_backward: T_max=%lld needs too large a grid", a.T_max);
    return launch_after("token_logprobs_backward launch", token_logprobs_bwd_kernel<kBf16, kThreads, kTeams, kUnroll>, ctas, kThreads * kTeams, 0, s, 1, a);
}

template <bool kBf16> static int run_bwd(BwdArgs a, cudaStream_t s) {
    const int nvec = a.V >> (kBf16 ? 3 : 2);
    const long long sms = sm_count(), T = a.T_max;
    a.chunks = 1; a.chunk_vecs = nvec;
    // A warp per row of up to 5 KB, its loads in rounds of four (20,011 x 1,021 f32: 27 us = 6.0 TB/s; rounds of two 30, of
    // eight 28); a round does not go past the end of a very short one (100,000 x 128 bf16: 46 us in rounds of four).  Fewer
    // rows than the SMs have places for warps go the quicker way below (300 x 2,000 bf16: 3.0 us in warps, 2.3).
    if (nvec <= 64 || (nvec <= 320 && T > (nvec <= 128 ? 3 : 8) * sms)) {
        if (nvec <= 32) return launch_bwd<kBf16, 32, 4, 1>(a, s);
        if (nvec <= 64) return launch_bwd<kBf16, 32, 4, 2>(a, s);
        return launch_bwd<kBf16, 32, 4, 4>(a, s);
    }
    // Longer rows in chunks, a CTA each, every thread's loads before its first store.
    auto cut = [&](int limit, int unit) {                          // equal chunks, of whole units
        a.chunks = (nvec + limit - 1) / limit;
        a.chunk_vecs = ((nvec + a.chunks - 1) / a.chunks + unit - 1) / unit * unit;
        a.chunks = (nvec + a.chunk_vecs - 1) / a.chunk_vecs;
    };
    // Little work, where latency counts: 128 threads of four loads (1,000 x 4,096 bf16 4.7 us, 7.6 with a warp per row; 64 x
    // 75,968 f32 8.2, 9.0 with the next), then for bf16, which has twice the exponentials in a load, 64 threads of eight (40 x
    // 151,936: 5.4 us, 5.8 with the one before).
    if (T * nvec < (nvec < 1024 || kBf16 ? 3 : 9) * sms * 1024) {
        cut(512, 64);
        return launch_bwd<kBf16, 128, 1, 4>(a, s);
    }
    if (kBf16 && T * nvec < 9 * sms * 1024) {
        a.chunk_vecs = 512;
        a.chunks = (nvec + 511) / 512;
        return launch_bwd<kBf16, 64, 1, 8>(a, s);
    }
    // Much: bf16 in 1024 vectors by 128 threads of eight loads, where that leaves no half-empty last chunk (8,192 x 151,936
    // 739 us, 6.7 TB/s read and written; 256 threads of four loads 830, 512 threads 988; 16,000 x 15,200 155, 162 with the next);
    if (kBf16 && nvec > 512 && (nvec >= 8192 || nvec % 1024 == 0 || nvec % 1024 >= 600)) {
        a.chunk_vecs = 1024;
        a.chunks = (nvec + 1023) / 1024;
        return launch_bwd<kBf16, 128, 1, 8>(a, s);
    }
    // otherwise equal chunks of up to 512 by 64 threads of eight (16,000 x 10,000 bf16 107 us, 118 with the one before; 4,000 x
    // 75,968 f32 366, 377).
    cut(512, 1);
    return launch_bwd<kBf16, 64, 1, 8>(a, s);
}

// Checks that both calls make; 0 or the error.
static int check(const dppo_logprob_params* p, const char* what, const void* logits, const void* other) {
    if (!p) return fail(DPPO_ERR_INVALID_ARG, "%s: NULL params", what);
    if (p->T_max < 0 || p->V < 1) return fail(DPPO_ERR_INVALID_ARG, "%s: T_max=%lld V=%d", what, (long long)p->T_max, p->V);
    if (p->dtype != DPPO_F32 && p->dtype != DPPO_BF16) return fail(DPPO_ERR_UNSUPPORTED, "%s: dtype %d", what, p->dtype);
    if (p->row_stride < p->V) return fail(DPPO_ERR_BAD_SHAPE, "%s: row_stride %lld < V %d", what, (long long)p->row_stride, p->V);
    if (!(p->temperature >= 1e-6) || !(p->temperature <= 1e6)) return fail(DPPO_ERR_INVALID_ARG, "%s: temperature must be in [1e-6, 1e6]", what);
    if (p->V > (1 << 30)) return fail(DPPO_ERR_BAD_SHAPE, "%s: V=%d, the limit is 2^30", what, p->V);
    if (p->T_max >= ((int64_t)1 << 31)) return fail(DPPO_ERR_BAD_SHAPE, "%s: T_max must be below 2^31", what);
    const size_t esize = p->dtype == DPPO_BF16 ? 2 : 4;
    if (p->T_max > 0 && !logits) return fail(DPPO_ERR_INVALID_ARG, "%s: NULL logits", what);
    if (((uintptr_t)logits & 15) || ((uintptr_t)other & 15) || ((size_t)p->row_stride * esize) % 16 != 0)
        return fail(DPPO_ERR_MISALIGNED, "%s: logits / dlogits / stats base and row stride must be multiples of 16 bytes", what);
    return DPPO_OK;
}

}  // namespace logprob
}  // namespace dppo

extern "C" int dppo_token_logprobs(const dppo_logprob_params* p, const void* logits, const int32_t* target,
                                   const int32_t* n_tokens_dev, float* logp_out, float* entropy_out, float* lse_out,
                                   int32_t* top_ids, float* top_logp, float* stats, int32_t* status, void* stream) {
    dppo::NvtxRange nvtx_range("dppo_token_logprobs");
    using namespace dppo;
    const int rc = logprob::check(p, "token_logprobs", logits, stats);
    if (rc != DPPO_OK) return rc;
    if (p->top_k < 0 || p->top_k > logprob::kMaxTop) return fail(DPPO_ERR_INVALID_ARG, "token_logprobs: top_k=%d (0..%d)", p->top_k, logprob::kMaxTop);
    if (p->variant < 0) return fail(DPPO_ERR_INVALID_ARG, "token_logprobs: variant %d", p->variant);
    if (p->T_max == 0) return DPPO_OK;
    if ((p->top_k > 0) != (top_ids != nullptr) || (p->top_k > 0) != (top_logp != nullptr))
        return fail(DPPO_ERR_INVALID_ARG, "token_logprobs: top_ids and top_logp go with top_k > 0");
    if (logp_out && !target) return fail(DPPO_ERR_INVALID_ARG, "token_logprobs: logp_out without target");
    logprob::Args a = {};
    a.logits = (const char*)logits; a.target = target; a.n_tokens_dev = n_tokens_dev;
    a.logp = logp_out; a.entropy = entropy_out; a.lse = lse_out; a.top_ids = top_ids; a.top_logp = top_logp;
    a.stats = (float4*)stats; a.status = status;
    a.T_max = p->T_max; a.row_bytes = (long long)p->row_stride * (p->dtype == DPPO_BF16 ? 2 : 4);
    a.V = p->V; a.k = p->top_k;
    a.c = (float)(1.4426950408889634 / p->temperature); a.inv_tau = (float)(1.0 / p->temperature);
    return p->dtype == DPPO_BF16 ? logprob::run_fwd<true>(a, p->variant, (cudaStream_t)stream)
                                 : logprob::run_fwd<false>(a, p->variant, (cudaStream_t)stream);
}

extern "C" int dppo_token_logprobs_backward(const dppo_logprob_params* p, const void* logits, const int32_t* target,
                                            const int32_t* n_tokens_dev, const float* stats, const float* dlogp,
                                            const float* dentropy, void* dlogits, int32_t* status, void* stream) {
    dppo::NvtxRange nvtx_range("dppo_token_logprobs_backward");
    using namespace dppo;
    int rc = logprob::check(p, "token_logprobs_backward", logits, stats);
    if (rc != DPPO_OK) return rc;
    if (p->T_max == 0) return DPPO_OK;
    if (!stats || !dlogits) return fail(DPPO_ERR_INVALID_ARG, "token_logprobs_backward: NULL stats or dlogits");
    if ((uintptr_t)dlogits & 15) return fail(DPPO_ERR_MISALIGNED, "token_logprobs_backward: dlogits base must be a multiple of 16 bytes");
    if (dlogp && !target) return fail(DPPO_ERR_INVALID_ARG, "token_logprobs_backward: dlogp without target");
    logprob::BwdArgs a = {};
    a.logits = (const char*)logits; a.dlogits = (char*)dlogits; a.target = target; a.n_tokens_dev = n_tokens_dev;
    a.stats = (const float4*)stats; a.dlogp = dlogp; a.dentropy = dentropy; a.status = status;
    a.T_max = p->T_max; a.row_bytes = (long long)p->row_stride * (p->dtype == DPPO_BF16 ? 2 : 4);
    a.V = p->V;
    a.c = (float)(1.4426950408889634 / p->temperature); a.inv_tau = (float)(1.0 / p->temperature);
    return p->dtype == DPPO_BF16 ? logprob::run_bwd<true>(a, (cudaStream_t)stream) : logprob::run_bwd<false>(a, (cudaStream_t)stream);
}
