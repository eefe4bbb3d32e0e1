// Sweeps over rows of logits: loads, maxima, and an online sum of exponentials (shared by the distillation and draft
// verification kernels; not part of the ABI).
#pragma once
#include "common.cuh"
#include "grpo_loss.cuh"

namespace dppo {
namespace sweep {
using namespace packed;

constexpr float kLowest = -3.402823466e38f;
constexpr int kRound = 4;                 // vectors that a thread has under way

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint4 load_vec(const void* p) {
    uint4 q;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p));
    return q;
}
// A vector that may be written by the same kernel (in place): not the read-only path.
__device__ __forceinline__ uint4 load_vec_rw(const void* p) {
    uint4 q;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "l"(p) : "memory");
    return q;
}
template <bool kBf16> __device__ __forceinline__ uint4 masked_vec() {
    constexpr uint32_t none = kBf16 ? 0xff80ff80u : 0xff800000u;  // -inf
    return make_uint4(none, none, none, none);
}

// What has been seen of a row: its largest entry (kLowest, with S = 0, if there is none but -inf), S = sum 2^((z - m) c), and
// whether a NaN or +inf was among them.
struct Part {
    float m, S;
    int bad;
};
__device__ __forceinline__ Part part_none() { return {kLowest, 0.0f, 0}; }
__device__ __forceinline__ void part_to(Part& p, float M, float c) {
    if (p.m != M) p.S = p.S > 0.0f ? p.S * ex2((p.m - M) * c) : 0.0f;
    p.m = M;
}
// The parts of a warp's lanes as one, in every lane.
__device__ __forceinline__ Part part_warp(Part p, float c) {
    part_to(p, warp_max_f32(p.m), c);
    p.S = warp_sum(p.S);
    p.bad = __any_sync(0xffffffffu, p.bad);
    return p;
}

// Running sum of a thread, in packed f32 pairs.  On ordinary rows ("quick") an exponent is one fma, z c - r with r = fl(m c);
// the sum then carries the shift m c - r (exact in f32), which comes out when m grows and at the end.  Rows whose maximum is
// far from zero against the temperature (|m c| > 2^20: masks of the type's lowest value with nothing above, logits of 10^6)
// take the differences z - m first, so they keep them.  Entries at -inf have exponent -inf, which ex2 turns into 0.
struct Sum {
    f32x2 S;
    float m, nr, res;
    uint32_t m2;                          // bf16 pair of m
    int quick, bad;
};
__device__ __forceinline__ void sum_frame(Sum& a, float m, float c) {
    const float r = m * c;
    a.quick = fabsf(r) <= 1048576.0f && fabsf(m) <= 1e37f;
    a.m = m; a.nr = -r;
    a.res = a.quick ? fmaf(m, c, -r) : 0.0f;
    const __nv_bfloat162 p = __float2bfloat162_rn(m);              // exact where the entries are bf16
    a.m2 = *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ void sum_init(Sum& a, float m, float c) {
    a.S = pair_of(0.0f, 0.0f); a.bad = 0;
    sum_frame(a, m, c);
}
__device__ __forceinline__ Part sum_part(const Sum& a) {
    float s0, s1;
    unpair(a.S, s0, s1);
    return {a.m, (s0 + s1) * ex2(-a.res), a.bad};
}
__device__ __forceinline__ void sum_grow(Sum& a, float vmax, float c) {
    const float x = (a.m - vmax) * c, res = a.res;
    sum_frame(a, vmax, c);
    const float f = ex2(x + (a.res - res));                        // x may be -inf: then there was nothing
    a.S = mul2(a.S, pair_of(f, f));
}
// The lanes of a warp together: they keep one maximum, and a larger one turns up a few times per row.
__device__ __forceinline__ void sum_grow_warp(Sum& a, float vmax, float c) {
    if (!(vmax < INFINITY)) { a.bad = 1; vmax = -INFINITY; }       // NaN or +inf: the row's results are NaN
    const float m = warp_max_f32(vmax);
    if (m > a.m) sum_grow(a, m, c);
}
__device__ __forceinline__ void sum_add(Sum& a, f32x2 y) {
    float y0, y1;
    unpair(y, y0, y1);
    a.S = add2(a.S, pair_of(ex2(y0), ex2(y1)));
}
template <bool kBf16> __device__ __forceinline__ void sum_vec(Sum& a, const uint4& q, float c) {
    const f32x2 c2 = pair_of(c, c);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    if (a.quick) {
        const f32x2 nr2 = pair_of(a.nr, a.nr);
        if constexpr (kBf16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum_add(a, fma2(pair_of(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u)), c2, nr2));
        } else {
#pragma unroll
            for (int i = 0; i < 4; i += 2) sum_add(a, fma2(pair_of(__uint_as_float(w[i]), __uint_as_float(w[i + 1])), c2, nr2));
        }
    } else {
        const f32x2 nm2 = pair_of(-a.m, -a.m);
        float f[Elems<kBf16>::kPerVec];
        Elems<kBf16>::unpack(q, f);
#pragma unroll
        for (int i = 0; i < Elems<kBf16>::kPerVec; i += 2) sum_add(a, mul2(add2(pair_of(f[i], f[i + 1]), nm2), c2));
    }
}
// Largest entry of kN vectors (NaN if there is one).
template <bool kBf16, int kN> __device__ __forceinline__ float vecs_max(const uint4 (&q)[kN], __nv_bfloat162& x) {
    if constexpr (kBf16) {
        x = *reinterpret_cast<const __nv_bfloat162*>(&q[0].x);
#pragma unroll
        for (int u = 0; u < kN; ++u) {
            const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
#pragma unroll
            for (int i = u == 0 ? 1 : 0; i < 4; ++i) x = __hmax2_nan(x, *reinterpret_cast<const __nv_bfloat162*>(&w[i]));
        }
        return __bfloat162float(__hmax_nan(__low2bfloat16(x), __high2bfloat16(x)));
    } else {
        float m = __uint_as_float(q[0].x);
#pragma unroll
        for (int u = 0; u < kN; ++u)
            m = max_nan(max_nan(m, max_nan(__uint_as_float(q[u].x), __uint_as_float(q[u].y))), max_nan(__uint_as_float(q[u].z), __uint_as_float(q[u].w)));
        return m;
    }
}
// kN vectors, by a whole warp.
template <bool kBf16, int kN> __device__ __forceinline__ void sum_vecs(Sum& a, const uint4 (&q)[kN], float c) {
    __nv_bfloat162 x;
    const float vmax = vecs_max<kBf16, kN>(q, x);
    if constexpr (kBf16) {
        if (__any_sync(0xffffffffu, !__hble2(x, *reinterpret_cast<const __nv_bfloat162*>(&a.m2)))) sum_grow_warp(a, vmax, c);
    } else {
        if (__any_sync(0xffffffffu, !(vmax <= a.m))) sum_grow_warp(a, vmax, c);
    }
    const int quick = a.quick;
    if (quick) {                                                   // one test per kN vectors: what follows is a straight line
#pragma unroll
        for (int u = 0; u < kN; ++u) { a.quick = 1; sum_vec<kBf16>(a, q[u], c); }
    } else {
#pragma unroll 1
        for (int u = 0; u < kN; ++u) {
            uint4 v = q[0];                                        // selects: q stays in registers
#pragma unroll
            for (int j = 1; j < kN; ++j) v = u == j ? q[j] : v;
            a.quick = 0;
            sum_vec<kBf16>(a, v, c);
        }
    }
}
// One entry of this lane's alone (-inf: nothing).
__device__ __forceinline__ void part_one(Part& p, float z, float c) {
    if (!(z < INFINITY)) { p.bad = 1; return; }
    if (z == -INFINITY) return;
    if (z > p.m) part_to(p, z, c);
    p.S += ex2((z - p.m) * c);
}

// ---- a row's scalars in 64 bits, short of the library's full precision -----------------------------------
// e^x for |x| <= 700 to a relative 2^-36: x = n ln 2 + f with |f| <= ln 2 / 2, the Taylor series of e^f to f^9 / 9! (remainder
// f^10 / 10! < 7e-12), in two halves that are under way together, and n added to the exponent.  Below it is 0, above infinity.
__device__ __forceinline__ double exp64(double x) {
    if (!(fabs(x) <= 700.0)) return x != x ? x : x > 0.0 ? (double)INFINITY : 0.0;
    const double n = rint(x * 1.4426950408889634);
    const double f = fma(n, -0.6931471805599453, x), f2 = f * f;
    const double even = fma(fma(fma(fma(1.0 / 40320, f2, 1.0 / 720), f2, 1.0 / 24), f2, 0.5), f2, 1.0);
    const double odd = fma(fma(fma(fma(1.0 / 362880, f2, 1.0 / 5040), f2, 1.0 / 120), f2, 1.0 / 6), f2, 1.0);
    const double r = fma(odd, f, even);
    return __hiloint2double(__double2hiint(r) + ((int)n << 20), __double2loint(r));
}
// ln x of a normal f32's range (or of 0, infinity, NaN) to 1e-11: one step of Newton's method from the f32 logarithm,
// l = l0 + d - d^2 / 2 with d = x e^-l0 - 1.
__device__ __forceinline__ double log64(double x) {
    const float l0 = logf((float)x);
    if (!(fabsf(l0) < 1e3f)) return (double)l0;
    const double d = fma(x, exp64(-(double)l0), -1.0);
    return (double)l0 + fma(-0.5 * d, d, d);
}
// 1 / x to 2^-46 of it, for x in the range of normal f32 values: Newton's step from the f32 quotient.
__device__ __forceinline__ double inv64(double x) {
    const double y = (double)(1.0f / (float)x);
    return y * fma(-x, y, 2.0);
}

}  // namespace sweep
}  // namespace dppo
