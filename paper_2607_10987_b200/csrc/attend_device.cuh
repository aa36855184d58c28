// Device helpers of the attention kernels: element types, warp matrix products, score function, asynchronous copies.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "attend_internal.h"

namespace aafkv {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// RAISE: weights are computed as 2^(x - m + RAISE), m the row's maximum, so that the largest is near the top of the type's range.
// f16 ends at 2^-24: with a largest weight of 1, weights below 2^-14 would lose bits and those below 2^-25 vanish from the
// products while the sum, in 32 bits, still counts them (131072 keys at 2^-24.6 of one: an error of five half steps).
// What is kept for the join and the log-sum is the base of the exponents, m - RAISE.
template <typename T> struct Elt;
template <> struct Elt<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ float lo(uint32_t v) { return __uint_as_float(v << 16); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
    static __device__ __forceinline__ float from(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
    static __device__ __forceinline__ uint16_t to(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
    static constexpr uint32_t EXP = 0x7f807f80u, ONE = 0x3f80u;
    static constexpr float RAISE = 0.0f;
    // magnitudes of at most the type's largest finite value, signs kept
    static __device__ __forceinline__ uint32_t bounded(uint32_t v) {
        uint32_t r;
        asm("min.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0x7f7f7f7fu));
        return r;
    }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};
template <> struct Elt<__half> {
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ float lo(uint32_t v) { return __half2float(__ushort_as_half((uint16_t)v)); }
    static __device__ __forceinline__ float hi(uint32_t v) { return __half2float(__ushort_as_half((uint16_t)(v >> 16))); }
    static __device__ __forceinline__ float from(uint16_t v) { return __half2float(__ushort_as_half(v)); }
    static __device__ __forceinline__ uint16_t to(float v) { return __half_as_ushort(__float2half_rn(v)); }
    static constexpr uint32_t EXP = 0x7c007c00u, ONE = 0x3c00u;
    static constexpr float RAISE = 15.0f;
    // magnitudes of at most the type's largest finite value, signs kept
    static __device__ __forceinline__ uint32_t bounded(uint32_t v) {
        uint32_t r;
        asm("min.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0x7bff7bffu));
        return r;
    }
    static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                               uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
                     "{%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};

// 8 x 8 transpose of 16-bit elements across the warp (accumulator layout -> operand layout)
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t s) {
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(s));
    return r;
}

// Tiles whose keys some rows see and others do not: a value that is not finite must reach only the rows that see it,
// but 0 * inf is NaN.  Such elements are taken as zero in the product itself (finite_only); what they add is counted
// with indicator products (1 where V is +inf or NaN, 1 where it is -inf or NaN, times 1 where the row sees the key).
template <typename T> __device__ __forceinline__ uint32_t finite_only(uint32_t v) {
    constexpr uint32_t e = Elt<T>::EXP;
    const uint32_t x = v & e;
    if ((x & 0xffffu) == (e & 0xffffu)) v &= 0xffff0000u;
    if ((x & 0xffff0000u) == (e & 0xffff0000u)) v &= 0xffffu;
    return v;
}
template <typename T> __device__ __forceinline__ uint32_t indicate(uint32_t v, bool up) {
    uint32_t r = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float x = Elt<T>::from((uint16_t)(v >> (16 * h)));
        if (up ? !(x < CUDART_INF_F) : !(x > -CUDART_INF_F)) r |= Elt<T>::ONE << (16 * h);
    }
    return r;
}
__device__ __forceinline__ float nonfinite_of(float up, float down) {
    return (up > 0.0f ? CUDART_INF_F : 0.0f) - (down > 0.0f ? CUDART_INF_F : 0.0f);
}
// what the elements of the first (second) operand that are not finite add to a 16 x 8 product; by value, so that the
// accumulators of the caller stay in registers
template <typename T>
__device__ __noinline__ float4 nonfinite_a(uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t vis0, uint32_t vis1) {
    float u[4] = {0, 0, 0, 0}, d[4] = {0, 0, 0, 0};
    Elt<T>::mma(u, indicate<T>(a0, true), indicate<T>(a1, true), indicate<T>(a2, true), indicate<T>(a3, true), vis0, vis1);
    Elt<T>::mma(d, indicate<T>(a0, false), indicate<T>(a1, false), indicate<T>(a2, false), indicate<T>(a3, false), vis0, vis1);
    return make_float4(nonfinite_of(u[0], d[0]), nonfinite_of(u[1], d[1]), nonfinite_of(u[2], d[2]), nonfinite_of(u[3], d[3]));
}
template <typename T>
__device__ __noinline__ float4 nonfinite_b(uint32_t vis0, uint32_t vis1, uint32_t vis2, uint32_t vis3, uint32_t b0, uint32_t b1) {
    float u[4] = {0, 0, 0, 0}, d[4] = {0, 0, 0, 0};
    Elt<T>::mma(u, vis0, vis1, vis2, vis3, indicate<T>(b0, true), indicate<T>(b1, true));
    Elt<T>::mma(d, vis0, vis1, vis2, vis3, indicate<T>(b0, false), indicate<T>(b1, false));
    return make_float4(nonfinite_of(u[0], d[0]), nonfinite_of(u[1], d[1]), nonfinite_of(u[2], d[2]), nonfinite_of(u[3], d[3]));
}
__device__ __forceinline__ void add4(float (&c)[4], float4 v) {
    c[0] += v.x;
    c[1] += v.y;
    c[2] += v.z;
    c[3] += v.w;
}

// 16-byte asynchronous copy global -> shared; bytes = 0 writes zeros and reads nothing
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// tanh(x) in single precision.  Large |x|: (1 - u) / (1 + u) with u = exp(-2|x|), relative error of a few ulp of u.
// Small |x|: the odd Taylor series to x^9, whose first left-out term is below 1e-8 of x for |x| < 0.25; there the
// quotient would lose the digits that 1 - u cancels.
__device__ __forceinline__ float tanh_f32(float x) {
    const float a = fabsf(x), z = x * x;
    const float u = ex2(-2.0f * LOG2E * a);
    const float big = (1.0f - u) * rcp(1.0f + u);
    const float small = a + a * z * (-1.0f / 3 + z * (2.0f / 15 + z * (-17.0f / 315 + z * (62.0f / 2835))));
    return copysignf(a < 0.25f ? small : big, x);
}

// Keys [lo, hi) that a query row sees and the distance that its bias is measured from.
// The bias of key t is -slope * |pos - t|.  Softmax does not change when a row's scores all move by the same
// amount, so the kernels use -slope * (|pos - t| - near) with near = the smallest distance within [lo, hi): the
// products that matter are then small and exact in 32 bits however far the span lies from the position, and the
// row's log-sum gets -slope * near back.
struct RowSpan {
    int lo, hi, pos, near;
};
__device__ __forceinline__ RowSpan row_span(const AttnParams &p, const AttnSeq &s, int j) {
    RowSpan r;
    r.pos = s.len - s.nq + j;
    r.lo = 0;
    r.hi = r.pos + 1;
    if (p.spans) {
        r.lo = max(0, p.spans[2 * (long long)(s.row0 + j)]);
        r.hi = min(s.len, p.spans[2 * (long long)(s.row0 + j) + 1]);
    }
    if (p.window) r.lo = max(r.lo, r.pos + 1 - p.window);
    if (r.hi < r.lo) r.hi = r.lo;
    r.near = r.pos < r.lo ? r.lo - r.pos : (r.pos >= r.hi ? r.pos - (r.hi - 1) : 0);
    return r;
}

// raw product -> score in the log2 domain
__device__ __forceinline__ float score2(const AttnParams &p, float x, float slope, const RowSpan &r, int t) {
    x *= p.scale;
    if (p.softcap != 0.0f) x = p.softcap * tanh_f32(x * p.inv_cap);
    if (p.slopes) x -= slope * (float)(abs(r.pos - t) - r.near);
    return x * LOG2E;
}

// an output from its weighted sum; a row without weights is zero, whatever it multiplied by zero
__device__ __forceinline__ float scaled(float o, float inv) { return inv == 0.0f ? 0.0f : o * inv; }

// sequence that a unit belongs to: the last one whose first unit is not behind it
__device__ __forceinline__ int find_seq(const AttnSeq *s, int n, int unit) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s[mid].unit0 <= unit) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// query token of a row
__device__ __forceinline__ int token_of(const AttnParams &p, int row) { return p.g_shift >= 0 ? row >> p.g_shift : row / p.G; }
__device__ __forceinline__ int block_of(int t, int BS, int shift) { return shift >= 0 ? t >> shift : t / BS; }

}  // namespace aafkv
