// Device helpers of the sparse attention kernels.
#pragma once
#include "attend_device.cuh"
#include "sparse_internal.h"

namespace aafkv {

// the smallest exponent from SUMMARY_LEAST_EXP with top <= 127 * 2^e, top not negative: 127 = 1.984375 * 2^6
__device__ __forceinline__ int code_exponent(float top) {
    const uint32_t b = __float_as_uint(top);
    return max(SUMMARY_LEAST_EXP, (int)(b >> 23) - 133 + ((b & 0x7fffffu) > 0x7e0000u ? 1 : 0));
}
// 2^e for -126 <= e <= 127
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// s if v = 2^s, else -1
__device__ __forceinline__ int log2_exact(int v) { return v & (v - 1) ? -1 : 31 - __clz(v); }

// Floats as unsigned numbers of the same order (no NaN).
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// Smallest distance of a row's position to a listed key that it sees: what its bias is measured from (see row_span).  A whole
// warp calls this.
__device__ __forceinline__ int listed_near(const AttnParams &p, const AttnSeq &s, const int *list, const RowSpan &r) {
    const int lane = threadIdx.x & 31, blocks = (s.len + p.BS - 1) / p.BS;
    int near = 0x7fffffff;
    for (int i = lane; i < p.keep; i += 32) {
        const int b = __ldg(list + i);
        if (b < 0 || b >= blocks) continue;
        const int a = max(r.lo, b * p.BS), e = (int)min((long long)r.hi, ((long long)b + 1) * p.BS);
        if (a < e) near = min(near, r.pos < a ? a - r.pos : (r.pos >= e ? r.pos - (e - 1) : 0));
    }
    near = (int)__reduce_min_sync(0xffffffffu, (unsigned)near);
    return near == 0x7fffffff ? 0 : near;
}

}  // namespace aafkv
