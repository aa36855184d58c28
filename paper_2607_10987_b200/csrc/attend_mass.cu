// Attention mass of cached tokens: mass_t = prev_t + sum over query rows r of exp(score_rt - lse_r).
//
// One pass over the keys; with the rows' log-sums given, every token is independent of the others.  A CTA takes a
// chunk of tokens of one sequence and all kv heads, so the sum over heads stays inside it and is taken in a fixed
// order (head by head, row block by row block): no atomics, the same bits every time.  Bound: the bytes of K.  A
// warp holds the keys of 32 tokens of one head in registers, in the layout of the products' first operand, straight
// from global memory (lane (g, t): 8 consecutive dimensions of tokens g, g + 8, g + 16, g + 24), and runs the rows
// past them eight at a time.
#include "attend_device.cuh"

namespace aafkv {

constexpr int MASS_WARPS = 8, MASS_TOKENS = 32;  // tokens of a warp's task

template <typename T, int DP>
__global__ void __launch_bounds__(MASS_WARPS * 32, DP <= 128 ? 2 : 1)
    attn_mass_kernel(const __grid_constant__ MassParams p, const __grid_constant__ SmallSeqs small) {
    extern __shared__ float part[];  // [head][chunk]
    const AttnParams &a = p.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t4 = lane & 3;
    const AttnSeq *seqs = a.seqs ? a.seqs : small.e;
    const int unit = blockIdx.x, si = find_seq(seqs, a.n, unit);
    const AttnSeq sq = seqs[si];
    const int c0 = (unit - sq.unit0) * p.chunk, cn = min(p.chunk, sq.len - c0);
    const int R = sq.nq * a.G, Hq = a.H * a.G;
    const int *table = a.tables + (long long)sq.ctx * a.max_blk;
    const int subs = (cn + MASS_TOKENS - 1) / MASS_TOKENS;

    for (int task = warp; task < subs * a.H; task += MASS_WARPS) {
        const int sub = task / a.H, head = task - sub * a.H, tb = c0 + sub * MASS_TOKENS;
        uint4 kf[4][DP / 32];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = tb + g + 8 * i;
            const char *src = a.kbase;
            if (t < c0 + cn) {
                const int b = block_of(t, a.BS, a.bs_shift);
                src += (long long)__ldg(table + b) * 2 * a.run + (long long)(t - b * a.BS) * a.row + (long long)head * a.D * 2;
            }
#pragma unroll
            for (int kk = 0; kk < DP / 32; ++kk) {
                const int d = kk * 32 + t4 * 8;
                kf[i][kk] = t < c0 + cn && d < a.D ? __ldg(reinterpret_cast<const uint4 *>(src + d * 2)) : make_uint4(0, 0, 0, 0);
            }
        }
        float w[4] = {0, 0, 0, 0};  // tokens g, g + 8, g + 16, g + 24, rows of this lane's columns
        for (int rb = 0; rb < R; rb += 8) {
            float s[2][4] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
            const int rq = min(rb + g, R - 1);
            const T *q = static_cast<const T *>(a.q) + (long long)(sq.row0 + rq / a.G) * a.q_stride +
                         (long long)(head * a.G + rq % a.G) * a.D;
#pragma unroll
            for (int kk = 0; kk < DP / 32; ++kk) {
                const int d = kk * 32 + t4 * 8;
                const uint4 qf = d < a.D ? __ldg(reinterpret_cast<const uint4 *>(q + d)) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint4 x = kf[2 * i][kk], y = kf[2 * i + 1][kk];
                    Elt<T>::mma(s[i], x.x, y.x, x.y, y.y, qf.x, qf.y);
                    Elt<T>::mma(s[i], x.z, y.z, x.w, y.w, qf.z, qf.w);
                }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int r = rb + 2 * t4 + c;
                if (r >= R) continue;
                const RowSpan sp = row_span(a, sq, r / a.G);
                const int hq = head * a.G + r % a.G;
                const float slope = a.slopes ? a.slopes[hq] : 0.0f;
                // the scores are measured from the nearest visible key, so is the log-sum
                const float lse = (p.lse_in[(long long)(sq.row0 + r / a.G) * Hq + hq] + slope * (float)sp.near) * LOG2E;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = tb + g + 8 * i;
                    const float x = score2(a, s[i >> 1][2 * (i & 1) + c], slope, sp, t);
                    if (t >= sp.lo && t < sp.hi && lse != -CUDART_INF_F) w[i] += ex2(x - lse);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] += __shfl_xor_sync(0xffffffffu, w[i], 1);
            w[i] += __shfl_xor_sync(0xffffffffu, w[i], 2);
        }
        const int t = sub * MASS_TOKENS + g + 8 * t4;  // lane (g, t4) writes token g + 8 t4 of the task
        const float mine = t4 == 0 ? w[0] : (t4 == 1 ? w[1] : (t4 == 2 ? w[2] : w[3]));
        if (t < cn) part[head * p.chunk + t] = mine;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < cn; t += MASS_WARPS * 32) {
        float sum = 0.0f;
        for (int h = 0; h < a.H; ++h) sum += part[h * p.chunk + t];
        const long long at = si * p.mass_stride + c0 + t;
        p.mass[at] = (p.prev ? p.prev[at] : 0.0f) + sum;
    }
}

template <typename T, int DP> static cudaError_t mass_go(const MassParams &p, const SmallSeqs &small, cudaStream_t st) {
    const size_t smem = sizeof(float) * (size_t)p.a.H * p.chunk;
    const cudaError_t e = cudaFuncSetAttribute(attn_mass_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    attn_mass_kernel<T, DP><<<(unsigned)p.a.total_units, MASS_WARPS * 32, smem, st>>>(p, small);
    return cudaGetLastError();
}
template <typename T> static cudaError_t mass_pick(const MassParams &p, const SmallSeqs &small, cudaStream_t st) {
    if (p.a.D <= 64) return mass_go<T, 64>(p, small, st);
    if (p.a.D <= 128) return mass_go<T, 128>(p, small, st);
    return mass_go<T, 256>(p, small, st);
}
cudaError_t launch_attn_mass(const MassParams &p, const SmallSeqs &small, int f16, cudaStream_t st) {
    return f16 ? mass_pick<__half>(p, small, st) : mass_pick<__nv_bfloat16>(p, small, st);
}

}  // namespace aafkv
