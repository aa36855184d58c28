// The blocks of a context with the largest bound on a query's scores, for every query token and kv head.
//
//   q_d in steps of 2^f: c_d = rint(F(q_d) / 2^f), |c_d| <= 127;   dot_b = sum_d max(c_d hi_bd, c_d lo_bd)
//   score_b = max over the group's heads of dot_b * 2^(e_b + f)
//
// max(c hi, c lo) = max(c, 0) hi + min(c, 0) lo: a product of [c+, c-] with the block's [hi, lo], in whole numbers, exact in any
// order, and so is the scaling by a power of two; equal scores go to the lower block.
#include "sparse_device.cuh"

namespace aafkv {

constexpr int SELECT_THREADS = 256;

template <typename T>
__global__ void __launch_bounds__(SELECT_THREADS)
    select_blocks_kernel(const __grid_constant__ SelectParams p, const __grid_constant__ SmallSeqs small) {
    extern __shared__ __align__(16) unsigned char smem_s[];
    uint32_t *keys = reinterpret_cast<uint32_t *>(smem_s);                               // [widest]
    int *codes = reinterpret_cast<int *>(smem_s + ((size_t)p.widest * 4 + 15) / 16 * 16);  // [G][2 D / 4]
    __shared__ int count_s[SELECT_THREADS / 32 + 1], exps[128];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int unit = blockIdx.x / p.H, head = blockIdx.x - unit * p.H;
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq s = seqs[find_seq(seqs, p.n, unit)];
    const int j = unit - s.unit0;
    const long long row = s.row0 + j;
    const int last = (s.len - s.nq + j) / p.BS, total = last + 1, words = p.D / 2;
    int *out = p.blocks + (row * p.H + head) * p.keep;
    float *out_s = p.scores ? p.scores + (row * p.H + head) * p.keep : nullptr;
    for (int b = threadIdx.x; b < total; b += SELECT_THREADS) keys[b] = 0;
    for (int g0 = 0; g0 < p.G; g0 += 16) {
        const int rows = min(16, p.G - g0);
        __syncthreads();
        for (int r = warp; r < rows; r += SELECT_THREADS / 32) {
            const T *q = static_cast<const T *>(p.q) + row * p.q_stride + (long long)(head * p.G + g0 + r) * p.D;
            float top = 0.0f;
            for (int d = lane; d < p.D; d += 32) {
                const float x = Elt<T>::from(reinterpret_cast<const uint16_t *>(q)[d]);
                if (x == x) top = fmaxf(top, fminf(fabsf(x), 127.0f * 0x1p113f));
            }
            const int f = code_exponent(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top))));
            signed char *c = reinterpret_cast<signed char *>(codes + r * words);
            for (int d = lane; d < p.D; d += 32) {
                const float x = Elt<T>::from(reinterpret_cast<const uint16_t *>(q)[d]);
                const int v = x != x ? 0 : __float2int_rn(fminf(fmaxf(x, -127.0f * 0x1p113f), 127.0f * 0x1p113f) * power_of_two(-f));
                c[d] = (signed char)max(v, 0);
                c[p.D + d] = (signed char)min(v, 0);
            }
            if (lane == 0) exps[r] = f;
        }
        __syncthreads();
        for (int b = threadIdx.x; b < total; b += SELECT_THREADS) {
            const signed char *rec = p.summary + (long long)__ldg(p.tables + (long long)s.ctx * p.max_blk + b) * p.record;
            const int e = rec[(long long)p.H * 2 * p.D + head];
            const int *code = reinterpret_cast<const int *>(rec + (long long)head * 2 * p.D);
            uint32_t best = keys[b];
            for (int r = 0; r < rows; ++r) {
                int dot = 0;
                for (int w = 0; w < words; ++w) dot = __dp4a(code[w], codes[r * words + w], dot);
                const int x = e + exps[r];  // -120 ... 226
                best = max(best, ordered((float)dot * power_of_two(min(x, 100)) * power_of_two(max(x, 100) - 100)));
            }
            keys[b] = best;
        }
    }
    __syncthreads();
    // the middle [sink, total - recent): the smallest key of those taken, bit by bit
    const int m0 = min(p.sink, total), m1 = max(m0, total - p.recent), want = p.keep - p.sink - p.recent;
    auto count = [&](uint32_t from) {
        int c = 0;
        for (int b = m0 + threadIdx.x; b < m1; b += SELECT_THREADS) c += keys[b] >= from;
        c = __reduce_add_sync(0xffffffffu, c);
        __syncthreads();
        if (lane == 0) count_s[warp] = c;
        __syncthreads();
        int t = 0;
        for (int w = 0; w < SELECT_THREADS / 32; ++w) t += count_s[w];
        return t;
    };
    uint32_t least = 0;
    int ties = 0x7fffffff;
    if (m1 - m0 > want) {
        if (want <= 0) {
            least = 0xffffffffu;
            ties = 0;
        } else {
            for (int bit = 31; bit >= 0; --bit)
                if (count(least | 1u << bit) >= want) least |= 1u << bit;
            ties = want - (least == 0xffffffffu ? 0 : count(least + 1));
        }
    }
    __syncthreads();
    if (warp == 0) {
        int at = 0, tied = 0;
        for (int b0 = 0; b0 < total; b0 += 32) {
            const int b = b0 + lane;
            const bool in = b < total, middle = in && b >= m0 && b < m1;
            const uint32_t k = in ? keys[b] : 0;
            const bool tie = middle && k == least;
            const unsigned tm = __ballot_sync(0xffffffffu, tie);
            const int before = tied + __popc(tm & ((1u << lane) - 1));
            const bool take = in && (!middle || k > least || (tie && before < ties));
            const unsigned mask = __ballot_sync(0xffffffffu, take);
            const int to = at + __popc(mask & ((1u << lane) - 1));
            if (take) {
                out[to] = b;
                if (out_s) out_s[to] = from_ordered(k);
            }
            at += __popc(mask);
            tied += __popc(tm);
        }
        for (int i = at + lane; i < p.keep; i += 32) {
            out[i] = -1;
            if (out_s) out_s[i] = -CUDART_INF_F;
        }
    }
}

template <typename T> static cudaError_t select_go(const SelectParams &p, const SmallSeqs &small, long long tokens, cudaStream_t st) {
    static SmemSeen seen{0};
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(select_blocks_kernel<T>), 220 * 1024, &seen);
    if (e != cudaSuccess) return e;
    const size_t smem = ((size_t)p.widest * 4 + 15) / 16 * 16 + (size_t)std::min(p.G, 16) * 2 * p.D;
    select_blocks_kernel<T><<<(unsigned)(tokens * p.H), SELECT_THREADS, smem, st>>>(p, small);
    return cudaGetLastError();
}
cudaError_t launch_select_blocks(const SelectParams &p, const SmallSeqs &small, int f16, long long tokens, cudaStream_t st) {
    return f16 ? select_go<__half>(p, small, tokens, st) : select_go<__nv_bfloat16>(p, small, tokens, st);
}

}  // namespace aafkv
