// Attention mass of many query rows on the tensor cores (see attend_mass.cu for the sums): a CTA takes 256 tokens, a thread
// one of them.  S^T = K Q^T for 64 rows of a kv head has the tokens as its rows, so a token's weights are the columns of its
// thread's row in tensor memory: the sum over rows and heads never leaves the thread, in a fixed order.  Bound: the bytes of K
// and, from 128 rows on, the exponentials (1024 cycles of an SM for 128 x 128 scores; the product takes 512).  A step is
// 64 rows of a head; keys have two stages, a head each, scores two, queries three: their copies are a chain of a wait, address
// arithmetic and a trip to L2, some 2 us, longer than a step's sums, so they run two steps ahead.  32763 tokens, 128 rows, 8 heads:
// 29 us (2.3 TB/s); 50 with 128 tokens a CTA and one stage of each.  Every wait is bounded (see attend_wide.cu).
#include "tensor_device.cuh"

namespace aafkv {

constexpr int MW_TOKENS = MASS_WIDE_CHUNK, MW_ROWS = 64, MW_Q = 3;
constexpr int MW_THREADS = 448;  // 8 warps sum, 4 copy queries, 1 issues products, 1 copies keys
static_assert(MW_TOKENS == 256, "a thread per token");

template <int D> struct MassWideShape {
    static constexpr int HALVES = D / 64, K_BYTES = HALVES * MW_TOKENS * 128, Q_BYTES = HALVES * MW_ROWS * 128;
    static constexpr int INFO = 2 * K_BYTES + MW_Q * Q_BYTES, LSE = INFO + MW_Q * MW_ROWS * 16,
                         SLOPE = LSE + MW_Q * MW_ROWS * 4, WORDS = SLOPE + MW_Q * MW_ROWS * 4;
    static constexpr int SMEM = WORDS + 192;
    static_assert(SMEM <= 227 * 1024, "shared memory of a CTA");
};

template <typename T, int D>
__global__ void __launch_bounds__(MW_THREADS, 1)
    attn_mass_wide_kernel(const __grid_constant__ MassParams p, const __grid_constant__ SmallSeqs small,
                          const __grid_constant__ CUtensorMap map, int layer) {
    using S = MassWideShape<D>;
    extern __shared__ __align__(1024) char smem[];
    const AttnParams &a = p.a;
    const uint32_t raw = (uint32_t)__cvta_generic_to_shared(smem), sK = raw, sQ = raw + 2 * S::K_BYTES;
    int4 *info = reinterpret_cast<int4 *>(smem + S::INFO);               // by stage of the queries: what the rows see,
    float *row_lse = reinterpret_cast<float *>(smem + S::LSE);           // their log-sums, slopes
    float *row_slope = reinterpret_cast<float *>(smem + S::SLOPE);
    uint32_t &sh_tmem = *reinterpret_cast<uint32_t *>(smem + S::WORDS);
    volatile int &sh_abort = *reinterpret_cast<volatile int *>(smem + S::WORDS + 4);
    volatile unsigned char *sh_all = reinterpret_cast<volatile unsigned char *>(smem + S::WORDS + 8);  // by stage and warp: rows that see all tokens
    const uint32_t k_full = raw + S::WORDS + 16, k_free = k_full + 16, q_full = k_free + 16, q_free = q_full + 24, s_full = q_free + 24,
                   s_free = s_full + 16, drain = s_free + 16;
    if (raw & 1023) {  // never: the swizzle goes by address bits
        if (threadIdx.x == 0) atomicCAS(a.status, 0, AAF_ERR_CORRUPT);
        return;
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const AttnSeq *seqs = a.seqs ? a.seqs : small.e;
    const int unit = blockIdx.x, si = find_seq(seqs, a.n, unit);
    const AttnSeq sq = seqs[si];
    const int tb = (unit - sq.unit0) * MW_TOKENS, R = sq.nq * a.G, Hq = a.H * a.G;
    const int row_blocks = (R + MW_ROWS - 1) / MW_ROWS, steps = row_blocks * a.H;  // step = head * row_blocks + block

    if (warp == 12) {
        if (lane == 0) {
            for (int i = 0; i < 2; ++i) {
                bar_init(k_full + 8 * i, 1);
                bar_init(k_free + 8 * i, 1);
                bar_init(s_full + 8 * i, 1);
                bar_init(s_free + 8 * i, 8);
            }
            for (int i = 0; i < MW_Q; ++i) {
                bar_init(q_full + 8 * i, 128);
                bar_init(q_free + 8 * i, 8);
            }
            bar_init(drain, 1);
            sh_abort = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 256;" ::"r"(
                         (uint32_t)__cvta_generic_to_shared(&sh_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    const uint32_t tmem = sh_tmem;

    if (warp < 8) {
        // ---------------------------------------------------------------- a thread per token: weights and their sum
        const int t = tb + threadIdx.x;
        const uint32_t tS = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * 2 * MW_ROWS;  // [token tile][stage][row]
        const float c2 = a.scale * LOG2E;
        const bool plain = a.softcap == 0.0f && !a.slopes;
        f2 sum[2] = {0, 0};
        float masked = 0.0f;
        for (int s = 0; s < steps; ++s) {
            const int e = s & 1, qs = s % MW_Q;
            if (!warp_wait(s_full + 8 * e, s >> 1 & 1, &sh_abort, a.status)) break;
            tmem_after();
            const float *lse = row_lse + qs * MW_ROWS;
            // every row of the block sees every token of the tile: the copying warps have looked
            const bool quick = plain && *reinterpret_cast<const volatile uint16_t *>(sh_all + 2 * qs) == 0x0101;
#pragma unroll 1
            for (int h = 0; h < MW_ROWS; h += 32) {
                float x[32];
                tmem_ld32(tS + e * MW_ROWS + h, x);
                tmem_wait_ld();
                if (quick) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 z = *reinterpret_cast<const float4 *>(lse + h + i);
                        float y[4];
                        unpair(fma2(pair(x[i], x[i + 1]), pair(c2, c2), pair(-z.x, -z.y)), y[0], y[1]);
                        unpair(fma2(pair(x[i + 2], x[i + 3]), pair(c2, c2), pair(-z.z, -z.w)), y[2], y[3]);
                        sum[0] = add2(sum[0], pair(ex2(y[0]), ex2(y[1])));
                        sum[1] = add2(sum[1], pair(ex2(y[2]), ex2(y[3])));
                    }
                } else if (plain) {  // a mask only: the CTAs at the end of a context, which would else be the last to finish
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int2 ri = *reinterpret_cast<const int2 *>(&info[qs * MW_ROWS + h + i]);
                        const float w = ex2(fmaf(x[i], c2, -lse[h + i]));
                        masked += t >= ri.x && t < ri.y ? w : 0.0f;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int4 ri = info[qs * MW_ROWS + h + i];
                        RowSpan sp;
                        sp.lo = ri.x;
                        sp.hi = ri.y;
                        sp.pos = ri.z;
                        sp.near = ri.w;
                        const float v = score2(a, x[i], a.slopes ? row_slope[qs * MW_ROWS + h + i] : 0.0f, sp, t) - lse[h + i];
                        masked += t >= sp.lo && t < sp.hi ? ex2(v) : 0.0f;
                    }
                }
            }
            // scores, log-sums and spans of this step have been read: others may take their place
            tmem_before();
            __syncwarp();
            if (lane == 0) {
                bar_arrive(s_free + 8 * e);
                bar_arrive(q_free + 8 * qs);
            }
        }
        float u, v;
        unpair(add2(sum[0], sum[1]), u, v);
        if (t < sq.len) {
            const long long o = si * p.mass_stride + t;
            p.mass[o] = (p.prev ? p.prev[o] : 0.0f) + (u + v + masked);
        }
    } else if (warp < 12) {
        // ---------------------------------------------------------------- queries, their log-sums and spans
        constexpr int PIECES = D / 8, AT_ONCE = 128 / PIECES;
        const int tid = threadIdx.x - 256, c = tid % PIECES;
        for (int s = 0; s < steps; ++s) {
            const int e = s % MW_Q, head = s / row_blocks, rb = (s - head * row_blocks) * MW_ROWS;
            if (s >= MW_Q && !warp_wait(q_free + 8 * e, s / MW_Q - 1 & 1, &sh_abort, a.status)) break;
#pragma unroll
            for (int i = 0; i < MW_ROWS / AT_ONCE; ++i) {
                const int r = i * AT_ONCE + tid / PIECES, rc = min(rb + r, R - 1), j = token_of(a, rc);  // behind the last: the last again
                const T *src = static_cast<const T *>(a.q) + (sq.row0 + j) * a.q_stride + (head * a.G + rc - j * a.G) * D + c * 8;
                copy16(sQ + e * S::Q_BYTES + r * 128 + (c >> 3) * (MW_ROWS * 128) + (((c & 7) ^ (r & 7)) << 4),
                       src, 16);
            }
            copy_commit();
            if (tid < MW_ROWS) {
                const int rq = rb + tid, rc = min(rq, R - 1), j = token_of(a, rc), hq = head * a.G + rc - j * a.G;
                const RowSpan sp = row_span(a, sq, j);
                float lse = p.lse_in[(long long)(sq.row0 + j) * Hq + hq];
                if (a.slopes) {  // scores are measured from the nearest visible key, so is the log-sum
                    row_slope[e * MW_ROWS + tid] = a.slopes[hq];
                    lse += a.slopes[hq] * (float)sp.near;
                }
                // a row without a sum adds nothing, nor does one behind the last
                row_lse[e * MW_ROWS + tid] = lse == -CUDART_INF_F || rq >= R ? CUDART_INF_F : lse * LOG2E;
                info[e * MW_ROWS + tid] = make_int4(sp.lo, rq < R ? sp.hi : 0, sp.pos, sp.near);
                const bool all = __all_sync(0xffffffffu, rq >= R || (sp.lo <= tb && sp.hi >= tb + MW_TOKENS));
                if (lane == 0) sh_all[2 * e + warp - 8] = all;
            }
            copy_wait<0>();
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            bar_arrive(q_full + 8 * e);
        }
        copy_wait<0>();
    } else if (warp == 13) {
        // ---------------------------------------------------------------- keys, a head ahead (64 copies of a block take some 3000
        // cycles to issue: the products' warp would not get to them in time)
        const int pages = MW_TOKENS / a.BS, at = tb + lane * a.BS;  // at most 32
        const bool mine = lane < pages && at < sq.len;
        const int slot = mine ? 2 * __ldg(a.tables + (long long)sq.ctx * a.max_blk + block_of(at, a.BS, a.bs_shift)) * a.BS : 0;
        const int count = __popc(__ballot_sync(0xffffffffu, mine));
        bool ok = true;
        int issued = 0;
        for (int head = 0; head < a.H; ++head) {
            const int e = head & 1;
            if (head > 1 && !(ok = warp_wait(k_free + 8 * e, (head >> 1) - 1 & 1, &sh_abort, a.status))) break;
            if (lane == 0) bar_expect(k_full + 8 * e, (uint32_t)(count * a.BS * D * 2));
            __syncwarp();
            if (mine)
#pragma unroll
                for (int h = 0; h < S::HALVES; ++h)
                    page_copy(sK + e * S::K_BYTES + h * (MW_TOKENS * 128) + lane * a.BS * 128, &map, k_full + 8 * e, head * D + h * 64, slot, layer);
            issued = head + 1;
        }
        if (!ok)  // nothing may be in flight when the CTA ends early
            for (int h = max(0, issued - 2); h < issued; ++h)
                for (int i = 0; i < WAIT_LIMIT && !bar_try(k_full + 8 * (h & 1), h >> 1 & 1); ++i) {}
    } else {
        // ---------------------------------------------------------------- products
        constexpr uint32_t F = WideFormat<T>::F;
        constexpr uint32_t QK = 1u << 4 | F << 7 | F << 10 | (MW_ROWS / 8) << 17 | (128 / 16) << 24;
        const uint64_t dK = smem_desc(sK, 16, 1024), dQ = smem_desc(sQ, 16, 1024);
        bool ok = true;
        int head = 0, block = 0;
        for (int s = 0; s < steps; ++s) {
            const int e = s & 1, ke = head & 1, qs = s % MW_Q;
            if (block == 0 && !(ok = warp_wait(k_full + 8 * ke, head >> 1 & 1, &sh_abort, a.status))) break;
            if (!(ok = warp_wait(q_full + 8 * qs, s / MW_Q & 1, &sh_abort, a.status))) break;
            if (s > 1 && !(ok = warp_wait(s_free + 8 * e, (s >> 1) - 1 & 1, &sh_abort, a.status))) break;
            tmem_after();
            if (elected()) {
#pragma unroll
                for (int i = 0; i < 2; ++i)  // the two token tiles
#pragma unroll
                    for (int h = 0; h < S::HALVES; ++h)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            mma_ss(tmem + (2 * i + e) * MW_ROWS, dK + ((ke * S::K_BYTES + h * (MW_TOKENS * 128) + i * (128 * 128)) >> 4) + 2 * k,
                                   dQ + ((qs * S::Q_BYTES + h * (MW_ROWS * 128)) >> 4) + 2 * k, QK, h + k > 0);
                mma_commit(s_full + 8 * e);
                if (block + 1 == row_blocks && head + 2 < a.H) mma_commit(k_free + 8 * ke);
            }
            __syncwarp();
            if (++block == row_blocks) {
                block = 0;
                ++head;
            }
        }
        if (!ok && lane == 0) {
            mma_commit(drain);
            for (int i = 0; i < WAIT_LIMIT && !bar_try(drain, 0); ++i) {}
        }
        __syncwarp();
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    if (warp == 12) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 256;" ::"r"(tmem));
}

template <typename T, int D> static cudaError_t mass_wide_go(const MassParams &p, const SmallSeqs &small, const void *map, int layer, cudaStream_t st) {
    static SmemSeen seen{0};
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(attn_mass_wide_kernel<T, D>), MassWideShape<D>::SMEM, &seen);
    if (e != cudaSuccess) return e;
    attn_mass_wide_kernel<T, D><<<(unsigned)p.a.total_units, MW_THREADS, MassWideShape<D>::SMEM, st>>>(
        p, small, *static_cast<const CUtensorMap *>(map), layer);
    return cudaGetLastError();
}
cudaError_t launch_attn_mass_wide(const MassParams &p, const SmallSeqs &small, int f16, const void *map, int layer, cudaStream_t st) {
    if (p.a.D == 64)
        return f16 ? mass_wide_go<__half, 64>(p, small, map, layer, st) : mass_wide_go<__nv_bfloat16, 64>(p, small, map, layer, st);
    return f16 ? mass_wide_go<__half, 128>(p, small, map, layer, st) : mass_wide_go<__nv_bfloat16, 128>(p, small, map, layer, st);
}

}  // namespace aafkv
