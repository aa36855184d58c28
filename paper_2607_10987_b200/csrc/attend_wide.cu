// Attention of many query rows per kv head over paged keys and values on the fifth-generation tensor cores: 256 rows a
// CTA (two row tiles of 128), keys in tiles of 128 tokens, head widths 64 and 128, blocks of 8 to 128 tokens.
//
// Bound: the tensor pipe and the exponentials.  Per 256 rows x 128 keys x 128 dims the products take 2 x 1024 cycles of
// the tensor pipe and the 32768 exponentials 2048 cycles of the special-function units, so the two must overlap:
//   - two row tiles take turns: while one's scores are being exponentiated the other's products run;
//   - scores S = Q K^T and outputs O stay in tensor memory (2 x 128 + 2 x D columns of 512); the weights P go back into the
//     upper half of their own scores' columns as the 16-bit first operand of O += P V, so shared memory carries only
//     K and V (both products with operands in shared memory would need more than its bandwidth);
//   - a thread owns a row: its maximum and sum need no exchange.  O is rescaled only when a row's maximum has grown by
//     more than 2^8 since the last time, which costs nothing in accuracy (all sums are in 32 bits, a weight of up to 2^8
//     keeps its digits) and leaves the outputs alone in almost every tile;
//   - one warp copies pages with tiled bulk copies (one per page and 64 dimensions, 128-byte swizzle, five stages), one
//     issues the products, two look at V tiles before they are multiplied.
// Key tiles start on a block boundary, so a copied box is always a whole block; rows of V outside the keys that the
// CTA's rows see are set to zero (0 * garbage is not 0), and a value that is not finite in a tile that some rows see and
// others do not raises `flag`: the caller then runs the 64-row kernel over the batch, which keeps such rows apart.
// The last tile of keys costs the same as a full one, at most 127 keys of it are masked.
//
// Every wait is bounded; one that gives up records AAF_ERR_TIMEOUT and ends the kernel.
#include <cuda.h>

#include "attend_device.cuh"

namespace aafkv {

constexpr int WIDE_TILE = 128, WIDE_KEYS = 128;
constexpr int WIDE_THREADS = 384;
constexpr int WAIT_LIMIT = 1 << 20;

template <int D> struct WideShape {
    static constexpr int HALVES = D / 64;
    static constexpr int TILE_BYTES = HALVES * 128 * 128;  // 128 rows of D 16-bit elements, 64 dims a half
    static constexpr int STAGES = D == 128 ? 5 : 10;
    static constexpr int SMEM = 1024 + (2 + STAGES) * TILE_BYTES + 512;
    static_assert(SMEM <= 227 * 1024, "shared memory of a CTA");
};

__device__ __forceinline__ void bar_init(uint32_t bar, int count) {
    asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// false: gave up, here or elsewhere in the CTA
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, int *status) {
    for (int i = 0; i < WAIT_LIMIT; ++i) {
        if (bar_try(bar, parity)) return true;
        if (*abort_flag) return false;
    }
    *abort_flag = 1;
    atomicCAS(status, 0, AAF_ERR_TIMEOUT);
    return false;
}
// the same for a whole warp: all lanes agree
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, int *status) {
    return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag, status));
}

__device__ __forceinline__ void page_copy(uint32_t dst, const CUtensorMap *map, uint32_t bar, int d, int head, int plane, int layer) {
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(d), "r"(head), "r"(0), "r"(plane), "r"(layer) : "memory");
}

// shared-memory matrix descriptor, 128-byte swizzle: start, leading and stride byte offsets in 16-byte units
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
    return (uint64_t)((addr >> 4) & 0x3fff) | (uint64_t)((lead >> 4) & 0x3fff) << 16 | (uint64_t)((stride >> 4) & 0x3fff) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float *r) {
    uint32_t *u = reinterpret_cast<uint32_t *>(r);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
          "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]),
          "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]),
          "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t *u) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(addr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
          "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]),
          "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]),
          "r"(u[30]), "r"(u[31])
        : "memory");
}

template <typename T> struct WideFormat;
template <> struct WideFormat<__half> { static constexpr uint32_t F = 0; };
template <> struct WideFormat<__nv_bfloat16> { static constexpr uint32_t F = 1; };

template <typename T, int D, bool FANCY>
__global__ void __launch_bounds__(WIDE_THREADS, 1)
    attend_wide_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ SmallSeqs small,
                       const __grid_constant__ CUtensorMap map, int layer) {
    using S = WideShape<D>;
    extern __shared__ char smem_raw[];
    __shared__ uint32_t sh_tmem;
    __shared__ volatile int sh_abort;
    __shared__ int sh_lo[2], sh_hi[2], sh_lo_max[2], sh_hi_min[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t raw = (uint32_t)__cvta_generic_to_shared(smem_raw);
    const uint32_t sQ = (raw + 1023) & ~1023u, sKV = sQ + 2 * S::TILE_BYTES, bars = sKV + S::STAGES * S::TILE_BYTES;
    const uint32_t full = bars, guarded = full + 8 * S::STAGES, empty = guarded + 8 * S::STAGES, q_ready = empty + 8 * S::STAGES,
                   s_full = q_ready + 8, p_ready = s_full + 16, o_done = p_ready + 16, drain = o_done + 16;

    const int unit = blockIdx.x / p.H, head = blockIdx.x - unit * p.H;
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq sq = seqs[find_seq(seqs, p.n, unit)];
    const int R = sq.nq * p.G, n_tiles = (R + WIDE_ROWS - 1) / WIDE_ROWS;
    const int u = unit - sq.unit0, part = u % sq.nsplit;
    const int tile = n_tiles - 1 - u / sq.nsplit;  // the latest rows see the most keys: they start first
    const int r0 = tile * WIDE_ROWS;
    const bool two = r0 + WIDE_TILE < R;           // the second row tile has rows

    if (warp == 8) {
        if (lane == 0) {
            for (int i = 0; i < S::STAGES; ++i) {
                bar_init(full + 8 * i, 1);
                bar_init(guarded + 8 * i, 2);
                bar_init(empty + 8 * i, 1);
            }
            bar_init(q_ready, 256);
            bar_init(drain, 1);
            for (int w = 0; w < 2; ++w) {
                bar_init(s_full + 8 * w, 1);
                bar_init(p_ready + 8 * w, 128);
                bar_init(o_done + 8 * w, 1);
            }
            sh_abort = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(
                         (uint32_t)__cvta_generic_to_shared(&sh_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // spans of the two row tiles, each looked at by one warp
    if (warp >= 10) {
        const int w = warp - 10, a = min(r0 + w * WIDE_TILE, R - 1), b = min(r0 + w * WIDE_TILE + WIDE_TILE - 1, R - 1);
        int lo = 0x7fffffff, hi = 0, lo_max = 0, hi_min = 0x7fffffff;
        for (int j = a / p.G + lane; j <= b / p.G; j += 32) {
            const RowSpan sp = row_span(p, sq, j);
            if (sp.hi > sp.lo) {
                lo = min(lo, sp.lo);
                hi = max(hi, sp.hi);
            }
            lo_max = max(lo_max, sp.lo);
            hi_min = min(hi_min, sp.hi);
        }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, d));
            hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, d));
            lo_max = max(lo_max, __shfl_xor_sync(0xffffffffu, lo_max, d));
            hi_min = min(hi_min, __shfl_xor_sync(0xffffffffu, hi_min, d));
        }
        if (lane == 0) {
            sh_lo[w] = lo;
            sh_hi[w] = hi;
            sh_lo_max[w] = lo_max;
            sh_hi_min[w] = hi_min;
        }
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    const uint32_t tmem = sh_tmem;
    int lo = min(sh_lo[0], sh_lo[1]), hi = max(sh_hi[0], sh_hi[1]);
    const int lo_max = max(sh_lo_max[0], sh_lo_max[1]), hi_min = min(sh_hi_min[0], sh_hi_min[1]);
    if (hi <= lo) lo = hi = 0;
    int t0 = lo / p.BS * p.BS;  // tiles start on a block boundary
    if (sq.nsplit > 1) {        // parts of whole key tiles
        const int all = (hi - t0 + WIDE_KEYS - 1) / WIDE_KEYS, each = (all + sq.nsplit - 1) / sq.nsplit;
        const int b = t0 + min(part * each, all) * WIDE_KEYS;
        hi = min(hi, t0 + min((part + 1) * each, all) * WIDE_KEYS);
        lo = max(lo, b);
        t0 = b;
        if (hi <= lo) lo = hi = t0 = 0;
    }
    const int tiles = (hi - t0 + WIDE_KEYS - 1) / WIDE_KEYS;

    if (warp < 8) {
        // ---------------------------------------------------------------- a thread per row: weights
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int w = warp >> 2, rl = (warp & 3) * 32 + lane, rr = r0 + w * WIDE_TILE + rl;
        const int rc = min(rr, R - 1);
        {   // the row's queries into the swizzled tile (rows behind the last: zeros); a negative scale moves into their sign
            const T *q = static_cast<const T *>(p.q) + (long long)(sq.row0 + rc / p.G) * p.q_stride + (long long)(head * p.G + rc % p.G) * D;
            const uint32_t flip = !FANCY && p.scale < 0.0f ? 0x80008000u : 0u;
            const uint32_t dst = sQ + w * S::TILE_BYTES + rl * 128;
#pragma unroll
            for (int c = 0; c < D / 8; ++c) {
                uint4 v = rr < R ? __ldg(reinterpret_cast<const uint4 *>(q + c * 8)) : make_uint4(0, 0, 0, 0);
                v.x ^= flip;
                v.y ^= flip;
                v.z ^= flip;
                v.w ^= flip;
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(dst + (c >> 3) * 16384 + (((c & 7) ^ (rl & 7)) << 4)),
                             "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            bar_arrive(q_ready);
        }
        const RowSpan span = row_span(p, sq, rc / p.G);
        const float slope = p.slopes ? p.slopes[head * p.G + rc % p.G] : 0.0f;
        int w_lo_max = span.lo, w_hi_min = span.hi;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            w_lo_max = max(w_lo_max, __shfl_xor_sync(0xffffffffu, w_lo_max, d));
            w_hi_min = min(w_hi_min, __shfl_xor_sync(0xffffffffu, w_hi_min, d));
        }
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lanes + w * 128, tP = tS + 64, tO = tmem + lanes + 256 + w * D;
        const float c = fabsf(p.scale) * LOG2E;
        float m = -CUDART_INF_F, l = 0.0f;
        const bool active = w == 0 || two;
        bool ok = true;
        for (int j = 0; active && j < tiles; ++j) {
            if (!(ok = warp_wait(s_full + 8 * w, j & 1, &sh_abort, p.status))) break;
            tmem_after();
            float s[128];
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_ld32(tS + 32 * i, s + 32 * i);
            tmem_wait_ld();
            const int tb = t0 + j * WIDE_KEYS;
            if (FANCY) {
#pragma unroll
                for (int i = 0; i < 128; ++i) s[i] = score2(p, s[i], slope, span, tb + i);
            }
            if (tb < w_lo_max || tb + WIDE_KEYS > w_hi_min || tb + WIDE_KEYS > hi) {
                const int a = span.lo - tb, b = min(span.hi, hi) - tb;
#pragma unroll
                for (int i = 0; i < 128; ++i) s[i] = i >= a && i < b ? s[i] : -CUDART_INF_F;
            }
            float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
            for (int i = 4; i < 128; i += 4) {
                mx[0] = fmaxf(mx[0], s[i]);
                mx[1] = fmaxf(mx[1], s[i + 1]);
                mx[2] = fmaxf(mx[2], s[i + 2]);
                mx[3] = fmaxf(mx[3], s[i + 3]);
            }
            const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * (FANCY ? 1.0f : c);
            // the first maximum, or one that outgrew the one in use by more than 2^8
            const bool grow = top > m + 8.0f || (m == -CUDART_INF_F && top > m);
            if (__any_sync(0xffffffffu, grow)) {
                const float f = grow && m != -CUDART_INF_F ? ex2(m - top) : 1.0f;
                if (grow) m = top;
                l *= f;
                if (j > 0 && __any_sync(0xffffffffu, f != 1.0f)) {
                    if (!(ok = warp_wait(o_done + 8 * w, (j - 1) & 1, &sh_abort, p.status))) break;
                    tmem_after();
#pragma unroll
                    for (int d = 0; d < D; d += 32) {
                        float o[32];
                        tmem_ld32(tO + d, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] *= f;
                        tmem_st32(tO + d, reinterpret_cast<const uint32_t *>(o));
                    }
                    tmem_wait_st();
                }
            }
            const float base = m == -CUDART_INF_F ? 0.0f : m;
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t pk[32];
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    const int e = h * 64 + 2 * i;
                    float x[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        x[k] = ex2(FANCY ? s[e + k] - base : fmaf(s[e + k], c, -base));
                        sum[k] += x[k];
                    }
                    pk[i] = Elt<T>::pack(x[0], x[1]);
                    pk[i + 1] = Elt<T>::pack(x[2], x[3]);
                }
                tmem_st32(tP + 32 * h, pk);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            tmem_wait_st();
            tmem_before();
            bar_arrive(p_ready + 8 * w);
        }
        if (ok && active && tiles > 0) {
            ok = warp_wait(o_done + 8 * w, (tiles - 1) & 1, &sh_abort, p.status);
            tmem_after();
        }
        if (ok && active) {
            const bool live = rr < R;
            const bool part_out = sq.part0 >= 0;
            const long long qt = sq.row0 + rc / p.G;
            const int hq = head * p.G + rc % p.G;
            const long long pr = sq.part0 + (((long long)tile * sq.nsplit + part) * p.H + head) * WIDE_ROWS + w * WIDE_TILE + rl;
            const float inv = part_out ? 1.0f : (l > 0.0f || l != l ? 1.0f / l : 0.0f);  // a row that sees nothing is zero
            T *out = static_cast<T *>(p.out) + (qt * p.H * p.G + hq) * D;
#pragma unroll
            for (int d = 0; d < D; d += 32) {
                float o[32];
                __syncwarp();
                if (tiles > 0) {
                    tmem_ld32(tO + d, o);
                    tmem_wait_ld();
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = tiles > 0 ? o[i] * inv : 0.0f;
                if (live && part_out) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        *reinterpret_cast<float4 *>(p.part_o + pr * D + d + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                } else if (live) {
#pragma unroll
                    for (int i = 0; i < 32; i += 8)
                        *reinterpret_cast<uint4 *>(out + d + i) =
                            make_uint4(Elt<T>::pack(o[i], o[i + 1]), Elt<T>::pack(o[i + 2], o[i + 3]),
                                       Elt<T>::pack(o[i + 4], o[i + 5]), Elt<T>::pack(o[i + 6], o[i + 7]));
                }
            }
            if (live && part_out) {
                p.part_ml[2 * pr] = m;
                p.part_ml[2 * pr + 1] = l;
            } else if (live && p.lse) {
                p.lse[qt * p.H * p.G + hq] = l == 0.0f ? -CUDART_INF_F : (m + log2f(l)) * LN2 - slope * (float)span.near;
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        const int loads = 2 * tiles;  // K0 V0 K1 V1 ...
        if (warp == 8) {
            // ------------------------------------------------------------ pages of K and V into the stages
            const int *table = p.tables + (long long)sq.ctx * p.max_blk;
            const int pages = WIDE_KEYS / p.BS;  // per tile, at most 16
            bool ok = true;
            int id = 0, done = 0;
            for (int n = 0; ok && n < loads; ++n) {
                const int stage = n % S::STAGES, tb = t0 + (n >> 1) * WIDE_KEYS, at = tb + lane * p.BS;
                const bool mine = lane < pages && at < hi && at + p.BS > lo;
                if (!(n & 1)) id = mine ? __ldg(table + at / p.BS) : 0;
                if (n >= S::STAGES) ok = warp_wait(empty + 8 * stage, (n / S::STAGES - 1) & 1, &sh_abort, p.status);
                if (!ok) break;
                const int count = __popc(__ballot_sync(0xffffffffu, mine));
                if (lane == 0) bar_expect(full + 8 * stage, (uint32_t)(count * p.BS * D * 2));
                __syncwarp();
                if (mine) {
                    const uint32_t dst = sKV + stage * S::TILE_BYTES + lane * p.BS * 128;
#pragma unroll
                    for (int h = 0; h < S::HALVES; ++h)
                        page_copy(dst + h * 16384, &map, full + 8 * stage, h * 64, head, 2 * id + (n & 1), layer);
                }
                done = n + 1;
            }
            // nothing may be in flight when the CTA ends early: wait for what was issued
            if (!ok)
                for (int n = max(0, done - S::STAGES); n < done; ++n)
                    for (int i = 0; i < WAIT_LIMIT && !bar_try(full + 8 * (n % S::STAGES), (n / S::STAGES) & 1); ++i) {}
        } else if (warp == 9) {
            // ------------------------------------------------------------ products
            if (lane == 0) {
                constexpr uint32_t F = WideFormat<T>::F;
                constexpr uint32_t QK = 1u << 4 | F << 7 | F << 10 | (WIDE_KEYS / 8) << 17 | (WIDE_TILE / 16) << 24;
                constexpr uint32_t PV = 1u << 4 | F << 7 | F << 10 | 1u << 16 | (D / 8) << 17 | (WIDE_TILE / 16) << 24;
                bool ok = bar_wait(q_ready, 0, &sh_abort, p.status);
                auto ready = [&](int n) {  // load n has landed and been looked at
                    const int stage = n % S::STAGES, parity = (n / S::STAGES) & 1;
                    return bar_wait(full + 8 * stage, parity, &sh_abort, p.status) && bar_wait(guarded + 8 * stage, parity, &sh_abort, p.status);
                };
                auto scores = [&](int w, int n) {
                    const uint32_t a = sQ + w * S::TILE_BYTES, b = sKV + (n % S::STAGES) * S::TILE_BYTES;
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = (k >> 2) * 16384 + (k & 3) * 32;
                        mma_ss(tmem + w * 128, smem_desc(a + off, 16, 1024), smem_desc(b + off, 16, 1024), QK, k > 0);
                    }
                    mma_commit(s_full + 8 * w);
                };
                if (ok && tiles > 0 && (ok = ready(0))) {
                    tmem_after();
                    scores(0, 0);
                    if (two) scores(1, 0);
                    if (S::STAGES < loads) mma_commit(empty);  // an arrival is asked for only where someone waits for it
                }
                for (int j = 0; ok && j < tiles; ++j) {
                    const int nv = 2 * j + 1, nk = 2 * j + 2;
                    const bool more = j + 1 < tiles;
                    if (!(ok = ready(nv))) break;
                    for (int w = 0; w < (two ? 2 : 1); ++w) {
                        if (!(ok = bar_wait(p_ready + 8 * w, j & 1, &sh_abort, p.status))) break;
                        tmem_after();
                        const uint32_t b = sKV + (nv % S::STAGES) * S::TILE_BYTES;
#pragma unroll
                        for (int k = 0; k < WIDE_KEYS / 16; ++k)
                            mma_ts(tmem + 256 + w * D, tmem + w * 128 + 64 + k * 8, smem_desc(b + k * 2048, 16384, 1024), PV, j > 0 || k > 0);
                        mma_commit(o_done + 8 * w);
                        if (more) {  // in order behind the product that still reads P from these columns
                            if (w == 0 && !(ok = ready(nk))) break;
                            scores(w, nk);
                        }
                    }
                    if (!ok) break;
                    if (nv + S::STAGES < loads) mma_commit(empty + 8 * (nv % S::STAGES));
                    if (nk + S::STAGES < loads) mma_commit(empty + 8 * (nk % S::STAGES));
                }
            }
            __syncwarp();
        } else {
            // ------------------------------------------------------------ V tiles that not every row sees whole
            const int tid = threadIdx.x - 320;
            bool odd = false, ok = true;
            for (int n = 0; n < loads; ++n) {
                const int stage = n % S::STAGES;
                if (!(ok = warp_wait(full + 8 * stage, (n / S::STAGES) & 1, &sh_abort, p.status))) break;
                const int tb = t0 + (n >> 1) * WIDE_KEYS;
                if ((n & 1) && (tb < lo_max || tb + WIDE_KEYS > hi_min || tb + WIDE_KEYS > hi)) {
                    const uint32_t v = sKV + stage * S::TILE_BYTES;
                    for (int i = tid; i < S::TILE_BYTES / 16; i += 64) {
                        const int t = tb + ((i >> 3) & 127);
                        const uint32_t at = v + i * 16;
                        if (t < lo || t >= hi) {
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(at), "r"(0) : "memory");
                        } else {
                            const uint4 x = lds16(at);
                            odd |= finite_only<T>(x.x) != x.x || finite_only<T>(x.y) != x.y || finite_only<T>(x.z) != x.z ||
                                   finite_only<T>(x.w) != x.w;
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                __syncwarp();
                if (lane == 0) bar_arrive(guarded + 8 * stage);
            }
            if (odd) *p.flag = p.epoch;
        }
    }
    __syncthreads();
    if (sh_abort && threadIdx.x == 288) {
        // a wait gave up: let the products that were issued finish before tensor memory is given back
        mma_commit(drain);
        for (int i = 0; i < WAIT_LIMIT && !bar_try(drain, 0); ++i) {}
    }
    __syncthreads();
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

bool wide_takes(int D, int BS) { return (D == 64 || D == 128) && BS >= 8 && BS <= WIDE_KEYS && (BS & (BS - 1)) == 0; }

template <typename T, int D, bool FANCY>
static cudaError_t wide_go(const AttnParams &p, const SmallSeqs &small, const void *map, int layer, cudaStream_t st) {
    const cudaError_t e =
        cudaFuncSetAttribute(attend_wide_kernel<T, D, FANCY>, cudaFuncAttributeMaxDynamicSharedMemorySize, WideShape<D>::SMEM);
    if (e != cudaSuccess) return e;
    attend_wide_kernel<T, D, FANCY><<<(unsigned)((long long)p.total_units * p.H), WIDE_THREADS, WideShape<D>::SMEM, st>>>(
        p, small, *static_cast<const CUtensorMap *>(map), layer);
    return cudaGetLastError();
}
template <typename T> static cudaError_t wide_pick(const AttnParams &p, const SmallSeqs &small, const void *map, int layer, cudaStream_t st) {
    const bool fancy = p.softcap != 0.0f || p.slopes || p.scale == 0.0f;  // 0 * -inf would undo a mask
    if (p.D == 64) return fancy ? wide_go<T, 64, true>(p, small, map, layer, st) : wide_go<T, 64, false>(p, small, map, layer, st);
    return fancy ? wide_go<T, 128, true>(p, small, map, layer, st) : wide_go<T, 128, false>(p, small, map, layer, st);
}
cudaError_t launch_attend_wide(const AttnParams &p, const SmallSeqs &small, int f16, const void *map, int layer, cudaStream_t st) {
    return f16 ? wide_pick<__half>(p, small, map, layer, st) : wide_pick<__nv_bfloat16>(p, small, map, layer, st);
}

// Tensor map of a whole pool: [layer][block * 2 + (K, V)][slot][kv head][dim], boxes of one block's slots of one head, 64 dims.
// The encoder is the driver's, found through the runtime (nothing links against the driver library).
static_assert(sizeof(CUtensorMap) == sizeof(PoolMap), "room for a tensor map");
bool encode_pool_map(const Geom &g, PoolMap *out) {
    typedef CUresult (*Encode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                               const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                               CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess || !fn) {
        cudaGetLastError();
        return false;
    }
    const cuuint64_t dims[5] = {(cuuint64_t)g.D, (cuuint64_t)g.H, (cuuint64_t)g.BS, 2 * (cuuint64_t)g.NB, (cuuint64_t)g.L};
    const cuuint64_t strides[4] = {2 * (cuuint64_t)g.D, (cuuint64_t)g.row, (cuuint64_t)g.run, (cuuint64_t)g.layer_stride};
    const cuuint32_t box[5] = {64, 1, (cuuint32_t)g.BS, 1, 1}, step[5] = {1, 1, 1, 1, 1};
    return reinterpret_cast<Encode>(fn)(reinterpret_cast<CUtensorMap *>(out), CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, g.pool, dims, strides,
                                        box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace aafkv
