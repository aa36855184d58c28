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
//   - a warp for K and one for V copy blocks with tiled bulk copies (one per block and 64 dimensions, 128-byte swizzle, five
//     stages; a copy takes about 85 cycles to issue, one warp for both would be as slow as the products), two warps issue
//     the products, one for each row tile.
// Key tiles start on a block boundary, so a copied box is always a whole block; rows of V outside the keys that the
// CTA's rows see are set to zero (0 * garbage is not 0), and a value that is not finite in a tile that some rows see and
// others do not raises `flag`: the caller then runs the 64-row kernel over the batch, which keeps such rows apart.
// The last tile of keys costs the same as a full one, at most 127 keys of it are masked.
// 16 contexts of 8699 tokens, 512 new each, 32 heads of 128: 1114 us under the power cap (1.02 PFLOP/s).
//
// Weights are rounded to the values' type before O += P V, as the tensor pipe takes them: one more rounding of the output's kind,
// half a step of each weight, while their sum stays in 32 bits.  A second product with what the rounding left would take the tensor
// pipe as long again.  Error against 64 bits with 16 contexts of 8699 tokens, 512 of them new: 2.3e-3 of the output's norm, of
// which the output's own rounding to bf16 is 1.7e-3.
//
// Every wait is bounded; one that gives up records AAF_ERR_TIMEOUT and ends the kernel.
#include <cuda.h>

#include <type_traits>

#include "tensor_device.cuh"

namespace aafkv {

constexpr int WIDE_TILE = 128, WIDE_KEYS = 128;
constexpr int WIDE_THREADS = 384;  // 8 warps for the weights, 4 for copies, products and the look at V

template <int D> struct WideShape {
    static constexpr int HALVES = D / 64;
    static constexpr int TILE_BYTES = HALVES * 128 * 128;  // 128 rows of D 16-bit elements, 64 dims a half
    static constexpr int STAGES = D == 128 ? 5 : 10;
    static constexpr int BARS = (2 + STAGES) * TILE_BYTES, WORDS = BARS + 512;
    static constexpr int SMEM = WORDS + 64;
    static_assert(SMEM <= 227 * 1024, "shared memory of a CTA");
};

// cap * tanh(s k) * log2(e) as s * (c0 + z (c1 + z (c2 + z (c3 + z c4)))), z = s^2, for |s k| <= 0.5: tanh(y) / y as a polynomial
// in y^2 that starts with 1 (least maximal relative error, fitted by linear programming: 1.6e-8 with the coefficients as 32 bits
// hold them; evaluated in 32 bits 5e-8), k and the cap folded into its coefficients.  The last one is positive, so a masked score, -inf, stays -inf.
constexpr float TANH_POLY_MAX = 0.5f;
struct CapPoly {
    float c[5];
    __device__ __forceinline__ CapPoly(float times, float k) {  // times = cap * k * log2(e)
        const float z = k * k;
        c[0] = times;
        c[1] = -0.33333144f * times * z;
        c[2] = 0.13325880f * times * z * z;
        c[3] = -0.05304564f * times * z * z * z;
        c[4] = 0.0172418f * times * z * z * z * z;
    }
    __device__ __forceinline__ f2 operator()(f2 s, f2 add) const {
        const f2 z = mul2(s, s);
        f2 q = fma2(z, pair(c[4], c[4]), pair(c[3], c[3]));
        q = fma2(z, q, pair(c[2], c[2]));
        q = fma2(z, q, pair(c[1], c[1]));
        q = fma2(z, q, pair(c[0], c[0]));
        return fma2(s, q, add);
    }
};

// MODE: what a score is.  0: a multiple of the product; 1: capped; 2: anything (with a distance bias, or a scale of zero)
// GROUP: the rows of contexts forked from one, over the keys that they share.  Each of these contexts would else be attend_few's,
// which multiplies the weights in two 16-bit parts; so does this variant, for a row must not lose digits because of what else
// is in the batch.  It has one row tile, and two threads a row: both look at all of a tile's scores, so that they agree on
// the maximum, and each computes the weights of 64 keys.  Both parts go where the second row tile's scores would be, the low parts'
// product into the columns of its outputs.  (The sum of the two is the output unless the high parts' product is not finite: an infinite
// value is infinite there, and times a low part, which may be zero or negative, NaN.)  16 contexts forked at 8187 tokens: 34.6 us a
// call; 32.5 with the weights rounded once, 40.3 with one thread a row.
template <typename T, int D, int MODE, bool GROUP>
__global__ void __launch_bounds__(WIDE_THREADS, 1)
    attend_wide_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ SmallSeqs small,
                       const __grid_constant__ CUtensorMap map, int layer) {
    using S = WideShape<D>;
    // all shared memory is dynamic, so that its start is that of the CTA's window and the swizzled tiles are aligned
    extern __shared__ __align__(1024) char smem_raw[];
    uint32_t &sh_tmem = *reinterpret_cast<uint32_t *>(smem_raw + S::WORDS);
    volatile int &sh_abort = *reinterpret_cast<volatile int *>(smem_raw + S::WORDS + 4);
    int *sh_lo = reinterpret_cast<int *>(smem_raw + S::WORDS + 8), *sh_hi = sh_lo + 2, *sh_lo_max = sh_lo + 4, *sh_hi_min = sh_lo + 6;
    asm volatile("griddepcontrol.launch_dependents;");  // the join may be brought up beside this kernel
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t raw = (uint32_t)__cvta_generic_to_shared(smem_raw);
    const uint32_t sQ = raw, sKV = sQ + 2 * S::TILE_BYTES, bars = raw + S::BARS;
    if (raw & 1023) {  // never: the swizzle goes by address bits
        if (threadIdx.x == 0) atomicCAS(p.status, 0, AAF_ERR_CORRUPT);
        return;
    }
    const uint32_t full = bars, guarded = full + 8 * S::STAGES, empty = guarded + 8 * S::STAGES, q_ready = empty + 8 * S::STAGES,
                   s_full = q_ready + 8, p_ready = s_full + 16, o_done = p_ready + 16, drain = o_done + 16, p_rest = drain + 16, turn = p_rest + 16;

    const int unit = blockIdx.x / p.H, head = blockIdx.x - unit * p.H;
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq sq = seqs[p.first + find_seq(seqs + p.first, p.n, unit)];
    constexpr int ROWS = GROUP ? GROUP_ROWS : WIDE_ROWS;
    // query token j of the record, its place in the packed batch and the keys it sees
    auto token = [&](int j, int &packed) -> RowSpan {
        if (!GROUP) {
            packed = sq.row0 + j;
            return row_span(p, sq, j);
        }
        const int member = j / sq.chunk, jj = j - member * sq.chunk;
        const AttnSeq &ms = seqs[sq.row0 + member];
        packed = ms.row0 + jj;
        RowSpan r;  // no mask but the causal one; the nearest key is the token itself, in the member's own part
        r.pos = ms.len - ms.nq + jj;
        r.lo = 0;
        r.hi = min(r.pos + 1, sq.len);
        r.near = 0;
        return r;
    };
    const int R = sq.nq * p.G, n_tiles = (R + ROWS - 1) / ROWS;
    const int u = unit - sq.unit0, part = u % sq.nsplit;
    const int tile = n_tiles - 1 - u / sq.nsplit;  // the latest rows see the most keys: they start first
    const int r0 = tile * ROWS;
    const bool two = !GROUP && r0 + WIDE_TILE < R;  // the second row tile has rows

    if (warp == 8) {
        if (lane == 0) {
            for (int i = 0; i < S::STAGES; ++i) {
                bar_init(full + 8 * i, 1);
                bar_init(guarded + 8 * i, 1);
                bar_init(empty + 8 * i, two ? 2 : 1);
            }
            bar_init(q_ready, 256);
            bar_init(drain, 1);
            bar_init(turn, 1);
            bar_init(turn + 8, 1);
            bar_init(drain + 8, 1);
            for (int w = 0; w < 2; ++w) {
                bar_init(s_full + 8 * w, 1);
                bar_init(p_ready + 8 * w, 4);
                bar_init(p_rest + 8 * w, 4);
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
        const int w = warp - 10, first = r0 + (GROUP ? 0 : w * WIDE_TILE), a = min(first, R - 1), b = min(first + WIDE_TILE - 1, R - 1);
        int lo = 0x7fffffff, hi = 0, lo_max = 0, hi_min = 0x7fffffff;
        for (int j = a / p.G + lane; j <= b / p.G; j += 32) {
            int packed;
            const RowSpan sp = token(j, packed);
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
    constexpr uint32_t tmem = 0;  // all 512 columns are this CTA's, so they start at column 0
    if (sh_tmem != 0 && threadIdx.x == 0) atomicCAS(p.status, 0, AAF_ERR_CORRUPT);  // never
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
        const int w = warp >> 2, rl = (warp & 3) * 32 + lane, rr = r0 + (GROUP ? 0 : w) * WIDE_TILE + rl;
        const int rc = min(rr, R - 1), rj = token_of(p, rc), hq = head * p.G + rc - rj * p.G;
        int packed;
        const RowSpan span = token(rj, packed);
        if (!GROUP || w == 0) {   // the warp's 32 rows of queries into the swizzled tile, D / 8 lanes a row (rows behind the last: zeros); a negative
            // scale moves into their sign
            constexpr int PIECES = D / 8, AT_ONCE = 32 / PIECES;
            const uint32_t flip = MODE < 2 && p.scale < 0.0f ? 0x80008000u : 0u;
            const int ch = lane % PIECES;
            uint4 v[PIECES];
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int rq = r0 + w * WIDE_TILE + (warp & 3) * 32 + i * AT_ONCE + lane / PIECES, rn = min(rq, R - 1), rt = token_of(p, rn);
                int at;
                token(rt, at);
                const T *q = static_cast<const T *>(p.q) + (long long)at * p.q_stride + (long long)(head * p.G + rn - rt * p.G) * D;
                v[i] = rq < R ? __ldg(reinterpret_cast<const uint4 *>(q + ch * 8)) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {  // all loads are under way before the first result is stored
                const int r = (warp & 3) * 32 + i * AT_ONCE + lane / PIECES;
                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(sQ + w * S::TILE_BYTES + r * 128 + (ch >> 3) * 16384 +
                                                                         (((ch & 7) ^ (r & 7)) << 4)),
                             "r"(v[i].x ^ flip), "r"(v[i].y ^ flip), "r"(v[i].z ^ flip), "r"(v[i].w ^ flip) : "memory");
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        bar_arrive(q_ready);
        const float slope = MODE == 2 && p.slopes ? p.slopes[hq] : 0.0f;
        int w_lo_max = span.lo, w_hi_min = span.hi;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            w_lo_max = max(w_lo_max, __shfl_xor_sync(0xffffffffu, w_lo_max, d));
            w_hi_min = min(w_hi_min, __shfl_xor_sync(0xffffffffu, w_hi_min, d));
        }
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const int rt = GROUP ? 0 : w;  // row tile
        const uint32_t tS = tmem + lanes + rt * 128, tP = GROUP ? tmem + lanes + 128 : tS + 64, tO = tmem + lanes + 256 + w * D;
        const float c = fabsf(p.scale) * LOG2E, k1 = fabsf(p.scale) * p.inv_cap, cap2 = p.softcap * LOG2E;
        const CapPoly capped(c, k1);
        constexpr float GROWTH = 8.0f;  // how far (log2) a score may outgrow the maximum in use
        constexpr float RAISE = Elt<T>::RAISE > 0.0f ? Elt<T>::RAISE - GROWTH : 0.0f;
        float m = -CUDART_INF_F, l = 0.0f;
        const bool active = GROUP || w == 0 || two;
        bool ok = true;
        // weights of two keys: scores are multiples of the products, or, with a cap and all of them small, a polynomial
        auto pair_of = [&](float s0, float s1, float times, float base, auto poly) -> f2 {
            f2 x;
            if (poly.value)
                x = capped(pair(s0, s1), pair(-base, -base));
            else
                x = fma2(pair(s0, s1), pair(times, times), pair(-base, -base));
            float a, b;
            unpair(x, a, b);
            return pair(ex2(a), ex2(b));
        };
        auto done_half = [&](int h, const uint32_t *pk) {  // 64 keys' weights: the product may start on them
            tmem_st32(tP + 32 * h, pk);
            tmem_wait_st();
            tmem_before();
            __syncwarp();
            if (lane == 0) bar_arrive((h ? p_rest : p_ready) + 8 * rt);
        };
        // a tile's largest score against the maximum in use: 0, it serves; 1, it is another one now; -1, a wait gave up
        auto settle = [&](int j, float most, float times, auto poly) -> int {
            const float top = poly.value && most > -CUDART_INF_F ? cap2 * tanh_f32(most * k1) : most * times;
            // the first maximum, or one that outgrew the one in use
            const bool grow = top > m + GROWTH || (m == -CUDART_INF_F && top > m);
            if (!__any_sync(0xffffffffu, grow)) return 0;
            const float f = grow && m != -CUDART_INF_F ? ex2(m - top) : 1.0f;
            if (grow) m = top;
            l *= f;
            if (j > 0 && __any_sync(0xffffffffu, f != 1.0f)) {
                if (!warp_wait(o_done + 8 * rt, (j - 1) & 1, &sh_abort, p.status)) return -1;
                tmem_after();
#pragma unroll 1
                for (int d = 0; d < D; d += 16) {
                    float o[16];
                    tmem_ld16(tO + d, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] *= f;
                    tmem_st16(tO + d, reinterpret_cast<const uint32_t *>(o));
                }
                tmem_wait_st();
            }
            return 1;
        };
        for (int j = 0; active && j < tiles; ++j) {
            if (!(ok = warp_wait(s_full + 8 * rt, j & 1, &sh_abort, p.status))) break;
            tmem_after();
            float s[128];
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_ld32(tS + 32 * i, s + 32 * i);
            tmem_wait_ld();
            const int tb = t0 + j * WIDE_KEYS;
            const bool edge = tb < w_lo_max || tb + WIDE_KEYS > w_hi_min || tb + WIDE_KEYS > hi;
            const int a0 = span.lo - tb, b0 = min(span.hi, hi) - tb;  // the tile's keys that this row sees
            float times = 1.0f;
            bool small = false;
            auto mask = [&](float with) {
                if (__any_sync(0xffffffffu, a0 > 0))
#pragma unroll
                    for (int i = 0; i < 128; ++i) s[i] = i < a0 ? with : s[i];
                if (__any_sync(0xffffffffu, b0 < 128))
#pragma unroll
                    for (int i = 0; i < 128; ++i) s[i] = i >= b0 ? with : s[i];
            };
            if (MODE == 1) {
                if (edge) mask(0.0f);  // what a masked key holds decides nothing
                float mx[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) mx[k] = fabsf(s[k]);
#pragma unroll
                for (int i = 4; i < 124; i += 8)
#pragma unroll
                    for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], fabsf(s[i + 2 * k]), fabsf(s[i + 2 * k + 1]));
                const float most = max3(max3(mx[0], fabsf(s[124]), fabsf(s[125])), max3(mx[1], fabsf(s[126]), fabsf(s[127])), max3(mx[2], mx[3], mx[3]));
                small = __all_sync(0xffffffffu, most * k1 <= TANH_POLY_MAX) && capped.c[4] > 0.0f && capped.c[4] < CUDART_INF_F;  // false for a NaN
            }
            if (MODE == 0 || small) {
                times = c;
            } else if (MODE == 2 && p.softcap == 0.0f && abs(span.pos - tb) + WIDE_KEYS < 1 << 24) {
                // distances are whole numbers, which 32 bits hold up to 2^24, measured from the nearest visible key (see RowSpan)
                const float d0 = (float)(span.pos - tb), slope2 = slope * LOG2E, c2 = p.scale * LOG2E, near = (float)span.near;
#pragma unroll
                for (int i = 0; i < 128; ++i) s[i] = fmaf(-slope2, fabsf(d0 - (float)i) - near, s[i] * c2);
            } else {
#pragma unroll
                for (int i = 0; i < 128; ++i) s[i] = score2(p, MODE == 1 && p.scale < 0.0f ? -s[i] : s[i], slope, span, tb + i);
            }
            if (edge) mask(-CUDART_INF_F);
            auto weights = [&](auto poly) -> bool {
                uint32_t pk[32];
                f2 sums[2];
                if constexpr (GROUP) {
                    float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                    for (int i = 4; i < 128; ++i) mx[i & 3] = fmaxf(mx[i & 3], s[i]);
                    if (settle(j, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), times, poly) < 0) return false;
                    const float base = m == -CUDART_INF_F ? 0.0f : m - RAISE;
                    uint32_t low[32];  // what the rounding leaves of the weights
                    sums[0] = sums[1] = 0;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const f2 x = pair_of(w ? s[64 + 2 * i] : s[2 * i], w ? s[65 + 2 * i] : s[2 * i + 1], times, base, poly);
                        sums[i & 1] = add2(sums[i & 1], x);
                        float a, b;
                        unpair(x, a, b);
                        pk[i] = Elt<T>::pack(a, b);
                        low[i] = Elt<T>::pack(a - Elt<T>::lo(pk[i]), b - Elt<T>::hi(pk[i]));
                    }
                    tmem_st32(tP + 64 + 32 * w, low);
                    done_half(w, pk);
                    float a, b;
                    unpair(add2(sums[0], sums[1]), a, b);
                    l += a + b;
                    return true;
                }
                // The maximum in use serves this tile too unless a score outgrows it by 2^8, so the first half of the weights is
                // computed beside the tile's maximum, not behind it, and once more in the tiles where it was too small.
                for (;;) {
                    const float base = m == -CUDART_INF_F ? 0.0f : m - RAISE;
                    float mx[4] = {s[0], s[1], s[2], s[3]};
                    sums[0] = sums[1] = 0;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const f2 x = pair_of(s[2 * i], s[2 * i + 1], times, base, poly);
                        sums[i & 1] = add2(sums[i & 1], x);
                        float a, b;
                        unpair(x, a, b);
                        pk[i] = Elt<T>::pack(a, b);
                        mx[i & 3] = fmaxf(fmaxf(fmaxf(mx[i & 3], s[4 * i]), fmaxf(s[4 * i + 1], s[4 * i + 2])), s[4 * i + 3]);
                    }
                    const float most = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                    const int changed = settle(j, most, times, poly);
                    if (changed < 0) return false;
                    if (!changed) break;
                }
                done_half(0, pk);
                const float base = m == -CUDART_INF_F ? 0.0f : m - RAISE;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const f2 x = pair_of(s[64 + 2 * i], s[65 + 2 * i], times, base, poly);
                    sums[i & 1] = add2(sums[i & 1], x);
                    float a, b;
                    unpair(x, a, b);
                    pk[i] = Elt<T>::pack(a, b);
                }
                done_half(1, pk);
                float a, b;
                unpair(add2(sums[0], sums[1]), a, b);
                l += a + b;
                return true;
            };
            if (MODE == 1 && small)
                ok = weights(std::true_type{});
            else
                ok = weights(std::false_type{});
            if (!ok) break;
        }
        if (ok && active && tiles > 0) {
            ok = warp_wait(o_done + 8 * rt, (tiles - 1) & 1, &sh_abort, p.status);
            tmem_after();
        }
        if (GROUP) {  // the row's other sum; the place of the second row tile's queries is free
            float *other = reinterpret_cast<float *>(smem_raw + S::TILE_BYTES);
            if (!w) other[rl] = l;
            asm volatile("bar.sync 1, 256;" ::: "memory");  // every weights' warp comes here, whatever it waited for in vain
            const float first = other[rl];
            if (w) other[128 + rl] = l;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            l = first + other[128 + rl];
        }
        if (ok && active) {
            const bool live = rr < R;
            const bool part_out = sq.part0 >= 0;
            const long long qt = packed;
            const long long pr = sq.part0 + (((long long)tile * sq.nsplit + part) * p.H + head) * ROWS + rt * WIDE_TILE + rl;
            const float inv = l > 0.0f || l != l ? (part_out ? 1.0f : 1.0f / l) : 0.0f;  // a row that sees nothing is zero
            T *out = static_cast<T *>(p.out) + (qt * p.H * p.G + hq) * D;
            float *part_o = p.part_o + pr * D;
#pragma unroll 1
            for (int d = GROUP ? w * (D / 2) : 0; d < (GROUP && !w ? D / 2 : D); d += 32) {
                float o[32];
                __syncwarp();
                if (tiles > 0) {
                    tmem_ld32(tmem + lanes + 256 + rt * D + d, o);
                    tmem_wait_ld();
                }
                if (GROUP && tiles > 0) {
                    float low[32];
                    tmem_ld32(tmem + lanes + 256 + D + d, low);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] += fabsf(o[i]) < CUDART_INF_F ? low[i] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = tiles > 0 ? scaled(o[i], inv) : 0.0f;
                if (live && part_out) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        *reinterpret_cast<float4 *>(part_o + d + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                } else if (live) {
#pragma unroll
                    for (int i = 0; i < 32; i += 8)
                        *reinterpret_cast<uint4 *>(out + d + i) =
                            make_uint4(Elt<T>::pack(o[i], o[i + 1]), Elt<T>::pack(o[i + 2], o[i + 3]),
                                       Elt<T>::pack(o[i + 4], o[i + 5]), Elt<T>::pack(o[i + 6], o[i + 7]));
                }
            }
            if (live && part_out) {  // (both threads of a group's row write the same)
                p.part_ml[2 * pr] = m - RAISE;
                p.part_ml[2 * pr + 1] = l;
            } else if (live && p.lse) {
                p.lse[qt * p.H * p.G + hq] = l == 0.0f ? -CUDART_INF_F : (m - RAISE + log2f(l)) * LN2 - slope * (float)span.near;
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        const int loads = 2 * tiles;  // K0 V0 K1 V1 ...
        if (warp == 8 || warp == 10) {
            // ------------------------------------------------------------ blocks of keys (values) into the stages
            const int *table = p.tables + (long long)sq.ctx * p.max_blk;
            const int pages = WIDE_KEYS / p.BS, which = warp == 8 ? 0 : 1;
            bool ok = true;
            int at_end = 0;
            uint32_t largest = 0;
            // V tiles that not every row sees whole: rows that none sees become zeros, values that are not finite are noticed
            auto look = [&](int n) -> bool {
                const int stage = n % S::STAGES, tb = t0 + (n >> 1) * WIDE_KEYS;
                if (tb >= lo_max && tb + WIDE_KEYS <= hi_min && tb + WIDE_KEYS <= hi) return true;
                if (!warp_wait(full + 8 * stage, (n / S::STAGES) & 1, &sh_abort, p.status)) return false;
                const uint32_t v = sKV + stage * S::TILE_BYTES + lane * 16;
#pragma unroll 1
                for (int i = 0; i < S::TILE_BYTES / 16; i += 256) {  // eight pieces at a time, 32 token rows
                    const int ta = tb + ((i >> 3) & 127);
                    if (ta >= lo_max && ta + 32 <= hi_min) continue;  // every row sees these tokens
                    uint4 x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = lds16(v + (i + 32 * e) * 16);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int t = ta + e * 4 + (lane >> 3);
                        if (t < lo || t >= hi)
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(v + (i + 32 * e) * 16), "r"(0) : "memory");
                        else
                            largest = WideFormat<T>::larger(WideFormat<T>::larger(WideFormat<T>::larger(
                                WideFormat<T>::larger(largest, x[e].x), x[e].y), x[e].z), x[e].w);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) bar_arrive(guarded + 8 * stage);
                return true;
            };
            for (int n = which; n < loads; n += 2) {
                const int stage = n % S::STAGES, tb = t0 + (n >> 1) * WIDE_KEYS, at = tb + lane * p.BS;
                const bool mine = lane < pages && at < hi && at + p.BS > lo;
                const int slot = mine ? (2 * __ldg(table + block_of(at, p.BS, p.bs_shift)) + which) * p.BS : 0;
                if (n >= S::STAGES && !(ok = warp_wait(empty + 8 * stage, (n / S::STAGES - 1) & 1, &sh_abort, p.status))) break;
                const int count = __popc(__ballot_sync(0xffffffffu, mine));
                if (lane == 0) bar_expect(full + 8 * stage, (uint32_t)(count * p.BS * D * 2));
                __syncwarp();
                if (mine) {
                    const uint32_t dst = sKV + stage * S::TILE_BYTES + lane * p.BS * 128;
#pragma unroll
                    for (int h = 0; h < S::HALVES; ++h)
                        page_copy(dst + h * 16384, &map, full + 8 * stage, head * D + h * 64, slot, layer);
                }
                at_end = n + 2;
                if (which && n > 1 && !(ok = look(n - 2))) break;  // the tile before: it has had time to land
            }
            if (ok && which && loads > 0) ok = look(loads - 1);
            if (finite_only<T>(largest) != largest) *p.flag = p.epoch;
            // nothing may be in flight when the CTA ends early: wait for what was issued
            if (!ok)
                for (int n = max(which, at_end - 2 * S::STAGES); n < at_end; n += 2)
                    for (int i = 0; i < WAIT_LIMIT && !bar_try(full + 8 * (n % S::STAGES), (n / S::STAGES) & 1); ++i) {}
        } else if (warp == 9 || two) {
            // ------------------------------------------------------------ products, a warp for each row tile
            // The whole warp keeps the loop, one lane issues: addresses and descriptors are then the same in all lanes and
            // stay in uniform registers.  A wait costs some 300 cycles even where there is nothing to wait for, so the row tiles
            // do not share a warp.
            constexpr uint32_t F = WideFormat<T>::F;
            constexpr uint32_t QK = 1u << 4 | F << 7 | F << 10 | (WIDE_KEYS / 8) << 17 | (WIDE_TILE / 16) << 24;
            constexpr uint32_t PV = 1u << 4 | F << 7 | F << 10 | 1u << 16 | (D / 8) << 17 | (WIDE_TILE / 16) << 24;
            const int n_tile = __shfl_sync(0xffffffffu, tiles, 0), w = __shfl_sync(0xffffffffu, warp == 9 ? 0 : 1, 0);
            const uint64_t dQ = smem_desc(sQ, 16, 1024) + w * (S::TILE_BYTES >> 4), dK = smem_desc(sKV, 16, 1024), dV = smem_desc(sKV, 16384, 1024);
            const uint32_t tS = w * 128, tP = GROUP ? 128 : tS + 64, tO = 256 + w * D;
            auto scores = [&](int stage, bool release) {
                if (elected()) {
                    uint64_t a = dQ, b = dK + stage * (S::TILE_BYTES >> 4);
#pragma unroll
                    for (int h = 0; h < S::HALVES; ++h, a += 16384 >> 4, b += 16384 >> 4)
#pragma unroll
                        for (int k = 0; k < 4; ++k) mma_ss(tS, a + 2 * k, b + 2 * k, QK, h + k > 0);
                    mma_commit(s_full + 8 * w);
                    if (release) mma_commit(empty + 8 * stage);  // an arrival is asked for only where someone waits for it
                }
                __syncwarp();
            };
            bool ok = warp_wait(q_ready, 0, &sh_abort, p.status);
            uint32_t looked = 0;  // parity of every stage's `guarded`
            int sv = 1 % S::STAGES, pv = 0, sk = 2 % S::STAGES, pk = 0;  // stage and parity of V_j and of K_j+1
            if (ok && n_tile > 0 && (ok = warp_wait(full, 0, &sh_abort, p.status))) {
                tmem_after();
                scores(0, S::STAGES < loads);
            }
            for (int j = 0; ok && j < n_tile; ++j) {
                const bool more = j + 1 < n_tile;
                const int tb = t0 + j * WIDE_KEYS;
                if (!(ok = warp_wait(full + 8 * sv, pv, &sh_abort, p.status))) break;
                if (more && !(ok = warp_wait(full + 8 * sk, pk, &sh_abort, p.status))) break;
                if (tb < lo_max || tb + WIDE_KEYS > hi_min || tb + WIDE_KEYS > hi) {
                    if (!(ok = warp_wait(guarded + 8 * sv, looked >> sv & 1, &sh_abort, p.status))) break;
                    looked ^= 1u << sv;
                }
                const uint64_t b = dV + sv * (S::TILE_BYTES >> 4);
                // the row tiles take turns, else both would exponentiate, then both multiply at the same time
                if (two && (w || j) && !(ok = warp_wait(turn + 8 * w, w ? j & 1 : (j - 1) & 1, &sh_abort, p.status))) break;
                if (!(ok = warp_wait(p_ready + 8 * w, j & 1, &sh_abort, p.status))) break;
                tmem_after();
                if (!GROUP && elected()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_ts(tO, tP + 8 * k, b + k * (2048 >> 4), PV, j > 0 || k > 0);
                }
                __syncwarp();
                if (!(ok = warp_wait(p_rest + 8 * w, j & 1, &sh_abort, p.status))) break;
                tmem_after();
                if (elected()) {
#pragma unroll
                    for (int k = GROUP ? 0 : 4; k < 8; ++k) {  // a group's first half too: the second half's warps may still rescale outputs
                        mma_ts(tO, tP + 8 * k, b + k * (2048 >> 4), PV, j > 0 || k > 0);
                        if (GROUP) mma_ts(tO + D, tP + 64 + 8 * k, b + k * (2048 >> 4), PV, j > 0 || k > 0);
                    }
                    mma_commit(o_done + 8 * w);
                    if (2 * j + 1 + S::STAGES < loads) mma_commit(empty + 8 * sv);
                }
                __syncwarp();
                if (more) scores(sk, 2 * j + 2 + S::STAGES < loads);  // in order behind the product that still reads P from these columns
                if (two && lane == 0) bar_arrive(turn + 8 * (w ^ 1));
                sv += 2;
                if (sv >= S::STAGES) sv -= S::STAGES, pv ^= 1;
                sk += 2;
                if (sk >= S::STAGES) sk -= S::STAGES, pk ^= 1;
            }
        }
    }
    __syncthreads();
    if (sh_abort && (warp == 9 || warp == 11) && lane == 0) {
        // a wait gave up: let the products that were issued finish before tensor memory is given back
        const uint32_t bar = drain + (warp == 11 ? 8 : 0);
        mma_commit(bar);
        for (int i = 0; i < WAIT_LIMIT && !bar_try(bar, 0); ++i) {}
    }
    __syncthreads();
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sh_tmem));
}

bool wide_takes(int D, int BS) { return (D == 64 || D == 128) && BS >= 8 && BS <= WIDE_KEYS && (BS & (BS - 1)) == 0; }

template <typename T, int D, int MODE, bool GROUP>
static cudaError_t wide_go(const AttnParams &p, const SmallSeqs &small, const void *map, int layer, cudaStream_t st) {
    static SmemSeen seen{0};
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(attend_wide_kernel<T, D, MODE, GROUP>), WideShape<D>::SMEM, &seen);
    if (e != cudaSuccess) return e;
    attend_wide_kernel<T, D, MODE, GROUP><<<(unsigned)((long long)p.total_units * p.H), WIDE_THREADS, WideShape<D>::SMEM, st>>>(
        p, small, *static_cast<const CUtensorMap *>(map), layer);
    return cudaGetLastError();
}
template <typename T, int D, bool GROUP>
static cudaError_t wide_mode(const AttnParams &p, const SmallSeqs &small, const void *map, int layer, cudaStream_t st) {
    // a scale of zero would undo a mask (0 * -inf) where scores are multiples of the product
    if (p.slopes || p.scale == 0.0f) return wide_go<T, D, 2, GROUP>(p, small, map, layer, st);
    return p.softcap != 0.0f ? wide_go<T, D, 1, GROUP>(p, small, map, layer, st) : wide_go<T, D, 0, GROUP>(p, small, map, layer, st);
}
template <typename T> static cudaError_t wide_pick(const AttnParams &p, const SmallSeqs &small, bool groups, const void *map, int layer, cudaStream_t st) {
    if (p.D == 64) return groups ? wide_mode<T, 64, true>(p, small, map, layer, st) : wide_mode<T, 64, false>(p, small, map, layer, st);
    return groups ? wide_mode<T, 128, true>(p, small, map, layer, st) : wide_mode<T, 128, false>(p, small, map, layer, st);
}
cudaError_t launch_attend_wide(const AttnParams &p, const SmallSeqs &small, int f16, bool groups, const void *map, int layer, cudaStream_t st) {
    return f16 ? wide_pick<__half>(p, small, groups, map, layer, st) : wide_pick<__nv_bfloat16>(p, small, groups, map, layer, st);
}

// Tensor map of a whole pool: [layer][slot of a block's keys or values][kv head and dim], boxes of a block's slots, 64 dims.
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
    const cuuint64_t dims[3] = {(cuuint64_t)g.H * g.D, 2 * (cuuint64_t)g.NB * g.BS, (cuuint64_t)g.L};
    const cuuint64_t strides[2] = {(cuuint64_t)g.row, (cuuint64_t)g.layer_stride};
    const cuuint32_t box[3] = {64, (cuuint32_t)g.BS, 1}, step[3] = {1, 1, 1};
    if (dims[1] >= (1ull << 31)) return false;
    return reinterpret_cast<Encode>(fn)(reinterpret_cast<CUtensorMap *>(out), CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, g.pool, dims, strides,
                                        box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace aafkv
