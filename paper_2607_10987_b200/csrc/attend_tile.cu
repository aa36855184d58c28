// Attention of many query rows per kv head over paged keys and values, 64 rows a CTA, any head width up to 256.
//
// The query heads that share a kv head are packed with the query tokens into the rows of one product (row = token * G +
// head of the group), so a shared key is read once for all of them.  A CTA walks the keys that any of its rows sees
// in tiles of 64 tokens: S = Q K^T, running maximum and sum per row, O += P V, all accumulators in registers; tiles
// of K and V come through the block table with 16-byte asynchronous copies into two swizzled shared-memory stages.
// When there are few row tiles the key range is cut into parts that attend_join adds up.
//
// P is rounded to the values' 16-bit type before P V: the error is that of one more rounding of the output's kind
// (each weight is off by at most half a step, the signs are independent), the sum of the weights stays in 32 bits.
//
// Bound: the issue of copies, ldmatrix and mma.sync by four warps.  4 contexts of 8699 tokens, 512 of them new, 32 heads, 8 kv
// heads: 96 wide 2962 us (72 TFLOP/s), 256 wide 9594 (59).
#include "attend_device.cuh"

namespace aafkv {

constexpr int TILE_WARPS = 4, TILE_KEYS = 64;

template <int DP> struct TileShape {
    static constexpr int ROW = DP * 2, CH = DP / 8;          // bytes and 16-byte pieces of a shared-memory row
    static constexpr int KV_BYTES = TILE_KEYS * ROW;         // one tile of K or V
    static constexpr int Q_BYTES = TILE_ROWS * ROW;
    static constexpr int SMEM = Q_BYTES + 4 * KV_BYTES;
    static constexpr bool Q_IN_REGS = DP <= 128;
};
// 16-byte piece c of row r: the piece index is XORed with the row so that eight rows of one column hit eight bank groups
template <int DP> __device__ __forceinline__ uint32_t swz(int r, int c) {
    return (uint32_t)(r * (DP * 2) + ((c ^ (r & 7)) << 4));
}

template <typename T, int DP>
__global__ void __launch_bounds__(TILE_WARPS * 32)
    attend_tile_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ SmallSeqs small) {
    using S = TileShape<DP>;
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t4 = lane & 3;
    asm volatile("griddepcontrol.launch_dependents;");
    if (p.flag && *p.flag != p.epoch) return;  // a second run that is not needed
    for (long long cta = blockIdx.x; cta < (long long)p.total_units * p.H; cta += gridDim.x) {
    const int unit = (int)(cta / p.H), head = (int)(cta - (long long)unit * p.H);
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq sq = seqs[find_seq(seqs, p.n, unit)];
    const int R = sq.nq * p.G, n_tiles = (R + TILE_ROWS - 1) / TILE_ROWS;
    const int u = unit - sq.unit0, part = u % sq.nsplit;
    const int tile = n_tiles - 1 - u / sq.nsplit;  // the latest rows see the most keys: they start first
    const int r0 = tile * TILE_ROWS;

    // keys that the CTA's rows see
    const int j0 = r0 / p.G, j1 = min(R - 1, r0 + TILE_ROWS - 1) / p.G;
    int lo = 0x7fffffff, hi = 0;
    for (int j = j0 + lane; j <= j1; j += 32) {
        const RowSpan sp = row_span(p, sq, j);
        if (sp.hi > sp.lo) {
            lo = min(lo, sp.lo);
            hi = max(hi, sp.hi);
        }
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    if (sq.nsplit > 1 && hi > lo) {
        const int chunk = ((hi - lo + sq.nsplit - 1) / sq.nsplit + TILE_KEYS - 1) / TILE_KEYS * TILE_KEYS;
        const long long b = lo + (long long)part * chunk;
        hi = (int)min((long long)hi, b + chunk);
        lo = (int)min(b, (long long)hi);
    }
    const int tiles = hi > lo ? (hi - lo + TILE_KEYS - 1) / TILE_KEYS : 0;

    const uint32_t sQ = (uint32_t)__cvta_generic_to_shared(smem), sK = sQ + S::Q_BYTES, sV = sK + 2 * S::KV_BYTES;
    const int *table = p.tables + (long long)sq.ctx * p.max_blk;
    const char *kb = p.kbase + (long long)head * p.D * 2;

    for (int i = threadIdx.x; i < TILE_ROWS * S::CH; i += TILE_WARPS * 32) {
        const int r = i / S::CH, c = i % S::CH, rr = r0 + r;
        const bool in = rr < R && c * 8 < p.D;
        const T *q = static_cast<const T *>(p.q) + (long long)(sq.row0 + min(rr, R - 1) / p.G) * p.q_stride +
                     (long long)(head * p.G + min(rr, R - 1) % p.G) * p.D + c * 8;
        copy16(sQ + swz<DP>(r, c), in ? q : static_cast<const T *>(p.q), in ? 16 : 0);
    }
    auto load_tile = [&](int it) {
        if (it < tiles) {
            const uint32_t k = sK + (it & 1) * S::KV_BYTES, v = sV + (it & 1) * S::KV_BYTES;
            for (int i = threadIdx.x; i < TILE_KEYS * S::CH; i += TILE_WARPS * 32) {
                const int r = i / S::CH, c = i % S::CH, t = lo + it * TILE_KEYS + r;
                const bool in = t < hi && c * 8 < p.D;
                const char *src = kb;
                if (in) {
                    const int b = block_of(t, p.BS, p.bs_shift);
                    src += (long long)__ldg(table + b) * 2 * p.run + (long long)(t - b * p.BS) * p.row + c * 16;
                }
                copy16(k + swz<DP>(r, c), src, in ? 16 : 0);
                copy16(v + swz<DP>(r, c), in ? src + p.run : src, in ? 16 : 0);
            }
        }
        copy_commit();
    };
    load_tile(0);

    // the two rows of this lane (g and g + 8 of the warp's 16) and what the warp's rows have in common
    RowSpan span[2];
    float slope[2];
    int lo_max = 0, hi_min = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int rr = min(r0 + warp * 16 + g + 8 * i, R - 1);
        span[i] = row_span(p, sq, rr / p.G);
        slope[i] = p.slopes ? p.slopes[head * p.G + rr % p.G] : 0.0f;
        lo_max = max(lo_max, span[i].lo);
        hi_min = min(hi_min, span[i].hi);
    }
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
        lo_max = max(lo_max, __shfl_xor_sync(0xffffffffu, lo_max, d));
        hi_min = min(hi_min, __shfl_xor_sync(0xffffffffu, hi_min, d));
    }

    float o[DP / 8][4];
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    float m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.0f, 0.0f};
    uint32_t qf[S::Q_IN_REGS ? DP / 16 : 1][4];
    auto load_q = [&](uint32_t(&f)[4], int ks) {
        ldmatrix4(f, sQ + swz<DP>(warp * 16 + (lane & 15), ks * 2 + (lane >> 4)));
    };

    for (int it = 0; it < tiles; ++it) {
        load_tile(it + 1);
        copy_wait<1>();
        __syncthreads();
        if (S::Q_IN_REGS && it == 0) {
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks) load_q(qf[S::Q_IN_REGS ? ks : 0], ks);
        }
        const uint32_t k = sK + (it & 1) * S::KV_BYTES, v = sV + (it & 1) * S::KV_BYTES;
        float s[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) {
            uint32_t a[4];
            if (S::Q_IN_REGS) {
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] = qf[S::Q_IN_REGS ? ks : 0][i];
            } else {
                load_q(a, ks);
            }
#pragma unroll
            for (int nt = 0; nt < 8; nt += 2) {  // matrices: keys nt*8.. k-half 0, 1; keys nt*8+8.. k-half 0, 1
                uint32_t b[4];
                ldmatrix4(b, k + swz<DP>(nt * 8 + (lane >> 4) * 8 + (lane & 7), ks * 2 + ((lane >> 3) & 1)));
                Elt<T>::mma(s[nt], a[0], a[1], a[2], a[3], b[0], b[1]);
                Elt<T>::mma(s[nt + 1], a[0], a[1], a[2], a[3], b[2], b[3]);
            }
        }
        const int tb = lo + it * TILE_KEYS;
        const bool full = lo_max <= tb && hi_min >= tb + TILE_KEYS && hi >= tb + TILE_KEYS;
        bool partial = false;  // some row misses a key that another of the CTA's rows may see
        float mx[2] = {-CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = tb + i * 8 + 2 * t4 + (e & 1), h = e >> 1;
                float x = score2(p, s[i][e], slope[h], span[h], t);
                if (!full) {
                    const bool see = t >= span[h].lo && t < span[h].hi && t < hi;
                    partial |= !see && t < hi;
                    x = see ? x : -CUDART_INF_F;
                }
                s[i][e] = x;
                mx[h] = fmaxf(mx[h], x);
            }
        float base[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
            const float n = fmaxf(m[h], mx[h]);
            const float a = n == -CUDART_INF_F ? 1.0f : ex2(m[h] - n);
            l[h] *= a;
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) {
                o[i][2 * h] *= a;
                o[i][2 * h + 1] *= a;
            }
            m[h] = n;
            base[h] = n == -CUDART_INF_F ? 0.0f : n - Elt<T>::RAISE;
        }
        partial = !full && __any_sync(0xffffffffu, partial);
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {  // 16 keys
            uint32_t a[4], vis[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float(&x)[4] = s[2 * kt + i];
                if (partial) {
                    const uint32_t one = Elt<T>::ONE;
                    vis[2 * i] = (x[0] != -CUDART_INF_F ? one : 0u) | (x[1] != -CUDART_INF_F ? one << 16 : 0u);
                    vis[2 * i + 1] = (x[2] != -CUDART_INF_F ? one : 0u) | (x[3] != -CUDART_INF_F ? one << 16 : 0u);
                }
                const float p0 = ex2(x[0] - base[0]), p1 = ex2(x[1] - base[0]), p2 = ex2(x[2] - base[1]), p3 = ex2(x[3] - base[1]);
                l[0] += p0 + p1;
                l[1] += p2 + p3;
                a[2 * i] = Elt<T>::pack(p0, p1);
                a[2 * i + 1] = Elt<T>::pack(p2, p3);
            }
#pragma unroll
            for (int dt = 0; dt < DP / 8; dt += 2) {  // matrices: key halves 0, 1 of dims dt*8.., then of dims dt*8+8..
                uint32_t b[4];
                ldmatrix4t(b, v + swz<DP>(kt * 16 + (lane & 15), dt + (lane >> 4)));
                if (partial) {
                    uint32_t f[4];
                    bool odd = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        f[i] = finite_only<T>(b[i]);
                        odd |= f[i] != b[i];
                    }
                    if (__any_sync(0xffffffffu, odd)) {
                        add4(o[dt], nonfinite_b<T>(vis[0], vis[1], vis[2], vis[3], b[0], b[1]));
                        add4(o[dt + 1], nonfinite_b<T>(vis[0], vis[1], vis[2], vis[3], b[2], b[3]));
#pragma unroll
                        for (int i = 0; i < 4; ++i) b[i] = f[i];
                    }
                }
                Elt<T>::mma(o[dt], a[0], a[1], a[2], a[3], b[0], b[1]);
                Elt<T>::mma(o[dt + 1], a[0], a[1], a[2], a[3], b[2], b[3]);
            }
        }
        __syncthreads();  // everyone is done with this stage before it is loaded again
    }
    copy_wait<0>();

#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float sum = l[h];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        const int rl = warp * 16 + g + 8 * h, rr = r0 + rl;
        if (rr >= R) continue;
        if (sq.part0 >= 0) {
            const long long pr = sq.part0 + (((long long)tile * sq.nsplit + part) * p.H + head) * TILE_ROWS + rl;
            const float some = sum == 0.0f ? 0.0f : 1.0f;
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) {
                const int d = i * 8 + 2 * t4;
                if (d < p.D)
                    *reinterpret_cast<float2 *>(p.part_o + pr * p.D + d) = make_float2(scaled(o[i][2 * h], some), scaled(o[i][2 * h + 1], some));
            }
            if (t4 == 0) {
                p.part_ml[2 * pr] = m[h] - Elt<T>::RAISE;
                p.part_ml[2 * pr + 1] = sum;
            }
            continue;
        }
        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;  // a row that sees nothing is zero
        const long long qt = sq.row0 + rr / p.G;
        const int hq = head * p.G + rr % p.G;
        T *out = static_cast<T *>(p.out) + (qt * p.H * p.G + hq) * p.D;
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
            const int d = i * 8 + 2 * t4;
            if (d < p.D) *reinterpret_cast<uint32_t *>(out + d) = Elt<T>::pack(scaled(o[i][2 * h], inv), scaled(o[i][2 * h + 1], inv));
        }
        if (p.lse && t4 == 0)
            p.lse[qt * p.H * p.G + hq] =
                sum == 0.0f ? -CUDART_INF_F : (m[h] - Elt<T>::RAISE + log2f(sum)) * LN2 - slope[h] * (float)span[h].near;
    }
    __syncthreads();  // the next unit loads over this one's tiles
    }
}

template <typename T, int DP> static cudaError_t tile_go(const AttnParams &p, const SmallSeqs &small, int sm_count, cudaStream_t st) {
    static SmemSeen seen{0};
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(attend_tile_kernel<T, DP>), TileShape<DP>::SMEM, &seen);
    if (e != cudaSuccess) return e;
    long long ctas = (long long)p.total_units * p.H;
    if (p.flag) ctas = min(ctas, 2ll * sm_count);  // what the GPU holds at once: most often they return at once
    attend_tile_kernel<T, DP><<<(unsigned)ctas, TILE_WARPS * 32, TileShape<DP>::SMEM, st>>>(p, small);
    return cudaGetLastError();
}
template <typename T> static cudaError_t tile_pick(const AttnParams &p, const SmallSeqs &small, int sm_count, cudaStream_t st) {
    if (p.D <= 64) return tile_go<T, 64>(p, small, sm_count, st);
    if (p.D <= 128) return tile_go<T, 128>(p, small, sm_count, st);
    return tile_go<T, 256>(p, small, sm_count, st);
}
cudaError_t launch_attend_tile(const AttnParams &p, const SmallSeqs &small, int f16, int sm_count, cudaStream_t st) {
    return f16 ? tile_pick<__half>(p, small, sm_count, st) : tile_pick<__nv_bfloat16>(p, small, sm_count, st);
}

}  // namespace aafkv
