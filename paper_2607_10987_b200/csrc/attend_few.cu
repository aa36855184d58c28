// Attention of a few query rows per kv head (one new token per sequence, or a handful) over paged keys and values.
//
//   s_rt = score(q_r . k_t),  o_r = sum_t exp(s_rt) v_t / sum_t exp(s_rt),  lse_r = log sum_t exp(s_rt)
//
// One pass over K and V with the running maximum m and sum l of every row; the key range of a sequence is cut into
// parts, each part leaves (m, l, o) and attend_join adds them up in part order, so results do not depend on timing.
//
// Bound: every cached row is used by at most 8 * NT query rows, so the bytes of K and V decide.  A warp owns one kv
// head of one part and shares nothing with the others: no barrier, only warps that wait for their own copies (cp.async,
// several tiles of 16 tokens in flight; a copy instruction covers whole rows, 256 contiguous bytes at 128 dims).
// The tensor products take the tokens as the M side (16) and the query rows as the N side (8): S^T = K Q^T and
// O^T = V^T P^T waste nothing for 8 rows, where rows as M would fill half a tile at best.  The order of the head
// dimensions inside a product is free as long as both operands agree, and so is the order of the output rows: lane
// (g, t) takes 8 consecutive dimensions of token g for K, and of tokens 2t, 2t+1, 2t+8, 2t+9 for V, whose pairs two
// byte permutes bring together; the 16-byte pieces of a row are stored so that neither pattern meets a bank twice.
//
// P is split into two 16-bit parts (p = hi + lo) and multiplied twice: the tensor pipe is idle anyway and the result
// then carries the output's own rounding only.
//
// 64 ragged contexts, 780 MB of keys and values: 145 us with the join (5.4 TB/s); one of 33787 tokens, 138 MB: 33.7.
#include "sparse_device.cuh"

namespace aafkv {

template <int DP> struct FewShape {
    static constexpr int PIECES = DP / 8;           // 16-byte pieces of a row
    static constexpr int ROW = DP * 2, HALF = 16 * ROW;  // bytes of a row, of a tile of 16 keys (or values)
    static constexpr int STAGE_BYTES = 2 * HALF;
    static constexpr int WARPS = DP <= 128 ? 4 : 3;
    static constexpr int STAGES = DP == 64 ? 6 : (DP == 128 ? 3 : 2);
    static constexpr int SMEM = WARPS * STAGES * STAGE_BYTES;  // 96 KB: two CTAs an SM, one starts while the other streams
    static_assert(2 * (SMEM + 1024) <= 228 * 1024, "shared memory of a CTA");
};

// SIMPLE: one query token a sequence, no cap, bias or spans: every row sees every key of its part, a score is a multiple of the
// product.  Two in five instructions of a tile go into the general case (486 at 128 dims).
template <typename T, int DP, int NT, bool SIMPLE>
__global__ void __launch_bounds__(FewShape<DP>::WARPS * 32, 2)
    attend_few_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ SmallSeqs small) {
    using S = FewShape<DP>;
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t4 = lane & 3;
    const long long task = (long long)blockIdx.x * S::WARPS + warp;
    if (task >= (long long)p.total_units * p.H) return;
    const int unit = (int)(task / p.H), head = (int)(task - (long long)unit * p.H);
    asm volatile("griddepcontrol.launch_dependents;");  // the join may be brought up beside this kernel
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq sq = seqs[find_seq(seqs, p.n, unit)];
    const int part = unit - sq.unit0;
    const int R = sq.nq * p.G;

    // rows of this lane: columns 2 t4, 2 t4 + 1 of every n-tile
    RowSpan span[SIMPLE ? 1 : NT][2];
    float slope[SIMPLE ? 1 : NT][2];
    int lo_all = SIMPLE ? 0 : 0x7fffffff, hi_all = SIMPLE ? sq.len : 0;
    if (!SIMPLE) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int r = nt * 8 + 2 * t4 + c;
            RowSpan &sp = span[SIMPLE ? 0 : nt][c];
            sp = row_span(p, sq, min(r, R - 1) / p.G);
            slope[SIMPLE ? 0 : nt][c] = p.slopes ? p.slopes[head * p.G + min(r, R - 1) % p.G] : 0.0f;
            if (sp.hi > sp.lo) {
                lo_all = min(lo_all, sp.lo);
                hi_all = max(hi_all, sp.hi);
            }
        }
#pragma unroll
    for (int d = 1; d < 4; d <<= 1) {
        lo_all = min(lo_all, __shfl_xor_sync(0xffffffffu, lo_all, d));
        hi_all = max(hi_all, __shfl_xor_sync(0xffffffffu, hi_all, d));
    }
    }
    // the part's keys: the host cut [key0, len) into chunks
    const long long c0 = sq.key0 + (long long)part * sq.chunk;
    int beg = (int)max((long long)lo_all, c0), end = (int)min((long long)hi_all, c0 + sq.chunk);
    if (end <= beg) beg = end = 0;  // nothing to see in this part: no token index is formed from an empty range
    const int tiles = (end - beg + 15) / 16;

    const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem) + warp * (S::STAGES * S::STAGE_BYTES);
    // where piece c of row r lies: lanes that read together have two rows and four pieces of K, four even (odd) rows and two
    // pieces of V
    auto k_at = [](int r, int c) { return (uint32_t)(r * S::ROW + ((c ^ ((r & 1) << 2)) << 4)); };
    auto v_at = [](int r, int c) { return (uint32_t)(S::HALF + r * S::ROW + ((c ^ (r & 6)) << 4)); };
    const int *table = p.tables + (long long)sq.ctx * p.max_blk;
    const char *kb = p.kbase + (long long)head * p.D * 2;

    auto table_id = [&](int tile) -> int {  // lane l: block of the tile's token l % 16
        const int t = beg + tile * 16 + (lane & 15);
        return t < end ? __ldg(table + block_of(t, p.BS, p.bs_shift)) : 0;
    };
    auto issue = [&](int tile, int id) {
        if (tile < tiles) {
            const int tm = beg + tile * 16 + (lane & 15);
            const int b = block_of(tm, p.BS, p.bs_shift);
            const long long off = (long long)id * 2 * p.run + (long long)(tm - b * p.BS) * p.row;
            const uint32_t st = base + (tile % S::STAGES) * S::STAGE_BYTES;
            constexpr int AT_ONCE = 32 / S::PIECES;  // rows of one copy instruction
            const int c = lane % S::PIECES;
#pragma unroll
            for (int i = 0; i < 16 / AT_ONCE; ++i) {
                const int r = i * AT_ONCE + lane / S::PIECES;
                const char *src = kb + __shfl_sync(0xffffffffu, off, r) + c * 16;
                const bool in = beg + tile * 16 + r < end && c * 8 < p.D;
                copy16(st + k_at(r, c), in ? src : kb, in ? 16 : 0);
                copy16(st + v_at(r, c), in ? src + p.run : kb, in ? 16 : 0);
            }
        }
        copy_commit();
    };

    int id = table_id(0);
#pragma unroll
    for (int s = 0; s < S::STAGES; ++s) {
        const int nxt = table_id(s + 1);
        issue(s, id);
        id = nxt;
    }

    // query fragments: row nt * 8 + g, 8 dimensions at kk * 32 + t4 * 8
    uint4 qf[NT][DP / 32];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 8 + g;
        const T *q = static_cast<const T *>(p.q) + (long long)(sq.row0 + min(r, R - 1) / p.G) * p.q_stride +
                     (long long)(head * p.G + min(r, R - 1) % p.G) * p.D;
#pragma unroll
        for (int kk = 0; kk < DP / 32; ++kk) {
            const int d = kk * 32 + t4 * 8;
            qf[nt][kk] = r < R && d < p.D ? __ldg(reinterpret_cast<const uint4 *>(q + d)) : make_uint4(0, 0, 0, 0);
        }
    }

    const float c2 = p.scale * LOG2E;
    float o[NT][DP / 16][4];
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = -CUDART_INF_F;
        l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.0f;
    }

    for (int tile = 0; tile < tiles; ++tile) {
        copy_wait<S::STAGES - 1>();
        __syncwarp();  // every lane's pieces have landed
        const uint32_t st = base + (tile % S::STAGES) * S::STAGE_BYTES;
        const int tb = beg + tile * 16;
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < DP / 32; ++kk) {
            const uint4 w = lds16(st + k_at(g, kk * 4 + t4)), x = lds16(st + k_at(g + 8, kk * 4 + t4));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                Elt<T>::mma(s[nt], w.x, x.x, w.y, x.y, qf[nt][kk].x, qf[nt][kk].y);
                Elt<T>::mma(s[nt], w.z, x.z, w.w, x.w, qf[nt][kk].z, qf[nt][kk].w);
            }
        }
        uint32_t ph[NT][2], pl[NT][2], vis[NT][2];
        bool partial = false;  // some row misses a token of the tile that is within the part
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mx[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int t = tb + g + 8 * h;
                    float &x = s[nt][2 * h + c];
                    if (SIMPLE) {
                        x = t < end ? x * c2 : -CUDART_INF_F;
                    } else {
                        const RowSpan &sp = span[SIMPLE ? 0 : nt][c];
                        const bool see = t >= sp.lo && t < sp.hi && t < end;
                        partial |= !see && t < end;
                        x = see ? score2(p, x, slope[SIMPLE ? 0 : nt][c], sp, t) : -CUDART_INF_F;
                    }
                }
                mx[c] = fmaxf(s[nt][c], s[nt][2 + c]);
            }
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) {
                mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], d));
                mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], d));
            }
            const float n0 = fmaxf(m[nt][0], mx[0]), n1 = fmaxf(m[nt][1], mx[1]);
            if (__any_sync(0xffffffffu, n0 > m[nt][0] || n1 > m[nt][1])) {  // a new maximum: rescale what is summed
                const float a0 = n0 == -CUDART_INF_F ? 1.0f : ex2(m[nt][0] - n0);
                const float a1 = n1 == -CUDART_INF_F ? 1.0f : ex2(m[nt][1] - n1);
                l[nt][0] *= a0;
                l[nt][1] *= a1;
#pragma unroll
                for (int i = 0; i < DP / 16; ++i) {
                    o[nt][i][0] *= a0;
                    o[nt][i][1] *= a1;
                    o[nt][i][2] *= a0;
                    o[nt][i][3] *= a1;
                }
                m[nt][0] = n0;
                m[nt][1] = n1;
            }
            const float b0 = n0 == -CUDART_INF_F ? 0.0f : n0 - Elt<T>::RAISE, b1 = n1 == -CUDART_INF_F ? 0.0f : n1 - Elt<T>::RAISE;
            const float p0 = ex2(s[nt][0] - b0), p1 = ex2(s[nt][1] - b1);
            const float p2 = ex2(s[nt][2] - b0), p3 = ex2(s[nt][3] - b1);
            l[nt][0] += p0 + p2;
            l[nt][1] += p1 + p3;
            const uint32_t h01 = Elt<T>::pack(p0, p1), h23 = Elt<T>::pack(p2, p3);
            const uint32_t l01 = Elt<T>::pack(p0 - Elt<T>::lo(h01), p1 - Elt<T>::hi(h01));
            const uint32_t l23 = Elt<T>::pack(p2 - Elt<T>::lo(h23), p3 - Elt<T>::hi(h23));
            ph[nt][0] = transpose8x8(h01);
            ph[nt][1] = transpose8x8(h23);
            pl[nt][0] = transpose8x8(l01);
            pl[nt][1] = transpose8x8(l23);
            if (SIMPLE) continue;
            const uint32_t one = Elt<T>::ONE;
            vis[nt][0] = (s[nt][0] != -CUDART_INF_F ? one : 0u) | (s[nt][1] != -CUDART_INF_F ? one << 16 : 0u);
            vis[nt][1] = (s[nt][2] != -CUDART_INF_F ? one : 0u) | (s[nt][3] != -CUDART_INF_F ? one << 16 : 0u);
        }
        partial = !SIMPLE && __any_sync(0xffffffffu, partial);
#pragma unroll
        for (int c = 0; c < DP / 64; ++c) {
            uint4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = lds16(st + v_at(2 * t4 + (i & 1) + (i >> 1) * 8, c * 8 + g));
            const uint32_t w0[4] = {v[0].x, v[0].y, v[0].z, v[0].w}, w1[4] = {v[1].x, v[1].y, v[1].z, v[1].w};
            const uint32_t w2[4] = {v[2].x, v[2].y, v[2].z, v[2].w}, w3[4] = {v[3].x, v[3].y, v[3].z, v[3].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t a[4] = {prmt(w0[j], w1[j], 0x5410), prmt(w0[j], w1[j], 0x7632), prmt(w2[j], w3[j], 0x5410),
                                 prmt(w2[j], w3[j], 0x7632)};
                if (partial) {
                    uint32_t f[4];
                    bool odd = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        f[i] = finite_only<T>(a[i]);
                        odd |= f[i] != a[i];
                    }
                    if (__any_sync(0xffffffffu, odd)) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            add4(o[nt][4 * c + j],
                                 nonfinite_a<T>(a[0], a[1], a[2], a[3], transpose8x8(vis[nt][0]), transpose8x8(vis[nt][1])));
#pragma unroll
                        for (int i = 0; i < 4; ++i) a[i] = f[i];
                    }
                }
                // An infinite value times the high part of its weight is infinite; times the low part, which may be zero or
                // negative, it would make a NaN of that: there it is the type's largest value.
                uint32_t b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = Elt<T>::bounded(a[i]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    Elt<T>::mma(o[nt][4 * c + j], a[0], a[1], a[2], a[3], ph[nt][0], ph[nt][1]);
                    Elt<T>::mma(o[nt][4 * c + j], b[0], b[1], b[2], b[3], pl[nt][0], pl[nt][1]);
                }
            }
        }
        const int nxt = table_id(tile + S::STAGES + 1);
        __syncwarp();  // every lane has read this stage
        issue(tile + S::STAGES, id);
        id = nxt;
    }
    copy_wait<0>();

#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float sum = l[nt][c];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            const int r = nt * 8 + 2 * t4 + c;
            if (r >= R) continue;
            if (sq.part0 >= 0) {  // a part of a longer range: (m, l, o) for the join
                const float some = sum == 0.0f ? 0.0f : 1.0f;
                const long long pr = sq.part0 + ((long long)part * p.H + head) * R + r;
#pragma unroll
                for (int cc = 0; cc < DP / 64; ++cc) {
                    const int d = cc * 64 + g * 8;
                    if (d >= p.D) continue;
                    float4 *dst = reinterpret_cast<float4 *>(p.part_o + pr * p.D + d);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        dst[i] = make_float4(scaled(o[nt][4 * cc + 2 * i][c], some), scaled(o[nt][4 * cc + 2 * i][2 + c], some),
                                             scaled(o[nt][4 * cc + 2 * i + 1][c], some), scaled(o[nt][4 * cc + 2 * i + 1][2 + c], some));
                }
                if (g == 0) {
                    p.part_ml[2 * pr] = m[nt][c] - Elt<T>::RAISE;
                    p.part_ml[2 * pr + 1] = sum;
                }
                continue;
            }
            const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;  // a row that sees nothing is zero
            const long long qt = sq.row0 + r / p.G;
            const int hq = head * p.G + r % p.G;
            T *out = static_cast<T *>(p.out) + (qt * p.H * p.G + hq) * p.D;
#pragma unroll
            for (int cc = 0; cc < DP / 64; ++cc) {
                const int d = cc * 64 + g * 8;
                if (d >= p.D) continue;
                uint4 w;
                w.x = Elt<T>::pack(scaled(o[nt][4 * cc][c], inv), scaled(o[nt][4 * cc][2 + c], inv));
                w.y = Elt<T>::pack(scaled(o[nt][4 * cc + 1][c], inv), scaled(o[nt][4 * cc + 1][2 + c], inv));
                w.z = Elt<T>::pack(scaled(o[nt][4 * cc + 2][c], inv), scaled(o[nt][4 * cc + 2][2 + c], inv));
                w.w = Elt<T>::pack(scaled(o[nt][4 * cc + 3][c], inv), scaled(o[nt][4 * cc + 3][2 + c], inv));
                *reinterpret_cast<uint4 *>(out + d) = w;
            }
            if (p.lse && g == 0)
                p.lse[qt * p.H * p.G + hq] =
                    sum == 0.0f ? -CUDART_INF_F
                                : (m[nt][c] - Elt<T>::RAISE + log2f(sum)) * LN2 - (SIMPLE ? 0.0f : slope[SIMPLE ? 0 : nt][c] * (float)span[SIMPLE ? 0 : nt][c].near);
        }
    asm volatile("griddepcontrol.wait;" ::: "memory");  // what it ran beside is done before it is
}

// As many rows as a lane's registers hold accumulators for; up to there this kernel is ahead of the ones for many rows.  16 contexts
// of 3300 tokens, 8 kv heads, here and there: 64 wide, 8 rows 32.0 and 47.8 us, 32 rows 45.7 and 47.8; 128 wide, 8 rows 43.8 and
// 54.1, 16 rows 47.5 and 54.0; 256 wide, 8 rows 94 and 592.  One context of 32768 tokens: 64 wide, 32 rows 33.4 and 35.5; 128 wide, 16
// rows 36.3 and 41.8.
int few_rows_limit(int D) { return D <= 64 ? 32 : (D <= 128 ? 16 : 8); }

template <typename T, int DP, int NT, bool SIMPLE>
static cudaError_t few_go(const AttnParams &p, const SmallSeqs &small, bool beside, cudaStream_t st) {
    static SmemSeen seen{0};
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(attend_few_kernel<T, DP, NT, SIMPLE>), FewShape<DP>::SMEM, &seen);
    if (e != cudaSuccess) return e;
    constexpr int W = FewShape<DP>::WARPS;
    const long long tasks = (long long)p.total_units * p.H;
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((tasks + W - 1) / W));
    cfg.blockDim = dim3(W * 32);
    cfg.dynamicSmemBytes = FewShape<DP>::SMEM;
    cfg.stream = st;
    cfg.attrs = &early;
    cfg.numAttrs = beside ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, attend_few_kernel<T, DP, NT, SIMPLE>, p, small);
    return e != cudaSuccess ? e : cudaGetLastError();
}
template <typename T, int DP, int NT>
static cudaError_t few_kind(const AttnParams &p, const SmallSeqs &small, bool simple, bool beside, cudaStream_t st) {
    return simple ? few_go<T, DP, NT, true>(p, small, beside, st) : few_go<T, DP, NT, false>(p, small, beside, st);
}
template <typename T>
static cudaError_t few_pick(const AttnParams &p, const SmallSeqs &small, int max_rows, bool single, bool beside, cudaStream_t st) {
    const bool simple = single && p.softcap == 0.0f && !p.slopes && !p.spans;
    if (p.D <= 64)
        return max_rows <= 8 ? few_kind<T, 64, 1>(p, small, simple, beside, st)
                             : (max_rows <= 16 ? few_kind<T, 64, 2>(p, small, simple, beside, st) : few_kind<T, 64, 4>(p, small, simple, beside, st));
    if (p.D <= 128) return max_rows <= 8 ? few_kind<T, 128, 1>(p, small, simple, beside, st) : few_kind<T, 128, 2>(p, small, simple, beside, st);
    return few_kind<T, 256, 1>(p, small, simple, beside, st);
}
cudaError_t launch_attend_few(const AttnParams &p, const SmallSeqs &small, int f16, int max_rows, bool single, bool beside,
                              cudaStream_t st) {
    return f16 ? few_pick<__half>(p, small, max_rows, single, beside, st) : few_pick<__nv_bfloat16>(p, small, max_rows, single, beside, st);
}

// ------------------------------------------------------------------------------------------ join
// Adds up the parts of a split row: o = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s.  SPREAD warps work on a query token's
// head, each with every SPREAD-th part, four dimensions a lane; a warp keeps its own running maximum and sum, and the
// warps meet once, in shared memory, in warp order.  Bound: latency (a trip to L2 for the parts' maxima and outputs, both asked for
// at once), which is why there are as many warps a row as fill the GPU.  64 rows of 141 parts, 4.6 MB: 9 us by itself, some 6 behind
// the kernel that it is brought up beside.
constexpr int JOIN_WARPS = 8, JOIN_AHEAD = 8;
template <typename T, int SPREAD>
__global__ void __launch_bounds__(JOIN_WARPS * 32)
    attend_join_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ SmallSeqs small, int tile_rows, int rows) {
    __shared__ float4 acc_s[JOIN_WARPS][2][32];
    __shared__ float sum_s[JOIN_WARPS], max_s[JOIN_WARPS];
    const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) % SPREAD, team = (threadIdx.x >> 5) / SPREAD;
    const int out_row = blockIdx.x * (JOIN_WARPS / SPREAD) + team;
    if (out_row >= rows) return;  // a whole team: only its own warps meet
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const int Hq = p.H * p.G;
    const int tok = out_row / Hq, hq = out_row - tok * Hq, head = hq / p.G;
    int lo = 0, hi = p.n - 1;  // record of the query token
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (seqs[mid].tok0 <= tok) lo = mid; else hi = mid - 1;
    }
    const AttnSeq sq = seqs[lo];
    if (sq.part0 < 0) return;
    const long long qt = sq.row0 + (tok - sq.tok0);
    const int j = (int)(qt - sq.row0), r = j * p.G + hq % p.G;
    // partial rows of a sequence: [part][head][R] for the few-row kernel, [tile][part][head][tile_rows] for the others; behind
    // them in order the parts of the keys that its group shares
    long long row, step, grow = 0, gstep = 0;
    if (tile_rows) {
        row = sq.part0 + ((long long)(r / tile_rows) * sq.nsplit * p.H + head) * tile_rows + r % tile_rows;
        step = (long long)p.H * tile_rows;
    } else {
        const int R = sq.nq * p.G;
        row = sq.part0 + (long long)head * R + r;
        step = (long long)p.H * R;
        const int gr = sq.grow + r;
        grow = sq.gpart0 + ((long long)(gr / GROUP_ROWS) * sq.gsplit * p.H + head) * GROUP_ROWS + gr % GROUP_ROWS;
        gstep = (long long)p.H * GROUP_ROWS;
    }
    const int parts = sq.nsplit + sq.gsplit, dims = p.D;
    auto at = [&](int s) { return s < sq.nsplit ? row + s * step : grow + (s - sq.nsplit) * gstep; };
    auto load = [&](int s, int d) {
        return s < parts && d < dims ? __ldcg(reinterpret_cast<const float4 *>(p.part_o + at(s) * dims + d)) : make_float4(0, 0, 0, 0);
    };
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the parts are written
    float m = -CUDART_INF_F, sum = 0.0f;
    float4 acc[2] = {make_float4(0, 0, 0, 0), make_float4(0, 0, 0, 0)};  // dimensions lane * 4 and 128 + lane * 4
    auto add = [&](int half, float w, const float4 &v) {
        acc[half].x += w * v.x;
        acc[half].y += w * v.y;
        acc[half].z += w * v.z;
        acc[half].w += w * v.w;
    };
    for (int c0 = warp; c0 < parts; c0 += 32 * SPREAD) {  // 32 parts, a lane looks after the weight of one
        const int count = min(32, (parts - c0 + SPREAD - 1) / SPREAD);
        float4 v[JOIN_AHEAD];
#pragma unroll
        for (int k = 0; k < JOIN_AHEAD; ++k) v[k] = load(c0 + k * SPREAD, lane * 4);
        const float2 ml = lane < count ? __ldcg(reinterpret_cast<const float2 *>(p.part_ml + 2 * at(c0 + lane * SPREAD)))
                                       : make_float2(-CUDART_INF_F, 0.0f);
        float top = ml.x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        top = fmaxf(top, m);
        const float base = top == -CUDART_INF_F ? 0.0f : top, old = top == -CUDART_INF_F ? 1.0f : ex2(m - top);
        const float w = ex2(ml.x - base);  // a part that saw nothing: m = -inf
        sum = sum * old + w * ml.y;
        m = top;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            acc[half].x *= old;
            acc[half].y *= old;
            acc[half].z *= old;
            acc[half].w *= old;
        }
        for (int i = 0; i < count; i += JOIN_AHEAD) {
            if (i)
#pragma unroll
                for (int k = 0; k < JOIN_AHEAD; ++k) v[k] = load(i + k < count ? c0 + (i + k) * SPREAD : parts, lane * 4);
#pragma unroll
            for (int k = 0; k < JOIN_AHEAD; ++k) add(0, __shfl_sync(0xffffffffu, w, (i + k) & 31), v[k]);
            if (dims > 128)
#pragma unroll
                for (int k = 0; k < JOIN_AHEAD; ++k)
                    add(1, __shfl_sync(0xffffffffu, w, (i + k) & 31), load(i + k < count ? c0 + (i + k) * SPREAD : parts, 128 + lane * 4));
        }
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (SPREAD > 1) {
        const int at_s = team * SPREAD;
        acc_s[at_s + warp][0][lane] = acc[0];
        acc_s[at_s + warp][1][lane] = acc[1];
        if (lane == 0) {
            sum_s[at_s + warp] = sum;
            max_s[at_s + warp] = m;
        }
        asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "n"(SPREAD * 32) : "memory");
        if (warp) return;
        float top = m;
#pragma unroll
        for (int w = 1; w < SPREAD; ++w) top = fmaxf(top, max_s[at_s + w]);
        const float base = top == -CUDART_INF_F ? 0.0f : top;
        sum = 0.0f;
        acc[0] = acc[1] = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < SPREAD; ++w) {
            const float f = ex2(max_s[at_s + w] - base);
            sum += f * sum_s[at_s + w];
            add(0, f, acc_s[at_s + w][0][lane]);
            add(1, f, acc_s[at_s + w][1][lane]);
        }
        m = top;
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    T *out = static_cast<T *>(p.out) + (qt * Hq + hq) * dims;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int d = half * 128 + lane * 4;
        if (d < dims)
            *reinterpret_cast<uint2 *>(out + d) = make_uint2(Elt<T>::pack(scaled(acc[half].x, inv), scaled(acc[half].y, inv)),
                                                             Elt<T>::pack(scaled(acc[half].z, inv), scaled(acc[half].w, inv)));
    }
    if (!p.lse) return;
    RowSpan sp = row_span(p, sq, j);
    const float slope = p.slopes ? p.slopes[hq] : 0.0f;
    if (p.lists && p.slopes) sp.near = listed_near(p, sq, p.lists + (qt * p.H + head) * p.keep, sp);
    if (lane == 0) {
        p.lse[qt * Hq + hq] = sum == 0.0f ? -CUDART_INF_F : (m + log2f(sum)) * LN2 - slope * (float)sp.near;
    }
}

template <typename T, int SPREAD>
static cudaError_t join_go(const AttnParams &p, const SmallSeqs &small, int tile_rows, int rows, cudaStream_t st) {
    // launched so that its CTAs come up while the parts are still being computed; it waits for them itself
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((rows + JOIN_WARPS / SPREAD - 1) / (JOIN_WARPS / SPREAD)));
    cfg.blockDim = dim3(JOIN_WARPS * 32);
    cfg.stream = st;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, attend_join_kernel<T, SPREAD>, p, small, tile_rows, rows);
    return e != cudaSuccess ? e : cudaGetLastError();
}
cudaError_t launch_attend_join(const AttnParams &p, const SmallSeqs &small, int f16, int tile_rows, int tokens, int max_parts,
                               int sm_count, cudaStream_t st) {
    const int rows = tokens * p.H * p.G;
    // warps a row: no more than its parts keep busy, nor than the GPU holds at once
    int spread = 1;
    while (spread < JOIN_WARPS && spread * JOIN_AHEAD < max_parts && (long long)rows * spread < 8ll * sm_count) spread *= 2;
    switch (spread) {
        case 1: return f16 ? join_go<__half, 1>(p, small, tile_rows, rows, st) : join_go<__nv_bfloat16, 1>(p, small, tile_rows, rows, st);
        case 2: return f16 ? join_go<__half, 2>(p, small, tile_rows, rows, st) : join_go<__nv_bfloat16, 2>(p, small, tile_rows, rows, st);
        case 4: return f16 ? join_go<__half, 4>(p, small, tile_rows, rows, st) : join_go<__nv_bfloat16, 4>(p, small, tile_rows, rows, st);
        default: return f16 ? join_go<__half, 8>(p, small, tile_rows, rows, st) : join_go<__nv_bfloat16, 8>(p, small, tile_rows, rows, st);
    }
}

}  // namespace aafkv
