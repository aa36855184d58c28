// Attention of query tokens over listed blocks of their contexts: every query token and kv head has a list of its own.
//
//   s_rt = score(q_r . k_t) for the tokens t of the listed blocks that the row sees,  o_r = sum_t exp(s_rt) v_t / sum_t exp(s_rt)
//
// Bound: a listed block's keys and values are used by one kv head's group of query heads only, so their bytes decide.  The products
// are those of the kernel for few rows: a warp takes 16 tokens at a time as the M side and its rows as the N side, waits for its
// own copies only, weights in two 16-bit parts.  What differs: a CTA takes a query token, a kv head and a part of the list, its warps
// every WARPS-th tile of 16 tokens, and puts their results together in shared memory, so that short lists need no join; tokens
// come through the list and then the table, two loads that are asked for ahead of the copies; and all rows of a CTA belong to one
// query token, so they see the same keys.  A key that is not seen is not read: its key and value are zeros, its score is -inf.
//
// 64 ragged contexts, up to 256 blocks for each kv head, 979 MB: 168 to 177 us with the join (5.5 to 5.8 TB/s); 16 contexts, 64 blocks, 67 MB:
// 18.5 us; 128 tokens, 128 blocks each, 1.07 GB of which 267 MB are distinct: 105 to 117 us, where instructions decide (450 a tile of 16
// keys), 121 with a bias, 134 with a cap, 119 and 127 in blocks of 8 and 24 tokens.
#include "sparse_device.cuh"

namespace aafkv {

__device__ __forceinline__ void copy16_all(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// CTAS of WARPS warps share an SM, as many as registers allow (a warp by itself waits for most of its time: twelve warps of two stages are
// ahead of eight of three); a CTA that has an SM to itself has the warps of all of them.
template <int DP, int NT> struct ListShape {
    static constexpr int PIECES = DP / 8;           // 16-byte pieces of a row
    static constexpr int ROW = DP * 2, HALF = 16 * ROW;  // bytes of a row, of a tile of 16 keys (or values)
    static constexpr int STAGE_BYTES = 2 * HALF;
    static constexpr int WARPS = DP <= 128 ? 4 : 3, CTAS = NT > 1 || DP > 128 ? 2 : (DP == 128 ? 3 : 4);
    static constexpr int STAGES = DP > 128 ? 2 : (NT > 1 ? 384 : 768 / CTAS) / DP;
    static constexpr int WARP_BYTES = STAGES * STAGE_BYTES;
    static_assert(CTAS * (WARPS * WARP_BYTES + 2048) <= 228 * 1024, "shared memory of a CTA");
};

// SIMPLE: neither cap nor bias, a score is a multiple of the product.  WHOLE: a tile of 16 tokens lies within a block (of a multiple of 16), so
// that one list entry, one table entry and one address do for all of it (1024 lists of 2048 keys: 109 us, looked up token by token 116)
template <typename T, int DP, int NT, bool SIMPLE, bool WHOLE, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, WARPS == ListShape<DP, NT>::WARPS ? ListShape<DP, NT>::CTAS : 1)
    attend_blocks_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ SmallSeqs small, int row_groups) {
    using S = ListShape<DP, NT>;
    extern __shared__ __align__(16) char smem[];
    __shared__ float2 ml_s[WARPS][NT * 8];  // of a warp's rows: base of the exponents, sum
    static_assert(NT * 8 * DP * 4 <= S::WARP_BYTES, "a warp's results fit where its copies were");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t4 = lane & 3;
    // One kv head after the other, so that query tokens of one context that list the same blocks find them in L2
    const int per_head = p.total_units * row_groups, head = blockIdx.x / per_head, rest = blockIdx.x - head * per_head;
    const int unit = rest / row_groups, first_row = (rest - unit * row_groups) * NT * 8;  // of the group's heads
    asm volatile("griddepcontrol.launch_dependents;");  // the join may be brought up beside this kernel
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq sq = seqs[find_seq(seqs, p.n, unit)];
    const int j = (unit - sq.unit0) / sq.nsplit, part = unit - sq.unit0 - j * sq.nsplit;
    const int R = min(NT * 8, p.G - first_row);
    const long long tok = sq.row0 + j;
    RowSpan span = row_span(p, sq, j);
    const int *list = p.lists + (tok * p.H + head) * p.keep;
    if (!SIMPLE && p.slopes) span.near = listed_near(p, sq, list, span);
    float slope[SIMPLE ? 1 : NT][2];
    if (!SIMPLE) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c)
                slope[nt][c] = p.slopes ? p.slopes[head * p.G + first_row + min(nt * 8 + 2 * t4 + c, R - 1)] : 0.0f;
    }
    // listed tokens, numbered through the list: those of this part
    const int blocks = (sq.len + p.BS - 1) / p.BS;
    int used = p.keep;
    if (p.keep > blocks) {  // such a list is filled up: its last entry that names a block
        used = 0;
        for (int i = lane; i < p.keep; i += 32) {
            const int b = __ldg(list + i);
            if (b >= 0 && b < blocks) used = i + 1;
        }
        used = (int)__reduce_max_sync(0xffffffffu, (unsigned)used);
    }
    const int beg = part * sq.chunk, end = part + 1 < sq.nsplit ? min(beg + sq.chunk, used * p.BS) : used * p.BS;
    const int tiles_all = max(0, end - beg + 15) / 16, tiles = (tiles_all - warp + WARPS - 1) / WARPS;  // of the part, of this warp
    auto first_of = [&](int tile) { return beg + (tile * WARPS + warp) * 16; };

    const uint32_t base = (uint32_t)__cvta_generic_to_shared(smem) + warp * S::WARP_BYTES;
    // where piece c of row r lies: lanes that read together have two rows and four pieces of K, four even (odd) rows and two
    // pieces of V
    auto k_at = [](int r, int c) { return (uint32_t)(r * S::ROW + ((c ^ ((r & 1) << 2)) << 4)); };
    auto v_at = [](int r, int c) { return (uint32_t)(S::HALF + r * S::ROW + ((c ^ (r & 6)) << 4)); };
    const int *table = p.tables + (long long)sq.ctx * p.max_blk;
    const char *kb = p.kbase + (long long)head * p.D * 2;

    // Lane l looks after the tile's token l % 16 (WHOLE: every lane after the first): its block's table position, then its position in the
    // context (-1: not seen; WHOLE: no token of the tile is) and where its key lies
    const int own = WHOLE ? 0 : lane & 15;
    auto listed = [&](int tile) -> int {
        const int u = first_of(tile) + own;
        return u < end ? __ldg(list + block_of(u, p.BS, p.bs_shift)) : -1;
    };
    struct Key {
        int t, id, slot;
    };
    auto key_of = [&](int tile, int entry) -> Key {
        Key k{-1, 0, 0};
        if (entry >= 0 && entry < blocks) {
            const int u = first_of(tile) + own;
            k.slot = u - block_of(u, p.BS, p.bs_shift) * p.BS;
            const int t = entry * p.BS + k.slot;
            if (t + (WHOLE ? 15 : 0) >= span.lo && t < span.hi) {
                k.t = t;
                k.id = __ldg(table + entry);
            }
        }
        return k;
    };
    constexpr int AT_ONCE = 32 / S::PIECES;  // rows of one copy instruction
    const int c = lane % S::PIECES, r0 = lane / S::PIECES;
    auto issue = [&](int tile, const Key &k) {
        if (WHOLE) {
            if (k.t >= 0) {  // else nothing of the tile is looked at
                const uint32_t st = base + (tile % S::STAGES) * S::STAGE_BYTES;
                const char *src = kb + (long long)k.id * 2 * p.run + (long long)(k.slot + r0) * p.row + c * 16;
                if (k.t >= span.lo && k.t + 16 <= span.hi && p.D == DP) {
                    const char *val = src + p.run;
                    const long long down = AT_ONCE * p.row;
#pragma unroll
                    for (int i = 0; i < 16 / AT_ONCE; ++i) {
                        copy16_all(st + k_at(i * AT_ONCE + r0, c), src);
                        copy16_all(st + v_at(i * AT_ONCE + r0, c), val);
                        src += down;
                        val += down;
                    }
                } else {
#pragma unroll 1
                    for (int i = 0; i < 16 / AT_ONCE; ++i) {
                        const int r = i * AT_ONCE + r0;
                        const bool in = k.t + r >= span.lo && k.t + r < span.hi && c * 8 < p.D;
                        copy16(st + k_at(r, c), in ? src : kb, in ? 16 : 0);
                        copy16(st + v_at(r, c), in ? src + p.run : kb, in ? 16 : 0);
                        src += AT_ONCE * p.row;
                    }
                }
            }
        } else if (tile < tiles) {
            const long long off = k.t < 0 ? -1 : (long long)k.id * 2 * p.run + (long long)k.slot * p.row;
            const uint32_t st = base + (tile % S::STAGES) * S::STAGE_BYTES;
#pragma unroll
            for (int i = 0; i < 16 / AT_ONCE; ++i) {
                const int r = i * AT_ONCE + r0;
                const long long at = __shfl_sync(0xffffffffu, off, r);
                const bool in = at >= 0 && c * 8 < p.D;
                const char *src = kb + at + c * 16;
                copy16(st + k_at(r, c), in ? src : kb, in ? 16 : 0);
                copy16(st + v_at(r, c), in ? src + p.run : kb, in ? 16 : 0);
            }
        }
        copy_commit();
    };

    int pos[S::STAGES];  // of the tokens whose copies are under way
    int entry = listed(0), after = listed(1);
    Key key = key_of(0, entry);
    entry = after;
#pragma unroll
    for (int s = 0; s < S::STAGES; ++s) {
        after = listed(s + 2);
        const Key nxt = key_of(s + 1, entry);
        issue(s, key);
        pos[s] = key.t;
        key = nxt;
        entry = after;
    }

    // query fragments: row nt * 8 + g, 8 dimensions at kk * 32 + t4 * 8
    uint4 qf[NT][DP / 32];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int r = nt * 8 + g;
        const T *q = static_cast<const T *>(p.q) + tok * p.q_stride + (long long)(head * p.G + first_row + min(r, R - 1)) * p.D;
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
        // the tile's tokens that are seen, a bit each
        const unsigned seen = !WHOLE ? __ballot_sync(0xffffffffu, pos[0] >= 0)
                                     : (pos[0] < 0 ? 0u : (1u << max(0, min(16, span.hi - pos[0]))) - (1u << max(0, min(16, span.lo - pos[0]))));
        if (seen) {
            const uint32_t st = base + (tile % S::STAGES) * S::STAGE_BYTES;
            float s[NT][4], s2[NT][4];  // two sums, which take turns: a product waits for the one before it in the same sum
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[nt][i] = s2[nt][i] = 0.0f;
#pragma unroll
            for (int kk = 0; kk < DP / 32; ++kk) {
                const uint4 w = lds16(st + k_at(g, kk * 4 + t4)), x = lds16(st + k_at(g + 8, kk * 4 + t4));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    Elt<T>::mma(s[nt], w.x, x.x, w.y, x.y, qf[nt][kk].x, qf[nt][kk].y);
                    Elt<T>::mma(s2[nt], w.z, x.z, w.w, x.w, qf[nt][kk].z, qf[nt][kk].w);
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[nt][i] += s2[nt][i];
            const int t_of[2] = {SIMPLE ? 0 : (WHOLE ? pos[0] + g : __shfl_sync(0xffffffffu, pos[0], g)),
                                 SIMPLE ? 0 : (WHOLE ? pos[0] + g + 8 : __shfl_sync(0xffffffffu, pos[0], g + 8))};
            uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float mx[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float &x = s[nt][2 * h + c];
                        x = seen >> (g + 8 * h) & 1 ? (SIMPLE ? x * c2 : score2(p, x, slope[SIMPLE ? 0 : nt][c], span, t_of[h])) : -CUDART_INF_F;
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
            }
#pragma unroll
            for (int c = 0; c < DP / 64; ++c) {
                uint4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = lds16(st + v_at(2 * t4 + (i & 1) + (i >> 1) * 8, c * 8 + g));
                const uint32_t w0[4] = {v[0].x, v[0].y, v[0].z, v[0].w}, w1[4] = {v[1].x, v[1].y, v[1].z, v[1].w};
                const uint32_t w2[4] = {v[2].x, v[2].y, v[2].z, v[2].w}, w3[4] = {v[3].x, v[3].y, v[3].z, v[3].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t a[4] = {prmt(w0[i], w1[i], 0x5410), prmt(w0[i], w1[i], 0x7632), prmt(w2[i], w3[i], 0x5410),
                                           prmt(w2[i], w3[i], 0x7632)};
                    // An infinite value times the high part of its weight is infinite; times the low part, which may be zero
                    // or negative, it would make a NaN of that: there it is the type's largest value.
                    uint32_t b[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) b[e] = Elt<T>::bounded(a[e]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        Elt<T>::mma(o[nt][4 * c + i], a[0], a[1], a[2], a[3], ph[nt][0], ph[nt][1]);
                        Elt<T>::mma(o[nt][4 * c + i], b[0], b[1], b[2], b[3], pl[nt][0], pl[nt][1]);
                    }
                }
            }
        }
        after = listed(tile + S::STAGES + 2);
        const Key nxt = key_of(tile + S::STAGES + 1, entry);
        __syncwarp();  // every lane has read this stage
        issue(tile + S::STAGES, key);
#pragma unroll
        for (int s = 0; s + 1 < S::STAGES; ++s) pos[s] = pos[s + 1];
        pos[S::STAGES - 1] = key.t;
        key = nxt;
        entry = after;
    }
    copy_wait<0>();
    __syncwarp();

    // every warp's results to shared memory, then (m, l, o) of the part from all of them, in warp order
    float *o_s = reinterpret_cast<float *>(smem + warp * S::WARP_BYTES);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            float sum = l[nt][c];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            const float some = sum == 0.0f ? 0.0f : 1.0f;
            const int r = nt * 8 + 2 * t4 + c;
            if (g == 0) ml_s[warp][r] = make_float2(m[nt][c] - Elt<T>::RAISE, sum);
#pragma unroll
            for (int cc = 0; cc < DP / 64; ++cc) {
                float4 *dst = reinterpret_cast<float4 *>(o_s + r * DP + cc * 64 + g * 8);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    dst[i] = make_float4(scaled(o[nt][4 * cc + 2 * i][c], some), scaled(o[nt][4 * cc + 2 * i][2 + c], some),
                                         scaled(o[nt][4 * cc + 2 * i + 1][c], some), scaled(o[nt][4 * cc + 2 * i + 1][2 + c], some));
            }
        }
    __syncthreads();
    const int quads = p.D / 4;
    for (int i = threadIdx.x; i < R * quads; i += WARPS * 32) {
        const int r = i / quads, d = (i - r * quads) * 4;
        float top = -CUDART_INF_F;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) top = fmaxf(top, ml_s[w][r].x);
        const float from = top == -CUDART_INF_F ? 0.0f : top;
        float sum = 0.0f;
        float4 acc = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float2 ml = ml_s[w][r];
            const float f = ex2(ml.x - from);  // a warp that saw nothing: 0
            const float4 v = *reinterpret_cast<const float4 *>(smem + w * S::WARP_BYTES + (r * DP + d) * 4);
            sum += f * ml.y;
            acc.x += f * v.x;
            acc.y += f * v.y;
            acc.z += f * v.z;
            acc.w += f * v.w;
        }
        const int hg = first_row + r;  // head of the group
        if (sq.part0 >= 0) {  // a part of the list, for the join; laid out as the kernel for few rows does
            const long long pr = sq.part0 + ((long long)part * p.H + head) * sq.nq * p.G + (long long)j * p.G + hg;
            *reinterpret_cast<float4 *>(p.part_o + pr * p.D + d) = acc;
            if (d == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * pr) = make_float2(top, sum);
            continue;
        }
        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;  // a row that sees nothing is zero
        const long long hq = tok * p.H * p.G + head * p.G + hg;
        *reinterpret_cast<uint2 *>(static_cast<T *>(p.out) + hq * p.D + d) =
            make_uint2(Elt<T>::pack(scaled(acc.x, inv), scaled(acc.y, inv)), Elt<T>::pack(scaled(acc.z, inv), scaled(acc.w, inv)));
        if (p.lse && d == 0)
            p.lse[hq] = sum == 0.0f ? -CUDART_INF_F : (top + log2f(sum)) * LN2 - (!SIMPLE && p.slopes ? p.slopes[head * p.G + hg] * (float)span.near : 0.0f);
    }
}

// rows that a lane's registers hold accumulators for, as in the kernel for few rows; larger groups go to several CTAs
static int list_tiles(int D, int G) { return std::min((G + 7) / 8, few_rows_limit(D) / 8); }
int attend_blocks_rows(int D, int G) {
    const int nt = list_tiles(D, G);
    return 8 * (nt == 3 ? 4 : nt);
}

int attend_blocks_warps(int D) { return D <= 128 ? ListShape<128, 1>::WARPS : ListShape<256, 1>::WARPS; }
int attend_blocks_ctas(int D, int G) {
    return list_tiles(D, G) > 1 || D > 128 ? ListShape<128, 2>::CTAS : (D <= 64 ? ListShape<64, 1>::CTAS : ListShape<128, 1>::CTAS);
}
static_assert(ListShape<64, 1>::WARPS == ListShape<128, 1>::WARPS && ListShape<256, 1>::CTAS == 2 && ListShape<64, 2>::CTAS == 2 &&
              ListShape<64, 4>::CTAS == 2, "what the two functions say");

template <typename T, int DP, int NT, bool SIMPLE, bool WHOLE, int WARPS>
static cudaError_t list_go(const AttnParams &p, const SmallSeqs &small, cudaStream_t st) {
    static SmemSeen seen{0};
    constexpr int bytes = WARPS * ListShape<DP, NT>::WARP_BYTES;
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(attend_blocks_kernel<T, DP, NT, SIMPLE, WHOLE, WARPS>), bytes, &seen);
    if (e != cudaSuccess) return e;
    const int groups = (p.G + NT * 8 - 1) / (NT * 8);
    attend_blocks_kernel<T, DP, NT, SIMPLE, WHOLE, WARPS><<<(unsigned)(p.total_units * p.H * groups), WARPS * 32, bytes, st>>>(p, small, groups);
    return cudaGetLastError();
}
template <typename T, int DP, int NT, bool SIMPLE> static cudaError_t list_whole(const AttnParams &p, const SmallSeqs &small, bool alone, cudaStream_t st) {
    constexpr int W = ListShape<DP, NT>::WARPS, ALL = W * ListShape<DP, NT>::CTAS;
    if (p.BS % 16 == 0) return alone ? list_go<T, DP, NT, SIMPLE, true, ALL>(p, small, st) : list_go<T, DP, NT, SIMPLE, true, W>(p, small, st);
    return alone ? list_go<T, DP, NT, SIMPLE, false, ALL>(p, small, st) : list_go<T, DP, NT, SIMPLE, false, W>(p, small, st);
}
template <typename T, int DP, int NT> static cudaError_t list_kind(const AttnParams &p, const SmallSeqs &small, bool alone, cudaStream_t st) {
    return p.softcap == 0.0f && !p.slopes ? list_whole<T, DP, NT, true>(p, small, alone, st) : list_whole<T, DP, NT, false>(p, small, alone, st);
}
template <typename T> static cudaError_t list_pick(const AttnParams &p, const SmallSeqs &small, bool alone, cudaStream_t st) {
    const int nt = list_tiles(p.D, p.G);
    if (p.D <= 64)
        return nt == 1 ? list_kind<T, 64, 1>(p, small, alone, st) : (nt == 2 ? list_kind<T, 64, 2>(p, small, alone, st) : list_kind<T, 64, 4>(p, small, alone, st));
    if (p.D <= 128) return nt == 1 ? list_kind<T, 128, 1>(p, small, alone, st) : list_kind<T, 128, 2>(p, small, alone, st);
    return list_kind<T, 256, 1>(p, small, alone, st);
}
cudaError_t launch_attend_blocks(const AttnParams &p, const SmallSeqs &small, int f16, bool alone, cudaStream_t st) {
    return f16 ? list_pick<__half>(p, small, alone, st) : list_pick<__nv_bfloat16>(p, small, alone, st);
}

}  // namespace aafkv
