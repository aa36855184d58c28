// Attention mass of cached tokens: mass_t = prev_t + sum over query rows r of exp(score_rt - lse_r).
//
// One pass over the keys; with the rows' log-sums given, every token is independent of the others.  A warp owns 16
// tokens and walks over all kv heads and query rows, so a token's sum stays in one lane quad and is taken in a fixed order
// (row block by row block, head by head, eight rows at a time): no atomics, the same bits every time.  Bound: the bytes of
// K while there are few rows, the exponentials' surroundings (masks, sums) from about a hundred rows on.  Keys come through
// the block table into stages of the warp's own, two heads ahead; the queries of as many heads as fit (64 rows) are shared by the
// CTA's four warps.  CTAs are small, three or four an SM: while one waits for its first keys or its next queries, the others
// work.  111 MB of keys, one token a context, four rows a head: 30 us (3.7 TB/s; 31.7 with two stages, 35.7 with four, when
// fewer CTAs fit; 32 with the rows fetched to L2 ahead).  Products as in attend_few.cu: tokens as the M side, eight query
// rows as the N side.
#include <type_traits>

#include "attend_device.cuh"

namespace aafkv {

constexpr int MASS_WARPS = 4, MASS_TOKENS = 16;  // tokens of a warp
static_assert(MASS_WARPS * MASS_TOKENS == MASS_CHUNK, "tokens of a CTA");

template <int DP> struct MassShape {
    static constexpr int ROW = DP * 2, PIECES = DP / 8, ROWS = DP <= 128 ? 64 : 32;  // rows of a batch of queries
    static constexpr int TILE_BYTES = MASS_TOKENS * ROW, STAGES = 3;
    static constexpr int K_BYTES = MASS_WARPS * STAGES * TILE_BYTES;
};
struct MassRow {  // what a query row of any head sees
    int lo, hi, pos, near;
};

template <typename T, int DP>
__global__ void __launch_bounds__(MASS_WARPS * 32, DP <= 128 ? 4 : 2)
    attn_mass_kernel(const __grid_constant__ MassParams p, const __grid_constant__ SmallSeqs small) {
    using S = MassShape<DP>;
    extern __shared__ __align__(16) char smem[];
    __shared__ MassRow row_info[S::ROWS];
    __shared__ __align__(8) float row_lse[S::ROWS];
    __shared__ float row_slope[S::ROWS];
    const AttnParams &a = p.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t4 = lane & 3;
    const AttnSeq *seqs = a.seqs ? a.seqs : small.e;
    const int unit = blockIdx.x, si = find_seq(seqs, a.n, unit);
    const AttnSeq sq = seqs[si];
    const int tb = (unit - sq.unit0) * MASS_CHUNK + warp * MASS_TOKENS;  // the warp's tokens
    const int R = sq.nq * a.G, Hq = a.H * a.G;
    const int block_rows = min((R + 7) / 8 * 8, S::ROWS), batch_heads = min(a.H, S::ROWS / block_rows);
    const int row_blocks = (R + block_rows - 1) / block_rows, batches = (a.H + batch_heads - 1) / batch_heads;
    const uint32_t sK = (uint32_t)__cvta_generic_to_shared(smem) + warp * S::STAGES * S::TILE_BYTES;
    const uint32_t sQ = (uint32_t)__cvta_generic_to_shared(smem) + S::K_BYTES;
    auto at = [](int r, int c) { return (uint32_t)(r * S::ROW + ((c ^ ((r & 1) << 2)) << 4)); };

    // keys: lane l knows where the warp's token l % 16 is
    long long off = 0;
    {
        const int t = tb + (lane & 15), b = block_of(t, a.BS, a.bs_shift);
        if (t < sq.len)
            off = (long long)__ldg(a.tables + (long long)sq.ctx * a.max_blk + b) * 2 * a.run + (long long)(t - b * a.BS) * a.row;
    }
    const int steps = tb < sq.len ? row_blocks * a.H : 0;  // one head of one row block each
    auto load_keys = [&](int step) {
        if (step < steps) {
            constexpr int AT_ONCE = 32 / S::PIECES;
            const int head = step % a.H, c = lane % S::PIECES;
            const uint32_t dst = sK + (step % S::STAGES) * S::TILE_BYTES;
#pragma unroll
            for (int i = 0; i < MASS_TOKENS / AT_ONCE; ++i) {
                const int r = i * AT_ONCE + lane / S::PIECES;
                const char *src = a.kbase + __shfl_sync(0xffffffffu, off, r) + (long long)head * a.D * 2 + c * 16;
                const bool in = tb + r < sq.len && c * 8 < a.D;
                copy16(dst + at(r, c), in ? src : a.kbase, in ? 16 : 0);
            }
        }
        copy_commit();
    };
    // Queries of a batch of heads: row hh * block_rows + r.  A row behind the last repeats the last one, with a log-sum of
    // infinity: it adds nothing unless the last row itself adds a NaN (zeros would make a NaN of an infinite key).
    auto load_queries = [&](int batch) {
        if (batch < row_blocks * batches) {
            const int rb = batch / batches * block_rows, h0 = batch % batches * batch_heads, heads = min(batch_heads, a.H - h0);
            const uint32_t dst = sQ;
            constexpr int AT_ONCE = MASS_WARPS * 32 / S::PIECES;
            const int c = threadIdx.x % S::PIECES;
            auto row_of = [&](int r, int &hh) {  // row of the sequence, capped at the last
                hh = batch_heads == 1 ? 0 : r / block_rows;
                return rb + r - hh * block_rows;
            };
#pragma unroll 4
            for (int r = threadIdx.x / S::PIECES; r < heads * block_rows; r += AT_ONCE) {
                int hh;
                const int rc = min(row_of(r, hh), R - 1), j = token_of(a, rc);
                const T *src = static_cast<const T *>(a.q) + (sq.row0 + j) * a.q_stride + ((h0 + hh) * a.G + rc - j * a.G) * a.D + c * 8;
                const bool in = c * 8 < a.D;
                copy16(dst + at(r, c), in ? src : static_cast<const T *>(a.q), in ? 16 : 0);
            }
            for (int r = threadIdx.x; r < heads * block_rows; r += MASS_WARPS * 32) {
                int hh;
                const int rc = min(row_of(r, hh), R - 1), j = token_of(a, rc), hq = (h0 + hh) * a.G + rc - j * a.G;
                float lse = p.lse_in[(long long)(sq.row0 + j) * Hq + hq];
                if (a.slopes) {  // scores are measured from the nearest visible key, so is the log-sum
                    row_slope[r] = a.slopes[hq];
                    lse += a.slopes[hq] * (float)row_span(a, sq, j).near;
                }
                // a row without a sum adds nothing, nor does one behind the last
                row_lse[r] = lse == -CUDART_INF_F || row_of(r, hh) >= R ? CUDART_INF_F : lse * LOG2E;
            }
        }
        copy_commit();
    };

    load_queries(0);
#pragma unroll
    for (int i = 0; i < S::STAGES - 1; ++i) load_keys(i);
    float w[2] = {0.0f, 0.0f};  // tokens g, g + 8, rows of this lane's columns
    const float c2 = a.scale * LOG2E;
    const bool plain = a.softcap == 0.0f && !a.slopes;
    int step = 0;
    bool quick = false;  // no score of the warp's tokens is masked, and scores are multiples of the products
    for (int batch = 0; batch < row_blocks * batches; ++batch) {
        const int rb = batch / batches * block_rows, h0 = batch % batches * batch_heads, heads = min(batch_heads, a.H - h0);
        copy_wait<0>();   // this batch's queries (and the keys asked for so far)
        __syncthreads();  // everyone's part of them; everyone is done with the batch before
        if (batch % batches == 0) {  // a new block of rows
            for (int r = threadIdx.x; r < block_rows; r += MASS_WARPS * 32) {
                const RowSpan sp = row_span(a, sq, token_of(a, min(rb + r, R - 1)));
                row_info[r] = MassRow{sp.lo, rb + r < R ? sp.hi : 0, sp.pos, sp.near};
            }
            __syncthreads();
            int lo = 0, hi = 0x7fffffff;  // tokens that every row of the block sees
            for (int r = lane; r < block_rows && rb + r < R; r += 32) {
                lo = max(lo, row_info[r].lo);
                hi = min(hi, row_info[r].hi);
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                lo = max(lo, __shfl_xor_sync(0xffffffffu, lo, d));
                hi = min(hi, __shfl_xor_sync(0xffffffffu, hi, d));
            }
            quick = plain && tb >= lo && tb + MASS_TOKENS <= hi;
        }
        for (int hh = 0; hh < heads && steps; ++hh, ++step) {
            load_keys(step + S::STAGES - 1);
            copy_wait<S::STAGES - 1>();
            __syncwarp();
            const uint32_t k = sK + (step % S::STAGES) * S::TILE_BYTES;
            uint4 kf[2][DP / 32];
#pragma unroll
            for (int kk = 0; kk < DP / 32; ++kk) {
                kf[0][kk] = lds16(k + at(g, kk * 4 + t4));
                kf[1][kk] = lds16(k + at(g + 8, kk * 4 + t4));
            }
            __syncwarp();
            const uint32_t q = sQ + hh * block_rows * S::ROW;
            // weights of UNITS groups of eight rows: independent products, one would wait for itself at every step
            auto rows = [&](int r0, auto units) {
                constexpr int U = decltype(units)::value;
                float s[U][4];
#pragma unroll
                for (int u = 0; u < U; ++u) s[u][0] = s[u][1] = s[u][2] = s[u][3] = 0.0f;
#pragma unroll
                for (int kk = 0; kk < DP / 32; ++kk)
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const uint4 qf = lds16(q + at(r0 + 8 * u + g, kk * 4 + t4));
                        Elt<T>::mma(s[u], kf[0][kk].x, kf[1][kk].x, kf[0][kk].y, kf[1][kk].y, qf.x, qf.y);
                        Elt<T>::mma(s[u], kf[0][kk].z, kf[1][kk].z, kf[0][kk].w, kf[1][kk].w, qf.z, qf.w);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int r = r0 + 8 * u + 2 * t4;
                    const float2 lse = *reinterpret_cast<const float2 *>(&row_lse[hh * block_rows + r]);
                    if (quick) {
                        w[0] += ex2(fmaf(s[u][0], c2, -lse.x)) + ex2(fmaf(s[u][1], c2, -lse.y));
                        w[1] += ex2(fmaf(s[u][2], c2, -lse.x)) + ex2(fmaf(s[u][3], c2, -lse.y));
                        continue;
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const MassRow ri = row_info[r + c];
                        RowSpan sp;
                        sp.lo = ri.lo;
                        sp.hi = ri.hi;
                        sp.pos = ri.pos;
                        sp.near = ri.near;
                        const float slope = a.slopes ? row_slope[hh * block_rows + r + c] : 0.0f;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int t = tb + g + 8 * h;
                            const float x = score2(a, s[u][2 * h + c], slope, sp, t) - (c ? lse.y : lse.x);
                            w[h] += t >= ri.lo && t < ri.hi ? ex2(x) : 0.0f;
                        }
                    }
                }
            };
            int r0 = 0;
            for (; r0 + 32 <= block_rows; r0 += 32) rows(r0, std::integral_constant<int, 4>{});
            for (; r0 < block_rows; r0 += 8) rows(r0, std::integral_constant<int, 1>{});
        }
        if (batch + 1 < row_blocks * batches) {
            __syncthreads();
            load_queries(batch + 1);
        }
    }
    copy_wait<0>();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        w[h] += __shfl_xor_sync(0xffffffffu, w[h], 1);
        w[h] += __shfl_xor_sync(0xffffffffu, w[h], 2);
        const int t = tb + g + 8 * h;
        if (t4 == 0 && t < sq.len) {
            const long long o = si * p.mass_stride + t;
            p.mass[o] = (p.prev ? p.prev[o] : 0.0f) + w[h];
        }
    }
}

template <typename T, int DP> static cudaError_t mass_go(const MassParams &p, const SmallSeqs &small, int max_rows, cudaStream_t st) {
    using S = MassShape<DP>;
    const int block = min((max_rows + 7) / 8 * 8, S::ROWS), rows = (int)min((long long)S::ROWS, (long long)block * p.a.H);
    const int smem = S::K_BYTES + rows * S::ROW;
    static SmemSeen seen{0};
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(attn_mass_kernel<T, DP>), S::K_BYTES + S::ROWS * S::ROW, &seen);
    if (e != cudaSuccess) return e;
    attn_mass_kernel<T, DP><<<(unsigned)p.a.total_units, MASS_WARPS * 32, smem, st>>>(p, small);
    return cudaGetLastError();
}
template <typename T> static cudaError_t mass_pick(const MassParams &p, const SmallSeqs &small, int max_rows, cudaStream_t st) {
    if (p.a.D <= 64) return mass_go<T, 64>(p, small, max_rows, st);
    if (p.a.D <= 128) return mass_go<T, 128>(p, small, max_rows, st);
    return mass_go<T, 256>(p, small, max_rows, st);
}
cudaError_t launch_attn_mass(const MassParams &p, const SmallSeqs &small, int f16, int max_rows, cudaStream_t st) {
    return f16 ? mass_pick<__half>(p, small, max_rows, st) : mass_pick<__nv_bfloat16>(p, small, max_rows, st);
}

}  // namespace aafkv
