// The blocks of a context with the largest bound on a query's scores, for every query token and kv head.
//
//   q_d in steps of 2^f: c_d = rint(F(q_d) / 2^f), |c_d| <= 127;   dot_b = sum_d max(c_d hi_bd, c_d lo_bd)
//   score_b = max over the group's heads of dot_b * 2^(e_b + f)
//
// max(c hi, c lo) = max(c, 0) hi + min(c, 0) lo: a product of [c+, c-] with the block's [hi, lo], in whole numbers, exact in any
// order, and so is the scaling by a power of two; equal scores go to the lower block.
//
// A unit is a tile of query tokens of a context and a kv head; a cluster of CTAs takes it, each CTA a stretch of the context's
// blocks.  Scores: 16 blocks as the M side of 8-bit products, the tile's query rows as the N side, codes straight from memory into
// the lanes that need them (the order of the channels is free as long as both sides agree: a lane takes 16 consecutive
// bytes).  They stay in shared memory, as whole numbers of the same order.  Selection: the smallest score that is taken is
// found eight bits at a time by histograms, which the CTAs of a cluster read from one another; then every CTA knows how many blocks come
// before its own and writes its part of the list.
//
// Bound: the bytes of the summaries where there is a token each; the selection's passes where there are many.
#include "sparse_device.cuh"

namespace aafkv {

constexpr int SELECT_WARPS = 8, SELECT_ROWS = 64;  // query rows of a pass over the summaries
constexpr int SELECT_TOKENS = 16;                  // of a tile, at most

__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// words of another CTA's shared memory: those that lie there where `addr` lies here
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, int cta) {
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(cta));
    return at;
}
__device__ __forceinline__ uint4 peer_words(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 peer_pair(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared::cluster.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}

// SPANS: 64-byte stretches of a head's codes (2 head_dim bytes); NT: n-tiles of 8 query rows that are accumulated at a time
template <int SPANS, int NT>
__global__ void __launch_bounds__(SELECT_WARPS * 32, 2)
    select_blocks_kernel(const __grid_constant__ SelectParams p, const __grid_constant__ SmallSeqs small, const __grid_constant__ SelectShape z) {
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t *keys = reinterpret_cast<uint32_t *>(smem);                    // [tile][room]
    uint32_t *hist = keys + z.tile * z.room;                                // [2][tile][256]
    unsigned char *codes = reinterpret_cast<unsigned char *>(hist + 2 * z.tile * 256);  // [rows][stride]
    __shared__ __align__(8) float units_s[SELECT_ROWS];                     // of a row's codes: 2^f
    __shared__ __align__(8) uint32_t range_s[2];                            // smallest and largest score of the stretch, of any token
    __shared__ int last_s[SELECT_TOKENS];                                   // a token's own block
    __shared__ uint32_t prefix_s[SELECT_TOKENS];                            // of a list: the threshold's leading bits
    __shared__ int want_s[SELECT_TOKENS];                                   // how many of those with these bits are taken; see below
    __shared__ uint32_t before_s[SELECT_TOKENS][2];                         // in other CTAs' earlier stretches: above the threshold, equal to it
    __shared__ uint32_t counts_s[SELECT_WARPS][2];                          // of a warp's piece: certainly taken, equal to the threshold
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t4 = lane & 3;
    const int cta = z.ctas > 1 ? (int)cluster_rank() : 0;
    const int unit = blockIdx.x / z.ctas / p.H, head = blockIdx.x / z.ctas - unit * p.H;
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq s = seqs[find_seq(seqs, p.n, unit)];
    const int j0 = (unit - s.unit0) * z.tile, tokens = min(z.tile, s.nq - j0);
    const int pos0 = s.len - s.nq + j0;  // position of the tile's first token
    const int total = (pos0 + tokens - 1) / p.BS + 1;  // blocks that some token of the tile may take
    const int stretch = ((total + z.ctas - 1) / z.ctas + 15) / 16 * 16;
    const int b0 = min(cta * stretch, total), count = min(stretch, total - b0);
    auto sync_all = [&]() {
        if (z.ctas > 1) cluster_sync();
        else __syncthreads();
    };
    auto key_at = [&](int list, int i) -> uint32_t & { return keys[list * z.room + i]; };

    for (int i = threadIdx.x; i < z.tile * 256; i += SELECT_WARPS * 32) hist[i] = 0;
    if (threadIdx.x < z.tile) {
        const int last = (pos0 + min((int)threadIdx.x, tokens - 1)) / p.BS;
        const int want = p.keep - p.sink - p.recent;
        last_s[threadIdx.x] = last;
        prefix_s[threadIdx.x] = before_s[threadIdx.x][0] = before_s[threadIdx.x][1] = 0;
        want_s[threadIdx.x] = last + 1 <= p.keep ? -1 : want;
    }

    if (threadIdx.x == 0) {
        range_s[0] = 0xffffffffu;
        range_s[1] = 0;
    }

    // ---- scores
    uint32_t least_k = 0xffffffffu, most_k = 0;
    const int *table = p.tables + (long long)s.ctx * p.max_blk + b0;
    auto id_of = [&](int m) {  // block of lane l's row l % 16 of an m-tile; behind the stretch its last one again
        return count ? __ldg(table + min(m * 16 + (lane & 15), count - 1)) : 0;
    };
    struct Codes {
        uint4 a[SPANS][2];
        int e[2];
    };
    const signed char *first = p.summary + (long long)head * 2 * p.D + t4 * 16;
    const int e_at = (p.H - head) * 2 * p.D + head - t4 * 16;  // the head's exponent, from there
    auto fetch = [&](int id, Codes &x) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const signed char *rec = first + (long long)__shfl_sync(0xffffffffu, id, g + 8 * h) * p.record;
            x.e[h] = __ldg(rec + e_at);
#pragma unroll
            for (int sp = 0; sp < SPANS; ++sp)
                x.a[sp][h] = sp * 64 + t4 * 16 < 2 * p.D ? __ldg(reinterpret_cast<const uint4 *>(rec + sp * 64)) : make_uint4(0, 0, 0, 0);
        }
    };
    constexpr bool AHEAD = SPANS <= 4;  // the next m-tile's codes are under way while one is multiplied, where registers allow it
    const int rows_all = z.tile * z.heads_p, hp_shift = z.heads_p >= 8 ? 3 : z.heads_p >> 1;  // rows of a token in an n-tile: 2^hp_shift
    for (int row0 = 0; row0 < rows_all; row0 += z.rows) {
        if (row0) __syncthreads();
        int id = id_of(warp);
        const int rows = min(z.rows, (rows_all - row0 + 7) / 8 * 8);
        for (int r = warp; r < rows; r += SELECT_WARPS) {  // a row's codes: [c+, c-], zeros behind them
            const int tok = min((row0 + r) / z.heads_p, tokens - 1), gh = min((row0 + r) % z.heads_p, p.G - 1);
            const uint16_t *q = static_cast<const uint16_t *>(p.q) + (long long)(s.row0 + j0 + tok) * p.q_stride + (long long)(head * p.G + gh) * p.D;
            const uint4 v = lane * 8 < p.D ? __ldg(reinterpret_cast<const uint4 *>(q) + lane) : make_uint4(0, 0, 0, 0);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            float x[8], top = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint16_t b = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
                x[i] = z.f16 ? Elt<__half>::from(b) : Elt<__nv_bfloat16>::from(b);
                x[i] = x[i] != x[i] ? 0.0f : fminf(fmaxf(x[i], -127.0f * 0x1p113f), 127.0f * 0x1p113f);
                top = fmaxf(top, fabsf(x[i]));
            }
            const int f = code_exponent(__uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top))));
            const float unit_inv = power_of_two(-f);
            uint32_t up[2] = {0, 0}, down[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = __float2int_rn(x[i] * unit_inv);
                up[i / 4] |= (uint32_t)max(c, 0) << (8 * (i & 3));
                down[i / 4] |= ((uint32_t)min(c, 0) & 255u) << (8 * (i & 3));
            }
            unsigned char *dst = codes + r * z.stride;
            if (lane * 8 < p.D) {
                *reinterpret_cast<uint2 *>(dst + lane * 8) = make_uint2(up[0], up[1]);
                *reinterpret_cast<uint2 *>(dst + p.D + lane * 8) = make_uint2(down[0], down[1]);
            }
            for (int i = 2 * p.D + lane * 8; i < SPANS * 64; i += 256) *reinterpret_cast<uint2 *>(dst + i) = make_uint2(0, 0);
            if (lane == 0) units_s[r] = power_of_two(f);
        }
        Codes even, odd;
        if (AHEAD) {
            fetch(id, even);
            id = id_of(warp + SELECT_WARPS);
        }
        __syncthreads();
        auto multiply = [&](int m, const Codes &x) {
            const float e[2] = {power_of_two(x.e[0]), power_of_two(x.e[1])};
            const int i0 = m * 16 + g;
            const bool in[2] = {i0 < count, i0 + 8 < count};
            for (int n0 = 0; n0 < rows; n0 += NT * 8) {
                int c[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    c[nt][0] = c[nt][1] = c[nt][2] = c[nt][3] = 0;
                    if (n0 + nt * 8 < rows) {
                        const unsigned char *src = codes + (n0 + nt * 8 + g) * z.stride + t4 * 16;
#pragma unroll
                        for (int sp = 0; sp < SPANS; ++sp) {
                            const uint4 b = *reinterpret_cast<const uint4 *>(src + sp * 64);
                            mma_s8(c[nt], x.a[sp][0].x, x.a[sp][1].x, x.a[sp][0].y, x.a[sp][1].y, b.x, b.y);
                            mma_s8(c[nt], x.a[sp][0].z, x.a[sp][1].z, x.a[sp][0].w, x.a[sp][1].w, b.z, b.w);
                        }
                    }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int r = n0 + nt * 8 + 2 * t4;  // this lane's rows: r, r + 1
                    if (n0 + nt * 8 >= rows) break;
                    // dot * 2^e * 2^f, the smaller power first: exact, and beyond the type's range only where the score is
                    const float2 f = *reinterpret_cast<const float2 *>(units_s + r);
                    float v[2][2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        v[h][0] = (float)c[nt][2 * h] * fminf(e[h], f.x) * fmaxf(e[h], f.x);
                        v[h][1] = (float)c[nt][2 * h + 1] * fminf(e[h], f.y) * fmaxf(e[h], f.y);
                    }
                    auto put = [&](int list, int h, float score) {
                        if (list < z.tile && in[h]) {
                            uint32_t k = ordered(score);
                            uint32_t &at = key_at(list, i0 + 8 * h);
                            if (z.heads_p > 8 && (row0 + n0 + nt * 8) % z.heads_p) k = max(k, at);  // a token's later rows
                            at = k;
                            least_k = min(least_k, k);
                            most_k = max(most_k, k);
                        }
                    };
                    const int list = z.heads_p > 8 ? (row0 + n0 + nt * 8) / z.heads_p : (row0 + r) >> hp_shift;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (hp_shift == 0) {
                            put(list, h, v[h][0]);
                            put(list + 1, h, v[h][1]);
                            continue;
                        }
                        float best = fmaxf(v[h][0], v[h][1]);
                        if (hp_shift >= 2) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 1));
                        if (hp_shift >= 3) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, 2));
                        if ((2 * t4 & ((1 << hp_shift) - 1)) == 0) put(list, h, best);
                    }
                }
            }
        };
        for (int m = warp; m * 16 < count; m += SELECT_WARPS) {
            if (AHEAD) {  // two m-tiles a round, so that no codes have to be moved from where they were loaded to
                fetch(id, odd);
                id = id_of(m + 2 * SELECT_WARPS);
                multiply(m, even);
                m += SELECT_WARPS;
                if (m * 16 >= count) break;
                fetch(id, even);
                id = id_of(m + 2 * SELECT_WARPS);
                multiply(m, odd);
            } else {
                fetch(id, even);
                id = id_of(m + SELECT_WARPS);
                multiply(m, even);
            }
        }
    }
    least_k = __reduce_min_sync(0xffffffffu, least_k);
    most_k = __reduce_max_sync(0xffffffffu, most_k);
    if (lane == 0) {
        atomicMin(&range_s[0], least_k);
        atomicMax(&range_s[1], most_k);
    }
    sync_all();

    // ---- selection: a list is looked after by `team` warps, each with a piece of the CTA's stretch.  The leading bits that all scores
    // have in common are skipped; then eight bits a pass.  want_s: -1 every block is taken; -2 those from prefix_s on; 0 none of the
    // middle; else those above prefix_s and so many of those equal to it.
    const int team = max(1, SELECT_WARPS / z.tile), wl = warp % team, lists_at_once = SELECT_WARPS / team;
    const int piece = ((count + team - 1) / team + 31) / 32 * 32, i0 = min(wl * piece, count), i1 = min(i0 + piece, count);
    if (z.ctas > 1) {
        uint2 r = make_uint2(0xffffffffu, 0);
        if (lane < z.ctas) r = peer_pair(peer_addr((uint32_t)__cvta_generic_to_shared(range_s), lane));
        least_k = __reduce_min_sync(0xffffffffu, r.x);
        most_k = __reduce_max_sync(0xffffffffu, r.y);
    } else {
        least_k = range_s[0];
        most_k = range_s[1];
    }
    int shift = 32 - __clz(least_k ^ most_k);  // bits that are not decided
    const uint32_t common = shift == 32 ? 0 : least_k >> shift << shift;
    for (int pass = 0; shift > 0; ++pass) {
        const int width = min(shift, 8);
        shift -= width;
        uint32_t *now = hist + (pass & 1) * z.tile * 256, *next = hist + (~pass & 1) * z.tile * 256;
        bool any = false;
        for (int list = 0; list < tokens; ++list) any |= want_s[list] > 0;
        if (!any) break;  // the same in all CTAs of the cluster
        for (int list = warp / team; list < tokens; list += lists_at_once) {
            if (want_s[list] <= 0) continue;
            const uint32_t prefix = (common | prefix_s[list]) >> shift >> width, mask = (1u << width) - 1;
            const int lo = max(i0, p.sink - b0), hi = min(i1, last_s[list] + 1 - p.recent - b0);
            for (int i = lo + lane; i < hi; i += 128) {
                uint32_t k[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) k[e] = i + 32 * e < hi ? key_at(list, i + 32 * e) : 0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + 32 * e < hi && k[e] >> shift >> width == prefix) atomicAdd(now + list * 256 + (k[e] >> shift & mask), 1u);
            }
        }
        sync_all();
        for (int i = threadIdx.x; i < z.tile * 256; i += SELECT_WARPS * 32) next[i] = 0;
        for (int list = warp / team; list < tokens; list += lists_at_once) {
            const int want = want_s[list];
            if (want <= 0 || wl) continue;
            uint32_t n[8], before[8];  // in all CTAs, in those with earlier stretches
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(now + list * 256 + lane * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) n[i] = before[i] = 0;
            if (z.ctas > 1) {
                uint4 v[8][2];  // all under way at once
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < z.ctas) {
                        const uint32_t there = peer_addr(at, c);
                        v[c][0] = peer_words(there);
                        v[c][1] = peer_words(there + 16);
                    }
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    if (c >= z.ctas) break;
                    const uint32_t w[8] = {v[c][0].x, v[c][0].y, v[c][0].z, v[c][0].w, v[c][1].x, v[c][1].y, v[c][1].z, v[c][1].w};
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        n[i] += w[i];
                        if (c < cta) before[i] += w[i];
                    }
                }
            } else {
                const uint4 a = lds16(at), b = lds16(at + 16);
                n[0] = a.x; n[1] = a.y; n[2] = a.z; n[3] = a.w;
                n[4] = b.x; n[5] = b.y; n[6] = b.z; n[7] = b.w;
            }
            uint32_t mine = 0, mine_before = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                mine += n[i];
                mine_before += before[i];
            }
            uint32_t above = mine, above_before = mine_before;  // of this lane's digits and larger ones
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t v = __shfl_down_sync(0xffffffffu, above, d), w = __shfl_down_sync(0xffffffffu, above_before, d);
                if (lane + d < 32) {
                    above += v;
                    above_before += w;
                }
            }
            above -= mine;
            above_before -= mine_before;
            if ((int)above < want && want <= (int)(above + mine)) {  // one lane
                uint32_t left = (uint32_t)want - above, here = 0, here_before = 0;
                int digit = 7;
#pragma unroll
                for (int i = 7; i >= 0; --i) {
                    if (digit == i && left > n[i]) {
                        left -= n[i];
                        above_before += before[i];
                        digit = i - 1;
                    }
                    if (digit == i) {
                        here = n[i];
                        here_before = before[i];
                    }
                }
                prefix_s[list] |= common | (uint32_t)(lane * 8 + digit) << shift;
                // all with these bits are taken: the threshold is the smallest number with them
                want_s[list] = here == left ? -2 : (int)left;
                before_s[list][0] += above_before + (here == left ? here_before : 0);
                before_s[list][1] = here_before;
            }
        }
        __syncthreads();
    }
    // nobody reads this CTA's memory any more once all have come here; they need not wait for its lists
    if (z.ctas > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    struct Rule {
        int first, end, want, last;  // of the middle, within the stretch
        uint32_t least;
    };
    auto rule_of = [&](int list) {
        const int last = last_s[list], want = want_s[list];
        Rule r{p.sink - b0, last + 1 - p.recent - b0, want, last - b0, common | prefix_s[list]};
        if (want == -1) r.end = -0x7fffffff;  // everything counts as first or last
        return r;
    };
    auto kind_of = [&](const Rule &r, int list, int i, bool &tie) -> bool {  // certainly taken
        tie = false;
        if (i > r.last) return false;
        if (i < r.first || i >= r.end) return true;
        const uint32_t k = key_at(list, i);
        if (r.want == -2) return k >= r.least;
        tie = r.want > 0 && k == r.least;
        return r.want > 0 && k > r.least;
    };
    if (team > 1) {  // a warp's piece comes behind those of the warps before it
        const int list = warp / team;
        uint32_t sure = 0, ties = 0;
        if (list < tokens) {
            const Rule rule = rule_of(list);
            for (int i = i0 + lane; i < i1; i += 32) {
                bool tie;
                sure += kind_of(rule, list, i, tie);
                ties += tie;
            }
        }
        sure = __reduce_add_sync(0xffffffffu, sure);
        ties = __reduce_add_sync(0xffffffffu, ties);
        if (lane == 0) {
            counts_s[warp][0] = sure;
            counts_s[warp][1] = ties;
        }
        __syncthreads();
    }
    for (int list = warp / team; list < tokens; list += lists_at_once) {
        const Rule rule = rule_of(list);
        const int ties_taken = max(rule.want, 0), own = last_s[list];
        // taken in earlier stretches: all of them, or the first, the last and those above the threshold
        uint32_t sure = rule.want == -1 ? (uint32_t)min(b0, own + 1)
                                        : (uint32_t)(min(b0, p.sink) + max(0, min(b0, own + 1) - (own + 1 - p.recent))) + before_s[list][0];
        uint32_t ties = before_s[list][1];
        if (least_k == most_k) ties = max(0, min(b0, own + 1 - p.recent) - p.sink);  // no pass: the middle is all equal
        if (rule.want <= 0) ties = 0;
        for (int w = 0; w < wl; ++w) {
            sure += counts_s[warp - wl + w][0];
            ties += counts_s[warp - wl + w][1];
        }
        const long long at0 = ((long long)(s.row0 + j0 + list) * p.H + head) * p.keep;
        for (int base = i0; base < i1; base += 32) {
            const int i = base + lane;
            bool tie = false;
            const bool certain = i < i1 && kind_of(rule, list, i, tie);
            const unsigned cm = __ballot_sync(0xffffffffu, certain), tm = __ballot_sync(0xffffffffu, tie), under = (1u << lane) - 1;
            const int ties_before = (int)ties + __popc(tm & under);
            if (certain || (tie && ties_before < ties_taken)) {
                const int to = (int)sure + __popc(cm & under) + min(ties_before, ties_taken);
                p.blocks[at0 + to] = b0 + i;
                if (p.scores) p.scores[at0 + to] = from_ordered(key_at(list, i));
            }
            sure += __popc(cm);
            ties += __popc(tm);
        }
        if (cta == 0)
            for (int i = min(p.keep, own + 1) + wl * 32 + lane; i < p.keep; i += team * 32) {
                p.blocks[at0 + i] = -1;
                if (p.scores) p.scores[at0 + i] = -CUDART_INF_F;
            }
    }
    if (z.ctas > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

static size_t select_smem(const SelectShape &z) { return (size_t)z.tile * z.room * 4 + (size_t)2 * z.tile * 256 * 4 + (size_t)z.rows * z.stride; }
constexpr size_t SELECT_SMEM = 220 * 1024;

// How a batch is cut: tokens of a tile, CTAs of a cluster.
SelectShape select_shape(const SelectParams &p, int max_nq, long long tokens, int sm_count, int f16) {
    SelectShape z{};
    z.f16 = f16;
    z.heads_p = p.G > 8 ? (p.G + 7) / 8 * 8 : (p.G > 4 ? 8 : (p.G > 2 ? 4 : p.G));
    const int spans = p.D <= 64 ? 2 : (p.D <= 128 ? 4 : 8);
    z.stride = spans * 64 + 64;
    for (z.tile = 1; z.tile < SELECT_TOKENS && z.tile < max_nq && 2 * z.tile * z.heads_p <= SELECT_ROWS; z.tile *= 2) {}
    for (;;) {
        z.rows = std::min((z.tile * z.heads_p + 7) / 8 * 8, SELECT_ROWS);
        const long long units = (tokens + z.tile - 1) / z.tile * p.H;
        for (z.ctas = 1;; z.ctas *= 2) {
            z.room = ((p.widest + z.ctas - 1) / z.ctas + 15) / 16 * 16;
            if (z.ctas == 8) break;
            const bool fits = select_smem(z) <= SELECT_SMEM / 2;  // two CTAs an SM
            if (fits && (units * z.ctas * 2 > 2ll * sm_count || z.room <= 256)) break;
        }
        if (z.tile == 1 || select_smem(z) <= SELECT_SMEM) return z;
        z.tile /= 2;
    }
}

template <int SPANS, int NT> static cudaError_t select_go(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, cudaStream_t st) {
    static SmemSeen seen{0};
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(select_blocks_kernel<SPANS, NT>), (int)SELECT_SMEM, &seen);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute cluster;
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = (unsigned)z.ctas;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(units * p.H * z.ctas));
    cfg.blockDim = dim3(SELECT_WARPS * 32);
    cfg.dynamicSmemBytes = select_smem(z);
    cfg.stream = st;
    cfg.attrs = &cluster;
    cfg.numAttrs = z.ctas > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, select_blocks_kernel<SPANS, NT>, p, small, z);
    return e != cudaSuccess ? e : cudaGetLastError();
}
template <int SPANS> static cudaError_t select_rows(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, cudaStream_t st) {
    return z.rows <= 8 ? select_go<SPANS, 1>(p, small, z, units, st) : (z.rows <= 16 ? select_go<SPANS, 2>(p, small, z, units, st) : select_go<SPANS, 4>(p, small, z, units, st));
}
cudaError_t launch_select_blocks(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, cudaStream_t st) {
    return p.D <= 64 ? select_rows<2>(p, small, z, units, st) : (p.D <= 128 ? select_rows<4>(p, small, z, units, st) : select_rows<8>(p, small, z, units, st));
}

}  // namespace aafkv
