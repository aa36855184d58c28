// The blocks of a context with the largest bound on a query's scores, for every query token and kv head.
//
//   q_d in steps of 2^f: c_d = rint(F(q_d) / 2^f), |c_d| <= 127;   dot_b = sum_d max(c_d hi_bd, c_d lo_bd)
//   score_b = max over the group's heads of dot_b * 2^(e_b + f)
//
// max(c hi, c lo) = max(c, 0) hi + min(c, 0) lo: a product of [c+, c-] with the block's [hi, lo], in whole numbers, exact in any
// order, and so is the scaling by a power of two; equal scores go to the lower block.
//
// Two kernels.  Scores: 128 blocks as the M side of 8-bit products on the fifth-generation tensor cores, the rows of a tile of query
// tokens as the N side, sums in tensor memory, where a thread finds all of a block's and takes the largest of every token's heads.  A CTA
// takes a kv head; those of one tile follow one another in the grid, so that the pieces of a block's record are asked for together.
// Selection: a CTA a list; the smallest score that is taken is found by histograms of eight bits, starting behind the bits that all
// scores share; a list's scores come from L2 and stay in shared memory where they fit.
//
// Bound: the bytes of the summaries where there is a token each (and the start of the two kernels); latency of the passes of the
// selection where there are many tokens.
#include "sparse_device.cuh"
#include "tensor_device.cuh"

namespace aafkv {

constexpr int SCORE_BLOCKS = 128;  // of an m-tile
constexpr int PICK_WARPS = 8, PICK_KEYS = 12288;  // scores of a list that are kept in shared memory

// 8-bit products, 32-bit sums
__device__ __forceinline__ void mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// HP: log2 of the rows that a token has in a stretch of 32 columns (its group's heads, repeated up to a power of two); THREADS: 128 for
// 32 rows or tokens of more, 256 for more rows
template <int HP, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 128 ? 5 : 3)
    score_blocks_kernel(const __grid_constant__ SelectParams p, const __grid_constant__ SmallSeqs small, const __grid_constant__ SelectShape z) {
    extern __shared__ unsigned char smem[];  // codes of the blocks (z.buffers of z.slabs * 16 KB), of the rows (z.slabs * z.n * 128)
    __shared__ __align__(8) uint64_t bar;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_s;
    __shared__ __align__(16) float units_s[SELECT_ROWS];  // of a row's codes: 2^(f - 64)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // First of all: the SM's next CTA does not start before this one has given up the right to allocate
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         (uint32_t)__cvta_generic_to_shared(&tmem_s)), "r"(z.n) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("griddepcontrol.launch_dependents;");
    const int unit = blockIdx.x / p.H, head = blockIdx.x - unit * p.H;
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq s = seqs[find_seq(seqs, p.n, unit)];
    const int tile = (unit - s.unit0) / s.nsplit, group = unit - s.unit0 - tile * s.nsplit;
    const int j0 = tile * z.tile, tokens = min(z.tile, s.nq - j0);
    const int total = (s.key0 + j0 + tokens - 1) / p.BS + 1;  // blocks that some token of the tile may take
    const int first = group * z.reps * SCORE_BLOCKS, m_tiles = min(z.reps, (total - first + SCORE_BLOCKS - 1) / SCORE_BLOCKS);
    if (m_tiles <= 0) {  // behind the tile's blocks
        if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_s), "r"(z.n));
        return;
    }
    const uint32_t s_0 = (uint32_t)__cvta_generic_to_shared(smem), s_a = (s_0 + 1023) & ~1023u, a_bytes = z.slabs * SCORE_BLOCKS * 128;
    const uint32_t s_b = s_a + z.buffers * a_bytes, s_bar = (uint32_t)__cvta_generic_to_shared(&bar);
    if (warp == 0) {
        if (lane == 0) {
            bar_init(s_bar, 1);
            abort_s = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    }

    // a warp copies the codes of OWN of an m-tile's blocks, 16 bytes a lane; a thread takes the sums of one block, every other 32 rows where
    // there are two threads for each
    constexpr int OWN = SCORE_BLOCKS / (THREADS / 32);
    const int *table = p.tables + (long long)s.ctx * p.max_blk;
    const int pieces = p.D / 8;  // of a block's codes, 16 bytes each
    auto block_id = [&](int m) { return __ldg(table + min(first + m * SCORE_BLOCKS + warp * OWN + (lane & (OWN - 1)), total - 1)); };
    const signed char *codes = p.summary + (long long)head * 2 * p.D;
    auto issue = [&](int m, int id) {
        const uint32_t dst = s_a + (m % z.buffers) * a_bytes + warp * (OWN * 128);
        auto copy = [&](int r, int c) {
            copy16(dst + (c >> 3) * (SCORE_BLOCKS * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4),
                   codes + (long long)__shfl_sync(0xffffffffu, id, r) * p.record + c * 16, 16);
        };
        // all lanes take part in every step, since they ask one another for the block
        if (32 % pieces == 0 && 32 / pieces <= OWN) {  // steps of whole rows
            const int at_once = 32 / pieces, c = lane & (pieces - 1), r0 = lane / pieces;
#pragma unroll 4
            for (int step = 0; step < OWN; step += at_once) copy(step + r0, c);
        } else {
            for (int i0 = 0; i0 < OWN * pieces; i0 += 32) {
                const int i = min(i0 + lane, OWN * pieces - 1);  // the last lanes may copy the same
                copy(i / pieces, i % pieces);
            }
        }
        copy_commit();
    };
    const int rows_token = z.heads_p, rows_all = tokens * rows_token;
    const int list_of_tile = s.tok0 + j0, mine = threadIdx.x & (SCORE_BLOCKS - 1);
    const long long list_pitch = p.H * p.pitch;
    bool ok = true;
    int parity = 0;
    const uint32_t idesc = 2u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(z.n / 8) << 17 | (SCORE_BLOCKS / 16) << 24;
    // a pass takes z.n rows: one, but for groups of more heads than that
    for (int row0 = 0; row0 < rows_all; row0 += z.n) {
        const int rows = min(z.n, rows_all - row0);
        if (row0) __syncthreads();
        const int lanes = p.D <= 128 ? 16 : 32, sub = lane & (lanes - 1);  // of a row, eight channels each
        const unsigned row_mask = lanes == 32 ? 0xffffffffu : 0xffffu << (lane & 16);
        constexpr int BATCH = THREADS == 128 ? 1 : 4;  // rows whose loads are under way together
        uint4 v[BATCH];
        auto load = [&](int base) {
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int rr = row0 + min(base + b * (THREADS / lanes), rows - 1), tok = HP == 5 ? rr / rows_token : rr >> HP;
                const uint16_t *q = static_cast<const uint16_t *>(p.q) + (long long)(s.row0 + j0 + tok) * p.q_stride +
                                    (long long)(head * p.G + min(rr - tok * rows_token, p.G - 1)) * p.D;
                v[b] = sub * 8 < p.D ? __ldg(reinterpret_cast<const uint4 *>(q) + sub) : make_uint4(0, 0, 0, 0);
            }
        };
        int id = block_id(0);
        load(threadIdx.x / lanes);  // under way beside the first block numbers
        issue(0, id);
        for (int base = threadIdx.x / lanes; base < (rows + 1) / 2 * 2; base += BATCH * (THREADS / lanes)) {
            if (base >= BATCH * (THREADS / lanes)) load(base);
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {  // a row's codes: [c+, c-], zeros up to a multiple of 32
                const int r = base + b * (THREADS / lanes);
                if (r >= (rows + 1) / 2 * 2) break;
                const uint32_t w[4] = {v[b].x, v[b].y, v[b].z, v[b].w};
                float x[8], top = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint16_t y = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
                    x[i] = z.f16 ? Elt<__half>::from(y) : Elt<__nv_bfloat16>::from(y);
                    x[i] = x[i] != x[i] ? 0.0f : fminf(fmaxf(x[i], -127.0f * 0x1p113f), 127.0f * 0x1p113f);
                    top = fmaxf(top, fabsf(x[i]));
                }
                const int f = code_exponent(__uint_as_float(__reduce_max_sync(row_mask, __float_as_uint(top))));
                const float unit_inv = power_of_two(-f);
                uint32_t up[2] = {0, 0}, down[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = __float2int_rn(x[i] * unit_inv);
                    up[i / 4] |= (uint32_t)max(c, 0) << (8 * (i & 3));
                    down[i / 4] |= ((uint32_t)min(c, 0) & 255u) << (8 * (i & 3));
                }
                unsigned char *dst = smem + (s_b - s_0) + r * 128;
                auto place = [&](int at) { return (at >> 7) * z.n * 128 + (((at >> 4 & 7) ^ (r & 7)) << 4) + (at & 15); };
                if (sub * 8 < p.D) {
                    *reinterpret_cast<uint2 *>(dst + place(sub * 8)) = make_uint2(up[0], up[1]);
                    *reinterpret_cast<uint2 *>(dst + place(p.D + sub * 8)) = make_uint2(down[0], down[1]);
                }
                if (2 * p.D % 32 && sub < 2) *reinterpret_cast<uint2 *>(dst + place(2 * p.D + sub * 8)) = make_uint2(0, 0);
                if (sub == 0) units_s[r] = power_of_two(f - 64);
            }
        }
        for (int m = 0; m < m_tiles; ++m) {
            const int e = __ldg(p.summary + (long long)(THREADS == 128 ? id : __ldg(table + min(first + m * SCORE_BLOCKS + mine, total - 1))) * p.record +
                                (long long)p.H * 2 * p.D + head);
            if (m + 1 < m_tiles && z.buffers > 1) {
                id = block_id(m + 1);
                issue(m + 1, id);
                copy_wait<1>();
            } else {
                copy_wait<0>();
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tmem_before();
            __syncthreads();
            tmem_after();
            const uint32_t tmem = tmem_s;
            if (warp == 0 && elected()) {
                const uint64_t da = smem_desc(s_a + (m % z.buffers) * a_bytes, 16, 1024), db = smem_desc(s_b, 16, 1024);
                const int steps = (2 * p.D + 31) / 32;
                for (int k = 0; k < steps; ++k)
                    mma_i8(tmem, da + (k >> 2) * (SCORE_BLOCKS * 128 >> 4) + 2 * (k & 3), db + (k >> 2) * (z.n * 128 >> 4) + 2 * (k & 3), idesc, k > 0);
                mma_commit(s_bar);
            }
            __syncwarp();
            ok = warp_wait(s_bar, parity, &abort_s, p.status) && ok;
            parity ^= 1;
            tmem_after();
            // dot * 2^(f - 64), the largest of a token's heads, * 2^(e + 64): exact, beyond the type's range only where the score is
            const float m1 = power_of_two(e < 0 ? e + 64 : 64), m2 = power_of_two(e < 0 ? 0 : e);
            const int block = first + m * SCORE_BLOCKS + mine;
            uint32_t *dst = p.keys + ((long long)list_of_tile * p.H + head) * p.pitch + block;
            for (int c0 = threadIdx.x / SCORE_BLOCKS * 32; c0 < rows; c0 += THREADS / SCORE_BLOCKS * 32) {
                float x[32];
                tmem_ld32(tmem + ((uint32_t)((warp & 3) * 32) << 16) + c0, x);
                tmem_wait_ld();
#pragma unroll
                for (int t = 0; t < 32 >> HP; ++t) {
                    const int row = row0 + c0 + (t << HP);
                    if (row >= rows_all) break;
                    float best = -CUDART_INF_F;
#pragma unroll
                    for (int i = t << HP; i < (t + 1) << HP; ++i) best = fmaxf(best, (float)__float_as_int(x[i]) * units_s[c0 + i]);
                    const uint32_t k = ordered(best * m1 * m2);
                    if (block < total) {
                        uint32_t &at = dst[(HP == 5 ? row / rows_token : row >> HP) * list_pitch];
                        at = HP == 5 && row % rows_token ? max(at, k) : k;  // a token of more than 32 heads: this thread has written `at`
                    }
                }
            }
            tmem_before();
            __syncthreads();  // sums and codes have been read
            tmem_after();
            if (m + 1 < m_tiles && z.buffers == 1) {
                id = block_id(m + 1);
                issue(m + 1, id);
            }
        }
    }
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_s), "r"(z.n));
}

// A list from its scores: the first `sink`, the last `recent`, the best others.  The scores of the middle are looked through three times:
// for their range; for a histogram of the eight bits behind those that all share, which finds the digit of the smallest score that is
// taken; and for the few that have this digit, among which a warp finds it.  (Where they are many, further histograms do.)  Then every
// warp writes what its piece of the context contributes.
constexpr int PICK_FEW = 128;
template <int WARPS>
__global__ void __launch_bounds__(WARPS * 32)
    pick_blocks_kernel(const __grid_constant__ SelectParams p, const __grid_constant__ SmallSeqs small, int room) {
    extern __shared__ __align__(16) uint32_t keys_s[];
    __shared__ __align__(16) uint32_t hist[4][256];
    __shared__ uint32_t range_s[2], counts_s[WARPS][2], few_s[PICK_FEW], few_count, least_s;
    __shared__ int want_s;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int token = blockIdx.x / p.H, head = blockIdx.x - token * p.H;  // tokens of this launch
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    int lo = 0, hi = p.n - 1;  // record of the token
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (seqs[mid].tok0 <= token) lo = mid; else hi = mid - 1;
    }
    const AttnSeq s = seqs[lo];
    const int j = token - s.tok0, total = (s.key0 + j) / p.BS + 1;
    for (int i = threadIdx.x; i < 4 * 256; i += WARPS * 32) hist[0][i] = 0;
    if (threadIdx.x == 0) {
        range_s[0] = 0xffffffffu;
        range_s[1] = few_count = 0;
    }
    const uint32_t *scores = p.keys + (long long)blockIdx.x * p.pitch;
    int *out = p.blocks + ((long long)(s.row0 + j) * p.H + head) * p.keep;
    float *out_s = p.scores ? p.scores + ((long long)(s.row0 + j) * p.H + head) * p.keep : nullptr;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the scores are written
    if (total <= p.keep) {  // every block
        for (int i = threadIdx.x; i < p.keep; i += WARPS * 32) {
            out[i] = i < total ? i : -1;
            if (out_s) out_s[i] = i < total ? from_ordered(__ldcg(scores + i)) : -CUDART_INF_F;
        }
        return;
    }
    const int m0 = p.sink, m1 = total - p.recent;  // the middle
    const bool stay = total <= room;
    int want = p.keep - p.sink - p.recent;
    uint32_t least = 0xffffffffu;  // what is taken of the middle: scores above it, and the first `want` equal to it
    // scores i ... i + 3, 0 (below all scores) outside the middle
    auto four = [&](int i) {
        uint4 v = __ldcg(reinterpret_cast<const uint4 *>(scores + i));
        if (i < m0 || i + 3 >= m1) {
            if (i < m0 || i >= m1) v.x = 0;
            if (i + 1 < m0 || i + 1 >= m1) v.y = 0;
            if (i + 2 < m0 || i + 2 >= m1) v.z = 0;
            if (i + 3 < m0 || i + 3 >= m1) v.w = 0;
        }
        return v;
    };
    auto again = [&](int i) { return stay ? *reinterpret_cast<const uint4 *>(keys_s + i) : four(i); };
    // a warp's piece: blocks i0 ... i1, a lane looks at four at a time
    const int piece = ((total + WARPS - 1) / WARPS + 127) / 128 * 128, i0 = min(warp * piece, total), i1 = min(i0 + piece, total);
    if (want > 0 || stay) {
        uint32_t a = 0xffffffffu, b = 0;
        for (int i = i0 + lane * 4; i < i1; i += 128) {
            const uint4 v = four(i);
            if (stay) *reinterpret_cast<uint4 *>(keys_s + i) = v;
            a = min(min(a, min(v.x - 1, v.y - 1)), min(v.z - 1, v.w - 1));  // a 0 becomes the largest number
            b = max(max(b, max(v.x, v.y)), max(v.z, v.w));
        }
        a = __reduce_min_sync(0xffffffffu, a);
        b = __reduce_max_sync(0xffffffffu, b);
        if (lane == 0) {
            atomicMin(&range_s[0], a);
            atomicMax(&range_s[1], b);
        }
    }
    __syncthreads();
    if (want > 0) {
        const uint32_t a = range_s[0] + 1, b = range_s[1];
        int shift = 32 - __clz(a ^ b);  // bits that are not decided
        least = shift == 32 ? 0 : a >> shift << shift;
        for (int pass = 0; shift > 0; ++pass) {
            const int width = min(shift, 8);
            shift -= width;
            const uint32_t prefix = least >> shift >> width, mask = (1u << width) - 1;
            for (int i = i0 + lane * 4; i < i1; i += 128) {
                const uint4 v = again(i);
                auto count = [&](uint32_t k) {
                    if (k && k >> shift >> width == prefix) atomicAdd(&hist[pass][k >> shift & mask], 1u);
                };
                count(v.x);
                count(v.y);
                count(v.z);
                count(v.w);
            }
            __syncthreads();
            // every warp looks for the digit: a lane sees eight of them
            const uint4 h0 = *reinterpret_cast<const uint4 *>(&hist[pass][lane * 8]), h1 = *reinterpret_cast<const uint4 *>(&hist[pass][lane * 8 + 4]);
            const uint32_t n[8] = {h0.x, h0.y, h0.z, h0.w, h1.x, h1.y, h1.z, h1.w};
            uint32_t mine = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) mine += n[i];
            uint32_t above = mine;  // of this lane's digits and larger ones
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t v = __shfl_down_sync(0xffffffffu, above, d);
                if (lane + d < 32) above += v;
            }
            above -= mine;
            const bool here = (int)above < want && want <= (int)(above + mine);  // one lane
            int left = want - (int)above, digit = 7, equal = 0;
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                if (digit == i && left > (int)n[i]) {
                    left -= (int)n[i];
                    digit = i - 1;
                }
                if (digit == i) equal = (int)n[i];
            }
            const int who = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
            want = __shfl_sync(0xffffffffu, left, who);
            least |= (uint32_t)__shfl_sync(0xffffffffu, lane * 8 + digit, who) << shift;
            const int have = __shfl_sync(0xffffffffu, equal, who);
            if (shift == 0) break;
            if (have == want) {  // all of them are taken
                least = max(least, 1u) - 1;  // scores are above 0
                want = 0;
                break;
            }
            if (have > PICK_FEW) continue;
            const uint32_t wanted = least >> shift;
            for (int i = i0 + lane * 4; i < i1; i += 128) {
                const uint4 v = again(i);
                auto gather = [&](uint32_t k) {
                    if (k && k >> shift == wanted) few_s[atomicAdd(&few_count, 1u)] = k;
                };
                gather(v.x);
                gather(v.y);
                gather(v.z);
                gather(v.w);
            }
            __syncthreads();
            // the smallest that is taken: fewer than `want` are larger, at least as many are not smaller
            if (threadIdx.x < PICK_FEW) {
                const int me = threadIdx.x;
                if (me < have) {
                    const uint32_t k = few_s[me];
                    int larger = 0, same = 0;
                    for (int i = 0; i < have; ++i) {
                        larger += few_s[i] > k;
                        same += few_s[i] == k;
                    }
                    if (larger < want && want <= larger + same) {  // equal scores all write the same
                        least_s = k;
                        want_s = want - larger;
                    }
                }
            }
            __syncthreads();
            least = least_s;
            want = want_s;
            break;
        }
    }
    // taken for certain and equal to the threshold, in this warp's piece: how many, then which
    auto kinds = [&](int i, const uint4 &v) {  // of blocks i ... i + 3: bits 0 ... 3, 16 ... 19
        const uint32_t k[4] = {v.x, v.y, v.z, v.w};
        uint32_t r = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (k[e] > least) r |= 1u << e;
            if (k[e] == least) r |= 0x10000u << e;
        }
        if (i < m0 || i + 3 >= m1) {  // the first and the last ones
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < i1 && (i + e < m0 || i + e >= m1)) r |= 1u << e;
        }
        return r;
    };
    uint32_t sure = 0, ties = 0;
    for (int i = i0 + lane * 4; i < i1; i += 128) {
        const uint32_t r = kinds(i, again(i));
        sure += __popc(r & 0xffffu);
        ties += __popc(r >> 16);
    }
    sure = __reduce_add_sync(0xffffffffu, sure);
    ties = __reduce_add_sync(0xffffffffu, ties);
    if (lane == 0) {
        counts_s[warp][0] = sure;
        counts_s[warp][1] = ties;
    }
    __syncthreads();
    const uint32_t taken = sure + ties;
    sure = ties = 0;
    for (int w = 0; w < warp; ++w) {
        sure += counts_s[w][0];
        ties += counts_s[w][1];
    }
    if (taken)
        for (int base = i0; base < i1; base += 128) {
            const int i = base + lane * 4;
            const uint4 v = i < i1 ? again(i) : make_uint4(0, 0, 0, 0);
            const uint32_t r = i < i1 ? kinds(i, v) : 0u, k[4] = {v.x, v.y, v.z, v.w};
            if (!__any_sync(0xffffffffu, r)) continue;
            const uint32_t mine = __popc(r & 0xffffu) | __popc(r >> 16) << 16;
            uint32_t upto = mine;  // of this lane and those before it
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t w = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += w;
            }
            const uint32_t whole = __shfl_sync(0xffffffffu, upto, 31);
            int s_at = (int)sure + (int)((upto - mine) & 0xffffu), t_at = (int)ties + (int)((upto - mine) >> 16);
            if (r)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool certain = r >> e & 1, tie = r >> (16 + e) & 1;
                    if (certain || (tie && t_at < want)) {
                        const int to = s_at + min(t_at, want);
                        out[to] = i + e;
                        if (out_s) out_s[to] = from_ordered(i + e < m0 || i + e >= m1 ? __ldcg(scores + i + e) : k[e]);
                    }
                    s_at += certain;
                    t_at += tie;
                }
            sure += whole & 0xffffu;
            ties += whole >> 16;
        }
}

static size_t score_smem(const SelectShape &z) { return (size_t)z.slabs * 128 * (z.buffers * SCORE_BLOCKS + z.n) + 1024; }
constexpr int SCORE_SMEM = (4 * 128 * (2 * SCORE_BLOCKS + SELECT_ROWS)) + 1024;

// How a batch is cut.  Rows of a tile: 32 where there is a token each (the sums' columns that a thread reads at once), else as many as
// the tokens fill, up to SELECT_ROWS.  A CTA takes so many m-tiles in turn that the CTAs are all there at once: its start (memory, record,
// rows' codes) costs as much as several of them.
SelectShape select_shape(const SelectParams &p, int n, int max_nq, long long m_tiles, int sm_count, int f16) {
    SelectShape z{};
    z.f16 = f16;
    z.heads_p = p.G > 32 ? (p.G + 31) / 32 * 32 : 1;
    while (z.heads_p < p.G) z.heads_p *= 2;
    for (z.n = 32; z.n < SELECT_ROWS && z.n < max_nq * z.heads_p; z.n *= 2) {}
    z.tile = std::max(1, z.n / z.heads_p);
    z.slabs = (2 * p.D + 127) / 128;
    const long long ctas = m_tiles * p.H / std::min(z.tile, max_nq);
    auto room = [&](int buffers) {
        z.buffers = buffers;
        return std::min<long long>(z.n == 32 ? 5 : 3, 227 * 1024 / (long long)(score_smem(z) + 2048)) * sm_count;
    };
    z.reps = 1;
    if (ctas > room(1)) {
        const long long most = std::max(room(2) - (long long)n * p.H / 2, room(2) / 2);  // contexts end with half of a CTA's m-tiles
        z.reps = (int)std::min<long long>(1 << 16, (ctas + most - 1) / most);
        if (z.reps == 1) z.buffers = 1;
    }
    return z;
}

template <int HP, int THREADS>
static cudaError_t score_go(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, cudaStream_t st) {
    static SmemSeen seen{0};
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(score_blocks_kernel<HP, THREADS>), SCORE_SMEM, &seen);
    if (e != cudaSuccess) return e;
    score_blocks_kernel<HP, THREADS><<<(unsigned)(units * p.H), THREADS, score_smem(z), st>>>(p, small, z);
    return cudaGetLastError();
}
template <int HP> static cudaError_t score_rows(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, cudaStream_t st) {
    // a token of more than 32 heads is put together by one thread
    return z.n == 32 || z.heads_p > 32 ? score_go<HP, 128>(p, small, z, units, st) : score_go<HP, 256>(p, small, z, units, st);
}
template <int WARPS> static cudaError_t pick_go(const SelectParams &p, const SmallSeqs &small, long long tokens, cudaStream_t st) {
    // launched so that its CTAs come up while the scores are still being computed; it waits for them itself
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(tokens * p.H));
    cfg.blockDim = dim3(WARPS * 32);
    const int room = p.widest <= PICK_KEYS ? (p.widest + 3) / 4 * 4 : 0;
    cfg.dynamicSmemBytes = (size_t)room * 4;
    cfg.stream = st;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    static SmemSeen seen{0};
    cudaError_t e = allow_smem(reinterpret_cast<const void *>(pick_blocks_kernel<WARPS>), PICK_KEYS * 4, &seen);
    if (e != cudaSuccess) return e;
    e = cudaLaunchKernelEx(&cfg, pick_blocks_kernel<WARPS>, p, small, room);
    return e != cudaSuccess ? e : cudaGetLastError();
}
cudaError_t launch_select_blocks(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, long long tokens, cudaStream_t st) {
    cudaError_t e;
    switch (log2_up(std::min(z.heads_p, 32))) {
        case 0: e = score_rows<0>(p, small, z, units, st); break;
        case 1: e = score_rows<1>(p, small, z, units, st); break;
        case 2: e = score_rows<2>(p, small, z, units, st); break;
        case 3: e = score_rows<3>(p, small, z, units, st); break;
        case 4: e = score_rows<4>(p, small, z, units, st); break;
        default: e = score_rows<5>(p, small, z, units, st); break;
    }
    if (e != cudaSuccess) return e;
    return p.widest <= 1024 ? pick_go<4>(p, small, tokens, st) : pick_go<PICK_WARPS>(p, small, tokens, st);
}

}  // namespace aafkv
