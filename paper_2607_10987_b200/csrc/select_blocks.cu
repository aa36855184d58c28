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
constexpr int SCORE_THREADS = 128, PICK_WARPS = 8, PICK_KEYS = 12288;  // scores of a list that are kept in shared memory

// 8-bit products, 32-bit sums
__device__ __forceinline__ void mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

// HP: log2 of the rows that a token has in a stretch of 32 columns (its group's heads, repeated up to a power of two)
template <int HP>
__global__ void __launch_bounds__(SCORE_THREADS)
    score_blocks_kernel(const __grid_constant__ SelectParams p, const __grid_constant__ SmallSeqs small, const __grid_constant__ SelectShape z) {
    extern __shared__ unsigned char smem[];  // codes of the blocks (z.buffers of z.slabs * 16 KB), of the rows (z.slabs * z.n * 128)
    __shared__ __align__(8) uint64_t bar;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_s;
    __shared__ __align__(16) float units_s[SELECT_ROWS];  // of a row's codes: 2^(f - 64)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    asm volatile("griddepcontrol.launch_dependents;");
    const int unit = blockIdx.x / p.H, head = blockIdx.x - unit * p.H;
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq s = seqs[find_seq(seqs, p.n, unit)];
    const int tile = (unit - s.unit0) / s.nsplit, group = unit - s.unit0 - tile * s.nsplit;
    const int j0 = tile * z.tile, tokens = min(z.tile, s.nq - j0);
    const int total = (s.key0 + j0 + tokens - 1) / p.BS + 1;  // blocks that some token of the tile may take
    const int first = group * z.reps * SCORE_BLOCKS, m_tiles = min(z.reps, (total - first + SCORE_BLOCKS - 1) / SCORE_BLOCKS);
    if (m_tiles <= 0) return;
    const uint32_t s_0 = (uint32_t)__cvta_generic_to_shared(smem), s_a = (s_0 + 1023) & ~1023u, a_bytes = z.slabs * SCORE_BLOCKS * 128;
    const uint32_t s_b = s_a + z.buffers * a_bytes, s_bar = (uint32_t)__cvta_generic_to_shared(&bar);
    if (warp == 0) {
        if (lane == 0) {
            bar_init(s_bar, 1);
            abort_s = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         (uint32_t)__cvta_generic_to_shared(&tmem_s)), "r"(z.n) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }

    // a thread looks after one block of an m-tile; a warp copies the codes of its 32 blocks, 16 bytes a lane
    const int *table = p.tables + (long long)s.ctx * p.max_blk;
    const int pieces = p.D / 8;  // of a block's codes, 16 bytes each
    auto record_of = [&](int m) {
        return p.summary + (long long)__ldg(table + min(first + m * SCORE_BLOCKS + (int)threadIdx.x, total - 1)) * p.record;
    };
    auto issue = [&](int m, const signed char *rec) {
        const uint32_t dst = s_a + (m % z.buffers) * a_bytes;
        for (int i = lane; i < 32 * pieces; i += 32) {  // 32 * pieces is a multiple of 32: all lanes take part
            const int r = i / pieces, c = i - r * pieces, row = warp * 32 + r;
            const signed char *src = reinterpret_cast<const signed char *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(rec), r));
            copy16(dst + (c >> 3) * (SCORE_BLOCKS * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4), src + (long long)head * 2 * p.D + c * 16, 16);
        }
        copy_commit();
    };
    const signed char *rec = record_of(0);
    issue(0, rec);

    const int rows_token = z.heads_p, rows_all = tokens * rows_token;
    const int list_of_tile = s.tok0 + j0;
    bool ok = true;
    int parity = 0;
    const uint32_t idesc = 2u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(z.n / 8) << 17 | (SCORE_BLOCKS / 16) << 24;
    // a pass takes z.n rows: one, but for groups of more heads than that
    for (int row0 = 0; row0 < rows_all; row0 += z.n) {
        const int rows = min(z.n, rows_all - row0);
        if (row0) {
            __syncthreads();
            rec = record_of(0);
            issue(0, rec);
        }
        for (int r = warp; r < rows; r += SCORE_THREADS / 32) {  // a row's codes: [c+, c-], zeros up to a multiple of 32
            const int tok = (row0 + r) / rows_token, gh = min((row0 + r) - tok * rows_token, p.G - 1);
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
            unsigned char *dst = smem + (s_b - s_0) + r * 128;
            auto place = [&](int at) { return (at >> 7) * z.n * 128 + (((at >> 4 & 7) ^ (r & 7)) << 4) + (at & 15); };
            if (lane * 8 < p.D) {
                *reinterpret_cast<uint2 *>(dst + place(lane * 8)) = make_uint2(up[0], up[1]);
                *reinterpret_cast<uint2 *>(dst + place(p.D + lane * 8)) = make_uint2(down[0], down[1]);
            }
            if (2 * p.D % 32 && lane < 2) *reinterpret_cast<uint2 *>(dst + place(2 * p.D + lane * 8)) = make_uint2(0, 0);
            if (lane == 0) units_s[r] = power_of_two(f - 64);
        }
        for (int m = 0; m < m_tiles; ++m) {
            const int e = __ldg(rec + (long long)p.H * 2 * p.D + head);
            if (m + 1 < m_tiles && z.buffers > 1) {
                rec = record_of(m + 1);
                issue(m + 1, rec);
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
            const int block = first + m * SCORE_BLOCKS + threadIdx.x;
            uint32_t *dst = p.keys + ((long long)list_of_tile * p.H + head) * p.pitch + block;
            for (int c0 = 0; c0 < rows; c0 += 32) {
                float x[32];
                tmem_ld32(tmem + ((uint32_t)(warp * 32) << 16) + c0, x);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float4 u = *reinterpret_cast<const float4 *>(units_s + c0 + i);
                    x[i] = (float)__float_as_int(x[i]) * u.x;
                    x[i + 1] = (float)__float_as_int(x[i + 1]) * u.y;
                    x[i + 2] = (float)__float_as_int(x[i + 2]) * u.z;
                    x[i + 3] = (float)__float_as_int(x[i + 3]) * u.w;
                }
#pragma unroll
                for (int t = 0; t < 32 >> HP; ++t) {
                    float best = x[t << HP];
#pragma unroll
                    for (int i = 1; i < 1 << HP; ++i) best = fmaxf(best, x[(t << HP) + i]);
                    const int row = row0 + c0 + (t << HP), tok = HP == 5 ? row / rows_token : row >> HP;
                    if (row < rows_all && block < total) {
                        uint32_t &at = dst[(long long)tok * p.H * p.pitch];
                        const uint32_t k = ordered(best * m1 * m2);
                        at = HP == 5 && row % rows_token ? max(at, k) : k;  // a token of more than 32 heads: this thread has written `at`
                    }
                }
            }
            tmem_before();
            __syncthreads();  // sums and codes have been read
            tmem_after();
            if (m + 1 < m_tiles && z.buffers == 1) {
                rec = record_of(m + 1);
                issue(m + 1, rec);
            }
        }
    }
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_s), "r"(z.n));
}

// A list from its scores: the first `sink`, the last `recent`, the best others.
template <int WARPS>
__global__ void __launch_bounds__(WARPS * 32)
    pick_blocks_kernel(const __grid_constant__ SelectParams p, const __grid_constant__ SmallSeqs small, int room) {
    extern __shared__ __align__(16) uint32_t keys_s[];
    __shared__ __align__(16) uint32_t hist[4][256];
    __shared__ uint32_t range_s[2], counts_s[WARPS][2];
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
        range_s[1] = 0;
    }
    const uint32_t *keys = p.keys + (long long)blockIdx.x * p.pitch;
    int *out = p.blocks + ((long long)(s.row0 + j) * p.H + head) * p.keep;
    float *out_s = p.scores ? p.scores + ((long long)(s.row0 + j) * p.H + head) * p.keep : nullptr;
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the scores are written
    const bool all = total <= p.keep;
    const int m0 = min(p.sink, total), m1 = max(m0, total - p.recent);  // the middle
    int want = p.keep - p.sink - p.recent;
    uint32_t least = 0;
    bool from = true;  // the threshold's equals are taken whole
    __syncthreads();
    if (!all && want > 0) {
        uint32_t a = 0xffffffffu, b = 0;
        const bool stay = total <= room;
        for (int i = threadIdx.x * 4; i < total; i += WARPS * 128) {
            const uint4 v = __ldcg(reinterpret_cast<const uint4 *>(keys + i));
            if (stay) *reinterpret_cast<uint4 *>(keys_s + i) = v;
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e >= m0 && i + e < m1) {
                    a = min(a, w[e]);
                    b = max(b, w[e]);
                }
        }
        a = __reduce_min_sync(0xffffffffu, a);
        b = __reduce_max_sync(0xffffffffu, b);
        if (lane == 0) {
            atomicMin(&range_s[0], a);
            atomicMax(&range_s[1], b);
        }
        __syncthreads();
        if (stay) keys = keys_s;
        a = range_s[0];
        b = range_s[1];
        int shift = 32 - __clz(a ^ b);  // bits that are not decided
        least = shift == 32 ? 0 : a >> shift << shift;
        from = false;
        for (int pass = 0; shift > 0 && !from; ++pass) {
            const int width = min(shift, 8);
            shift -= width;
            const uint32_t prefix = least >> shift >> width, mask = (1u << width) - 1;
            for (int i = m0 + (int)threadIdx.x; i < m1; i += WARPS * 128) {
                uint32_t k[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) k[e] = i + e * WARPS * 32 < m1 ? keys[i + e * WARPS * 32] : 0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e * WARPS * 32 < m1 && k[e] >> shift >> width == prefix) atomicAdd(&hist[pass][k[e] >> shift & mask], 1u);
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
            from = __shfl_sync(0xffffffffu, equal, who) == want;  // all with these bits are taken
        }
    }
    // a warp's piece of the context: how many it takes, then which.  `from`: scores from `least` on, else those above it and the first `want`
    // of its equals
    const int piece = ((total + WARPS - 1) / WARPS + 31) / 32 * 32, i0 = min(warp * piece, total), i1 = min(i0 + piece, total);
    const bool none = !all && p.keep == p.sink + p.recent;
    auto kind_of = [&](int i, bool &tie) -> bool {  // certainly taken
        tie = false;
        if (all || i < m0 || i >= m1) return true;
        if (none) return false;
        const uint32_t k = keys[i];
        tie = !from && k == least;
        return from ? k >= least : k > least;
    };
    uint32_t sure = 0, ties = 0;
    if (!all) {
        for (int i = i0 + lane; i < i1; i += 32) {
            bool tie;
            sure += kind_of(i, tie);
            ties += tie;
        }
        sure = __reduce_add_sync(0xffffffffu, sure);
        ties = __reduce_add_sync(0xffffffffu, ties);
        if (lane == 0) {
            counts_s[warp][0] = sure;
            counts_s[warp][1] = ties;
        }
        __syncthreads();
        sure = ties = 0;
        for (int w = 0; w < warp; ++w) {
            sure += counts_s[w][0];
            ties += counts_s[w][1];
        }
    } else {
        sure = i0;
    }
    for (int base = i0; base < i1; base += 32) {
        const int i = base + lane;
        bool tie = false;
        const bool certain = i < i1 && kind_of(i, tie);
        const unsigned cm = __ballot_sync(0xffffffffu, certain), tm = __ballot_sync(0xffffffffu, tie), under = (1u << lane) - 1;
        const int ties_before = (int)ties + __popc(tm & under);
        if (certain || (tie && ties_before < want)) {
            const int to = (int)sure + __popc(cm & under) + min(ties_before, from ? 0 : want);
            out[to] = i;
            if (out_s) out_s[to] = from_ordered(keys[i]);
        }
        sure += __popc(cm);
        ties += __popc(tm);
    }
    for (int i = min(p.keep, total) + (int)threadIdx.x; i < p.keep; i += WARPS * 32) {
        out[i] = -1;
        if (out_s) out_s[i] = -CUDART_INF_F;
    }
}

static size_t score_smem(const SelectShape &z) { return (size_t)z.slabs * 128 * (z.buffers * SCORE_BLOCKS + z.n) + 1024; }
constexpr int SCORE_SMEM = (4 * 128 * (2 * SCORE_BLOCKS + SELECT_ROWS)) + 1024;

// How a batch is cut.  Rows of a tile: 32 where there is a token each (the sums' columns that a thread reads at once), else as many as
// the tokens fill, up to SELECT_ROWS.  A CTA takes several m-tiles in turn, so that its rows' codes are made once, where that leaves four
// CTAs an SM.
SelectShape select_shape(const SelectParams &p, int max_nq, long long m_tiles, int sm_count, int f16) {
    SelectShape z{};
    z.f16 = f16;
    z.heads_p = p.G > 32 ? (p.G + 31) / 32 * 32 : 1;
    while (z.heads_p < p.G) z.heads_p *= 2;
    for (z.n = 32; z.n < SELECT_ROWS && z.n < max_nq * z.heads_p; z.n *= 2) {}
    z.tile = std::max(1, z.n / z.heads_p);
    z.slabs = (2 * p.D + 127) / 128;
    z.reps = (int)std::max<long long>(1, std::min<long long>(8, m_tiles * p.H / z.tile / (4ll * sm_count)));
    if (max_nq == 1) z.reps = 1;
    z.buffers = z.reps > 1 ? 2 : 1;
    return z;
}

template <int HP> static cudaError_t score_go(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, cudaStream_t st) {
    static SmemSeen seen{0};
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(score_blocks_kernel<HP>), SCORE_SMEM, &seen);
    if (e != cudaSuccess) return e;
    score_blocks_kernel<HP><<<(unsigned)(units * p.H), SCORE_THREADS, score_smem(z), st>>>(p, small, z);
    return cudaGetLastError();
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
        case 0: e = score_go<0>(p, small, z, units, st); break;
        case 1: e = score_go<1>(p, small, z, units, st); break;
        case 2: e = score_go<2>(p, small, z, units, st); break;
        case 3: e = score_go<3>(p, small, z, units, st); break;
        case 4: e = score_go<4>(p, small, z, units, st); break;
        default: e = score_go<5>(p, small, z, units, st); break;
    }
    if (e != cudaSuccess) return e;
    return p.widest <= 1024 ? pick_go<4>(p, small, tokens, st) : pick_go<PICK_WARPS>(p, small, tokens, st);
}

}  // namespace aafkv
