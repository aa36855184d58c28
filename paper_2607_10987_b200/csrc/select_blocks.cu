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
// Selection: a CTA a list; a histogram over the scores' range finds where the smallest one that is taken lies, the few that lie there are
// compared with one another; a list's scores come from L2 and stay in shared memory where they fit.
//
// Bound: the bytes of the summaries where there is a token each (and the start of the two kernels); instructions of the sums' and the
// scores' passes where there are many tokens.  16 contexts of 544 blocks, 18 MB of summaries: 16.5 us; 32 ragged ones of 512 to 4096, 113 MB:
// 47.5 us, of which the scores 32 (5.4 TB/s once they are under way); 128 tokens behind 4096 blocks: 44 us.
#include "sparse_device.cuh"
#include "tensor_device.cuh"

namespace aafkv {

constexpr int SCORE_BLOCKS = 128;  // of an m-tile
constexpr int PICK_KEYS = 12288;  // scores of a list that are kept in shared memory

// 8-bit products, 32-bit sums
__device__ __forceinline__ void mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

__device__ __forceinline__ uint32_t max16(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Eight channels of a query row that `lanes` lanes share: codes [c+, c-] to where `place` says within the row, zeros up to a multiple of
// 32 bytes; 2^(f - 64)
template <typename Place>
__device__ __forceinline__ float row_codes(const uint4 &v, int f16, int D, int sub, unsigned lanes, unsigned char *row, Place place) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    // magnitudes of 16-bit floats have the order of their bits; what is not finite, and bf16 beyond 127 * 2^113, is looked at one by one
    const uint32_t m = max16(max16(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), max16(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
    const uint32_t top = __reduce_max_sync(lanes, max(m & 0xffffu, m >> 16));
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = f16 ? Elt<__half>::lo(w[i]) : Elt<__nv_bfloat16>::lo(w[i]);
        x[2 * i + 1] = f16 ? Elt<__half>::hi(w[i]) : Elt<__nv_bfloat16>::hi(w[i]);
    }
    float most = f16 ? Elt<__half>::from((uint16_t)top) : Elt<__nv_bfloat16>::from((uint16_t)top);
    if (!(most <= 127.0f * 0x1p113f)) {
        most = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = x[i] != x[i] ? 0.0f : fminf(fmaxf(x[i], -127.0f * 0x1p113f), 127.0f * 0x1p113f);
            most = fmaxf(most, fabsf(x[i]));
        }
        most = __uint_as_float(__reduce_max_sync(lanes, __float_as_uint(most)));
    }
    const int f = code_exponent(most);
    const float unit_inv = power_of_two(-f);
    uint32_t up[2], down[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        // x / 2^f + 1.5 * 2^23: rounded to a whole number, half to even, whose low byte is that of the sum's bits
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(fmaf(x[4 * h + i], unit_inv, 12582912.0f));
        const uint32_t c = prmt(prmt(b[0], b[1], 0x0040), prmt(b[2], b[3], 0x0040), 0x5410);
        const uint32_t negative = (c >> 7 & 0x01010101u) * 255u;
        up[h] = c & ~negative;
        down[h] = c & negative;
    }
    if (sub * 8 < D) {
        *reinterpret_cast<uint2 *>(row + place(sub * 8)) = make_uint2(up[0], up[1]);
        *reinterpret_cast<uint2 *>(row + place(D + sub * 8)) = make_uint2(down[0], down[1]);
    }
    if (2 * D % 32 && sub < 2) *reinterpret_cast<uint2 *>(row + place(2 * D + sub * 8)) = make_uint2(0, 0);
    return power_of_two(f - 64);
}
// dot * 2^(f - 64), the largest of a token's heads, * 2^(e + 64): exact, beyond the type's range only where the score is
__device__ __forceinline__ uint32_t score_key(float best, int e) {
    return ordered(best * power_of_two(e < 0 ? e + 64 : 64) * power_of_two(e < 0 ? 0 : e));
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
                auto place = [&](int at) { return (at >> 7) * z.n * 128 + (((at >> 4 & 7) ^ (r & 7)) << 4) + (at & 15); };
                const float unit = row_codes(v[b], z.f16, p.D, sub, row_mask, smem + (s_b - s_0) + r * 128, place);
                if (sub == 0) units_s[r] = unit;
            }
        }
        for (int m = 0; m < m_tiles; ++m) {
            const int e = __ldg(p.summary + (long long)(THREADS == 128 ? id : __ldg(table + min(first + m * SCORE_BLOCKS + mine, total - 1))) * p.record +
                                (long long)p.H * 2 * p.D + head);
            if (m + 1 < m_tiles) {  // into the other buffer: there are two where there are several m-tiles
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
            warp_wait(s_bar, parity, &abort_s, p.status);  // if it gives up, the status says so and the scores are void
            parity ^= 1;
            tmem_after();
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
                    const uint32_t k = score_key(best, e);
                    if (block < total) {
                        uint32_t &at = dst[(HP == 5 ? row / rows_token : row >> HP) * list_pitch];
                        at = HP == 5 && row % rows_token ? max(at, k) : k;  // a token of more than 32 heads: this thread has written `at`
                    }
                }
            }
            tmem_before();
            __syncthreads();  // sums and codes have been read
            tmem_after();
        }
    }
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_s), "r"(z.n));
}

// The same for a token each: an m-tile is all kv heads of some blocks, so that whole records are read from memory, and is multiplied with
// the rows of all heads; of the sums, those of a kv head with its own rows are used.  Row (head, block) of the m-tile is head *
// z.blocks + block, column (head, query head of its group) is head * z.heads_p + query head.
template <int HP>
__global__ void __launch_bounds__(128, 5)
    score_records_kernel(const __grid_constant__ SelectParams p, const __grid_constant__ SmallSeqs small, const __grid_constant__ SelectShape z) {
    extern __shared__ unsigned char smem[];
    __shared__ __align__(8) uint64_t bar;
    __shared__ uint32_t tmem_s;
    __shared__ int abort_s;
    __shared__ __align__(16) float units_s[SELECT_ROWS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // First of all: the SM's next CTA does not start before this one has given up the right to allocate
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         (uint32_t)__cvta_generic_to_shared(&tmem_s)), "r"(z.n) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("griddepcontrol.launch_dependents;");
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq s = seqs[find_seq(seqs, p.n, blockIdx.x)];
    const int total = s.key0 / p.BS + 1;
    const int first = ((int)blockIdx.x - s.unit0) * z.reps * z.blocks, m_tiles = min(z.reps, (total - first + z.blocks - 1) / z.blocks);
    const uint32_t s_0 = (uint32_t)__cvta_generic_to_shared(smem), s_a = (s_0 + 1023) & ~1023u;
    const uint32_t a_bytes = z.slabs * SCORE_BLOCKS * 128, s_b = s_a + z.buffers * a_bytes, s_bar = (uint32_t)__cvta_generic_to_shared(&bar);
    if (threadIdx.x == 0) {
        bar_init(s_bar, 1);
        abort_s = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const int *table = p.tables + (long long)s.ctx * p.max_blk;
    const int pieces = p.D / 8, shift = log2_exact(pieces), chunks = p.H * pieces;  // 16 bytes each; of a head, of a record
    auto block_id = [&](int at) { return __ldg(table + min(at, total - 1)); };
    auto issue = [&](int m, int id) {  // lane l holds the number of the warp's l-th block
        for (int k = 0; k < z.blocks / 4; ++k) {
            const int b = 4 * k + warp;
            const signed char *rec = p.summary + (long long)__shfl_sync(0xffffffffu, id, k) * p.record;
            for (int i = lane; i < chunks; i += 32) {
                const int h = shift >= 0 ? i >> shift : i / pieces, c = i - h * pieces, row = h * z.blocks + b;
                copy16(s_a + (m & (z.buffers - 1)) * a_bytes + (c >> 3) * (SCORE_BLOCKS * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4), rec + i * 16, 16);
            }
        }
        copy_commit();
    };
    const int lanes = p.D <= 128 ? 16 : 32, sub = lane & (lanes - 1), rows = p.H * z.heads_p;
    const unsigned row_mask = lanes == 32 ? 0xffffffffu : 0xffffu << (lane & 16);
    auto load = [&](int r) {
        const int rr = min(r, rows - 1), h = rr / z.heads_p;
        const uint16_t *q = static_cast<const uint16_t *>(p.q) + (long long)s.row0 * p.q_stride + (long long)(h * p.G + min(rr - h * z.heads_p, p.G - 1)) * p.D;
        return sub * 8 < p.D ? __ldg(reinterpret_cast<const uint4 *>(q) + sub) : make_uint4(0, 0, 0, 0);
    };
    const int step = 128 / lanes;
    int id = block_id(first + 4 * lane + warp);
    uint4 v[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) v[b] = load(threadIdx.x / lanes + b * step);  // under way beside the block numbers
    issue(0, id);
    if (m_tiles > 1) issue(1, block_id(first + z.blocks + 4 * lane + warp));
    for (int base = threadIdx.x / lanes; base < (rows + 1) / 2 * 2; base += 4 * step) {
        if (base >= 4 * step)
#pragma unroll
            for (int b = 0; b < 4; ++b) v[b] = load(base + b * step);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int r = base + b * step;
            if (r >= (rows + 1) / 2 * 2) break;
            auto place = [&](int at) { return (at >> 7) * z.n * 128 + (((at >> 4 & 7) ^ (r & 7)) << 4) + (at & 15); };
            const float unit = row_codes(v[b], z.f16, p.D, sub, row_mask, smem + (s_b - s_0) + r * 128, place);
            if (sub == 0) units_s[r] = unit;
        }
    }
    const int b_shift = log2_exact(z.blocks), head = threadIdx.x >> b_shift, mine = threadIdx.x & (z.blocks - 1);
    const int column = min((warp * 32 >> b_shift) << HP, z.n - 32), off = (head << HP) - column;  // where this warp's sums are, this thread's
    const uint32_t idesc = 2u << 4 | 1u << 7 | 1u << 10 | (uint32_t)(z.n / 8) << 17 | (SCORE_BLOCKS / 16) << 24;
    int parity = 0;
    if (m_tiles > 2) id = block_id(first + 2 * z.blocks + 4 * lane + warp);
    for (int m = 0; m < m_tiles; ++m) {
        const int block = first + m * z.blocks + mine;
        const int e = head < p.H ? __ldg(p.summary + (long long)block_id(block) * p.record + (long long)p.H * 2 * p.D + head) : 0;
        if (m + 1 < m_tiles) copy_wait<1>();
        else copy_wait<0>();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tmem_before();
        __syncthreads();
        tmem_after();
        const uint32_t tmem = tmem_s;
        if (warp == 0 && elected()) {
            const uint64_t da = smem_desc(s_a + (m & (z.buffers - 1)) * a_bytes, 16, 1024), db = smem_desc(s_b, 16, 1024);
            const int steps = (2 * p.D + 31) / 32;
            for (int k = 0; k < steps; ++k)
                mma_i8(tmem, da + (k >> 2) * (SCORE_BLOCKS * 128 >> 4) + 2 * (k & 3), db + (k >> 2) * (z.n * 128 >> 4) + 2 * (k & 3), idesc, k > 0);
            mma_commit(s_bar);
        }
        __syncwarp();
        warp_wait(s_bar, parity, &abort_s, p.status);  // if it gives up, the status says so and the scores are void
        parity ^= 1;
        tmem_after();
        if (m + 2 < m_tiles) {  // into the buffer whose codes have been multiplied
            issue(m + 2, id);
            if (m + 3 < m_tiles) id = block_id(first + (m + 3) * z.blocks + 4 * lane + warp);
        }
        float x[32];
        tmem_ld32(tmem + ((uint32_t)(warp * 32) << 16) + column, x);
        tmem_wait_ld();
        float best = -CUDART_INF_F;
#pragma unroll
        for (int t = 0; t < 32 >> HP; ++t)
            if (off == t << HP) {
#pragma unroll
                for (int i = t << HP; i < (t + 1) << HP; ++i) best = fmaxf(best, (float)__float_as_int(x[i]) * units_s[column + i]);
            }
        if (head < p.H && block < total) p.keys[((long long)s.tok0 * p.H + head) * p.pitch + block] = score_key(best, e);
    }
    tmem_before();
    __syncthreads();
    tmem_after();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_s), "r"(z.n));
}

// A list from its scores: the first `sink`, the last `recent`, the best others.  The scores of the middle are looked through three times:
// for their range; for a histogram of 256 equal parts of it, which finds the part of the smallest score that is taken; and for the few in
// this part, among which each counts those above it.  (Where they are many, the part's range is cut on.)  Then every warp writes what
// its piece of the context contributes.
constexpr int PICK_FEW = 128;
constexpr int PICK_PASSES = 5;  // a histogram leaves 1/256 of the range, or 1 % more: 2^32, 2^24 ... below 256, one by one
template <int WARPS>
__global__ void __launch_bounds__(WARPS * 32)
    pick_blocks_kernel(const __grid_constant__ SelectParams p, const __grid_constant__ SmallSeqs small, int room) {
    extern __shared__ __align__(16) uint32_t keys_s[];
    __shared__ __align__(16) uint32_t hist[PICK_PASSES][256];
    __shared__ uint32_t range_s[2], counts_s[WARPS], few_s[PICK_FEW], few_count, least_s;
    __shared__ uint2 bits_s[PICK_KEYS / 32];
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
    for (int i = threadIdx.x; i < PICK_PASSES * 256; i += WARPS * 32) hist[0][i] = 0;
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
        for (int at = i0 + lane * 4; at < i1; at += 4 * 128) {
            uint4 v[4];  // under way together
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = at + u * 128 < i1 ? four(at + u * 128) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (stay && at + u * 128 < i1) *reinterpret_cast<uint4 *>(keys_s + at + u * 128) = v[u];
                a = min(min(a, min(v[u].x - 1, v[u].y - 1)), min(v[u].z - 1, v[u].w - 1));  // a 0 becomes the largest number
                b = max(max(b, max(v[u].x, v[u].y)), max(v[u].z, v[u].w));
            }
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
        uint32_t a = range_s[0] + 1, b = range_s[1];  // what the threshold lies between
        for (int pass = 0;; ++pass) {
            const uint32_t range = b - a;
            const bool exact = range < 256;
            const uint32_t mult = exact ? 0 : (uint32_t)((1ull << 40) / (range + 1ull));
            auto bin = [&](uint32_t k) { return exact ? k - a : __umulhi(k - a, mult); };  // below 256 for a <= k <= b
            for (int i = i0 + lane * 4; i < i1; i += 128) {
                const uint4 v = again(i);
                auto count = [&](uint32_t k) {
                    if (k - a <= range) atomicAdd(&hist[pass][bin(k)], 1u);
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
            const unsigned where = __ballot_sync(0xffffffffu, here);
            if (!where) {  // fewer scores than are wanted: void ones, among them zeros, which no block has (a wait ran out).  All, then zeros
                want -= __shfl_sync(0xffffffffu, (int)(above + mine), 0);
                least = 0;
                break;
            }
            const int who = __ffs(where) - 1;
            want = __shfl_sync(0xffffffffu, left, who);
            const uint32_t found = __shfl_sync(0xffffffffu, lane * 8 + digit, who);
            const int have = __shfl_sync(0xffffffffu, equal, who);
            if (exact) {
                least = a + found;
                break;
            }
            if (have > PICK_FEW) {  // on with the numbers of this bin: from ceil(found * 2^32 / mult) on
                const uint32_t from = (uint32_t)((((unsigned long long)found << 32) + mult - 1) / mult);
                const unsigned long long upto = (((unsigned long long)(found + 1) << 32) + mult - 1) / mult;
                b = (uint32_t)min((unsigned long long)b, a + upto - 1);
                a += from;
                continue;
            }
            for (int i = i0 + lane * 4; i < i1; i += 128) {
                const uint4 v = again(i);
                auto gather = [&](uint32_t k) {
                    if (k - a <= range && bin(k) == found) {
                        const uint32_t to = atomicAdd(&few_count, 1u);
                        if (to < PICK_FEW) few_s[to] = k;  // always, unless the scores change meanwhile
                    }
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
    // A bit for every block: taken for certain, equal to the threshold.  A thread then has 32 blocks, counts what is taken before them and
    // writes what is taken of them.
    uint32_t sure = 0, ties = 0;  // in the windows and rounds before
    for (int w0 = 0; w0 < total; w0 += PICK_KEYS) {
        const int words = (min(PICK_KEYS, total - w0) + 31) / 32;
        if (w0) __syncthreads();
        for (int w = warp; w < words; w += WARPS) {
            const int i = w0 + w * 32 + lane;
            const bool middle = i >= m0 && i < m1;
            const uint32_t k = !middle ? 0u : (stay ? keys_s[i] : __ldcg(scores + i));
            const uint2 v = make_uint2(__ballot_sync(0xffffffffu, middle ? k > least : i < total), __ballot_sync(0xffffffffu, middle && k == least));
            if (lane == 0) bits_s[w] = v;
        }
        __syncthreads();
        for (int c = 0; c < words; c += WARPS * 32) {
            const int w = c + threadIdx.x;
            const uint2 v = w < words ? bits_s[w] : make_uint2(0, 0);
            const uint32_t mine = __popc(v.x) | __popc(v.y) << 16;
            uint32_t upto = mine;  // of this lane and those before it
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += x;
            }
            if (c) __syncthreads();
            if (lane == 31) counts_s[warp] = upto;
            __syncthreads();
            int s_at = (int)(sure + ((upto - mine) & 0xffffu)), t_at = (int)(ties + ((upto - mine) >> 16));
#pragma unroll
            for (int x = 0; x < WARPS; ++x) {
                const uint32_t n = counts_s[x];
                if (x < warp) {
                    s_at += (int)(n & 0xffffu);
                    t_at += (int)(n >> 16);
                }
                sure += n & 0xffffu;
                ties += n >> 16;
            }
            for (uint32_t left = v.x | v.y; left; left &= left - 1) {
                const int b = __ffs(left) - 1, i = w0 + w * 32 + b;
                const bool tie = v.y >> b & 1;
                if (!tie || t_at < want) {
                    const int to = s_at + min(t_at, want);
                    if ((unsigned)to >= (unsigned)p.keep) break;  // never, unless the scores change meanwhile
                    out[to] = i;
                    if (out_s) out_s[to] = from_ordered(stay && i >= m0 && i < m1 ? keys_s[i] : __ldcg(scores + i));
                }
                if (tie) ++t_at;
                else ++s_at;
            }
        }
    }
}

static size_t score_smem(const SelectShape &z) { return (size_t)z.slabs * 128 * (z.buffers * SCORE_BLOCKS + z.n) + 1024; }
constexpr int SCORE_SMEM = (4 * 128 * (2 * SCORE_BLOCKS + SELECT_ROWS)) + 1024;

// How a batch is cut.  Rows of a tile: 32 (the sums' columns that a thread reads at once), or as many as the tokens fill, up to SELECT_ROWS
// (128 tokens behind 65531: 45 us with 128 rows and 256 threads, 49 with 128 threads, 49 with 64 rows, 60 with 32).  A CTA takes so many m-tiles
// in turn that the CTAs are all there at once: its start (memory, record, rows' codes) costs as much as several of them.  A token each:
// whole records, where the CTAs of single heads would not be there at once (32 ragged contexts, 55 thousand blocks: 46.8 us, head by head
// 50.6; 16 contexts of 544 blocks: 18.5 and 16.5, since every CTA makes the codes of all heads' rows).
SelectShape select_shape(const SelectParams &p, int n, int max_nq, long long m_tiles, int sm_count, int f16) {
    SelectShape z{};
    z.f16 = f16;
    // `all` m-tiles; `ends` of them are what is lost where contexts end with half of a CTA's
    auto cut = [&](long long all, long long ends) {
        auto room = [&](int buffers) {
            z.buffers = buffers;
            return std::min<long long>(z.n == 32 ? 5 : 3, 227 * 1024 / (long long)(score_smem(z) + 2048)) * sm_count;
        };
        z.reps = 1;
        if (all > room(1)) {
            const long long most = std::max(room(2) - ends, room(2) / 2);
            z.reps = (int)std::min<long long>(1 << 16, (all + most - 1) / most);
            if (z.reps == 1) z.buffers = 1;
        }
    };
    z.heads_p = p.G > 32 ? (p.G + 31) / 32 * 32 : 1;
    while (z.heads_p < p.G) z.heads_p *= 2;
    z.slabs = (2 * p.D + 127) / 128;
    z.blocks = SCORE_BLOCKS;
    z.n = 32;
    z.buffers = 1;
    const bool at_once = m_tiles * p.H <= std::min<long long>(5, 227 * 1024 / (long long)(score_smem(z) + 2048)) * sm_count;
    if (max_nq == 1 && !at_once && p.H * z.heads_p <= SELECT_ROWS && z.heads_p <= 32 && p.H <= 16) {
        z.together = 1;
        z.tile = 1;
        for (z.n = 32; z.n < p.H * z.heads_p; z.n *= 2) {}
        for (int h = 1; h < p.H; h *= 2) z.blocks /= 2;
        cut(m_tiles * (SCORE_BLOCKS / z.blocks), n / 2);
        return z;
    }
    for (z.n = 32; z.n < SELECT_ROWS && z.n < max_nq * z.heads_p; z.n *= 2) {}
    z.tile = std::max(1, z.n / z.heads_p);
    cut(m_tiles * p.H / std::min(z.tile, max_nq), (long long)n * p.H / 2);
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
template <int HP> static cudaError_t records_go(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, cudaStream_t st) {
    static SmemSeen seen{0};
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(score_records_kernel<HP>), SCORE_SMEM, &seen);
    if (e != cudaSuccess) return e;
    score_records_kernel<HP><<<(unsigned)units, 128, score_smem(z), st>>>(p, small, z);
    return cudaGetLastError();
}
cudaError_t launch_select_blocks(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, long long tokens, int sm_count,
                                 cudaStream_t st) {
    cudaError_t e;
    switch (log2_up(std::min(z.heads_p, 32))) {
        case 0: e = z.together ? records_go<0>(p, small, z, units, st) : score_rows<0>(p, small, z, units, st); break;
        case 1: e = z.together ? records_go<1>(p, small, z, units, st) : score_rows<1>(p, small, z, units, st); break;
        case 2: e = z.together ? records_go<2>(p, small, z, units, st) : score_rows<2>(p, small, z, units, st); break;
        case 3: e = z.together ? records_go<3>(p, small, z, units, st) : score_rows<3>(p, small, z, units, st); break;
        case 4: e = z.together ? records_go<4>(p, small, z, units, st) : score_rows<4>(p, small, z, units, st); break;
        default: e = z.together ? records_go<5>(p, small, z, units, st) : score_rows<5>(p, small, z, units, st); break;
    }
    if (e != cudaSuccess) return e;
    // few lists: more warps for each (128 lists of 544 blocks 17.0 us with eight, 18.5 with four; 1024 lists of 4096 45.1 and 43.1)
    return tokens * p.H > 2ll * sm_count ? pick_go<4>(p, small, tokens, st) : pick_go<8>(p, small, tokens, st);
}

}  // namespace aafkv
