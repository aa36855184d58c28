// Summaries of cache blocks: per block and kv head, the largest and smallest key of every channel.
//
//   hi_d = max_t F(k_td), lo_d = min_t F(k_td) over the block's stored tokens, F(x) = x within +-127 * 2^113, a NaN counting as
//   the largest and as the smallest value;  e = the smallest exponent >= -60 with all |hi_d|, |lo_d| <= 127 * 2^e;
//   codes ceil(hi_d / 2^e), floor(lo_d / 2^e)
//
// Every step is exact (comparisons, divisions by a power of two), so the codes bound the keys and do not depend on any order.
//
// Bound: the bytes of the keys, read once.  D / 8 lanes take a head's channels, 16 bytes each, and walk the block's tokens with
// the loads of SUMMARY_AHEAD tokens under way; maxima stay in the type itself, two channels an instruction.  8187 tokens in 32 layers, 537 MB
// read: 92 to 95 us (5.7 to 5.8 TB/s); one block of 16 contexts: 6 us, three loads one behind the other.
#include "attend_device.cuh"
#include "sparse_device.cuh"

namespace aafkv {

constexpr int SUMMARY_WARPS = 4, SUMMARY_AHEAD = 16;

template <typename T> struct Extreme;
template <> struct Extreme<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t top(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t least(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
};
template <> struct Extreme<__half> {
    static __device__ __forceinline__ uint32_t top(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t least(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
};

template <typename T>
__global__ void __launch_bounds__(SUMMARY_WARPS * 32)
    summarize_kernel(const __grid_constant__ SummaryParams p, const __grid_constant__ SmallSeqs small) {
    const int lane = threadIdx.x & 31, pieces = p.D / 8, teams = 32 / pieces;  // lanes of a head, heads of a warp
    const int groups = (p.H + teams - 1) / teams;
    const long long task = (long long)blockIdx.x * SUMMARY_WARPS + (threadIdx.x >> 5);
    if (task >= (long long)p.blocks * groups * p.layers) return;
    const long long item_l = task / groups;
    const int layer = (int)(item_l / p.blocks), item = (int)(item_l - (long long)layer * p.blocks);
    const int team = lane / pieces, head = (int)(task - item_l * groups) * teams + team, c = lane - team * pieces;
    const AttnSeq *seqs = p.seqs ? p.seqs : small.e;
    const AttnSeq s = seqs[find_seq(seqs, p.n, item)];
    const int column = (s.len - s.nq) / p.BS + (item - s.unit0);
    const int count = min(p.BS, s.len - column * p.BS);  // stored tokens
    const int id = __ldg(p.tables + (long long)s.ctx * p.max_blk + column);
    if (team >= teams || head >= p.H) return;
    const char *src = p.pool + layer * p.layer_stride + (long long)id * 2 * p.run + ((long long)head * p.D + c * 8) * 2;
    uint4 hi, lo;
    for (int t0 = 0; t0 < count; t0 += SUMMARY_AHEAD) {
        uint4 v[SUMMARY_AHEAD];
#pragma unroll
        for (int i = 0; i < SUMMARY_AHEAD; ++i)  // behind the last token the first one again
            v[i] = __ldg(reinterpret_cast<const uint4 *>(src + (long long)(t0 + i < count ? t0 + i : t0) * p.row));
        if (t0 == 0) hi = lo = v[0];
#pragma unroll
        for (int i = 0; i < SUMMARY_AHEAD; ++i) {
            hi.x = Extreme<T>::top(hi.x, v[i].x); lo.x = Extreme<T>::least(lo.x, v[i].x);
            hi.y = Extreme<T>::top(hi.y, v[i].y); lo.y = Extreme<T>::least(lo.y, v[i].y);
            hi.z = Extreme<T>::top(hi.z, v[i].z); lo.z = Extreme<T>::least(lo.z, v[i].z);
            hi.w = Extreme<T>::top(hi.w, v[i].w); lo.w = Extreme<T>::least(lo.w, v[i].w);
        }
    }
    const float most = 127.0f * 0x1p113f;
    const uint32_t hw[4] = {hi.x, hi.y, hi.z, hi.w}, lw[4] = {lo.x, lo.y, lo.z, lo.w};
    float h[8], l[8], amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = i & 1 ? Elt<T>::hi(hw[i / 2]) : Elt<T>::lo(hw[i / 2]), b = i & 1 ? Elt<T>::hi(lw[i / 2]) : Elt<T>::lo(lw[i / 2]);
        h[i] = a != a ? most : fminf(fmaxf(a, -most), most);
        l[i] = b != b ? -most : fminf(fmaxf(b, -most), most);
        amax = fmaxf(amax, fmaxf(fabsf(h[i]), fabsf(l[i])));
    }
    // the head's largest magnitude: the bits of numbers that are not negative have their order
    const unsigned mask = (pieces == 32 ? 0xffffffffu : ((1u << pieces) - 1)) << (team * pieces);
    const int e = code_exponent(__uint_as_float(__reduce_max_sync(mask, __float_as_uint(amax))));
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);  // 2^-e, -113 <= -e <= 60
    uint32_t up[2] = {0, 0}, down[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        up[i / 4] |= ((uint32_t)__float2int_ru(h[i] * inv) & 255u) << (8 * (i & 3));
        down[i / 4] |= ((uint32_t)__float2int_rd(l[i] * inv) & 255u) << (8 * (i & 3));
    }
    signed char *rec = p.summary + layer * p.summary_stride + (long long)id * p.record;
    signed char *dst = rec + (long long)head * 2 * p.D + c * 8;
    *reinterpret_cast<uint2 *>(dst) = make_uint2(up[0], up[1]);
    *reinterpret_cast<uint2 *>(dst + p.D) = make_uint2(down[0], down[1]);
    if (c == 0) rec[(long long)p.H * 2 * p.D + head] = (signed char)e;
}

cudaError_t launch_summarize(const SummaryParams &p, const SmallSeqs &small, int f16, cudaStream_t st) {
    const int teams = 32 / (p.D / 8), groups = (p.H + teams - 1) / teams;
    const long long tasks = (long long)p.blocks * groups * p.layers;
    const unsigned grid = (unsigned)((tasks + SUMMARY_WARPS - 1) / SUMMARY_WARPS);
    if (f16) summarize_kernel<__half><<<grid, SUMMARY_WARPS * 32, 0, st>>>(p, small);
    else summarize_kernel<__nv_bfloat16><<<grid, SUMMARY_WARPS * 32, 0, st>>>(p, small);
    return cudaGetLastError();
}

// ------------------------------------------------------------------------------------------ tables of a batch
// Block tables, lengths and offsets of a batch's contexts, and row, position and slot of every new token, in one launch: the
// first CTAs copy the tables, a row's stretch each, the others take the tokens, one a thread.  Bound: the launch (16 contexts of 544 blocks 4 us,
// 256 ragged ones with 61 thousand new tokens 6 us); beyond some 10 MB the bytes.
constexpr int TABLES_THREADS = 256, TABLES_STRETCH = 1024;

template <int N>
__global__ void __launch_bounds__(TABLES_THREADS)
    batch_tables_kernel(const __grid_constant__ TablesParams p, const __grid_constant__ SmallRows<N> small, int table_ctas) {
    const TableRow *seqs = p.seqs ? p.seqs : small.e;
    const int cta = blockIdx.x;
    if (cta < table_ctas) {
        const int per_row = table_ctas / p.rows, row = cta / per_row, c0 = (cta - row * per_row) * TABLES_STRETCH;
        const int count = row < p.n ? (seqs[row].len + p.BS - 1) / p.BS : 0;
        const int *src = p.src + (long long)(row < p.n ? seqs[row].ctx : 0) * p.max_blk;
        const int end = min(p.cols, c0 + TABLES_STRETCH);
        for (int c = c0 + threadIdx.x; c < end; c += TABLES_THREADS) p.tables[(long long)row * p.cols + c] = c < count ? __ldg(src + c) : -1;
        return;
    }
    const int i = (cta - table_ctas) * TABLES_THREADS + threadIdx.x;
    if (p.lens && i < p.rows) p.lens[i] = i < p.n ? seqs[i].len : 0;
    if (p.offsets && i <= p.rows) p.offsets[i] = i < p.n ? seqs[i].row0 : p.total;
    if (i >= p.tokens) return;
    int row = -1;
    long long pos = 0, slot = -1;
    if (i < p.total) {
        int lo = 0, hi = p.n - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (seqs[mid].row0 <= i) lo = mid; else hi = mid - 1;
        }
        row = lo;
        const int at = seqs[row].len - seqs[row].nq + (i - seqs[row].row0), b = at / p.BS;
        pos = at;
        if (p.slots) slot = (long long)__ldg(p.src + (long long)seqs[row].ctx * p.max_blk + b) * p.BS + (at - b * p.BS);
    }
    if (p.token_row) p.token_row[i] = row;
    if (p.positions) p.positions[i] = pos;
    if (p.slots) p.slots[i] = slot;
}

template <int N> static cudaError_t tables_go(const TablesParams &p, const TableRow *rows, cudaStream_t st) {
    SmallRows<N> small;
    if (!p.seqs) std::copy(rows, rows + p.n, small.e);
    const int table_ctas = p.tables && p.rows ? (p.cols + TABLES_STRETCH - 1) / TABLES_STRETCH * p.rows : 0;
    const long long items = std::max<long long>(p.tokens, (long long)p.rows + 1);
    const unsigned grid = (unsigned)(table_ctas + (items + TABLES_THREADS - 1) / TABLES_THREADS);
    batch_tables_kernel<N><<<grid, TABLES_THREADS, 0, st>>>(p, small, table_ctas);
    return cudaGetLastError();
}
cudaError_t launch_batch_tables(const TablesParams &p, const TableRow *rows, cudaStream_t st) {
    return p.seqs || p.n <= 64 ? tables_go<64>(p, rows, st) : tables_go<SMALL_ROWS>(p, rows, st);
}

}  // namespace aafkv
