// Rotary positions and the write of new keys and values into their cache slots; selection and gather of a pruned context.
#include "attend_device.cuh"

namespace aafkv {

// ------------------------------------------------------------------------------------------ store
// A pair (a, b) of a head's rotated dimensions at position p, frequency f: (a cos - b sin, a sin + b cos) with the angle
// p * f; pairs are (i, i + rot/2) or (2i, 2i + 1).  The angle of a far position has lost its fraction in 32 bits, so
// position * frequency is taken in 64 bits, reduced to (-1, 1] half turns there, and only then rounded.  Sine and
// cosine are computed once per (token, frequency) into shared memory and used by all heads; results are rounded to the
// payload's type once.  Bound: bytes (q read and written, k and v read and written).  A thread handles units of 16 bytes, or
// two of them where the halves of pairs lie apart, the same unit of two tokens at a time: the loads are under way together and the
// place of a unit is worked out once.  Rows are fetched to L2 while the angles are computed.  201 MB moved in 41 us (4.9 TB/s;
// 44.7 with a prefetch for each line instead of each row, 53.3 with none and eight tokens a CTA, four at a time).
constexpr int STORE_THREADS = 256;
constexpr int STORE_ANGLES = 2048;  // (token, frequency) pairs of a CTA
constexpr int STORE_AHEAD = 2;
constexpr int STORE_TOKENS = 4;     // tokens of a CTA at most

template <typename T> __device__ __forceinline__ void unpack8(const uint4 &v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = Elt<T>::lo(w[i]);
        f[2 * i + 1] = Elt<T>::hi(w[i]);
    }
}
template <typename T> __device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
    return make_uint4(Elt<T>::pack(f[0], f[1]), Elt<T>::pack(f[2], f[3]), Elt<T>::pack(f[4], f[5]), Elt<T>::pack(f[6], f[7]));
}

template <typename T>
__global__ void __launch_bounds__(STORE_THREADS)
    store_kernel(const __grid_constant__ StoreParams p, const __grid_constant__ SmallStores small, int tokens) {
    __shared__ float2 turn[STORE_ANGLES];
    __shared__ char *slot_of[STORE_TOKENS];
    const StoreSeq *seqs = p.seqs ? p.seqs : small.e;
    const int t0 = blockIdx.x * tokens, cnt = min(tokens, p.total - t0);
    const int half = p.rot / 2;
    auto seq_of = [&](int tok) {
        int lo = 0, hi = p.n - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (seqs[mid].row0 <= tok) lo = mid; else hi = mid - 1;
        }
        return lo;
    };
    // the CTA's rows are on their way to L2 while the angles are computed
    auto ahead = [&](const void *src, long long stride, int heads, int tl) {
        if (tl >= 0 && tl < cnt)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(static_cast<const char *>(src) + (t0 + tl) * stride * 2),
                         "r"((uint32_t)(heads * p.D * 2)) : "memory");
    };
    if (p.q) ahead(p.q, p.q_stride, p.Hq, (int)threadIdx.x - 32);
    ahead(p.k, p.k_stride, p.H, (int)threadIdx.x - 64);
    ahead(p.v, p.v_stride, p.H, (int)threadIdx.x - 96);
    if (threadIdx.x < cnt) {
        const int tok = t0 + threadIdx.x;
        const StoreSeq s = seqs[seq_of(tok)];
        const int at = s.len - s.n_new + (tok - s.row0), b = block_of(at, p.BS, p.bs_shift);
        slot_of[threadIdx.x] = p.kbase + (long long)p.tables[(long long)s.ctx * p.max_blk + b] * 2 * p.run +
                               (long long)(at - b * p.BS) * p.row;
    }
    for (int i = threadIdx.x; i < cnt * half; i += STORE_THREADS) {
        const int tok = t0 + i / half;
        long long pos;
        if (p.pos) {
            pos = p.pos[tok];
        } else {
            const StoreSeq s = seqs[seq_of(tok)];
            pos = s.len - s.n_new + (tok - s.row0);
        }
        double x = (double)pos * p.inv_freq[i % half] * 0.3183098861837906715;  // half turns
        x -= 2.0 * rint(0.5 * x);
        float sn, cs;
        sincospif((float)x, &sn, &cs);
        turn[i] = make_float2(cs * p.mscale, sn * p.mscale);
    }
    __syncthreads();
    // Units of a head, 16 bytes each: in the half layout the unit of a pair's first elements carries the second ones with it.
    // (Pairs that straddle units, rot / 2 no multiple of 8, are left to one thread per head.)
    const int pieces = p.D / 8;
    const bool apart = p.rot && !p.interleaved, paired = apart && half % 8 == 0;
    const int turned = paired ? half / 8 : 0;  // units with a second piece
    auto copy_heads = [&](const T *src, long long src_stride, int heads, int which) {
        const bool rotate = which < 2 && p.rot > 0;
        const int units = rotate ? (paired ? pieces - turned : pieces) : pieces;
        const unsigned per_unit = 0xffffffffu / (unsigned)units + 1;  // i / units = high word of i * per_unit while i * units < 2^32
        for (int i = threadIdx.x; i < heads * units; i += STORE_THREADS) {  // the same unit of all the CTA's tokens
            const int h = units == 1 ? i : (int)__umulhi((unsigned)i, per_unit), u = i - h * units;
            const int d = (rotate && paired && u >= turned ? u + turned : u) * 8;
            const bool two = rotate && paired && u < turned;
            const T *s = src + t0 * src_stride + (long long)h * p.D;
            for (int tl0 = 0; tl0 < cnt; tl0 += STORE_AHEAD) {
                uint4 x[STORE_AHEAD], y[STORE_AHEAD];
#pragma unroll
                for (int e = 0; e < STORE_AHEAD; ++e)
                    if (tl0 + e < cnt) {
                        x[e] = *reinterpret_cast<const uint4 *>(s + (tl0 + e) * src_stride + d);
                        if (two) y[e] = *reinterpret_cast<const uint4 *>(s + (tl0 + e) * src_stride + d + half);
                    }
#pragma unroll
                for (int e = 0; e < STORE_AHEAD; ++e) {
                    const int tl = tl0 + e;
                    if (tl >= cnt) continue;
                    uint16_t *dst = which == 0 ? static_cast<uint16_t *>(p.q_out) + (t0 + tl) * p.q_out_stride + (long long)h * p.D
                                               : reinterpret_cast<uint16_t *>(slot_of[tl] + (which == 2 ? p.run : 0)) + (long long)h * p.D;
                    const float2 *tn = turn + tl * half;
                    uint4 *out = reinterpret_cast<uint4 *>(dst + d);
                    if (!rotate || d >= p.rot) {
                        *out = x[e];
                    } else if (p.interleaved) {
                        float v[8];
                        unpack8<T>(x[e], v);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (d / 2 + k < half) {
                                const float2 r = tn[d / 2 + k];
                                const float a = v[2 * k], b = v[2 * k + 1];
                                v[2 * k] = a * r.x - b * r.y;
                                v[2 * k + 1] = a * r.y + b * r.x;
                            }
                        *out = pack8<T>(v);
                    } else if (paired) {
                        float v[8], w[8];
                        unpack8<T>(x[e], v);
                        unpack8<T>(y[e], w);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float2 r = tn[d + k];
                            const float a = v[k], b = w[k];
                            v[k] = a * r.x - b * r.y;
                            w[k] = a * r.y + b * r.x;
                        }
                        *out = pack8<T>(v);
                        *reinterpret_cast<uint4 *>(dst + d + half) = pack8<T>(w);
                    } else if (d == 0) {
                        // pairs straddle units: the thread of the head's first one turns all of them, reading both elements of a
                        // pair before it writes them (q_out may be q); units behind the rotated part are other threads'
                        const uint16_t *in = reinterpret_cast<const uint16_t *>(s) + tl * src_stride;
                        for (int k = 0; k < half; ++k) {
                            const float2 r = tn[k];
                            const float a = Elt<T>::from(in[k]), b = Elt<T>::from(in[k + half]);
                            dst[k] = Elt<T>::to(a * r.x - b * r.y);
                            dst[k + half] = Elt<T>::to(a * r.y + b * r.x);
                        }
                        for (int k = p.rot; k < min(p.D, (p.rot + 7) / 8 * 8); ++k) dst[k] = in[k];  // the last unit's unrotated rest
                    }
                }
            }
        }
    };
    if (p.q) copy_heads(static_cast<const T *>(p.q), p.q_stride, p.Hq, 0);
    copy_heads(static_cast<const T *>(p.k), p.k_stride, p.H, 1);
    copy_heads(static_cast<const T *>(p.v), p.v_stride, p.H, 2);
}

cudaError_t launch_store(const StoreParams &p, const SmallStores &small, int f16, int sm_count, cudaStream_t st) {
    // tokens of a CTA: eight CTAs an SM while there are few tokens, at most 4 (41 us; 44 at 6 and 8) and the angle table's room
    int tokens = max(1, min(STORE_TOKENS, p.total / (8 * sm_count)));
    if (p.rot) tokens = max(1, min(tokens, STORE_ANGLES / (p.rot / 2)));
    const unsigned grid = (unsigned)((p.total + tokens - 1) / tokens);
    if (f16)
        store_kernel<__half><<<grid, STORE_THREADS, 0, st>>>(p, small, tokens);
    else
        store_kernel<__nv_bfloat16><<<grid, STORE_THREADS, 0, st>>>(p, small, tokens);
    return cudaGetLastError();
}

// ------------------------------------------------------------------------------------------ prune: selection
// Keeps the first `sink` tokens, the last `recent` ones and, of the rest, those with the largest scores until `budget`
// tokens are kept; equal scores go to the lower position, a NaN ranks below everything.  The threshold score is found
// digit by digit, largest first, with a histogram of the candidates that match the digits so far; then each warp counts the
// kept tokens of a contiguous stretch, one scan gives it its place, and it writes them.  Bound: the latency of one CTA's
// passes; the rows that are moved afterwards cost several times as much.
constexpr int SELECT_THREADS = 1024;
__device__ __forceinline__ uint32_t score_key(float f) {
    if (f != f) return 0u;
    const uint32_t u = __float_as_uint(f + 0.0f);  // -0 + 0 = +0: the two zeros tie
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// 11 bits at a time (11, 11, 10).  The order-preserving keys of up to SELECT_CACHED candidates are kept in shared memory, so
// that the scores are read once: 34 us for 40960 with planner and gather, 56 for 45000, which are read in every pass, 178 for 131072.
constexpr int SELECT_CACHED = 40960, SELECT_BINS = 2048;
__global__ void __launch_bounds__(SELECT_THREADS)
    select_kernel(const float *__restrict__ scores, int len, int budget, int sink, int recent, int *__restrict__ kept,
                  float *__restrict__ kept_scores, int cached) {
    extern __shared__ uint32_t keys[];
    __shared__ unsigned hist[SELECT_BINS];
    __shared__ unsigned warp_sums[32];
    __shared__ uint32_t sh_prefix;
    __shared__ unsigned sh_need;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int lo = sink, n = len - recent - sink;  // candidates
    const unsigned want = (unsigned)(budget - sink - recent);
    auto key_of = [&](int i) { return cached ? keys[i] : score_key(scores[lo + i]); };
    auto scan = [&](unsigned v) {  // exclusive prefix over the CTA
        unsigned incl = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned t = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += t;
        }
        __syncthreads();
        if (lane == 31) warp_sums[warp] = incl;
        __syncthreads();
        unsigned before = lane < warp ? warp_sums[lane] : 0;
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) before += __shfl_xor_sync(0xffffffffu, before, d);
        return before + incl - v;
    };
    if (cached)
        for (int i = threadIdx.x; i < n; i += SELECT_THREADS) keys[i] = score_key(scores[lo + i]);
    uint32_t prefix = 0, mask = 0;
    unsigned need = want;
    for (int pass = 0; pass < 3 && want; ++pass) {
        const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bits = pass == 2 ? 10 : 11;
        for (int i = threadIdx.x; i < SELECT_BINS; i += SELECT_THREADS) hist[i] = 0;
        __syncthreads();
        for (int i0 = 0; i0 < n; i0 += SELECT_THREADS) {
            const int i = i0 + threadIdx.x;
            const uint32_t k = i < n ? key_of(i) : 0;
            const bool in = i < n && (k & mask) == prefix;
            const uint32_t bin = (k >> shift) & ((1u << bits) - 1);
            if (in) atomicAdd(&hist[bin], 1u);
        }
        __syncthreads();
        // thread t owns the two bins 2047 - 2t and 2046 - 2t: from the largest digit down
        const unsigned c0 = hist[SELECT_BINS - 1 - 2 * threadIdx.x], c1 = hist[SELECT_BINS - 2 - 2 * threadIdx.x];
        const unsigned above = scan(c0 + c1);
        if (above < need && need <= above + c0 + c1) {
            const bool second = need > above + c0;
            sh_prefix = prefix | (uint32_t)(SELECT_BINS - 1 - 2 * threadIdx.x - second) << shift;
            sh_need = need - above - (second ? c0 : 0);
        }
        __syncthreads();
        prefix = sh_prefix;
        need = sh_need;
        mask |= ((1u << bits) - 1) << shift;
        __syncthreads();
    }
    // need = how many of the candidates equal to the threshold are kept (the first ones).  A warp takes a contiguous stretch, 32
    // candidates at a time, so that its writes are together; where it starts follows from what the warps before it keep.
    const int per = (n + SELECT_THREADS - 1) / SELECT_THREADS * 32, b = min(warp * per, n), e = min(b + per, n);
    unsigned gt = 0, eq = 0;
    if (want)
        for (int i0 = b; i0 < e; i0 += 32) {
            const uint32_t k = i0 + lane < e ? key_of(i0 + lane) : 0;
            gt += __popc(__ballot_sync(0xffffffffu, i0 + lane < e && k > prefix));
            eq += __popc(__ballot_sync(0xffffffffu, i0 + lane < e && k == prefix));
        }
    const unsigned gt0 = scan(lane == 0 ? gt : 0), eq0 = scan(lane == 0 ? eq : 0);  // lane 0: before this warp
    unsigned more = __shfl_sync(0xffffffffu, gt0, 0), equal = __shfl_sync(0xffffffffu, eq0, 0);
    if (want)
        for (int i0 = b; i0 < e; i0 += 32) {
            const uint32_t k = i0 + lane < e ? key_of(i0 + lane) : 0;
            const unsigned g = __ballot_sync(0xffffffffu, i0 + lane < e && k > prefix);
            const unsigned q = __ballot_sync(0xffffffffu, i0 + lane < e && k == prefix);
            const unsigned below = (1u << lane) - 1;
            const unsigned seen = equal + __popc(q & below);
            if ((g >> lane & 1) || ((q >> lane & 1) && seen < need)) {
                const unsigned at = sink + more + __popc(g & below) + min(seen, need);
                kept[at] = lo + i0 + lane;
                if (kept_scores) kept_scores[at] = scores[lo + i0 + lane];
            }
            more += __popc(g);
            equal += __popc(q);
        }
    for (int i = threadIdx.x; i < sink + recent; i += SELECT_THREADS) {
        const int src = i < sink ? i : len - recent + (i - sink), dst = i < sink ? i : budget - recent + (i - sink);
        kept[dst] = src;
        if (kept_scores) kept_scores[dst] = scores[src];
    }
}

cudaError_t launch_select(const float *scores, int len, int budget, int sink, int recent, int *kept, float *kept_scores,
                          cudaStream_t st) {
    const int n = len - sink - recent, cached = n <= SELECT_CACHED;
    static SmemSeen seen{0};
    const cudaError_t e = allow_smem(reinterpret_cast<const void *>(select_kernel), SELECT_CACHED * 4, &seen);
    if (e != cudaSuccess) return e;
    select_kernel<<<1, SELECT_THREADS, cached ? 4 * (size_t)n : 0, st>>>(scores, len, budget, sink, recent, kept, kept_scores, cached);
    return cudaGetLastError();
}

// ------------------------------------------------------------------------------------------ prune: gather
// Row `kept[i]` of the source context becomes row i of the new one, in every layer, K and V.  A warp takes one row
// (n_kv_heads * head_dim elements) of one plane; neighbouring warps take neighbouring rows of the same plane.
// The new context's blocks are read from the planner's piece list, which alternates between two buffers: the next planner
// need not wait for this kernel.
constexpr int GATHER_THREADS = 256;
__global__ void __launch_bounds__(GATHER_THREADS)
    gather_rows_kernel(Geom g, const int *__restrict__ src_table, const Piece *__restrict__ dst_blocks,
                       const int *__restrict__ kept, int budget) {
    const int lane = threadIdx.x & 31;
    const long long rows = (long long)budget * 2 * g.L;
    const int words = (int)(g.row / 16);
    for (long long w = (blockIdx.x * (long long)GATHER_THREADS + threadIdx.x) >> 5; w < rows;
         w += (long long)gridDim.x * GATHER_THREADS >> 5) {
        const int plane = (int)(w / budget), i = (int)(w - (long long)plane * budget);
        const int t = kept[i], sb = t / g.BS, db = i / g.BS;
        const long long at = (long long)(plane >> 1) * g.layer_stride + (plane & 1) * g.run;
        const uint4 *src = reinterpret_cast<const uint4 *>(g.pool + at + (long long)src_table[sb] * 2 * g.run + (long long)(t - sb * g.BS) * g.row);
        uint4 *dst = reinterpret_cast<uint4 *>(dst_blocks[db].dst + at + (long long)(i - db * g.BS) * g.row);
        int c = lane;
        for (; c + 96 < words; c += 128) {
            const uint4 a = src[c], b = src[c + 32], d = src[c + 64], e = src[c + 96];
            dst[c] = a;
            dst[c + 32] = b;
            dst[c + 64] = d;
            dst[c + 96] = e;
        }
        for (; c < words; c += 32) dst[c] = src[c];
    }
}

cudaError_t launch_gather_rows(const Geom &g, const int *src_table, const Piece *dst_blocks, const int *kept, int budget,
                               int sm_count, cudaStream_t st) {
    const long long rows = (long long)budget * 2 * g.L, per_cta = GATHER_THREADS / 32;
    const long long need = (rows + per_cta - 1) / per_cta, most = (long long)sm_count * 8 * 16;
    gather_rows_kernel<<<(unsigned)(need < most ? need : most), GATHER_THREADS, 0, st>>>(g, src_table, dst_blocks, kept, budget);
    return cudaGetLastError();
}

}  // namespace aafkv
