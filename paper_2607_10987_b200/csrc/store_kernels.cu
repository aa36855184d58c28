// Rotary positions and the write of new keys and values into their cache slots; selection and gather of a pruned context.
#include "attend_device.cuh"

namespace aafkv {

// ------------------------------------------------------------------------------------------ store
// A pair (a, b) of a head's rotated dimensions at position p, frequency f: (a cos - b sin, a sin + b cos) with the angle
// p * f; pairs are (i, i + rot/2) or (2i, 2i + 1).  The angle of a far position has lost its fraction in 32 bits, so
// position * frequency is taken in 64 bits, reduced to (-1, 1] half turns there, and only then rounded.  Sine and
// cosine are computed once per (token, frequency) into shared memory and used by all heads; results are rounded to the
// payload's type once.  Bound: bytes (q read and written, k and v read and written); a CTA takes a few tokens so that a
// step of one token per sequence still fills its CTAs with one head's 16-byte pieces a thread.
constexpr int STORE_THREADS = 256;
constexpr int STORE_ANGLES = 2048;  // (token, frequency) pairs of a CTA

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
    __shared__ char *slot_of[64];
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
    // 16-byte pieces: [token][q heads, k heads, v heads][dim / 8].  In the half layout the piece that holds the first
    // elements of pairs is handled together with the one that holds the second; its partner has no work of its own.
    const int pieces = p.D / 8, heads = (p.q ? p.Hq : 0) + 2 * p.H;
    const bool paired = half % 8 == 0;  // half layout with whole pieces on both sides
    for (int i = threadIdx.x; i < cnt * heads * pieces; i += STORE_THREADS) {
        const int c = i % pieces, hh = i / pieces % heads, tl = i / pieces / heads;
        const long long tok = t0 + tl;
        const T *src;
        T *dst;
        bool rotate = true;
        const int kh = hh - (p.q ? p.Hq : 0);
        if (kh < 0) {
            src = static_cast<const T *>(p.q) + tok * p.q_stride + (long long)hh * p.D;
            dst = static_cast<T *>(p.q_out) + tok * p.q_out_stride + (long long)hh * p.D;
        } else if (kh < p.H) {
            src = static_cast<const T *>(p.k) + tok * p.k_stride + (long long)kh * p.D;
            dst = reinterpret_cast<T *>(slot_of[tl]) + (long long)kh * p.D;
        } else {
            src = static_cast<const T *>(p.v) + tok * p.v_stride + (long long)(kh - p.H) * p.D;
            dst = reinterpret_cast<T *>(slot_of[tl] + p.run) + (long long)(kh - p.H) * p.D;
            rotate = false;
        }
        const int d = c * 8;
        if (!rotate || d >= p.rot) {
            *reinterpret_cast<uint4 *>(dst + d) = *reinterpret_cast<const uint4 *>(src + d);
            continue;
        }
        const float2 *tn = turn + tl * half;
        float x[8];
        if (p.interleaved) {
            unpack8<T>(*reinterpret_cast<const uint4 *>(src + d), x);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (d / 2 + e < half) {
                    const float2 r = tn[d / 2 + e];
                    const float a = x[2 * e], b = x[2 * e + 1];
                    x[2 * e] = a * r.x - b * r.y;
                    x[2 * e + 1] = a * r.y + b * r.x;
                }
            *reinterpret_cast<uint4 *>(dst + d) = pack8<T>(x);
        } else if (paired) {
            if (d >= half) continue;
            float y[8];
            unpack8<T>(*reinterpret_cast<const uint4 *>(src + d), x);
            unpack8<T>(*reinterpret_cast<const uint4 *>(src + d + half), y);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 r = tn[d + e];
                const float a = x[e], b = y[e];
                x[e] = a * r.x - b * r.y;
                y[e] = a * r.y + b * r.x;
            }
            *reinterpret_cast<uint4 *>(dst + d) = pack8<T>(x);
            *reinterpret_cast<uint4 *>(dst + d + half) = pack8<T>(y);
        } else {
            // pairs straddle pieces: the thread that owns piece 0 of the head does all of the rotated part, reading
            // both elements of a pair before it writes them (q_out may be q)
            if (c) continue;
            uint16_t *o = reinterpret_cast<uint16_t *>(dst);
            const uint16_t *in = reinterpret_cast<const uint16_t *>(src);
            for (int e = 0; e < half; ++e) {
                const float2 r = tn[e];
                const float a = Elt<T>::from(in[e]), b = Elt<T>::from(in[e + half]);
                o[e] = Elt<T>::to(a * r.x - b * r.y);
                o[e + half] = Elt<T>::to(a * r.y + b * r.x);
            }
            for (int e = p.rot; e < min(p.D, (p.rot + 7) / 8 * 8); ++e) o[e] = in[e];  // the last piece's unrotated rest
        }
    }
}

cudaError_t launch_store(const StoreParams &p, const SmallStores &small, int f16, cudaStream_t st) {
    // tokens of a CTA: enough CTAs for every SM while there are few tokens, at most 64 and the angle table's room
    int tokens = max(1, min(8, p.total / 1184));
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
// digit by digit (eight bits at a time, largest first) with a histogram of the candidates that match the digits so far;
// then each thread counts the kept tokens of a contiguous stretch, one scan gives it its place, and it writes them.
constexpr int SELECT_THREADS = 1024;
__device__ __forceinline__ uint32_t score_key(float f) {
    if (f != f) return 0u;
    const uint32_t u = __float_as_uint(f + 0.0f);  // -0 + 0 = +0: the two zeros tie
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(SELECT_THREADS)
    select_kernel(const float *__restrict__ scores, int len, int budget, int sink, int recent, int *__restrict__ kept,
                  float *__restrict__ kept_scores) {
    __shared__ unsigned hist[256];
    __shared__ unsigned warp_sums[32];
    __shared__ uint32_t sh_prefix;
    __shared__ unsigned sh_need;
    const int lo = sink, hi = len - recent;
    const unsigned want = (unsigned)(budget - sink - recent);
    uint32_t prefix = 0, mask = 0;
    unsigned need = want;
    if (want)
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (threadIdx.x < 256) hist[threadIdx.x] = 0;
            __syncthreads();
            for (int i = lo + threadIdx.x; i < hi; i += SELECT_THREADS) {
                const uint32_t k = score_key(scores[i]);
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1u);
            }
            __syncthreads();
            if (threadIdx.x < 32) {  // lane l owns bins 255 - 8l .. 248 - 8l, from the largest digit down
                unsigned c[8], sum = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += c[e] = hist[255 - 8 * threadIdx.x - e];
                unsigned incl = sum;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const unsigned t = __shfl_up_sync(0xffffffffu, incl, d);
                    if ((int)threadIdx.x >= d) incl += t;
                }
                unsigned above = incl - sum;
                if (above < need && need <= incl) {
                    int e = 0;
                    while (above + c[e] < need) above += c[e++];
                    sh_prefix = prefix | (uint32_t)(255 - 8 * threadIdx.x - e) << shift;
                    sh_need = need - above;
                }
            }
            __syncthreads();
            prefix = sh_prefix;
            need = sh_need;
            mask |= 255u << shift;
            __syncthreads();
        }
    // need = how many of the candidates equal to the threshold are kept (the first ones)
    const int per = (hi - lo + SELECT_THREADS - 1) / SELECT_THREADS;
    const int b = lo + min((int)threadIdx.x * per, hi - lo), e = min(b + per, hi);
    unsigned gt = 0, eq = 0;
    if (want)
        for (int i = b; i < e; ++i) {
            const uint32_t k = score_key(scores[i]);
            gt += k > prefix;
            eq += k == prefix;
        }
    auto scan = [&](unsigned v) {  // exclusive prefix over the CTA
        unsigned incl = v;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned t = __shfl_up_sync(0xffffffffu, incl, d);
            if ((int)(threadIdx.x & 31) >= d) incl += t;
        }
        __syncthreads();
        if ((threadIdx.x & 31) == 31) warp_sums[threadIdx.x >> 5] = incl;
        __syncthreads();
        unsigned before = 0;
        for (int w = 0; w < (int)(threadIdx.x >> 5); ++w) before += warp_sums[w];
        return before + incl - v;
    };
    const unsigned gt0 = scan(gt), eq0 = scan(eq);
    unsigned at = sink + gt0 + min(eq0, need), seen = eq0;
    if (want)
        for (int i = b; i < e; ++i) {
            const uint32_t k = score_key(scores[i]);
            if (k > prefix || (k == prefix && seen++ < need)) {
                kept[at] = i;
                if (kept_scores) kept_scores[at] = scores[i];
                ++at;
            }
        }
    for (int i = threadIdx.x; i < sink + recent; i += SELECT_THREADS) {
        const int src = i < sink ? i : len - recent + (i - sink), dst = i < sink ? i : budget - recent + (i - sink);
        kept[dst] = src;
        if (kept_scores) kept_scores[dst] = scores[src];
    }
}

cudaError_t launch_select(const float *scores, int len, int budget, int sink, int recent, int *kept, float *kept_scores,
                          cudaStream_t st) {
    select_kernel<<<1, SELECT_THREADS, 0, st>>>(scores, len, budget, sink, recent, kept, kept_scores);
    return cudaGetLastError();
}

// ------------------------------------------------------------------------------------------ prune: gather
// Row `kept[i]` of the source context becomes row i of the new one, in every layer, K and V.  A warp takes one row
// (n_kv_heads * head_dim elements) of one plane; neighbouring warps take neighbouring rows of the same plane.
constexpr int GATHER_THREADS = 256;
__global__ void __launch_bounds__(GATHER_THREADS)
    gather_rows_kernel(Geom g, const int *__restrict__ src_table, const int *__restrict__ dst_table,
                       const int *__restrict__ kept, int budget) {
    const int lane = threadIdx.x & 31;
    const long long rows = (long long)budget * 2 * g.L;
    const int words = (int)(g.row / 16);
    for (long long w = (blockIdx.x * (long long)GATHER_THREADS + threadIdx.x) >> 5; w < rows;
         w += (long long)gridDim.x * GATHER_THREADS >> 5) {
        const int plane = (int)(w / budget), i = (int)(w - (long long)plane * budget);
        const int t = kept[i], sb = t / g.BS, db = i / g.BS;
        char *base = g.pool + (long long)(plane >> 1) * g.layer_stride + (plane & 1) * g.run;
        const uint4 *src = reinterpret_cast<const uint4 *>(base + (long long)src_table[sb] * 2 * g.run + (long long)(t - sb * g.BS) * g.row);
        uint4 *dst = reinterpret_cast<uint4 *>(base + (long long)dst_table[db] * 2 * g.run + (long long)(i - db * g.BS) * g.row);
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

cudaError_t launch_gather_rows(const Geom &g, const int *src_table, const int *dst_table, const int *kept, int budget,
                               int sm_count, cudaStream_t st) {
    const long long rows = (long long)budget * 2 * g.L, per_cta = GATHER_THREADS / 32;
    const long long need = (rows + per_cta - 1) / per_cta, most = (long long)sm_count * 8 * 16;
    gather_rows_kernel<<<(unsigned)(need < most ? need : most), GATHER_THREADS, 0, st>>>(g, src_table, dst_table, kept, budget);
    return cudaGetLastError();
}

}  // namespace aafkv
