// Declarations shared by the kernels that compute with the pool's bytes (attention over the block tables, the
// attention mass of cached tokens, rotary stores, token pruning) and their host side in pool.cu.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "aafkv_internal.h"

namespace aafkv {

// One sequence of an attention batch.  Its queries are the last nq tokens of the context; row r of a kv head is
// query token r / G, head r % G of the head's group.  Units are what the kernels are launched over; they are
// numbered over the batch, unit0 is the sequence's first.
struct AttnSeq {          // 56 bytes
    int ctx;
    int len;              // tokens of the context (an int: max_ctx * max_blk and the block size bound it, see pool.cu)
    int nq;
    int row0;             // first query token of the sequence in the packed batch
    int unit0;            // first unit
    int nsplit;           // parts that the key range of a row tile is cut into
    int chunk;            // few-row kernel: keys of a part; a group: query tokens of each member
    int part0;            // first row of the sequence's partial results, -1: written straight to the output
    int key0;             // few-row kernel: first key
    int gpart0;           // parts of the keys before key0, which a group of sequences shares (GROUP_ROWS rows a unit)
    int gsplit;           // how many, 0: none
    int grow;             // the sequence's first row within the group
    int tok0;             // query tokens of the records before this one
    int pad;
};
static_assert(sizeof(AttnSeq) == 56, "AttnSeq layout");
// Sequences forked from one context hold the same blocks up to where they were forked.  A group record of the wide kernel stands
// for several of them: the rows of all of them over the shared keys [0, len); row0 is then the first member's place
// in the record array, members are consecutive there.
constexpr int SMALL_SEQS = 64;  // sequences that travel as kernel parameters
struct SmallSeqs {
    AttnSeq e[SMALL_SEQS];
};

struct AttnParams {
    const void *q;
    void *out;
    float *lse;           // may be null
    float *part_o;        // [partial rows][D]
    float *part_ml;       // [partial rows][2]: base of the exponents (log2 domain) and sum
    const AttnSeq *seqs;  // device records, null: the kernel parameter holds them
    const int *tables;
    const char *kbase;    // layer's first byte
    const float *slopes;  // per query head, may be null
    const int *spans;     // [query tokens][2], may be null
    long long q_stride;   // elements between query tokens
    long long run, row;   // bytes
    int max_blk, BS, bs_shift;  // bs_shift: log2 of the block size, -1 if it is no power of two
    int H, G, D, g_shift, n, total_units, first;  // records [first, first + n) are launched over  // g_shift as bs_shift, of G
    int window;           // 0: none
    int epoch;            // what `flag` holds when a CTA of the wide kernel has met values it cannot keep apart
    int *flag;            // wide kernel: written; tile kernel: run only if it holds `epoch` (null: always)
    int *status;          // sticky device status of the pool
    float scale, softcap, inv_cap;  // softcap 0: none
    const int *lists;     // attention over listed blocks: table positions [query tokens][H][keep]; else null
    int keep;
};

struct MassParams {
    AttnParams a;
    const float *lse_in;
    const float *prev;    // may be null
    float *mass;
    long long mass_stride;
};

struct StoreSeq {         // 24 bytes
    int ctx, len, n_new, row0, pad0, pad1;
};
struct SmallStores {
    StoreSeq e[SMALL_SEQS];
};
struct StoreParams {
    const void *q, *k, *v;
    void *q_out;
    long long q_stride, q_out_stride, k_stride, v_stride;  // elements between tokens
    const double *inv_freq;
    const long long *pos;
    const StoreSeq *seqs;
    const int *tables;
    char *kbase;
    long long run, row;
    int max_blk, BS, bs_shift;
    int Hq, H, D, rot, interleaved, n, total;
    float mscale;
};

// Shared memory beyond 48 KB is allowed once per kernel and device; `seen` is the kernel's own.  Pools of several threads share it:
// two that come first together both ask, which does no harm.
typedef std::atomic<unsigned long long> SmemSeen;
inline cudaError_t allow_smem(const void *kernel, int bytes, SmemSeen *seen) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < 64 && (seen->load(std::memory_order_acquire) >> dev & 1))) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) seen->fetch_or(1ull << dev, std::memory_order_release);
    return e;
}

// ---- launchers (each returns cudaGetLastError() of its launches); f16: 1 = half, 0 = bfloat16
constexpr int FEW_MAX_DIM = 256;
int few_rows_limit(int D);                       // most rows of a kv head that the few-row kernel takes
constexpr int TILE_ROWS = 64;                    // rows of a unit of the tile kernel
constexpr int MASS_CHUNK = 64;                   // keys of a CTA of the mass kernel
// single: one query token each; beside: brought up beside the kernel launched before it, which it does not depend on
cudaError_t launch_attend_few(const AttnParams &p, const SmallSeqs &small, int f16, int max_rows, bool single, bool beside,
                              cudaStream_t st);
cudaError_t launch_attend_tile(const AttnParams &p, const SmallSeqs &small, int f16, int sm_count, cudaStream_t st);
constexpr int WIDE_ROWS = 256;                   // rows of a unit of the wide kernel
constexpr int GROUP_ROWS = 128;                  // the same over the keys that a group of sequences shares
bool wide_takes(int D, int BS);                  // pool geometries of the wide kernel
// groups: the records are groups
cudaError_t launch_attend_wide(const AttnParams &p, const SmallSeqs &small, int f16, bool groups, const void *map, int layer,
                               cudaStream_t st);
struct alignas(64) PoolMap {                     // a tensor map, opaque to the host side
    unsigned char bytes[128];
};
bool encode_pool_map(const Geom &g, PoolMap *out);
cudaError_t launch_attend_join(const AttnParams &p, const SmallSeqs &small, int f16, int tile_rows, int tokens, int max_parts,
                               int sm_count, cudaStream_t st);
cudaError_t launch_attn_mass(const MassParams &p, const SmallSeqs &small, int f16, int max_rows, cudaStream_t st);
constexpr int MASS_WIDE_CHUNK = 256;             // keys of a CTA of the mass kernel for many rows
cudaError_t launch_attn_mass_wide(const MassParams &p, const SmallSeqs &small, int f16, const void *map, int layer,
                                  cudaStream_t st);
cudaError_t launch_store(const StoreParams &p, const SmallStores &small, int f16, int sm_count, cudaStream_t st);
// keep list of a pruned context: kept[budget] ascending, kept_scores (may be null); then the row gather
cudaError_t launch_select(const float *scores, int len, int budget, int sink, int recent, int *kept, float *kept_scores,
                          cudaStream_t st);
cudaError_t launch_gather_rows(const Geom &g, const int *src_table, const Piece *dst_blocks, const int *kept, int budget,
                               int sm_count, cudaStream_t st);

}  // namespace aafkv
