// Declarations shared by the kernels of sparse attention (block summaries, selection, attention over listed blocks) and of a
// batch's tables, and their host side in sparse.cu.
#pragma once
#include "attend_internal.h"

namespace aafkv {

// A block's summary of one layer: [H][2][D] codes (upper, lower bound of every channel's keys), H exponents, filled up to 16
// bytes.  Bounds are code * 2^exponent.
constexpr int SUMMARY_LEAST_EXP = -60;
inline long long summary_record(int H, int D) { return (long long)H * 2 * D + (H + 15) / 16 * 16; }

struct SummaryParams {
    const AttnSeq *seqs;  // device records, null: the kernel parameter holds them.  nq: tokens whose blocks are summed up, unit0: first block
    const int *tables;
    const char *pool;     // first layer's first byte
    signed char *summary; // that layer's first record
    long long layer_stride, run, row, record, summary_stride;  // bytes
    int max_blk, BS, H, D, n, blocks, layers;
};

struct SelectParams {
    const void *q;
    // Records: the tokens of a context that one launch takes.  nq: how many, row0: the first in the batch, key0: its position, tok0: its
    // place in this launch; unit0: first unit (a tile of tokens and z.reps * 128 blocks), nsplit: units of a tile
    const AttnSeq *seqs;
    const int *tables;
    const signed char *summary;  // the layer's first record
    uint32_t *keys;       // scores, as numbers of the same order: [tokens of the launch][H][pitch]
    int *blocks;          // [query tokens][H][keep]
    float *scores;        // the same shape, may be null
    int *status;
    long long q_stride;   // elements
    long long record;     // bytes
    long long pitch;      // a multiple of 4
    int max_blk, BS, H, G, D, n, keep, sink, recent, widest;  // widest: blocks of the longest context
};
constexpr int SELECT_ROWS = 128;  // of a pass over the summaries
struct SelectShape {
    int tile;      // query tokens of a unit
    int heads_p;   // rows of a token: the group's heads, repeated up to a power of two or a multiple of 32
    int n;         // rows that are multiplied at a time
    int slabs;     // 128-byte stretches of a head's codes
    int reps;      // m-tiles of a CTA
    int buffers;   // for their codes: two where reps > 1, else one
    int together;  // all kv heads of some blocks make an m-tile
    int blocks;    // of an m-tile
    int f16;
};

struct TableRow {
    int ctx, len, nq, row0;
};
// Rows that travel as kernel parameters: a batch of up to 64 in 1 KB, up to 512 in 8 KB (256 rows: 7 us of the host's time less than
// through pinned memory and a copy)
template <int N> struct SmallRows {
    TableRow e[N];
};
constexpr int SMALL_ROWS = 512;
struct TablesParams {
    const TableRow *seqs;  // device records, null: the kernel parameter holds them
    const int *src;       // the pool's tables
    int *tables, *lens, *offsets, *token_row;
    long long *positions, *slots;
    int max_blk, BS, n, cols, rows, tokens, total;
};

inline int log2_up(int v) {  // of a power of two
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

cudaError_t launch_summarize(const SummaryParams &p, const SmallSeqs &small, int f16, cudaStream_t st);
SelectShape select_shape(const SelectParams &p, int n, int max_nq, long long m_tiles, int sm_count, int f16);
cudaError_t launch_select_blocks(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, long long tokens, int sm_count,
                                 cudaStream_t st);
// p.first is not read; a record's nsplit parts of `chunk` listed keys (lists of `keep` blocks); units are (query token, part).
// alone: CTAs that have an SM to themselves
cudaError_t launch_attend_blocks(const AttnParams &p, const SmallSeqs &small, int f16, bool alone, cudaStream_t st);
int attend_blocks_rows(int D, int G);  // query rows of a CTA
int attend_blocks_warps(int D);        // of a CTA that is not alone
int attend_blocks_ctas(int D, int G);  // of those, that share an SM; one that is alone has the warps of all of them
cudaError_t launch_batch_tables(const TablesParams &p, const TableRow *rows, cudaStream_t st);  // rows: the batch, on the host

}  // namespace aafkv
