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
    const AttnSeq *seqs;  // unit0: first unit (a tile of query tokens)
    const int *tables;
    const signed char *summary;  // the layer's first record
    int *blocks;          // [query tokens][H][keep]
    float *scores;        // the same shape, may be null
    long long q_stride;   // elements
    long long record;     // bytes
    int max_blk, BS, H, G, D, n, keep, sink, recent, widest;  // widest: blocks of the longest context
};
// How a batch is cut (see select_shape)
struct SelectShape {
    int tile;      // query tokens of a unit
    int heads_p;   // rows of a token: the group's heads, repeated up to a power of two or a multiple of 8
    int ctas;      // of a cluster
    int room;      // blocks of a CTA's stretch at most
    int stride;    // bytes from one row's codes to the next in shared memory
    int rows;      // rows that are held at a time
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

cudaError_t launch_summarize(const SummaryParams &p, const SmallSeqs &small, int f16, cudaStream_t st);
SelectShape select_shape(const SelectParams &p, int max_nq, long long tokens, int sm_count, int f16);
cudaError_t launch_select_blocks(const SelectParams &p, const SmallSeqs &small, const SelectShape &z, long long units, cudaStream_t st);
// p.first is not read; a record's nsplit parts of `chunk` listed keys (lists of `keep` blocks); units are (query token, part).
// alone: CTAs of twice as many warps that have an SM to themselves
cudaError_t launch_attend_blocks(const AttnParams &p, const SmallSeqs &small, int f16, bool alone, cudaStream_t st);
int attend_blocks_rows(int D, int G);  // query rows of a CTA
int attend_blocks_warps(int D);        // of a CTA that is not alone
cudaError_t launch_batch_tables(const TablesParams &p, const TableRow *rows, cudaStream_t st);  // rows: the batch, on the host

}  // namespace aafkv
