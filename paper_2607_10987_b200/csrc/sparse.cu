// Host side of sparse attention over the paged pool (block summaries, selection, attention over listed blocks) and of a batch's
// tables: the entry points, their checks, the cut of the work into units.
#include "pool_state.h"
#include "sparse_internal.h"

using namespace aafkv;

namespace {

// what the summaries and their readers ask of a pool
bool summary_takes(const aaf_kv_pool *p) { return p->g.E == 2 && p->g.D % 8 == 0 && p->g.D <= AAF_ATTN_MAX_HEAD_DIM; }
long long record_of(const aaf_kv_pool *p) { return summary_record(p->g.H, p->g.D); }
size_t summary_size(const aaf_kv_pool *p) { return (size_t)p->g.L * (size_t)p->g.NB * (size_t)record_of(p); }

// records of a batch; nq null: `all` says whether that means every token of a context or its last one
int batch_records(const aaf_kv_pool *p, int32_t n, const aaf_ctx_t *ctxs, const int32_t *nq, bool all, std::vector<AttnSeq> &rec,
                  long long *total) {
    if (n > p->lay.max_batch) return AAF_ERR_TOO_MANY;
    rec.resize((size_t)n);
    long long sum = 0;
    for (int i = 0; i < n; ++i) {
        if (!is_live(p, ctxs[i])) return AAF_ERR_BAD_CTX;
        const long long T = p->len[ctxs[i]];
        if (nq && (nq[i] < 1 || nq[i] > T)) return AAF_ERR_INVALID_ARG;
        if (T > (1ll << 30)) return AAF_ERR_TOO_LONG;  // token indices are ints in the kernels
        AttnSeq &s = rec[(size_t)i];
        s = AttnSeq{};
        s.ctx = ctxs[i];
        s.len = (int)T;
        s.nq = nq ? nq[i] : (all ? (int)T : 1);
        s.row0 = (int)sum;
        s.nsplit = 1;
        s.part0 = -1;
        sum += s.nq;
        if (sum > (1ll << 30)) return AAF_ERR_TOO_MANY;
    }
    *total = sum;
    return AAF_OK;
}

}  // namespace
extern "C" {

size_t aaf_kv_summary_bytes(const aaf_kv_pool *p) { return p && summary_takes(p) ? summary_size(p) : 0; }

int aaf_kv_summarize(aaf_kv_pool *p, int32_t layer, int32_t dtype, int32_t n, const aaf_ctx_t *ctxs, const int32_t *n_new,
                     void *summary_dev, size_t summary_bytes, void *stream) try {
    AAF_RANGE("aaf_kv_summarize");
    if (!p || n < 1 || !ctxs || !aligned16(summary_dev)) return AAF_ERR_INVALID_ARG;
    if (p->broken) return AAF_ERR_CUDA;
    if (layer < AAF_ALL_LAYERS || layer >= p->g.L || !dtype_ok(dtype)) return AAF_ERR_INVALID_ARG;
    if (!summary_takes(p)) return AAF_ERR_INCOMPAT;
    if (summary_bytes < summary_size(p)) return AAF_ERR_DST_TOO_SMALL;
    std::vector<AttnSeq> rec;
    long long total = 0, blocks = 0;
    const int rc = batch_records(p, n, ctxs, n_new, true, rec, &total);
    if (rc != AAF_OK) return rc;
    for (AttnSeq &s : rec) {
        s.unit0 = (int)blocks;
        blocks += (s.len + p->g.BS - 1) / p->g.BS - (s.len - s.nq) / p->g.BS;
    }
    SummaryParams k{};
    const int first = layer < 0 ? 0 : layer;
    k.layers = layer < 0 ? p->g.L : 1;
    if (blocks * k.layers > (1ll << 31) / p->g.H) return AAF_ERR_TOO_MANY;  // a warp of the grid takes one head of a block at least
    DeviceGuard guard(p->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (capturing(st)) return AAF_ERR_INVALID_ARG;
    k.tables = p->s.tables;
    k.layer_stride = p->g.layer_stride;
    k.pool = p->g.pool + first * k.layer_stride;
    k.record = record_of(p);
    k.summary_stride = (long long)p->g.NB * k.record;
    k.summary = static_cast<signed char *>(summary_dev) + first * k.summary_stride;
    k.run = p->g.run; k.row = p->g.row;
    k.max_blk = p->g.max_blk; k.BS = p->g.BS; k.H = p->g.H; k.D = p->g.D;
    k.n = n; k.blocks = (int)blocks;
    p->last_stream = st;
    if (!begin_read(p, ctxs, n, st)) return broke(p);
    SmallSeqs small;
    const bool ok = place_records(p, rec, small, &k.seqs, 0, st) && launch_summarize(k, small, dtype == AAF_DTYPE_F16, st) == cudaSuccess;
    return ok && end_read(p, st) ? AAF_OK : broke(p);
} catch (const std::bad_alloc &) {
    return AAF_ERR_INVALID_ARG;  // the host has no memory for the records; nothing was launched
}

int aaf_kv_select(aaf_kv_pool *p, int32_t layer, const aaf_kv_select_desc *d, int32_t n, const aaf_ctx_t *ctxs, const int32_t *n_q,
                  const void *q_dev, const void *summary_dev, size_t summary_bytes, int32_t *blocks_dev, float *scores_dev,
                  void *workspace_dev, size_t workspace_bytes, void *stream) try {
    AAF_RANGE("aaf_kv_select");
    if (!p || !d || d->struct_size != sizeof(aaf_kv_select_desc) || n < 1 || !ctxs || !aligned16(q_dev) || !aligned16(summary_dev) ||
        !aligned16(workspace_dev))
        return AAF_ERR_INVALID_ARG;
    if (!blocks_dev || ((reinterpret_cast<uintptr_t>(blocks_dev) | reinterpret_cast<uintptr_t>(scores_dev)) & 3u)) return AAF_ERR_INVALID_ARG;
    if (p->broken) return AAF_ERR_CUDA;
    if (layer < 0 || layer >= p->g.L || !dtype_ok(d->dtype)) return AAF_ERR_INVALID_ARG;
    if (!summary_takes(p)) return AAF_ERR_INCOMPAT;
    if (d->n_q_heads < 1 || d->n_q_heads % p->g.H != 0 || (long long)d->n_q_heads * p->g.D >= 1ll << 31) return AAF_ERR_INVALID_ARG;
    if (d->q_stride % 8 != 0 || d->q_stride < (long long)d->n_q_heads * p->g.D) return AAF_ERR_INVALID_ARG;
    if (d->keep < 1 || d->keep > AAF_LIST_MAX_BLOCKS || d->sink < 0 || d->recent < 1 || d->sink > d->keep - d->recent) return AAF_ERR_INVALID_ARG;
    if (summary_bytes < summary_size(p) || workspace_bytes < attend_ws_bytes(p)) return AAF_ERR_DST_TOO_SMALL;
    std::vector<AttnSeq> rec;
    long long total = 0, m_tiles = 0;
    const int rc = batch_records(p, n, ctxs, n_q, false, rec, &total);
    if (rc != AAF_OK) return rc;
    SelectParams k{};
    int max_nq = 1;
    for (const AttnSeq &s : rec) {
        const int blocks = (s.len + p->g.BS - 1) / p->g.BS;
        k.widest = std::max(k.widest, blocks);
        max_nq = std::max(max_nq, s.nq);
        m_tiles += (blocks + 127ll) / 128 * s.nq;
    }
    // the scores of so many tokens fit into the workspace at a time
    k.pitch = (k.widest + 3) / 4 * 4;
    const long long at_once = (long long)(attend_ws_bytes(p) / 4) / (k.pitch * p->g.H);
    if (at_once < 1) return AAF_ERR_TOO_LONG;
    k.q = q_dev;
    k.tables = p->s.tables;
    k.record = record_of(p);
    k.summary = static_cast<const signed char *>(summary_dev) + (long long)layer * p->g.NB * k.record;
    k.keys = static_cast<uint32_t *>(workspace_dev);
    k.blocks = blocks_dev;
    k.scores = scores_dev;
    k.status = &p->s.ctl->status;
    k.q_stride = d->q_stride;
    k.max_blk = p->g.max_blk; k.BS = p->g.BS; k.H = p->g.H; k.G = d->n_q_heads / p->g.H; k.D = p->g.D;
    k.keep = d->keep; k.sink = d->sink; k.recent = d->recent;
    const SelectShape z = select_shape(k, n, max_nq, m_tiles, p->sm_count, d->dtype == AAF_DTYPE_F16);
    if (std::min(at_once, total) * p->g.H > (1ll << 31) - 1) return AAF_ERR_TOO_MANY;
    // what one launch takes: `units` CTAs a head, `tokens` lists a head
    struct Launch {
        size_t first, end;
        long long units, tokens;
    };
    std::vector<AttnSeq> parts;
    std::vector<Launch> launches;
    for (const AttnSeq &s : rec)
        for (int j = 0; j < s.nq;) {
            if (launches.empty() || launches.back().tokens == at_once || (long long)(launches.back().end - launches.back().first) == p->lay.max_batch)
                launches.push_back(Launch{parts.size(), parts.size(), 0, 0});
            Launch &l = launches.back();
            AttnSeq x = s;
            x.nq = (int)std::min<long long>(s.nq - j, at_once - l.tokens);
            x.row0 = s.row0 + j;
            x.key0 = s.len - s.nq + j;
            x.tok0 = (int)l.tokens;
            x.unit0 = (int)l.units;
            x.nsplit = (int)(((x.key0 + x.nq - 1) / p->g.BS + (long long)z.blocks * z.reps) / ((long long)z.blocks * z.reps));
            l.units += (long long)((x.nq + z.tile - 1) / z.tile) * x.nsplit;
            l.tokens += x.nq;
            l.end += 1;
            if (l.units * p->g.H > (1ll << 31) - 1) return AAF_ERR_TOO_MANY;
            parts.push_back(x);
            j += x.nq;
        }
    DeviceGuard guard(p->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (capturing(st)) return AAF_ERR_INVALID_ARG;
    p->last_stream = st;
    if (!begin_read(p, ctxs, n, st)) return broke(p);
    bool ok = true;
    for (size_t i = 0; i < launches.size() && ok; ++i) {  // nothing is allocated from here on
        const Launch &l = launches[i];
        SmallSeqs small;
        k.n = (int)(l.end - l.first);
        ok = place_records(p, parts.data() + l.first, l.end - l.first, small, &k.seqs, 0, st) &&
             launch_select_blocks(k, small, z, l.units, l.tokens, p->sm_count, st) == cudaSuccess;
    }
    return ok && end_read(p, st) ? AAF_OK : broke(p);
} catch (const std::bad_alloc &) {
    return AAF_ERR_INVALID_ARG;  // the host has no memory for the records; nothing was launched
}

int aaf_kv_attend_blocks(aaf_kv_pool *p, int32_t layer, const aaf_kv_attn *a, int32_t n, const aaf_ctx_t *ctxs, const int32_t *n_q,
                         const void *q_dev, const int32_t *blocks_dev, int32_t keep, void *out_dev, float *lse_dev,
                         void *workspace_dev, size_t workspace_bytes, void *stream) try {
    AAF_RANGE("aaf_kv_attend_blocks");
    if (!p) return AAF_ERR_INVALID_ARG;
    if (p->broken) return AAF_ERR_CUDA;
    long long total = 0;
    int rc = attn_check(p, layer, a, n, ctxs, n_q, q_dev, &total);
    if (rc != AAF_OK) return rc;
    if (!blocks_dev || (reinterpret_cast<uintptr_t>(blocks_dev) & 3u) || keep < 1 || keep > AAF_LIST_MAX_BLOCKS) return AAF_ERR_INVALID_ARG;
    if (!aligned16(out_dev) || (reinterpret_cast<uintptr_t>(lse_dev) & 3u) || !aligned16(workspace_dev)) return AAF_ERR_INVALID_ARG;
    if (workspace_bytes < attend_ws_bytes(p)) return AAF_ERR_DST_TOO_SMALL;
    const long long BS = p->g.BS;
    if (keep * BS > 1ll << 30) return AAF_ERR_TOO_MANY;  // listed tokens are numbered in ints
    std::vector<AttnSeq> rec;
    rc = batch_records(p, n, ctxs, n_q, false, rec, &total);
    if (rc != AAF_OK) return rc;
    AttnParams k = attn_params(p, layer, a, q_dev);
    k.out = out_dev;
    k.lse = lse_dev;
    k.part_o = static_cast<float *>(workspace_dev);
    k.part_ml = k.part_o + PART_ROWS * p->g.D;
    k.lists = blocks_dev;
    k.keep = keep;
    const int Hq = k.H * k.G, groups = (k.G + attend_blocks_rows(k.D, k.G) - 1) / attend_blocks_rows(k.D, k.G);
    // Lists are cut into parts so that the GPU is filled a whole number of times, by CTAs that share an SM or, where there is one for
    // each of them, by CTAs that have it to themselves and more warps: a round costs its part's keys per warp and a start (about 72
    // keys' time), a join twice that.  Microseconds with 1, 2, 3, 4, 6 parts: 1024 lists of 2048 keys 105, 111, 118, 124, 139; 512 ragged
    // ones of up to 4096 197, 179, 171, 169, 169; 128 of 1024 20.3, 19.8, 19.5, 19.6, 20.5, and 17.2 with an SM for each.  The figures are
    // those of groups of 4, heads of 128 and blocks of 16; with blocks of 8, 24 and 40, heads of 64 and 256, groups of 16 and 32, with a
    // bias and a cap (32 batches of 8 to 1024 lists) what the rule takes is within 4 % of the best of 1 to 12 parts, but for 64 lists of
    // 1024 keys in heads of 256: 22.9 us in one part, 20.0 in two.
    int longest = 0;
    for (AttnSeq &s : rec) {
        s.chunk = (int)(std::min<long long>(keep, nblk_of(p, s.len)) * BS);  // keys of a full list, for now
        longest = std::max(longest, s.chunk);
    }
    const int warps = attend_blocks_warps(k.D), ctas = attend_blocks_ctas(k.D, k.G);
    int chunk = 16;
    long long best = 1ll << 62;
    bool alone = false;
    for (int parts = 1; parts <= 64 && (parts == 1 || longest / 64 >= parts); parts += parts < 4 ? 1 : parts / 2) {
        const int c = ((longest + parts - 1) / parts + 15) / 16 * 16;
        long long t = 0;
        for (const AttnSeq &s : rec) t += (long long)((s.chunk + c - 1) / c) * s.nq;
        if (parts > 1 && t * Hq > PART_ROWS) break;  // partial results have to fit
        for (int one = 0; one < 2; ++one) {
            const long long at_once = (one ? 1 : ctas) * p->sm_count, rounds = (t * k.H * groups + at_once - 1) / at_once;
            const long long cost = rounds * (c / (one ? warps * ctas : warps) + 72) + (parts > 1 ? 144 : 0);
            if (cost < best && (!one || rounds == 1)) {
                best = cost;
                chunk = c;
                alone = one;
            }
        }
        if (t * k.H * groups > 16ll * p->sm_count) break;  // enough for even rounds
    }
    long long units = 0, rows = 0;
    int max_parts = 1;
    bool joined = false;
    for (AttnSeq &s : rec) {
        s.nsplit = (s.chunk + chunk - 1) / chunk;
        s.chunk = chunk;
        s.unit0 = (int)units;
        s.tok0 = s.row0;
        units += (long long)s.nsplit * s.nq;
        max_parts = std::max(max_parts, s.nsplit);
        if (s.nsplit > 1) {
            s.part0 = (int)rows;
            rows += (long long)s.nsplit * s.nq * Hq;
            joined = true;
        }
    }
    if (units * k.H * groups > (1ll << 31) - 1) return AAF_ERR_TOO_MANY;
    DeviceGuard guard(p->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (capturing(st)) return AAF_ERR_INVALID_ARG;
    k.n = n;
    k.total_units = (int)units;
    k.status = &p->s.ctl->status;
    p->last_stream = st;
    if (!begin_read(p, ctxs, n, st)) return broke(p);
    const int f16 = a->dtype == AAF_DTYPE_F16;
    SmallSeqs small;
    bool ok = place_records(p, rec, small, &k.seqs, 0, st) && launch_attend_blocks(k, small, f16, alone, st) == cudaSuccess;
    if (ok && joined) ok = launch_attend_join(k, small, f16, 0, (int)total, max_parts, p->sm_count, st) == cudaSuccess;
    return ok && end_read(p, st) ? AAF_OK : broke(p);
} catch (const std::bad_alloc &) {
    return AAF_ERR_INVALID_ARG;  // the host has no memory for the records; nothing was launched
}

int aaf_kv_batch_tables(aaf_kv_pool *p, const aaf_kv_batch_desc *d, int32_t n, const aaf_ctx_t *ctxs, const int32_t *n_new,
                        void *stream) try {
    AAF_RANGE("aaf_kv_batch_tables");
    if (!p || !d || d->struct_size != sizeof(aaf_kv_batch_desc) || n < 1 || !ctxs) return AAF_ERR_INVALID_ARG;
    if (p->broken) return AAF_ERR_CUDA;
    if ((reinterpret_cast<uintptr_t>(d->tables) | reinterpret_cast<uintptr_t>(d->lens) | reinterpret_cast<uintptr_t>(d->offsets) |
         reinterpret_cast<uintptr_t>(d->token_row)) & 3u)
        return AAF_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(d->positions) | reinterpret_cast<uintptr_t>(d->slots)) & 7u) return AAF_ERR_INVALID_ARG;
    if (!d->tables && !d->lens && !d->offsets && !d->token_row && !d->positions && !d->slots) return AAF_ERR_INVALID_ARG;
    if (d->rows > (1 << 30) || d->tokens > (1 << 30) || (d->tables && d->cols > (1 << 30))) return AAF_ERR_TOO_MANY;  // ints in the kernel
    std::vector<AttnSeq> rec;
    long long total = 0;
    const int rc = batch_records(p, n, ctxs, n_new, false, rec, &total);
    if (rc != AAF_OK) return rc;
    if (d->rows < n || d->tokens < total) return AAF_ERR_DST_TOO_SMALL;
    std::vector<TableRow> row(rec.size());
    std::transform(rec.begin(), rec.end(), row.begin(), [](const AttnSeq &s) { return TableRow{s.ctx, s.len, s.nq, s.row0}; });
    if (d->tables)
        for (const AttnSeq &s : rec)
            if (d->cols < nblk_of(p, s.len)) return AAF_ERR_DST_TOO_SMALL;
    if (d->tables && (long long)d->rows * ((long long)d->cols / 1024 + 1) > 1ll << 30) return AAF_ERR_TOO_MANY;
    DeviceGuard guard(p->device);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (capturing(st)) return AAF_ERR_INVALID_ARG;
    TablesParams k{};
    k.src = p->s.tables;
    k.tables = d->tables; k.lens = d->lens; k.offsets = d->offsets; k.token_row = d->token_row;
    k.positions = reinterpret_cast<long long *>(d->positions);
    k.slots = reinterpret_cast<long long *>(d->slots);
    k.max_blk = p->g.max_blk; k.BS = p->g.BS;
    k.n = n; k.cols = d->cols; k.rows = d->rows; k.tokens = d->tokens; k.total = (int)total;
    p->last_stream = st;
    if (!begin_read(p, ctxs, n, st)) return broke(p);
    SmallRows<SMALL_SEQS> none;
    const bool ok = (n <= SMALL_ROWS || place_records(p, row, none, &k.seqs, 0, st)) && launch_batch_tables(k, row.data(), st) == cudaSuccess;
    return ok && end_read(p, st) ? AAF_OK : broke(p);
} catch (const std::bad_alloc &) {
    return AAF_ERR_INVALID_ARG;  // the host has no memory for the records; nothing was launched
}

}  // extern "C"
