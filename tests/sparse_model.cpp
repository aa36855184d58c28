// The model of the CUDA runtime with the launchers of sparse attention and of a batch's tables beside the others.
#include "order_model.cpp"

#include "sparse_internal.h"

namespace aafkv {
cudaError_t launch_summarize(const SummaryParams &, const SmallSeqs &, int, cudaStream_t st) { return launch("summarize", st); }
SelectShape select_shape(const SelectParams &, int, int, long long, int, int f16) {
    SelectShape z{};
    z.tile = 16;
    z.heads_p = 1;
    z.n = 32;
    z.slabs = z.reps = z.buffers = 1;
    z.blocks = 128;
    z.f16 = f16;
    return z;
}
cudaError_t launch_select_blocks(const SelectParams &, const SmallSeqs &, const SelectShape &, long long, long long, int, cudaStream_t st) {
    return launch("choose", st);
}
cudaError_t launch_attend_blocks(const AttnParams &, const SmallSeqs &, int, bool, cudaStream_t st) { return launch("attend_blocks", st); }
int attend_blocks_rows(int, int) { return 8; }
int attend_blocks_warps(int) { return 4; }
int attend_blocks_ctas(int, int) { return 2; }
cudaError_t launch_batch_tables(const TablesParams &, const TableRow *, cudaStream_t st) { return launch("tables", st); }
}  // namespace aafkv
