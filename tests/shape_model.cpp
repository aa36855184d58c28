// How a choice of blocks is cut (select_shape of select_blocks.cu, whose text SHAPE_SOURCE is) on the CPU.
#include <algorithm>
#include <cstdint>

#include "sparse_internal.h"

namespace aafkv {
constexpr int SCORE_BLOCKS = 128;
#include SHAPE_SOURCE
}  // namespace aafkv

extern "C" void shape_of(int H, int G, int D, int n, int max_nq, long long m_tiles, int sm_count, long long *out) {
    aafkv::SelectParams p{};
    p.H = H, p.G = G, p.D = D;
    const aafkv::SelectShape z = aafkv::select_shape(p, n, max_nq, m_tiles, sm_count, 0);
    const long long v[] = {z.tile, z.heads_p, z.n, z.slabs, z.reps, z.buffers, z.together, z.blocks, (long long)aafkv::score_smem(z), aafkv::SCORE_SMEM};
    std::copy(v, v + 10, out);
}
