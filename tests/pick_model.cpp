// The selection kernel of select_blocks.cu on the CPU: a thread of the host for every thread of a CTA, warp functions and barriers as
// meetings of threads.  PICK_SOURCE is the kernel's text.  Built with the address sanitizer, so that an access beyond the list, the
// scores or the kernel's own shared arrays ends the process.
//
//   pick_model WARPS total keep sink recent room < scores > blocks
#include <cuda_runtime.h>

#include <atomic>
#include <barrier>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <limits>
#include <memory>
#include <thread>
#include <vector>

#undef __shared__
#undef __global__
#undef __device__
#undef __forceinline__
#undef __launch_bounds__
#undef __grid_constant__
#define __shared__ static
#define __global__
#define __device__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __grid_constant__

#define CUDART_INF_F std::numeric_limits<float>::infinity()

namespace {
struct Place {
    unsigned x;
};
thread_local Place threadIdx_, blockIdx_;
#define threadIdx threadIdx_
#define blockIdx blockIdx_
int warps = 0;
std::unique_ptr<std::barrier<>> cta;
std::vector<std::unique_ptr<std::barrier<>>> meet;
std::vector<unsigned long long> slots;  // a lane's word in a warp function

void __syncthreads() { cta->arrive_and_wait(); }
// every lane gives a word and sees those of its warp
template <typename F> auto together(unsigned long long mine, F &&f) {
    const unsigned w = threadIdx.x / 32;
    slots[threadIdx.x] = mine;
    meet[w]->arrive_and_wait();
    auto r = f(&slots[w * 32]);
    meet[w]->arrive_and_wait();
    return r;
}
unsigned lane_() { return threadIdx.x & 31; }
template <typename T> T from_lane(T v, int lane) {
    return together((unsigned long long)(uint32_t)v, [&](unsigned long long *s) { return (T)(uint32_t)s[lane & 31]; });
}
template <typename T> T __shfl_sync(unsigned, T v, int lane) { return from_lane(v, lane); }
template <typename T> T __shfl_down_sync(unsigned, T v, int d) { return from_lane(v, (int)lane_() + d < 32 ? (int)lane_() + d : (int)lane_()); }
template <typename T> T __shfl_up_sync(unsigned, T v, int d) { return from_lane(v, (int)lane_() >= d ? (int)lane_() - d : (int)lane_()); }
unsigned __ballot_sync(unsigned, bool p) {
    return together(p, [](unsigned long long *s) {
        unsigned r = 0;
        for (int i = 0; i < 32; ++i) r |= (unsigned)(s[i] != 0) << i;
        return r;
    });
}
unsigned __reduce_min_sync(unsigned, unsigned v) {
    return together(v, [](unsigned long long *s) { unsigned long long r = s[0]; for (int i = 1; i < 32; ++i) r = s[i] < r ? s[i] : r; return (unsigned)r; });
}
unsigned __reduce_max_sync(unsigned, unsigned v) {
    return together(v, [](unsigned long long *s) { unsigned long long r = s[0]; for (int i = 1; i < 32; ++i) r = s[i] > r ? s[i] : r; return (unsigned)r; });
}
uint32_t atomicAdd(uint32_t *p, uint32_t v) { return __atomic_fetch_add(p, v, __ATOMIC_SEQ_CST); }
void atomicMin(uint32_t *p, uint32_t v) {
    for (uint32_t o = __atomic_load_n(p, __ATOMIC_SEQ_CST); v < o && !__atomic_compare_exchange_n(p, &o, v, false, __ATOMIC_SEQ_CST, __ATOMIC_SEQ_CST);) {}
}
void atomicMax(uint32_t *p, uint32_t v) {
    for (uint32_t o = __atomic_load_n(p, __ATOMIC_SEQ_CST); v > o && !__atomic_compare_exchange_n(p, &o, v, false, __ATOMIC_SEQ_CST, __ATOMIC_SEQ_CST);) {}
}
uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((unsigned long long)a * b >> 32); }
int __popc(uint32_t v) { return __builtin_popcount(v); }
int __ffs(uint32_t v) { return __builtin_ffs((int)v); }
float __uint_as_float(uint32_t v) {
    float f;
    memcpy(&f, &v, 4);
    return f;
}
template <typename T> T __ldcg(const T *p) { return *p; }
template <typename T> T min(T a, T b) { return b < a ? b : a; }
template <typename T> T max(T a, T b) { return a < b ? b : a; }

uint32_t *shared_keys = nullptr;
struct AttnSeq {
    int row0, tok0, key0;
};
struct SmallSeqs {
    AttnSeq e[1];
};
struct SelectParams {
    const AttnSeq *seqs;
    const uint32_t *keys;
    int *blocks;
    float *scores;
    long long pitch;
    int BS, H, n, keep, sink, recent;
};
constexpr int PICK_KEYS = 12288;
float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

#include PICK_SOURCE

template <int WARPS> void run(const SelectParams &p, int room) {
    warps = WARPS;
    cta = std::make_unique<std::barrier<>>(WARPS * 32);
    for (int w = 0; w < WARPS; ++w) meet.push_back(std::make_unique<std::barrier<>>(32));
    slots.resize(WARPS * 32);
    SmallSeqs small{};
    std::vector<std::thread> all;
    for (int t = 0; t < WARPS * 32; ++t)
        all.emplace_back([&, t] {
            threadIdx.x = (unsigned)t;
            blockIdx.x = 0;
            pick_blocks_kernel<WARPS>(p, small, room);
        });
    for (auto &t : all) t.join();
}
}  // namespace

int main(int, char **a) {
    const int w = atoi(a[1]), total = atoi(a[2]), room = atoi(a[6]);
    SelectParams p{};
    p.pitch = (total + 3) / 4 * 4;
    p.BS = p.H = p.n = 1;
    p.keep = atoi(a[3]), p.sink = atoi(a[4]), p.recent = atoi(a[5]);
    AttnSeq s{0, 0, total - 1};
    p.seqs = &s;
    auto keys = std::make_unique<uint32_t[]>((size_t)p.pitch);
    if (fread(keys.get(), 4, (size_t)total, stdin) != (size_t)total) return 2;
    auto blocks = std::make_unique<int[]>((size_t)p.keep);
    auto scores = std::make_unique<float[]>((size_t)p.keep);
    auto own = std::make_unique<uint32_t[]>((size_t)room + 4);
    for (int i = 0; i < p.keep; ++i) blocks[(size_t)i] = -2;
    shared_keys = reinterpret_cast<uint32_t *>((reinterpret_cast<uintptr_t>(own.get()) + 15) / 16 * 16);
    p.keys = keys.get(), p.blocks = blocks.get(), p.scores = scores.get();
    if (w == 4) run<4>(p, room);
    else run<8>(p, room);
    fwrite(blocks.get(), 4, (size_t)p.keep, stdout);
    return 0;
}
