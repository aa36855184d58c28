// Two threads that launch the same kernels for the first time; built with the thread sanitizer.
#include <thread>

#include "attend_internal.h"

extern "C" {
cudaError_t CUDARTAPI cudaGetDevice(int *d) {
    *d = 0;
    return cudaSuccess;
}
cudaError_t CUDARTAPI cudaFuncSetAttribute(const void *, cudaFuncAttribute, int) { return cudaSuccess; }
}

int main() {
    static aafkv::SmemSeen seen[64];
    auto run = [] {
        for (auto &s : seen)
            if (aafkv::allow_smem(nullptr, 1 << 17, &s) != cudaSuccess) return;
    };
    std::thread a(run), b(run);
    a.join();
    b.join();
    for (auto &s : seen)
        if (s != 1) return 1;
    return 0;
}
