// The model of the CUDA runtime with an allocator that gives nothing large any more once a call has launched something: what a
// call needs of the host it has to have by then.
#include "sparse_model.cpp"

#include <cstdlib>
#include <new>

namespace {
int armed = -1;  // launches so far when the test began to look; -1: not looking
}
extern "C" void order_no_memory_behind_launches(int on) { armed = on ? (int)ops.size() : -1; }

static void *get(size_t n) {
    if (armed >= 0 && (int)ops.size() > armed && n > 8192) throw std::bad_alloc();  // the model's own needs are smaller
    void *q = std::malloc(n ? n : 1);
    if (!q) throw std::bad_alloc();
    return q;
}
void *operator new(size_t n) { return get(n); }
void *operator new[](size_t n) { return get(n); }
void operator delete(void *q) noexcept { std::free(q); }
void operator delete[](void *q) noexcept { std::free(q); }
void operator delete(void *q, size_t) noexcept { std::free(q); }
void operator delete[](void *q, size_t) noexcept { std::free(q); }
