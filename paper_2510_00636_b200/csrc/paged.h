// Shared by the translation units of the paged cache.
#pragma once

#include <atomic>

#include "ea_internal.h"

// Called by one thread of each of `parts` CTAs, once the threads that wrote have met at a barrier: whether the others have all
// been here (and what they wrote can be read).  The last one puts the counter back to zero.
__device__ __forceinline__ bool arrives_last(unsigned* counter, int parts) {
    __threadfence();
    const bool last = atomicAdd(counter, 1u) == (unsigned)parts - 1u;
    if (last) {
        *counter = 0;
        __threadfence();
    }
    return last;
}

// Whether all others have arrived already (then the caller is the last, and the counter is put back to zero).
__device__ __forceinline__ bool others_arrived(unsigned* counter, int parts) {
    const bool last = *reinterpret_cast<volatile unsigned*>(counter) == (unsigned)parts - 1u;
    if (last) {
        __threadfence();
        *counter = 0;
    }
    return last;
}

// Lets a kernel use more than 48 KiB of dynamic shared memory: once per device (a runtime call that a generation step
// would otherwise pay at each layer); `done` belongs to the kernel.
template <class Kernel>
static inline ea_status ea_allow_smem(Kernel kernel, int bytes, int device, std::atomic<uint64_t>& done) {
    const uint64_t bit = 1ull << (device & 63);
    if (device < 64 && (done.load(std::memory_order_acquire) & bit)) return EA_OK;
    EA_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    if (device < 64) done.fetch_or(bit, std::memory_order_release);
    return EA_OK;
}

// A buffer of a call.  Kernels read inputs in any order beside their writes, so that an output may overlap nothing else.
struct Span {
    const void* at;
    long long bytes;
    bool output;
};
template <int N>
static inline bool outputs_overlap(const Span (&spans)[N]) {
    for (int i = 0; i < N; ++i)
        for (int j = 0; j < i; ++j) {
            const uintptr_t a = reinterpret_cast<uintptr_t>(spans[i].at), b = reinterpret_cast<uintptr_t>(spans[j].at);
            if ((spans[i].output || spans[j].output) && a && b && spans[i].bytes > 0 && spans[j].bytes > 0 &&
                a < b + (unsigned long long)spans[j].bytes && b < a + (unsigned long long)spans[i].bytes)
                return true;
        }
    return false;
}

ea_status ea_check_paged_shape(const ea_paged_shape* s);
// Workspace of ea_paged_attention (partial results of lists that several CTAs share).
size_t ea_paged_attn_ws_bytes(const ea_paged_shape& s, int max_q);
