// Internal to libqllm: the limit of dynamic LDS of kernels whose launches ask for different amounts.
#ifndef QLLM_LDS_LIMIT_H
#define QLLM_LDS_LIMIT_H

#include <hip/hip_runtime.h>

#include <stdint.h>

#include <mutex>

#include "qllm.h"

extern "C" void qllm_note_hip_error(const char *step, const char *name);

namespace qllm_detail {

// The limit belongs to all threads that launch the kernel: written for each launch, it could be lowered by one thread's smaller launch
// between another's limit and launch.  It is raised once per kernel and device, to `most`, which no launch of the kernel goes beyond.
inline int32_t raise_lds_limit(const void *kernel, int most, const char *step)
{
    constexpr int ROOM = 128; // kernels; one that finds no room is raised to the same `most` for every launch
    struct Raised {
        const void *kernel;
        uint64_t devices;
    };
    static std::mutex lock;
    static Raised raised[ROOM];
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess) {
        std::lock_guard<std::mutex> hold(lock);
        int at = 0;
        while (at < ROOM && raised[at].kernel && raised[at].kernel != kernel) ++at;
        const bool kept = at < ROOM && device < 64;
        if (kept && (raised[at].devices >> device & 1u)) return QLLM_OK;
        e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, most);
        if (e == hipSuccess) {
            if (kept) raised[at].kernel = kernel, raised[at].devices |= 1ull << device;
            return QLLM_OK;
        }
    }
    (void)hipGetLastError();
    qllm_note_hip_error(step, hipGetErrorName(e));
    return QLLM_ERR_HIP;
}

} // namespace qllm_detail

#endif
