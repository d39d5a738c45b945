// What the translation units of libgrawa share on the host side.
#pragma once
#include "../../include/grawa.h"

#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

namespace grawa {

extern std::atomic<int64_t> g_launches;                              // kernels launched since the library was loaded
bool dependent_launch();                                             // the "dependent_launch" option
grawa_status cuda_fail(cudaError_t err, const char* what);           // keeps the text for grawa_last_cuda_error()

#define GRAWA_CUDA_TRY(expr)                                        \
    do {                                                            \
        cudaError_t err__ = (expr);                                 \
        if (err__ != cudaSuccess) return cuda_fail(err__, #expr);   \
    } while (0)

}  // namespace grawa
