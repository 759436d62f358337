// What the entry points share: the launch counter, the record of the last error, and the checks of arguments.
#pragma once
#include <algorithm>
#include <atomic>
#include <cstdio>

#include "carnator.h"
#include "common.cuh"

#define CARNATOR_HIDDEN __attribute__((visibility("hidden")))

namespace carnator {

CARNATOR_HIDDEN extern std::atomic<long long> g_launches;
CARNATOR_HIDDEN extern thread_local char g_cuda_error[256];
CARNATOR_HIDDEN carnator_status check_device();      // whether the current device is an sm_100 one

inline carnator_status cuda_fail(cudaError_t e, const char* where) { return cuda_error(e, where, g_cuda_error, sizeof(g_cuda_error)); }

#define CUDA_TRY(expr)                                              \
    do {                                                            \
        cudaError_t e__ = (expr);                                   \
        if (e__ != cudaSuccess) return cuda_fail(e__, #expr);       \
    } while (0)

#define LAUNCH_CHECK(name)                                          \
    do {                                                            \
        g_launches.fetch_add(1, std::memory_order_relaxed);         \
        cudaError_t e__ = cudaGetLastError();                       \
        if (e__ != cudaSuccess) return cuda_fail(e__, name);        \
    } while (0)

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline bool dtype_ok(int32_t d) { return d == CARNATOR_DTYPE_F32 || d == CARNATOR_DTYPE_BF16; }
inline int64_t dtype_bytes(int32_t d) { return d == CARNATOR_DTYPE_F32 ? 4 : d == CARNATOR_DTYPE_BF16 ? 2 : 1; }
inline int64_t dtype_unit(int32_t d) { return 16 / dtype_bytes(d); }       // elements in 16 bytes

// Element strides of an operand with `n` axes in front of `row` contiguous elements: whole 16-byte steps and at most 2^38, not
// negative.  For one that is written (or read through TMA, `positive`) no two rows may overlap (be the same).
inline bool axes_ok(const int64_t* stride, const int64_t* size, int n, int64_t row, int32_t dtype, bool written, bool positive) {
    int64_t st[3], sz[3];
    int used = 0;
    for (int i = 0; i < n; ++i) {
        if (size[i] == 1) continue;                   // never used
        if (stride[i] < 0 || stride[i] % dtype_unit(dtype) || stride[i] > (int64_t(1) << 38) || (positive && stride[i] == 0)) return false;
        st[used] = stride[i]; sz[used] = size[i]; ++used;
    }
    if (!written) return true;
    int64_t extent = row;
    for (int k = 0; k < used; ++k) {                  // from the innermost axis out
        int at = k;
        for (int i = k + 1; i < used; ++i) if (st[i] < st[at]) at = i;
        std::swap(st[k], st[at]); std::swap(sz[k], sz[at]);
        if (st[k] < extent) return false;
        extent += st[k] * (sz[k] - 1);
    }
    return true;
}
inline bool rows32(const void* p, const int64_t st[2], int32_t dtype) {      // whether every row starts on a 32-byte boundary
    return !p || (aligned(p, 32) && st[0] % (2 * dtype_unit(dtype)) == 0 && st[1] % (2 * dtype_unit(dtype)) == 0);
}
inline bool vec16(const void* p, int64_t stride, int32_t dtype) { return !p || (aligned(p, 16) && stride % dtype_unit(dtype) == 0); }

}  // namespace carnator
