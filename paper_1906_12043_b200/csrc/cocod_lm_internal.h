// What the translation units of the language-model operators share: the handle and the host-side helpers.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "cocod_host.h"
#include "cocod_lm.h"

struct cocod_lm {
    int *order = nullptr;                  // device: the groups by size
    float *parts = nullptr;                // device: parts of tiles, 256 x 256 for each pair of CTAs
    int *flag = nullptr;                   // device: what the kernels met
    int device = -1;                       // the one current at creation
    long long launches = 0;
};

#define TRY_CUDA(call) do { if ((call) != cudaSuccess) { cudaGetLastError(); return COCOD_ERR_CUDA; } ++h->launches; } while (0)

namespace cocod {

constexpr int64_t MAX_DIM = (1ll << 31) - 1024;

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int size_of(int type) { return type == COCOD_BF16 ? 2 : type == COCOD_F32 ? 4 : 0; }

inline int sm_count()
{
    static int count[MAX_DEVICES] = {};
    const int dev = current_device();
    if (dev < 0) return 0;
    if (count[dev] == 0 && cudaDeviceGetAttribute(&count[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        count[dev] = 0;
    }
    return count[dev];
}

}  // namespace cocod
