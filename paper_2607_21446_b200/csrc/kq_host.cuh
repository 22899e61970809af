// Host helpers that the translation units of the library share: the launch counter, device properties, once-per-device set-up,
// alignment checks and launches.  Everything but the counter has internal linkage: each unit (and each build of the library
// loaded into one process) keeps its own "done once" flags for its own kernels.
#pragma once
#include <atomic>
#include <utility>

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/kroquant.h"

// kernels launched by the process (defined in kroquant_api.cu)
extern std::atomic<int64_t> g_launches __attribute__((visibility("hidden")));

namespace {

int sm_count() {
    static int cached[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (cached[dev] == 0) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
        cached[dev] = n;
    }
    return cached[dev];
}

// Per-device "do once" for set-up that belongs to a device (function attributes).  needed() is true until
// done() has been called with the same device current; a race between two first calls only repeats the set-up.
struct DeviceOnce {
    std::atomic<int> flag[64];
    DeviceOnce() { for (auto& f : flag) f.store(0); }
    static int dev() {
        int d = -1;
        if (cudaGetDevice(&d) != cudaSuccess || d < 0 || d >= 64) return -1;
        return d;
    }
    bool needed() const { const int d = dev(); return d < 0 || !flag[d].load(std::memory_order_acquire); }
    void done() { const int d = dev(); if (d >= 0) flag[d].store(1, std::memory_order_release); }
};

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int type_size(int t) { return t == KQ_OUT_F32 ? 4 : 2; }
bool known_type(int t) { return t == KQ_OUT_F32 || t == KQ_OUT_BF16 || t == KQ_OUT_FP16; }
bool element_aligned(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % type_size(type) == 0; }
// pointer and pitch (in elements) both keep rows on `bytes`-byte boundaries
bool rows_aligned(const void* p, int64_t pitch, int type, int bytes) {
    return !p || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && pitch * type_size(type) % bytes == 0);
}

// a launch that may set up while the kernel before it drains (every kernel here waits for it before it touches memory)
void launch_config(cudaLaunchConfig_t* cfg, cudaLaunchAttribute* attr, dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st) {
    *cfg = {};
    cfg->gridDim = grid;
    cfg->blockDim = block;
    cfg->dynamicSmemBytes = smem;
    cfg->stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg->attrs = attr;
    cfg->numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = (unsigned)cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg->numAttrs = 2;
    }
}
template <typename... Params, typename... Args>
kq_status_t launch(const cudaLaunchConfig_t& cfg, void (*kernel)(Params...), Args&&... args) {
    if (cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...) != cudaSuccess) {
        (void)cudaGetLastError();
        return KQ_ERR_CUDA;
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return KQ_OK;
}

}  // namespace
