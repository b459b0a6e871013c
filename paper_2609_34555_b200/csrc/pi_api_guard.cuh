// What the entry points beside pi_api.cu share: the context's device as the current one, the checks of layer and batch, and the
// device's view of a store.
#pragma once

#include "pi_common.cuh"

namespace {

class DeviceGuard {
public:
    explicit DeviceGuard(int device) {
        if (cudaGetDevice(&before_) != cudaSuccess) { (void)cudaGetLastError(); ok_ = false; return; }
        if (before_ != device) {
            if (cudaSetDevice(device) != cudaSuccess) { (void)cudaGetLastError(); ok_ = false; return; }
            changed_ = true;
        }
    }
    ~DeviceGuard() { if (changed_) (void)cudaSetDevice(before_); }
    DeviceGuard(const DeviceGuard&) = delete;
    DeviceGuard& operator=(const DeviceGuard&) = delete;
    bool ok() const { return ok_; }
private:
    int before_ = 0;
    bool changed_ = false, ok_ = true;
};

bool valid(const pi_ctx* ctx, int layer, int batch) {
    return ctx && layer >= 0 && layer < ctx->cfg.n_layers && batch >= 1 && batch <= ctx->cfg.max_batch;
}

// The device's address of a store in device memory or in pinned host memory.
int device_view(const void* p, void** out) {
    cudaPointerAttributes attr;
    if (cudaPointerGetAttributes(&attr, p) != cudaSuccess) { (void)cudaGetLastError(); return PI_ERR_NOT_PINNED; }
    *out = const_cast<void*>(p);
    if (attr.type == cudaMemoryTypeHost) {
        if (!attr.devicePointer) return PI_ERR_NOT_PINNED;
        *out = attr.devicePointer;
    } else if (attr.type != cudaMemoryTypeDevice && attr.type != cudaMemoryTypeManaged) {
        return PI_ERR_NOT_PINNED;
    }
    return PI_OK;
}

}  // namespace
