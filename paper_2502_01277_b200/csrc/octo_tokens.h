// What the token calls (octo_tokens.cu, octo_attend*.cu) share on the host.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "octo.h"
#include "octo_kernels.h"

namespace octo {

// Makes `device` current for the length of a call and puts the caller's device back.
struct DeviceScope {
    int before = -1;
    cudaError_t error;
    explicit DeviceScope(int device) {
        error = cudaGetDevice(&before);
        if (error == cudaSuccess && before != device) error = cudaSetDevice(device);
        else if (error == cudaSuccess) before = -1;  // nothing to put back
    }
    ~DeviceScope() {
        if (before >= 0) cudaSetDevice(before);
    }
};

inline bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Number of SMs of a device (looked up once per device and process).
cudaError_t sm_count_of(int device, int* out);

cudaError_t launch_positions(const octo_item_t* d_items, int max_items, const int* d_n_items, int slot_w, int slot_h,
                             int patch, int keep_aspect, const float* d_times, int n_frames, float* d_positions,
                             uint8_t* d_visible, cudaStream_t stream);

}  // namespace octo
