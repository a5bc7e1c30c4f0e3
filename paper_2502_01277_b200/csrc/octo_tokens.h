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
// An output whose rows or heads lie on one another (an expanded tensor, windows of one that overlap, row r + 1 of head h in
// the place of row r of head h + 1): what stayed there would be a matter of time.
inline bool rows_coincide(const octo_heads_t& t, int64_t rows, int heads, int dim) {
    auto near = [&](int64_t stride) { return stride > -dim && stride < dim; };
    if (rows < 1 || heads < 1) return false;
    return (rows > 1 && near(t.row_stride)) || (heads > 1 && near(t.head_stride)) ||
           (rows > 1 && heads > 1 && (near(t.row_stride - t.head_stride) || near(t.row_stride + t.head_stride)));
}
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Division by a number that is the same for a whole launch: exact for 0 <= n < 2^31 (multiply by the reciprocal rounded
// up to 33 bits, whose top bit is the addition of n).
struct FastDiv {
    unsigned mul, shift;
    void set(unsigned d) {
        shift = 0;
        while ((1ull << shift) < d) ++shift;
        mul = (unsigned)(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ int div(int n) const { return (int)((__umulhi(mul, (unsigned)n) + (unsigned)n) >> shift); }
};

// Number of SMs of a device (looked up once per device and process).
cudaError_t sm_count_of(int device, int* out);

}  // namespace octo
