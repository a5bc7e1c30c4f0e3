// What the attention kernels share: arguments, segments, the layout of partial results.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "octo_tokens.h"

namespace octo {

// Range checks of the checked build for kernels whose status word may be missing (see OCTO_IN_RANGE).
#ifdef OCTO_BOUNDS_CHECK
__device__ __forceinline__ bool token_in_range(bool ok, unsigned int* status) {
    if (!ok && status) atomicOr(status, OCTO_STATUS_BOUNDS);
    return ok;
}
#define OCTO_TOKEN_IN_RANGE(cond, status_ptr) token_in_range((cond), (status_ptr))
#else
#define OCTO_TOKEN_IN_RANGE(cond, status_ptr) (true)
#endif

struct AttendArgs {
    const void *q, *k, *v;
    void* out;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;  // strides, elements
    const int* q_offsets;
    const int* k_offsets;
    int64_t q_rows, k_rows, q_first, k_first, q_total, k_total, max_q, max_k;
    const uint8_t* mask;
    float scale_log2;  // scale * log2(e): the softmax is taken to base 2
    int segments, heads, kv_heads, group, dim;
    FastDiv group_div;
    // Work split over the keys: split i of a segment takes its key rows [i * chunk, (i + 1) * chunk).  A
    // segment of at most `chunk` keys has one active split, which writes the result itself; those of more
    // leave (unnormalised sum, reference maximum, sum of weights) of every row for the joining kernel.
    int splits, chunk;
    float* part_o;    // [splits][q_total][heads][dim]
    float2* part_ml;  // [splits][q_total][heads]
    unsigned int* status;
};

struct Segment {
    int64_t q0, k0;
    int qn, kn;
};

__device__ __forceinline__ int64_t clip_row(int64_t v, int64_t total) { return v < 0 ? 0 : (v > total ? total : v); }

__device__ __forceinline__ Segment segment_of(const AttendArgs& a, int s) {
    const int64_t qb = a.q_offsets ? a.q_offsets[s] : s, qe = a.q_offsets ? a.q_offsets[s + 1] : s + 1;
    const int64_t kb = a.k_offsets ? a.k_offsets[s] : s, ke = a.k_offsets ? a.k_offsets[s + 1] : s + 1;
    Segment g;
    g.q0 = clip_row((qb - a.q_first) * a.q_rows, a.q_total);
    g.k0 = clip_row((kb - a.k_first) * a.k_rows, a.k_total);
    const int64_t qn = clip_row((qe - a.q_first) * a.q_rows, a.q_total) - g.q0;
    const int64_t kn = clip_row((ke - a.k_first) * a.k_rows, a.k_total) - g.k0;
    g.qn = (int)(qn < 0 ? 0 : (qn < a.max_q ? qn : a.max_q));
    g.kn = (int)(kn < 0 ? 0 : (kn < a.max_k ? kn : a.max_k));
    return g;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

}  // namespace octo
