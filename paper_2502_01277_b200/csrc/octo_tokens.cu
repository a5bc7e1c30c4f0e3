// Tokens of a transformer behind the stage: positions of the patches of packed crops, and the norm of query
// and key heads together with their rotation by those positions (include/octo.h).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <atomic>

#include "octo_tokens.h"

namespace octo {

// ---------------------------------------------------------------------------------------
// Positions.  One CTA per item: its threads first make one coordinate per patch column and patch row (a
// division in binary64 each, of which a patch of its own would need two), then write the item's block of
// (time, y, x) triples with neighbouring threads on neighbouring words.  Bound by the bytes written.
// ---------------------------------------------------------------------------------------
constexpr int kPosThreads = 128;
constexpr int kPosMaxSide = 2048;  // patches along a side of a slot

// Image size and place inside the slot, in integers (the fit of an aspect-preserving crop).
__device__ __forceinline__ void fit_in_slot(int cw, int ch, int ow, int oh, int keep_aspect, int& nw, int& nh, int& pl,
                                            int& pt) {
    nw = ow;
    nh = oh;
    if (keep_aspect) {
        if ((long long)ow * ch <= (long long)oh * cw) nh = max(1, (int)((2LL * ow * ch + cw) / (2LL * cw)));
        else nw = max(1, (int)((2LL * oh * cw + ch) / (2LL * ch)));
    }
    pl = (ow - nw) / 2;
    pt = (oh - nh) / 2;
}

__global__ void __launch_bounds__(kPosThreads)
positions_kernel(const octo_item_t* __restrict__ items, int max_items, const int* __restrict__ n_items, int slot_w,
                 int slot_h, int patch, int keep_aspect, const float* __restrict__ times, int n_frames,
                 float* __restrict__ positions, uint8_t* __restrict__ visible) {
    extern __shared__ float s_axis[];  // [gw] x, [gh] y, then one byte per column and row: shows the image
    const int gw = slot_w / patch, gh = slot_h / patch, patches = gw * gh;
    float* s_x = s_axis;
    float* s_y = s_axis + gw;
    uint8_t* s_vx = reinterpret_cast<uint8_t*>(s_axis + gw + gh);
    uint8_t* s_vy = s_vx + gw;
    const int i = blockIdx.x;
    pdl_wait();
    if (n_items && i >= *n_items) return;
    const octo_item_t it = items[i];
    const int cw = it.rx1 - it.rx0, ch = it.ry1 - it.ry0;
    const bool good = cw > 0 && ch > 0 && it.rx1 > it.rx0 && it.ry1 > it.ry0 && it.frame >= 0 && it.frame < n_frames;
    int nw = 1, nh = 1, pl = 0, pt = 0;
    if (good) fit_in_slot(cw, ch, slot_w, slot_h, keep_aspect, nw, nh, pl, pt);
    for (int k = threadIdx.x; k < gw + gh; k += kPosThreads) {
        const bool col = k < gw;
        const int g = col ? k : k - gw, pad = col ? pl : pt, n = col ? nw : nh, size = col ? cw : ch;
        const int origin = col ? it.rx0 : it.ry0;
        // the centre of the patch, in halves of a slot pixel from the image's edge; one rounding at the end
        const double off = (double)((2 * g + 1) * patch - 2 * pad) * (double)size / (double)(2 * n);
        s_axis[k] = good ? (float)((double)origin + off) : 0.0f;
        s_vx[k] = good && g * patch < pad + n && (g + 1) * patch > pad ? 1 : 0;
    }
    __syncthreads();
    const float t = good && times ? times[it.frame] : 0.0f;
    float* out = positions + (size_t)i * patches * 3;
    // word f of the block is component f % 3 of patch f / 3; the pair (row, column) follows by steps
    for (int f = threadIdx.x; f < patches * 3; f += kPosThreads) {
        const int p = f / 3, c = f - 3 * p, gy = p / gw, gx = p - gy * gw;
        out[f] = c == 0 ? t : (c == 1 ? s_y[gy] : s_x[gx]);
    }
    if (visible) {
        uint8_t* vis = visible + (size_t)i * patches;
        for (int p = threadIdx.x; p < patches; p += kPosThreads) {
            const int gy = p / gw, gx = p - gy * gw;
            vis[p] = s_vy[gy] & s_vx[gx];
        }
    }
}

cudaError_t launch_positions(const octo_item_t* d_items, int max_items, const int* d_n_items, int slot_w, int slot_h,
                             int patch, int keep_aspect, const float* d_times, int n_frames, float* d_positions,
                             uint8_t* d_visible, cudaStream_t stream) {
    if (max_items < 1) return cudaSuccess;
    const size_t smem = 5 * (size_t)(slot_w / patch + slot_h / patch);
    return launch_kernel(positions_kernel, dim3((unsigned)max_items), dim3(kPosThreads), smem, stream, d_items, max_items,
                         d_n_items, slot_w, slot_h, patch, keep_aspect, d_times, n_frames, d_positions, d_visible);
}

cudaError_t sm_count_of(int device, int* out) {
    static std::atomic<int> known[64];
    int n = device >= 0 && device < 64 ? known[device].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        const cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device);
        if (e != cudaSuccess) return e;
        if (device < 64) known[device].store(n, std::memory_order_relaxed);
    }
    *out = n;
    return cudaSuccess;
}

// ---------------------------------------------------------------------------------------
// Norm and rotation.  Bound by HBM: every element is read once and written once.  A group of lanes owns a
// token and walks over its heads, so that the sine and cosine of the token's pairs are made once and stay in
// registers for all heads.  A lane owns VP pairs of every head, both elements of each: for halves two runs of
// VP elements that lie `pairs` apart, for neighbours one run of 2 VP, so that no element changes lanes;
// elements behind the rotated ones are given to lanes as pairs with the angle zero.
// ---------------------------------------------------------------------------------------
struct RotTensor {
    const void* in;
    void* out;
    const void* weight;
    int64_t in_row, in_head, out_row, out_head;
    int heads;
};
struct RotArgs {
    RotTensor t[2];
    const void* positions;
    const float* freqs;
    const int* axes;
    const int* n_items;
    int64_t rows, item_rows;
    int head_dim, pairs, num_axes, positions_are_int;
    float eps;
};

constexpr int kRotThreads = 256;
constexpr int kRotBatch = 4;  // heads of a lane group that are in flight together

template <typename T> struct Conv;
template <> struct Conv<__half> {
    static __device__ __forceinline__ float up(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half down(float v) { return __float2half_rn(v); }
};
template <> struct Conv<__nv_bfloat16> {
    static __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 down(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Conv<float> {
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};

// N elements of T that start on a multiple of their own size (at most 16 bytes at a time).
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Run {
    T v[N];
};

// Sine and cosine of position * freq.  The product of two binary32 numbers is exact in binary64, and so is
// the subtraction of the whole turns up to 2^-53 of their number: the phase keeps binary32's precision
// however far the position.
__device__ __forceinline__ void turn_of(double position, float freq, float& c, float& s) {
    const double turns = position * (double)freq * 0.15915494309189533577;
    const double half_turns = 2.0 * (turns - rint(turns));  // in [-1, 1]
    const float h = (float)half_turns;
    const float rest = (float)(half_turns - (double)h) * 3.14159265f;  // what the rounding of h left, as an angle
    float s0, c0;
    sincospif(h, &s0, &c0);
    s = fmaf(c0, rest, s0);
    c = fmaf(-s0, rest, c0);
}

// Lanes per token: LP (a power of two).  ILV: pairs are neighbours.  NU units of VP pairs per lane.
template <typename T, int VP, int NU, bool ILV>
__global__ void __launch_bounds__(kRotThreads)
rotate_kernel(const __grid_constant__ RotArgs a, int lp_log, int heads_per_group) {
    pdl_wait();
    const int lp = 1 << lp_log, lane = threadIdx.x & (lp - 1);
    const int64_t row = ((int64_t)blockIdx.x * kRotThreads + threadIdx.x) >> lp_log;
    int64_t rows = a.rows;
    if (a.n_items) {
        const int64_t n = *a.n_items;
        rows = n <= 0 ? 0 : (n < rows / a.item_rows + 1 ? min(rows, n * a.item_rows) : rows);
    }
    if (row >= rows) return;  // a group leaves as a whole; the shuffles below stay inside a group
    const unsigned group = (lp == 32 ? 0xffffffffu : ((1u << lp) - 1u)) << ((threadIdx.x & 31) & ~(lp - 1));
    const int total = a.t[0].heads + a.t[1].heads;
    const int h0 = blockIdx.y * heads_per_group, h1 = min(total, h0 + heads_per_group);

    // which elements this lane owns, and how they turn
    const int half = a.head_dim / 2, rest = half - a.pairs;  // pairs that turn, pairs that do not
    int e0[NU], e1[NU];  // first element of the two runs of a unit (ILV: e1 = e0 + VP)
    bool own[NU];
    float cs[NU * VP], sn[NU * VP];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const int p = (lane + u * lp) * VP;  // first pair of the unit
        own[u] = p < half;
        const bool turning = p < a.pairs;
        if (ILV) {
            e0[u] = 2 * p;
            e1[u] = 2 * p + VP;
        } else {
            e0[u] = turning ? p : p + a.pairs;
            e1[u] = e0[u] + (turning ? a.pairs : rest);
        }
#pragma unroll
        for (int j = 0; j < VP; ++j) {
            float c = 1.0f, s = 0.0f;
            if (turning) {
                const int axis = a.axes[p + j];
                if (axis >= 0 && axis < a.num_axes) {
                    const int64_t at = row * a.num_axes + axis;
                    const double pos = a.positions_are_int ? (double)static_cast<const int*>(a.positions)[at]
                                                           : (double)static_cast<const float*>(a.positions)[at];
                    turn_of(pos, a.freqs[p + j], c, s);
                }
            }
            cs[u * VP + j] = c;
            sn[u * VP + j] = s;
        }
    }

    const float inv_dim = 1.0f / (float)a.head_dim;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const RotTensor& t = a.t[which];
        const int first = which ? a.t[0].heads : 0;
        const int b = max(h0, first) - first, e = min(h1, first + t.heads) - first;
        if (b >= e) continue;
        const T* in = static_cast<const T*>(t.in) + row * t.in_row;
        T* out = static_cast<T*>(t.out) + row * t.out_row;
        const T* weight = static_cast<const T*>(t.weight);
        for (int h = b; h < e; h += kRotBatch) {
            Run<T, VP> x[kRotBatch][NU][2];
#pragma unroll
            for (int k = 0; k < kRotBatch; ++k) {
                const T* head = in + (int64_t)min(h + k, e - 1) * t.in_head;
#pragma unroll
                for (int u = 0; u < NU; ++u)
                    if (own[u]) {
                        x[k][u][0] = *reinterpret_cast<const Run<T, VP>*>(head + e0[u]);
                        x[k][u][1] = *reinterpret_cast<const Run<T, VP>*>(head + e1[u]);
                    }
            }
#pragma unroll
            for (int k = 0; k < kRotBatch; ++k) {
                if (h + k >= e) break;
                float v[NU][2 * VP];
                float sum = 0.0f;
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int j = 0; j < VP; ++j) {
                        v[u][j] = own[u] ? Conv<T>::up(x[k][u][0].v[j]) : 0.0f;
                        v[u][VP + j] = own[u] ? Conv<T>::up(x[k][u][1].v[j]) : 0.0f;
                        sum += v[u][j] * v[u][j] + v[u][VP + j] * v[u][VP + j];
                    }
                if (weight) {
                    for (int m = lp >> 1; m > 0; m >>= 1) sum += __shfl_xor_sync(group, sum, m);
                    const float r = 1.0f / sqrtf(sum * inv_dim + a.eps);
#pragma unroll
                    for (int u = 0; u < NU; ++u)
                        if (own[u]) {
                            const Run<T, VP> w0 = *reinterpret_cast<const Run<T, VP>*>(weight + e0[u]);
                            const Run<T, VP> w1 = *reinterpret_cast<const Run<T, VP>*>(weight + e1[u]);
#pragma unroll
                            for (int j = 0; j < VP; ++j) {
                                v[u][j] *= r * Conv<T>::up(w0.v[j]);
                                v[u][VP + j] *= r * Conv<T>::up(w1.v[j]);
                            }
                        }
                }
                T* head = out + (int64_t)(h + k) * t.out_head;
#pragma unroll
                for (int u = 0; u < NU; ++u)
                    if (own[u]) {
                        Run<T, VP> y0, y1;
#pragma unroll
                        for (int j = 0; j < VP; ++j) {
                            const float c = cs[u * VP + j], s = sn[u * VP + j];
                            const int m = ILV ? 2 * j : j, n = ILV ? 2 * j + 1 : VP + j;  // the pair inside v
                            const float r0 = v[u][m] * c - v[u][n] * s, r1 = v[u][n] * c + v[u][m] * s;
                            if (m < VP) y0.v[m] = Conv<T>::down(r0); else y1.v[m - VP] = Conv<T>::down(r0);
                            if (n < VP) y0.v[n] = Conv<T>::down(r1); else y1.v[n - VP] = Conv<T>::down(r1);
                        }
                        *reinterpret_cast<Run<T, VP>*>(head + e0[u]) = y0;
                        *reinterpret_cast<Run<T, VP>*>(head + e1[u]) = y1;
                    }
            }
        }
    }
}

template <typename T, int VP, int NU>
static cudaError_t launch_rotate(const RotArgs& a, bool interleaved, int sm_count, cudaStream_t stream) {
    const int units = ceil_div(a.head_dim / 2, VP);
    int lp_log = 0;
    while ((1 << lp_log) * NU < units) ++lp_log;
    const int total = a.t[0].heads + a.t[1].heads;
    // Few tokens: their heads are spread over more groups of lanes until there are about 1024 threads per SM, a
    // multiple of kRotBatch heads each while that is enough.
    const int64_t groups = a.rows << lp_log, want = (int64_t)sm_count * 1024;
    int per = total;
    if (groups < want) {
        const int64_t split = (want + groups - 1) / groups;
        per = split >= total ? 1 : ceil_div(total, (int)split);
        if (per > kRotBatch) per = ceil_div(per, kRotBatch) * kRotBatch;
    }
    const int64_t blocks = (groups + kRotThreads - 1) / kRotThreads;
    const dim3 grid((unsigned)blocks, (unsigned)ceil_div(total, per));
    auto kernel = interleaved ? rotate_kernel<T, VP, NU, true> : rotate_kernel<T, VP, NU, false>;
    return launch_kernel(kernel, grid, dim3(kRotThreads), 0, stream, a, lp_log, per);
}

// Runs of VP elements may be taken together when every address they start at is a multiple of their size.
static bool runs_of(const octo_rotate_t& c, const RotArgs& a, int vp, int esize) {
    const int rest = a.head_dim / 2 - a.pairs;
    if (a.pairs % vp || rest % vp) return false;
    const uintptr_t bytes = (uintptr_t)(vp * esize < 16 ? vp * esize : 16);
    for (const RotTensor& t : a.t) {
        if (t.heads == 0) continue;
        if (!aligned_to(t.in, bytes) || !aligned_to(t.out, bytes) || !aligned_to(t.weight, bytes)) return false;
        for (int64_t s : {t.in_row, t.in_head, t.out_row, t.out_head})
            if ((uintptr_t)(s * esize) % bytes) return false;
    }
    // a run may start at any multiple of vp inside a head, so its size has to divide 16 bytes' worth of them
    return (vp * esize) % (int)bytes == 0 && (c.interleaved == 0 || a.head_dim % (2 * vp) == 0);
}

template <typename T>
static cudaError_t rotate_typed(const octo_rotate_t& c, const RotArgs& a, int sm_count, cudaStream_t stream) {
    if (runs_of(c, a, 8, (int)sizeof(T))) return launch_rotate<T, 8, 1>(a, c.interleaved != 0, sm_count, stream);
    if (runs_of(c, a, 4, (int)sizeof(T))) return launch_rotate<T, 4, 1>(a, c.interleaved != 0, sm_count, stream);
    return launch_rotate<T, 1, 4>(a, c.interleaved != 0, sm_count, stream);
}

}  // namespace octo

using namespace octo;

extern "C" int octo_patch_positions(int32_t device, const octo_item_t* d_items, int32_t max_items, const int32_t* d_n_items,
                                    int32_t slot_w, int32_t slot_h, int32_t patch, int32_t keep_aspect,
                                    const float* d_times, int32_t n_frames, float* d_positions, uint8_t* d_visible,
                                    void* cuda_stream) {
    if (device < 0 || max_items < 0 || n_frames < 0) return OCTO_E_INVALID_ARG;
    if (slot_w < 1 || slot_w > kPosMaxSide || slot_h < 1 || slot_h > kPosMaxSide || patch < 1) return OCTO_E_INVALID_ARG;
    if (slot_w % patch || slot_h % patch || (keep_aspect != 0 && keep_aspect != 1)) return OCTO_E_INVALID_ARG;
    if (max_items == 0) return OCTO_OK;
    if (!d_items || !d_positions) return OCTO_E_INVALID_ARG;
    if (!aligned_to(d_items, 4) || !aligned_to(d_n_items, 4) || !aligned_to(d_times, 4) || !aligned_to(d_positions, 4))
        return OCTO_E_ALIGNMENT;
    DeviceScope scope(device);
    if (scope.error != cudaSuccess) return report_cuda_error(scope.error, "octo_patch_positions");
    const cudaError_t e = launch_positions(d_items, max_items, d_n_items, slot_w, slot_h, patch, keep_aspect, d_times,
                                           n_frames, d_positions, d_visible, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? OCTO_OK : report_cuda_error(e, "octo_patch_positions");
}

extern "C" int octo_norm_rotate(const octo_rotate_t* c, void* cuda_stream) {
    if (!c || c->device < 0) return OCTO_E_INVALID_ARG;
    if (c->dtype != OCTO_F16 && c->dtype != OCTO_BF16 && c->dtype != OCTO_F32) return OCTO_E_INVALID_ARG;
    if (c->heads < 0 || c->kv_heads < 0 || c->heads > 16384 || c->kv_heads > 16384 || c->heads + c->kv_heads < 1)
        return OCTO_E_INVALID_ARG;
    if (c->head_dim < 2 || c->head_dim > 256 || (c->head_dim & 1)) return OCTO_E_INVALID_ARG;
    if (c->pairs < 0 || 2 * c->pairs > c->head_dim) return OCTO_E_INVALID_ARG;
    if (c->interleaved != 0 && c->interleaved != 1) return OCTO_E_INVALID_ARG;
    if (c->num_axes < 1 || c->num_axes > 8 || (c->positions_are_int != 0 && c->positions_are_int != 1))
        return OCTO_E_INVALID_ARG;
    if (c->rows < 0 || c->rows > (int64_t)1 << 31 || !(c->eps >= 0.0f) || c->eps > 1e30f) return OCTO_E_INVALID_ARG;
    if (c->d_n_items && c->item_rows < 1) return OCTO_E_INVALID_ARG;
    if (c->rows == 0) return OCTO_OK;
    if (c->pairs > 0 && (!c->d_positions || !c->d_freqs || !c->d_axes)) return OCTO_E_INVALID_ARG;
    if (c->heads > 0 && (!c->q.d_data || !c->q_out.d_data)) return OCTO_E_INVALID_ARG;
    if (c->kv_heads > 0 && (!c->k.d_data || !c->k_out.d_data)) return OCTO_E_INVALID_ARG;
    const uintptr_t esize = c->dtype == OCTO_F32 ? 4 : 2;
    for (const void* p : {(const void*)c->q.d_data, (const void*)c->k.d_data, (const void*)c->q_out.d_data,
                          (const void*)c->k_out.d_data, c->d_q_weight, c->d_k_weight})
        if (!aligned_to(p, esize)) return OCTO_E_ALIGNMENT;
    for (const void* p : {c->d_positions, (const void*)c->d_freqs, (const void*)c->d_axes, (const void*)c->d_n_items})
        if (!aligned_to(p, 4)) return OCTO_E_ALIGNMENT;

    RotArgs a;
    a.t[0] = {c->q.d_data, c->q_out.d_data, c->d_q_weight, c->q.row_stride, c->q.head_stride, c->q_out.row_stride,
              c->q_out.head_stride, c->heads};
    a.t[1] = {c->k.d_data, c->k_out.d_data, c->d_k_weight, c->k.row_stride, c->k.head_stride, c->k_out.row_stride,
              c->k_out.head_stride, c->kv_heads};
    a.positions = c->d_positions;
    a.freqs = c->d_freqs;
    a.axes = c->d_axes;
    a.n_items = c->d_n_items;
    a.rows = c->rows;
    a.item_rows = c->item_rows;
    a.head_dim = c->head_dim;
    a.pairs = c->pairs;
    a.num_axes = c->num_axes;
    a.positions_are_int = c->positions_are_int;
    a.eps = c->eps;
    DeviceScope scope(c->device);
    if (scope.error != cudaSuccess) return report_cuda_error(scope.error, "octo_norm_rotate");
    int sms = 0;
    cudaError_t e = sm_count_of(c->device, &sms);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (e == cudaSuccess) {
        if (c->dtype == OCTO_F16) e = rotate_typed<__half>(*c, a, sms, stream);
        else if (c->dtype == OCTO_BF16) e = rotate_typed<__nv_bfloat16>(*c, a, sms, stream);
        else e = rotate_typed<float>(*c, a, sms, stream);
    }
    return e == cudaSuccess ? OCTO_OK : report_cuda_error(e, "octo_norm_rotate");
}
