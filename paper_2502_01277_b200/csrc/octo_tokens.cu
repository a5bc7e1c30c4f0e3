// Tokens of a transformer behind the stage: positions of the patches of packed crops, and the norm of query
// and key heads together with their rotation by those positions (include/octo.h).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "octo_tokens.h"

namespace octo {

// ---------------------------------------------------------------------------------------
// Positions.  The threads of an item first make one coordinate per patch column and patch row (a division in
// binary64 each, of which a patch of its own would need two), then write the item's block of (time, y, x) triples
// with neighbouring threads on neighbouring words.  A batch of many items gives a warp to each, which lets all
// of a server's batch be under way at once; a few items get a CTA each (7356 items of 196 patches: 13.1 us with a CTA
// per item, 8.5 with a warp; 22 items 2.4).  What grows with the items is instructions: each word picks its source.
// ---------------------------------------------------------------------------------------
constexpr int kPosThreads = 128;
constexpr int kPosMaxSide = 2048;  // patches along a side of a slot

// Image size and place inside the slot, in integers (the fit of an aspect-preserving crop).
__device__ __forceinline__ void fit_in_slot(int cw, int ch, int ow, int oh, int keep_aspect, int& nw, int& nh, int& pl,
                                            int& pt) {
    nw = ow;
    nh = oh;
    if (keep_aspect && (cw | ch) < 1 << 18) {  // everything fits 32 bits: a fifth of a 64-bit division's instructions
        if (ow * ch <= oh * cw) nh = max(1, (int)((2u * ow * ch + cw) / (2u * cw)));
        else nw = max(1, (int)((2u * oh * cw + ch) / (2u * ch)));
    } else if (keep_aspect) {
        if ((long long)ow * ch <= (long long)oh * cw) nh = max(1, (int)((2LL * ow * ch + cw) / (2LL * cw)));
        else nw = max(1, (int)((2LL * oh * cw + ch) / (2LL * ch)));
    }
    pl = (ow - nw) / 2;
    pt = (oh - nh) / 2;
}

// PER: threads of an item, 32 or kPosThreads.
template <int PER>
__global__ void __launch_bounds__(kPosThreads)
positions_kernel(const octo_item_t* __restrict__ items, int max_items, const int* __restrict__ n_items, int slot_w,
                 int slot_h, int patch, int gw, int gh, FastDiv by_gw, int wide, int keep_aspect, const float* __restrict__ times,
                 int n_frames, float* __restrict__ positions, uint8_t* __restrict__ visible) {
    extern __shared__ float s_all[];  // per item: [gw] x, [gh] y, then one byte per column and row: shows the image
    const int local = PER == 32 ? threadIdx.x >> 5 : 0, t = threadIdx.x & (PER - 1), words = gw + gh + (gw + gh + 3) / 4;
    float* const s_x = s_all + local * words;
    float* const s_y = s_x + gw;
    uint8_t* const s_vx = reinterpret_cast<uint8_t*>(s_y + gh);
    uint8_t* const s_vy = s_vx + gw;
    const int i = blockIdx.x * (kPosThreads / PER) + local;
    pdl_wait();
    if (i >= max_items || (n_items && i >= *n_items)) return;
    const octo_item_t it = items[i];
    const int cw = it.rx1 - it.rx0, ch = it.ry1 - it.ry0;
    const bool good = cw > 0 && ch > 0 && it.rx1 > it.rx0 && it.ry1 > it.ry0 && it.frame >= 0 && it.frame < n_frames;
    const float time = good && times ? times[it.frame] : 0.0f;
    int nw = 1, nh = 1, pl = 0, pt = 0;
    if (good) fit_in_slot(cw, ch, slot_w, slot_h, keep_aspect, nw, nh, pl, pt);
    for (int k = t; k < gw + gh; k += PER) {
        const bool col = k < gw;
        const int g = col ? k : k - gw, pad = col ? pl : pt, n = col ? nw : nh, size = col ? cw : ch;
        const int origin = col ? it.rx0 : it.ry0;
        // the centre of the patch, in halves of a slot pixel from the image's edge; one rounding at the end
        const double off = (double)((2 * g + 1) * patch - 2 * pad) * (double)size / (double)(2 * n);
        s_x[k] = good ? (float)((double)origin + off) : 0.0f;
        s_vx[k] = good && g * patch < pad + n && (g + 1) * patch > pad ? 1 : 0;
    }
    if (PER == 32) __syncwarp();
    else __syncthreads();
    const int patches = gw * gh;
    float* const out = positions + (size_t)i * patches * 3;
    if (wide) {  // four words, or the bytes of four patches, at a time
        for (int f = 4 * t; f < patches * 3; f += 4 * PER) {
            int p = f / 3, c = f - 3 * p, gy = by_gw.div(p), gx = p - gy * gw;
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k] = c == 0 ? time : (c == 1 ? s_y[gy] : s_x[gx]);
                if (++c == 3) {
                    c = 0;
                    if (++gx == gw) {
                        gx = 0;
                        ++gy;  // (one past the last row after the last word: not read)
                    }
                }
            }
            *reinterpret_cast<float4*>(out + f) = make_float4(v[0], v[1], v[2], v[3]);
        }
        for (int p = 4 * t; visible && p < patches; p += 4 * PER) {
            int gy = by_gw.div(p), gx = p - gy * gw;
            uint32_t v = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v |= (uint32_t)(s_vy[gy] & s_vx[gx]) << (8 * k);
                if (++gx == gw) {
                    gx = 0;
                    ++gy;
                }
            }
            *reinterpret_cast<uint32_t*>(visible + (size_t)i * patches + p) = v;
        }
        return;
    }
    // word f of the block is component f % 3 of patch f / 3
    for (int f = t; f < patches * 3; f += PER) {
        const int p = f / 3, c = f - 3 * p, gy = by_gw.div(p), gx = p - gy * gw;
        out[f] = c == 0 ? time : (c == 1 ? s_y[gy] : s_x[gx]);
    }
    if (visible) {
        uint8_t* const vis = visible + (size_t)i * patches;
        for (int p = t; p < patches; p += PER) {
            const int gy = by_gw.div(p), gx = p - gy * gw;
            vis[p] = s_vy[gy] & s_vx[gx];
        }
    }
}

cudaError_t launch_positions(const octo_item_t* d_items, int max_items, const int* d_n_items, int slot_w, int slot_h,
                             int patch, int keep_aspect, const float* d_times, int n_frames, float* d_positions,
                             uint8_t* d_visible, int sm_count, cudaStream_t stream) {
    if (max_items < 1) return cudaSuccess;
    const int gw = slot_w / patch, gh = slot_h / patch;
    const size_t words = (size_t)(gw + gh) + (size_t)(gw + gh + 3) / 4;
    FastDiv by_gw;
    by_gw.set((unsigned)gw);
    // a warp per item from two CTAs per SM on, and where four items' tables still fit beside one another
    const bool warps = max_items >= 2 * sm_count && words <= 2048;
    const int wide = gw * gh % 4 == 0 && aligned_to(d_positions, 16) && aligned_to(d_visible, 4);
    const int per_cta = warps ? kPosThreads / 32 : 1;
    return launch_kernel(warps ? positions_kernel<32> : positions_kernel<kPosThreads>, dim3((unsigned)ceil_div(max_items, per_cta)),
                         dim3(kPosThreads), words * per_cta * sizeof(float), stream, d_items, max_items, d_n_items, slot_w, slot_h,
                         patch, gw, gh, by_gw, wide, keep_aspect, d_times, n_frames, d_positions, d_visible);
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
// registers for all heads, multiplied with the norm's weights: a pair (x0, x1) of a head with 1 / rms r becomes
// r (x0 w0 c - x1 w1 s), r (x1 w1 c + x0 w0 s), six operations.  A lane owns VP pairs of every head, both elements of
// each: for halves two runs of VP elements that lie `pairs` apart, for neighbours one run of 2 VP, so that no
// element changes lanes.  Elements behind the rotated ones are given to lanes as pairs too, but pairs that do not turn are
// only scaled: as turns by zero an infinity in one element would make its partner NaN (infinity times a sine of zero).
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

// N elements of T that start on a multiple of their own size (at most 16 bytes at a time).
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Run {
    T v[N];
};

__device__ __forceinline__ float one_up(__half v) { return __half2float(v); }
__device__ __forceinline__ float one_up(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float one_up(float v) { return v; }
__device__ __forceinline__ void one_down(float f, __half& v) { v = __float2half_rn(f); }
__device__ __forceinline__ void one_down(float f, __nv_bfloat16& v) { v = __float2bfloat16_rn(f); }
__device__ __forceinline__ void one_down(float f, float& v) { v = f; }
__device__ __forceinline__ void two_up(uint32_t w, float& a, float& b, __half) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
}
__device__ __forceinline__ void two_up(uint32_t w, float& a, float& b, __nv_bfloat16) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t two_down(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t two_down(float a, float b, __nv_bfloat16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// A run to binary32 and back; 16-bit types two at a time.
template <typename T, int N>
__device__ __forceinline__ void run_up(const Run<T, N>& r, float* f) {
    if constexpr (sizeof(T) == 2 && N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) two_up(reinterpret_cast<const uint32_t*>(&r)[i / 2], f[i], f[i + 1], T());
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = one_up(r.v[i]);
    }
}
template <typename T, int N>
__device__ __forceinline__ Run<T, N> run_down(const float* f) {
    Run<T, N> r;
    if constexpr (sizeof(T) == 2 && N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) reinterpret_cast<uint32_t*>(&r)[i / 2] = two_down(f[i], f[i + 1], T());
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) one_down(f[i], r.v[i]);
    }
    return r;
}

// Sine and cosine of position * freq, from the whole turns' remainder.  In binary64 (the product of two binary32
// numbers is exact, of an int32 and a binary32 number off by 2^-53) for positions of any size ...
__device__ __noinline__ void turn_far(double position, float freq, float& c, float& s) {
    const double turns = position * (double)freq * 0.15915494309189533577;
    const double half_turns = 2.0 * (turns - rint(turns));  // in [-1, 1]
    const float h = (float)half_turns;
    const float rest = (float)(half_turns - (double)h) * 3.14159265f;  // what the rounding of h left, as an angle
    float s0, c0;
    sincospif(h, &s0, &c0);
    s = fmaf(c0, rest, s0);
    c = fmaf(-s0, rest, c0);
}
// ... and in pairs of binary32 numbers below 2^22 turns: freq / 2 pi and the product with the position are each held as
// a sum of two (an error of 2^-46 of the turns, 2^-24 of a turn at most), the first of which loses its whole turns
// exactly.  Conversions and products in binary64 took most of a token's time where it has few heads.
// COARSE, for results of 16 bits: the rest of the turns is rounded to binary32 (2^-25 turns, 2^-24 near 2^22 turns), and the
// hardware's sine and cosine, off by up to 2^-21.2 in [-pi, pi], are taken of it: 1.4e-6 (2^-19.4) with everything, where
// half a step of fp16 is 2^-12 at 1.  Near the zeros up to 4.1e-7 was seen in 25 million angles.
template <bool COARSE>
__device__ __forceinline__ void turn_of(float position, float freq, float& c, float& s) {
    const float f1 = freq * 0.15915494f, f2 = fmaf(freq, 6.4206383e-9f, fmaf(freq, 0.15915494f, -f1));  // 1 / 2 pi in two parts
    const float p1 = position * f1;
    if (!(fabsf(p1) < 4194304.0f)) return turn_far((double)position, freq, c, s);
    const float p2 = fmaf(position, f2, fmaf(position, f1, -p1));
    const float whole = p1 - rintf(p1);
    float t = whole + p2;
    if (COARSE) {
        __sincosf((t - rintf(t)) * 6.28318531f, &s, &c);
        return;
    }
    const float left = p2 - (t - whole);
    t -= rintf(t);
    const float h = 2.0f * t, rest = left * 6.28318531f;  // what the rounding of t left, as an angle
    float s0, c0;
    sincospif(h, &s0, &c0);
    s = fmaf(c0, rest, s0);
    c = fmaf(-s0, rest, c0);
}

// Sum over the lanes of a group of `size` neighbouring lanes that starts at lane `first`, in every one of them.
__device__ __forceinline__ float group_sum(float v, unsigned mask, int first, int size, int in) {
    if ((size & (size - 1)) == 0) {
        for (int m = size >> 1; m > 0; m >>= 1) v += __shfl_xor_sync(mask, v, m);
        return v;
    }
    for (int m = 16; m > 0; m >>= 1) {
        const float w = __shfl_down_sync(mask, v, m);
        if (m < size && in + m < size && in < m) v += w;
    }
    return __shfl_sync(mask, v, first);
}

// CTAs an SM should hold: many where few heads are in flight, since the wait for a token's angles and heads is then
// covered by other tokens.
template <typename T, int VP, int NU, int BATCH>
constexpr int rotate_ctas() {
    return BATCH * VP >= 4 * 8 || sizeof(T) * VP * NU * BATCH >= 64 ? 2 : (sizeof(T) * VP * NU > 16 ? 3 : 4);
}

// ILV: pairs are neighbours.  `lanes` lanes per token, NU units of VP pairs per lane, BATCH heads of a group in flight together.
template <typename T, int VP, int NU, bool ILV, int BATCH>
__global__ void __launch_bounds__(kRotThreads, rotate_ctas<T, VP, NU, BATCH>())
rotate_kernel(const __grid_constant__ RotArgs a, int lanes, int heads_per_group) {
    constexpr int N = VP * NU;
    pdl_wait();
    const int lane = threadIdx.x & 31, tokens = 32 / lanes, mine = lane / lanes, in = lane - mine * lanes;
    const int64_t row = ((int64_t)blockIdx.x * (kRotThreads / 32) + (threadIdx.x >> 5)) * tokens + mine;
    int64_t rows = a.rows;
    if (a.n_items) {
        const int64_t n = *a.n_items;
        rows = n <= 0 ? 0 : (n < rows / a.item_rows + 1 ? min(rows, n * a.item_rows) : rows);
    }
    const bool live = mine < tokens && row < rows;
    const unsigned mask = __ballot_sync(0xffffffffu, live);
    if (!live) return;  // a group leaves as a whole; shuffles name the lanes that stay
    const int first = mine * lanes;
    const int total = a.t[0].heads + a.t[1].heads;
    const int h0 = blockIdx.y * heads_per_group, h1 = min(total, h0 + heads_per_group);

    // which elements this lane owns, and how they turn
    const int half = a.head_dim / 2, rest = half - a.pairs;  // pairs that turn and do not: `half` in all
    int e0[NU], e1[NU];  // first element of the two runs of a unit (ILV: e1 = e0 + VP)
    bool own[NU];
    unsigned still = 0;  // bit k: pair k of the lane does not turn
    float cs[N], sn[N];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        const int p = (in + u * lanes) * VP;  // first pair of the unit
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
            if (own[u]) still |= 1u << (u * VP + j);
            if (turning) {
                const int axis = a.axes[p + j];
                if (axis >= 0 && axis < a.num_axes) {
                    still &= ~(1u << (u * VP + j));
                    const int64_t at = row * a.num_axes + axis;
                    if (a.positions_are_int) {
                        const int pos = static_cast<const int*>(a.positions)[at];
                        if (pos >= -(1 << 24) && pos <= 1 << 24) turn_of<sizeof(T) == 2>((float)pos, a.freqs[p + j], c, s);
                        else turn_far((double)pos, a.freqs[p + j], c, s);
                    } else {
                        turn_of<sizeof(T) == 2>(static_cast<const float*>(a.positions)[at], a.freqs[p + j], c, s);
                    }
                }
            }
            cs[u * VP + j] = c;
            sn[u * VP + j] = s;
        }
    }

    const bool some_still = __any_sync(mask, still != 0);
    const float inv_dim = 1.0f / (float)a.head_dim;
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const RotTensor& t = a.t[which];
        const int from = which ? a.t[0].heads : 0;
        const int b = max(h0, from) - from, e = min(h1, from + t.heads) - from;
        if (b >= e) continue;
        const T* const in_row = static_cast<const T*>(t.in) + row * t.in_row;
        T* const out_row = static_cast<T*>(t.out) + row * t.out_row;
        const T* const weight = static_cast<const T*>(t.weight);
        // (w0 c, w1 s, w1 c, w0 s) of every pair
        float m00[N], m01[N], m11[N], m10[N];
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float w[2 * VP];
#pragma unroll
            for (int j = 0; j < 2 * VP; ++j) w[j] = 1.0f;
            if (weight && own[u]) {
                run_up<T, VP>(*reinterpret_cast<const Run<T, VP>*>(weight + e0[u]), w);
                run_up<T, VP>(*reinterpret_cast<const Run<T, VP>*>(weight + e1[u]), w + VP);
            }
#pragma unroll
            for (int j = 0; j < VP; ++j) {
                const int m = ILV ? 2 * j : j, n = ILV ? 2 * j + 1 : VP + j;  // the pair inside the unit's 2 VP elements
                const int k = u * VP + j;
                m00[k] = w[m] * cs[k];
                m01[k] = w[n] * sn[k];
                m11[k] = w[n] * cs[k];
                m10[k] = w[m] * sn[k];
            }
        }
        for (int h = b; h < e; h += BATCH) {
            Run<T, VP> x[BATCH][NU][2];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const T* const head = in_row + (int64_t)min(h + k, e - 1) * t.in_head;
#pragma unroll
                for (int u = 0; u < NU; ++u)
                    if (own[u]) {
                        x[k][u][0] = *reinterpret_cast<const Run<T, VP>*>(head + e0[u]);
                        x[k][u][1] = *reinterpret_cast<const Run<T, VP>*>(head + e1[u]);
                    }
            }
            float r[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                r[k] = 1.0f;
                if (weight) {
                    float sum = 0.0f;
#pragma unroll
                    for (int u = 0; u < NU; ++u) {
                        float f[2 * VP];
                        run_up<T, VP>(x[k][u][0], f);
                        run_up<T, VP>(x[k][u][1], f + VP);
                        float part = 0.0f;
#pragma unroll
                        for (int j = 0; j < 2 * VP; ++j) part = fmaf(f[j], f[j], part);
                        if (own[u]) sum += part;
                    }
                    r[k] = rsqrtf(fmaf(group_sum(sum, mask, first, lanes, in), inv_dim, a.eps));
                }
            }
            auto write = [&](auto some) {
                constexpr bool SOME_STILL = decltype(some)::value;
                unsigned kept = still;
                if (SOME_STILL) asm volatile("" : "+r"(kept));  // (else a predicate per pair is kept over the whole loop, and spilled)
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    if (h + k >= e) break;
                    T* const head = out_row + (int64_t)(h + k) * t.out_head;
#pragma unroll
                    for (int u = 0; u < NU; ++u)
                        if (own[u]) {
                            float f[2 * VP], y[2 * VP];
                            run_up<T, VP>(x[k][u][0], f);
                            run_up<T, VP>(x[k][u][1], f + VP);
#pragma unroll
                            for (int j = 0; j < VP; ++j) {
                                const int m = ILV ? 2 * j : j, n = ILV ? 2 * j + 1 : VP + j, i = u * VP + j;
                                const float x0 = r[k] * f[m], x1 = r[k] * f[n];
                                const bool turns = !SOME_STILL || !((kept >> i) & 1u);
                                y[m] = fmaf(x0, m00[i], turns ? -(x1 * m01[i]) : -0.0f);
                                y[n] = fmaf(x1, m11[i], turns ? x0 * m10[i] : -0.0f);
                            }
                            *reinterpret_cast<Run<T, VP>*>(head + e0[u]) = run_down<T, VP>(y);
                            *reinterpret_cast<Run<T, VP>*>(head + e1[u]) = run_down<T, VP>(y + VP);
                        }
                }
            };
            // (decided once for the heads in flight; us without the choice, with it here, and with it per head: 274 000 tokens of 16 +
            // 16 heads of 64, all pairs turning, 393 / 406 / 416; 196 000 tokens of 5 + 5 heads 122 / 129 / 141)
            if (some_still) write(std::true_type());
            else write(std::false_type());
        }
    }
}

// How a call is carried out (octo_rotate_plan).
struct RotateForm {
    int run, per, in_flight;
};

// Launches, or with `form` only says how it would.
template <typename T, int VP, int NU>
static cudaError_t launch_rotate(const RotArgs& a, bool interleaved, int sm_count, cudaStream_t stream, RotateForm* form) {
    const int lanes = ceil_div(ceil_div(a.head_dim / 2, VP), NU), tokens = 32 / lanes;
    const int total = a.t[0].heads + a.t[1].heads;
    const int64_t warps = (a.rows + tokens - 1) / tokens;
    // Few tokens: their heads are spread over more warps until there are about 16 per SM, a multiple of 4 heads each
    // while that is enough.
    const int64_t want = (int64_t)sm_count * 16;
    int per = total;
    if (warps < want) {
        const int64_t split = (want + warps - 1) / warps;
        per = split >= total ? 1 : ceil_div(total, (int)split);
        if (per > 4) per = ceil_div(per, 4) * 4;
    }
    const int64_t blocks = (warps + kRotThreads / 32 - 1) / (kRotThreads / 32);
    const dim3 grid((unsigned)blocks, (unsigned)ceil_div(total, per));
    // Heads in flight.  One head: one.  Few heads: two, and more CTAs (us two / four: 196 000 tokens, 5 + 5 heads of 64 129 / 135).
    // Else what 16 registers of a lane hold (four of 16 bits, two of binary32; two / four: 274 000 tokens, 16 + 16 heads of 64
    // 458 / 404).  Runs of less than eight elements: two (four took 303 instead of 324 for 137 000 tokens of 16 + 16 heads of 72;
    // fewer heads were not compared).
    const int most = std::min(per, std::max(a.t[0].heads, a.t[1].heads));
    auto start = [&](auto batch) {
        constexpr int BATCH = decltype(batch)::value;
        if (form) {
            *form = {VP, per, BATCH};
            return cudaSuccess;
        }
        auto kernel = interleaved ? rotate_kernel<T, VP, NU, true, BATCH> : rotate_kernel<T, VP, NU, false, BATCH>;
        return launch_kernel(kernel, grid, dim3(kRotThreads), 0, stream, a, lanes, per);
    };
    if (most == 1) return start(std::integral_constant<int, 1>());
    if constexpr (VP == 8 && sizeof(T) == 2) {
        if (most > 5) return start(std::integral_constant<int, 4>());
    }
    return start(std::integral_constant<int, 2>());
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
static cudaError_t rotate_typed(const octo_rotate_t& c, const RotArgs& a, int sm_count, cudaStream_t stream, RotateForm* form) {
    if (runs_of(c, a, 8, (int)sizeof(T))) return launch_rotate<T, 8, 1>(a, c.interleaved != 0, sm_count, stream, form);
    if (runs_of(c, a, 4, (int)sizeof(T))) return launch_rotate<T, 4, 1>(a, c.interleaved != 0, sm_count, stream, form);
    // Shorter runs: two units per lane where a warp then takes two tokens or more rather than one (one fp32 head of 72 with
    // 18 turning pairs in q and k, 835 000 tokens: 600 us with one unit, 269 with two).
    const int half = c.head_dim / 2;
    const bool ilv = c.interleaved != 0;
    if (runs_of(c, a, 2, (int)sizeof(T)))
        return half <= 32 ? launch_rotate<T, 2, 1>(a, ilv, sm_count, stream, form)
                          : launch_rotate<T, 2, 2>(a, ilv, sm_count, stream, form);
    if (half <= 16) return launch_rotate<T, 1, 1>(a, ilv, sm_count, stream, form);
    if (half <= 32) return launch_rotate<T, 1, 2>(a, ilv, sm_count, stream, form);
    return launch_rotate<T, 1, 4>(a, ilv, sm_count, stream, form);
}

}  // namespace octo

using namespace octo;

extern "C" int octo_patch_positions(int32_t device, const octo_item_t* d_items, int32_t max_items, const int32_t* d_n_items,
                                    int32_t slot_w, int32_t slot_h, int32_t patch, int32_t keep_aspect,
                                    const float* d_times, int32_t n_frames, float* d_positions, uint8_t* d_visible,
                                    void* cuda_stream) {
    if (device < 0 || max_items < 0 || max_items > 1 << 30 || n_frames < 0) return OCTO_E_INVALID_ARG;
    if (slot_w < 1 || slot_w > kPosMaxSide || slot_h < 1 || slot_h > kPosMaxSide || patch < 1) return OCTO_E_INVALID_ARG;
    if (slot_w % patch || slot_h % patch || (keep_aspect != 0 && keep_aspect != 1)) return OCTO_E_INVALID_ARG;
    if (max_items == 0) return OCTO_OK;
    if (!d_items || !d_positions) return OCTO_E_INVALID_ARG;
    if (!aligned_to(d_items, 4) || !aligned_to(d_n_items, 4) || !aligned_to(d_times, 4) || !aligned_to(d_positions, 4))
        return OCTO_E_ALIGNMENT;
    DeviceScope scope(device);
    if (scope.error != cudaSuccess) return report_cuda_error(scope.error, "octo_patch_positions");
    int sms = 0;
    cudaError_t e = sm_count_of(device, &sms);
    if (e == cudaSuccess)
        e = launch_positions(d_items, max_items, d_n_items, slot_w, slot_h, patch, keep_aspect, d_times, n_frames, d_positions,
                             d_visible, sms, static_cast<cudaStream_t>(cuda_stream));
    return e == cudaSuccess ? OCTO_OK : report_cuda_error(e, "octo_patch_positions");
}

static int rotate_call(const octo_rotate_t* c, void* cuda_stream, RotateForm* form) {
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
    if (rows_coincide(c->q_out, c->rows, c->heads, c->head_dim) || rows_coincide(c->k_out, c->rows, c->kv_heads, c->head_dim)) return OCTO_E_INVALID_ARG;
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
        if (c->dtype == OCTO_F16) e = rotate_typed<__half>(*c, a, sms, stream, form);
        else if (c->dtype == OCTO_BF16) e = rotate_typed<__nv_bfloat16>(*c, a, sms, stream, form);
        else e = rotate_typed<float>(*c, a, sms, stream, form);
    }
    return e == cudaSuccess ? OCTO_OK : report_cuda_error(e, "octo_norm_rotate");
}

extern "C" int octo_norm_rotate(const octo_rotate_t* c, void* cuda_stream) { return rotate_call(c, cuda_stream, nullptr); }

extern "C" int octo_rotate_plan(const octo_rotate_t* c, int32_t* run, int32_t* heads_per_warp, int32_t* heads_in_flight) {
    if (!run || !heads_per_warp || !heads_in_flight) return OCTO_E_INVALID_ARG;
    RotateForm form = {0, 0, 0};
    const int rc = rotate_call(c, nullptr, &form);
    *run = form.run;
    *heads_per_warp = form.per;
    *heads_in_flight = form.in_flight;
    return rc;
}
