// Attention of one set of tokens to another set's states (include/octo.h): the plan of a call, the kernel for
// few query rows, and the kernel that joins work split over the keys.
#include <math.h>

#include <type_traits>

#include "octo_attend.cuh"
#include "octo_attend_tile.h"

namespace octo {

// ---------------------------------------------------------------------------------------
// Few query rows (one new token per item): bound by reading every key and value once.  A CTA takes the rows -- pairs
// (query row, head) that share a key head, at most 16 -- of one segment and one split; each of its warps walks
// over the keys in groups of 16, four warps side by side, with a softmax of its own that the warps join at the end.
// Keys are the long side of the matrix instruction (16 x 8 x 16) and rows the short one, S^T = K Q^T and O^T = V^T P^T, so
// that eight rows fill it.  Keys and values go from global memory straight into its operand registers: which element
// of a head an operand's slot holds is free as long as both operands agree, so the slots are dealt out such
// that a lane's part of a key is 16 bytes in a row, and a lane's part of the values the same 16 bytes of four
// keys, paired up by byte permutes.  No shared memory and no barrier before the end; the loads of the next
// group are in flight while the current one is worked on.  Under a mask the visible keys are listed first, a
// window at a time, and only those are fetched.
// ---------------------------------------------------------------------------------------
constexpr int kStepThreads = 128;
constexpr int kStepWarps = kStepThreads / 32;
constexpr int kStepRows = 16;
constexpr int kStepKeys = 16 * kStepWarps;  // keys a CTA takes per turn
constexpr int kStepFill = 9;
constexpr int kStepWindow = 2048;           // keys that are looked through for visible ones at a time
constexpr float kStepSlack = 8.0f;          // a row's reference follows its maximum when that has grown by 2^8

template <typename T>
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1);
template <>
__device__ __forceinline__ void mma_16816<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                                  uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma_16816<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                                         uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint4 ldg128(const void* p, bool take) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);  // a hidden key counts as zeros, whatever its place holds
    if (take) asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// 8 x 8 elements of 16 bits, two in a row per lane: the transposed matrix.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// DB: 64-element blocks of a head.  NT: groups of eight rows.
template <typename T, int DB, int NT, bool MASKED>
__global__ void __launch_bounds__(kStepThreads, (DB == 1 ? 2 : 1) * (NT == 1 ? 3 : 2) - (DB == 1 ? 1 : 0))
attend_step_kernel(const __grid_constant__ AttendArgs a, int row_tiles) {
    constexpr int KB = 2 * DB;  // 32-element blocks
    constexpr int SP = DB * 64 + 4, ROWS = 8 * NT;
    __shared__ float s_o[kStepWarps][ROWS][SP];
    __shared__ float s_m[kStepWarps][ROWS], s_l[kStepWarps][ROWS];
    __shared__ int s_list[MASKED ? kStepWindow : 1], s_seen[kStepWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    unsigned x = blockIdx.x;
    const int split = (int)(x % (unsigned)a.splits);
    x /= (unsigned)a.splits;
    const int row0 = (int)(x % (unsigned)row_tiles) * ROWS;
    x /= (unsigned)row_tiles;
    const int kvh = (int)(x % (unsigned)a.kv_heads), seg_no = (int)(x / (unsigned)a.kv_heads);
    pdl_wait();
    const Segment seg = segment_of(a, seg_no);
    const int rows = min(seg.qn * a.group - row0, ROWS);
    if (rows <= 0) return;
    const int kb = min(split * a.chunk, seg.kn), ke = min(kb + a.chunk, seg.kn);
    if (split > 0 && kb >= ke) return;
    const int active = a.splits == 1 ? 1 : (seg.kn + a.chunk - 1) / a.chunk;

    // queries: row g of every group, 8 elements at 32 b + 8 t
    uint4 q[NT][KB];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int r = 8 * n + g, row = a.group_div.div(row0 + r), head = kvh * a.group + (row0 + r - row * a.group);
        const T* p = static_cast<const T*>(a.q) + (seg.q0 + row) * a.q_row + head * a.q_head;
#pragma unroll
        for (int b = 0; b < KB; ++b)
            q[n][b] = ldg128(p + 32 * b + 8 * t, r < rows && 32 * b + 8 * t < a.dim &&
                                                     OCTO_TOKEN_IN_RANGE(seg.q0 + row < a.q_total && head < a.heads, a.status));
    }

    const T* const kp = static_cast<const T*>(a.k) + seg.k0 * a.k_row + kvh * a.k_head + 8 * t;
    const T* const vp = static_cast<const T*>(a.v) + seg.k0 * a.v_row + kvh * a.v_head + 8 * g;
    float o[NT][DB * 4][4];
    float ref[NT][2], sum[NT][2];  // rows 2 t and 2 t + 1 of every group: what the exponents are taken against, sum of weights
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        ref[n][0] = ref[n][1] = -INFINITY;
        sum[n][0] = sum[n][1] = 0.0f;
#pragma unroll
        for (int i = 0; i < DB * 4; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.0f;
    }

    for (int wb = kb; wb < ke; wb += kStepWindow) {
        int count = ke - wb;
        if (MASKED) {
            // the visible keys of the window, every warp's one after the other
            const uint8_t* const mask = a.mask + seg.k0 + wb;
            unsigned bits = 0;
            int mine = 0;
            const int limit = min(count, kStepWindow);
#pragma unroll
            for (int j = 0; j < kStepWindow / kStepThreads; ++j) {
                const int at = j * kStepThreads + (int)threadIdx.x;
                if (at < limit && mask[at] != 0) bits |= 1u << j;
            }
#pragma unroll
            for (int j = 0; j < kStepWindow / kStepThreads; ++j) mine += __popc(__ballot_sync(0xffffffffu, (bits >> j) & 1u));
            __syncthreads();  // (the list of the window before has been read)
            if (lane == 0) s_seen[warp] = mine;
            __syncthreads();
            int at = 0;
            count = 0;
#pragma unroll
            for (int w = 0; w < kStepWarps; ++w) {
                if (w < warp) at += s_seen[w];
                count += s_seen[w];
            }
#pragma unroll
            for (int j = 0; j < kStepWindow / kStepThreads; ++j) {
                const bool seen = (bits >> j) & 1u;
                const unsigned ballot = __ballot_sync(0xffffffffu, seen);
                if (seen) s_list[at + __popc(ballot & ((1u << lane) - 1u))] = j * kStepThreads + (int)threadIdx.x;
                at += __popc(ballot);
            }
            __syncthreads();
        }
        auto key_at = [&](int n) -> int64_t { return wb + (MASKED ? s_list[n] : n); };
        auto in_keys = [&](int n) { return n >= 0 && (!MASKED || n < kStepWindow) && key_at(n) < ke && seg.k0 + key_at(n) < a.k_total; };
        uint4 kr[2][KB], vr[4][DB];
        auto load_k = [&](int first) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int n = first + 8 * j + g;
                const bool there = n < count && OCTO_TOKEN_IN_RANGE(in_keys(n), a.status);
                const T* p = kp + (there ? key_at(n) : 0) * a.k_row;
#pragma unroll
                for (int b = 0; b < KB; ++b) kr[j][b] = ldg128(p + 32 * b, there && 32 * b + 8 * t < a.dim);
            }
        };
        auto load_v = [&](int first) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = first + 2 * t + (j & 1) + 8 * (j >> 1);
                const bool there = n < count && OCTO_TOKEN_IN_RANGE(in_keys(n), a.status);
                const T* p = vp + (there ? key_at(n) : 0) * a.v_row;
#pragma unroll
                for (int b = 0; b < DB; ++b) vr[j][b] = ldg128(p + 64 * b, there && 64 * b + 8 * g < a.dim);
            }
        };
        int first = 16 * warp;
        load_k(first);
        load_v(first);
        for (; first < count; first += kStepKeys) {
            float s[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
                for (int b = 0; b < KB; ++b) {
                    mma_16816<T>(s[n], kr[0][b].x, kr[1][b].x, kr[0][b].y, kr[1][b].y, q[n][b].x, q[n][b].y);
                    mma_16816<T>(s[n], kr[0][b].z, kr[1][b].z, kr[0][b].w, kr[1][b].w, q[n][b].z, q[n][b].w);
                }
            }
            load_k(first + kStepKeys);
            // this lane's scores: keys g (0, 1) and g + 8 (2, 3), rows 2 t (0, 2) and 2 t + 1 (1, 3)
            const bool in0 = first + g < count, in1 = first + g + 8 < count;
            bool grown = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[n][i] = (i < 2 ? in0 : in1) ? s[n][i] * a.scale_log2 : -INFINITY;
                    grown = grown || s[n][i] > ref[n][i & 1] + kStepSlack || (ref[n][i & 1] == -INFINITY && s[n][i] > -INFINITY);
                }
            if (__any_sync(0xffffffffu, grown)) {  // (not for NaN, which comes through the weights)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float top = fmaxf(s[n][c], s[n][c + 2]);
#pragma unroll
                        for (int m = 4; m < 32; m <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
                        top = fmaxf(top, ref[n][c]);
                        const float f = top == -INFINITY ? 1.0f : ex2(ref[n][c] - top);  // what was summed shrinks
                        ref[n][c] = top;
                        sum[n][c] *= f;
#pragma unroll
                        for (int i = 0; i < DB * 4; ++i) {
                            o[n][i][c] *= f;
                            o[n][i][c + 2] *= f;
                        }
                    }
            }
            uint32_t p0[NT], p1[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][i] = ex2(s[n][i] - (ref[n][i & 1] == -INFINITY ? 0.0f : ref[n][i & 1]));
                sum[n][0] += s[n][0] + s[n][2];
                sum[n][1] += s[n][1] + s[n][3];
                // the weights in the type of the values: what the matrix instruction takes (the sum keeps them unrounded)
                p0[n] = transpose8x8(pack2<T>(s[n][0], s[n][1]));
                p1[n] = transpose8x8(pack2<T>(s[n][2], s[n][3]));
            }
#pragma unroll
            for (int b = 0; b < DB; ++b) {
                const uint32_t* v0 = reinterpret_cast<const uint32_t*>(&vr[0][b]);
                const uint32_t* v1 = reinterpret_cast<const uint32_t*>(&vr[1][b]);
                const uint32_t* v2 = reinterpret_cast<const uint32_t*>(&vr[2][b]);
                const uint32_t* v3 = reinterpret_cast<const uint32_t*>(&vr[3][b]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // elements 64 b + 8 g + 2 i and + 1 of this lane's piece
                    const uint32_t a0 = __byte_perm(v0[i], v1[i], 0x5410), a1 = __byte_perm(v0[i], v1[i], 0x7632);
                    const uint32_t a2 = __byte_perm(v2[i], v3[i], 0x5410), a3 = __byte_perm(v2[i], v3[i], 0x7632);
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_16816<T>(o[n][4 * b + i], a0, a1, a2, a3, p0[n], p1[n]);
                }
            }
            load_v(first + kStepKeys);
        }
        if (!MASKED) break;
    }

    // join the warps: o[n][4 b + i] of this lane are elements 64 b + 8 g + 2 i (0, 1) and + 1 (2, 3) of rows 2 t (0, 2), 2 t + 1 (1, 3)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
            for (int m = 4; m < 32; m <<= 1) sum[n][c] += __shfl_xor_sync(0xffffffffu, sum[n][c], m);
            const int r = 8 * n + 2 * t + c;
            if (g == 0) {
                s_m[warp][r] = ref[n][c];
                s_l[warp][r] = sum[n][c];
            }
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int i = 0; i < 4; i += 2)
                    *reinterpret_cast<float4*>(&s_o[warp][r][64 * b + 8 * g + 2 * i]) =
                        make_float4(o[n][4 * b + i][c], o[n][4 * b + i][c + 2], o[n][4 * b + i + 1][c], o[n][4 * b + i + 1][c + 2]);
        }
    __syncthreads();
    constexpr int PER = kStepThreads / ROWS;  // threads of a row, 8 elements of it at a time
    const int r = threadIdx.x / PER, part_of = threadIdx.x % PER;
    if (r >= rows || !OCTO_TOKEN_IN_RANGE(seg.q0 + a.group_div.div(row0 + r) < a.q_total, a.status)) return;
    float top = s_m[0][r];
#pragma unroll
    for (int w = 1; w < kStepWarps; ++w) top = fmaxf(top, s_m[w][r]);
    const float base = top == -INFINITY ? 0.0f : top;
    float share[kStepWarps], total = 0.0f;
#pragma unroll
    for (int w = 0; w < kStepWarps; ++w) {
        share[w] = ex2(s_m[w][r] - base);
        total += share[w] * s_l[w][r];
    }
    const int row = a.group_div.div(row0 + r), head = kvh * a.group + (row0 + r - row * a.group);
    const int64_t part = ((int64_t)split * a.q_total + seg.q0 + row) * a.heads + head;
    const bool last = active <= 1;
    const float inv = last ? (total > 0.0f || total != total ? 1.0f / total : 0.0f) : 1.0f;
    T* const out = static_cast<T*>(a.out) + (seg.q0 + row) * a.o_row + head * a.o_head;
    for (int d = 8 * part_of; d < a.dim; d += 8 * PER) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < kStepWarps; ++w) f[i] += share[w] * s_o[w][r][d + i];
            f[i] *= inv;
        }
        if (last) {
            uint4 y;
            y.x = pack2<T>(f[0], f[1]);
            y.y = pack2<T>(f[2], f[3]);
            y.z = pack2<T>(f[4], f[5]);
            y.w = pack2<T>(f[6], f[7]);
            *reinterpret_cast<uint4*>(out + d) = y;
        } else {
            float4* p = reinterpret_cast<float4*>(a.part_o + part * a.dim + d);
            p[0] = make_float4(f[0], f[1], f[2], f[3]);
            p[1] = make_float4(f[4], f[5], f[6], f[7]);
        }
    }
    if (!last && part_of == 0) a.part_ml[part] = make_float2(top, total);
}

// ---------------------------------------------------------------------------------------
// Joins the splits of a row: a warp per (query row, head), four elements of it per lane, the splits in order.
// ---------------------------------------------------------------------------------------
constexpr int kJoinThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kJoinThreads)
attend_join_kernel(const __grid_constant__ AttendArgs a) {
    pdl_wait();
    const int64_t at = ((int64_t)blockIdx.x * kJoinThreads + threadIdx.x) >> 5;  // row * heads + head
    const int lane = threadIdx.x & 31;
    if (at >= a.q_total * a.heads) return;
    const int64_t row = at / a.heads;
    const int head = (int)(at - row * a.heads);
    // the segment this row belongs to
    const int64_t step = row / a.q_rows + a.q_first;
    int s;
    if (a.q_offsets) {
        int lo = 0, hi = a.segments;  // last s with offsets[s] <= step
        if (a.q_offsets[0] > step) return;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.q_offsets[mid] <= step) lo = mid; else hi = mid;
        }
        s = lo;
    } else {
        if (step < 0 || step >= a.segments) return;
        s = (int)step;
    }
    const Segment seg = segment_of(a, s);
    if (row < seg.q0 || row >= seg.q0 + seg.qn) return;
    const int active = (seg.kn + a.chunk - 1) / a.chunk;
    if (active <= 1) return;
    const int64_t step_part = a.q_total * a.heads;
    float top = -INFINITY;
    for (int i = lane; i < active; i += 32) top = fmaxf(top, a.part_ml[i * step_part + at].x);
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    const float ref = top == -INFINITY ? 0.0f : top;
    const int d = 4 * lane;
    float sum = 0.0f;
    float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int i = 0; i < active; ++i) {
        const float2 ml = a.part_ml[i * step_part + at];
        const float w = ex2(ml.x - ref);
        sum += w * ml.y;
        if (d < a.dim) {
            const float4 p = *reinterpret_cast<const float4*>(a.part_o + (i * step_part + at) * a.dim + d);
            f.x += w * p.x;
            f.y += w * p.y;
            f.z += w * p.z;
            f.w += w * p.w;
        }
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    if (d < a.dim) {
        T* out = static_cast<T*>(a.out) + row * a.o_row + head * a.o_head + d;
        *reinterpret_cast<uint2*>(out) = make_uint2(pack2<T>(f.x * inv, f.y * inv), pack2<T>(f.z * inv, f.w * inv));
    }
}

// ---------------------------------------------------------------------------------------
// The plan of a call: which kernel, and into how many splits.  It follows from sizes alone.
// ---------------------------------------------------------------------------------------
struct AttendPlan {
    bool tile;            // attend_tile_kernel, else attend_step_kernel
    int64_t row_tiles;    // per segment and key head
    int splits, chunk;
    int64_t ctas;
    int64_t workspace;
};

static int validate(const octo_attend_t* c) {
    if (!c || c->device < 0) return OCTO_E_INVALID_ARG;
    if (c->dtype != OCTO_F16 && c->dtype != OCTO_BF16) return OCTO_E_INVALID_ARG;
    if (c->segments < 1 || c->heads < 1 || c->kv_heads < 1 || c->heads > 16384 || c->heads % c->kv_heads)
        return OCTO_E_INVALID_ARG;
    if (c->head_dim < 8 || c->head_dim > 128 || c->head_dim % 8) return OCTO_E_INVALID_ARG;
    const int64_t most = 1 << 30;
    if (c->q_total < 0 || c->k_total < 0 || c->q_total > most || c->k_total > most) return OCTO_E_INVALID_ARG;
    if (c->q_total * c->heads > INT32_MAX - 511) return OCTO_E_CAPACITY;  // rows of the last tile are numbered in 32 bits too
    if (c->q_rows < 1 || c->k_rows < 1 || c->q_rows > most || c->k_rows > most) return OCTO_E_INVALID_ARG;
    if (c->q_first < -most || c->q_first > most || c->k_first < -most || c->k_first > most) return OCTO_E_INVALID_ARG;
    if (c->max_q < 0 || c->max_k < 0) return OCTO_E_INVALID_ARG;
    if (!(fabsf(c->scale) <= 1e30f)) return OCTO_E_INVALID_ARG;
    if ((c->d_q_offsets || c->d_k_offsets) && c->segments > OCTO_MAX_SEGMENTS) return OCTO_E_CAPACITY;
    return OCTO_OK;
}

static int64_t bound_of(int64_t given, const int32_t* offsets, int64_t rows, int64_t total) {
    int64_t b = offsets ? total : (rows < total ? rows : total);
    if (given > 0 && given < b) b = given;
    return b < 1 ? 1 : b;
}

static int make_plan(const octo_attend_t* c, int sms, AttendPlan* p) {
    const int64_t group = c->heads / c->kv_heads;
    const int64_t max_q = bound_of(c->max_q, c->d_q_offsets, c->q_rows, c->q_total);
    const int64_t max_k = bound_of(c->max_k, c->d_k_offsets, c->k_rows, c->k_total);
    // Up to 16 rows a segment the step kernel reads every key once and is always ahead.  More rows take several of its
    // CTAs, which read the keys again, but a CTA is through in 3 us where a tile takes 7 to 9: it stays ahead while the
    // whole call is small.  Work in key rows read, with what a CTA costs beside them (256); us on the GPU tile / step:
    // 4 segments of 64 rows, 8 key heads of 128, 512 keys 13.9 / 9.5, 2048 keys 18.0 / 25.3; 64 segments of 32 rows, 128
    // keys 22.8 / 19.4, 512 keys 42 / 53; 64 of 64 rows, 8 key heads of 64, 128 keys 20.6 / 19.8; 8 of 128 rows, 2 key heads,
    // 512 keys 12.8 / 7.4.  Where it goes wrong: many segments of a dozen keys (216 of 28 rows and 18 keys, 16 heads of 64,
    // 82 / 44), which count as large.
    const double step_ctas = (double)c->segments * c->kv_heads * (double)((max_q * group + kStepRows - 1) / kStepRows);
    const double work = step_ctas * (double)(max_k + 256) * (c->head_dim > 64 ? 2 : 1);
    p->tile = max_q * group > kStepRows && work > (step_ctas >= 4.0 * sms ? 800e3 : 300e3);
    const int64_t tile_rows = p->tile ? kTileRows : kStepRows, step = p->tile ? kTileKeys : kStepKeys;
    p->row_tiles = (max_q * group + tile_rows - 1) / tile_rows;
    if ((double)c->segments * c->kv_heads * (double)p->row_tiles > (double)INT64_MAX / 1024) return OCTO_E_CAPACITY;
    const int64_t units = (int64_t)c->segments * c->kv_heads * p->row_tiles;
    // no more tiles than the rows make, with one that is not full in every segment
    const int64_t rows_make = (c->q_total * group + tile_rows - 1) / tile_rows + c->segments;
    const int64_t busy = units < rows_make * c->kv_heads ? units : rows_make * c->kv_heads;
    // Work is split over the keys, into splits of one size.  Few rows: up to kStepFill CTAs per SM, 512 keys at least.  Tiles:
    // up to one per SM at 512 keys at least, and beyond that up to four per SM at 2048 keys at least, since tiles of
    // uneven length on one CTA per SM end at different times.  us with up to one / up to four tiles per SM: 14 segments of 196
    // rows and 8000 to 32 000 keys, heads of 64, four heads 246 / 211, one head whose longest segment is not known 343 / 175
    // (where it is known 60 / 81: shorter splits than it needs); 5 segments of 300 rows, four heads of 128 190 / 147.
    auto at_most = [&](int64_t want, int64_t keys) {
        const int64_t a = want / busy, b = max_k / keys;
        return a < b ? a : b;
    };
    int64_t splits = p->tile ? at_most(sms, 512) : at_most((int64_t)sms * kStepFill + busy - 1, 512);
    if (p->tile && at_most((int64_t)sms * 4, 2048) > splits) splits = at_most((int64_t)sms * 4, 2048);
    if (splits < 1) splits = 1;
    const int64_t chunk = ((max_k + splits - 1) / splits + step - 1) / step * step;
    splits = (max_k + chunk - 1) / chunk;
    p->splits = (int)splits;
    p->chunk = splits == 1 ? (int)max_k : (int)chunk;
    p->ctas = p->tile ? (busy * splits < sms ? busy * splits : sms) : units * splits;
    p->workspace = splits == 1 ? 0 : splits * c->q_total * c->heads * (c->head_dim + 2) * (int64_t)sizeof(float);
    if (p->ctas > INT32_MAX || (!c->d_q_offsets && units > INT32_MAX)) return OCTO_E_CAPACITY;
    return OCTO_OK;
}

template <typename T>
static cudaError_t launch_attend(const AttendArgs& a, const AttendPlan& p, cudaStream_t stream) {
    cudaError_t e;
    if (p.tile) {
        e = launch_attend_tile(a, std::is_same<T, __nv_bfloat16>::value, (int)p.ctas, (int)p.row_tiles, stream);
    } else {
        const bool eight = a.max_q * a.group <= 8;
        void (*kernel)(const AttendArgs, int);
        if (a.dim <= 64)
            kernel = a.mask ? (eight ? attend_step_kernel<T, 1, 1, true> : attend_step_kernel<T, 1, 2, true>)
                            : (eight ? attend_step_kernel<T, 1, 1, false> : attend_step_kernel<T, 1, 2, false>);
        else
            kernel = a.mask ? (eight ? attend_step_kernel<T, 2, 1, true> : attend_step_kernel<T, 2, 2, true>)
                            : (eight ? attend_step_kernel<T, 2, 1, false> : attend_step_kernel<T, 2, 2, false>);
        e = launch_kernel(kernel, dim3((unsigned)p.ctas), dim3(kStepThreads), 0, stream, a, (int)p.row_tiles);
    }
    if (e == cudaSuccess && a.splits > 1) {
        const int64_t blocks = (a.q_total * a.heads * 32 + kJoinThreads - 1) / kJoinThreads;
        e = launch_kernel(attend_join_kernel<T>, dim3((unsigned)blocks), dim3(kJoinThreads), 0, stream, a);
    }
    return e;
}

}  // namespace octo

using namespace octo;

// The plan of a call; `work` says whether there is any.
static int plan_of(const octo_attend_t* c, AttendPlan* p, bool* work, const char* where) {
    *work = false;
    const int rc = validate(c);
    if (rc != OCTO_OK || c->q_total == 0) return rc;
    int sms = 0;
    const cudaError_t e = sm_count_of(c->device, &sms);
    if (e != cudaSuccess) return report_cuda_error(e, where);
    *work = true;
    return make_plan(c, sms, p);
}

extern "C" int octo_attend_workspace(const octo_attend_t* c, int64_t* bytes) {
    if (!bytes) return OCTO_E_INVALID_ARG;
    *bytes = 0;
    AttendPlan p;
    bool work;
    const int rc = plan_of(c, &p, &work, "octo_attend_workspace");
    if (rc == OCTO_OK && work) *bytes = p.workspace;
    return rc;
}

extern "C" int octo_attend_plan(const octo_attend_t* c, int32_t* tile, int32_t* splits) {
    if (!tile || !splits) return OCTO_E_INVALID_ARG;
    *tile = *splits = 0;
    AttendPlan p;
    bool work;
    const int rc = plan_of(c, &p, &work, "octo_attend_plan");
    if (rc == OCTO_OK && work) {
        *tile = p.tile ? 1 : 0;
        *splits = p.splits;
    }
    return rc;
}

extern "C" int octo_cross_attention(const octo_attend_t* c, void* d_workspace, int64_t workspace_bytes, void* cuda_stream) {
    const int rc = validate(c);
    if (rc != OCTO_OK) return rc;
    if (c->q_total == 0) return OCTO_OK;
    if (!c->q.d_data || !c->out.d_data || (c->k_total > 0 && (!c->k.d_data || !c->v.d_data))) return OCTO_E_INVALID_ARG;
    for (const octo_heads_t* t : {&c->q, &c->k, &c->v, &c->out})
        if (!aligned_to(t->d_data, 16) || t->row_stride % 8 || t->head_stride % 8) return OCTO_E_ALIGNMENT;
    for (const octo_heads_t* t : {&c->q, &c->k, &c->v, &c->out})
        for (int64_t s : {t->row_stride, t->head_stride})
            if (s < 0 || s >= (int64_t)1 << 30) return OCTO_E_INVALID_ARG;
    if (rows_coincide(c->out, c->q_total, c->heads, c->head_dim)) return OCTO_E_INVALID_ARG;
    if (!aligned_to(c->d_q_offsets, 4) || !aligned_to(c->d_k_offsets, 4) || !aligned_to(c->d_status, 4) ||
        !aligned_to(d_workspace, 16))
        return OCTO_E_ALIGNMENT;
    DeviceScope scope(c->device);
    if (scope.error != cudaSuccess) return report_cuda_error(scope.error, "octo_cross_attention");
    int sms = 0;
    cudaError_t e = sm_count_of(c->device, &sms);
    if (e != cudaSuccess) return report_cuda_error(e, "octo_cross_attention");
    AttendPlan p;
    const int prc = make_plan(c, sms, &p);
    if (prc != OCTO_OK) return prc;
    if (p.workspace > 0 && (!d_workspace || workspace_bytes < p.workspace)) return OCTO_E_CAPACITY;

    AttendArgs a;
    a.q = c->q.d_data;
    a.k = c->k.d_data;
    a.v = c->v.d_data;
    a.out = c->out.d_data;
    a.q_row = c->q.row_stride;
    a.q_head = c->q.head_stride;
    a.k_row = c->k.row_stride;
    a.k_head = c->k.head_stride;
    a.v_row = c->v.row_stride;
    a.v_head = c->v.head_stride;
    a.o_row = c->out.row_stride;
    a.o_head = c->out.head_stride;
    a.q_offsets = c->d_q_offsets;
    a.k_offsets = c->d_k_offsets;
    a.q_rows = c->q_rows;
    a.k_rows = c->k_rows;
    a.q_first = c->q_first;
    a.k_first = c->k_first;
    a.q_total = c->q_total;
    a.k_total = c->k_total;
    a.max_q = bound_of(c->max_q, c->d_q_offsets, c->q_rows, c->q_total);
    a.max_k = bound_of(c->max_k, c->d_k_offsets, c->k_rows, c->k_total);
    a.mask = c->d_key_mask;
    a.scale_log2 = (float)((double)c->scale * 1.44269504088896340736);
    // Equal weights, and still no weight for what is hidden (-infinity): the smallest number there is, 1.4e-45, makes of any
    // finite score at most 2^-21.
    if (a.scale_log2 == 0.0f) a.scale_log2 = 1e-45f;
    a.segments = c->segments;
    a.heads = c->heads;
    a.kv_heads = c->kv_heads;
    a.group = c->heads / c->kv_heads;
    a.group_div.set((unsigned)a.group);
    a.dim = c->head_dim;
    a.splits = p.splits;
    a.chunk = p.chunk;
    a.part_o = static_cast<float*>(d_workspace);
    a.part_ml = p.workspace > 0 ? reinterpret_cast<float2*>(a.part_o + (int64_t)p.splits * c->q_total * c->heads * c->head_dim)
                                : nullptr;
    a.status = c->d_status;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    e = c->dtype == OCTO_F16 ? launch_attend<__half>(a, p, stream) : launch_attend<__nv_bfloat16>(a, p, stream);
    return e == cudaSuccess ? OCTO_OK : report_cuda_error(e, "octo_cross_attention");
}
