// Attention for many query rows: both products on the tensor cores (tcgen05), accumulators in tensor memory.
//
// Work items are tiles of 256 rows -- pairs (query row, head) that share a key head -- of one segment and one split
// of its keys; a persistent grid of one CTA per SM walks over them.  Inside a CTA
//   warps 0-3, 4-7   one softmax group per half (128 rows, a thread per row): scores from tensor memory, running
//                    maximum and sum in registers, weights back into tensor memory over the scores they came from;
//                    at the end the half's rows of the result.
//   warp 8           issues all matrix instructions: S_h = Q_h K^T, O_h += P_h V.
//   warps 9-11       fetch queries, keys and values with 16-byte asynchronous copies into shared memory, in the
//                    128-byte swizzle that the matrix instructions read.  Copies by row (rather than by tensor
//                    map) let a tile consist of the VISIBLE keys only, wherever they lie: hidden keys cost a byte
//                    of mask and nothing else, and what they hold is never looked at.
// Keys are fetched 128 at a time and worked on 64 at a time: tensor memory holds two score buffers per half (S0a S0b
// S1a S1b, 64 columns each, then O0 and O1, 128 each), so that the scores of the next 64 keys are made while the
// softmax works on these and a half never waits for the matrix instructions of its own weights.
// A rescaling of O is rare: the reference that the exponents are taken against only follows the row's maximum
// when it has grown by more than 2^8 (weights up to 2^8 lose nothing in binary32 sums or 16-bit weights); the
// group then waits for the products under way and rescales O itself.
#include <math.h>

#include "octo_attend.cuh"
#include "octo_attend_tile.h"

namespace octo {

constexpr int kTileThreads = 384;
constexpr int kHalf = 128;            // rows of a half, keys of a tile
constexpr int kSub = 64;              // keys of a turn
constexpr int kLoaders = 96;
constexpr int kBlockBytes = 128 * 128;  // 128 rows of 64 elements
constexpr int kListInts = 256;
constexpr float kSlack = 8.0f;        // growth of the maximum, as a power of two, before the reference follows

template <int DB>
struct TileShape {
    static constexpr int kStages = DB == 1 ? 8 : 4;  // 16 or 32 KB each
    static constexpr int kStageBytes = DB * kBlockBytes;
    static constexpr int kQBytes = 2 * kStageBytes;
};

// What the other roles need to know of an item, left by the loaders.
struct TileInfo {
    int64_t q0, work;       // first query row of the segment; number of the item
    int kvh, split, row0, rows, last;
};

struct TileShared {
    uint64_t full[8], empty[8];
    uint64_t q_full, q_empty, done;
    uint64_t s_full[2][2], p_full[2][2], pv_done[2][2], o_empty[2];  // [half][turn & 1]: see below
    int meta[16];         // per key tile, by the loaders: visible keys | last << 16
    int half_meta[2][4];  // per half and turn, by the issuing warp: keys | kLast | item << kItemShift | kStop
    TileInfo info[4];
    uint32_t tmem;
    int list[3][kListInts];
    uint4 stage[8][32 * 4];  // per softmax warp: 32 rows of 32 elements on their way out
};
// A wait names the parity of one phase, so a barrier may be at most one phase away from the one that is waited for.  The
// scores, weights and products of a half therefore have a barrier for even and one for odd turns: turn n + 2 is not
// begun before turn n's weights are there, but turn n + 1 may be through before anyone has asked for turn n.
constexpr int kLast = 1 << 8, kStop = 1 << 9, kItemShift = 16;

// ---- tensor core and tensor memory ----------------------------------------------------------------------
// Descriptor of a shared-memory operand in the 128-byte swizzle.  Low word: start address and leading offset (distance
// of 64-element blocks for the values, unused else) in units of 16 bytes; high word: 8-row groups of 1024 bytes,
// version 1, swizzle mode.  The issuing thread keeps low words and adds to them: one thread issues everything, so
// a descriptor put together anew for every instruction was what the kernel waited for (145 clocks each).
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t lead) { return ((addr & 0x3ffffu) >> 4) | ((lead >> 4) << 16); }
__device__ __forceinline__ uint64_t desc_of(uint32_t low) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(low), "r"(kDescHigh));
    return d;
}
template <typename T> struct MmaFormat;
template <> struct MmaFormat<__half> { static constexpr uint32_t kCode = 0; };
template <> struct MmaFormat<__nv_bfloat16> { static constexpr uint32_t kCode = 1; };
template <typename T>
__device__ __forceinline__ uint32_t instr_desc(int n, bool b_mn_major) {
    // binary32 accumulator, both operands of type T, A along K, B along K or along N
    const uint32_t fmt = MmaFormat<T>::kCode;
    return (1u << 4) | (fmt << 7) | (fmt << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define OCTO_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define OCTO_P8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define OCTO_W8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of the warp's 32 lanes; lane l holds row l
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : OCTO_R8(r, 0), OCTO_R8(r, 8), OCTO_R8(r, 16), OCTO_R8(r, 24)
        : "r"(addr)
        : "memory");
}
// The 32 registers of the latest load are there from here on (they pass through, so that no use moves above).
__device__ __forceinline__ void tmem_landed(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : OCTO_P8(r, 0), OCTO_P8(r, 8), OCTO_P8(r, 16), OCTO_P8(r, 24)::"memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
        "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::OCTO_W8(r, 0), OCTO_W8(r, 8), OCTO_W8(r, 16), OCTO_W8(r, 24), "r"(addr)
        : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool take) {
    const uint32_t bytes = take ? 16u : 0u;  // nothing is read, zeros are written
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// ---- work items -------------------------------------------------------------------------------------------
struct TileItem {
    Segment seg;
    int kvh, split, row0, rows;  // first row of the tile and rows in it (1 .. 256)
    int kb, ke;                  // key rows of this split, inside the segment
    bool last;                   // the segment's only split: writes the result
};

// Item w of the grid's list; false where there is nothing to do.  prefix: first tile of every segment (ragged
// queries), or null: tiles_per_segment each.
__device__ __forceinline__ bool tile_item(const AttendArgs& a, const int* prefix, int tiles_per_segment, int64_t w, TileItem& it) {
    it.split = (int)(w % a.splits);
    const int64_t u = w / a.splits;
    int s, tiles, first;
    if (prefix) {
        int lo = 0, hi = a.segments;  // last s with prefix[s] * kv_heads <= u
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((int64_t)prefix[mid] * a.kv_heads <= u) lo = mid; else hi = mid;
        }
        s = lo;
        first = prefix[s];
        tiles = prefix[s + 1] - first;
    } else {
        s = (int)(u / ((int64_t)tiles_per_segment * a.kv_heads));
        tiles = tiles_per_segment;
        first = s * tiles_per_segment;
    }
    const int in = (int)(u - (int64_t)first * a.kv_heads);
    it.kvh = in / tiles;
    it.row0 = (in - it.kvh * tiles) * (2 * kHalf);
    it.seg = segment_of(a, s);
    it.rows = min(it.seg.qn * a.group - it.row0, 2 * kHalf);
    it.kb = min(it.split * a.chunk, it.seg.kn);
    it.ke = min(it.kb + a.chunk, it.seg.kn);
    it.last = it.seg.kn <= a.chunk;
    return it.rows > 0 && (it.split == 0 || it.kb < it.ke);
}

// Row r (of a segment and key head) -> query row and head.
__device__ __forceinline__ void tile_row(const AttendArgs& a, int kvh, int r, int& qrow, int& head) {
    qrow = a.group_div.div(r);
    head = kvh * a.group + (r - qrow * a.group);
}

// One wait of a role.  A wait that runs out is reported; the role then leaves, and so do the others in turn.
__device__ __forceinline__ bool tile_wait(uint64_t* bar, uint32_t parity, unsigned int* status) {
    if (mbar_wait_bounded(bar, parity)) return true;
    if (status) atomicOr(status, OCTO_STATUS_COPY_TIMEOUT);
    return false;
}

template <int DB>
struct Loader {
    unsigned int* status;
    int lane, warp;
    uint32_t slot = 0;             // ring slots issued so far
    uint64_t *oldest, *second, *newest;  // barriers of the groups in flight
    int in_flight = 0;
    bool dead = false;

    __device__ __forceinline__ void arrive_oldest() {
        fence_proxy_async();  // the matrix instructions read through the asynchronous proxy
        mbar_arrive(oldest);
        oldest = second;
        second = newest;
        --in_flight;
    }
    __device__ __forceinline__ void issued(uint64_t* bar) {
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (in_flight == 0) oldest = bar;
        else if (in_flight == 1) second = bar;
        else newest = bar;
        if (++in_flight == 3) {
            asm volatile("cp.async.wait_group 2;" ::: "memory");
            arrive_oldest();
        }
    }
    __device__ __forceinline__ void flush() {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        while (in_flight > 0) arrive_oldest();
    }
    // Whoever waits hands over what has landed first: the wait may be for a consumer of just that.
    __device__ __forceinline__ void wait(uint64_t* bar, uint32_t parity) {
        if (__all_sync(0xffffffffu, mbar_test_wait(bar, parity))) return;
        flush();
        if (!__all_sync(0xffffffffu, tile_wait(bar, parity, status))) dead = true;
    }

    // A warp takes every third group of 8 rows, kRowsAtOnce rows per instruction; the swizzle of a lane's row inside
    // its group, and so its place in shared memory, is the same for every group.
    static constexpr int kLanesPerRow = 8 * DB, kRowsAtOnce = 32 / kLanesPerRow, kTurns = 8 / kRowsAtOnce;
    uint32_t place[kTurns];  // of the lane's piece of row kRowsAtOnce * i + its own in a group
    bool wide;               // the lane's piece lies inside the head
    __device__ __forceinline__ void layout(int dim_bytes) {
        const int c = lane & (kLanesPerRow - 1), own = lane / kLanesPerRow;
        wide = c * 16 < dim_bytes;
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int r = kRowsAtOnce * i + own;
            place[i] = (uint32_t)(c >> 3) * kBlockBytes + (uint32_t)r * 128u + (uint32_t)(((c & 7) ^ r) << 4);
        }
    }
    // Rows [0, count) of a tile, count a multiple of 8; row_at(r) gives a row's address or null for zeros.
    template <typename F>
    __device__ __forceinline__ void rows(uint32_t dst, int count, F row_at) {
        const int c = lane & (kLanesPerRow - 1), own = lane / kLanesPerRow;
        for (int g = warp; g < (count >> 3); g += 3) {
            const uint32_t at = dst + (uint32_t)g * 1024u;
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                const char* p = row_at(8 * g + kRowsAtOnce * i + own);
                const bool take = wide && p != nullptr;
                cp_async16(at + place[i], take ? p + c * 16 : zero_row, take);
            }
        }
    }
    // 128 rows that lie side by side from `src` on, `stride` bytes apart.
    __device__ __forceinline__ void full_rows(uint32_t dst, const char* src, int64_t stride) {
        const int c = lane & (kLanesPerRow - 1), own = lane / kLanesPerRow;
        const char* p = wide ? src + (8 * warp + own) * stride + c * 16 : zero_row;
        const int64_t turn = wide ? kRowsAtOnce * stride : 0, group = wide ? 24 * stride : 0;
        uint32_t at = dst + (uint32_t)warp * 1024u;
        for (int g = warp; g < 16; g += 3) {
#pragma unroll
            for (int i = 0; i < kTurns; ++i) cp_async16(at + place[i], p + i * turn, wide);
            p += group;
            at += 3 * 1024u;
        }
    }
    const char* zero_row;  // any valid address
};

template <typename T, int DB>
__global__ void __launch_bounds__(kTileThreads, 1)
attend_tile_kernel(const __grid_constant__ AttendArgs a, int tiles_per_segment, int ragged) {
    using Shape = TileShape<DB>;
    extern __shared__ uint8_t raw[];
    uint8_t* const base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    TileShared* const sh = reinterpret_cast<TileShared*>(base + Shape::kQBytes + Shape::kStages * Shape::kStageBytes);
    int* const prefix = ragged ? reinterpret_cast<int*>(sh + 1) : nullptr;
    const uint32_t q_base = smem_u32(base), ring = q_base + Shape::kQBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < Shape::kStages; ++i) {
            mbar_init(&sh->full[i], kLoaders);
            mbar_init(&sh->empty[i], 1);
        }
        mbar_init(&sh->q_full, kLoaders);
        mbar_init(&sh->q_empty, 1);
        mbar_init(&sh->done, 1);
        for (int h = 0; h < 2; ++h) {
            mbar_init(&sh->s_full[h][0], 2);
            mbar_init(&sh->s_full[h][1], 2);
            mbar_init(&sh->p_full[h][0], kHalf);
            mbar_init(&sh->p_full[h][1], kHalf);
            mbar_init(&sh->pv_done[h][0], 1);
            mbar_init(&sh->pv_done[h][1], 1);
            mbar_init(&sh->o_empty[h], kHalf);
        }
        mbar_fence_init();
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sh->tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    pdl_wait();
    if (ragged) {
        for (int s = threadIdx.x; s < a.segments; s += kTileThreads)
            prefix[s + 1] = (segment_of(a, s).qn * a.group + 2 * kHalf - 1) / (2 * kHalf);
        __syncthreads();
        if (warp == 0) {  // inclusive sums, a strip of segments per lane
            const int strip = (a.segments + 31) >> 5, b = lane * strip, e = min(a.segments, b + strip);
            int64_t sum = 0;
            for (int s = b; s < e; ++s) sum += prefix[s + 1];
            int64_t run = sum;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int64_t t = __shfl_up_sync(0xffffffffu, run, off);
                if (lane >= off) run += t;
            }
            run -= sum;
            for (int s = b; s < e; ++s) {
                run += prefix[s + 1];
                prefix[s + 1] = (int)min(run, (int64_t)1 << 30);  // (more than rows that do not overlap can make)
            }
            if (lane == 0) prefix[0] = 0;
        }
    }
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh->tmem, 0);
    const int64_t total = (ragged ? (int64_t)prefix[a.segments] : (int64_t)a.segments * tiles_per_segment) * a.kv_heads * a.splits;

    if (warp < 8) {
        // ---------------- softmax of one half ----------------
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const int h = warp >> 2, row = threadIdx.x & (kHalf - 1);
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);  // the warp's 32 lanes of tensor memory
        const uint32_t o_at = lanes + 256u + 128u * h;
        const float sc = a.scale_log2;
        const int o_chunks = (a.dim + 31) >> 5;
        uint32_t turn = 0;  // turns so far; the scores of turn n are in buffer n & 1
        int64_t done_work = -1;
        bool dead = false;
        for (;;) {
            float ref = -INFINITY, sum = 0.0f;  // what the exponents are taken against; sum of the weights
            bool first = true;
            int meta = 0;
            while (!(meta & (kLast | kStop))) {
                if (!__all_sync(0xffffffffu, tile_wait(&sh->s_full[h][turn & 1], (turn >> 1) & 1, a.status))) {
                    dead = true;
                    break;
                }
                tmem_after_sync();
                meta = sh->half_meta[h][turn & 3];
                if (meta & kStop) break;
                const int take = meta & 0xff;
                const uint32_t s_at = lanes + 128u * h + 64u * (turn & 1);
                // Weights against the reference so far, and the scores' maximum beside them: the exponentials do not wait
                // for the maximum.  Only if a row's has outgrown the reference (and for the first turn, whose
                // scores are looked through before) is the reference moved and the turn, still in tensor memory, taken again.
                uint32_t p[32];
                unsigned long long part = 0ull;
                for (bool look = first;;) {
                    if (look) {
                        float top = -INFINITY;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            if (32 * c >= take) break;
                            uint32_t s[32];
                            tmem_ld32(s_at + 32 * c, s);
                            tmem_landed(s);
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (32 * c + i < take) top = fmaxf(top, __uint_as_float(s[i]) * sc);
                        }
                        const float now = fmaxf(ref, top);
                        const float f = now == -INFINITY ? 1.0f : ex2(ref - now);
                        sum *= f;
                        ref = now;
                        if (!first) {  // (of the products, all but the last turn's are complete: the scores came after them)
                            if (!__all_sync(0xffffffffu, tile_wait(&sh->pv_done[h][(turn - 1) & 1], ((turn - 1) >> 1) & 1, a.status))) dead = true;
                            tmem_after_sync();
                            for (int c = 0; c < o_chunks; ++c) {
                                uint32_t o[32];
                                tmem_ld32(o_at + 32 * c, o);
                                tmem_landed(o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tmem_st32(o_at + 32 * c, o);
                            }
                        }
                    }
                    const float minus = ref == -INFINITY ? 0.0f : -ref;
                    const unsigned long long sc2 = f32x2(sc, sc), minus2 = f32x2(minus, minus);
                    float top = -INFINITY;  // above the reference
                    part = 0ull;
                    uint32_t s[2][32];
                    tmem_ld32(s_at, s[0]);
                    tmem_landed(s[0]);
                    if (take > 32) tmem_ld32(s_at + 32, s[1]);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (c > 0) {
                            if (take <= 32) {  // (the matrix instruction reads the first 32 weights then)
#pragma unroll
                                for (int i = 0; i < 16; ++i) p[16 + i] = 0u;
                                break;
                            }
                            tmem_landed(s[1]);
                        }
                        if (take < 32 * (c + 1)) {  // columns behind the last visible key weigh nothing
                            const uint32_t none = __float_as_uint(sc < 0.0f ? INFINITY : -INFINITY);
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (32 * c + i >= take) s[c][i] = none;
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t* const in = s[c] + 2 * i;
                            float x, y;
                            asm("mov.b64 {%0, %1}, %2;"
                                : "=f"(x), "=f"(y)
                                : "l"(fma_f32x2(f32x2(__uint_as_float(in[0]), __uint_as_float(in[1])), sc2, minus2)));
                            top = max3(top, x, y);
                            x = ex2(x);
                            y = ex2(y);
                            part = add_f32x2(part, f32x2(x, y));
                            // the weights in the type of the values: what the matrix instruction takes (the sum keeps them unrounded)
                            p[16 * c + i] = pack2<T>(x, y);
                        }
                    }
                    // (false for NaN: it leaves the reference and comes through the exponentials)
                    if (look || !__any_sync(0xffffffffu, (ref == -INFINITY && top > -INFINITY) || top > kSlack)) break;
                    look = true;
                }
                first = false;
                tmem_st32(s_at, p);
                {
                    float x, y;
                    asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(part));
                    sum += x + y;
                }
                tmem_wait_st();
                tmem_before_sync();
                mbar_arrive(&sh->p_full[h][turn & 1]);
                ++turn;
            }
            if (dead || (meta & kStop)) break;
            // the half's rows of the result
            const TileInfo it = sh->info[meta >> kItemShift];
            if (!__all_sync(0xffffffffu, tile_wait(&sh->pv_done[h][(turn - 1) & 1], ((turn - 1) >> 1) & 1, a.status))) {
                dead = true;
                break;
            }
            tmem_after_sync();
            done_work = it.work;
            const int r0 = it.row0 + h * kHalf, end = it.row0 + it.rows;
            const float inv = it.last ? (sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f) : 1.0f;
            if (it.last) {
                // four lanes to a row and 64 bytes of it at once, by way of shared memory
                uint4* const stage = sh->stage[warp];
                T* row_out[4];
                bool real[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int r = r0 + (row & ~31) + 8 * k + (lane >> 2);
                    int qrow, head;
                    tile_row(a, it.kvh, r, qrow, head);
                    real[k] = r < end;
                    row_out[k] = static_cast<T*>(a.out) + (it.q0 + qrow) * a.o_row + head * a.o_head + 8 * (lane & 3);
                }
                for (int c = 0; c < o_chunks; ++c) {
                    uint32_t o[32];
                    tmem_ld32(o_at + 32 * c, o);
                    tmem_landed(o);
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t y[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            y[j] = pack2<T>(__uint_as_float(o[8 * i + 2 * j]) * inv, __uint_as_float(o[8 * i + 2 * j + 1]) * inv);
                        stage[4 * lane + (i ^ ((lane >> 1) & 3))] = make_uint4(y[0], y[1], y[2], y[3]);
                    }
                    __syncwarp();
                    const bool inside = 32 * c + 8 * (lane & 3) < a.dim;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int l = 8 * k + (lane >> 2);
                        const uint4 v = stage[4 * l + ((lane & 3) ^ ((l >> 1) & 3))];
                        if (real[k] && inside) *reinterpret_cast<uint4*>(row_out[k] + 32 * c) = v;
                    }
                }
            } else {
                const int r = r0 + row;
                int qrow, head;
                tile_row(a, it.kvh, r, qrow, head);
                const int64_t at = ((int64_t)it.split * a.q_total + it.q0 + qrow) * a.heads + head;
                for (int c = 0; c < o_chunks; ++c) {
                    uint32_t o[32];
                    __syncwarp();
                    tmem_ld32(o_at + 32 * c, o);
                    tmem_landed(o);
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        if (r < end && 32 * c + i < a.dim)
                            *reinterpret_cast<uint4*>(a.part_o + at * a.dim + 32 * c + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                }
                if (r < end) a.part_ml[at] = make_float2(ref, sum);
            }
            __syncwarp();
            tmem_before_sync();
            mbar_arrive(&sh->o_empty[h]);
        }
        if (dead) {  // a wait has run out: rows that are not done say so
            const float nan = __int_as_float(0x7fffffff);
            for (int64_t w = done_work < 0 ? blockIdx.x : done_work + gridDim.x; w < total; w += gridDim.x) {
                TileItem it;
                if (!tile_item(a, prefix, tiles_per_segment, w, it)) continue;
                const int r = it.row0 + h * kHalf + row;
                if (r >= it.row0 + it.rows) continue;
                int qrow, head;
                tile_row(a, it.kvh, r, qrow, head);
                T* const out = static_cast<T*>(a.out) + (it.seg.q0 + qrow) * a.o_row + head * a.o_head;
                const int64_t at = ((int64_t)it.split * a.q_total + it.seg.q0 + qrow) * a.heads + head;
                if (!it.last) a.part_ml[at] = make_float2(0.0f, nan);
                for (int d = 0; it.last && d < a.dim; d += 2) *reinterpret_cast<uint32_t*>(out + d) = pack2<T>(nan, nan);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        if (warp == 8) {
            {
                // ---------------- matrix instructions ----------------
                // The whole warp walks through the loop and one elected lane issues, so that descriptors and addresses
                // are the warp's and stay in uniform registers.
                const int ksteps = (a.dim + 15) >> 4;
                const uint32_t idesc_pv = instr_desc<T>(16 * ksteps, true), idesc_qk = instr_desc<T>(0, false);
                uint32_t slot = 0, tile = 0, items = 0;
                uint32_t turns[2] = {0, 0}, weights[2] = {0, 0}, half_items[2] = {0, 0};  // scores issued, weights used
                bool ok = true;
                auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, tile_wait(bar, parity, a.status)); };
                auto commit = [&](uint64_t* bar) {
                    if (elect_one()) mma_commit(bar);
                    __syncwarp();
                };
                auto full_wait = [&](uint32_t n) { wait(&sh->full[n % Shape::kStages], (n / Shape::kStages) & 1); };
                auto slot_at = [&](uint32_t n) { return ring + (n % Shape::kStages) * Shape::kStageBytes; };
                // S_h = Q_h K^T over keys [64 sub, 64 sub + keys) of the tile in k_slot
                auto scores = [&](int h, uint32_t k_slot, int sub, int keys, int flags) {
                    const int n = max(16, (keys + 15) & ~15);
                    const uint32_t idesc = idesc_qk + ((uint32_t)(n >> 3) << 17), d = tmem + 128u * h + 64u * (turns[h] & 1);
                    const uint32_t qa = desc_low(q_base + h * Shape::kStageBytes, 0), ka = desc_low(slot_at(k_slot) + 8192u * sub, 0);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 4 * DB; ++k) {
                            const uint32_t off = ((uint32_t)(k >> 2) * kBlockBytes + (uint32_t)(k & 3) * 32u) >> 4;
                            if (k < ksteps) mma_ss(d, desc_of(qa + off), desc_of(ka + off), idesc, k > 0);
                        }
                        sh->half_meta[h][turns[h] & 3] = keys | flags;
                        mma_commit(&sh->s_full[h][turns[h] & 1]);
                        mbar_arrive(&sh->s_full[h][turns[h] & 1]);
                    }
                    __syncwarp();
                    ++turns[h];
                };
                for (;;) {
                    wait(&sh->q_full, items & 1);
                    if (!ok) break;
                    const int rows = __shfl_sync(0xffffffffu, sh->info[items & 3].rows, 0);
                    if (rows == 0) break;  // no more items
                    const int halves = rows > kHalf ? 2 : 1, tag = (int)(items & 3) << kItemShift;
                    // One walk over the turns of the item: the scores of turn j + 1 are issued ahead of the products
                    // of turn j.  (k_slot, k_sub, k_keys): where the scores are; v_*: where the products are.
                    uint32_t k_slot = slot;
                    full_wait(k_slot);
                    if (!ok) break;
                    tmem_after_sync();
                    int k_meta = __shfl_sync(0xffffffffu, sh->meta[tile & 15], 0), k_sub = 0;
                    ++tile;
                    bool more = true, first = true;
                    int v_keys = 0, v_sub = 0;
                    uint32_t v_slot = 0;
                    bool v_frees = false;
                    for (;;) {
                        int keys = 0, sub = 0;
                        uint32_t at = 0;
                        bool frees = false;
                        if (more) {
                            const int left = (k_meta & 0xffff) - kSub * k_sub;
                            keys = min(left, kSub);
                            sub = k_sub;
                            at = k_slot;
                            frees = left <= kSub;  // the tile's last turn
                            const bool last = frees && (k_meta >> 16);
                            for (int h = 0; h < halves; ++h) scores(h, k_slot, sub, keys, (last ? kLast : 0) | tag);
                            if (frees) {
                                commit(&sh->empty[k_slot % Shape::kStages]);
                                if (last) commit(&sh->q_empty);
                            }
                            more = !last;
                            ++k_sub;
                        }
                        if (!first) {
                            // O_h += P_h V over the turn before
                            if (v_sub == 0) full_wait(v_slot);
                            const bool start = v_slot == slot + 1 && v_sub == 0, stop = keys == 0 && !frees;
                            const uint32_t va = desc_low(slot_at(v_slot) + 8192u * v_sub, kBlockBytes);
                            const int steps = max(1, (v_keys + 15) >> 4);
                            for (int h = 0; h < halves && ok; ++h) {
                                wait(&sh->p_full[h][weights[h] & 1], (weights[h] >> 1) & 1);
                                if (start) wait(&sh->o_empty[h], (half_items[h] & 1) ^ 1);
                                if (!ok) break;
                                tmem_after_sync();
                                const uint32_t pa = tmem + 128u * h + 64u * (weights[h] & 1);
                                if (elect_one()) {
#pragma unroll
                                    for (int k = 0; k < 4; ++k)
                                        if (k < steps)
                                            mma_ts(tmem + 256u + 128u * h, pa + 8u * k, desc_of(va + 128u * k), idesc_pv, !start || k > 0);
                                    mma_commit(&sh->pv_done[h][weights[h] & 1]);
                                }
                                __syncwarp();
                                ++weights[h];
                                if (stop) ++half_items[h];
                            }
                            if (!ok) break;
                            if (v_frees) commit(&sh->empty[v_slot % Shape::kStages]);
                            if (stop) {
                                slot = v_slot + 1;
                                break;
                            }
                        }
                        first = false;
                        v_keys = keys;
                        v_sub = sub;
                        v_slot = at + 1;
                        v_frees = frees;
                        if (more && frees) {  // on to the next tile's keys
                            k_slot += 2;
                            k_sub = 0;
                            full_wait(k_slot);
                            if (!ok) break;
                            tmem_after_sync();
                            k_meta = __shfl_sync(0xffffffffu, sh->meta[tile & 15], 0);
                            ++tile;
                        }
                    }
                    if (!ok) break;
                    ++items;
                }
                if (ok) {  // the softmax groups may leave
                    if (elect_one()) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            sh->half_meta[h][turns[h] & 3] = kStop;
                            mbar_arrive(&sh->s_full[h][turns[h] & 1]);
                            mbar_arrive(&sh->s_full[h][turns[h] & 1]);
                        }
                    }
                    __syncwarp();
                }
                commit(&sh->done);  // nothing of this CTA is under way when it gives its memory back
                tile_wait(&sh->done, 0, a.status);
            }
        } else {
            // ---------------- loads ----------------
            Loader<DB> ld;
            ld.status = a.status;
            ld.lane = lane;
            ld.warp = warp - 9;
            ld.zero_row = static_cast<const char*>(a.q);
            int* const list = sh->list[warp - 9];
            ld.layout(2 * a.dim);
            uint32_t items = 0, tile = 0;
            for (int64_t w = blockIdx.x; w < total && !ld.dead; w += gridDim.x) {
                TileItem it;
                if (!tile_item(a, prefix, tiles_per_segment, w, it)) continue;
                // the queries follow the first keys and values: their place is free only when the last item's scores are made
                auto load_queries = [&]() {
                    ld.wait(&sh->q_empty, (items & 1) ^ 1);
                    if (ld.dead) return;
                    const int64_t row = 2 * a.q_row, head = 2 * a.q_head;
                    const char* const q = static_cast<const char*>(a.q) + it.seg.q0 * row + (int64_t)it.kvh * a.group * head;
                    for (int b = 0; b < it.rows; b += kHalf) {
                        if (a.group == 1 && it.rows - b >= kHalf)
                            ld.full_rows(q_base + (b / kHalf) * Shape::kStageBytes, q + (it.row0 + b) * row, row);
                        else
                            ld.rows(q_base + (b / kHalf) * Shape::kStageBytes, kHalf, [&](int r) -> const char* {
                                int qrow, hd;
                                tile_row(a, 0, it.row0 + b + r, qrow, hd);
                                return b + r < it.rows ? q + qrow * row + hd * head : nullptr;
                            });
                    }
                    if (warp == 9 && lane == 0) {
                        TileInfo& info = sh->info[items & 3];
                        info.q0 = it.seg.q0;
                        info.work = w;
                        info.kvh = it.kvh;
                        info.split = it.split;
                        info.row0 = it.row0;
                        info.rows = it.rows;
                        info.last = it.last;
                    }
                    ld.issued(&sh->q_full);
                    ++items;
                };
                bool queries = false;
                const char* const k = reinterpret_cast<const char*>(static_cast<const T*>(a.k) + it.seg.k0 * a.k_row + it.kvh * a.k_head);
                const char* const v = reinterpret_cast<const char*>(static_cast<const T*>(a.v) + it.seg.k0 * a.v_row + it.kvh * a.v_head);
                const uint8_t* const mask = a.mask ? a.mask + it.seg.k0 : nullptr;
                int cursor = it.kb, listed = 0;
                for (bool last = false; !last && !ld.dead; ++tile) {
                    // the next 128 visible keys
                    int take, from = cursor;
                    if (mask) {
                        while (listed <= kHalf && cursor < it.ke) {
                            bool seen[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const int key = cursor + 32 * j + lane;
                                seen[j] = key < it.ke && mask[key] != 0;
                            }
                            // (at most 128 are listed here, and 128 more fit)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const unsigned ballot = __ballot_sync(0xffffffffu, seen[j]);
                                if (seen[j]) list[listed + __popc(ballot & ((1u << lane) - 1u))] = cursor + 32 * j + lane;
                                listed += __popc(ballot);
                            }
                            cursor += 128;
                        }
                        __syncwarp();
                        take = min(listed, kHalf);
                        last = listed <= kHalf;
                    } else {
                        take = min(it.ke - cursor, kHalf);
                        cursor += take;
                        last = cursor >= it.ke;
                    }
                    const int padded = max(16, (take + 15) & ~15);  // rows that the matrix instructions read
                    if (warp == 9 && lane == 0) sh->meta[tile & 15] = take | (last ? 1 << 16 : 0);
#pragma unroll
                    for (int which = 0; which < 2; ++which) {
                        const uint32_t n = ld.slot;
                        ld.wait(&sh->empty[n % Shape::kStages], ((n / Shape::kStages) & 1) ^ 1);
                        if (ld.dead) break;
                        const char* const src = which ? v : k;
                        const int64_t stride = 2 * (which ? a.v_row : a.k_row);
                        const uint32_t dst = ring + (n % Shape::kStages) * Shape::kStageBytes;
                        if (mask)
                            ld.rows(dst, padded, [&](int r) -> const char* { return r < take ? src + list[r] * stride : nullptr; });
                        else if (take == kHalf)
                            ld.full_rows(dst, src + from * stride, stride);
                        else
                            ld.rows(dst, padded, [&](int r) -> const char* { return r < take ? src + (from + r) * stride : nullptr; });
                        ld.issued(&sh->full[n % Shape::kStages]);
                        ++ld.slot;
                    }
                    if (!queries && !ld.dead) {
                        load_queries();
                        queries = true;
                    }
                    if (mask) {  // what is left over moves to the front
                        listed -= take;
                        int rest[4];
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 4; ++j) rest[j] = 32 * j + lane < listed ? list[kHalf + 32 * j + lane] : 0;
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (32 * j + lane < listed) list[32 * j + lane] = rest[j];
                        __syncwarp();
                    }
                }
            }
            if (!ld.dead) ld.wait(&sh->q_empty, (items & 1) ^ 1);
            ld.flush();
            if (!ld.dead) {  // an item without rows: there are no more
                if (warp == 9 && lane == 0) sh->info[items & 3].rows = 0;
                __syncwarp();
                mbar_arrive(&sh->q_full);
            }
        }
    }
    tmem_before_sync();
    __syncthreads();
    if (warp == 8) {
        __syncwarp();
        tmem_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
}

template <typename T, int DB>
static cudaError_t launch_shape(const AttendArgs& a, int grid, int tiles_per_segment, cudaStream_t stream) {
    using Shape = TileShape<DB>;
    const bool ragged = a.q_offsets != nullptr;
    const size_t fixed = 1024 + Shape::kQBytes + Shape::kStages * Shape::kStageBytes + sizeof(TileShared);
    const size_t most = fixed + sizeof(int) * (OCTO_MAX_SEGMENTS + 1);
    static_assert(1024 + Shape::kQBytes + Shape::kStages * Shape::kStageBytes + sizeof(TileShared) +
                          sizeof(int) * (OCTO_MAX_SEGMENTS + 1) <= 232448,
                  "shared memory of a CTA");
    auto kernel = attend_tile_kernel<T, DB>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e != cudaSuccess) return e;
    const size_t smem = fixed + (ragged ? sizeof(int) * ((size_t)a.segments + 1) : 0);
    return launch_kernel(kernel, dim3((unsigned)grid), dim3(kTileThreads), smem, stream, a, tiles_per_segment, ragged ? 1 : 0);
}

cudaError_t launch_attend_tile(const AttendArgs& a, int bf16, int grid, int tiles_per_segment, cudaStream_t stream) {
    if (a.dim <= 64)
        return bf16 ? launch_shape<__nv_bfloat16, 1>(a, grid, tiles_per_segment, stream)
                    : launch_shape<__half, 1>(a, grid, tiles_per_segment, stream);
    return bf16 ? launch_shape<__nv_bfloat16, 2>(a, grid, tiles_per_segment, stream)
                : launch_shape<__half, 2>(a, grid, tiles_per_segment, stream);
}

}  // namespace octo
