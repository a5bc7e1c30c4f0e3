// Attention for many query rows: both products on the tensor cores (tcgen05), accumulators in tensor memory.
//
// Work items are tiles of 256 rows -- pairs (query row, head) that share a key head -- of one segment and one split
// of its keys; a persistent grid of one CTA per SM walks over them.  Inside a CTA
//   warps 0-3, 4-7   one softmax group per half (128 rows, a thread per row): scores from tensor memory, running
//                    maximum and sum in registers, weights back into tensor memory over the scores they came from;
//                    at the end the half's rows of the result.
//   warps 8, 9       issue the matrix instructions of one half each: S_h = Q_h K^T, O_h += P_h V.  (One warp for both was
//                    what the kernel waited for: its waits, about 150 clocks each though satisfied, left the tensor
//                    cores idle for 40 % of the time.)
//   warps 10-13      fetch queries, keys and values with 16-byte asynchronous copies into shared memory, in the
//                    128-byte swizzle that the matrix instructions read.  Copies by row (rather than by tensor
//                    map) let a tile consist of the VISIBLE keys only, wherever they lie: hidden keys cost a byte
//                    of mask and nothing else, and what they hold is never looked at.
// Keys are fetched 128 at a time and worked on 64 at a time: tensor memory holds two score buffers per half (S0a S0b
// S1a S1b, 64 columns each, then O0 and O1, 128 each), so that the scores of the next 64 keys are made while the
// softmax works on these and a half never waits for the matrix instructions of its own weights.
// A rescaling of O is rare: the reference that the exponents are taken against only follows the row's maximum when the
// weights have grown large (kMostInTurn); the group then waits for the products under way and rescales O itself.
#include <math.h>

#include "octo_attend.cuh"
#include "octo_attend_tile.h"

namespace octo {

constexpr int kTileThreads = 512;
constexpr int kHalf = 128;            // rows of a half, keys of a tile
constexpr int kSub = 64;              // keys of a turn
constexpr int kLoadWarps = 4, kLoaders = 32 * kLoadWarps;
constexpr int kBlockBytes = 128 * 128;  // 128 rows of 64 elements
constexpr int kListInts = 256;
// The reference that exponents are taken against stays while a turn's 64 weights sum to no more than 2^10 (weights that
// large lose nothing in binary32 sums, and fp16 holds them); where they sum to more, one of them is above 2^4.
constexpr float kMostInTurn = 1024.0f, kGrown = 4.0f;

// Both halves begin an item together and stay in step, so that their exponentials share the special-function unit at one
// time and leave it alone at another.  Half a turn of delay for the second half, once an item, sets them apart.
// us without / with: crops of 32 frames, heads of 128, 1600 keys 1699 / 1589 at 1965 MHz (ten calls), 1927 / 1827 at
// 1730 / 1660 MHz (1.5 s of calls, power cap); of 64 frames, 49 rows, heads of 64, 900 visible keys 552 / 542; ragged
// items of a few turns, heads of 80 23.5 / 22.6 (400, 1000 and 1400 clocks gave less on the first).
constexpr int kStagger = 700;

template <int DB>
struct TileShape {
    static constexpr int kStages = DB == 1 ? 8 : 4;  // 16 or 32 KB each
    static constexpr int kStageBytes = DB * kBlockBytes;
    static constexpr int kQBytes = 2 * kStageBytes;
};

// What the other roles need to know of an item, left by the loaders.  The record of item n takes the place of item n - 4's
// once the queries' place of item n - 1 is free.  A half without rows gives that place back at once, so only its softmax
// group's last arrival orders the group's read of a record before the writing of the next one in its place.
struct TileInfo {
    int64_t q0, work;       // first query row of the segment; number of the item
    int kvh, split, row0, rows, last;
};

struct TileShared {
    uint64_t full[8], empty[8];
    uint64_t q_full, q_empty, done[2];
    uint64_t s_full[2][2], p_full[2][2], pv_done[2][2], o_empty[2];  // [half][turn & 1]: see below
    int meta[16];         // per key tile, by the loaders: visible keys | last << 16
    int half_meta[2][4];  // per half and turn, by the issuing warp: keys | kLast | item << kItemShift | kStop
    TileInfo info[4];
    uint32_t tmem;
    int list[kLoadWarps][kListInts];
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
__device__ __forceinline__ void halves_of(unsigned long long v, float& x, float& y) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
}
__device__ __forceinline__ unsigned long long pair_of(float v) { return f32x2(v, v); }

// Weights of 32 scores: 2^(s * scale + minus), packed in the type of the values, and their sum (of the unrounded ones).
// (A polynomial on the multiply-add pipe for every fourth pair, to relieve the special-function unit, cost more issue
// slots than it freed: 2230 -> 2325 us over 64 segments of 1024 queries and 4096 keys, 16 heads of 128.)
template <typename T>
__device__ __forceinline__ void weigh(const uint32_t* s, unsigned long long scale, unsigned long long minus, uint32_t* p,
                                      unsigned long long& sum) {
    // (All exponents, then all exponentials, then sums and weights: left to itself the compiler went through pairs one
    // after the other and waited for each: crops of 32 frames, heads of 128 1637 -> 1589 us at 1965 MHz; heads of 64 the same.)
    float e[32];
#pragma unroll
    for (int i = 0; i < 16; ++i)
        halves_of(fma_f32x2(f32x2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), scale, minus), e[2 * i], e[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("ex2.approx.ftz.f32 %0, %0;" : "+f"(e[i]));
    unsigned long long odd = 0ull;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        if (i & 1) odd = add_f32x2(odd, f32x2(e[2 * i], e[2 * i + 1]));
        else sum = add_f32x2(sum, f32x2(e[2 * i], e[2 * i + 1]));
        p[i] = pack2<T>(e[2 * i], e[2 * i + 1]);  // what the matrix instruction takes
    }
    sum = add_f32x2(sum, odd);
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

// One wait of a role.  A wait that runs out is reported; the role then leaves, and so do the others in turn.  2^23 polls are 17 s
// or more.  What takes longest in a call that works is looking through hidden keys: 5 s for the 2^30 that there can be,
// during which all other roles wait.  (Asking the loaders for signs of life instead cost 5 % of every call.)
constexpr int kTilePolls = 1 << 23;
__device__ __forceinline__ bool tile_wait(uint64_t* bar, uint32_t parity, unsigned int* status) {
#pragma unroll 1  // (the loops of five roles were a third of the kernel's code)
    for (int i = 0; i < kTilePolls; ++i)
        if (mbar_try_wait(bar, parity)) return true;
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
#pragma unroll 1
        while (in_flight > 0) arrive_oldest();
    }
    // Whoever waits hands over what has landed first: the wait may be for a consumer of just that.
    __device__ __forceinline__ void wait(uint64_t* bar, uint32_t parity) {
        if (__all_sync(0xffffffffu, mbar_test_wait(bar, parity))) return;
        flush();
        if (!__all_sync(0xffffffffu, tile_wait(bar, parity, status))) dead = true;
    }

    // The warps take groups of 8 rows in turn, kRowsAtOnce rows per instruction; the swizzle of a lane's row inside
    // its group, and so its place in shared memory, is the same for every group.
    static constexpr int kLanesPerRow = 8 * DB, kRowsAtOnce = 32 / kLanesPerRow, kTurns = 8 / kRowsAtOnce;
    static constexpr int kGroups = 16 / kLoadWarps, kOwn = kGroups * kTurns;  // groups of a warp, rows of a lane
    uint32_t place[kTurns];  // of the lane's piece of row kRowsAtOnce * i + its own in a group
    bool wide;               // the lane's piece lies inside the head
    __device__ __forceinline__ int own() const { return lane / kLanesPerRow; }
    __device__ __forceinline__ int column() const { return lane & (kLanesPerRow - 1); }
    __device__ __forceinline__ void layout(int dim_bytes) {
        wide = column() * 16 < dim_bytes;
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int r = kRowsAtOnce * i + own();
            place[i] = (uint32_t)(column() >> 3) * kBlockBytes + (uint32_t)r * 128u + (uint32_t)(((column() & 7) ^ r) << 4);
        }
    }
    // The lane's rows of a tile of 128: row(j) for j < kOwn.
    __device__ __forceinline__ int row(int j) const { return 8 * (warp + kLoadWarps * (j / kTurns)) + kRowsAtOnce * (j % kTurns) + own(); }
    // One tile: key(r) is the row of `src` that row r of the tile holds, r < take; zeros from there on.
    template <typename F>
    __device__ __forceinline__ void tile(uint32_t dst, int take, const char* src, int stride, F key) {
        src += column() * 16;
        const int groups = (max(16, (take + 15) & ~15)) >> 3;  // that the matrix instructions read
#pragma unroll 1
        for (int b = 0; b < kOwn; b += 8) {
            if (warp + kLoadWarps * (b / kTurns) >= groups) break;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int g = warp + kLoadWarps * ((b + i) / kTurns), r = row(b + i);
                const bool take_it = wide && r < take && OCTO_TOKEN_IN_RANGE(key(r) >= 0 && key(r) < end, status);
                const char* const p = take_it ? src + (int64_t)key(r) * stride : zero_row;
                if (g < groups) cp_async16(dst + (uint32_t)g * 1024u + place[i % kTurns], p, take_it);
            }
        }
    }
    // 128 rows that lie side by side from `src` on.
    __device__ __forceinline__ void full_tile(uint32_t dst, const char* src, int stride) {
        const char* p = wide ? src + (int64_t)(8 * warp + own()) * stride + column() * 16 : zero_row;
        const int64_t turn = wide ? (int64_t)kRowsAtOnce * stride : 0, group = wide ? (int64_t)(8 * kLoadWarps) * stride : 0;
        uint32_t at = dst + (uint32_t)warp * 1024u;
#pragma unroll 4
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
            for (int i = 0; i < kTurns; ++i) cp_async16(at + place[i], p + i * turn, wide);
            p += group;
            at += kLoadWarps * 1024u;
        }
    }
    // The queries' tile; at(r) gives a row's address, or null for zeros.
    template <typename F>
    __device__ __forceinline__ void queries(uint32_t dst, F at) {
#pragma unroll 4
        for (int j = 0; j < kOwn; ++j) {
            const char* p = at(row(j));
            const bool take = wide && p != nullptr;
            cp_async16(dst + (uint32_t)(warp + kLoadWarps * (j / kTurns)) * 1024u + place[j % kTurns], take ? p + column() * 16 : zero_row, take);
        }
    }
    const char* zero_row;  // any valid address
    int end;               // key rows of the segment
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
            mbar_init(&sh->empty[i], 2);
        }
        mbar_init(&sh->q_full, kLoaders);
        mbar_init(&sh->q_empty, 2);
        mbar_init(&sh->done[0], 1);
        mbar_init(&sh->done[1], 1);
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
        asm volatile("setmaxnreg.inc.sync.aligned.u32 144;");
        const int h = warp >> 2, row = threadIdx.x & (kHalf - 1);
        const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);  // the warp's 32 lanes of tensor memory
        const uint32_t o_at = lanes + 256u + 128u * h;
        const float sc = a.scale_log2;
        const int o_chunks = (a.dim + 31) >> 5;
        uint32_t turn = 0;  // turns so far; the scores of turn n are in buffer n & 1
        const unsigned long long sc2 = pair_of(sc);
        int64_t done_work = -1;
        bool dead = false;
        for (;;) {
            float ref = -INFINITY, sum = 0.0f;  // what the exponents are taken against; sum of the weights
            bool look = true;    // the scores have to be looked through before they are weighed
            bool first = true;
            int meta = 0;
            TileInfo it = {};
            uint32_t s0[32], s1[32], p[32];
            while (!(meta & (kLast | kStop))) {
                if (!__all_sync(0xffffffffu, tile_wait(&sh->s_full[h][turn & 1], (turn >> 1) & 1, a.status))) {
                    dead = true;
                    break;
                }
                tmem_after_sync();
                meta = sh->half_meta[h][turn & 3];
                if (meta & kStop) break;
                if (first && h == 1) {  // (see kStagger)
                    const long long began = clock64();
                    while (clock64() - began < kStagger) {
                    }
                }
                const int take = meta & 0xff;
                const uint32_t s_at = lanes + 128u * h + 64u * (turn & 1);
                unsigned long long part = 0ull;
                bool again = look || take < kSub;
                if (!again) {
                    // Weights against the reference so far: the exponentials do not wait for a maximum.
                    const unsigned long long minus = pair_of(-ref);
                    tmem_ld32(s_at, s0);
                    tmem_landed(s0);
                    tmem_ld32(s_at + 32, s1);
                    weigh<T>(s0, sc2, minus, p, part);
                    tmem_landed(s1);
                    weigh<T>(s1, sc2, minus, p + 16, part);
                    float x, y;
                    halves_of(part, x, y);
                    // A weight far above the reference shows in the sum (false for NaN: it comes through the weights).
                    again = __any_sync(0xffffffffu, x + y > kMostInTurn);
                }
                if (again) {
                    // The first turn, the last one where it is not full, and turns in which a row has outgrown its reference: the
                    // scores, still in tensor memory, are looked through, the reference follows, and they are weighed.
                    const uint32_t none = __float_as_uint(sc < 0.0f ? INFINITY : -INFINITY);  // behind the last visible key
                    float top = -INFINITY;
                    tmem_ld32(s_at, s0);
                    tmem_landed(s0);
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        if (i >= take) s0[i] = none;
                        else top = fmaxf(top, __uint_as_float(s0[i]) * sc);
                    }
                    if (take > 32) {
                        tmem_ld32(s_at + 32, s1);
                        tmem_landed(s1);
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            if (32 + i >= take) s1[i] = none;
                            else top = fmaxf(top, __uint_as_float(s1[i]) * sc);
                        }
                    }
                    const bool grown = top > ref + kGrown || (ref == -INFINITY && top > -INFINITY);
                    if (__any_sync(0xffffffffu, grown)) {
                        const float now = fmaxf(ref, top);
                        const float f = now == -INFINITY ? 1.0f : ex2(ref - now);
                        sum *= f;
                        ref = now;
                        if (!first) {  // (of the products, all but the last turn's are complete: the scores came after them)
                            if (!__all_sync(0xffffffffu, tile_wait(&sh->pv_done[h][(turn - 1) & 1], ((turn - 1) >> 1) & 1, a.status))) dead = true;
                            tmem_after_sync();
#pragma unroll 1
                            for (int c = 0; c < o_chunks; ++c) {
                                tmem_ld32(o_at + 32 * c, p);
                                tmem_landed(p);
#pragma unroll
                                for (int i = 0; i < 32; ++i) p[i] = __float_as_uint(__uint_as_float(p[i]) * f);
                                tmem_st32(o_at + 32 * c, p);
                            }
                        }
                    }
                    look = __any_sync(0xffffffffu, ref == -INFINITY);
                    const unsigned long long minus = pair_of(ref == -INFINITY ? 0.0f : -ref);
                    part = 0ull;
                    weigh<T>(s0, sc2, minus, p, part);
                    if (take > 32) {
                        weigh<T>(s1, sc2, minus, p + 16, part);
                    } else {  // (the matrix instruction reads the first 32 weights then)
#pragma unroll
                        for (int i = 16; i < 32; ++i) p[i] = 0u;
                    }
                }
                first = false;
                tmem_st32(s_at, p);
                float x, y;
                halves_of(part, x, y);
                sum += x + y;
                tmem_wait_st();
                tmem_before_sync();
                // (before the arrival: from there on the record's place may be written again, see TileInfo)
                if (meta & kLast) it = sh->info[OCTO_TOKEN_IN_RANGE((unsigned)(meta >> kItemShift) < 4u, a.status) ? meta >> kItemShift : 0];
                mbar_arrive(&sh->p_full[h][turn & 1]);
                ++turn;
            }
            if (dead || (meta & kStop)) break;
            // the half's rows of the result
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
                    real[k] = r < end && OCTO_TOKEN_IN_RANGE(it.q0 >= 0 && it.q0 + qrow < a.q_total && head < a.heads, a.status);
                    row_out[k] = static_cast<T*>(a.out) + (it.q0 + qrow) * a.o_row + head * a.o_head + 8 * (lane & 3);
                }
#pragma unroll 1
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
#pragma unroll 1
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
#pragma unroll 1
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
#pragma unroll 1
                for (int d = 0; it.last && d < a.dim; d += 2) *reinterpret_cast<uint32_t*>(out + d) = pack2<T>(nan, nan);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 112;");
        if (warp < 10) {
            // ---------------- matrix instructions of one half ----------------
            // The whole warp walks through the loop and one elected lane issues, so that descriptors and addresses are the
            // warp's and stay in uniform registers.
            const int h = warp - 8;
            const int ksteps = (a.dim + 15) >> 4;
            const uint32_t idesc_pv = instr_desc<T>(16 * ksteps, true), idesc_qk = instr_desc<T>(0, false);
            const uint32_t s_at = tmem + 128u * h, o_at = tmem + 256u + 128u * h;
            const uint32_t qa = desc_low(q_base + h * Shape::kStageBytes, 0);
            uint32_t slot = 0, tile = 0, items = 0;             // ring slots, key tiles and items so far
            uint32_t turns = 0, weights = 0, half_items = 0;    // scores issued, weights used, items with rows in this half
            bool ok = true;
            auto wait = [&](uint64_t* bar, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, tile_wait(bar, parity, a.status)); };
            auto commit = [&](uint64_t* bar) {
                if (elect_one()) mma_commit(bar);
                __syncwarp();
            };
            auto full_wait = [&](uint32_t n) { wait(&sh->full[n % Shape::kStages], (n / Shape::kStages) & 1); };
            auto slot_at = [&](uint32_t n) { return ring + (n % Shape::kStages) * Shape::kStageBytes; };
            auto next_meta = [&]() { return __shfl_sync(0xffffffffu, sh->meta[tile++ & 15], 0); };
            for (;;) {
                wait(&sh->q_full, items & 1);
                if (!ok) break;
                const int rows = __shfl_sync(0xffffffffu, sh->info[items & 3].rows, 0), tag = (int)(items & 3) << kItemShift;
                if (rows == 0) break;  // no more items
                ++items;
                if (rows <= h * kHalf) {  // nothing in this half: only give the places back
                    if (elect_one()) mbar_arrive(&sh->q_empty);
                    for (bool last = false; !last;) {
                        full_wait(slot);
                        if (!ok) break;
                        last = next_meta() >> 16;
                        if (elect_one()) mbar_arrive(&sh->empty[slot % Shape::kStages]);
                        // (not before it is full: the arrival could count for the tile that lies there still)
                        full_wait(slot + 1);
                        if (!ok) break;
                        if (elect_one()) mbar_arrive(&sh->empty[(slot + 1) % Shape::kStages]);
                        __syncwarp();
                        slot += 2;
                    }
                    if (!ok) break;
                    continue;
                }
                // The turns of the item in order; scores run two turns ahead of products, into the buffer that the products
                // before them have just read.  From the arrival of a turn's weights to the next scores nothing is
                // waited for: places of keys and values are seen to while the softmax works.
                struct Turn {
                    uint32_t k;       // descriptor of its keys
                    uint32_t slot;    // of its keys; the values follow
                    int sub, keys;
                    bool frees, last; // the tile's last turn; the item's
                };
                uint32_t k_slot = slot;
                int k_meta = 0, k_sub = 0;
                auto prepare = [&](Turn& t) {
                    if (k_sub == 0) {
                        full_wait(k_slot);
                        if (!ok) return;
                        k_meta = next_meta();
                    }
                    const int left = (k_meta & 0xffff) - kSub * k_sub;
                    t.k = desc_low(slot_at(k_slot) + 8192u * k_sub, 0);
                    t.slot = k_slot;
                    t.sub = k_sub;
                    t.keys = min(left, kSub);
                    t.frees = left <= kSub;
                    t.last = t.frees && (k_meta >> 16);
                    k_sub = t.frees ? 0 : k_sub + 1;
                    if (t.frees) k_slot += 2;
                };
                auto scores = [&](const Turn& t) {  // S = Q K^T, by the elected lane
                    const uint32_t idesc = idesc_qk + ((uint32_t)(max(16, (t.keys + 15) & ~15) >> 3) << 17), d = s_at + 64u * (turns & 1);
#pragma unroll
                    for (int k = 0; k < 4 * DB; ++k) {
                        const uint32_t off = ((uint32_t)(k >> 2) * kBlockBytes + (uint32_t)(k & 3) * 32u) >> 4;
                        if (k < ksteps) mma_ss(d, desc_of(qa + off), desc_of(t.k + off), idesc, k > 0);
                    }
                    sh->half_meta[h][turns & 3] = t.keys | (t.last ? kLast : 0) | tag;
                    mma_commit(&sh->s_full[h][turns & 1]);
                    mbar_arrive(&sh->s_full[h][turns & 1]);
                    if (t.frees) mma_commit(&sh->empty[t.slot % Shape::kStages]);
                    if (t.last) mma_commit(&sh->q_empty);
                };
                Turn now, next, after;
                prepare(now);
                if (!ok) break;
                tmem_after_sync();
                if (elect_one()) scores(now);
                __syncwarp();
                ++turns;
                next = now;
                if (!now.last) {
                    prepare(next);
                    if (!ok) break;
                    if (elect_one()) scores(next);
                    __syncwarp();
                    ++turns;
                }
                for (bool start = true;; start = false) {
                    const bool more = !now.last && !next.last;
                    after = next;
                    if (more) prepare(after);
                    if (now.sub == 0) full_wait(now.slot + 1);
                    if (start) wait(&sh->o_empty[h], (half_items & 1) ^ 1);
                    const uint32_t va = desc_low(slot_at(now.slot + 1) + 8192u * now.sub, kBlockBytes), pa = s_at + 64u * (weights & 1);
                    const int steps = max(1, (now.keys + 15) >> 4);
                    wait(&sh->p_full[h][weights & 1], (weights >> 1) & 1);
                    if (!ok) break;
                    tmem_after_sync();
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)  // O += P V
                            if (k < steps) mma_ts(o_at, pa + 8u * k, desc_of(va + 128u * k), idesc_pv, !start || k > 0);
                        mma_commit(&sh->pv_done[h][weights & 1]);
                        if (now.frees) mma_commit(&sh->empty[(now.slot + 1) % Shape::kStages]);
                        if (more) scores(after);
                    }
                    __syncwarp();
                    ++weights;
                    if (more) ++turns;
                    if (now.last) break;
                    now = next;
                    next = after;
                }
                if (!ok) break;
                slot = k_slot;
                ++half_items;
            }
            if (ok) {  // the softmax group may leave
                if (elect_one()) {
                    sh->half_meta[h][turns & 3] = kStop;
                    mbar_arrive(&sh->s_full[h][turns & 1]);
                    mbar_arrive(&sh->s_full[h][turns & 1]);
                }
                __syncwarp();
            }
            commit(&sh->done[h]);  // nothing of this CTA is under way when it gives its memory back
            tile_wait(&sh->done[h], 0, a.status);
        } else if (warp < 10 + kLoadWarps) {
            // ---------------- loads ----------------
            Loader<DB> ld;
            ld.status = a.status;
            ld.lane = lane;
            ld.warp = warp - 10;
            ld.zero_row = static_cast<const char*>(a.q);
            int* const list = sh->list[warp - 10];
            ld.layout(2 * a.dim);
            uint32_t items = 0, tile = 0;
            for (int64_t w = blockIdx.x; w < total && !ld.dead; w += gridDim.x) {
                TileItem it;
                if (!tile_item(a, prefix, tiles_per_segment, w, it)) continue;
                // the queries follow the first keys and values: their place is free only when the last item's scores are made
                auto load_queries = [&]() {
                    ld.wait(&sh->q_empty, (items & 1) ^ 1);
                    if (ld.dead) return;
                    const int row = (int)(2 * a.q_row), head = (int)(2 * a.q_head);
                    const char* const q = static_cast<const char*>(a.q) + it.seg.q0 * 2 * a.q_row + (int64_t)it.kvh * a.group * 2 * a.q_head;
                    for (int b = 0; b < it.rows; b += kHalf)
                        ld.queries(q_base + (b / kHalf) * Shape::kStageBytes, [&](int r) -> const char* {
                            int qrow, hd;
                            tile_row(a, 0, it.row0 + b + r, qrow, hd);
                            if (!OCTO_TOKEN_IN_RANGE(b + r >= it.rows || (it.seg.q0 + qrow < a.q_total && hd < a.group), a.status)) return nullptr;
                            return b + r < it.rows ? q + (int64_t)qrow * row + (int64_t)hd * head : nullptr;
                        });
                    if (warp == 10 && lane == 0) {
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
                ld.end = OCTO_TOKEN_IN_RANGE(it.seg.k0 >= 0 && it.seg.k0 + it.ke <= a.k_total && it.kvh < a.kv_heads, a.status) ? it.ke : 0;
                const char* const k = reinterpret_cast<const char*>(static_cast<const T*>(a.k) + it.seg.k0 * a.k_row + it.kvh * a.k_head);
                const char* const v = reinterpret_cast<const char*>(static_cast<const T*>(a.v) + it.seg.k0 * a.v_row + it.kvh * a.v_head);
                const uint8_t* const mask = a.mask ? a.mask + it.seg.k0 : nullptr;
                int cursor = it.kb, listed = 0;
                bool seen[4];  // of the 128 keys from the cursor on, fetched ahead
                auto look_ahead = [&]() {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = cursor + 32 * j + lane;
                        seen[j] = key < it.ke && mask[key] != 0;
                    }
                };
                if (mask) look_ahead();
                for (bool last = false; !last && !ld.dead; ++tile) {
                    // The next 128 visible keys: those that are listed, and then the keys that follow without a gap where there
                    // are enough of them (the states of a frame between its canvas bands); else the list is filled up.
                    int take, from = cursor, kept = 0;  // rows below `kept` from the list, the others from `from` on
                    if (mask) {
                        bool gapless = false;
                        while (listed <= kHalf) {
                            unsigned ballot[4];
                            bool all = true;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                ballot[j] = __ballot_sync(0xffffffffu, seen[j]);
                                const int wanted = min(max(kHalf - listed - 32 * j, 0), 32);  // of these 32
                                const unsigned those = wanted == 32 ? 0xffffffffu : (1u << wanted) - 1u;
                                all = all && (ballot[j] & those) == those;
                            }
                            gapless = all && listed < kHalf;
                            if (gapless || cursor >= it.ke) break;
                            const int hidden = ballot[0] ? __ffs(ballot[0]) - 1 : 32;
                            if (listed == 0 && hidden > 0) {  // begin at a visible key
                                cursor += ballot[0] | ballot[1] | ballot[2] | ballot[3] ? hidden : 128;
                            } else {  // (at most 128 are listed here, and 128 more fit)
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    if (seen[j]) list[listed + __popc(ballot[j] & ((1u << lane) - 1u))] = cursor + 32 * j + lane;
                                    listed += __popc(ballot[j]);
                                }
                                cursor += 128;
                            }
                            look_ahead();
                        }
                        __syncwarp();
                        kept = gapless ? listed : kHalf;
                        take = gapless ? kHalf : min(listed, kHalf);
                        from = cursor;
                        if (gapless) {  // is there any key left?
                            cursor += kHalf - listed;
                            look_ahead();
                            while (!__any_sync(0xffffffffu, seen[0] || seen[1] || seen[2] || seen[3]) && cursor < it.ke) {
                                cursor += 128;
                                look_ahead();
                            }
                            last = cursor >= it.ke;
                            listed = take;  // (none is left over)
                        } else {
                            last = listed <= kHalf;
                        }
                    } else {
                        take = min(it.ke - cursor, kHalf);
                        cursor += take;
                        last = cursor >= it.ke;
                    }
                    if (warp == 10 && lane == 0) sh->meta[tile & 15] = take | (last ? 1 << 16 : 0);
#pragma unroll 1
                    for (int which = 0; which < 2; ++which) {
                        const uint32_t n = ld.slot;
                        ld.wait(&sh->empty[n % Shape::kStages], ((n / Shape::kStages) & 1) ^ 1);
                        if (ld.dead) break;
                        const char* const src = which ? v : k;
                        const int stride = (int)(2 * (which ? a.v_row : a.k_row));
                        const uint32_t dst = ring + (n % Shape::kStages) * Shape::kStageBytes;
                        if (mask && kept > 0) ld.tile(dst, take, src, stride, [&](int r) { return r < kept ? list[r] : from + r - kept; });
                        else if (take == kHalf && OCTO_TOKEN_IN_RANGE(from >= 0 && from + kHalf <= it.ke, a.status)) ld.full_tile(dst, src + (int64_t)from * stride, stride);
                        else ld.tile(dst, take, src, stride, [&](int r) { return from + r; });
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
                if (warp == 10 && lane == 0) sh->info[items & 3].rows = 0;
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
