// Matrix products on the fifth-generation tensor cores (skew_product.h): a persistent kernel whose warps bring operands, multiply (one thread)
// and write out at the same time. A pair of CTAs shares a tile of 256 x 256: each holds half of either operand and gets the sums of its rows.
//
// A CTA brings 128 lines of A and 128 of B, 64 elements of each at a time (a stage of 32 KiB, in a ring of six), to shared
// memory in 128-byte rows whose 16-byte units are permuted by the row's number (unit u of row L lies at u ^ (L & 7)), which is the layout that
// tcgen05.mma reads without bank conflicts. The same layout serves both orders of an operand: lines along the summed index
// ("K-major"), or 64 steps of the summed index, each a line along the tile ("MN-major"), 64 columns to a block of 8 KiB. Lines on 16-byte boundaries come by tensor
// copies that one thread asks for, others by eight warps (Loose), an operand at a time.
// Sums stay in tensor memory in fp32, in two halves: the next tile is multiplied into one while the other is written out.
//
// Rows of the group behind this one, which a tile's last lines may hold, cost nothing: a row of C has its own row of A (or, in a turned tile, column of its
// own). Where the rows are summed over (OUTER) they are zeros in shared memory, so that nothing of another group, NaN included, enters.
//
// What bounds it. At the tensor cores' rate a CTA takes 64 bytes a clock from L2, as many as it can, and reads as many from shared memory, so that this is busy
// throughout: 8192 x 4096 times 4096 x 16384 runs at 1.80 PFLOP/s in bursts (574 us without the logits' sums, 611 with; the library's product 2.05) and at what the power
// limit leaves in a row (1.66). Tiles of few steps are bound by what becomes of their sums, some 3000 to 5500 clocks a tile; a tile of 512 rows to an expert
// takes 4096 to multiply (the gradient of 128 matrices of 4096 x 4096 from 512 rows each: 1.52 ms in bursts, 1.19 without writing out).
#include "skew_product.h"

#include <cuda.h>

#include <atomic>

#include "skew_lines.h"
#include "skew_ops.h"

namespace skew {
namespace {

constexpr int kLines = kOperandLines;
constexpr int kStep = 64;                      // elements of the summed index in a stage
constexpr uint32_t kOperandBytes = kLines * kStep * 2;
constexpr uint32_t kStageBytes = 2 * kOperandBytes;
constexpr int kStages = 6;                     // 5 where there are many groups
constexpr int kMaxGroups = 1024;
constexpr int kBandRows = 2048;                // rows of tiles that are walked together (what 152 SMs have under way then stays in L2)

constexpr int kTile = 256;                     // rows and columns of a tile, which a pair of CTAs shares

constexpr int kMulWarp = 0, kMemWarp = 1, kCopyWarp = 2, kCutWarp = 3, kFirstEnd = 4;  // of the warps from 4 on, each reads lanes 32 (warp % 4) on of tensor memory
constexpr int kEndWarps = 8, kEndCols = kTile * 4 / kEndWarps, kFirstLoad = kFirstEnd + kEndWarps, kLoadWarps = 8;

// How an operand lies in its lines: along the summed index, or across it.
template <int KIND>
constexpr bool kMajorA = KIND != kOuter && KIND != kGroupRows;
template <int KIND>
constexpr bool kMajorB = KIND != kOuter && KIND != kByRows;
// The tile's rows are the matrices' columns, and its columns the group's rows.
template <int KIND>
constexpr bool kTurned = KIND == kGroupRows || KIND == kGroupCols;
constexpr int kRowBox = 32;                    // lines of a copy of a group's rows where they do not fill a tile (one of 128 is 8 % quicker where they do)

// COPY: the operands (1: A, 2: B) whose stages come by tensor copies, which one thread asks for. Eight more warps load the others.
constexpr int kCopyA = 1, kCopyB = 2;
template <int COPY>
constexpr int kThreads = 32 * (kFirstLoad + (COPY == 3 ? 0 : kLoadWarps));

struct Shared {
    uint64_t full[kStages], empty[kStages], landed[kStages], sums[2], freed[2];
    uint32_t acc;                     // where the sums are in tensor memory
    uint32_t gave_up;
    uint32_t asked;                   // OUTER: stages that copies were asked for
    int32_t total[32];
    int32_t begin[1];                 // [groups + 1]: first row of each group, and the end of the last; then
                                      // [groups + 1]: tiles of rows before it (BY_ROWS, BY_COLS)
};

constexpr int kOutBytes = 32 * 128;            // 32 rows of 128 bytes, of each warp that writes out
constexpr size_t kMaxSharedBytes = 232448;
constexpr size_t shared_bytes(int stages, size_t raw, int groups) {
    return 1024 + size_t(stages) * kStageBytes + raw + size_t(kEndWarps) * kOutBytes + sizeof(Shared) + size_t(groups + 1) * 8;
}
// Stages that loaded lines are on their way for, and the stages of the ring beside them.
template <int COPY>
constexpr int kRawStages = COPY ? 4 : 3;
template <int COPY>
constexpr int kRing = COPY == 3 ? kStages : COPY ? 3 : 2;
template <int COPY>
constexpr size_t kRawBytes = COPY == 3 ? 0 : size_t(kRawStages<COPY>) * (COPY ? 1 : 2) * kLines * kRawLine;
static_assert(shared_bytes(kStages - 1, 0, kMaxGroups) <= kMaxSharedBytes && shared_bytes(kRing<1>, kRawBytes<1>, kMaxGroups) <= kMaxSharedBytes &&
              shared_bytes(kRing<0>, kRawBytes<0>, kMaxGroups) <= kMaxSharedBytes, "shared memory of a CTA");

// A place in the ring of stages, and how often it was there before (odd or even).
struct Place {
    uint32_t s = 0, phase = 0;
    __device__ __forceinline__ void next(uint32_t stages) {
        if (++s == stages) s = 0, phase ^= 1;
    }
};

__device__ uint32_t g_status;  // 1: a wait gave up

__device__ __forceinline__ uint32_t shared_address(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void bar_init(uint64_t *b, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(b)), "r"(count) : "memory");
}

// The address of `p` in the pair's first CTA.
__device__ __forceinline__ uint32_t in_first(const void *p) {
    uint32_t a = shared_address(p);
    asm("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(a));
    return a;
}

__device__ __forceinline__ void bar_arrive(uint64_t *b) {  // the first CTA's
    // (Scope cta: what is handed over lies in shared or tensor memory, and goes by the proxies' own fences. At cluster scope the release waits for this
    // thread's stores to memory.)
    asm volatile("mbarrier.arrive.release.cta.shared::cluster.b64 _, [%0];" ::"r"(in_first(b)) : "memory");
}

// Arrives at a barrier of this address, which then also waits for `bytes`. (Relaxed: nothing that this thread wrote is read after it. A release
// waits for what is under way, copies among it: 0.6 us a stage.)
__device__ __forceinline__ void bar_expect(uint32_t address, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(address), "r"(bytes) : "memory");
}

__device__ __forceinline__ bool bar_poll(uint64_t *b, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(shared_address(b)), "r"(parity), "n"(2000) : "memory");
    return ok != 0;
}

// False once this or another of the CTA's waits has given up, after some four seconds: the kernel then ends as it stands and
// leaves its mark for skew_ops_sync_status. A wait that may be for much later, at any step of the work before it, is given a count of those steps: its four
// seconds start anew with each.
__device__ __forceinline__ bool bar_wait(uint64_t *b, uint32_t parity, Shared &S, const uint32_t *progress = nullptr) {
    if (bar_poll(b, parity)) return true;
    uint32_t seen = 0;
    for (uint32_t i = 0; i < 1u << 20; ++i) {
        if (bar_poll(b, parity)) return true;
        if (*reinterpret_cast<volatile uint32_t *>(&S.gave_up)) return false;
        if (!progress) continue;
        const uint32_t now = *reinterpret_cast<const volatile uint32_t *>(progress);
        if (now != seen) seen = now, i = 0;
    }
    *reinterpret_cast<volatile uint32_t *>(&S.gave_up) = 1;
    atomicOr(&g_status, 1u);
    return false;
}

// One lane waits for its warp.
__device__ __forceinline__ bool warp_wait(uint64_t *b, uint32_t parity, Shared &S, const uint32_t *progress = nullptr) {
    bool ok = true;
    if ((threadIdx.x & 31) == 0) ok = bar_wait(b, parity, S, progress);
    return __shfl_sync(kFullMask, ok, 0);
}

__device__ __forceinline__ void drain(uint64_t *b, uint32_t parity) {
    for (int i = 0; i < 1 << 20 && !bar_poll(b, parity); ++i) {}
}

__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---------------------------------------------------------------------------
// Tiles
// ---------------------------------------------------------------------------
struct Tile {
    int32_t group, m0, n0;        // first row (of the matrices' `rows`, or OUTER's i) and column
    int32_t r0, r1;               // the group's rows
    int32_t k0, steps;            // of the summed index: the first, and how many
    int32_t unit;                 // of the tile and its share of the summed index, where that is split
    bool ends;                    // the share's last step is the group's
    // GROUP: columns of the tile, which the products take 64 at a time
    __device__ __forceinline__ int width() const { return min(kTile, (r1 - m0 + 63) / 64 * 64); }
};

__device__ __forceinline__ int32_t *tiles_of(const ProductArgs &A, Shared &S) { return S.begin + A.groups + 1; }

// The groups' rows, in order and within [0, rows) whatever `offsets` hold, and the tiles before each.
template <int KIND, int THREADS>
__device__ __forceinline__ void groups_of(const ProductArgs &A, Shared &S) {
    const int G = A.groups, per = (G + THREADS) / THREADS, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rows = int(A.rows);
    if (!A.offsets) {
        if (threadIdx.x == 0) {
            int32_t *const tile = tiles_of(A, S);
            S.begin[0] = tile[0] = 0;
            S.begin[1] = rows;
            tile[1] = (rows + kTile - 1) / kTile;
        }
        __syncthreads();
        return;
    }
    const int i0 = threadIdx.x * per, i1 = min(i0 + per, G + 1);
    auto scan = [&](int v, auto join) {  // what the threads before this one have together; -1 for none
        int x = v;
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(kFullMask, x, d);
            if (lane >= d) x = join(x, y);
        }
        __syncthreads();
        if (lane == 31) S.total[warp] = x;
        __syncthreads();
        int before = __shfl_up_sync(kFullMask, x, 1);
        if (!lane) before = 0;
        for (int w = 0; w < warp; ++w) before = join(before, S.total[w]);
        return before;
    };
    auto most = [](int a, int b) { return max(a, b); };
    auto both = [](int a, int b) { return a + b; };
    auto at = [&](int i) { return min(max(A.offsets[i], 0), rows); };
    int m = 0;
    for (int i = i0; i < i1; ++i) m = max(m, at(i));
    m = scan(m, most);
    for (int i = i0; i < i1; ++i) S.begin[i] = m = max(m, at(i));
    __syncthreads();
    if (KIND != kOuter) {
        int32_t *const tile = tiles_of(A, S);
        auto tiles = [&](int i) { return i < G ? (S.begin[i + 1] - S.begin[i] + kTile - 1) / kTile : 0; };
        int n = 0;
        for (int i = i0; i < i1; ++i) n += tiles(i);
        n = scan(n, both);
        for (int i = i0; i < i1; ++i) tile[i] = n, n += tiles(i);
    }
    __syncthreads();
}

// The pair's tiles, one after another: its own number, + the pairs, ... (Their number fits 31 bits: launch_of sees to it.) A whole warp walks: each lane works
// out one of the next 32 tiles, which takes four divisions.
template <int KIND>
struct Walk {
    static constexpr uint32_t kBand = kBandRows / kTile;
    const ProductArgs &A;
    const int32_t *begin, *tile;
    uint32_t at, all, nt, mt;
    Tile mine;
    int32_t ahead;     // tiles that the lanes have left

    __device__ __forceinline__ Walk(const ProductArgs &a, Shared &s) : A(a), begin(s.begin), tile(tiles_of(a, s)), at(blockIdx.x / 2), ahead(0) {
        nt = (uint32_t(A.cols) + kTile - 1) / kTile;
        mt = (uint32_t(A.inner) + kTile - 1) / kTile;
        all = (KIND == kOuter ? mt * A.groups : tile[A.groups]) * nt * A.splits;
    }

    __device__ __forceinline__ void work_out(uint32_t at) {
        uint32_t here = at, split = 0, mt = this->mt, group;
        if (A.splits > 1) here /= uint32_t(A.splits), split = at - here * A.splits;
        const uint32_t row = here / nt;  // tiles of rows before this one's, over all groups
        if (KIND == kOuter) {
            group = row / mt;
            here -= group * mt * nt;
        } else {  // its group is the last that begins at or before it
            uint32_t lo = 0, hi = A.groups;
            while (hi - lo > 1) {
                const uint32_t mid = (lo + hi) >> 1;
                if (uint32_t(tile[mid]) <= row) lo = mid; else hi = mid;
            }
            group = lo;
            here -= tile[group] * nt;
            mt = tile[group + 1] - tile[group];
        }
        const uint32_t band = here / (kBand * nt), first = band * kBand, in = min(kBand, mt - first), left = here - first * nt;
        const uint32_t n = left / in, m = first + left - n * in;
        mine.group = group;
        mine.r0 = begin[group];
        mine.r1 = begin[group + 1];
        mine.m0 = m * kTile + (KIND == kOuter ? 0 : mine.r0);
        mine.n0 = n * kTile;
        const int steps = ((KIND == kOuter ? mine.r1 - mine.r0 : A.inner) + kStep - 1) / kStep, share = A.splits > 1 ? (steps + A.splits - 1) / A.splits : steps;
        mine.k0 = split * share;
        mine.steps = max(min(share, steps - mine.k0), 0);
        mine.ends = mine.k0 + mine.steps == steps;
        mine.unit = (((KIND == kOuter ? group * mt : 0) + m) * nt + n) * A.splits + split;
    }

    __device__ __forceinline__ bool next(Tile &t) {
        if (at >= all) return false;
        const uint32_t step = gridDim.x / 2;
        if (!ahead) {
            const uint32_t lane = threadIdx.x & 31;
            if (at + uint64_t(lane) * step < all) work_out(at + lane * step);
            ahead = 32;
        }
        const int from = 32 - ahead--;
        t.group = __shfl_sync(kFullMask, mine.group, from);
        t.m0 = __shfl_sync(kFullMask, mine.m0, from);
        t.n0 = __shfl_sync(kFullMask, mine.n0, from);
        t.r0 = __shfl_sync(kFullMask, mine.r0, from);
        t.r1 = __shfl_sync(kFullMask, mine.r1, from);
        t.k0 = __shfl_sync(kFullMask, mine.k0, from);
        t.steps = __shfl_sync(kFullMask, mine.steps, from);
        t.unit = __shfl_sync(kFullMask, mine.unit, from);
        t.ends = __shfl_sync(kFullMask, int(mine.ends), from);
        at += step;
        return true;
    }
};

// ---------------------------------------------------------------------------
// Loads
// ---------------------------------------------------------------------------
// Lines that start off a 16-byte boundary, or lie an odd number of elements apart, come as the 16-byte units that hold them, by asynchronous copies, to memory of the
// warp's own (144 bytes a line), a few stages ahead; from there each unit of a stage is cut out of two of those. (A unit is read only where it holds an element
// that is there, so that no access leaves the units of the matrix itself.)
constexpr int kLooseLines = (2 * kLines) / kLoadWarps;  // of a warp, of one operand, where both are loaded; half of that of each operand's lines where one is

// Those lines (skew_lines.h), to the warp's own memory and from there to a stage.
template <bool MAJOR, int N>
struct Loose : Lines<MAJOR, N> {
    using Lines<MAJOR, N>::Lines;

    __device__ __forceinline__ void ask(uint32_t raw, const void *any, int lane) const {
        this->units(lane, [&](uint32_t to, const char *from, bool there) { copy_unit(raw + to, there ? from : any, there); });
    }

    static __device__ __forceinline__ void copy_unit(uint32_t to, const void *from, bool there) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
    }

    // To lines `from` on of the stage.
    __device__ __forceinline__ void cut(const char *raw, char *to, int from, int lane) const {
        const int c = lane % 8, have = this->n - c * 8;
        raw += lane / 8 * kRawLine + c * 16;
        uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(this->at)) & 15;
        constexpr int kDeep = 4;
#pragma unroll
        for (int i0 = 0; i0 < N / 4; i0 += kDeep) {
            uint4 a[kDeep], b[kDeep];  // (all read before the first is stored: for the compiler a store might write what the next read reads)
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                a[i] = *reinterpret_cast<const uint4 *>(raw + (i0 + i) * 4 * kRawLine);
                b[i] = *reinterpret_cast<const uint4 *>(raw + (i0 + i) * 4 * kRawLine + 16);
            }
#pragma unroll
            for (int i = 0; i < kDeep; ++i, off = (off + uint32_t(this->four)) & 15) {
                const int L = from + (i0 + i) * 4 + lane / 8;
                uint32_t w[8] = {a[i].x, a[i].y, a[i].z, a[i].w, b[i].x, b[i].y, b[i].z, b[i].w};
#pragma unroll
                for (int k = 0; k < 6; ++k) w[k] = off & 8 ? w[k + 2] : w[k];
#pragma unroll
                for (int k = 0; k < 5; ++k) w[k] = off & 4 ? w[k + 1] : w[k];
                const uint32_t turn = off & 2 ? 0x5432u : 0x3210u;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = __byte_perm(w[k], w[k + 1], turn);
                if (have < 8) {  // (what the units hold behind the line is not zeros)
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] = have >= 2 * k + 2 ? w[k] : have == 2 * k + 1 ? w[k] & 0xFFFFu : 0u;
                }
                *reinterpret_cast<uint4 *>(to + L * 128 + (c ^ (L & 7)) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
};

// A box of a tensor map, from column x, line y of group z, to shared memory at `to`; its bytes count at the barrier of this address.
__device__ __forceinline__ void copy_box(const CUtensorMap &map, uint32_t to, uint32_t bar, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(to), "l"(&map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}

// One operand's 128 lines, where Loose would put them. Beyond the matrix the boxes hold zeros.
template <bool MAJOR>
__device__ __forceinline__ void copy_lines(const CUtensorMap &map, uint32_t to, uint32_t bar, int l0, int s0, int group) {
    if constexpr (MAJOR) {
        copy_box(map, to, bar, s0, l0, group);
    } else {
        copy_box(map, to, bar, l0, s0, group);
        copy_box(map, to + kOperandBytes / 2, bar, l0 + 64, s0, group);
    }
}

// ---------------------------------------------------------------------------
// Tensor cores
// ---------------------------------------------------------------------------
// How tcgen05.mma finds an operand in shared memory. Along the summed index: groups of 8 lines, 1024 bytes apart. Across it: blocks of 64
// columns 8192 bytes apart, of groups of 8 lines 1024 bytes apart.
template <bool MAJOR>
__device__ __forceinline__ uint64_t operand(uint32_t address) {
    return uint64_t(address >> 4 & 0x3FFF) | uint64_t(MAJOR ? 1 : 8192 >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}

// 16 steps of the summed index further on: 32 bytes along lines, or 16 lines.
template <bool MAJOR>
constexpr uint32_t kNext16 = (MAJOR ? 32 : 16 * 128) >> 4;

template <bool A_MAJOR, bool B_MAJOR>
constexpr uint32_t kInstruction = 1u << 4 /* sums fp32 */ | 1u << 7 | 1u << 10 /* bf16 */ | uint32_t(!A_MAJOR) << 15 | uint32_t(!B_MAJOR) << 16 |
                                  uint32_t(kTile >> 4) << 24;  // and the tile's columns >> 3 at bit 17

// 16 steps of a tile: each CTA of the pair holds half of A's rows and of B's columns, and gets the sums of its rows.
__device__ __forceinline__ void multiply(uint32_t acc, uint64_t a, uint64_t b, uint32_t instruction, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(acc), "l"(a), "l"(b), "r"(instruction), "r"(uint32_t(add)) : "memory");
}

// Arrives, in each CTA of the pair, once what was issued before is done.
__device__ __forceinline__ void commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(shared_address(bar)), "h"(uint16_t(3)) : "memory");
}

__device__ __forceinline__ void take_tensor_memory(uint32_t *address) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(address)), "n"(2 * kTile) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void give_tensor_memory(uint32_t acc) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(acc), "n"(2 * kTile) : "memory");
}

__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 lanes, x[c] of this lane: there after sums_read.
__device__ __forceinline__ void read_sums(uint32_t at, float (&x)[32]) {
    uint32_t *u = reinterpret_cast<uint32_t *>(x);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]),
          "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]),
          "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(at) : "memory");
}

__device__ __forceinline__ void sums_read(float (&x)[32]) {  // (x: so that nothing that reads it moves before)
    uint32_t *u = reinterpret_cast<uint32_t *>(x);
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]), "+r"(u[9]), "+r"(u[10]), "+r"(u[11]),
          "+r"(u[12]), "+r"(u[13]), "+r"(u[14]), "+r"(u[15]), "+r"(u[16]), "+r"(u[17]), "+r"(u[18]), "+r"(u[19]), "+r"(u[20]), "+r"(u[21]), "+r"(u[22]),
          "+r"(u[23]), "+r"(u[24]), "+r"(u[25]), "+r"(u[26]), "+r"(u[27]), "+r"(u[28]), "+r"(u[29]), "+r"(u[30]), "+r"(u[31])
        :: "memory");
}

// ---------------------------------------------------------------------------
// What becomes of the sums
// ---------------------------------------------------------------------------
__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What a row's logits are taken off before their exponentials: an infinite one would make NaN of itself.
__device__ __forceinline__ float finite_or_0(float x) { return fabsf(x) < INFINITY ? x : 0.f; }

__device__ __forceinline__ void store16(void *p, uint4 u) {
    asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory");
}

// Where 32 rows of a warp go, in elements: of the first row and the matrix's first column, and the rows' distance.
struct Target {
    int64_t at, ldo;
    int rows;
};

// What lanes have of their rows leaves through 32 x 128 bytes of shared memory of the warp's own, 16-byte units permuted as in a stage, and from there row by row,
// so that accesses are whole 32-byte sectors (stores of the lanes' own rows took twice the time, and tensor copies of them a wait for each).

// 64 columns, from `column` on, scaled, in bf16; the rows' units are on 16-byte boundaries.
__device__ __forceinline__ void put_64(const ProductArgs &A, char *buffer, const Target &to, int column, float scale, const float (&x)[64]) {
    const int lane = threadIdx.x & 31, unit = lane % 8;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const float *y = x + u * 8;
        *reinterpret_cast<uint4 *>(buffer + lane * 128 + (u ^ (lane & 7)) * 16) = make_uint4(pack_bf16(y[0] * scale, y[1] * scale), pack_bf16(y[2] * scale, y[3] * scale),
                                                                                             pack_bf16(y[4] * scale, y[5] * scale), pack_bf16(y[6] * scale, y[7] * scale));
    }
    __syncwarp();
    uint4 y[8];  // (all read before the first is stored: for the compiler a store might write what the next read reads)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = *reinterpret_cast<const uint4 *>(buffer + (i * 4 + lane / 8) * 128 + (unit ^ ((i * 4 + lane / 8) & 7)) * 16);
    __syncwarp();
    char *out = static_cast<char *>(A.out) + (to.at + column + lane / 8 * to.ldo) * 2 + unit * 16;
    const int64_t next = to.ldo * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i, out += next)
        if (i * 4 + lane / 8 < to.rows) store16(out, y[i]);
}

// 32 columns, from `column` on, of which `n` are there: base + scale * x, in any type.
__device__ __forceinline__ void put_32(const ProductArgs &A, char *buffer, const Target &to, int column, int n, float scale, const float (&x)[32]) {
    const int lane = threadIdx.x & 31;
    const bool o32 = A.flags & kOut32, b32 = A.flags & kBase32;
#pragma unroll
    for (int u = 0; u < 8; ++u)
        *reinterpret_cast<float4 *>(buffer + lane * 128 + (u ^ (lane & 7)) * 16) = make_float4(x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]);
    __syncwarp();
    if (A.flags & kOutVec && n >= 32) {  // eight lanes to a row, four columns to a lane
        const int unit = lane % 8;
        const int64_t at = to.at + column + unit * 4;
        float4 y[8], b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + lane / 8;
            y[i] = *reinterpret_cast<const float4 *>(buffer + r * 128 + (unit ^ (r & 7)) * 16);
            b[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (!A.base || r >= to.rows) continue;
            if (b32) {
                b[i] = *reinterpret_cast<const float4 *>(elem_ptr<true>(A.base, at + r * to.ldo));
            } else {
                const uint2 u = *reinterpret_cast<const uint2 *>(elem_ptr<false>(A.base, at + r * to.ldo));
                b[i] = make_float4(bf16_low(u.x), bf16_high(u.x), bf16_low(u.y), bf16_high(u.y));
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = i * 4 + lane / 8;
            const int64_t e = at + r * to.ldo;
            const float4 z = A.base ? make_float4(fmaf(y[i].x, scale, b[i].x), fmaf(y[i].y, scale, b[i].y), fmaf(y[i].z, scale, b[i].z), fmaf(y[i].w, scale, b[i].w))
                                    : make_float4(y[i].x * scale, y[i].y * scale, y[i].z * scale, y[i].w * scale);
            if (r >= to.rows) continue;
            if (o32) store16(static_cast<float *>(A.out) + e, make_uint4(__float_as_uint(z.x), __float_as_uint(z.y), __float_as_uint(z.z), __float_as_uint(z.w)));
            else *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(A.out) + e) = make_uint2(pack_bf16(z.x, z.y), pack_bf16(z.z, z.w));
        }
    } else {  // a row at a time, a column to a lane
        const int64_t at = to.at + column + lane;
        constexpr int kDeep = 16;
        for (int r0 = 0; r0 < to.rows; r0 += kDeep) {
            float b[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                b[i] = 0.f;
                if (!A.base || lane >= n || r0 + i >= to.rows) continue;
                b[i] = b32 ? load1<true>(A.base, at + (r0 + i) * to.ldo) : load1<false>(A.base, at + (r0 + i) * to.ldo);
            }
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                const int r = r0 + i;
                if (lane >= n || r >= to.rows) continue;
                const float y = *reinterpret_cast<const float *>(buffer + r * 128 + ((lane / 4) ^ (r & 7)) * 16 + lane % 4 * 4), z = A.base ? fmaf(y, scale, b[i]) : y * scale;
                if (o32) store1<true>(A.out, at + r * to.ldo, z); else store1<false>(A.out, at + r * to.ldo, z);
            }
        }
    }
    __syncwarp();
}

__device__ __forceinline__ int64_t target_of(const ProductArgs &A, int64_t row) {  // -1: none
    const int64_t v = A.flags & kIds64 ? static_cast<const int64_t *>(A.targets)[row] : static_cast<const int32_t *>(A.targets)[row];
    return v < 0 || v >= A.vocab ? -1 : v;
}

// The largest of a call's peaks (all of one warp ask); 1 where that divides nothing.
__device__ __forceinline__ float peak_of(const float *peaks) {
    if (!peaks) return 1.f;
    float m = 0.f;
    for (int i = threadIdx.x & 31; i < kPeaks; i += 32) m = fmaxf(m, peaks[i]);
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(kFullMask, m, d));
    return m > 0.f && m < INFINITY ? m : 1.f;
}

constexpr int kPart = 128;  // columns of a LOSS part: what one warp has of a tile
constexpr float kLog2e = 1.44269504088896340736f;

// The sums in tensor memory, one half after the other, as a warp that writes out sees them.
struct Sums {
    Shared &S;
    Place half;
    uint32_t first;
    __device__ __forceinline__ bool wait(uint32_t &at) {  // for the next; false if that gave up
        if (!warp_wait(&S.sums[half.s], half.phase, S)) return false;
        after_sync();
        at = first + half.s * kTile;
        return true;
    }
    __device__ __forceinline__ void free() {
        before_sync();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) bar_arrive(&S.freed[half.s]);
        half.next(2);
    }
};

// What a warp does with 32 rows and COLS columns of a tile, from row `row0` and column `col0` of it; false if a wait gave up. Sums of more than A.chunk
// steps come in several parts, which are added here: the tensor cores round every addition towards zero, so that errors do not cancel but grow with the
// number of steps (measured: 1e-9 of the result for each product).
template <int KIND, int END, int COLS>
__device__ __forceinline__ bool end_tile(const ProductArgs &A, char *buffer, const Tile &t, float peak, int row0, int col0, Sums &sums) {
    const bool parts = A.splits > 1;  // of the sums, each to a tile of its own
    const int64_t first = int64_t(t.m0) + row0, row = first + (threadIdx.x & 31);
    const int64_t end = KIND == kOuter ? A.inner : t.r1;
    const bool mine = row < end;
    const int start = t.n0 + col0, stop = min(start + COLS, A.cols);
    const bool any = first < end && start < stop;
    const Target to{parts ? int64_t(t.unit) * (kTile * kTile) + row0 * kTile - t.n0 : (KIND == kOuter ? t.group * A.o_group : 0) + first * A.ldo,
                    parts ? kTile : A.ldo, int(min(end - first, int64_t(32)))};
    // LOSS, LOGITS_GRAD: in powers of two, exp(x) = 2^(x log2 e)
    const float scale = A.scale * peak, scale2 = A.scale * kLog2e;
    const int64_t target = END != kStore && mine ? target_of(A, row) : -1;
    const float g = END == kLogitsGrad && target >= 0 ? A.dloss[row] / peak : 0.f;
    const float lse2 = END == kLogitsGrad && target >= 0 ? A.lse[row] * kLog2e : INFINITY;  // (padding: no probability)
    float top = -INFINITY, sum = 0.f;

    // The target's column, here; where no column is meant, one that no tile has.
    const int picked = target >= A.first && target < A.first + A.cols ? int(target - A.first) : -kTile;
    auto turn = [&](int column, auto &x) {  // LOGITS_GRAD: logits to their gradients
        constexpr int N = sizeof(x) / 4;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = exp2_of(fmaf(x[i], scale2, -lse2));
        if (picked >= column && picked < column + N) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] -= picked == column + i ? 1.f : 0.f;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= g;
        if (target < 0) {  // (padding: its zeros times an infinity of the table are NaN)
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = 0.f;
        }
    };
    auto pick = [&](int column, const auto &x) {  // LOSS: the target's logit
        constexpr int N = sizeof(x) / 4;
        if (picked < column || picked >= column + N) return;
        float p = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) p = picked == column + i ? x[i] : p;
        A.picked[row] = p * scale2;
    };
    auto sum_up = [&](const float (&x)[64]) {  // LOSS: 64 logits, all there
        float far[4] = {x[0], x[1], x[2], x[3]}, part[4] = {};
        if (scale2 >= 0.f) {
#pragma unroll
            for (int i = 4; i < 64; ++i) far[i % 4] = fmaxf(far[i % 4], x[i]);
            far[0] = fmaxf(fmaxf(far[0], far[1]), fmaxf(far[2], far[3]));
        } else {
#pragma unroll
            for (int i = 4; i < 64; ++i) far[i % 4] = fminf(far[i % 4], x[i]);
            far[0] = fminf(fminf(far[0], far[1]), fminf(far[2], far[3]));
        }
        const float most = fmaxf(top, far[0] * scale2), from = finite_or_0(most);
#pragma unroll
        for (int i = 0; i < 64; ++i) part[i % 4] += exp2_of(fmaf(x[i], scale2, -from));
        sum = fmaf(sum, exp2_of(top - from), (part[0] + part[1]) + (part[2] + part[3]));
        top = most;
    };
    auto chunk = [&](int column, float (&x)[32]) {  // 32 columns
        const int n = stop - column;
        if constexpr (END == kStore) {
            put_32(A, buffer, to, column, n, scale, x);
        } else if constexpr (END == kLoss) {
            pick(column, x);
            float high[4] = {top, -INFINITY, -INFINITY, -INFINITY}, part[4] = {};
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                x[i] = i < n ? x[i] * scale2 : -INFINITY;
                high[i % 4] = fmaxf(high[i % 4], x[i]);
            }
            const float most = fmaxf(fmaxf(high[0], high[1]), fmaxf(high[2], high[3])), from = finite_or_0(most);
#pragma unroll
            for (int i = 0; i < 32; ++i) part[i % 4] += exp2_of(x[i] - from);
            sum = fmaf(sum, exp2_of(top - from), (part[0] + part[1]) + (part[2] + part[3]));
            top = most;
        } else {
            turn(column, x);
            put_32(A, buffer, to, column, n, 1.f, x);
        }
    };
    // Below, one loop for what comes from tensor memory, from several parts of it, or is zeros, and not unrolled: what becomes of 32 columns is long, and code
    // that is there several times waits for instructions (2.2 us more a tile, measured with four copies).
    float run[COLS / 32][32];
    const bool several = t.steps > A.chunk;
    if (several) {
#pragma unroll
        for (int c = 0; c < COLS / 32; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i) run[c][i] = 0.f;
#pragma unroll 1
        for (int k = 0; k < t.steps; k += A.chunk) {
            uint32_t acc;
            if (!sums.wait(acc)) return false;
#pragma unroll
            for (int c = 0; c < COLS / 32; ++c) {
                float x[32];
                read_sums(acc + c * 32, x);
                sums_read(x);
#pragma unroll
                for (int i = 0; i < 32; ++i) run[c][i] += x[i];
            }
            sums.free();
        }
    }
    const bool here = t.steps && !several;
    uint32_t acc = 0;
    if (here && !sums.wait(acc)) return false;
    if (any) {
        int c = 0;
        if (here && (END == kLoss || (A.flags & kOutVec && !(A.flags & kOut32) && !A.base))) {
#pragma unroll 1
            for (; c < COLS && start + c + 64 <= stop; c += 64) {
                float x[64];
                read_sums(acc + c, *reinterpret_cast<float (*)[32]>(x));
                read_sums(acc + c + 32, *reinterpret_cast<float (*)[32]>(x + 32));
                sums_read(*reinterpret_cast<float (*)[32]>(x));
                sums_read(*reinterpret_cast<float (*)[32]>(x + 32));
                if constexpr (END == kLoss) {
                    pick(start + c, x);
                    sum_up(x);
                } else {
                    if (END == kLogitsGrad) turn(start + c, x);
                    put_64(A, buffer, to, start + c, END == kLogitsGrad ? 1.f : scale, x);
                }
            }
        }
#pragma unroll(END == kLoss ? COLS / 32 : 1)
        for (; c < COLS; c += 32) {
            if (start + c >= stop) break;
            float x[32];
            if (here) {
                read_sums(acc + c, x);
                sums_read(x);
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    x[i] = 0.f;
                    if (several) {
#pragma unroll
                        for (int j = 0; j < COLS / 32; ++j) x[i] = c == 32 * j ? run[j][i] : x[i];
                    }
                }
            }
            chunk(start + c, x);
        }
    }
    if (here) sums.free();
    if (END == kLoss && any && mine) A.part[int64_t(start / kPart) * A.rows + row] = make_float2(top, sum);  // lanes side by side
    return true;
}

// The same for a turned tile: a lane has a column of the matrices, and 32 of the tile's columns are 32 rows, so that a store of the warp is 64 or 128 bytes of a row,
// wherever it starts. `which`: of the two warps that have these lanes; they take every other 32 rows.
template <int KIND>
__device__ __forceinline__ bool end_turned(const ProductArgs &A, const Tile &t, int row0, int which, Sums &sums) {
    const int column = t.n0 + row0 + (threadIdx.x & 31), width = t.width();
    const bool mine = column < A.cols, several = t.steps > A.chunk;
    float run[kTile / 64][32];
    if (several) {
#pragma unroll
        for (int c = 0; c < kTile / 64; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i) run[c][i] = 0.f;
#pragma unroll 1
        for (int k = 0; k < t.steps; k += A.chunk) {
            uint32_t acc;
            if (!sums.wait(acc)) return false;
#pragma unroll
            for (int c = 0; c < kTile / 64; ++c) {
                if (c * 64 >= width) break;
                float x[32];
                read_sums(acc + (2 * c + which) * 32, x);
                sums_read(x);
#pragma unroll
                for (int i = 0; i < 32; ++i) run[c][i] += x[i];
            }
            sums.free();
        }
    }
    uint32_t acc = 0;
    if (!several && !sums.wait(acc)) return false;
#pragma unroll 1
    for (int c = 0; c < width; c += 64) {
        float x[32];
        if (!several) {
            read_sums(acc + c + which * 32, x);
            sums_read(x);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
#pragma unroll
                for (int j = 0; j < kTile / 64; ++j) x[i] = c == 64 * j ? run[j][i] : x[i];
        }
        const int first = t.m0 + c + which * 32, rows = t.r1 - first;
        if (!mine || rows <= 0) continue;
        if (A.flags & kOut32) {
            float *out = static_cast<float *>(A.out) + first * A.ldo + column;
#pragma unroll
            for (int i = 0; i < 32; ++i, out += A.ldo)
                if (i < rows) *out = x[i];
        } else {
            uint16_t *out = static_cast<uint16_t *>(A.out) + first * A.ldo + column;
#pragma unroll
            for (int i = 0; i < 32; ++i, out += A.ldo)
                if (i < rows) *out = uint16_t(pack_bf16(x[i], x[i]));
        }
    }
    if (!several) sums.free();
    return true;
}

// Rows of no group are zeros.
__device__ __forceinline__ void clear_rows(const ProductArgs &A, const Shared &S, int warp, int lane) {
    const int64_t before = S.begin[0], behind = A.rows - S.begin[A.groups];
    for (int64_t i = int64_t(blockIdx.x) * kEndWarps + warp; i < before + behind; i += int64_t(gridDim.x) * kEndWarps) {
        const int64_t row = i < before ? i : S.begin[A.groups] + i - before;
        if (A.flags & kOutVec) {
            for (int c = lane * 8; c < A.cols; c += 256) {
                char *q = static_cast<char *>(A.out) + (row * A.ldo + c) * (A.flags & kOut32 ? 4 : 2);
                reinterpret_cast<uint4 *>(q)[0] = make_uint4(0, 0, 0, 0);
                if (A.flags & kOut32) reinterpret_cast<uint4 *>(q)[1] = make_uint4(0, 0, 0, 0);
            }
        } else {
            for (int c = lane; c < A.cols; c += 32) {
                if (A.flags & kOut32) store1<true>(A.out, row * A.ldo + c, 0.f); else store1<false>(A.out, row * A.ldo + c, 0.f);
            }
        }
    }
}

// The stages of one operand, as one of the warps has them that load it.
template <int KIND, int COPY, bool MAJOR, int N>
__device__ __forceinline__ bool load_stages(const ProductArgs &A, Shared &S, Walk<KIND> &walk, char *raw, char *ring, uint32_t stages, int from, int rank, bool second) {
    constexpr bool TURNED = kTurned<KIND>;
    constexpr int kDeep = kRawStages<COPY>;
    const int lane = threadIdx.x & 31;
    const void *const any = reinterpret_cast<const void *>(reinterpret_cast<uintptr_t>(second ? A.b : A.a) & ~uintptr_t(15));
    auto lines_of = [&](const Tile &t) {
        const int64_t s0 = (KIND == kOuter ? t.r0 : 0) + int64_t(t.k0) * kStep, s_end = KIND == kOuter ? t.r1 : A.inner;
        if (!second) {
            const int64_t l0 = (TURNED ? t.n0 : t.m0) + rank * kLines;
            return Loose<MAJOR, N>(static_cast<const uint16_t *>(A.a) + (TURNED ? t.group * A.a_group : 0), A.lda, l0, TURNED ? A.cols : KIND == kOuter ? A.inner : t.r1, s0,
                                   s_end, from, lane);
        }
        const int half = TURNED ? t.width() / 2 : kLines;
        const int64_t l0 = TURNED ? t.m0 + rank * half : t.n0 + rank * kLines;
        return Loose<MAJOR, N>(static_cast<const uint16_t *>(A.b) + (KIND == kByRows ? t.group * A.b_group : 0), A.ldb, l0, TURNED ? min(int64_t(t.r1), l0 + half) : A.cols, s0, s_end, from, lane);
    };
    Walk<KIND> walk_ahead = walk;
    Tile t, ta;
    ta.steps = 0;
    int ka = 0;
    uint32_t asked = 0, slot = 0;
    Loose<MAJOR, N> ahead(nullptr, 0, 0, 0, 0, 0, 0, 0);
    auto ask = [&] {  // for the next stage, if there is one
        bool more = true;
        if (ka == ta.steps) {
            do more = walk_ahead.next(ta); while (more && !ta.steps);
            ka = 0;
            if (more) ahead = lines_of(ta); else ta.steps = 0;
        }
        if (more) {
            ahead.ask(shared_address(raw + asked * N * kRawLine), any, lane);
            ahead.next();
            ++ka;
            asked = asked + 1 == kDeep ? 0 : asked + 1;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int i = 1; i < kDeep; ++i) ask();
    Place p;
    bool ok = true;
    while (ok && walk.next(t)) {
        if (!t.steps) continue;
        Loose<MAJOR, N> lines = lines_of(t);
        for (int k = 0; k < t.steps; ++k, p.next(stages), lines.next()) {
            ask();
            asm volatile("cp.async.wait_group %0;" ::"n"(kDeep - 1) : "memory");
            if (!(ok = warp_wait(&S.empty[p.s], p.phase ^ 1, S))) break;
            __syncwarp();
            lines.cut(raw + slot * N * kRawLine, ring + p.s * kStageBytes, from, lane);
            slot = slot + 1 == kDeep ? 0 : slot + 1;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (!lane) bar_arrive(&S.full[p.s]);
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    return ok;
}

template <int KIND, int END, int COPY>
__global__ void __launch_bounds__(kThreads<COPY>, 1) k_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                               const __grid_constant__ CUtensorMap map_few, const ProductArgs A, const uint32_t stages) {
    extern __shared__ char raw[];
    constexpr bool COPY_A = COPY & kCopyA, COPY_B = COPY & kCopyB;
    char *const ring = raw + (1024 - (shared_address(raw) & 1023)) % 1024, *const out_at = ring + stages * kStageBytes + kRawBytes<COPY>;
    Shared &S = *reinterpret_cast<Shared *>(out_at + kEndWarps * kOutBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = blockIdx.x & 1;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) bar_init(&S.full[i], 2 * ((COPY ? 1 : 0) + (COPY == 3 ? 0 : kLoadWarps))), bar_init(&S.empty[i], 1), bar_init(&S.landed[i], 1);
        for (int i = 0; i < 2; ++i) bar_init(&S.sums[i], 1), bar_init(&S.freed[i], 2 * kEndWarps);
        S.gave_up = S.asked = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (COPY && threadIdx.x == 32 * kCopyWarp) {
        if (COPY_A) asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        if (COPY_B) asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
    }
    if (warp == kMemWarp) take_tensor_memory(&S.acc);
    before_sync();
    pair_sync();
    after_sync();
    wait_launch_before();  // (what is above reads nothing that the launch before wrote, and goes on beside its end)
    if (A.flags & kRelease) release_launch_after();
    groups_of<KIND, kThreads<COPY>>(A, S);
    const uint32_t acc = S.acc;
    constexpr bool A_MAJOR = kMajorA<KIND>, B_MAJOR = kMajorB<KIND>, TURNED = kTurned<KIND>;
    Walk<KIND> walk(A, S);
    Tile t;
    Place p;
    bool ok = true;

    // Registers, of the 168 (96) that a thread starts with: a warp that writes out holds 128 columns of sums, and what becomes of them.
    if (warp < kFirstEnd) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(COPY == 3 ? 56 : 40));
    if (COPY && warp == kCopyWarp) {  // one lane, as where the products are issued: 32 that wait for a barrier slow down what runs beside them by 3 %
        uint32_t n = 0;
        while (ok && walk.next(t)) {
            if (!lane) {
                const int half = TURNED ? t.width() / 2 : kLines;  // lines of B
                const int m0 = TURNED ? t.n0 + rank * kLines : t.m0 + rank * kLines, n0 = TURNED ? t.m0 + rank * half : t.n0 + rank * kLines;
                // A CTA that has none of the rows needs nothing of A: its sums are not read.
                const bool rows = COPY_A && (TURNED || KIND == kOuter || m0 < t.r1);
                for (int k = 0; k < t.steps; ++k, ++n, p.next(stages)) {
                    const int s0 = (KIND == kOuter ? t.r0 : 0) + (t.k0 + k) * kStep;
                    if (!(ok = bar_wait(&S.empty[p.s], p.phase ^ 1, S))) break;
                    // The last lines of a group that ends within a stage go to the warp that clears what is behind them.
                    const bool cut = KIND == kOuter && s0 + kStep > t.r1;
                    const uint32_t to = shared_address(ring) + p.s * kStageBytes, bar = cut ? shared_address(&S.landed[p.s]) : in_first(&S.full[p.s]);
                    if (KIND == kOuter) *reinterpret_cast<volatile uint32_t *>(&S.asked) = n + 1;
                    bar_expect(bar, (rows ? kOperandBytes : 0) + (COPY_B ? half * 128 : 0));
                    if (rows) copy_lines<A_MAJOR>(map_a, to, bar, m0, s0, TURNED ? t.group : 0);
                    if (COPY_B && TURNED && half < kLines) {
                        for (int l = 0; l < half; l += kRowBox) copy_box(map_few, to + kOperandBytes + l * 128, bar, s0, n0 + l, 0);
                    } else if (COPY_B) {
                        copy_lines<B_MAJOR>(map_b, to + kOperandBytes, bar, n0, s0, KIND == kByRows ? t.group : 0);
                    }
                }
            }
            ok = __shfl_sync(kFullMask, ok, 0);
        }
        // what was asked for arrives before the shared memory is given back
        if (!ok && !rank && !lane)
            for (uint32_t i = n > stages ? n - stages : 0; i < n; ++i) drain(&S.full[i % stages], i / stages & 1);
    } else if (COPY && KIND == kOuter && warp == kCutWarp) {
        uint32_t phases = 0, n = 0;
        while (ok && walk.next(t)) {
            const int left = t.ends && t.steps ? (t.r1 - t.r0) % kStep : 0;
            n = (n + t.steps) % stages;
            if (!left) continue;
            const uint32_t s = n ? n - 1 : stages - 1;
            // (all groups before this one may have whole stages, for as long as they take)
            if (!(ok = warp_wait(&S.landed[s], phases >> s & 1, S, &S.asked))) break;
            phases ^= 1u << s;
            char *const at = ring + s * kStageBytes;
            for (int i = left * 8 + lane; i < kStep * 8; i += 32)  // 16-byte units of a block's lines
#pragma unroll
                for (int b = COPY_A ? 0 : 2; b < (COPY_B ? 4 : 2); ++b) *reinterpret_cast<uint4 *>(at + b * (kOperandBytes / 2) + i * 16) = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (!lane) bar_arrive(&S.full[s]);
            __syncwarp();
        }
    } else if (COPY != 3 && warp >= kFirstLoad) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        // A warp has 16 lines of the operand that is not copied, or 32 of one of both.
        constexpr int N = COPY ? kLooseLines / 2 : kLooseLines;
        const int w = warp - kFirstLoad, from = w * N % kLines;
        char *const raw = ring + stages * kStageBytes + size_t(w) * kRawStages<COPY> * N * kRawLine;
        if (COPY ? COPY_A : w * N >= kLines)
            ok = load_stages<KIND, COPY, B_MAJOR, N>(A, S, walk, raw, ring + kOperandBytes, stages, from, rank, true);
        else
            ok = load_stages<KIND, COPY, A_MAJOR, N>(A, S, walk, raw, ring, stages, from, rank, false);
    } else if (warp == kMulWarp && !rank) {
        Place h;  // of the two halves of tensor memory
        bool some = false;
        while (ok && walk.next(t)) {
            if (!lane && t.steps) {
                uint32_t to = 0;
                const uint32_t instruction = kInstruction<A_MAJOR, B_MAJOR> | uint32_t(TURNED ? t.width() : kTile) >> 3 << 17;
                for (int k = 0, in = 0; k < t.steps; ++k, ++in) {
                    if (in == A.chunk) {
                        commit(&S.sums[h.s]);
                        h.next(2);
                        in = 0;
                    }
                    if (in == 0) {
                        if (!(ok = bar_wait(&S.freed[h.s], h.phase ^ 1, S))) break;
                        to = acc + h.s * kTile;
                    }
                    if (!(ok = bar_wait(&S.full[p.s], p.phase, S))) break;
                    after_sync();
                    const uint32_t at = shared_address(ring) + p.s * kStageBytes;
                    const uint64_t a = operand<A_MAJOR>(at), b = operand<B_MAJOR>(at + kOperandBytes);
#pragma unroll
                    for (int i = 0; i < kStep / 16; ++i)
                        multiply(to, a + i * kNext16<A_MAJOR>, b + i * kNext16<B_MAJOR>, instruction, in | i);
                    commit(&S.empty[p.s]);
                    p.next(stages);
                    some = true;
                }
                if (ok) commit(&S.sums[h.s]);
                h.next(2);
            }
            ok = __shfl_sync(kFullMask, ok, 0);
        }
        // what was issued ends before the tensor memory is given back
        if (!ok && some) drain(&S.empty[p.s ? p.s - 1 : stages - 1], p.s ? p.phase : p.phase ^ 1);
    } else if (warp >= kFirstEnd && warp < kFirstLoad) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(COPY == 3 ? 224 : 152));
        const int q = warp % 4, col0 = (warp - kFirstEnd) / 4 * kEndCols;
        char *const buffer = out_at + (warp - kFirstEnd) * kOutBytes;
        Sums sums{S, {}, acc + (TURNED ? 0 : col0) + (uint32_t(q * 32) << 16)};
        const float peak = END == kLoss ? 1.f : peak_of(A.peaks);
        while (ok && walk.next(t)) {
            if (!t.steps && KIND == kOuter && A.base) continue;  // (there already, or k_keep's)
            if constexpr (TURNED)
                ok = end_turned<KIND>(A, t, rank * kLines + q * 32, col0 / kEndCols, sums);
            else
                ok = end_tile<KIND, END, kEndCols>(A, buffer, t, peak, rank * kLines + q * 32, col0, sums);
        }
        if (TURNED || (KIND == kByRows && A.offsets)) clear_rows(A, S, warp - kFirstEnd, lane);
    }
    before_sync();
    __syncwarp();
    pair_sync();
    if (warp == kMemWarp) give_tensor_memory(acc);
}

// out = base + scale * (the sum, in order, of a tile's shares), four columns to a thread. (Tiles that are cut are few: their elements' numbers fit 32 bits.)
constexpr int kSumThreads = 256;

__global__ void __launch_bounds__(kSumThreads) k_sum(const ProductArgs A, const int32_t splits, const uint32_t height) {
    wait_launch_before();
    if (A.flags & kRelease) release_launch_after();
    const float scale = A.scale * peak_of(A.peaks);
    const uint32_t mt = (height + kTile - 1) / kTile, nt = (uint32_t(A.cols) + kTile - 1) / kTile, fours = (uint32_t(A.cols) + 3) / 4, all = A.groups * height * fours;
    for (uint32_t i = blockIdx.x * kSumThreads + threadIdx.x; i < all; i += gridDim.x * kSumThreads) {
        const uint32_t q = i / fours, c = (i - q * fours) * 4, g = q / height, r = q - g * height;
        const uint32_t unit = ((g * mt + r / kTile) * nt + c / kTile) * splits;
        const float4 *p = reinterpret_cast<const float4 *>(A.parts + int64_t(unit) * (kTile * kTile) + r % kTile * kTile + c % kTile);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int s = 0; s < splits; ++s) {
            const float4 y = p[s * (kTile * kTile / 4)];
            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
        }
        const int64_t at = g * A.o_group + r * A.ldo + c;
        const float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (c + k >= uint32_t(A.cols) || (A.base == A.out && v[k] == 0.f)) continue;  // (in place: a matrix without rows is not touched)
            if (A.base && v[k] == 0.f && bool(A.flags & kOut32) == bool(A.flags & kBase32)) {  // (nor are its bits changed on the way to another tensor)
                if (A.flags & kOut32) static_cast<uint32_t *>(A.out)[at + k] = static_cast<const uint32_t *>(A.base)[at + k];
                else static_cast<uint16_t *>(A.out)[at + k] = static_cast<const uint16_t *>(A.base)[at + k];
                continue;
            }
            const float b = !A.base ? 0.f : A.flags & kBase32 ? load1<true>(A.base, at + k) : load1<false>(A.base, at + k);
            const float y = A.base ? fmaf(v[k], scale, b) : v[k] * scale;
            if (A.flags & kOut32) store1<true>(A.out, at + k, y); else store1<false>(A.out, at + k, y);
        }
    }
}

// The matrices of groups without rows stay as the base has them, bit for bit, in another tensor of its type: each one run of memory in both, copied in 16-byte
// units where both lie alike in those, and the elements before the first and behind the last. (By the warps that write out tiles this was slower for every call: the
// registers that it needed went to and from memory in each tile. The gradient of 65,536 rows took 143 us, 104 now, by one expert of 1024 x 1024, and 1942, 1878 now, by 128 of
// 4096 x 4096; that of 20 rows by 60 experts onto an fp32 base 270, 245 now, of 1304 x 1304, and 915, 376 now, of 1300 x 1301. A call whose experts all have rows pays 2 us.)
constexpr int kKeepThreads = 256, kKeepDeep = 8, kKeepBytes = kKeepThreads * kKeepDeep * 16;  // of a CTA at a time

template <typename T>
__global__ void __launch_bounds__(kKeepThreads) k_keep(const ProductArgs A, const int64_t size /* elements of a matrix */) {
    __shared__ __align__(16) char memory[sizeof(Shared) + (kMaxGroups + 1) * 8];
    Shared &S = *reinterpret_cast<Shared *>(memory);
    wait_launch_before();
    release_launch_after();
    groups_of<kOuter, kKeepThreads>(A, S);
    const int64_t shares = (size * int64_t(sizeof(T)) + kKeepBytes - 1) / kKeepBytes, all = shares * A.groups;
    for (int64_t u = blockIdx.x; u < all;) {
        const int64_t g = u / shares, first = (u - g * shares) * kKeepBytes / int64_t(sizeof(T));
        if (S.begin[g] != S.begin[g + 1]) {  // on to the next group
            u += ((g + 1) * shares - u + gridDim.x - 1) / gridDim.x * gridDim.x;
            continue;
        }
        u += gridDim.x;
        const T *const p = static_cast<const T *>(A.base) + g * A.o_group;
        T *const q = static_cast<T *>(A.out) + g * A.o_group;
        constexpr int kUnit = 16 / sizeof(T);
        if (((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15) == 0) {
            const int64_t before = min(int64_t(-(reinterpret_cast<uintptr_t>(p) / sizeof(T)) & (kUnit - 1)), size), units = (size - before) / kUnit;
            uint4 x[kKeepDeep];
#pragma unroll
            for (int k = 0; k < kKeepDeep; ++k) {
                const int64_t i = first / kUnit + k * kKeepThreads + threadIdx.x;
                if (i < units) x[k] = ld_stream(p + before + i * kUnit);
            }
#pragma unroll
            for (int k = 0; k < kKeepDeep; ++k) {
                const int64_t i = first / kUnit + k * kKeepThreads + threadIdx.x;
                if (i < units) st_stream(q + before + i * kUnit, x[k]);
            }
            const int64_t rest = threadIdx.x, i = rest < before ? rest : units * kUnit + rest;
            if (!first && i < size && rest < 2 * kUnit) q[i] = p[i];
        } else {
#pragma unroll 1
            for (int64_t i0 = first; i0 < first + kKeepBytes / int(sizeof(T)) && i0 < size; i0 += kKeepThreads * kKeepDeep) {
                T x[kKeepDeep];
#pragma unroll
                for (int k = 0; k < kKeepDeep; ++k) {
                    const int64_t i = i0 + k * kKeepThreads + threadIdx.x;
                    if (i < size) x[k] = p[i];
                }
#pragma unroll
                for (int k = 0; k < kKeepDeep; ++k) {
                    const int64_t i = i0 + k * kKeepThreads + threadIdx.x;
                    if (i < size) q[i] = x[k];
                }
            }
        }
    }
}

// One wait as the kernel's, for what nothing completes.
__global__ void k_wait_in_vain() {
    __shared__ Shared S;
    bar_init(&S.full[0], 1);
    S.gave_up = 0;
    bar_wait(&S.full[0], 0, S);
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
int64_t sms() {
    const int n = ops_sm_count();
    return n > 0 ? n : 152;
}

using Encode = decltype(&cuTensorMapEncodeTiled);

Encode encoder() {
    static const Encode f = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult got;
        return cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &got) == cudaSuccess && got == cudaDriverEntryPointSuccess
                   ? reinterpret_cast<Encode>(p) : nullptr;
    }();
    return f;
}

// Lines of `x` elements, `ld` apart, y of them in a group and z groups; boxes of `lines` lines of 128 bytes.
bool map_of(CUtensorMap *m, const void *p, int64_t x, int64_t ld, int64_t y, int64_t group, int64_t z, uint32_t lines) {
    const cuuint64_t dims[3] = {cuuint64_t(x), cuuint64_t(y), cuuint64_t(z)}, strides[2] = {cuuint64_t(ld) * 2, cuuint64_t(z > 1 ? group : ld) * 2};
    const cuuint32_t box[3] = {64, lines, 1}, step[3] = {1, 1, 1};
    const Encode f = encoder();
    return f && f(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), dims, strides, box, step,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether tensor copies can move a matrix: lines on 16-byte boundaries, strides that their maps hold.
bool copies(const void *p, int64_t ld, int64_t group, int64_t groups) {
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && (groups == 1 || (group % 8 == 0 && group < int64_t(1) << 38));
}

template <int KIND, int END, int COPY>
cudaError_t launch_of(const ProductArgs &A, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &few, cudaStream_t s) {
    constexpr auto k = k_product<KIND, END, COPY>;
    const cudaError_t e = ops_allow_smem<k>(int(kMaxSharedBytes));
    if (e != cudaSuccess) return e;
    uint32_t stages = kRing<COPY>;
    while (shared_bytes(stages, kRawBytes<COPY>, A.groups) > kMaxSharedBytes) --stages;
    const int64_t nt = (A.cols + kTile - 1) / kTile;
    const int64_t most = (KIND == kOuter ? int64_t((A.inner + kTile - 1) / kTile) * A.groups : A.rows / kTile + A.groups) * nt * A.splits;
    if (most > INT32_MAX) return cudaErrorInvalidValue;
    const int64_t pairs = sms() / 2;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = 2;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(uint32_t(most < pairs ? most : pairs) * 2);
    cfg.blockDim = dim3(kThreads<COPY>);
    cfg.dynamicSmemBytes = shared_bytes(stages, kRawBytes<COPY>, A.groups);
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k, a, b, few, A, stages);
}

// Steps between two additions outside of the tensor cores: 512 products (an error of 5e-7 of the result); 1024 (9e-7) for logits, of which an epilogue makes more
// (at 4096 columns 597 us for 8192 x 16384 of them, 619 with 512, 574 with all); 8192 (8e-6) where bf16 is made of it. The logits that the gradient makes anew
// are summed as the loss's are, though bf16 is made of them too: their bits are then the same, and an error that lse and a logit share leaves exp(l - lse), which
// is subtracted from 1 at a certain target (l = 60, 8192 columns: 4e-4 of dloss with 8192 products, where nothing should be left).
constexpr int kChunk32 = 512 / kStep, kChunkLoss = 1024 / kStep, kChunk16 = 8192 / kStep;

constexpr int kMostWaves = 4;  // of shares: what their sums' memory is sized for

// How many shares the summed index is cut into, so that few tiles keep the SMs busy: the fewest steps (of 64 products, about 0.3 us) that a pair of CTAs does in
// turn, a share's start and end counted as 6, and the launch that adds the shares as 10 and 0.4 for each: an estimate, which reckons with even loads and lines on 16-byte
// boundaries. us by the rule, with the best of 1 to 32 shares, and uncut: the gradient of 65,536 rows by one expert of 1024 x 1024 103, 103, 300; of 30,000 by 3 of
// 256 x 256 27, 24, 92; of 8192 by one of 4096 x 4096 176, 170, 170; of 5000 by 9 of 1000 x 511 46, 46, 46; the head's gradients of 44 tokens over 20879 x 520 78, 77, 152;
// of 512 over 50304 x 4096 489, 486, 577; of 4096 over 50257 x 768 667, 662, 691.
int shares_of(int64_t tiles, int64_t steps, int64_t pairs) {
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 4 * pairs && (s == 1 || (tiles * s <= kMostWaves * pairs && (steps + s - 1) / s >= 4)); ++s) {
        const int64_t units = tiles * s, waves = (units + pairs - 1) / pairs;
        const double cost = double(waves) * double((steps + s - 1) / s + 6) + (s > 1 ? 10 + 0.4 * double(units) : 0);
        if (s == 1 || cost < least) best = s, least = cost;
    }
    return best;
}

template <int KIND, int END, int COPY>
cudaError_t launch_split(ProductArgs A, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &few, cudaStream_t s) {
    const int64_t height = KIND == kOuter ? A.inner : A.rows, mt = (height + kTile - 1) / kTile, nt = (A.cols + kTile - 1) / kTile, tiles = mt * nt * A.groups;
    const int64_t steps = KIND == kOuter ? (A.rows + int64_t(kStep) * A.groups - 1) / (int64_t(kStep) * A.groups) : (A.inner + kStep - 1) / kStep;
    const int shares = END == kStore && A.parts ? shares_of(tiles, steps, sms() / 2) : 1;
    if (shares == 1) {
        if (KIND == kOuter && A.base && A.base != A.out && (A.offsets || !A.rows)) {
            const int64_t size = A.inner * A.ldo, ctas = (size * (A.flags & kOut32 ? 4 : 2) + kKeepBytes - 1) / kKeepBytes * A.groups, most = sms() * 8;
            const cudaError_t e = ops_launch(true, A.flags & kOut32 ? k_keep<uint32_t> : k_keep<uint16_t>, uint32_t(ctas < most ? ctas : most), kKeepThreads, 0, s, A, size);
            if (e != cudaSuccess) return e;
        }
        return launch_of<KIND, END, COPY>(A, a, b, few, s);
    }
    ProductArgs P = A;
    P.splits = shares;
    P.out = A.parts;
    P.base = nullptr;
    P.peaks = nullptr;
    P.scale = 1.f;
    P.flags = kOut32 | kOutVec | kRelease;
    P.chunk = kChunk32;
    const cudaError_t e = launch_of<KIND, END, COPY>(P, a, b, few, s);
    if (e != cudaSuccess) return e;
    const int64_t blocks = (A.groups * height * ((A.cols + 3) / 4) + kSumThreads - 1) / kSumThreads;
    return ops_launch(true, k_sum, uint32_t(blocks < sms() * 8 ? blocks : sms() * 8), kSumThreads, 0, s, A, shares, uint32_t(height));
}

template <int KIND, int END>
cudaError_t launch(ProductArgs A, cudaStream_t s) {
    CUtensorMap a{}, b{}, few{};
    A.splits = 1;
    A.chunk = END != kStore ? kChunkLoss : A.flags & kOut32 ? kChunk32 : kChunk16;
    constexpr bool A_MAJOR = kMajorA<KIND>, B_MAJOR = kMajorB<KIND>, TURNED = kTurned<KIND>, OUTER = KIND == kOuter;
    // lines of an operand: how long, how many, in how many groups, and in a copy
    const int64_t long_a = TURNED && !A_MAJOR ? A.cols : A.inner, lines_a = TURNED ? (A_MAJOR ? A.cols : A.inner) : A.rows, groups_a = TURNED ? A.groups : 1;
    const int64_t groups_b = KIND == kByRows ? A.groups : 1, long_b = B_MAJOR ? A.inner : A.cols, lines_b = TURNED || OUTER ? A.rows : B_MAJOR ? A.cols : A.inner;
    const bool copy_a = A.rows && copies(A.a, A.lda, A.a_group, groups_a) && map_of(&a, A.a, long_a, A.lda, lines_a, A.a_group, groups_a, A_MAJOR ? kLines : kStep);
    const bool copy_b = A.rows && copies(A.b, A.ldb, A.b_group, groups_b) && map_of(&b, A.b, long_b, A.ldb, lines_b, A.b_group, groups_b, B_MAJOR ? kLines : kStep) &&
                        (!TURNED || map_of(&few, A.b, long_b, A.ldb, lines_b, 0, 1, kRowBox));
    if (copy_a && copy_b) return launch_split<KIND, END, 3>(A, a, b, few, s);
    if (copy_a) return launch_split<KIND, END, kCopyA>(A, a, b, few, s);
    if (copy_b) return launch_split<KIND, END, kCopyB>(A, a, b, few, s);
    return launch_split<KIND, END, 0>(A, a, b, few, s);
}

}  // namespace

int32_t product_loss_columns() { return kPart; }

size_t product_parts_bytes(int64_t groups, int64_t height, int64_t cols) {
    const int64_t tiles = groups * ((height + kTile - 1) / kTile) * ((cols + kTile - 1) / kTile), units = kMostWaves * (sms() / 2);
    return tiles > 0 && 2 * tiles <= units ? size_t(units / tiles * tiles) * kTile * kTile * 4 : 0;
}

cudaError_t product_launch(ProductKind kind, ProductEnd end, const ProductArgs &A, cudaStream_t s) {
    if (end == kLoss) return launch<kByCols, kLoss>(A, s);
    if (end == kLogitsGrad) return launch<kByCols, kLogitsGrad>(A, s);
    switch (kind) {
        case kByRows: return launch<kByRows, kStore>(A, s);
        case kGroupRows: return launch<kGroupRows, kStore>(A, s);
        case kGroupCols: return launch<kGroupCols, kStore>(A, s);
        default: return launch<kOuter, kStore>(A, s);
    }
}

int product_status(cudaStream_t s) {
    void *p = nullptr;
    uint32_t word = 0;
    int rc = ops_cuda(cudaStreamSynchronize(s), "synchronise");
    if (rc || (rc = ops_cuda(cudaGetSymbolAddress(&p, g_status), "status")) || (rc = ops_cuda(cudaMemcpy(&word, p, 4, cudaMemcpyDeviceToHost), "status"))) return rc;
    if (!word) return SKEW_OK;
    if ((rc = ops_cuda(cudaMemsetAsync(p, 0, 4, s), "status")) || (rc = ops_cuda(cudaStreamSynchronize(s), "status"))) return rc;
    return ops_fail(SKEW_ETIMEOUT, "a wait on the device gave up");
}

}  // namespace skew

extern "C" int skew_ops_sync_status(void *stream) { return skew::product_status((cudaStream_t)stream); }

extern "C" int skew_ops_selftest_wait_timeout(void *stream) {
    return skew::ops_cuda(skew::ops_launch(false, skew::k_wait_in_vain, 1, 1, 0, (cudaStream_t)stream), "k_wait_in_vain");
}
