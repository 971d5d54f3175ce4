// Matrix products on the fifth-generation tensor cores (skew_product.h): a persistent kernel whose warps load
// (8 warps), multiply (one thread) and write out (4 warps) at the same time.
//
// A CTA brings 128 lines of A and 128 of B, 64 elements of each at a time (a stage of 32 KiB, in a ring of six), to shared
// memory in 128-byte rows whose 16-byte units are permuted by the row's number (unit u of row L lies at u ^ (L & 7)), which is the layout that
// tcgen05.mma reads without bank conflicts. The same layout serves both orders of an operand: lines along the summed index
// ("K-major"), or 64 steps of the summed index, each a line along the tile ("MN-major"), 64 columns to a block of 8 KiB.
// Sums stay in tensor memory in fp32, in two halves: the next tile is multiplied into one while the other is written out.
//
// Rows of the group behind this one, which a tile's last lines may hold, cost nothing: a row of C has its own row of A. Where the
// rows are summed over (OUTER) they are zeros in shared memory, so that nothing of another group, NaN included, enters.
#include "skew_product.h"

#include <cuda.h>

#include <atomic>

#include "skew_ops.h"

namespace skew {
namespace {

constexpr int kLines = 128;                    // of each operand, in a CTA's stage
constexpr int kStep = 64;                      // elements of the summed index in a stage
constexpr uint32_t kOperandBytes = kLines * kStep * 2;
constexpr uint32_t kStageBytes = 2 * kOperandBytes;
constexpr int kStages = 6;                     // 5 where there are many groups
constexpr int kMaxGroups = 1024;
constexpr int kBandRows = 2048;                // rows of tiles that are walked together (what 152 SMs have under way then stays in L2)

constexpr int kMulWarp = 0, kMemWarp = 1, kCopyWarp = 2, kCutWarp = 3, kFirstEnd = 4;  // of the warps from 4 on, each reads lanes 32 (warp % 4) on of tensor memory
constexpr int kLoadWarps = 8;

// COPY: stages come by tensor copies (one thread), and eight warps write out; else eight warps load, and four write out.
template <bool COPY>
constexpr int kEndWarps = COPY ? 8 : 4;
template <bool COPY>
constexpr int kThreads = 32 * (kFirstEnd + kEndWarps<COPY> + (COPY ? 0 : kLoadWarps));
// PAIR: CTAs that share a tile, 1 or 2.
template <int PAIR>
constexpr int kTile = 128 * PAIR;              // rows and columns of a tile

struct Shared {
    uint64_t full[kStages], empty[kStages], landed[kStages], sums[2], freed[2];
    uint32_t acc;                     // where the sums are in tensor memory
    uint32_t gave_up;
    int32_t total[32];
    int32_t begin[1];                 // [groups + 1]: first row of each group, and the end of the last; then
                                      // [groups + 1]: tiles of rows before it (BY_ROWS, BY_COLS)
};

constexpr int kOutBytes = 32 * 128;            // 32 rows of 128 bytes, of each warp that writes out
constexpr size_t kMaxSharedBytes = 232448;
constexpr size_t shared_bytes(int stages, int end_warps, int groups) {
    return 1024 + size_t(stages) * kStageBytes + size_t(end_warps) * kOutBytes + sizeof(Shared) + size_t(groups + 1) * 8;
}
static_assert(shared_bytes(kStages - 1, 8, kMaxGroups) <= kMaxSharedBytes, "shared memory of a CTA");

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
template <int PAIR>
__device__ __forceinline__ uint32_t in_first(const void *p) {
    uint32_t a = shared_address(p);
    if constexpr (PAIR == 2) asm("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(a));
    return a;
}

template <int PAIR>
__device__ __forceinline__ void bar_arrive(uint64_t *b) {  // the first CTA's
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(in_first<PAIR>(b)) : "memory");
}

// Arrives at a barrier of this address, which then also waits for `bytes`. (Relaxed: nothing that this thread wrote is read after it. A release
// waits for what is under way, copies among it: 0.6 us a stage.)
__device__ __forceinline__ void bar_expect(uint32_t address, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(address), "r"(bytes) : "memory");
}

__device__ __forceinline__ bool bar_poll(uint64_t *b, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(shared_address(b)), "r"(parity), "n"(2000) : "memory");
    return ok != 0;
}

// False once this or another of the CTA's waits has given up, after some two seconds: the kernel then ends as it stands and
// leaves its mark for skew_ops_sync_status.
__device__ __forceinline__ bool bar_wait(uint64_t *b, uint32_t parity, Shared &S) {
    if (bar_poll(b, parity)) return true;
    for (uint32_t i = 0; i < 1u << 20; ++i) {
        if (bar_poll(b, parity)) return true;
        if (*reinterpret_cast<volatile uint32_t *>(&S.gave_up)) return false;
    }
    *reinterpret_cast<volatile uint32_t *>(&S.gave_up) = 1;
    atomicOr(&g_status, 1u);
    return false;
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
};

__device__ __forceinline__ int32_t *tiles_of(const ProductArgs &A, Shared &S) { return S.begin + A.groups + 1; }

// The groups' rows, in order and within [0, rows) whatever `offsets` hold, and the tiles before each.
template <int KIND, int THREADS, int TILE>
__device__ __forceinline__ void groups_of(const ProductArgs &A, Shared &S) {
    const int G = A.groups, per = (G + THREADS) / THREADS, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rows = int(A.rows);
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
    auto at = [&](int i) { return A.offsets ? min(max(A.offsets[i], 0), rows) : i ? rows : 0; };
    int m = 0;
    for (int i = i0; i < i1; ++i) m = max(m, at(i));
    m = scan(m, most);
    for (int i = i0; i < i1; ++i) S.begin[i] = m = max(m, at(i));
    __syncthreads();
    if (KIND != kOuter) {
        int32_t *const tile = tiles_of(A, S);
        auto tiles = [&](int i) { return i < G ? (S.begin[i + 1] - S.begin[i] + TILE - 1) / TILE : 0; };
        int n = 0;
        for (int i = i0; i < i1; ++i) n += tiles(i);
        n = scan(n, both);
        for (int i = i0; i < i1; ++i) tile[i] = n, n += tiles(i);
    }
    __syncthreads();
}

// The pair's tiles, one after another: its own number, + the pairs, ...
template <int KIND, int PAIR>
struct Walk {
    static constexpr int kT = kTile<PAIR>, kBand = kBandRows / kT;
    const ProductArgs &A;
    const int32_t *begin, *tile;
    int64_t at, all;
    int64_t each;      // OUTER: tiles of a group
    int32_t nt, group;

    __device__ __forceinline__ Walk(const ProductArgs &a, Shared &s) : A(a), begin(s.begin), tile(tiles_of(a, s)), at(blockIdx.x / PAIR), group(0) {
        nt = (A.cols + kT - 1) / kT;
        if (KIND == kOuter) {
            each = int64_t((A.inner + kT - 1) / kT) * nt;
            all = each * A.groups;
        } else {
            all = int64_t(tile[A.groups]) * nt;
        }
        all *= A.splits;
    }

    __device__ __forceinline__ bool next(Tile &t) {
        if (at >= all) return false;
        int64_t here = at;
        int mt, split = 0;
        if (A.splits > 1) here /= A.splits, split = int(at - here * A.splits);
        if (KIND == kOuter) {
            group = int(here / each);
            here -= group * each;
            mt = (A.inner + kT - 1) / kT;
        } else {
            const int row = int(here / nt);  // tiles of rows before this one's, over all groups: its group is the last that begins at or before it
            int lo = group, hi = A.groups;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (tile[mid] <= row) lo = mid; else hi = mid;
            }
            group = lo;
            here -= int64_t(tile[group]) * nt;
            mt = tile[group + 1] - tile[group];
        }
        const int64_t span = int64_t(kBand) * nt;
        const int band = int(here / span), first = band * kBand, in = min(kBand, mt - first), left = int(here - band * span);
        t.group = group;
        t.r0 = begin[group];
        t.r1 = begin[group + 1];
        t.m0 = (first + left % in) * kT + (KIND == kOuter ? 0 : t.r0);
        t.n0 = left / in * kT;
        const int steps = ((KIND == kOuter ? t.r1 - t.r0 : A.inner) + kStep - 1) / kStep, share = (steps + A.splits - 1) / A.splits;
        t.k0 = split * share;
        t.steps = max(min(share, steps - t.k0), 0);
        t.ends = t.k0 + t.steps == steps;
        t.unit = ((KIND == kOuter ? group * mt : 0) + first + left % in) * nt + left / in;
        t.unit = t.unit * A.splits + split;
        at += gridDim.x / PAIR;
        return true;
    }
};

// ---------------------------------------------------------------------------
// Loads
// ---------------------------------------------------------------------------
// Eight elements from `p`, of which `n` are there.
__device__ __forceinline__ uint4 eight(const uint16_t *p, int n) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
        u = *reinterpret_cast<const uint4 *>(p);
    } else if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 3) == 0) {
        const uint32_t *q = reinterpret_cast<const uint32_t *>(p);
        u = make_uint4(q[0], q[1], q[2], q[3]);
    } else if (n > 0) {
        uint32_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0;
        u = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
    }
    return u;
}

// One operand's 128 lines of a stage. MAJOR: lines along the summed index, numbered l0 on, of which those before l_end are there; elements from s0, before s_end.
// Else two blocks of 64 lines, one for each step of the summed index (s0 on, before s_end), of elements from l0 (and l0 + 64), before l_end.
template <bool MAJOR>
__device__ __forceinline__ void load_lines(const uint16_t *p, int64_t ld, int64_t l0, int64_t l_end, int64_t s0, int64_t s_end, char *to, int warp, int lane) {
    constexpr int kRounds = kLines / (kLoadWarps / 2) / 4;
    uint4 u[kRounds];
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int L = (warp * kRounds + i) * 4 + lane / 8, c = lane % 8 * 8;
        const int64_t line = MAJOR ? l0 + L : s0 + L % 64, elem = MAJOR ? s0 + c : l0 + L / 64 * 64 + c;
        const int64_t left = (MAJOR ? s_end : l_end) - elem;
        u[i] = line < (MAJOR ? l_end : s_end) && left > 0 ? eight(p + line * ld + elem, left < 8 ? int(left) : 8) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int L = (warp * kRounds + i) * 4 + lane / 8;
        *reinterpret_cast<uint4 *>(to + L * 128 + ((lane % 8) ^ (L & 7)) * 16) = u[i];
    }
}

// A box of a tensor map, from column x, line y of group z, to shared memory at `to`; its bytes count at the barrier of this address.
template <int PAIR>
__device__ __forceinline__ void copy_box(const CUtensorMap &map, uint32_t to, uint32_t bar, int x, int y, int z) {
    if constexpr (PAIR == 2)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(to), "l"(&map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                     ::"r"(to), "l"(&map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}

// One operand's 128 lines, as load_lines brings them. Beyond the matrix the boxes hold zeros.
template <bool MAJOR, int PAIR>
__device__ __forceinline__ void copy_lines(const CUtensorMap &map, uint32_t to, uint32_t bar, int l0, int s0, int group) {
    if constexpr (MAJOR) {
        copy_box<PAIR>(map, to, bar, s0, l0, group);
    } else {
        copy_box<PAIR>(map, to, bar, l0, s0, group);
        copy_box<PAIR>(map, to + kOperandBytes / 2, bar, l0 + 64, s0, group);
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

template <bool A_MAJOR, bool B_MAJOR, int PAIR>
constexpr uint32_t kInstruction = 1u << 4 /* sums fp32 */ | 1u << 7 | 1u << 10 /* bf16 */ | uint32_t(!A_MAJOR) << 15 | uint32_t(!B_MAJOR) << 16 |
                                  uint32_t(kTile<PAIR> >> 3) << 17 | uint32_t(kTile<PAIR> >> 4) << 24;

// 16 steps of the tile: for a pair of CTAs, each holds half of A's rows and of B's columns, and takes the sums of its rows.
template <int PAIR>
__device__ __forceinline__ void multiply(uint32_t acc, uint64_t a, uint64_t b, uint32_t instruction, bool add) {
    if constexpr (PAIR == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(acc), "l"(a), "l"(b), "r"(instruction), "r"(uint32_t(add)) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(acc), "l"(a), "l"(b), "r"(instruction), "r"(uint32_t(add)) : "memory");
}

// Arrives, in each CTA of the pair, once what was issued before is done.
template <int PAIR>
__device__ __forceinline__ void commit(uint64_t *bar) {
    if constexpr (PAIR == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(shared_address(bar)), "h"(uint16_t(3)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_address(bar)) : "memory");
}

template <int PAIR>
__device__ __forceinline__ void take_tensor_memory(uint32_t *address) {
    if constexpr (PAIR == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(address)), "n"(2 * kTile<PAIR>) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(address)), "n"(2 * kTile<PAIR>) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}

template <int PAIR>
__device__ __forceinline__ void give_tensor_memory(uint32_t acc) {
    if constexpr (PAIR == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(acc), "n"(2 * kTile<PAIR>) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(acc), "n"(2 * kTile<PAIR>) : "memory");
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

// y = base + scale * x for 32 columns of a row, of which `n` are there.
template <bool B32>
__device__ __forceinline__ void add_base(const ProductArgs &A, float scale, int64_t at, int n, float (&x)[32]) {
    if (!A.base) {
#pragma unroll
        for (int c = 0; c < 32; ++c) x[c] *= scale;
    } else if (n >= 32 && A.flags & kOutVec) {
        Vec8<B32> b[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) b[c] = load8_cached<B32>(A.base, at + 8 * c);
#pragma unroll
        for (int c = 0; c < 32; ++c) x[c] = fmaf(x[c], scale, b[c / 8].at(c % 8));
    } else {
#pragma unroll
        for (int c = 0; c < 32; ++c) x[c] = c < n ? fmaf(x[c], scale, load1<B32>(A.base, at + c)) : 0.f;
    }
}

// 32 columns of a row, of which `n` are there, to memory.
template <bool O32>
__device__ __forceinline__ void put_columns(const ProductArgs &A, int64_t at, int n, const float (&y)[32]) {
    if (n >= 32 && A.flags & kOutVec) {
        uint4 *q = reinterpret_cast<uint4 *>(const_cast<char *>(elem_ptr<O32>(A.out, at)));
#pragma unroll
        for (int c = 0; c < 32; c += O32 ? 4 : 8)
            q[c / (O32 ? 4 : 8)] = O32 ? make_uint4(__float_as_uint(y[c]), __float_as_uint(y[c + 1]), __float_as_uint(y[c + 2]), __float_as_uint(y[c + 3]))
                                       : make_uint4(pack_bf16(y[c], y[c + 1]), pack_bf16(y[c + 2], y[c + 3]), pack_bf16(y[c + 4], y[c + 5]), pack_bf16(y[c + 6], y[c + 7]));
        return;
    }
#pragma unroll
    for (int c = 0; c < 32; ++c)
        if (c < n) store1<O32>(A.out, at + c, y[c]);
}

// The 32 columns to the lane's row of the warp's 32 x 128 bytes of shared memory, 16-byte units permuted as in a stage; the last of the 128 bytes then
// leave by a tensor copy, which keeps to the matrix. `column`: the first of the 32.
template <bool O32>
__device__ __forceinline__ void copy_columns(const CUtensorMap &map, char *to, int column, int row0, int group, bool last, const float (&y)[32]) {
    const int lane = threadIdx.x & 31;
    constexpr int kWide = O32 ? 32 : 64;  // columns of 128 bytes
    const int part = column % kWide;
    if (part == 0) {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    }
#pragma unroll
    for (int c = 0; c < 32; c += O32 ? 4 : 8) {
        const uint4 u = O32 ? make_uint4(__float_as_uint(y[c]), __float_as_uint(y[c + 1]), __float_as_uint(y[c + 2]), __float_as_uint(y[c + 3]))
                            : make_uint4(pack_bf16(y[c], y[c + 1]), pack_bf16(y[c + 2], y[c + 3]), pack_bf16(y[c + 4], y[c + 5]), pack_bf16(y[c + 6], y[c + 7]));
        *reinterpret_cast<uint4 *>(to + lane * 128 + ((((part + c) / (O32 ? 4 : 8)) ^ (lane & 7)) * 16)) = u;
    }
    if (part + 32 == kWide || last) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                         ::"l"(&map), "r"(shared_address(to)), "r"(column - part), "r"(row0), "r"(group) : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
    }
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

// What a warp does with 32 rows and COLS columns of a tile, from row `row0` and column `col0` of it. read(f) has f see the sums in tensor memory, at an
// address, once they are there; false if the wait for them gave up. Sums of more than A.chunk steps come in several parts, which are added here: the tensor
// cores round every addition towards zero, so that errors do not cancel but grow with the number of steps (measured: 1e-9 of the result for each product).
template <int KIND, int END, int COLS, typename Read>
__device__ __forceinline__ bool end_tile(const ProductArgs &A, const CUtensorMap &map, char *buffer, const Tile &t, float peak, int row0, int col0, const Read &read) {
    const bool parts = A.splits > 1;  // of the sums, each to a tile of its own
    const int64_t first = int64_t(t.m0) + row0, row = first + (threadIdx.x & 31);
    const int64_t end = KIND == kOuter ? A.inner : t.r1;
    const bool mine = row < end;
    const int start = t.n0 + col0, stop = min(start + COLS, A.cols);
    const bool any = first < end && start < stop;
    // STORE: whole by a tensor copy, unless rows of the group behind would be written.
    const bool copy = A.flags & kOutCopy && (KIND == kOuter || !A.offsets || first + 32 <= end);
    const int64_t at = (KIND == kOuter ? t.group * A.o_group : 0) + row * A.ldo;
    const int to_col = parts ? t.n0 : 0, to_row = parts ? row0 : int(first), to_group = parts ? t.unit : KIND == kOuter ? t.group : 0;
    // LOSS, LOGITS_GRAD: in powers of two, exp(x) = 2^(x log2 e)
    const float scale = A.scale * peak, scale2 = A.scale * kLog2e;
    const int64_t target = END != kStore && mine ? target_of(A, row) : -1;
    const float g = END == kLogitsGrad && target >= 0 ? A.dloss[row] / peak : 0.f, lse2 = END == kLogitsGrad && target >= 0 ? A.lse[row] * kLog2e : 0.f;
    float top = -INFINITY, sum = 0.f;

    auto chunk = [&](int column, float (&x)[32]) {  // 32 columns
        const int n = stop - column;
        if constexpr (END == kStore) {
            if (mine) {
                if (A.flags & kBase32) add_base<true>(A, scale, at + column, n, x); else add_base<false>(A, scale, at + column, n, x);
            }
            if (copy) {
                if (A.flags & kOut32) copy_columns<true>(map, buffer, column - to_col, to_row, to_group, n <= 32, x); else copy_columns<false>(map, buffer, column - to_col, to_row, to_group, n <= 32, x);
            } else if (mine) {
                if (A.flags & kOut32) put_columns<true>(A, at + column, n, x); else put_columns<false>(A, at + column, n, x);
            }
        } else if constexpr (END == kLoss) {
            const int64_t here = target - column;
            if (here >= 0 && here < 32 && target >= 0) {
                float p = 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i) p = here == i ? x[i] : p;
                A.picked[row] = p * A.scale;
            }
            float high = top;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                x[i] = i < n ? x[i] * scale2 : -INFINITY;
                high = fmaxf(high, x[i]);
            }
            const float from = high == -INFINITY ? 0.f : high;
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) part += exp2_of(x[i] - from);
            sum = fmaf(sum, exp2_of(top - from), part);
            top = high;
        } else {
            const int64_t here = target - A.first - column;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float p = exp2_of(fmaf(x[i], scale2, -lse2)) - (here == i ? 1.f : 0.f);
                x[i] = target >= 0 ? p * g : 0.f;
            }
            if (copy) {
                copy_columns<false>(map, buffer, column, int(first), 0, n <= 32, x);
            } else if (mine) {
                put_columns<false>(A, at + column, n, x);
            }
        }
    };
    if (!t.steps) {
        float x[32];
        for (int c = start; any && c < stop; c += 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = 0.f;
            chunk(c, x);
        }
        return true;
    }
    if (t.steps <= A.chunk) {
        const bool ok = read([&](uint32_t acc) {
            if (!any) return;
            float x[2][32];
            read_sums(acc, x[0]);
#pragma unroll
            for (int c = 0; c < COLS / 32; ++c) {  // the next 32 columns are on their way while 32 are dealt with
                sums_read(x[c % 2]);
                if (c + 1 < COLS / 32) read_sums(acc + (c + 1) * 32, x[(c + 1) % 2]);
                if (start + c * 32 < stop) chunk(start + c * 32, x[c % 2]);
                __syncwarp();
            }
        });
        if (!ok) return false;
    } else {
        float run[COLS / 32][32];
#pragma unroll
        for (int c = 0; c < COLS / 32; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i) run[c][i] = 0.f;
#pragma unroll 1
        for (int k = 0; k < t.steps; k += A.chunk) {
            const bool ok = read([&](uint32_t acc) {
#pragma unroll
                for (int c = 0; c < COLS / 32; ++c) {
                    float x[32];
                    read_sums(acc + c * 32, x);
                    sums_read(x);
#pragma unroll
                    for (int i = 0; i < 32; ++i) run[c][i] += x[i];
                }
            });
            if (!ok) return false;
        }
        if (any) {
#pragma unroll
            for (int c = 0; c < COLS / 32; ++c) {
                if (start + c * 32 < stop) chunk(start + c * 32, run[c]);
                __syncwarp();
            }
        }
    }
    if (END == kLoss && any && mine) A.part[int64_t(start / kPart) * A.rows + row] = make_float2(top, sum);  // lanes side by side
    return true;
}

// Rows of no group are zeros.
template <int WARPS>
__device__ __forceinline__ void clear_rows(const ProductArgs &A, const Shared &S, int warp, int lane) {
    const int64_t before = S.begin[0], behind = A.rows - S.begin[A.groups];
    for (int64_t i = int64_t(blockIdx.x) * WARPS + warp; i < before + behind; i += int64_t(gridDim.x) * WARPS) {
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

template <int KIND, int END, bool COPY, int PAIR>
__global__ void __launch_bounds__(kThreads<COPY>, 1) k_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                               const __grid_constant__ CUtensorMap map_out, const ProductArgs A, const uint32_t stages) {
    extern __shared__ char raw[];
    constexpr int kT = kTile<PAIR>, kEnds = kEndWarps<COPY>, kEndCols = kT * 4 / kEnds;
    char *const ring = raw + (1024 - (shared_address(raw) & 1023)) % 1024, *const out_at = ring + stages * kStageBytes;
    Shared &S = *reinterpret_cast<Shared *>(out_at + kEnds * kOutBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = PAIR == 2 ? blockIdx.x & 1 : 0;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) bar_init(&S.full[i], PAIR * (COPY ? 1 : kLoadWarps)), bar_init(&S.empty[i], 1), bar_init(&S.landed[i], 1);
        for (int i = 0; i < 2; ++i) bar_init(&S.sums[i], 1), bar_init(&S.freed[i], PAIR * kEnds);
        S.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMemWarp) take_tensor_memory<PAIR>(&S.acc);
    groups_of<KIND, kThreads<COPY>, kT>(A, S);
    before_sync();
    if (PAIR == 2) pair_sync(); else __syncthreads();
    after_sync();
    const uint32_t acc = S.acc;
    constexpr bool A_MAJOR = KIND != kOuter, B_MAJOR = KIND == kByCols;
    Walk<KIND, PAIR> walk(A, S);
    Tile t;
    Place p;
    bool ok = true;

    // Registers, of the 168 (128) that a thread starts with: a warp that writes out holds 128 columns of sums, and what becomes of them.
    if (warp < kFirstEnd)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(COPY ? 56 : 48));
    if (COPY && warp == kCopyWarp) {
        if (!lane) {
            uint32_t n = 0;
            while (ok && walk.next(t)) {
                const int m0 = t.m0 + rank * kLines, n0 = t.n0 + rank * kLines;
                // A CTA whose rows all belong to the groups behind needs none of them: its sums are not read.
                const bool rows = KIND == kOuter || m0 < t.r1;
                for (int k = 0; k < t.steps; ++k, ++n, p.next(stages)) {
                    const int s0 = (KIND == kOuter ? t.r0 : 0) + (t.k0 + k) * kStep;
                    if (!(ok = bar_wait(&S.empty[p.s], p.phase ^ 1, S))) break;
                    // The last lines of a group that ends within a stage go to the warp that clears what is behind them.
                    const bool cut = KIND == kOuter && s0 + kStep > t.r1;
                    const uint32_t to = shared_address(ring) + p.s * kStageBytes, bar = cut ? shared_address(&S.landed[p.s]) : in_first<PAIR>(&S.full[p.s]);
                    bar_expect(bar, rows ? kStageBytes : kOperandBytes);
                    if (rows) copy_lines<A_MAJOR, PAIR>(map_a, to, bar, m0, s0, 0);
                    copy_lines<B_MAJOR, PAIR>(map_b, to + kOperandBytes, bar, n0, s0, KIND == kOuter ? 0 : t.group);
                }
            }
            // what was asked for arrives before the shared memory is given back
            if (!ok && !rank)
                for (uint32_t i = n > stages ? n - stages : 0; i < n; ++i) drain(&S.full[i % stages], i / stages & 1);
        }
    } else if (COPY && KIND == kOuter && warp == kCutWarp) {
        uint32_t phases = 0, n = 0;
        while (ok && walk.next(t)) {
            const int left = t.ends && t.steps ? (t.r1 - t.r0) % kStep : 0;
            n = (n + t.steps) % stages;
            if (!left) continue;
            const uint32_t s = n ? n - 1 : stages - 1;
            if (!(ok = bar_wait(&S.landed[s], phases >> s & 1, S))) break;
            phases ^= 1u << s;
            char *const at = ring + s * kStageBytes;
            for (int i = left * 8 + lane; i < kStep * 8; i += 32)  // 16-byte units of a block's lines
#pragma unroll
                for (int b = 0; b < 4; ++b) *reinterpret_cast<uint4 *>(at + b * (kOperandBytes / 2) + i * 16) = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (!lane) bar_arrive<PAIR>(&S.full[s]);
        }
    } else if (!COPY && warp >= kFirstEnd + kEnds) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 96;");
        const int w = (warp - kFirstEnd - kEnds) % (kLoadWarps / 2);
        const bool second = warp - kFirstEnd - kEnds >= kLoadWarps / 2;
        while (ok && walk.next(t)) {
            const uint16_t *b = static_cast<const uint16_t *>(A.b) + (KIND != kOuter ? t.group * A.b_group : 0);
            for (int k = 0; k < t.steps; ++k, p.next(stages)) {
                if (!(ok = bar_wait(&S.empty[p.s], p.phase ^ 1, S))) break;
                char *to = ring + p.s * kStageBytes;
                const int64_t s0 = (KIND == kOuter ? t.r0 : 0) + int64_t(t.k0 + k) * kStep, s_end = KIND == kOuter ? t.r1 : A.inner;
                if (!second)
                    load_lines<A_MAJOR>(static_cast<const uint16_t *>(A.a), A.lda, t.m0 + rank * kLines, KIND == kOuter ? A.inner : t.r1, s0, s_end, to, w, lane);
                else
                    load_lines<B_MAJOR>(b, A.ldb, t.n0 + rank * kLines, A.cols, s0, s_end, to + kOperandBytes, w, lane);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (!lane) bar_arrive<PAIR>(&S.full[p.s]);
            }
        }
    } else if (warp == kMulWarp && !rank) {
        if (!lane) {
            Place h;  // of the two halves of tensor memory
            bool some = false;
            while (ok && walk.next(t)) {
                if (!t.steps) continue;
                uint32_t to = 0;
                for (int k = 0, in = 0; k < t.steps; ++k, ++in) {
                    if (in == A.chunk) {
                        commit<PAIR>(&S.sums[h.s]);
                        h.next(2);
                        in = 0;
                    }
                    if (in == 0) {
                        if (!(ok = bar_wait(&S.freed[h.s], h.phase ^ 1, S))) break;
                        after_sync();
                        to = acc + h.s * kT;
                    }
                    if (!(ok = bar_wait(&S.full[p.s], p.phase, S))) break;
                    after_sync();
                    const uint32_t at = shared_address(ring) + p.s * kStageBytes;
                    const uint64_t a = operand<A_MAJOR>(at), b = operand<B_MAJOR>(at + kOperandBytes);
#pragma unroll
                    for (int i = 0; i < kStep / 16; ++i)
                        multiply<PAIR>(to, a + i * kNext16<A_MAJOR>, b + i * kNext16<B_MAJOR>, kInstruction<A_MAJOR, B_MAJOR, PAIR>, in | i);
                    commit<PAIR>(&S.empty[p.s]);
                    p.next(stages);
                    some = true;
                }
                if (ok) commit<PAIR>(&S.sums[h.s]);
                h.next(2);
            }
            // what was issued ends before the tensor memory is given back
            if (!ok && some) drain(&S.empty[p.s ? p.s - 1 : stages - 1], p.s ? p.phase : p.phase ^ 1);
        }
    } else if (warp >= kFirstEnd && warp < kFirstEnd + kEnds) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(COPY ? 224 : 216));
        const int q = warp % 4, col0 = (warp - kFirstEnd) / 4 * kEndCols;
        char *const buffer = out_at + (warp - kFirstEnd) * kOutBytes;
        Place h;
        const float peak = END == kLoss ? 1.f : peak_of(A.peaks);
        while (ok && walk.next(t)) {
            if (!t.steps && KIND == kOuter && A.base == A.out) continue;
            ok = end_tile<KIND, END, kEndCols>(A, map_out, buffer, t, peak, rank * kLines + q * 32, col0, [&](auto &&see) {
                if (!bar_wait(&S.sums[h.s], h.phase, S)) return false;
                after_sync();
                see(acc + h.s * kT + col0 + (uint32_t(q * 32) << 16));
                before_sync();
                __syncwarp();
                if (!lane) bar_arrive<PAIR>(&S.freed[h.s]);
                h.next(2);
                return true;
            });
        }
        if (KIND != kOuter && END == kStore && A.offsets) clear_rows<kEnds>(A, S, warp - kFirstEnd, lane);
        if (!lane) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    before_sync();
    __syncwarp();
    if (PAIR == 2) pair_sync(); else __syncthreads();
    if (warp == kMemWarp) give_tensor_memory<PAIR>(acc);
}

// out = base + scale * (the sum, in order, of a tile's shares), four columns to a thread.
constexpr int kSumThreads = 256;

template <int TILE>
__global__ void __launch_bounds__(kSumThreads) k_sum(const ProductArgs A, const int32_t splits, const int64_t height) {
    wait_launch_before();
    const float scale = A.scale * peak_of(A.peaks);
    const int64_t mt = (height + TILE - 1) / TILE, nt = (A.cols + TILE - 1) / TILE, fours = (A.cols + 3) / 4;
    for (int64_t i = blockIdx.x * int64_t(kSumThreads) + threadIdx.x; i < A.groups * height * fours; i += int64_t(gridDim.x) * kSumThreads) {
        const int64_t c = i % fours * 4, r = i / fours % height, g = i / fours / height;
        const float4 *p = reinterpret_cast<const float4 *>(A.parts + ((g * mt + r / TILE) * nt + c / TILE) * splits * (TILE * TILE) + r % TILE * TILE + c % TILE);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int s = 0; s < splits; ++s) {
            const float4 y = p[s * (TILE * TILE / 4)];
            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
        }
        const int64_t at = g * A.o_group + r * A.ldo + c;
        const float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (c + k >= A.cols || (A.base == A.out && v[k] == 0.f)) continue;  // (in place: a matrix without rows is not touched)
            const float b = !A.base ? 0.f : A.flags & kBase32 ? load1<true>(A.base, at + k) : load1<false>(A.base, at + k);
            const float y = A.base ? fmaf(v[k], scale, b) : v[k] * scale;
            if (A.flags & kOut32) store1<true>(A.out, at + k, y); else store1<false>(A.out, at + k, y);
        }
    }
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
bool map_of(CUtensorMap *m, const void *p, bool f32, int64_t x, int64_t ld, int64_t y, int64_t group, int64_t z, uint32_t lines) {
    const int es = f32 ? 4 : 2;
    const cuuint64_t dims[3] = {cuuint64_t(x), cuuint64_t(y), cuuint64_t(z)}, strides[2] = {cuuint64_t(ld) * es, cuuint64_t(z > 1 ? group : ld) * es};
    const cuuint32_t box[3] = {cuuint32_t(128 / es), lines, 1}, step[3] = {1, 1, 1};
    const Encode f = encoder();
    return f && f(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), dims, strides, box, step,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether tensor copies can move a matrix: lines on 16-byte boundaries, strides that their maps hold.
bool copies(const void *p, bool f32, int64_t ld, int64_t group, int64_t groups) {
    const int64_t unit = f32 ? 4 : 8;
    return ((uintptr_t)p & 15) == 0 && ld % unit == 0 && (groups == 1 || (group % unit == 0 && group < int64_t(1) << 37));
}

template <int KIND, int END, bool COPY, int PAIR>
cudaError_t launch_of(const ProductArgs &A, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &out, cudaStream_t s) {
    constexpr auto k = k_product<KIND, END, COPY, PAIR>;
    const cudaError_t e = ops_allow_smem<k>(int(kMaxSharedBytes));
    if (e != cudaSuccess) return e;
    uint32_t stages = kStages;
    while (shared_bytes(stages, kEndWarps<COPY>, A.groups) > kMaxSharedBytes) --stages;
    constexpr int kT = kTile<PAIR>;
    const int64_t nt = (A.cols + kT - 1) / kT;
    const int64_t most = (KIND == kOuter ? int64_t((A.inner + kT - 1) / kT) * A.groups : A.rows / kT + A.groups) * nt * A.splits;
    const int64_t pairs = sms() / PAIR;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = PAIR;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(uint32_t(most < pairs ? most : pairs) * PAIR);
    cfg.blockDim = dim3(kThreads<COPY>);
    cfg.dynamicSmemBytes = shared_bytes(stages, kEndWarps<COPY>, A.groups);
    cfg.stream = s;
    cfg.attrs = &at;
    cfg.numAttrs = PAIR > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k, a, b, out, A, stages);
}

// Steps between two additions outside of the tensor cores: 512 products (an error of 5e-7 of the result); 1024 (9e-7) for logits, of which an epilogue makes more
// (at 4096 columns 597 us a 8192 x 16384 table, 619 with 512, 574 with all of them); 8192 (8e-6) where bf16 is made of it.
constexpr int kChunk32 = 512 / kStep, kChunkLoss = 1024 / kStep, kChunk16 = 8192 / kStep;


constexpr int kMostWaves = 4;  // of shares: what their sums' memory is sized for

// How many shares the summed index is cut into, so that few tiles keep the SMs busy: the fewest steps (of 64 products, about 0.3 us) that a pair of CTAs does in
// turn, a share's start and end counted as 6, and the launch that adds the shares as 10 and 0.4 for each.
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

template <int KIND, int END, bool COPY, int PAIR>
cudaError_t launch_split(ProductArgs A, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &out, cudaStream_t s) {
    constexpr int kT = kTile<PAIR>;
    const int64_t height = KIND == kOuter ? A.inner : A.rows, mt = (height + kT - 1) / kT, nt = (A.cols + kT - 1) / kT, tiles = mt * nt * A.groups;
    const int64_t steps = KIND == kOuter ? (A.rows + int64_t(kStep) * A.groups - 1) / (int64_t(kStep) * A.groups) : (A.inner + kStep - 1) / kStep;
    const int shares = END == kStore && A.parts && (KIND == kOuter || !A.offsets) ? shares_of(tiles, steps, sms() / PAIR) : 1;
    CUtensorMap to{};
    if (shares == 1 || !map_of(&to, A.parts, true, kT, kT, kT, kT * kT, tiles * shares, 32)) return launch_of<KIND, END, COPY, PAIR>(A, a, b, out, s);
    ProductArgs P = A;
    P.splits = shares;
    P.out = A.parts;
    P.base = nullptr;
    P.peaks = nullptr;
    P.scale = 1.f;
    P.flags = (A.flags & ~uint32_t(kBase32)) | kOut32 | kOutCopy;
    P.chunk = kChunk32;
    const cudaError_t e = launch_of<KIND, END, COPY, PAIR>(P, a, b, to, s);
    if (e != cudaSuccess) return e;
    const int64_t blocks = (A.groups * height * ((A.cols + 3) / 4) + kSumThreads - 1) / kSumThreads;
    return ops_launch(true, k_sum<kT>, uint32_t(blocks < sms() * 8 ? blocks : sms() * 8), kSumThreads, 0, s, A, shares, height);
}

template <int KIND, int END>
cudaError_t launch(ProductArgs A, cudaStream_t s) {
    CUtensorMap a{}, b{}, out{};
    A.splits = 1;
    A.chunk = END == kLoss ? kChunkLoss : END == kStore && A.flags & kOut32 ? kChunk32 : kChunk16;
    constexpr bool A_MAJOR = KIND != kOuter, B_MAJOR = KIND == kByCols;
    const bool outer = KIND == kOuter, o32 = A.flags & kOut32;
    const int64_t groups = outer ? 1 : A.groups, o_groups = outer ? A.groups : 1;
    if (END != kLoss && copies(A.out, o32, A.ldo, A.o_group, o_groups) &&
        map_of(&out, A.out, o32, A.cols, A.ldo, outer ? A.inner : A.rows, A.o_group, o_groups, 32))
        A.flags |= kOutCopy;
    if (A.rows && copies(A.a, false, A.lda, 0, 1) && copies(A.b, false, A.ldb, A.b_group, groups) &&
        map_of(&a, A.a, false, A.inner, A.lda, A.rows, 0, 1, A_MAJOR ? kLines : kStep) &&
        map_of(&b, A.b, false, B_MAJOR ? A.inner : A.cols, A.ldb, B_MAJOR ? A.cols : outer ? A.rows : A.inner, A.b_group, groups, B_MAJOR ? kLines : kStep))
        return launch_split<KIND, END, true, 2>(A, a, b, out, s);
    return launch_split<KIND, END, false, 1>(A, a, b, out, s);
}

}  // namespace

int32_t product_loss_columns() { return kPart; }

size_t product_parts_bytes() { return size_t(kMostWaves) * (sms() / 2) * kTile<2> * kTile<2> * 4; }

cudaError_t product_launch(ProductKind kind, ProductEnd end, const ProductArgs &A, cudaStream_t s) {
    if (end == kLoss) return launch<kByCols, kLoss>(A, s);
    if (end == kLogitsGrad) return launch<kByCols, kLogitsGrad>(A, s);
    return kind == kByRows ? launch<kByRows, kStore>(A, s) : kind == kByCols ? launch<kByCols, kStore>(A, s) : launch<kOuter, kStore>(A, s);
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
