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

#include <atomic>

#include "skew_ops.h"

namespace skew {
namespace {

constexpr int kLines = 128;                    // of each operand, in a stage
constexpr int kStep = 64;                      // elements of the summed index in a stage
constexpr uint32_t kOperandBytes = kLines * kStep * 2;
constexpr uint32_t kStageBytes = 2 * kOperandBytes;
constexpr int kStages = 6;
constexpr int kMaxGroups = 1024;
constexpr int kTileRows = 128, kTileCols = 128;
constexpr int kAccCols = 2 * kTileCols;        // of tensor memory: two tiles of sums
constexpr int kBand = 16;                      // tiles of rows that are walked together (A and B of 152 tiles then stay in L2)

constexpr int kLoadWarps = 8, kEndWarps = 4;
constexpr int kMulWarp = 0, kFirstEnd = 4, kFirstLoad = 8;  // warps 4 to 7 read lanes 32 (warp % 4) on of tensor memory
constexpr int kThreads = 32 * (kFirstLoad + kLoadWarps);

struct Shared {
    uint64_t full[kStages], empty[kStages], sums[2], freed[2];
    uint32_t acc;                     // where the sums are in tensor memory
    uint32_t gave_up;
    int32_t total[kThreads / 32];
    int32_t begin[kMaxGroups + 1];    // first row of each group; the end of the last
    int32_t tile[kMaxGroups + 1];     // tiles of rows before it (BY_ROWS, BY_COLS)
};

constexpr size_t kSharedBytes = 1024 + size_t(kStages) * kStageBytes + sizeof(Shared);

__device__ uint32_t g_status;  // 1: a wait gave up

__device__ __forceinline__ uint32_t shared_address(const void *p) { return uint32_t(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void bar_init(uint64_t *b, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(shared_address(b)), "r"(count) : "memory");
}

__device__ __forceinline__ void bar_arrive(uint64_t *b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(shared_address(b)) : "memory");
}

__device__ __forceinline__ bool bar_poll(uint64_t *b, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
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

// ---------------------------------------------------------------------------
// Tiles
// ---------------------------------------------------------------------------
struct Tile {
    int32_t group, m0, n0;        // first row (of the matrices' `rows`, or OUTER's i) and column
    int32_t r0, r1;               // the group's rows
    int32_t steps;                // of the summed index
};

// The groups' rows, in order and within [0, rows) whatever `offsets` hold, and the tiles before each.
template <int KIND>
__device__ __forceinline__ void groups_of(const ProductArgs &A, Shared &S) {
    const int G = A.groups, per = (G + kThreads) / kThreads, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
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
        auto tiles = [&](int i) { return i < G ? (S.begin[i + 1] - S.begin[i] + kTileRows - 1) / kTileRows : 0; };
        int n = 0;
        for (int i = i0; i < i1; ++i) n += tiles(i);
        n = scan(n, both);
        for (int i = i0; i < i1; ++i) S.tile[i] = n, n += tiles(i);
    }
    __syncthreads();
}

// The CTA's tiles, one after another: blockIdx.x, + gridDim.x, ...
template <int KIND>
struct Walk {
    const ProductArgs &A;
    const Shared &S;
    int64_t at, all;
    int64_t each;      // OUTER: tiles of a group
    int32_t nt, group;

    __device__ __forceinline__ Walk(const ProductArgs &a, const Shared &s) : A(a), S(s), at(blockIdx.x), group(0) {
        nt = (A.cols + kTileCols - 1) / kTileCols;
        if (KIND == kOuter) {
            each = int64_t((A.inner + kTileRows - 1) / kTileRows) * nt;
            all = each * A.groups;
        } else {
            all = int64_t(S.tile[A.groups]) * nt;
        }
    }

    __device__ __forceinline__ bool next(Tile &t) {
        if (at >= all) return false;
        int64_t here;
        int mt;
        if (KIND == kOuter) {
            group = int(at / each);
            here = at - group * each;
            mt = (A.inner + kTileRows - 1) / kTileRows;
        } else {
            const int row = int(at / nt);  // tiles of rows before this one's, over all groups: its group is the last that begins at or before it
            int lo = group, hi = A.groups;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (S.tile[mid] <= row) lo = mid; else hi = mid;
            }
            group = lo;
            here = at - int64_t(S.tile[group]) * nt;
            mt = S.tile[group + 1] - S.tile[group];
        }
        const int64_t span = int64_t(kBand) * nt;
        const int band = int(here / span), first = band * kBand, in = min(kBand, mt - first), left = int(here - band * span);
        t.group = group;
        t.r0 = S.begin[group];
        t.r1 = S.begin[group + 1];
        t.m0 = (first + left % in) * kTileRows + (KIND == kOuter ? 0 : t.r0);
        t.n0 = left / in * kTileCols;
        t.steps = ((KIND == kOuter ? t.r1 - t.r0 : A.inner) + kStep - 1) / kStep;
        at += gridDim.x;
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
                                  uint32_t(kTileCols >> 3) << 17 | uint32_t(kTileRows >> 4) << 24;

__device__ __forceinline__ void multiply(uint32_t acc, uint64_t a, uint64_t b, uint32_t instruction, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(acc), "l"(a), "l"(b), "r"(instruction), "r"(uint32_t(add)) : "memory");
}

// Arrives once what was issued before is done.
__device__ __forceinline__ void commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(shared_address(bar)) : "memory");
}

__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 lanes: x[c] of this lane.
__device__ __forceinline__ void read_sums(uint32_t at, float (&x)[32]) {
    __syncwarp();
    uint32_t *u = reinterpret_cast<uint32_t *>(x);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]),
          "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]),
          "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(at) : "memory");
}

// ---------------------------------------------------------------------------
// What becomes of the sums
// ---------------------------------------------------------------------------
__device__ __forceinline__ float exp2_of(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// out = base + scale * x for 32 columns of a row, of which `n` are there.
template <bool O32, bool B32>
__device__ __forceinline__ void store_sums(const ProductArgs &A, int64_t at, int n, bool vec, const float (&x)[32]) {
    if (n >= 32 && vec) {
#pragma unroll
        for (int c = 0; c < 32; c += 8) {
            float y[8];
            if (A.base) {
                const Vec8<B32> b = load8_cached<B32>(A.base, at + c);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = fmaf(x[c + i], A.scale, b.at(i));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = x[c + i] * A.scale;
            }
            char *q = const_cast<char *>(elem_ptr<O32>(A.out, at + c));
            if constexpr (O32) {
                reinterpret_cast<float4 *>(q)[0] = make_float4(y[0], y[1], y[2], y[3]);
                reinterpret_cast<float4 *>(q)[1] = make_float4(y[4], y[5], y[6], y[7]);
            } else {
                *reinterpret_cast<uint4 *>(q) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
            }
        }
        return;
    }
#pragma unroll
    for (int c = 0; c < 32; ++c)
        if (c < n) store1<O32>(A.out, at + c, A.base ? fmaf(x[c], A.scale, load1<B32>(A.base, at + c)) : x[c] * A.scale);
}

__device__ __forceinline__ int64_t target_of(const ProductArgs &A, int64_t row) {  // -1: none
    const int64_t v = A.flags & kIds64 ? static_cast<const int64_t *>(A.targets)[row] : static_cast<const int32_t *>(A.targets)[row];
    return v < 0 || v >= A.vocab ? -1 : v;
}

constexpr float kLog2e = 1.44269504088896340736f;

// A tile's 32 rows of one warp, read from tensor memory at `acc` (`none`: the sums are zero).
template <int KIND, int END>
__device__ __forceinline__ void end_tile(const ProductArgs &A, const Tile &t, uint32_t acc, bool none, int row_in_tile) {
    const int64_t row = t.m0 + row_in_tile;
    const bool mine = row < (KIND == kOuter ? A.inner : t.r1);
    float x[32];
    if constexpr (END == kStore) {
        const int64_t at = t.group * A.o_group * (KIND == kOuter) + row * A.ldo;
        for (int c = 0; c < kTileCols && t.n0 + c < A.cols; c += 32) {
            if (none) {
#pragma unroll
                for (int i = 0; i < 32; ++i) x[i] = 0.f;
            } else {
                read_sums(acc + c, x);
            }
            const int n = A.cols - t.n0 - c;
            const bool vec = A.flags & kOutVec;
            if (!mine) {
            } else if (A.flags & kOut32) {
                store_sums<true, true>(A, at + t.n0 + c, n, vec, x);
            } else if (A.flags & kBase32) {
                store_sums<false, true>(A, at + t.n0 + c, n, vec, x);
            } else {
                store_sums<false, false>(A, at + t.n0 + c, n, vec, x);
            }
        }
    } else if constexpr (END == kLoss) {
        // in powers of two: exp(x) = 2^(x log2 e)
        const float scale2 = A.scale * kLog2e;
        const int64_t target = mine ? target_of(A, row) : -1;
        float top = -INFINITY, sum = 0.f;
        for (int c = 0; c < kTileCols && t.n0 + c < A.cols; c += 32) {
            read_sums(acc + c, x);
            const int n = A.cols - t.n0 - c;
            const int64_t at = target - t.n0 - c;
            if (at >= 0 && at < 32 && target >= 0) {
                float p = 0.f;
#pragma unroll
                for (int i = 0; i < 32; ++i) p = at == i ? x[i] : p;
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
        }
        if (mine) A.part[row * A.tiles + t.n0 / kTileCols] = make_float2(top, sum);
    } else {
        const float scale2 = A.scale * kLog2e;
        const int64_t target = mine ? target_of(A, row) : -1;
        const float g = target >= 0 ? A.dloss[row] : 0.f, lse2 = target >= 0 ? A.lse[row] * kLog2e : 0.f;
        for (int c = 0; c < kTileCols && t.n0 + c < A.cols; c += 32) {
            read_sums(acc + c, x);
            const int64_t at = target - A.first - t.n0 - c;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float p = exp2_of(fmaf(x[i], scale2, -lse2)) - (at == i ? 1.f : 0.f);
                x[i] = target >= 0 ? p * g : 0.f;
            }
            const int n = mine ? A.cols - t.n0 - c : 0;
            uint16_t *q = static_cast<uint16_t *>(A.out) + row * A.ldo + t.n0 + c;
#pragma unroll
            for (int i = 0; i < 32; i += 8) {  // the matrix's lines are 16-byte aligned and have room for whole units
                if (i < n)
                    *reinterpret_cast<uint4 *>(q + i) = make_uint4(pack_bf16(x[i], x[i + 1]), pack_bf16(x[i + 2], x[i + 3]), pack_bf16(x[i + 4], x[i + 5]), pack_bf16(x[i + 6], x[i + 7]));
            }
        }
    }
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

template <int KIND, int END>
__global__ void __launch_bounds__(kThreads, 1) k_product(const ProductArgs A) {
    extern __shared__ char raw[];
    char *const ring = raw + (1024 - (shared_address(raw) & 1023)) % 1024;
    Shared &S = *reinterpret_cast<Shared *>(ring + size_t(kStages) * kStageBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) bar_init(&S.full[i], kLoadWarps), bar_init(&S.empty[i], 1);
        for (int i = 0; i < 2; ++i) bar_init(&S.sums[i], 1), bar_init(&S.freed[i], kEndWarps);
        S.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(shared_address(&S.acc)), "n"(kAccCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    groups_of<KIND>(A, S);
    before_sync();
    __syncthreads();
    after_sync();
    const uint32_t acc = S.acc;
    constexpr bool A_MAJOR = KIND != kOuter, B_MAJOR = KIND == kByCols;
    Walk<KIND> walk(A, S);
    Tile t;

    if (warp >= kFirstLoad) {
        const int w = (warp - kFirstLoad) % (kLoadWarps / 2);
        const bool second = warp - kFirstLoad >= kLoadWarps / 2;
        uint32_t n = 0;
        bool ok = true;
        while (ok && walk.next(t)) {
            const uint16_t *b = static_cast<const uint16_t *>(A.b) + t.group * A.b_group * (KIND != kOuter);
            for (int k = 0; k < t.steps; ++k, ++n) {
                const int s = n % kStages;
                if (n >= kStages && !(ok = bar_wait(&S.empty[s], (n / kStages - 1) & 1, S))) break;
                char *to = ring + size_t(s) * kStageBytes;
                const int64_t s0 = (KIND == kOuter ? t.r0 : 0) + int64_t(k) * kStep, s_end = KIND == kOuter ? t.r1 : A.inner;
                if (!second)
                    load_lines<A_MAJOR>(static_cast<const uint16_t *>(A.a), A.lda, t.m0, KIND == kOuter ? A.inner : t.r1, s0, s_end, to, w, lane);
                else
                    load_lines<B_MAJOR>(b, A.ldb, t.n0, A.cols, s0, s_end, to + kOperandBytes, w, lane);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (!lane) bar_arrive(&S.full[s]);
            }
        }
    } else if (warp == kMulWarp) {
        if (!lane) {
            uint32_t n = 0, tiles = 0;
            bool ok = true;
            while (ok && walk.next(t)) {
                if (!t.steps) continue;
                const uint32_t half = tiles & 1, to = acc + half * kTileCols;
                if (tiles >= 2 && !(ok = bar_wait(&S.freed[half], (tiles / 2 - 1) & 1, S))) break;
                after_sync();
                for (int k = 0; k < t.steps; ++k, ++n) {
                    const int s = n % kStages;
                    if (!(ok = bar_wait(&S.full[s], n / kStages & 1, S))) break;
                    after_sync();
                    const uint32_t at = shared_address(ring + size_t(s) * kStageBytes);
                    const uint64_t a = operand<A_MAJOR>(at), b = operand<B_MAJOR>(at + kOperandBytes);
#pragma unroll
                    for (int i = 0; i < kStep / 16; ++i)
                        multiply(to, a + i * kNext16<A_MAJOR>, b + i * kNext16<B_MAJOR>, kInstruction<A_MAJOR, B_MAJOR>, k | i);
                    commit(&S.empty[s]);
                }
                if (ok) commit(&S.sums[half]);
                ++tiles;
            }
            // what was issued ends before the tensor memory is given back
            if (!ok && n) {
                const uint32_t s = (n - 1) % kStages;
                for (int i = 0; i < 1 << 20 && !bar_poll(&S.empty[s], (n - 1) / kStages & 1); ++i) {}
            }
        }
    } else if (warp >= kFirstEnd && warp < kFirstEnd + kEndWarps) {
        const int q = warp - kFirstEnd;
        uint32_t tiles = 0;
        bool ok = true;
        while (ok && walk.next(t)) {
            const uint32_t half = tiles & 1;
            if (t.steps) {
                if (!(ok = bar_wait(&S.sums[half], tiles / 2 & 1, S))) break;
                after_sync();
            } else if (KIND == kOuter && A.base == A.out) {
                continue;
            }
            end_tile<KIND, END>(A, t, acc + half * kTileCols + (uint32_t(q * 32) << 16), !t.steps, q * 32 + lane);
            if (t.steps) {
                before_sync();
                __syncwarp();
                if (!lane) bar_arrive(&S.freed[half]);
                ++tiles;
            }
        }
        if (KIND != kOuter && END == kStore && A.offsets) clear_rows(A, S, q, lane);
    }
    before_sync();
    __syncwarp();
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(acc), "n"(kAccCols) : "memory");
}

template <int KIND, int END>
cudaError_t launch(const ProductArgs &A, cudaStream_t s) {
    constexpr auto k = k_product<KIND, END>;
    const cudaError_t e = ops_allow_smem<k>(int(kSharedBytes));
    if (e != cudaSuccess) return e;
    const int64_t nt = (A.cols + kTileCols - 1) / kTileCols;
    const int64_t most = (KIND == kOuter ? int64_t((A.inner + kTileRows - 1) / kTileRows) * A.groups : A.rows / kTileRows + A.groups) * nt;
    const int64_t sms = ops_sm_count();
    return ops_launch(false, k, uint32_t(most < sms ? most : sms), kThreads, kSharedBytes, s, A);
}

}  // namespace

int32_t product_loss_columns() { return kTileCols; }

cudaError_t product_launch(ProductKind kind, ProductEnd end, ProductArgs &A, cudaStream_t s) {
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
