// Embedding lookup and its gradient (skew_embed_* in include/skewadam.h).
//
//   y[t] = scale W[id_t],   dW[v] = base[v] + scale sum over t with id_t = v of dy[t]
//
// Both are bound by memory. The gradient sorts the tokens by id, stably, so that a row's terms are added
// in the tokens' order whatever runs first; then each warp takes up to kChunk consecutive places of the sorted
// list and kCols columns, and adds up the runs that start there. A run of more places than that (a
// frequent word) is cut at the chunks' ends into pieces, which the warps that finish last add up in their
// order. The same warps write the rows without tokens while their copies are under way.
// One GB300, 50304 x 4096, bf16, 32768 tokens with frequencies of 1 / rank, the kernels alone: lookup 57 us (354 MB, 6.2 TB/s), gradient
// 4 + 9 us of sorting and 112 us for 681 MB (6.1 TB/s). Whole calls: 59, 125, and 94 where the gradient is added in place.
#include "skew_ops.h"

#include <cmath>

namespace skew {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kOwnerBits = 7;
constexpr uint32_t kOwners = 1u << kOwnerBits;  // CTAs of the sort: about as many as there are SMs
constexpr uint32_t kSortRows = 1024;  // rows that a CTA of the sort has counters for at a time
// Most tokens that every CTA of the sort reads itself; more are split by owner first (one launch more, us for the gradient of 50257
// x 64: 2048 tokens 19 and 21, 4096 21 and 22, 8192 26 and 24, 16384 32 and 24).
constexpr int64_t kDirect = 4096;
constexpr int kParts = 4;        // loads of the sort under way at a time
constexpr int kChunk = 32;       // most places of the sorted list to a warp: one to a lane
constexpr int kCols = 256;       // columns to a warp: 8 to a lane
// Chunks are halved, down to 4 places, while there are fewer warps than this (322 tokens of 7266 x 255: 15 us at 4 places, 30 at 32).
constexpr int kFewWarps = 152 * 8;
constexpr uint32_t kFillWarps = 152 * 48;  // at least so many warps, if they find rows without tokens to write
constexpr int kGradThreads = 128;
// Bytes of shared memory that a warp has rows copied to: half in use, half under way. 16 rows of 256 bf16, five CTAs an SM (us for 32768
// tokens of 50304 x 4096 at 12, 16, 20, 24 and 32 rows: 128 126 127 129 139).
constexpr int kRing = 16 * (kCols * 2 + 32);
constexpr uint32_t kJoin = 16;   // pieces that one warp adds up
constexpr int kLookups = 4;      // most tokens to a warp of the lookup (at full occupancy; 2 and 8: 68 and 59 us where 4 take 57)
constexpr int64_t kMaxTokens = int64_t(1) << 30;  // places and what is added to them stay in 32 bits

__device__ __forceinline__ int64_t load_id(const void *ids, bool wide, int64_t t) {
    return wide ? static_cast<const int64_t *>(ids)[t] : static_cast<const int32_t *>(ids)[t];
}

// ---------------------------------------------------------------------------
// Lookup
// ---------------------------------------------------------------------------
struct LookupArgs {
    const void *table, *ids;
    void *out;
    int64_t rows, width, tokens, ld_out;
    uint32_t tiles;
    int32_t per;
    float scale;
    int32_t wide;
};

// A warp to `per` tokens and kCols columns: all rows are under way before the first is stored. VEC: rows of both
// sides start on 16-byte boundaries.
template <bool TF32, bool YF32, bool VEC>
__global__ void __launch_bounds__(kThreads, TF32 ? 5 : 8) k_lookup(const __grid_constant__ LookupArgs A) {
    const int lane = threadIdx.x & 31;
    const int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const int64_t t0 = w / A.tiles * A.per, c0 = (w - w / A.tiles * A.tiles) * kCols;
    if (t0 >= A.tokens) return;
    const int n = int(A.tokens - t0 < A.per ? A.tokens - t0 : A.per);
    int64_t id = lane < n ? load_id(A.ids, A.wide, t0 + lane) : -1;
    if (id >= A.rows) id = -1;
    if constexpr (VEC) {
        const bool on = c0 + 8 * lane < A.width;
        const uint32_t real = __ballot_sync(kFullMask, id >= 0);
        // a lane to a token: where its row is; then the row to the lanes
        const uint64_t mine = reinterpret_cast<uint64_t>(A.table) + (id * A.width + c0) * (TF32 ? 4 : 2);
        Vec8<TF32> v[kLookups];
#pragma unroll
        for (int b = 0; b < kLookups; ++b) {
            const char *row = reinterpret_cast<const char *>(__shfl_sync(kFullMask, mine, b));
            v[b] = Vec8<TF32>{};
            if (on && (real >> b & 1)) v[b] = load8_cached<TF32>(row, 8 * lane);
        }
        char *to = static_cast<char *>(A.out) + (t0 * A.ld_out + c0) * (YF32 ? 4 : 2);
#pragma unroll
        for (int b = 0; b < kLookups; ++b, to += A.ld_out * (YF32 ? 4 : 2))
            if (on && b < n) {
                if (TF32 == YF32 && A.scale == 1.f) {  // as it is
                    st_stream(to + 8 * lane * (YF32 ? 4 : 2), v[b].u[0]);
                    if constexpr (TF32) st_stream(to + 8 * lane * 4 + 16, v[b].u[1]);
                } else {
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = v[b].at(k) * A.scale;
                    store8<YF32>(to, 8 * lane, y);
                }
            }
    } else {  // an element an access (the same lookup with 4095 columns: 133 us)
#pragma unroll
        for (int b = 0; b < kLookups; ++b) {
            const int64_t row = __shfl_sync(kFullMask, id, b);
            if (b >= n) break;
            float v[kCols / 32];
#pragma unroll
            for (int k = 0; k < kCols / 32; ++k) {
                const int64_t c = c0 + 32 * k + lane;
                v[k] = row >= 0 && c < A.width ? load1<TF32>(A.table, row * A.width + c) * A.scale : 0.f;
            }
#pragma unroll
            for (int k = 0; k < kCols / 32; ++k)
                if (c0 + 32 * k + lane < A.width) store1<YF32>(A.out, (t0 + b) * A.ld_out + c0 + 32 * k + lane, v[k]);
        }
    }
}

// ---------------------------------------------------------------------------
// Gradient
// ---------------------------------------------------------------------------
struct EmbedGradArgs {
    const void *ids, *dy, *base;
    void *dw;
    int64_t rows, width, tokens, ld_dy;
    float scale;
    uint32_t own_rows, splits;  // rows of the table to an owner; CTAs of k_embed_split
    int32_t chunk;              // places of the list to a warp: at most kChunk, a power of two
    uint32_t chunks, tiles, fill;  // chunks of the list, tiles of columns, shares of 32 rows to look through for rows without tokens (0: they stay)
    // workspace
    int32_t *first;    // [kOwners * own_rows + 1]: where each row's run starts in the list, by packed()
    uint32_t *start;   // [kOwners + 1][splits]
    uint2 *part;       // [splits][1024]: (id, token)
    int32_t *order;    // [tokens]: the list: tokens by id
    int32_t *key;      // [tokens]: their ids
    uint32_t *done;    // [chunks][3][tiles]: by the chunk where they start, pieces done of kJoin (of a run that came in, of one
                       // that starts there), and such sums done of a run that starts there
    float *piece;      // [2 * chunks][width padded]: sums of pieces that start before a chunk, and in it
};

// The tokens are sorted by (id mod kOwners, id), stably. Rows go round the kOwners CTAs of k_embed_sort, so that
// frequent ids, which are neighbours in most vocabularies, do not meet in one. Over kDirect tokens,
// k_embed_split first divides every 1024 of them by owner; an owner then reads its parts alone. Counts, places
// and orders do not depend on timing, and no CTA waits for another of its launch.
// Where a row's run is in `first`:
__device__ __forceinline__ uint32_t packed(const EmbedGradArgs &A, uint32_t row) { return (row & (kOwners - 1)) * A.own_rows + row / kOwners; }

constexpr uint32_t kNobody = 0xFFFFFFFFu;  // padding: past any owner's rows

__device__ __forceinline__ uint32_t read_id(const EmbedGradArgs &A, bool wide, int64_t t) {
    const int64_t id = t < A.tokens ? load_id(A.ids, wide, t) : -1;
    return id >= 0 && id < A.rows ? uint32_t(id) : kNobody;
}

// Of the lanes in `in`, those whose `bits` low bits of x are this lane's.
__device__ __forceinline__ uint32_t same_lanes(uint32_t in, uint32_t x, int bits) {
    if (in & (in - 1))
        for (int i = 0; i < bits; ++i) {
            const uint32_t ones = __ballot_sync(kFullMask, x >> i & 1);
            in &= x >> i & 1 ? ones : ~ones;
        }
    return in;
}

// Exclusive sum over the threads of a CTA of kSortThreads, and the total.
__device__ __forceinline__ uint32_t cta_exclusive(uint32_t x, uint32_t &total) {
    __shared__ uint32_t warp_sum[kSortWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t upto = x;
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(kFullMask, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    uint32_t sums = warp_sum[lane];  // kSortWarps is 32
    const uint32_t before = __reduce_add_sync(kFullMask, lane < warp ? sums : 0u);
    total = __reduce_add_sync(kFullMask, sums);
    __syncthreads();
    return before + upto - x;
}

// Divides 1024 tokens by owner: part[1024 b ..] holds them by owner, each owner's in the tokens' order;
// start[o][b] is where owner o's begin.
template <bool WIDE>
__global__ void __launch_bounds__(kSortThreads) k_embed_split(const __grid_constant__ EmbedGradArgs A) {
    __shared__ uint32_t hist[kSortWarps][kOwners];
    release_launch_after();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int i = threadIdx.x; i < kSortWarps * kOwners; i += kSortThreads) hist[0][i] = 0;
    const int64_t t = int64_t(blockIdx.x) * kSortThreads + threadIdx.x;
    const uint32_t id = read_id(A, WIDE, t), owner = id & (kOwners - 1);
    const uint32_t same = same_lanes(__ballot_sync(kFullMask, id != kNobody), owner, kOwnerBits);
    __syncthreads();
    if (id != kNobody && lane == __ffs(same) - 1) hist[warp][owner] = __popc(same);
    __syncthreads();
    uint32_t n = 0, all;
    if (threadIdx.x < kOwners)
        for (int w = 0; w < kSortWarps; ++w) n += hist[w][threadIdx.x];
    uint32_t at = cta_exclusive(n, all);
    if (threadIdx.x <= kOwners) A.start[int64_t(threadIdx.x) * A.splits + blockIdx.x] = at;  // at kOwners: all of them
    if (threadIdx.x < kOwners)
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t h = hist[w][threadIdx.x];
            hist[w][threadIdx.x] = at;
            at += h;
        }
    __syncthreads();
    if (id != kNobody) A.part[int64_t(blockIdx.x) * kSortThreads + hist[warp][owner] + __popc(same & ((1u << lane) - 1))] = make_uint2(id, uint32_t(t));
}

// Sorts an owner's tokens by row: counts by (warp, row), each warp its own run of the owner's tokens, then places.
// Rows are taken kSortRows at a time. SPLIT: the tokens come from k_embed_split's parts, else from the ids themselves.
// Walking the tokens twice is much of what many tokens of few columns take (126113 of 12777 x 176, fp32: 49 us, the bytes 16).
template <bool WIDE, bool SPLIT>
__global__ void __launch_bounds__(kSortThreads, 1) k_embed_sort(const __grid_constant__ EmbedGradArgs A) {
    extern __shared__ uint32_t hist[];  // [warp][row], then each warp's next place
    release_launch_after();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t me = blockIdx.x, window = A.own_rows < kSortRows ? A.own_rows : kSortRows;
    const int bits = 32 - __clz(window - 1);
    uint32_t *mine = hist + warp * window;
    for (uint32_t i = threadIdx.x; i < kSortWarps * window; i += kSortThreads) hist[i] = 0;
    if constexpr (SPLIT) wait_launch_before();
    for (uint32_t i = me * kSortThreads + threadIdx.x; i < 3 * A.chunks * A.tiles; i += kOwners * kSortThreads) A.done[i] = 0;
    // a warp's run of tokens: parts [from, to) of k_embed_split, or 32 ids each
    const uint32_t pieces = SPLIT ? A.splits : uint32_t((A.tokens + 31) / 32), share = (pieces + kSortWarps - 1) / kSortWarps;
    const uint32_t from = warp * share < pieces ? warp * share : pieces, to = from + share < pieces ? from + share : pieces;
    // f(row, token, whether there is one) for the run, 32 at a time
    auto each = [&](auto &&f) {
        if constexpr (SPLIT) {
            for (uint32_t p0 = from; p0 < to; p0 += 32) {
                const uint32_t p = p0 + lane;
                const uint32_t a = p < to ? A.start[int64_t(me) * A.splits + p] : 0, b = p < to ? A.start[int64_t(me + 1) * A.splits + p] : 0;
                const uint32_t n = to - p0 < 32 ? to - p0 : 32;
                for (uint32_t q0 = 0; q0 < n; q0 += kParts) {  // the first 32 of kParts parts under way at a time
                    uint2 e[kParts];
#pragma unroll
                    for (int k = 0; k < kParts; ++k) {
                        const uint32_t pa = __shfl_sync(kFullMask, a, (q0 + k) & 31), pb = __shfl_sync(kFullMask, b, (q0 + k) & 31);
                        e[k] = make_uint2(kNobody, 0);
                        if (q0 + k < n && pa + lane < pb) e[k] = A.part[int64_t(p0 + q0 + k) * kSortThreads + pa + lane];
                    }
#pragma unroll
                    for (int k = 0; k < kParts; ++k) {
                        if (q0 + k >= n) break;
                        const uint32_t pa = __shfl_sync(kFullMask, a, q0 + k), pb = __shfl_sync(kFullMask, b, q0 + k);
                        if (pa < pb) f(e[k].x / kOwners, e[k].y, e[k].x != kNobody);
                        for (uint32_t i = pa + 32; i < pb; i += 32) {
                            uint2 more = make_uint2(kNobody, 0);
                            if (i + lane < pb) more = A.part[int64_t(p0 + q0 + k) * kSortThreads + i + lane];
                            f(more.x / kOwners, more.y, more.x != kNobody);
                        }
                    }
                }
            }
        } else {
            for (uint32_t p = from; p < to; p += kParts) {
                uint32_t id[kParts];
#pragma unroll
                for (int k = 0; k < kParts; ++k) id[k] = p + k < to ? read_id(A, WIDE, int64_t(p + k) * 32 + lane) : kNobody;
#pragma unroll
                for (int k = 0; k < kParts; ++k) {
                    const bool in = id[k] != kNobody && (id[k] & (kOwners - 1)) == me;
                    if (__any_sync(kFullMask, in)) f(id[k] / kOwners, (p + k) * 32 + lane, in);
                }
            }
        }
    };
    uint32_t lower = 0;  // tokens of the owners before
    if constexpr (SPLIT) {
        for (uint32_t p = threadIdx.x; p < A.splits; p += kSortThreads) lower += A.start[int64_t(me) * A.splits + p];
    } else {
        for (int64_t t = threadIdx.x; t < A.tokens; t += kSortThreads) {
            const uint32_t id = read_id(A, WIDE, t);
            lower += id != kNobody && (id & (kOwners - 1)) < me;
        }
    }
    uint32_t at0;
    cta_exclusive(lower, at0);
    for (uint32_t v0 = 0; v0 < A.own_rows; v0 += window) {
        const uint32_t n = A.own_rows - v0 < window ? A.own_rows - v0 : window;
        __syncthreads();
        each([&](uint32_t row, uint32_t, bool in) {
            if (in && row - v0 < n) atomicAdd(mine + (row - v0), 1u);
        });
        __syncthreads();
        // places: rows in order, within a row the warps in order
        const uint32_t v = threadIdx.x;  // a thread to a row
        uint32_t total = 0, all;
        if (v < n)
            for (int w = 0; w < kSortWarps; ++w) total += hist[w * window + v];
        uint32_t at = at0 + cta_exclusive(total, all);
        if (v < n) {
            A.first[me * A.own_rows + v0 + v] = int32_t(at);
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t h = hist[w * window + v];
                hist[w * window + v] = at;
                at += h;
            }
        }
        at0 += all;
        __syncthreads();
        each([&](uint32_t row, uint32_t token, bool in) {
            in = in && row - v0 < n;
            const uint32_t same = same_lanes(__ballot_sync(kFullMask, in), row - v0, bits);
            if (in) {
                const uint32_t place = mine[row - v0] + __popc(same & ((1u << lane) - 1));
                A.order[place] = int32_t(token);
                A.key[place] = int32_t(row * kOwners + me);
            }
            __syncwarp();
            if (in && lane == __ffs(same) - 1) mine[row - v0] += __popc(same);
            __syncwarp();
        });
        if (v0 + window < A.own_rows) {  // counters of the next rows
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < kSortWarps * window; i += kSortThreads) hist[i] = 0;
        }
    }
    if (me == kOwners - 1 && threadIdx.x == 0) A.first[kOwners * A.own_rows] = int32_t(at0);
}

// A lane's 8 columns of the tile at c0: consecutive (VEC), or every 32nd.
template <bool VEC>
__device__ __forceinline__ int64_t column(int64_t c0, int k) {
    return VEC ? c0 + 8 * (threadIdx.x & 31) + k : c0 + 32 * k + (threadIdx.x & 31);
}

// dW = base, or zero, over `count` elements from `at` on: whole rows without tokens, one after another, or a part of them.
template <bool F32, bool BASE>
__device__ __forceinline__ void fill(const EmbedGradArgs &A, int64_t at, int64_t count) {
    constexpr int kElem = F32 ? 4 : 2;
    const int lane = threadIdx.x & 31;
    char *to = static_cast<char *>(A.dw) + at * kElem;
    const char *from = BASE ? static_cast<const char *>(A.base) + at * kElem : nullptr;
    auto one = [&](int64_t i) { store1<F32>(A.dw, at + i, BASE ? load1<F32>(A.base, at + i) : 0.f); };
    int64_t done = 0;
    if (!BASE || (((uintptr_t)to ^ (uintptr_t)from) & 15) == 0) {
        const int64_t head = (-(intptr_t)to & 15) / kElem < count ? (-(intptr_t)to & 15) / kElem : count, units = (count - head) * kElem / 16;
        if (lane < head) one(lane);
        to += head * kElem;
        from += BASE ? head * kElem : 0;
        constexpr int kUnits = 8;  // under way at a time
        for (int64_t u = lane; u < units; u += 32 * kUnits) {
            uint4 v[kUnits];
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                v[k] = make_uint4(0, 0, 0, 0);
                if (BASE && u + 32 * k < units) v[k] = ld_stream(from + 16 * (u + 32 * k));
            }
#pragma unroll
            for (int k = 0; k < kUnits; ++k)
                if (u + 32 * k < units) st_stream(to + 16 * (u + 32 * k), v[k]);
        }
        done = head + units * 16 / kElem;
    }
    for (int64_t i = done + lane; i < count; i += 32) one(i);
}

// Stores a row's 8 columns of a lane: without VEC an element at a time, as they are read from shared memory (25090 tokens of 4594 x 4519 to
// fp32: 101 us, where the bytes take 42).
template <bool TF32, bool VEC>
__device__ __forceinline__ void put_row(const EmbedGradArgs &A, int64_t row, int64_t c0, const float (&y)[8]) {
    if constexpr (VEC) {
        if (column<VEC>(c0, 0) < A.width) store8<TF32>(A.dw, row * A.width + column<VEC>(c0, 0), y);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (column<VEC>(c0, k) < A.width) store1<TF32>(A.dw, row * A.width + column<VEC>(c0, k), y[k]);
    }
}

// A piece of a cut run [r0, r1). Of every kJoin pieces the last one done adds them up in order, and of those sums
// the last one done again (two short chains of loads instead of a long one): then `sum` is the run's, and the answer true.
__device__ __forceinline__ bool put_piece(const EmbedGradArgs &A, int r0, int r1, uint32_t chunk, uint32_t tile, float2 (&sum)[4]) {
    const int lane = threadIdx.x & 31;
    const int64_t pitch = int64_t(A.tiles) * kCols;
    const uint32_t first = uint32_t(r0 / A.chunk), last = uint32_t((r1 - 1) / A.chunk);
    auto place = [&](uint32_t c) { return reinterpret_cast<float4 *>(A.piece + (2 * int64_t(c) + (c == first)) * pitch + int64_t(tile) * kCols + 8 * lane); };
    uint32_t at = first + (chunk - first) / kJoin * kJoin, mine = chunk, step = 1, to = last + 1 - at < kJoin ? last + 1 : at + kJoin;
#pragma unroll 1
    for (int level = 0; level < 2; ++level) {  // pieces at, at + step, ... before `to`
        float4 *p = place(mine);
        __stcg(p, make_float4(sum[0].x, sum[0].y, sum[1].x, sum[1].y));
        __stcg(p + 1, make_float4(sum[2].x, sum[2].y, sum[3].x, sum[3].y));
        __threadfence();
        __syncwarp();
        uint32_t before = 0;
        if (lane == 0) before = atomicAdd(A.done + (3 * int64_t(at) + (level ? 2 : at == first)) * A.tiles + tile, 1u);
        before = __shfl_sync(kFullMask, before, 0);
        __threadfence();
        if (before + 1 != (to - at + step - 1) / step) return false;
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] = make_float2(0.f, 0.f);
        for (uint32_t c = at; c < to; c += 4 * step) {
            float4 a[4], b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j * step < to) a[j] = __ldcg(place(c + j * step)), b[j] = __ldcg(place(c + j * step) + 1);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c + j * step < to) {
                    sum[0].x += a[j].x, sum[0].y += a[j].y, sum[1].x += a[j].z, sum[1].y += a[j].w;
                    sum[2].x += b[j].x, sum[2].y += b[j].y, sum[3].x += b[j].z, sum[3].y += b[j].w;
                }
        }
        if (last - first < kJoin) break;  // one sum
        mine = at;
        at = first;
        step = kJoin;
        to = last + 1;
    }
    return true;
}

__device__ __forceinline__ void copy16(uint32_t dst, const char *src, uint32_t bytes) {  // the rest of the 16 as zeros
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// One row's kCols columns in shared memory. VEC: as they lie; else from the 16-byte boundary before them on, so that rows
// of any alignment come by 16-byte copies ([lo, hi) is the whole array: no byte outside of it is read).
template <bool F32, bool VEC>
struct Staged {
    static constexpr int kElem = F32 ? 4 : 2, kBytes = kCols * kElem + (VEC ? 0 : 32);
    // `bytes` of a row from `from` on
    static __device__ __forceinline__ void fetch(uint32_t to, const char *from, int bytes, const char *lo, const char *hi) {
        const int lane = threadIdx.x & 31;
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < kElem / 2; ++j)
                if (16 * lane + 512 * j < bytes) copy16(to + 16 * lane + 512 * j, from + 16 * lane + 512 * j, 16);
        } else {
            const int off = int((uintptr_t)from & 15);
            for (int j = 16 * lane; j < off + bytes; j += 512) {
                const char *src = from - off + j;
                if (src < lo) {  // the array's first bytes
                    for (int i = 0; i < 16; i += kElem)
                        if (src + i >= lo && src + i < hi) {
                            if constexpr (F32)
                                asm volatile("st.shared.u32 [%0], %1;" ::"r"(to + j + i), "r"(*reinterpret_cast<const uint32_t *>(src + i)) : "memory");
                            else
                                asm volatile("st.shared.u16 [%0], %1;" ::"r"(to + j + i), "h"(*reinterpret_cast<const uint16_t *>(src + i)) : "memory");
                        }
                } else {
                    copy16(to + j, src, hi - src < 16 ? uint32_t(hi - src) : 16u);
                }
            }
        }
    }
    // this lane's 8 columns of a row that was fetched to `at`, as they lie; `from`: the low bits of where the row lies
    uint32_t raw[VEC ? 2 * kElem : 8];
    __device__ __forceinline__ void read(const char *at, uint32_t from) {
        const int lane = threadIdx.x & 31;
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < kElem / 2; ++j) {
                const uint4 u = *reinterpret_cast<const uint4 *>(at + 8 * kElem * lane + 16 * j);
                raw[4 * j] = u.x, raw[4 * j + 1] = u.y, raw[4 * j + 2] = u.z, raw[4 * j + 3] = u.w;
            }
        } else {
            at += from & 15;
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if constexpr (F32)
                    raw[k] = reinterpret_cast<const uint32_t *>(at)[32 * k + lane];
                else
                    raw[k] = reinterpret_cast<const uint16_t *>(at)[32 * k + lane];
        }
    }
    __device__ __forceinline__ float2 pair(int k) const {  // columns 2 k and 2 k + 1 of the 8
        if constexpr (F32)
            return make_float2(__uint_as_float(raw[2 * k]), __uint_as_float(raw[2 * k + 1]));
        else if constexpr (VEC)
            return make_float2(bf16_low(raw[k]), bf16_high(raw[k]));
        else
            return make_float2(bf16_low(raw[2 * k]), bf16_low(raw[2 * k + 1]));
    }
};

// A warp to (chunk, tile of columns): it has the chunk's rows of dy copied to shared memory, kRound at a time, writes its
// share of the rows without tokens while they come, and adds up the runs. Warps past the last chunk only do the latter.
// BASE: A.base is there; the rows of it that the round's runs need come by copies of their own.
template <bool TF32, bool YF32, bool VEC, bool BASE>
__global__ void __launch_bounds__(kGradThreads, 5) k_embed_grad(const __grid_constant__ EmbedGradArgs A) {
    using Y = Staged<YF32, VEC>;
    using T = Staged<TF32, VEC>;
    constexpr int kSlot = Y::kBytes + (BASE ? T::kBytes : 0), kRound = kRing / kSlot / 2;  // rows of a round: two rounds at a time are under way or in use
    static_assert(kRound >= 1, "two rounds fit the warp's shared memory");
    extern __shared__ __align__(16) char ring_all[];
    const char *ring = ring_all + (threadIdx.x >> 5) * kRing;
    const uint32_t ring_at = uint32_t(__cvta_generic_to_shared(ring));
    const int lane = threadIdx.x & 31;
    const uint32_t w = blockIdx.x * (kGradThreads / 32) + (threadIdx.x >> 5);
    wait_launch_before();
    const uint32_t chunk = w / A.tiles, tile = w - chunk * A.tiles;
    const int64_t c0 = int64_t(tile) * kCols;
    const int cols = A.width - c0 < kCols ? int(A.width - c0) : kCols;
    const int n = chunk < A.chunks ? A.first[kOwners * A.own_rows] : 0, C = A.chunk;  // places in the list, in a chunk
    const bool some = chunk < A.chunks && int64_t(chunk) * C < n;
    const int s0 = some ? int(chunk) * C : 0, end = !some ? 0 : n - s0 < C ? n : s0 + C, s_mine = s0 + lane;
    const char *dy = static_cast<const char *>(A.dy), *dy_end = dy + ((A.tokens - 1) * A.ld_dy + A.width) * Y::kElem;
    const char *base = static_cast<const char *>(A.base), *base_end = base + A.rows * A.width * T::kElem;
    // a lane to a place of the chunk: its run, and where its row of dy lies; `after`: the row of C places on
    const bool has = s_mine < end;
    const int row = has ? A.key[s_mine] : 0;
    const uint64_t mine = reinterpret_cast<uint64_t>(dy + ((has ? A.order[s_mine] : 0) * A.ld_dy + c0) * Y::kElem);
    const uint64_t after = reinterpret_cast<uint64_t>(dy + ((has && C < n - s_mine ? A.order[s_mine + C] : 0) * A.ld_dy + c0) * Y::kElem);
    const uint32_t run = packed(A, uint32_t(row));
    const int r0 = has ? A.first[run] : 0, r1 = has ? A.first[run + 1] : 0;
    const bool cut = r1 - r0 > C;
    const uint32_t own = __ballot_sync(kFullMask, has && (cut || r0 >= s0));  // others: a run of the chunk before
    const uint32_t ends = __ballot_sync(kFullMask, has && (s_mine + 1 == r1 || (cut && s_mine + 1 == end)));
    const int tail = some ? end - 1 - s0 : 0;  // a run that starts here and is not cut is followed to its end
    const int stop = own ? __shfl_sync(kFullMask, cut ? end : r1, tail) : 0, go = own ? s0 + __ffs(own) - 1 : 0;
    auto in_round = [&](int s) { return stop - s < kRound ? stop - s : kRound; };
    auto ends_from = [&](int s) {  // bit i: a run, or a piece of one, ends at place s + i
        const uint32_t m = s - s0 < 32 ? ends >> (s - s0) : 0;
        return stop > s && stop - s <= 32 ? m | 1u << (stop - 1 - s) : m;
    };
    auto place_row = [&](int i) { return __shfl_sync(kFullMask, row, i < tail ? i : tail); };
    auto fetch = [&](int s, int half) {  // (nothing past `stop`)
        const uint32_t to = ring_at + half * (kRound * kSlot);
        const int count = in_round(s);
        const uint32_t done = ends_from(s);
#pragma unroll 4
        for (int i = 0; i < count; ++i) {
            const int q = s - s0 + i;
            Y::fetch(to + i * kSlot, reinterpret_cast<const char *>(__shfl_sync(kFullMask, q < C ? mine : after, q & (C - 1))), cols * Y::kElem, dy, dy_end);
            if constexpr (BASE)
                if (done >> i & 1)
                    T::fetch(to + i * kSlot + Y::kBytes, base + (int64_t(place_row(q)) * A.width + c0) * T::kElem, cols * T::kElem, base, base_end);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    fetch(go, 0);
    fetch(go + kRound, 1);
    for (uint32_t f = w; f < A.fill; f += gridDim.x * (kGradThreads / 32)) {  // a share of 32 rows
        const uint32_t v0 = f / A.tiles * 32, share = f - f / A.tiles * A.tiles;
        const uint32_t p = packed(A, v0 + lane < A.rows ? v0 + lane : 0);
        uint32_t empty = __ballot_sync(kFullMask, v0 + lane < A.rows && A.first[p] == A.first[p + 1]);
        if constexpr (VEC) {  // a tile of columns of each
            const int64_t fc = int64_t(share) * kCols;
            const int bytes = int(A.width - fc < kCols ? A.width - fc : kCols) * T::kElem;
            const int64_t row0 = (v0 * A.width + fc) * T::kElem + 16 * lane, pitch = A.width * T::kElem;
            while (empty) {
                uint4 v[4][T::kElem / 2];
                int64_t to[4];
                uint32_t there[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    there[i] = empty;
                    to[i] = row0 + (__ffs(empty) - 1) * pitch;
                    empty &= empty - 1;
#pragma unroll
                    for (int j = 0; j < T::kElem / 2; ++j) {
                        v[i][j] = make_uint4(0, 0, 0, 0);
                        if (BASE && there[i] && 16 * lane + 512 * j < bytes) v[i][j] = ld_stream(base + to[i] + 512 * j);
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < T::kElem / 2; ++j)
                        if (there[i] && 16 * lane + 512 * j < bytes) st_stream(static_cast<char *>(A.dw) + to[i] + 512 * j, v[i][j]);
            }
        } else {
            while (empty) {  // runs of them: this share of each
                const int r = __ffs(empty) - 1, n = __ffs(~(empty >> r)) - 1 < 0 ? 32 - r : __ffs(~(empty >> r)) - 1;
                empty &= r + n < 32 ? ~0u << (r + n) : 0u;
                const int64_t all = n * A.width, part = (all / A.tiles + 63) / 64 * 64, at = share * part;
                if (at < all) fill<TF32, BASE>(A, (int64_t(v0) + r) * A.width + at, share + 1 == A.tiles || at + part > all ? all - at : part);
            }
        }
    }
    if (!own) return;
    float2 sum[4] = {};
    int half = 0;
    for (int s = go; s < stop; s += kRound, half ^= 1) {
        const char *at = ring + half * (kRound * kSlot);
        const int count = in_round(s);
        const uint32_t done = ends_from(s);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        constexpr int kRead = VEC && !YF32 ? 4 : 2;
        for (int i0 = 0; i0 < count; i0 += kRead) {
            Y y[kRead];
#pragma unroll
            for (int j = 0; j < kRead; ++j) {
                const int q = s - s0 + i0 + j;
                const uint32_t from = VEC ? 0u : __shfl_sync(kFullMask, uint32_t(q < C ? mine : after), q & (C - 1));
                if (i0 + j < kRound) y[j].read(at + (i0 + j) * kSlot, from);
            }
#pragma unroll
            for (int j = 0; j < kRead; ++j) {
                if (i0 + j >= count) break;
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] = __fadd2_rn(sum[k], y[j].pair(k));
                if (!(done >> (i0 + j) & 1)) continue;
                const int q = s - s0 + i0 + j, from = q < tail ? q : tail;
                const int r = place_row(q), a0 = __shfl_sync(kFullMask, r0, from), a1 = __shfl_sync(kFullMask, r1, from);
                if (a1 - a0 <= C || put_piece(A, a0, a1, chunk, tile, sum)) {
                    float out[8];
                    T b;
                    if constexpr (BASE) b.read(at + (i0 + j) * kSlot + Y::kBytes, uint32_t(reinterpret_cast<uint64_t>(base + (int64_t(r) * A.width + c0) * T::kElem)));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        out[2 * k] = BASE ? fmaf(sum[k].x, A.scale, b.pair(k).x) : sum[k].x * A.scale;
                        out[2 * k + 1] = BASE ? fmaf(sum[k].y, A.scale, b.pair(k).y) : sum[k].y * A.scale;
                    }
                    put_row<TF32, VEC>(A, r, c0, out);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] = make_float2(0.f, 0.f);
            }
        }
        __syncwarp();
        fetch(s + 2 * kRound, half);
    }
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
constexpr uint32_t kFlags = SKEW_EMBED_TABLE_FP32 | SKEW_EMBED_ACT_FP32 | SKEW_EMBED_IDS_64;

int check(const skew_embed_config_t *c, int64_t tokens) {
    if (!c) return ops_fail(SKEW_EINVAL, "config is NULL");
    if (c->rows < 1 || c->rows > INT32_MAX) return ops_fail(SKEW_EINVAL, "rows must be in [1, 2^31)");
    if (c->width < 1 || c->width > int64_t(1) << 20) return ops_fail(SKEW_EINVAL, "width must be in [1, 2^20]");
    if (!std::isfinite(c->scale)) return ops_fail(SKEW_EINVAL, "scale must be finite");
    if (c->flags & ~kFlags) return ops_fail(SKEW_EINVAL, "unknown flags");
    if (tokens < 0 || tokens > kMaxTokens) return ops_fail(SKEW_EINVAL, "tokens must be in [0, 2^30]");
    return SKEW_OK;
}

int check_ptr(const char *what, const void *p, uintptr_t es, bool needed) {
    if ((needed && !p) || ((uintptr_t)p & (es - 1))) return ops_fail(SKEW_EINVAL, "%s must be a device pointer aligned to its type", what);
    return SKEW_OK;
}

struct Layout {
    uint32_t chunk, chunks, tiles, own_rows, splits;
    size_t first, start, part, order, key, done, piece, bytes;
};

Layout layout(const skew_embed_config_t *c, int64_t tokens) {
    Layout L{};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    L.own_rows = uint32_t((c->rows + kOwners - 1) / kOwners);
    L.splits = tokens > kDirect ? uint32_t((tokens + kSortThreads - 1) / kSortThreads) : 0;
    L.tiles = uint32_t((c->width + kCols - 1) / kCols);
    // few tokens: shorter chunks, so that they spread over the SMs
    L.chunk = kChunk;
    while (L.chunk > 4 && (tokens + L.chunk - 1) / L.chunk * L.tiles < kFewWarps) L.chunk >>= 1;
    L.chunks = uint32_t((tokens + L.chunk - 1) / L.chunk);
    L.first = take((size_t(L.own_rows) * kOwners + 1) * 4);
    L.start = take(size_t(L.splits) * (kOwners + 1) * 4);
    L.part = take(size_t(L.splits) * kSortThreads * 8);
    L.order = take(size_t(tokens) * 4);
    L.key = take(size_t(tokens) * 4);
    L.done = take(size_t(L.chunks) * L.tiles * 12);
    L.piece = take(size_t(L.chunks) * 2 * L.tiles * kCols * 4);
    L.bytes = at;
    return L;
}

template <bool TF32, bool YF32>
cudaError_t launch_lookup(const LookupArgs &A, bool vec, cudaStream_t s) {
    const int64_t warps = (A.tokens + A.per - 1) / A.per * A.tiles;
    const uint32_t grid = uint32_t((warps + kWarps - 1) / kWarps);
    return vec ? ops_launch(false, k_lookup<TF32, YF32, true>, grid, kThreads, 0, s, A) : ops_launch(false, k_lookup<TF32, YF32, false>, grid, kThreads, 0, s, A);
}

template <bool WIDE, bool SPLIT>
cudaError_t launch_sort_of(const EmbedGradArgs &A, cudaStream_t s) {
    constexpr auto k = k_embed_sort<WIDE, SPLIT>;
    const cudaError_t e = ops_allow_smem<k>(kSortWarps * (int)kSortRows * 4);
    if (e != cudaSuccess) return e;
    return ops_launch(SPLIT, k, kOwners, kSortThreads, size_t(kSortWarps) * (A.own_rows < kSortRows ? A.own_rows : kSortRows) * 4, s, A);
}

template <bool WIDE>
cudaError_t launch_sort(const EmbedGradArgs &A, cudaStream_t s) {
    if (!A.splits) return launch_sort_of<WIDE, false>(A, s);
    const cudaError_t e = ops_launch(false, k_embed_split<WIDE>, A.splits, kSortThreads, 0, s, A);
    return e != cudaSuccess ? e : launch_sort_of<false, true>(A, s);
}

template <bool TF32, bool YF32, bool VEC, bool BASE>
cudaError_t launch_grad_of(const EmbedGradArgs &A, cudaStream_t s) {
    constexpr auto k = k_embed_grad<TF32, YF32, VEC, BASE>;
    constexpr int kSmem = kGradThreads / 32 * kRing;
    // warps of their own for the rows without tokens where there are few chunks
    uint32_t warps = A.fill < kFillWarps ? A.fill : kFillWarps;
    if (warps < A.chunks * A.tiles) warps = A.chunks * A.tiles;
    if (!warps) return cudaSuccess;
    const cudaError_t e = ops_allow_smem<k>(kSmem);
    return e != cudaSuccess ? e : ops_launch(true, k, (warps + kGradThreads / 32 - 1) / (kGradThreads / 32), kGradThreads, kSmem, s, A);
}

template <bool TF32, bool YF32>
cudaError_t launch_grad(const EmbedGradArgs &A, bool vec, cudaStream_t s) {
    return vec ? (A.base ? launch_grad_of<TF32, YF32, true, true>(A, s) : launch_grad_of<TF32, YF32, true, false>(A, s))
               : (A.base ? launch_grad_of<TF32, YF32, false, true>(A, s) : launch_grad_of<TF32, YF32, false, false>(A, s));
}

}  // namespace
}  // namespace skew

using namespace skew;

extern "C" {

int skew_embed_lookup(const skew_embed_config_t *c, const void *table, const void *ids, int64_t tokens, void *out, int64_t ld_out, void *stream) {
    if (const int rc = check(c, tokens)) return rc;
    const bool tf = c->flags & SKEW_EMBED_TABLE_FP32, yf = c->flags & SKEW_EMBED_ACT_FP32, wide = c->flags & SKEW_EMBED_IDS_64;
    int rc;
    if ((rc = check_ptr("table", table, tf ? 4 : 2, true)) || (rc = check_ptr("ids", ids, wide ? 8 : 4, tokens > 0)) || (rc = check_ptr("out", out, yf ? 4 : 2, tokens > 0)))
        return rc;
    if (ld_out < c->width || ld_out > int64_t(1) << 31) return ops_fail(SKEW_EINVAL, "row stride must be in [width, 2^31]");
    if (!tokens) return SKEW_OK;
    // few tokens: one to a warp, so that they spread
    const int64_t tiles = (c->width + kCols - 1) / kCols;
    int per = kLookups;
    while (per > 1 && (tokens + per - 1) / per * tiles < int64_t(ops_sm_count()) * 32) per >>= 1;
    if ((tokens + per - 1) / per * tiles > int64_t(INT32_MAX) * kWarps) return ops_fail(SKEW_EINVAL, "too many tokens for this width");
    const LookupArgs A{table, ids, out, c->rows, c->width, tokens, ld_out, (uint32_t)tiles, per, c->scale, wide};
    const bool vec = c->width % 8 == 0 && ld_out % (yf ? 4 : 8) == 0 && (((uintptr_t)table | (uintptr_t)out) & 15) == 0;
    cudaStream_t s = (cudaStream_t)stream;
    return ops_cuda(tf ? (yf ? launch_lookup<true, true>(A, vec, s) : launch_lookup<true, false>(A, vec, s))
                       : (yf ? launch_lookup<false, true>(A, vec, s) : launch_lookup<false, false>(A, vec, s)), "k_lookup");
}

size_t skew_embed_workspace_bytes(const skew_embed_config_t *c, int64_t tokens) { return check(c, tokens) == SKEW_OK ? layout(c, tokens).bytes : 0; }

int skew_embed_grad(const skew_embed_config_t *c, const void *ids, int64_t tokens, const void *dout, int64_t ld_dout, const void *base, void *dtable,
                    void *workspace, size_t workspace_bytes, void *stream) {
    if (const int rc = check(c, tokens)) return rc;
    const bool tf = c->flags & SKEW_EMBED_TABLE_FP32, yf = c->flags & SKEW_EMBED_ACT_FP32, wide = c->flags & SKEW_EMBED_IDS_64;
    int rc;
    if ((rc = check_ptr("ids", ids, wide ? 8 : 4, tokens > 0)) || (rc = check_ptr("dout", dout, yf ? 4 : 2, tokens > 0)) ||
        (rc = check_ptr("base", base, tf ? 4 : 2, false)) || (rc = check_ptr("dtable", dtable, tf ? 4 : 2, true)))
        return rc;
    if (ld_dout < c->width || ld_dout > int64_t(1) << 31) return ops_fail(SKEW_EINVAL, "row stride must be in [width, 2^31]");
    const Layout L = layout(c, tokens);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < L.bytes)
        return ops_fail(SKEW_EINVAL, "workspace must be 256-byte aligned and at least %zu bytes", L.bytes);
    const int64_t fill = base == dtable ? 0 : (c->rows + 31) / 32 * L.tiles;
    if (fill > INT32_MAX || int64_t(L.chunks) * L.tiles > INT32_MAX / 3) return ops_fail(SKEW_EINVAL, "too many rows or tokens for this width");
    EmbedGradArgs A{};
    char *ws = (char *)workspace;
    A.ids = ids;
    A.dy = dout;
    A.base = base;
    A.dw = dtable;
    A.rows = c->rows;
    A.width = c->width;
    A.tokens = tokens;
    A.ld_dy = ld_dout;
    A.scale = c->scale;
    A.chunks = L.chunks;
    A.tiles = L.tiles;
    A.fill = (uint32_t)fill;
    A.first = (int32_t *)(ws + L.first);
    A.order = (int32_t *)(ws + L.order);
    A.key = (int32_t *)(ws + L.key);
    A.done = (uint32_t *)(ws + L.done);
    A.piece = (float *)(ws + L.piece);
    A.own_rows = L.own_rows;
    A.splits = L.splits;
    A.chunk = (int32_t)L.chunk;
    A.start = (uint32_t *)(ws + L.start);
    A.part = (uint2 *)(ws + L.part);
    const bool vec = c->width % 8 == 0 && ld_dout % (yf ? 4 : 8) == 0 && (((uintptr_t)dout | (uintptr_t)base | (uintptr_t)dtable) & 15) == 0;
    cudaStream_t s = (cudaStream_t)stream;
    if ((rc = ops_cuda(wide ? launch_sort<true>(A, s) : launch_sort<false>(A, s), "k_embed_sort"))) return rc;
    return ops_cuda(tf ? (yf ? launch_grad<true, true>(A, vec, s) : launch_grad<true, false>(A, vec, s))
                       : (yf ? launch_grad<false, true>(A, vec, s) : launch_grad<false, false>(A, vec, s)), "k_embed_grad");
}

}  // extern "C"
