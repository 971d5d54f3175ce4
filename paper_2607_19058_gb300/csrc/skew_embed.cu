// Embedding lookup and its gradient (skew_embed_* in include/skewadam.h).
//
//   y[t] = scale W[id_t],   dW[v] = base[v] + scale sum over t with id_t = v of dy[t]
//
// Both are bound by memory. The gradient sorts the tokens by id, stably, so that a row's terms are added
// in the tokens' order whatever runs first; then each warp takes kChunk consecutive places of the sorted
// list and kCols columns, and adds up the runs that start there. A run of more than kChunk tokens (a
// frequent word) is cut at the chunks' ends into pieces; the warp that finishes last adds the pieces up in
// their order. Rows without tokens are written by warps of their own.
#include "skew_ops.h"

#include <cmath>

namespace skew {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kOwnerBits = 7;
constexpr uint32_t kOwners = 1u << kOwnerBits;  // CTAs of the sort: about as many as there are SMs
constexpr uint32_t kSortRows = 1024;  // rows that a CTA of the sort has counters for at a time
constexpr int64_t kDirect = 2048;     // most tokens that every CTA of the sort reads itself
constexpr int kParts = 4;
constexpr int kChunk = 32;       // most places of the sorted list to a warp: one to a lane
constexpr int kCols = 256;       // columns to a warp: 8 to a lane
constexpr int kFewWarps = 152 * 8;
constexpr int kFill = 8;         // rows of the table to a warp that writes those without tokens
constexpr int kJoin = 4;         // pieces that are under way at a time where they are added up
constexpr int kLookups = 8;      // most tokens to a warp of the lookup

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
__global__ void __launch_bounds__(kThreads) k_lookup(const __grid_constant__ LookupArgs A) {
    const int lane = threadIdx.x & 31;
    const int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const int64_t t0 = w / A.tiles * A.per, c0 = (w - w / A.tiles * A.tiles) * kCols;
    if (t0 >= A.tokens) return;
    const int n = int(A.tokens - t0 < A.per ? A.tokens - t0 : A.per);
    int64_t id = lane < n ? load_id(A.ids, A.wide, t0 + lane) : -1;
    if (id >= A.rows) id = -1;
    if constexpr (VEC) {
        const int64_t c = c0 + 8 * lane;
        const bool on = c < A.width;
        const uint32_t real = __ballot_sync(kFullMask, id >= 0);
        Vec8<TF32> v[kLookups];
#pragma unroll
        for (int b = 0; b < kLookups; ++b) {
            const int64_t row = __shfl_sync(kFullMask, id, b);
            if (on && row >= 0) v[b] = load8_cached<TF32>(A.table, row * A.width + c);
        }
#pragma unroll
        for (int b = 0; b < kLookups; ++b)
            if (on && b < n) {
                float y[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = real >> b & 1 ? v[b].at(k) * A.scale : 0.f;
                store8<YF32>(A.out, (t0 + b) * A.ld_out + c, y);
            }
    } else {
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
    int32_t wide;
    uint32_t own_rows, splits;  // rows of the table to an owner; CTAs of k_embed_split
    int32_t chunk;              // places of the list to a warp: at most kChunk, a power of two
    uint32_t chunks, tiles, fill;  // chunks of the list, tiles of columns, warps' shares of the rows without tokens (0: they stay)
    // workspace
    int32_t *first;    // [kOwners * own_rows + 1]: where each row's run starts in the list, by packed()
    uint32_t *start;   // [kOwners + 1][splits]
    uint2 *part;       // [splits][1024]: (id, token)
    int32_t *order;    // [tokens]: the list: tokens by id
    int32_t *key;      // [tokens]: their ids
    uint32_t *done;    // [chunks * tiles]: pieces done of the run that is cut first at a chunk's end
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
    for (uint32_t i = me * kSortThreads + threadIdx.x; i < A.chunks * A.tiles; i += kOwners * kSortThreads) A.done[i] = 0;
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
            for (uint32_t p = from; p < to; ++p) {
                const uint32_t id = read_id(A, WIDE, int64_t(p) * 32 + lane);
                const bool in = id != kNobody && (id & (kOwners - 1)) == me;
                if (__any_sync(kFullMask, in)) f(id / kOwners, p * 32 + lane, in);
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

// A lane's 8 elements of a row, as they are loaded.
template <bool F32, bool VEC>
struct Cells {
    Vec8<F32> v;
    __device__ __forceinline__ void load(const void *p, int64_t row_at, int64_t c0, int64_t width) {
        if (column<true>(c0, 0) < width) v = load8<F32>(p, row_at + column<true>(c0, 0));
    }
    __device__ __forceinline__ float at(int k) const { return v.at(k); }
};
template <bool F32>
struct Cells<F32, false> {
    float v[8];
    __device__ __forceinline__ void load(const void *p, int64_t row_at, int64_t c0, int64_t width) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (column<false>(c0, k) < width) v[k] = load1<F32>(p, row_at + column<false>(c0, k));
    }
    __device__ __forceinline__ float at(int k) const { return v[k]; }
};

// Stores a row's 8 columns of a lane.
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

// A piece of a cut run [r0, r1) of `row`; the last piece done adds them all, in order.
template <bool TF32, bool VEC>
__device__ __forceinline__ void put_piece(const EmbedGradArgs &A, int row, int r0, int r1, uint32_t chunk, uint32_t tile, const float (&sum)[8]) {
    const int lane = threadIdx.x & 31;
    const int64_t pitch = int64_t(A.tiles) * kCols;
    const uint32_t first = uint32_t(r0 / A.chunk), last = uint32_t((r1 - 1) / A.chunk);
    auto place = [&](uint32_t c) { return reinterpret_cast<float4 *>(A.piece + (2 * int64_t(c) + (c == first)) * pitch + int64_t(tile) * kCols + 8 * lane); };
    float4 *p = place(chunk);
    __stcg(p, make_float4(sum[0], sum[1], sum[2], sum[3]));
    __stcg(p + 1, make_float4(sum[4], sum[5], sum[6], sum[7]));
    __threadfence();
    __syncwarp();
    uint32_t before = 0;
    if (lane == 0) before = atomicAdd(A.done + int64_t(first) * A.tiles + tile, 1u);
    before = __shfl_sync(kFullMask, before, 0);
    if (before != last - first) return;
    __threadfence();
    float all[8] = {};
    for (uint32_t c = first; c <= last; c += kJoin) {
        float4 a[kJoin], b[kJoin];
#pragma unroll
        for (int j = 0; j < kJoin; ++j)
            if (c + j <= last) a[j] = __ldcg(place(c + j)), b[j] = __ldcg(place(c + j) + 1);
#pragma unroll
        for (int j = 0; j < kJoin; ++j)
            if (c + j <= last) {
                all[0] += a[j].x, all[1] += a[j].y, all[2] += a[j].z, all[3] += a[j].w;
                all[4] += b[j].x, all[5] += b[j].y, all[6] += b[j].z, all[7] += b[j].w;
            }
    }
    Cells<TF32, VEC> base;
    if (A.base) base.load(A.base, int64_t(row) * A.width, int64_t(tile) * kCols, A.width);
#pragma unroll
    for (int k = 0; k < 8; ++k) all[k] = A.base ? fmaf(all[k], A.scale, base.at(k)) : all[k] * A.scale;
    put_row<TF32, VEC>(A, row, int64_t(tile) * kCols, all);
}

// The first chunks x tiles warps add up the runs, the others write the rows without tokens. BASE: A.base is there.
template <bool TF32, bool YF32, bool VEC, bool BASE>
__global__ void __launch_bounds__(kThreads, 2) k_embed_grad(const __grid_constant__ EmbedGradArgs A) {
    constexpr int kBatch = VEC && !YF32 && !BASE ? 8 : 4;  // rows of dy that are under way at a time
    const int lane = threadIdx.x & 31;
    const int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    wait_launch_before();
    if (w < int64_t(A.chunks) * A.tiles) {
        const uint32_t chunk = uint32_t(w / A.tiles), tile = uint32_t(w - int64_t(chunk) * A.tiles);
        const int64_t c0 = int64_t(tile) * kCols;
        const int n = A.first[kOwners * A.own_rows], C = A.chunk;  // places in the list, in a chunk
        if (int64_t(chunk) * C >= n) return;
        const int s0 = int(chunk) * C, end = n - s0 < C ? n : s0 + C, s_mine = s0 + lane;
        // a lane to a place of the chunk: its token and its run; `after`: the token C places on
        const bool has = s_mine < end;
        const int row = has ? A.key[s_mine] : 0, token = has ? A.order[s_mine] : 0, after = has && s_mine + C < n ? A.order[s_mine + C] : 0;
        const uint32_t at = packed(A, uint32_t(row));
        const int r0 = has ? A.first[at] : 0, r1 = has ? A.first[at + 1] : 0;
        const bool cut = r1 - r0 > C;
        const uint32_t whole = __ballot_sync(kFullMask, has && !cut && r0 >= s0);  // runs that start here and are not cut
        const uint32_t ends = __ballot_sync(kFullMask, s_mine + 1 == r1);
        auto token_at = [&](int i) { return int64_t(__shfl_sync(kFullMask, i < C ? token : after, i & (C - 1))); };
        if (whole) {
            const int tail = 31 - __clz(whole), stop = __shfl_sync(kFullMask, r1, tail);  // the last one is followed to its end
            float sum[8] = {};
            for (int s = s0 + __ffs(whole) - 1; s < stop; s += kBatch) {
                Cells<YF32, VEC> v[kBatch];
                Cells<TF32, VEC> base[BASE ? kBatch : 1];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int i = s + b - s0;
                    const int64_t t = token_at(i);
                    if (s + b < stop) v[b].load(A.dy, t * A.ld_dy, c0, A.width);
                    if constexpr (BASE) {
                        const int64_t r = __shfl_sync(kFullMask, row, i < tail ? i : tail);
                        if (s + b + 1 == stop || (i < tail && (ends >> i & 1))) base[b].load(A.base, r * A.width, c0, A.width);
                    }
                }
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    if (s + b < stop) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum[k] += v[b].at(k);
                    }
                    const int i = s + b - s0;
                    const int r = __shfl_sync(kFullMask, row, i < tail ? i : tail);
                    if (s + b + 1 == stop || (i < tail && (ends >> i & 1))) {
                        float y[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            y[k] = BASE ? fmaf(sum[k], A.scale, base[BASE ? b : 0].at(k)) : sum[k] * A.scale;
                            sum[k] = 0.f;
                        }
                        put_row<TF32, VEC>(A, r, c0, y);
                    }
                }
            }
        }
        // pieces of cut runs: of one that comes in (or fills the chunk), of one that goes on
#pragma unroll 1
        for (int which = 0; which < 2; ++which) {
            const int at = which ? end - 1 - s0 : 0;
            const int a0 = __shfl_sync(kFullMask, r0, at), a1 = __shfl_sync(kFullMask, r1, at), r = __shfl_sync(kFullMask, row, at);
            if (a1 - a0 <= C || (a0 >= s0) != bool(which)) continue;
            const int from = which ? a0 : s0, to = a1 < end ? a1 : end;
            float sum[8] = {};
            for (int s = from; s < to; s += kBatch) {
                Cells<YF32, VEC> v[kBatch];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int64_t t = token_at(s + b - s0);
                    if (s + b < to) v[b].load(A.dy, t * A.ld_dy, c0, A.width);
                }
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (s + b < to)
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum[k] += v[b].at(k);
            }
            put_piece<TF32, VEC>(A, r, a0, a1, chunk, tile, sum);
        }
    } else {
        const int64_t f = w - int64_t(A.chunks) * A.tiles, v0 = f * kFill, left = A.rows - v0;
        if (f >= A.fill) return;
        const uint32_t at = lane < kFill && lane < left ? packed(A, uint32_t(v0 + lane)) : 0;
        const uint32_t empty = __ballot_sync(kFullMask, lane < kFill && lane < left && A.first[at] == A.first[at + 1]);
        for (uint32_t tile = 0; tile < A.tiles; ++tile) {
            const int64_t c0 = int64_t(tile) * kCols;
            Cells<TF32, VEC> base[BASE ? kFill : 1];
            if constexpr (BASE)
#pragma unroll
                for (int i = 0; i < kFill; ++i)
                    if (empty >> i & 1) base[i].load(A.base, (v0 + i) * A.width, c0, A.width);
#pragma unroll
            for (int i = 0; i < kFill; ++i)
                if (empty >> i & 1) {
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = BASE ? base[BASE ? i : 0].at(k) : 0.f;
                    put_row<TF32, VEC>(A, v0 + i, c0, y);
                }
        }
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
    if (tokens < 0 || tokens > INT32_MAX) return ops_fail(SKEW_EINVAL, "tokens must be in [0, 2^31)");
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
    L.done = take(size_t(L.chunks) * L.tiles * 4);
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

template <bool WIDE>
cudaError_t launch_sort(const EmbedGradArgs &A, cudaStream_t s) {
    cudaError_t e = cudaSuccess;
    auto sort = [&](bool after, auto k) {
        e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortWarps * (int)kSortRows * 4);
        return e != cudaSuccess ? e : ops_launch(after, k, kOwners, kSortThreads, size_t(kSortWarps) * (A.own_rows < kSortRows ? A.own_rows : kSortRows) * 4, s, A);
    };
    if (!A.splits) return sort(false, k_embed_sort<WIDE, false>);
    e = ops_launch(false, k_embed_split<WIDE>, A.splits, kSortThreads, 0, s, A);
    return e != cudaSuccess ? e : sort(true, k_embed_sort<false, true>);
}

template <bool TF32, bool YF32>
cudaError_t launch_grad(const EmbedGradArgs &A, bool vec, cudaStream_t s) {
    const int64_t warps = int64_t(A.chunks) * A.tiles + A.fill;
    const uint32_t grid = uint32_t((warps + kWarps - 1) / kWarps);
    if (!grid) return cudaSuccess;
    auto go = [&](auto k) { return ops_launch(true, k, grid, kThreads, 0, s, A); };
    return vec ? (A.base ? go(k_embed_grad<TF32, YF32, true, true>) : go(k_embed_grad<TF32, YF32, true, false>))
               : (A.base ? go(k_embed_grad<TF32, YF32, false, true>) : go(k_embed_grad<TF32, YF32, false, false>));
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
    const int64_t fill = base == dtable ? 0 : (c->rows + kFill - 1) / kFill;
    if (int64_t(L.chunks) * L.tiles + fill > int64_t(INT32_MAX) * kWarps || int64_t(L.chunks) * L.tiles > INT32_MAX)
        return ops_fail(SKEW_EINVAL, "too many tokens for this width");
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
    A.wide = wide;
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
