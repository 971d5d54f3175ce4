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
constexpr int kSortRows = 1024;  // most rows of the table to a CTA of the sort: its counters fit shared memory
constexpr int kChunk = 32;       // places of the sorted list to a warp: one to a lane
constexpr int kCols = 256;       // columns to a warp: 8 to a lane
constexpr int kFill = 8;         // rows without tokens to a warp
constexpr int kBatch = 4;        // rows of dy a lane loads before it adds them

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
    float scale;
    int32_t wide;
};

// A warp to (token, kCols columns). VEC: rows of both sides start on 16-byte boundaries.
template <bool TF32, bool YF32, bool VEC>
__global__ void __launch_bounds__(kThreads) k_lookup(const __grid_constant__ LookupArgs A) {
    const int lane = threadIdx.x & 31;
    const uint32_t tiles = uint32_t((A.width + kCols - 1) / kCols);
    const int64_t total = A.tokens * tiles;
    for (int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); w < total; w += int64_t(gridDim.x) * kWarps) {
        const int64_t t = w / tiles, c0 = (w - t * tiles) * kCols;
        const int64_t id = load_id(A.ids, A.wide, t);
        const bool there = id >= 0 && id < A.rows;
        if constexpr (VEC) {
            const int64_t c = c0 + 8 * lane;
            if (c < A.width) {
                float y[8];
                if (there) {
                    const Vec8<TF32> v = load8<TF32>(A.table, id * A.width + c);
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = v.at(k) * A.scale;
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = 0.f;
                }
                store8<YF32>(A.out, t * A.ld_out + c, y);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kCols / 32; ++k) {
                const int64_t c = c0 + 32 * k + lane;
                if (c < A.width) store1<YF32>(A.out, t * A.ld_out + c, there ? load1<TF32>(A.table, id * A.width + c) * A.scale : 0.f);
            }
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
    uint32_t sort_rows;  // rows of the table to a CTA of the sort
    uint32_t chunks, tiles, fill;  // chunks of the list, tiles of columns, warps' shares of the rows without tokens (0: they stay)
    // workspace
    int32_t *first;    // [rows + 1]: where each row's run starts in the list
    int32_t *order;    // [tokens]: the list: tokens by id
    int32_t *key;      // [tokens]: their ids
    uint32_t *done;    // [chunks * tiles]: pieces done of the run that is cut first at a chunk's end
    float *piece;      // [2 * chunks][width padded]: sums of pieces that start before a chunk, and in it
};

// Stable counting sort of the tokens by id. A CTA owns sort_rows rows of the table and reads all ids: it counts those
// of lower rows (its place in the list), and those of its own rows by warp, each warp its own run of tokens; so no
// CTA waits for another, and no count or place depends on timing.
template <bool WIDE>
__global__ void __launch_bounds__(kSortThreads, 1) k_embed_sort(const __grid_constant__ EmbedGradArgs A) {
    extern __shared__ uint32_t hist[];  // [warp][row], then each warp's next place
    __shared__ uint32_t warp_sum[kSortWarps], below[kSortWarps];
    release_launch_after();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t R = A.sort_rows;
    const int64_t v0 = int64_t(blockIdx.x) * R;
    const uint32_t rows = uint32_t(A.rows - v0 < R ? A.rows - v0 : R);
    for (uint32_t i = threadIdx.x; i < kSortWarps * R; i += kSortThreads) hist[i] = 0;
    for (uint32_t i = blockIdx.x * kSortThreads + threadIdx.x; i < A.chunks * A.tiles; i += gridDim.x * kSortThreads) A.done[i] = 0;
    __syncthreads();
    uint32_t *mine = hist + warp * R;
    const int64_t share = ((A.tokens + kSortWarps - 1) / kSortWarps + 31) / 32 * 32;
    const int64_t from = warp * share < A.tokens ? warp * share : A.tokens, to = from + share < A.tokens ? from + share : A.tokens;
    uint32_t lower = 0;
    for (int64_t t0 = from; t0 < to; t0 += 32) {
        const int64_t t = t0 + lane, id = t < to ? load_id(A.ids, WIDE, t) : -1;
        lower += id >= 0 && id < v0;
        const bool in = id >= v0 && id < v0 + rows;
        if (__any_sync(kFullMask, in)) {
            const uint32_t same = __match_any_sync(kFullMask, in ? uint32_t(id - v0) : kFullMask);
            if (in && lane == __ffs(same) - 1) mine[id - v0] += __popc(same);
            __syncwarp();
        }
    }
    lower = __reduce_add_sync(kFullMask, lower);
    if (lane == 0) below[warp] = lower;
    __syncthreads();
    // places: rows in order, within a row the warps in order
    const uint32_t v = threadIdx.x;  // a thread to a row: R <= kSortThreads
    uint32_t total = 0;
    if (v < rows)
        for (int w = 0; w < kSortWarps; ++w) total += hist[w * R + v];
    uint32_t upto = total;
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t o = __shfl_up_sync(kFullMask, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    uint32_t at = upto - total;
    for (int w = 0; w < kSortWarps; ++w) at += below[w] + (w < warp ? warp_sum[w] : 0u);
    if (v < rows) {
        A.first[v0 + v] = int32_t(at);
        if (v0 + v + 1 == A.rows) A.first[A.rows] = int32_t(at + total);
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t n = hist[w * R + v];
            hist[w * R + v] = at;
            at += n;
        }
    }
    __syncthreads();
    for (int64_t t0 = from; t0 < to; t0 += 32) {
        const int64_t t = t0 + lane, id = t < to ? load_id(A.ids, WIDE, t) : -1;
        const bool in = id >= v0 && id < v0 + rows;
        if (__any_sync(kFullMask, in)) {
            const uint32_t same = __match_any_sync(kFullMask, in ? uint32_t(id - v0) : kFullMask);
            if (in) {
                const uint32_t place = mine[id - v0] + __popc(same & ((1u << lane) - 1));
                A.order[place] = int32_t(t);
                A.key[place] = int32_t(id);
            }
            __syncwarp();
            if (in && lane == __ffs(same) - 1) mine[id - v0] += __popc(same);
            __syncwarp();
        }
    }
}

// A lane's 8 columns of the tile at c0: consecutive (VEC), or every 32nd.
template <bool VEC>
__device__ __forceinline__ int64_t column(int64_t c0, int k) {
    return VEC ? c0 + 8 * (threadIdx.x & 31) + k : c0 + 32 * k + (threadIdx.x & 31);
}

// Adds rows [from, to) of the list to `sum`, in order.
template <bool YF32, bool VEC>
__device__ __forceinline__ void add_rows(const EmbedGradArgs &A, int from, int to, int64_t c0, float (&sum)[8]) {
    const bool on = column<VEC>(c0, 0) < A.width;
    for (int s0 = from; s0 < to; s0 += 32) {
        const int lane = threadIdx.x & 31;
        const int token = s0 + lane < to ? A.order[s0 + lane] : 0, n = to - s0 < 32 ? to - s0 : 32;
        for (int s = 0; s < n; s += kBatch) {
            if constexpr (VEC) {
                Vec8<YF32> v[kBatch];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int64_t t = __shfl_sync(kFullMask, token, (s + b) & 31);
                    if (on && s + b < n) v[b] = load8<YF32>(A.dy, t * A.ld_dy + column<VEC>(c0, 0));
                }
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (s + b < n)
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum[k] += v[b].at(k);
            } else {
                float v[kBatch][8];
#pragma unroll
                for (int b = 0; b < kBatch; ++b) {
                    const int64_t t = __shfl_sync(kFullMask, token, (s + b) & 31);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        v[b][k] = s + b < n && column<VEC>(c0, k) < A.width ? load1<YF32>(A.dy, t * A.ld_dy + column<VEC>(c0, k)) : 0.f;
                }
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (s + b < n)
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum[k] += v[b][k];
            }
        }
    }
}

// dW[row] = base[row] + scale * sum, 8 columns a lane.
template <bool TF32, bool VEC>
__device__ __forceinline__ void write_row(const EmbedGradArgs &A, int64_t row, int64_t c0, const float (&sum)[8]) {
    const int64_t at = row * A.width;
    if constexpr (VEC) {
        const int64_t c = column<VEC>(c0, 0);
        if (c >= A.width) return;
        float y[8];
        if (A.base) {
            const Vec8<TF32> b = load8<TF32>(A.base, at + c);
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = fmaf(sum[k], A.scale, b.at(k));
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = sum[k] * A.scale;
        }
        store8<TF32>(A.dw, at + c, y);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t c = column<VEC>(c0, k);
            if (c < A.width) store1<TF32>(A.dw, at + c, A.base ? fmaf(sum[k], A.scale, load1<TF32>(A.base, at + c)) : sum[k] * A.scale);
        }
    }
}

// A piece of a cut run; the last piece done adds them all.
template <bool TF32, bool VEC>
__device__ __forceinline__ void put_piece(const EmbedGradArgs &A, int row, uint32_t chunk, uint32_t tile, bool starts, const float (&sum)[8]) {
    const int lane = threadIdx.x & 31;
    const int64_t pitch = int64_t(A.tiles) * kCols;
    auto place = [&](uint32_t c, bool head) { return A.piece + (2 * int64_t(c) + head) * pitch + int64_t(tile) * kCols + 8 * lane; };
    float4 *p = reinterpret_cast<float4 *>(place(chunk, starts));
    __stcg(p, make_float4(sum[0], sum[1], sum[2], sum[3]));
    __stcg(p + 1, make_float4(sum[4], sum[5], sum[6], sum[7]));
    const uint32_t c0 = uint32_t(A.first[row]) / kChunk, c1 = uint32_t(A.first[row + 1] - 1) / kChunk;
    __threadfence();
    __syncwarp();
    uint32_t before = 0;
    if (lane == 0) before = atomicAdd(A.done + int64_t(c0) * A.tiles + tile, 1u);
    before = __shfl_sync(kFullMask, before, 0);
    if (before != c1 - c0) return;
    __threadfence();
    float all[8] = {};
    for (uint32_t c = c0; c <= c1; ++c) {
        const float4 *q = reinterpret_cast<const float4 *>(place(c, c == c0));
        const float4 a = __ldcg(q), b = __ldcg(q + 1);
        all[0] += a.x, all[1] += a.y, all[2] += a.z, all[3] += a.w;
        all[4] += b.x, all[5] += b.y, all[6] += b.z, all[7] += b.w;
    }
    write_row<TF32, VEC>(A, row, int64_t(tile) * kCols, all);
}

template <bool TF32, bool YF32, bool VEC>
__global__ void __launch_bounds__(kThreads) k_embed_grad(const __grid_constant__ EmbedGradArgs A) {
    const int lane = threadIdx.x & 31;
    const int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    wait_launch_before();
    if (w < int64_t(A.chunks) * A.tiles) {
        const uint32_t chunk = uint32_t(w / A.tiles), tile = uint32_t(w - int64_t(chunk) * A.tiles);
        const int64_t c0 = int64_t(tile) * kCols;
        const int n = A.first[A.rows];  // places in the list
        const int64_t s0 = int64_t(chunk) * kChunk;
        if (s0 >= n) return;
        const int end = n - s0 < kChunk ? n : int(s0) + kChunk;
        int s = int(s0);
        const int mine = s + lane < end ? A.key[s + lane] : 0;
        while (s < end) {
            const int row = __shfl_sync(kFullMask, mine, s - int(s0));
            const int r0 = A.first[row], r1 = A.first[row + 1];
            float sum[8] = {};
            if (r1 - r0 <= kChunk) {  // whole, by the chunk that it starts in
                if (r0 == s) {
                    add_rows<YF32, VEC>(A, r0, r1, c0, sum);
                    write_row<TF32, VEC>(A, row, c0, sum);
                }
            } else {
                add_rows<YF32, VEC>(A, s, r1 < end ? r1 : end, c0, sum);
                put_piece<TF32, VEC>(A, row, chunk, tile, r0 == s, sum);
            }
            s = r1;
        }
    } else {
        const int64_t f = w - int64_t(A.chunks) * A.tiles;
        if (f >= A.fill) return;
        const float zero[8] = {};
        for (int64_t row = f * kFill; row < (f + 1) * kFill && row < A.rows; ++row)
            if (A.first[row] == A.first[row + 1])
                for (uint32_t tile = 0; tile < A.tiles; ++tile) write_row<TF32, VEC>(A, row, int64_t(tile) * kCols, zero);
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
    uint32_t chunks, tiles;
    size_t first, order, key, done, piece, bytes;
};

Layout layout(const skew_embed_config_t *c, int64_t tokens) {
    Layout L{};
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    L.chunks = uint32_t((tokens + kChunk - 1) / kChunk);
    L.tiles = uint32_t((c->width + kCols - 1) / kCols);
    L.first = take((size_t(c->rows) + 1) * 4);
    L.order = take(size_t(tokens) * 4);
    L.key = take(size_t(tokens) * 4);
    L.done = take(size_t(L.chunks) * L.tiles * 4);
    L.piece = take(size_t(L.chunks) * 2 * L.tiles * kCols * 4);
    L.bytes = at;
    return L;
}

template <bool TF32, bool YF32>
cudaError_t launch_lookup(const LookupArgs &A, bool vec, cudaStream_t s) {
    const int64_t warps = A.tokens * ((A.width + kCols - 1) / kCols), ctas = (warps + kWarps - 1) / kWarps;
    const uint32_t grid = uint32_t(ctas < INT32_MAX ? ctas : INT32_MAX);
    return vec ? ops_launch(false, k_lookup<TF32, YF32, true>, grid, kThreads, 0, s, A) : ops_launch(false, k_lookup<TF32, YF32, false>, grid, kThreads, 0, s, A);
}

template <bool WIDE>
cudaError_t launch_sort(const EmbedGradArgs &A, uint32_t grid, cudaStream_t s) {
    constexpr int kMost = kSortWarps * kSortRows * 4;
    const cudaError_t e = cudaFuncSetAttribute(k_embed_sort<WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    return e != cudaSuccess ? e : ops_launch(false, k_embed_sort<WIDE>, grid, kSortThreads, size_t(kSortWarps) * A.sort_rows * 4, s, A);
}

template <bool TF32, bool YF32>
cudaError_t launch_grad(const EmbedGradArgs &A, bool vec, cudaStream_t s) {
    const int64_t warps = int64_t(A.chunks) * A.tiles + A.fill;
    const uint32_t grid = uint32_t((warps + kWarps - 1) / kWarps);
    if (!grid) return cudaSuccess;
    return vec ? ops_launch(true, k_embed_grad<TF32, YF32, true>, grid, kThreads, 0, s, A) : ops_launch(true, k_embed_grad<TF32, YF32, false>, grid, kThreads, 0, s, A);
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
    const LookupArgs A{table, ids, out, c->rows, c->width, tokens, ld_out, c->scale, wide};
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
    // a CTA to an SM, unless that is more rows than a CTA has counters for
    const int sms = ops_sm_count() > 0 ? ops_sm_count() : 1;
    const int64_t even = (c->rows + sms - 1) / sms;
    A.sort_rows = uint32_t(even < kSortRows ? even : kSortRows);
    const uint32_t grid = uint32_t((c->rows + A.sort_rows - 1) / A.sort_rows);
    const bool vec = c->width % 8 == 0 && ld_dout % (yf ? 4 : 8) == 0 && (((uintptr_t)dout | (uintptr_t)base | (uintptr_t)dtable) & 15) == 0;
    cudaStream_t s = (cudaStream_t)stream;
    if ((rc = ops_cuda(wide ? launch_sort<true>(A, grid, s) : launch_sort<false>(A, grid, s), "k_embed_sort"))) return rc;
    return ops_cuda(tf ? (yf ? launch_grad<true, true>(A, vec, s) : launch_grad<true, false>(A, vec, s))
                       : (yf ? launch_grad<false, true>(A, vec, s) : launch_grad<false, false>(A, vec, s)), "k_embed_grad");
}

}  // extern "C"
