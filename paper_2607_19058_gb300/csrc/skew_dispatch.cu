// Rows by expert and back (skewadam.h): the order of the chosen experts' entries, the tokens' rows spread in that order, the rows combined
// token by token, and the gradients of both.
//
// The order is a stable counting sort of n = tokens * top_k small keys. A CTA takes a run of entries, a few thousand at a time, a warp 256 of
// those: entries of one expert within 32 are found by a match, so that a count or a place is one access to the warp's own counters for all of them, and
// no atomic decides an order. One launch up to kRun entries, else a launch that counts every CTA's run goes before it.
//
// The other kernels move rows, and are bound by memory: 16-byte accesses, several of them under way for each lane, and rows
// read once from DRAM (a token's row is held while it is written to each of its places).
#include <limits.h>

#include "skew_ops.h"

namespace skew {
namespace {

constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kPerWarp = 256;                        // entries of a warp between two barriers: 16-bit counters hold them
constexpr int kRun = kSortWarps * kPerWarp;
constexpr int kMaxExperts = 1024, kMaxTopK = 64;
constexpr int kSortCtas = 304;                       // runs get longer beyond: what a CTA reads of the others' counts stays short

struct OrderArgs {
    const int32_t *chosen;
    int32_t *offsets, *places, *counts;  // counts[cta][expert]
    int64_t n;
    int32_t experts, runs;               // of kRun entries, of a CTA
};

__device__ __forceinline__ int expert_of(const OrderArgs &A, int64_t i, int64_t end) {  // -1: none
    const int e = i < end ? A.chosen[i] : -1;
    return e >= 0 && e < A.experts ? e : -1;
}

__global__ void __launch_bounds__(kSortThreads) k_order_count(const OrderArgs A) {
    __shared__ int32_t count[kMaxExperts];
    for (int e = threadIdx.x; e < A.experts; e += kSortThreads) count[e] = 0;
    __syncthreads();
    const int64_t run = int64_t(A.runs) * kRun, i0 = blockIdx.x * run, end = min(A.n, i0 + run);
    for (int64_t i = i0 + threadIdx.x; i - threadIdx.x % 32 < end; i += kSortThreads) {
        const int e = expert_of(A, i, end);
        const uint32_t same = __match_any_sync(kFullMask, e);
        if (e >= 0 && (same & ((1u << (threadIdx.x & 31)) - 1)) == 0) atomicAdd(&count[e], __popc(same));  // (integers: any order gives the same)
    }
    __syncthreads();
    release_launch_after();
    for (int e = threadIdx.x; e < A.experts; e += kSortThreads) A.counts[int64_t(blockIdx.x) * A.experts + e] = count[e];
}

// What the threads before this one have together.
__device__ __forceinline__ int block_scan(int v, int32_t *of_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(kFullMask, x, d);
        if (lane >= d) x += y;
    }
    if (lane == 31) of_warp[warp] = x;
    __syncthreads();
    int before = x - v;
    for (int w = 0; w < warp; ++w) before += of_warp[w];
    return before;
}

// COUNTED: after k_order_count, in several CTAs.
template <bool COUNTED>
__global__ void __launch_bounds__(kSortThreads) k_order_place(const OrderArgs A) {
    __shared__ int32_t next[kMaxExperts], in_run[kMaxExperts];   // place of the next entry of each expert, and the entries of this run
    extern __shared__ uint16_t mine[];                           // [warp][expert]: entries of this run
    __shared__ int32_t of_warp[kSortWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = A.experts;
    uint16_t *const own = mine + warp * E;
    const uint32_t below = (1u << lane) - 1;
    const int64_t run = int64_t(A.runs) * kRun, end = min(A.n, blockIdx.x * run + run);

    int e_here[kPerWarp / 32];
    uint32_t same[kPerWarp / 32];
    auto count = [&](int64_t i0) {  // the warp's entries of the run that starts at i0, and how many of each expert every warp has
        for (int e = threadIdx.x; e < E * kSortWarps; e += kSortThreads) mine[e] = 0;
#pragma unroll
        for (int k = 0; k < kPerWarp / 32; ++k) e_here[k] = expert_of(A, i0 + warp * kPerWarp + k * 32 + lane, end);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPerWarp / 32; ++k) {
            same[k] = __match_any_sync(kFullMask, e_here[k]);
            if (e_here[k] >= 0 && !(same[k] & below)) own[e_here[k]] += __popc(same[k]);
            __syncwarp();
        }
        __syncthreads();
    };

    // the first place of each expert, and of this CTA's entries of it
    constexpr int kEach = kMaxExperts / kSortThreads;
    int total[kEach], before[kEach];
    if constexpr (COUNTED) {
        wait_launch_before();
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int e = threadIdx.x * kEach + j;
            total[j] = before[j] = 0;
            if (e >= E) continue;
            for (int c = 0; c < int(gridDim.x); ++c) {
                const int v = A.counts[int64_t(c) * E + e];
                total[j] += v;
                if (c < int(blockIdx.x)) before[j] += v;
            }
        }
    } else {
        count(0);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int e = threadIdx.x * kEach + j;
            total[j] = before[j] = 0;
            if (e < E)
                for (int w = 0; w < kSortWarps; ++w) total[j] += mine[w * E + e];
        }
    }
    int at = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) at += total[j];
    at = block_scan(at, of_warp);
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int e = threadIdx.x * kEach + j;
        if (e < E) {
            next[e] = at + before[j];
            if (blockIdx.x == 0) A.offsets[e] = at;
        }
        at += total[j];
        if (blockIdx.x == 0 && e == E - 1) A.offsets[E] = at;
    }
    __syncthreads();

    for (int64_t i0 = blockIdx.x * run; i0 < end; i0 += kRun) {
        if (COUNTED) count(i0);
        for (int e = threadIdx.x; e < E; e += kSortThreads) {  // the entries of the warps before each
            int n = 0;
            for (int w = 0; w < kSortWarps; ++w) {
                const int c = mine[w * E + e];
                mine[w * E + e] = uint16_t(n);
                n += c;
            }
            in_run[e] = n;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPerWarp / 32; ++k) {
            const int e = e_here[k];
            const int64_t i = i0 + warp * kPerWarp + k * 32 + lane;
            if (i < end) A.places[i] = e >= 0 ? next[e] + own[e] + __popc(same[k] & below) : -1;
            __syncwarp();
            if (e >= 0 && !(same[k] & below)) own[e] += __popc(same[k]);
            __syncwarp();
        }
        __syncthreads();
        for (int e = threadIdx.x; e < E; e += kSortThreads) next[e] += in_run[e];
    }
}

// ---------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------
constexpr int kThreads = 256, kWarps = kThreads / 32;

struct RowsArgs {
    const void *tokens;                 // x or dout
    const void *rows;
    void *out;                          // spread, combine_grad: rows; combine: tokens
    const float *weights;
    float *dweights;
    const int32_t *offsets, *places;
    int64_t n_tokens, n_rows, width, ld;  // ld: of the tokens' rows
    int32_t top_k, experts;
    int32_t lanes;                      // to a row (a power of two), the others take the next rows
    bool wide;                          // a CTA to a row instead: its warps share the columns
};

// Eight elements of a row: side by side, as one or two 16-byte accesses; or one access each, 32 apart, so that the lanes of a warp access
// neighbours (`n`: elements from the first to the row's end).
template <bool F32, bool VEC>
struct Piece {
    float x[8];
    __device__ __forceinline__ void read(const void *p, int64_t i, int n) {
        if constexpr (VEC) {
            const Vec8<F32> v = load8_cached<F32>(p, i);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = v.at(k);
        } else {
            p = elem_ptr<F32>(p, i);
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = k * 32 < n ? load1<F32>(p, k * 32) : 0.f;
        }
    }
    __device__ __forceinline__ void write(void *p, int64_t i, int n) const {
        if constexpr (VEC) {
            store8<F32>(p, i, x);
        } else {
            p = const_cast<char *>(elem_ptr<F32>(p, i));
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k * 32 < n) store1<F32>(p, k * 32, x[k]);
        }
    }
};

// A lane's row, of `total`; the first column of its first piece, and the columns from a piece to its next.
#define SKEW_ROW_OF_LANES(total)                                                                                      \
    const int lane = threadIdx.x & 31, in = A.wide ? int(threadIdx.x) : lane & (A.lanes - 1);                         \
    const int64_t first = VEC ? in * 8 : A.wide ? threadIdx.x / 32 * 256 + lane : in, step = (A.wide ? kThreads : A.lanes) * 8; \
    const int64_t per = 32 / A.lanes;                                                                                 \
    const int64_t i = A.wide ? blockIdx.x : (blockIdx.x * int64_t(kWarps) + threadIdx.x / 32) * per + lane / A.lanes; \
    const bool there = i < (total);

// rows[place(t, j)] = x[t]; rows behind the last place: zeros.
template <bool TF32, bool RF32, bool VEC>
__global__ void __launch_bounds__(kThreads) k_spread(const RowsArgs A) {
    SKEW_ROW_OF_LANES(A.n_tokens)
    if (!there) return;
    const int64_t used = A.offsets[A.experts];
    constexpr int kDeep = 4;
    for (int64_t c0 = first; c0 < A.width; c0 += step * kDeep) {
        Piece<TF32, VEC> x[kDeep];
#pragma unroll
        for (int q = 0; q < kDeep; ++q) {
            const int64_t c = c0 + q * step;
            if (c < A.width) x[q].read(A.tokens, i * A.ld + c, int(A.width - c));
        }
        for (int j = 0; j < A.top_k; ++j) {
            const int64_t entry = i * A.top_k + j, place = A.places[entry];
            const bool put = place >= 0 && place < A.n_rows, clear = entry >= used;
#pragma unroll
            for (int q = 0; q < kDeep; ++q) {
                const int64_t c = c0 + q * step;
                if (c >= A.width) break;
                if (put) reinterpret_cast<const Piece<RF32, VEC> &>(x[q]).write(A.out, place * A.width + c, int(A.width - c));
                if (clear) Piece<RF32, VEC>{}.write(A.out, entry * A.width + c, int(A.width - c));
            }
        }
    }
}

// out[t] = sum over j of weights[t, j] * rows[place(t, j)]: kRows rows at a time, of kPieces pieces of columns.
template <bool TF32, bool RF32, bool VEC, int kRows, int kPieces>
__device__ __forceinline__ void combine(const RowsArgs &A, int64_t i, int64_t first, int64_t step) {
    for (int64_t c0 = first; c0 < A.width; c0 += step * kPieces) {
        Piece<TF32, VEC> y[kPieces] = {};
        for (int j0 = 0; j0 < A.top_k; j0 += kRows) {
            Piece<RF32, VEC> x[kRows][kPieces];
            float w[kRows];
#pragma unroll
            for (int q = 0; q < kRows; ++q) {
                const int64_t entry = i * A.top_k + j0 + q;
                const int64_t place = j0 + q < A.top_k ? A.places[entry] : -1;
                const bool put = place >= 0 && place < A.n_rows;
                w[q] = put ? (A.weights ? A.weights[entry] : 1.f) : 0.f;
#pragma unroll
                for (int p = 0; p < kPieces; ++p) {
                    const int64_t c = c0 + p * step;
                    x[q][p] = {};
                    if (put && c < A.width) x[q][p].read(A.rows, place * A.width + c, int(A.width - c));
                }
            }
#pragma unroll
            for (int q = 0; q < kRows; ++q)
#pragma unroll
                for (int p = 0; p < kPieces; ++p)
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[p].x[k] = fmaf(w[q], x[q][p].x[k], y[p].x[k]);
        }
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int64_t c = c0 + p * step;
            if (c < A.width) y[p].write(A.out, i * A.ld + c, int(A.width - c));
        }
    }
}

template <bool TF32, bool RF32, bool VEC>
__global__ void __launch_bounds__(kThreads) k_combine(const RowsArgs A) {
    SKEW_ROW_OF_LANES(A.n_tokens)
    if (!there) return;
    // Four rows' loads under way, or two rows' of two pieces: with one or two experts a token, half of them would be none.
    if (A.top_k <= 2)
        combine<TF32, RF32, VEC, 2, 2>(A, i, first, step);
    else
        combine<TF32, RF32, VEC, 4, 1>(A, i, first, step);
}

// drows[place] = weights[t, j] * dout[t], dweights[t, j] = <dout[t], rows[place]>; an entry (t, j) to `lanes` lanes. Two loads and a store at a time, and as many
// warps as fit: with more under way for each, fewer fit (65,536 rows of 4096 columns: 211 us, 253 with two pieces of columns at a time, 379 with four).
template <bool TF32, bool RF32, bool VEC>
__global__ void __launch_bounds__(kThreads, 6) k_combine_grad(const RowsArgs A) {
    SKEW_ROW_OF_LANES(A.n_tokens * A.top_k)
    const int64_t place = there ? A.places[i] : -1;
    const bool put = place >= 0 && place < A.n_rows, clear = there && i >= A.offsets[A.experts];
    const float w = put ? A.weights[i] : 0.f;
    const int64_t from = there ? i / A.top_k * A.ld : 0;
    float dot = 0.f;
    if (put || clear) {
        for (int64_t c = first; c < A.width; c += step) {
            const int n = int(A.width - c);
            if (put) {
                Piece<TF32, VEC> g;
                Piece<RF32, VEC> x;
                g.read(A.tokens, from + c, n);
                x.read(A.rows, place * A.width + c, n);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    dot = fmaf(g.x[k], x.x[k], dot);
                    x.x[k] = w * g.x[k];
                }
                x.write(A.out, place * A.width + c, n);
            }
            if (clear) Piece<RF32, VEC>{}.write(A.out, i * A.width + c, n);
        }
    }
    for (int d = A.lanes / 2; d; d >>= 1) dot += __shfl_xor_sync(kFullMask, dot, d);
    if (A.wide) {
        __shared__ float of_warp[kWarps];
        if (!lane) of_warp[threadIdx.x / 32] = dot;
        __syncthreads();
        dot = 0.f;
        for (int w = 0; w < kWarps; ++w) dot += of_warp[w];
    }
    if (there && !in) A.dweights[i] = dot;
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------
int check(const skew_dispatch_config_t *c, int64_t tokens) {
    if (!c) return ops_fail(SKEW_EINVAL, "config is NULL");
    if (c->experts < 1 || c->experts > kMaxExperts) return ops_fail(SKEW_EINVAL, "experts must be in [1, %d]", kMaxExperts);
    if (c->top_k < 1 || c->top_k > kMaxTopK) return ops_fail(SKEW_EINVAL, "top_k must be in [1, %d]", kMaxTopK);
    if (c->flags & ~(SKEW_DISPATCH_TOKENS_FP32 | SKEW_DISPATCH_ROWS_FP32) || c->zero) return ops_fail(SKEW_EINVAL, "unknown flags");
    if (tokens < 0 || tokens > (int64_t(1) << 30) / c->top_k) return ops_fail(SKEW_EINVAL, "tokens * top_k must be in [0, 2^30]");
    return SKEW_OK;
}

int check_ptr(const char *what, const void *p, uintptr_t es, bool needed) {
    if ((needed && !p) || ((uintptr_t)p & (es - 1))) return ops_fail(SKEW_EINVAL, "%s must be a device pointer aligned to its type", what);
    return SKEW_OK;
}

int check_width(int64_t width, int64_t ld) {
    if (width < 1 || width > int64_t(1) << 20) return ops_fail(SKEW_EINVAL, "width must be in [1, 2^20]");
    if (ld < width || ld > int64_t(1) << 31) return ops_fail(SKEW_EINVAL, "row stride must be in [width, 2^31]");
    return SKEW_OK;
}

struct Runs {
    int64_t ctas, runs;
};

Runs runs_of(int64_t n) {
    const int64_t runs = (n + kRun - 1) / kRun, per = (runs + kSortCtas - 1) / kSortCtas;
    return {per ? (runs + per - 1) / per : 1, per ? per : 1};
}

// `rows`: of lanes' rows.
template <template <bool, bool, bool> class K>
cudaError_t launch_rows(const skew_dispatch_config_t *c, RowsArgs &A, int64_t items, bool vec, cudaStream_t s) {
    A.lanes = 32;
    while (A.lanes > 1 && (vec ? int64_t(A.lanes) * 4 >= A.width : A.lanes / 2 >= A.width)) A.lanes >>= 1;  // (one access each: a piece's first element alone is there)
    const int64_t warps = (items + 32 / A.lanes - 1) / (32 / A.lanes);
    // few rows, of some width: a CTA to each (2 tokens of 10 rows of 5197 columns, combined: 72 us by a warp each)
    A.wide = A.lanes == 32 && A.width > 512 && items <= int64_t(ops_sm_count()) * 4;
    const uint32_t grid = uint32_t(A.wide ? items : (warps + kWarps - 1) / kWarps);
    auto run = [&](auto k) { return ops_launch(false, k, grid, kThreads, 0, s, A); };
    const bool t = c->flags & SKEW_DISPATCH_TOKENS_FP32, r = c->flags & SKEW_DISPATCH_ROWS_FP32;
    if (vec) return t ? (r ? run(K<true, true, true>::k) : run(K<true, false, true>::k)) : (r ? run(K<false, true, true>::k) : run(K<false, false, true>::k));
    return t ? (r ? run(K<true, true, false>::k) : run(K<true, false, false>::k)) : (r ? run(K<false, true, false>::k) : run(K<false, false, false>::k));
}

template <bool T, bool R, bool V> struct Spread { static constexpr auto k = k_spread<T, R, V>; };
template <bool T, bool R, bool V> struct Combine { static constexpr auto k = k_combine<T, R, V>; };
template <bool T, bool R, bool V> struct CombineGrad { static constexpr auto k = k_combine_grad<T, R, V>; };

bool whole_units(const skew_dispatch_config_t *c, int64_t width, int64_t ld, const void *tokens, const void *rows, const void *more) {
    return width % 8 == 0 && ld % (c->flags & SKEW_DISPATCH_TOKENS_FP32 ? 4 : 8) == 0 && (((uintptr_t)tokens | (uintptr_t)rows | (uintptr_t)more) & 15) == 0;
}

}  // namespace
}  // namespace skew

using namespace skew;

extern "C" {

size_t skew_dispatch_workspace_bytes(const skew_dispatch_config_t *c, int64_t tokens) {
    if (check(c, tokens) != SKEW_OK) return 0;
    return (size_t(runs_of(tokens * c->top_k).ctas) * c->experts * 4 + 255) / 256 * 256;
}

int skew_dispatch_order(const skew_dispatch_config_t *c, const int32_t *chosen, int64_t tokens, int32_t *offsets, int32_t *places, void *workspace,
                        size_t workspace_bytes, void *stream) {
    int rc;
    if ((rc = check(c, tokens)) || (rc = check_ptr("chosen", chosen, 4, tokens > 0)) || (rc = check_ptr("offsets", offsets, 4, true)) ||
        (rc = check_ptr("places", places, 4, tokens > 0)))
        return rc;
    const size_t need = skew_dispatch_workspace_bytes(c, tokens);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)
        return ops_fail(SKEW_EINVAL, "workspace must be 256-byte aligned and at least %zu bytes", need);
    const Runs r = runs_of(tokens * c->top_k);
    const OrderArgs A{chosen, offsets, places, (int32_t *)workspace, tokens * c->top_k, c->experts, (int32_t)r.runs};
    cudaStream_t s = (cudaStream_t)stream;
    const size_t smem = size_t(kSortWarps) * c->experts * 2;
    if (r.ctas == 1 && r.runs == 1) return ops_cuda(ops_launch(false, k_order_place<false>, 1, kSortThreads, smem, s, A), "k_order_place");
    if ((rc = ops_cuda(ops_launch(false, k_order_count, (uint32_t)r.ctas, kSortThreads, 0, s, A), "k_order_count"))) return rc;
    return ops_cuda(ops_launch(true, k_order_place<true>, (uint32_t)r.ctas, kSortThreads, smem, s, A), "k_order_place");
}

int skew_dispatch_spread(const skew_dispatch_config_t *c, const void *x, int64_t ld_x, const int32_t *offsets, const int32_t *places, int64_t tokens,
                         int64_t width, void *rows, void *stream) {
    int rc;
    const int tf = c && c->flags & SKEW_DISPATCH_TOKENS_FP32 ? 4 : 2, rf = c && c->flags & SKEW_DISPATCH_ROWS_FP32 ? 4 : 2;
    if ((rc = check(c, tokens)) || (rc = check_width(width, ld_x)) || (rc = check_ptr("x", x, tf, tokens > 0)) || (rc = check_ptr("offsets", offsets, 4, true)) ||
        (rc = check_ptr("places", places, 4, tokens > 0)) || (rc = check_ptr("rows", rows, rf, tokens > 0)))
        return rc;
    if (!tokens) return SKEW_OK;
    RowsArgs A{x, nullptr, rows, nullptr, nullptr, offsets, places, tokens, tokens * c->top_k, width, ld_x, c->top_k, c->experts, 0, false};
    return ops_cuda(launch_rows<Spread>(c, A, tokens, whole_units(c, width, ld_x, x, rows, nullptr), (cudaStream_t)stream), "k_spread");
}

int skew_dispatch_combine(const skew_dispatch_config_t *c, const void *rows, const float *weights, const int32_t *places, int64_t tokens, int64_t width,
                          void *out, int64_t ld_out, void *stream) {
    int rc;
    const int tf = c && c->flags & SKEW_DISPATCH_TOKENS_FP32 ? 4 : 2, rf = c && c->flags & SKEW_DISPATCH_ROWS_FP32 ? 4 : 2;
    if ((rc = check(c, tokens)) || (rc = check_width(width, ld_out)) || (rc = check_ptr("rows", rows, rf, tokens > 0)) || (rc = check_ptr("weights", weights, 4, false)) ||
        (rc = check_ptr("places", places, 4, tokens > 0)) || (rc = check_ptr("out", out, tf, tokens > 0)))
        return rc;
    if (!tokens) return SKEW_OK;
    RowsArgs A{nullptr, rows, out, weights, nullptr, nullptr, places, tokens, tokens * c->top_k, width, ld_out, c->top_k, c->experts, 0, false};
    return ops_cuda(launch_rows<Combine>(c, A, tokens, whole_units(c, width, ld_out, out, rows, nullptr), (cudaStream_t)stream), "k_combine");
}

int skew_dispatch_combine_grad(const skew_dispatch_config_t *c, const void *dout, int64_t ld_dout, const void *rows, const float *weights,
                               const int32_t *offsets, const int32_t *places, int64_t tokens, int64_t width, void *drows, float *dweights, void *stream) {
    int rc;
    const int tf = c && c->flags & SKEW_DISPATCH_TOKENS_FP32 ? 4 : 2, rf = c && c->flags & SKEW_DISPATCH_ROWS_FP32 ? 4 : 2;
    if ((rc = check(c, tokens)) || (rc = check_width(width, ld_dout)) || (rc = check_ptr("dout", dout, tf, tokens > 0)) || (rc = check_ptr("rows", rows, rf, tokens > 0)) ||
        (rc = check_ptr("weights", weights, 4, tokens > 0)) || (rc = check_ptr("offsets", offsets, 4, true)) || (rc = check_ptr("places", places, 4, tokens > 0)) ||
        (rc = check_ptr("drows", drows, rf, tokens > 0)) || (rc = check_ptr("dweights", dweights, 4, tokens > 0)))
        return rc;
    if (!tokens) return SKEW_OK;
    RowsArgs A{dout, rows, drows, weights, dweights, offsets, places, tokens, tokens * c->top_k, width, ld_dout, c->top_k, c->experts, 0, false};
    return ops_cuda(launch_rows<CombineGrad>(c, A, tokens * c->top_k, whole_units(c, width, ld_dout, dout, rows, drows), (cudaStream_t)stream), "k_combine_grad");
}

}  // extern "C"
