// Global gradient norm and clipping over many tensors (skew_clip_* in include/skewadam.h).
//
//   norm = sqrt(sum g^2), gamma = min(1, max_norm / (norm + 1e-6)), out = gamma g.
//
// The tensors are cut into tiles, one entry each in a table written at bind that holds all a CTA needs to know
// (one trip to L2 ahead of the data). Both kernels are bound by memory: the sum of squares reads every
// gradient once, 2 flops an element; the factor depends on all of them, so clipping reads them again,
// the last tiles first, which are the ones that L2 still holds. One GB300, whole calls: norm of 13.6 GB in 407 tensors
// 1.78 ms (7.6 TB/s); norm and clipping of 157 MB 76 us (in place 80), of 1.08 GB of fp32 to bf16 397 us (2.7 GB, 6.8 TB/s).
#include "skew_ops.h"

#include <cmath>
#include <cstring>
#include <new>
#include <vector>

namespace skew {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kMaxCtas = 8192;   // partial sums that the workspace has room for
constexpr int kBatch = 4;             // 8-element units a thread loads before it uses them
// Bytes of gradient in a tile: smaller ones where tiles are few for the SMs, larger ones where reading the table tells. From 1 GB on
// the norm gains a little by larger tiles and clipping loses a little (16 and 32 KiB, us, for 0.94, 1.75, 3.4, 6.6 and 13 GB of bf16: norm 133.5
// 132.7, 239.7 238.4, 451 449, 877 868, 1749 1709; norm and clipping 426 430, 787 789, 1505 1519, 2952 2962, 5801 5808).
constexpr int64_t kTileBytes = 16384, kLargeTileBytes = 32768, kLargeSet = int64_t(2) << 30;
// What the norm's pass asks L2 to keep for clipping (0, 48, 64, 96 and 112 MiB, us for 157 MB, one set: 81.8 77.6 77.7 78.9 79.5).
constexpr int64_t kKeepBytes = 64 << 20;

enum : uint32_t { kGradF32 = SKEW_CLIP_GRAD_FP32, kOutF32 = SKEW_CLIP_OUT_FP32, kVectors = 4u, kNoVectors = 8u };

// A run of elements of one tensor. kVectors: g and out start on 16-byte boundaries; kNoVectors: g does not.
struct alignas(16) ClipTile {
    const void *g;
    void *out;
    uint32_t n, flags, zero[2];
};

// A tensor, cut into `tiles` tiles from `first` on: its first `head` elements, if any, then `step` at a time.
struct ClipTensor {
    const char *g;
    char *out;
    int64_t numel;
    uint32_t head, step, flags, first, tiles, zero;
};

struct ClipArgs {
    const ClipTile *tiles;
    double *part;
    uint32_t *ticket;
    float *result;
    uint32_t n_tiles, keep;  // tiles from `keep` on are to stay in L2
    float max_norm;
};

// Sums of squares outside [2^-100, 2^100] may have lost elements to overflow or underflow: with at most
// 2^17 elements and inside that range, no square has overflowed, and what squares below 2^-126 lose (2^-150
// each) is below 2^-32 of the sum. Outside, the elements are summed again, scaled into the range.
constexpr float kSumLow = 0x1p-100f, kSumHigh = 0x1p100f;
constexpr float kScaleUp = 0x1p100f, kScaleDown = 0x1p-80f;

// Eight elements, with an L2 eviction policy.
template <bool F32>
__device__ __forceinline__ Vec8<F32> load8_policy(const void *p, int64_t i, uint64_t policy) {
    Vec8<F32> v;
#pragma unroll
    for (int q = 0; q < (F32 ? 2 : 1); ++q)
        asm volatile("ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0,%1,%2,%3}, [%4], %5;"
                     : "=r"(v.u[q].x), "=r"(v.u[q].y), "=r"(v.u[q].z), "=r"(v.u[q].w)
                     : "l"(elem_ptr<F32>(p, i) + 16 * q), "l"(policy));
    return v;
}

__device__ __forceinline__ uint64_t evict_last() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ uint64_t evict_first() {
    uint64_t p;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}

template <bool F32, class F>
__device__ __forceinline__ void each_unit(const ClipTile &t, uint64_t policy, F &&f) {  // f(8 elements) for the thread's units
    const uint32_t units = t.n >> 3;
    uint32_t u = threadIdx.x;
    for (; u + (kBatch - 1) * kThreads < units; u += kBatch * kThreads) {
        Vec8<F32> v[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) v[b] = load8_policy<F32>(t.g, int64_t(u + b * kThreads) * 8, policy);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) f(v[b]);
    }
    for (; u < units; u += kThreads) f(load8_policy<F32>(t.g, int64_t(u) * 8, policy));
}

// Sum of (scale x)^2 over the thread's elements of a tile; `any`: the OR of their magnitudes' bits.
template <bool F32, bool SCALED>
__device__ __forceinline__ float tile_squares(const ClipTile &t, uint64_t policy, float scale, uint32_t &any) {
    float s0 = 0.f, s1 = 0.f;
    any = 0;
    uint32_t left = threadIdx.x;  // elements one at a time: what 8 does not divide, or all
    if (!(t.flags & kNoVectors)) {
        each_unit<F32>(t, policy, [&](const Vec8<F32> &v) {
#pragma unroll
            for (int q = 0; q < (F32 ? 2 : 1); ++q) any |= v.u[q].x | v.u[q].y | v.u[q].z | v.u[q].w;
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                const float a = SCALED ? v.at(k) * scale : v.at(k), b = SCALED ? v.at(k + 1) * scale : v.at(k + 1);
                s0 = fmaf(a, a, s0);
                s1 = fmaf(b, b, s1);
            }
        });
        any &= F32 ? 0x7FFFFFFFu : 0x7FFF7FFFu;
        left += t.n & ~7u;
    }
    for (uint32_t i = left; i < t.n; i += kThreads) {
        const float a = load1<F32>(t.g, i);
        any |= __float_as_uint(a) & 0x7FFFFFFFu;
        s0 = fmaf(SCALED ? a * scale : a, SCALED ? a * scale : a, s0);
    }
    return s0 + s1;
}

// The thread's sum of squares: a two-term fp32 sum, and in fp64 what fp32 does not hold.
struct Squares {
    float hi = 0.f, lo = 0.f;
    double rest = 0.0;
    template <bool F32>
    __device__ __forceinline__ void add(const ClipTile &t, uint64_t policy) {
        uint32_t any, unused;
        const float s = tile_squares<F32, false>(t, policy, 1.f, any);
        if (s >= kSumLow && s <= kSumHigh) {
            const float sum = hi + s, back = sum - hi;
            lo += (hi - (sum - back)) + (s - back);
            hi = sum;
        } else if (any) {
            const float scale = s < kSumLow ? kScaleUp : kScaleDown;  // a NaN stays one either way
            const double r = 1.0 / double(scale);
            rest += double(tile_squares<F32, true>(t, policy, scale, unused)) * r * r;
        }
    }
};

__device__ __forceinline__ double cta_sum(double x) {  // the sum, in thread 0
    __shared__ double warp[kThreads / 32];
    for (int d = 16; d; d >>= 1) x += __shfl_down_sync(kFullMask, x, d);
    if ((threadIdx.x & 31) == 0) warp[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kThreads / 32; ++w) x += warp[w];
    __syncthreads();
    return x;
}

// Norm and factor. The CTAs' sums are joined by whichever ends last, in the order of the CTAs.
__global__ void __launch_bounds__(kThreads) k_clip_norm(const __grid_constant__ ClipArgs A) {
    Squares sq;
    const uint64_t keep = evict_last(), drop = evict_first();
    for (uint32_t k = blockIdx.x; k < A.n_tiles; k += gridDim.x) {
        const ClipTile t = A.tiles[k];
        const uint64_t policy = k >= A.keep ? keep : drop;
        if (t.flags & kGradF32)
            sq.add<true>(t, policy);
        else
            sq.add<false>(t, policy);
    }
    const double mine = cta_sum(double(sq.hi) + double(sq.lo) + sq.rest);
    __shared__ bool last;
    if (threadIdx.x == 0) {
        A.part[blockIdx.x] = mine;
        __threadfence();
        last = atomicInc(A.ticket, gridDim.x - 1) == gridDim.x - 1;  // back at 0 for the next call
        __threadfence();
    }
    __syncthreads();
    if (!last) return;
    double x = 0.0;
    for (uint32_t k = threadIdx.x; k < gridDim.x; k += kThreads) x += __ldcg(A.part + k);
    x = cta_sum(x);
    if (threadIdx.x == 0) {
        const float norm = float(sqrt(x)), gamma = A.max_norm / (norm + 1e-6f);
        A.result[0] = norm;
        A.result[1] = gamma > 1.f ? 1.f : gamma;  // a NaN stays one
    }
}

// Writes the tiles' table: a row of CTAs to a tensor.
__global__ void __launch_bounds__(kThreads) k_clip_tiles(const ClipTensor *tensors, ClipTile *tiles) {
    const ClipTensor t = tensors[blockIdx.y];
    const int64_t ge = t.flags & kGradF32 ? 4 : 2, oe = t.flags & kOutF32 ? 4 : 2;
    const uint32_t heads = t.head != 0;
    for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < t.tiles; i += gridDim.x * kThreads) {
        const bool head = i < heads;
        const int64_t at = head ? 0 : t.head + int64_t(i - heads) * t.step, left = t.numel - at;
        tiles[t.first + i] = ClipTile{t.g + at * ge, t.out ? t.out + at * oe : nullptr, head ? t.head : uint32_t(left < t.step ? left : t.step),
                                      head ? (t.flags & ~kVectors) | kNoVectors : t.flags, {0, 0}};
    }
}

template <bool GF32, bool OF32>
__device__ __forceinline__ void scale_tile(const ClipTile &t, uint64_t policy, float gamma) {
    constexpr int kUnits = GF32 ? kBatch / 2 : kBatch;  // under way at a time
    uint32_t left = threadIdx.x;
    if (t.flags & kVectors) {
        auto scale = [&](uint32_t u, const Vec8<GF32> &v) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = v.at(k) * gamma;
            store8<OF32>(t.out, int64_t(u) * 8, x);
        };
        const uint32_t units = t.n >> 3;
        uint32_t u = threadIdx.x;
        for (; u + (kUnits - 1) * kThreads < units; u += kUnits * kThreads) {
            Vec8<GF32> v[kUnits];
#pragma unroll
            for (int b = 0; b < kUnits; ++b) v[b] = load8_policy<GF32>(t.g, int64_t(u + b * kThreads) * 8, policy);
#pragma unroll
            for (int b = 0; b < kUnits; ++b) scale(u + b * kThreads, v[b]);
        }
        for (; u < units; u += kThreads) scale(u, load8_policy<GF32>(t.g, int64_t(u) * 8, policy));
        left += t.n & ~7u;
    }
    // what 8 does not divide; or all, where g and out lie differently in their 16-byte units (157 MB: 226 us, aligned 76)
    for (uint32_t i = left; i < t.n; i += kThreads) store1<OF32>(t.out, i, load1<GF32>(t.g, i) * gamma);
}

__global__ void __launch_bounds__(kThreads, 4) k_clip_apply(const __grid_constant__ ClipArgs A) {
    wait_launch_before();
    const float gamma = __ldcg(A.result + 1);
    const uint64_t drop = evict_first();
    for (uint32_t k = blockIdx.x; k < A.n_tiles; k += gridDim.x) {
        const ClipTile t = A.tiles[A.n_tiles - 1 - k];
        if (t.g == t.out && gamma == 1.f) continue;
        if (!(t.flags & kGradF32))
            scale_tile<false, false>(t, drop, gamma);
        else if (t.flags & kOutF32)
            scale_tile<true, true>(t, drop, gamma);
        else
            scale_tile<true, false>(t, drop, gamma);
    }
}

}  // namespace
}  // namespace skew

using namespace skew;

struct skew_clip {
    std::vector<ClipTensor> tensors;
    uint32_t n_tiles = 0;
    bool writes = true;  // every tensor has an `out`
    uint32_t keep = 0;   // the first of the tiles that skew_clip_apply finds in L2
    size_t ws_ticket = 0, ws_tensors = 0, ws_tiles = 0, ws_bytes = 0;
    char *ws = nullptr;
    bool bound = false;
    uint32_t norm_ctas = 1, apply_ctas = 1;
};

extern "C" {

int skew_clip_create(const skew_clip_desc_t *tensors, int32_t n, skew_clip_t **out) {
    if (!out) return ops_fail(SKEW_EINVAL, "out is NULL");
    *out = nullptr;
    if (n < 0 || (n > 0 && !tensors)) return ops_fail(SKEW_EINVAL, "bad tensor list");
    int64_t total = 0;
    bool writes = true, reads_only = true;
    for (int32_t k = 0; k < n; ++k) {
        const skew_clip_desc_t &d = tensors[k];
        if (d.flags & ~(SKEW_CLIP_GRAD_FP32 | SKEW_CLIP_OUT_FP32) || d.zero) return ops_fail(SKEW_EINVAL, "tensor %d: unknown flags", k);
        const int64_t ge = d.flags & SKEW_CLIP_GRAD_FP32 ? 4 : 2, oe = d.flags & SKEW_CLIP_OUT_FP32 ? 4 : 2;
        if (oe > ge) return ops_fail(SKEW_EINVAL, "tensor %d: a bf16 gradient is clipped to bf16", k);
        if (d.numel < 0 || d.numel > (int64_t(1) << 40)) return ops_fail(SKEW_EINVAL, "tensor %d: numel must be in [0, 2^40]", k);
        if (d.numel && !d.grad) return ops_fail(SKEW_EINVAL, "tensor %d: null grad", k);
        if ((uintptr_t)d.grad & (ge - 1) || (uintptr_t)d.out & (oe - 1)) return ops_fail(SKEW_EINVAL, "tensor %d: pointers must be aligned to their type", k);
        if (d.out == d.grad && d.grad && oe != ge) return ops_fail(SKEW_EINVAL, "tensor %d: in place needs one type", k);
        if (d.numel) (d.out ? reads_only : writes) = false;
        if ((total += d.numel * ge) > int64_t(1) << 46) return ops_fail(SKEW_EINVAL, "too many elements");
    }
    if (!writes && !reads_only) return ops_fail(SKEW_EINVAL, "`out` is given for some tensors and not for others");
    skew_clip *h = new (std::nothrow) skew_clip();
    if (!h) return ops_fail(SKEW_ENOMEM, "out of host memory");
    h->writes = writes;
    const int64_t tile_bytes = total < kLargeSet ? kTileBytes : kLargeTileBytes;
    try {
        h->tensors.reserve(n);
        for (int32_t k = 0; k < n; ++k) {
            const skew_clip_desc_t &d = tensors[k];
            if (!d.numel) continue;
            const int64_t ge = d.flags & SKEW_CLIP_GRAD_FP32 ? 4 : 2, oe = d.flags & SKEW_CLIP_OUT_FP32 ? 4 : 2;
            // The first elements, up to where vectors may start: of both if there is such a place, else of g.
            int64_t head = -1, head_g = 0;
            for (int64_t e = 7; e >= 0; --e) {
                const bool ga = (((uintptr_t)d.grad + e * ge) & 15) == 0, oa = (((uintptr_t)d.out + e * oe) & 15) == 0;
                if (ga) head_g = e;
                if (ga && oa) head = e;
            }
            const uint32_t flags = d.flags | (head >= 0 ? kVectors : 0u);
            if (head < 0) head = head_g;
            if (head > d.numel) head = d.numel;
            const int64_t step = tile_bytes / ge, tiles = (head > 0) + (d.numel - head + step - 1) / step;
            h->tensors.push_back(ClipTensor{(const char *)d.grad, (char *)d.out, d.numel, (uint32_t)head, (uint32_t)step, flags, h->n_tiles, (uint32_t)tiles, 0});
            h->n_tiles += (uint32_t)tiles;
        }
    } catch (...) {
        delete h;
        return ops_fail(SKEW_ENOMEM, "out of host memory");
    }
    h->keep = h->n_tiles;
    int64_t keep = kKeepBytes / tile_bytes;
    for (size_t k = h->tensors.size(); k-- > 0 && keep > 0;) {  // whole tiles, a tensor's last and smaller ones among them
        const int64_t take = h->tensors[k].tiles < keep ? h->tensors[k].tiles : keep;
        h->keep -= (uint32_t)take;
        keep -= take;
    }
    auto after = [](size_t at, size_t bytes) { return (at + bytes + 255) / 256 * 256; };
    h->ws_ticket = kMaxCtas * sizeof(double);
    h->ws_tensors = h->ws_ticket + 256;
    h->ws_tiles = after(h->ws_tensors, h->tensors.size() * sizeof(ClipTensor));
    h->ws_bytes = after(h->ws_tiles, size_t(h->n_tiles) * sizeof(ClipTile));
    *out = h;
    return SKEW_OK;
}

int skew_clip_destroy(skew_clip_t *h) {
    delete h;
    return SKEW_OK;
}

size_t skew_clip_workspace_bytes(const skew_clip_t *h) { return h ? h->ws_bytes : 0; }

int skew_clip_bind(skew_clip_t *h, void *workspace, size_t workspace_bytes, void *stream) {
    if (!h) return ops_fail(SKEW_EINVAL, "handle is NULL");
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes != h->ws_bytes)
        return ops_fail(SKEW_EINVAL, "workspace must be 256-byte aligned and exactly %zu bytes", h->ws_bytes);
    cudaStream_t s = (cudaStream_t)stream;
    const int sms = ops_sm_count();
    int norm_occ = 0, apply_occ = 0, rc;
    if ((rc = ops_cuda(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&norm_occ, k_clip_norm, kThreads, 0), "occupancy")) ||
        (rc = ops_cuda(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&apply_occ, k_clip_apply, kThreads, 0), "occupancy")))
        return rc;
    h->bound = false;
    char *ws = (char *)workspace;
    if ((rc = ops_cuda(cudaMemsetAsync(ws, 0, h->ws_tensors, s), "zero-fill of the workspace"))) return rc;
    if (!h->tensors.empty()) {
        if ((rc = ops_cuda(cudaMemcpyAsync(ws + h->ws_tensors, h->tensors.data(), h->tensors.size() * sizeof(ClipTensor), cudaMemcpyHostToDevice, s), "upload of the tensors")))
            return rc;
        // (a grid holds 65535 rows)
        for (size_t k = 0; k < h->tensors.size(); k += 65535) {
            const size_t rows = h->tensors.size() - k < 65535 ? h->tensors.size() - k : 65535;
            k_clip_tiles<<<dim3(rows < 64 ? 32 : 4, (uint32_t)rows), kThreads, 0, s>>>(reinterpret_cast<const ClipTensor *>(ws + h->ws_tensors) + k,
                                                                                       reinterpret_cast<ClipTile *>(ws + h->ws_tiles));
            if ((rc = ops_cuda(cudaGetLastError(), "k_clip_tiles"))) return rc;
        }
    }
    if ((rc = ops_cuda(cudaStreamSynchronize(s), "bind"))) return rc;
    auto ctas = [&](int occ) {
        const uint64_t most = uint64_t(sms > 0 ? sms : 1) * (occ > 0 ? occ : 1), n = h->n_tiles;
        const uint64_t c = n < most ? n : most;
        return (uint32_t)(c < 1 ? 1 : c < kMaxCtas ? c : kMaxCtas);
    };
    h->norm_ctas = ctas(norm_occ);
    h->apply_ctas = ctas(apply_occ);
    h->ws = ws;
    h->bound = true;
    return SKEW_OK;
}

static int clip_args(skew_clip_t *h, float max_norm, float *result, ClipArgs &A) {
    if (!h) return ops_fail(SKEW_EINVAL, "handle is NULL");
    if (!h->bound) return ops_fail(SKEW_ESTATE, "call before skew_clip_bind");
    if (!std::isfinite(max_norm) || max_norm < 0.f) return ops_fail(SKEW_EINVAL, "max_norm must be finite and >= 0");
    if (!result || ((uintptr_t)result & 3)) return ops_fail(SKEW_EINVAL, "result must be a 4-byte aligned device pointer");
    A.tiles = reinterpret_cast<const ClipTile *>(h->ws + h->ws_tiles);
    A.part = reinterpret_cast<double *>(h->ws);
    A.ticket = reinterpret_cast<uint32_t *>(h->ws + h->ws_ticket);
    A.result = result;
    A.n_tiles = h->n_tiles;
    A.keep = A.n_tiles;
    A.max_norm = max_norm;
    return SKEW_OK;
}

int skew_clip_norm(skew_clip_t *h, float max_norm, float *result, void *stream) {
    ClipArgs A{};
    if (const int rc = clip_args(h, max_norm, result, A)) return rc;
    return ops_cuda(ops_launch(false, k_clip_norm, h->norm_ctas, kThreads, 0, (cudaStream_t)stream, A), "k_clip_norm");
}

int skew_clip_apply(skew_clip_t *h, float max_norm, float *result, void *stream) {
    ClipArgs A{};
    if (const int rc = clip_args(h, max_norm, result, A)) return rc;
    if (!h->writes) return ops_fail(SKEW_ESTATE, "the handle was planned without `out`");
    A.keep = h->keep;
    int rc = ops_cuda(ops_launch(false, k_clip_norm, h->norm_ctas, kThreads, 0, (cudaStream_t)stream, A), "k_clip_norm");
    if (rc || !A.n_tiles) return rc;
    return ops_cuda(ops_launch(true, k_clip_apply, h->apply_ctas, kThreads, 0, (cudaStream_t)stream, A), "k_clip_apply");
}

}  // extern "C"
