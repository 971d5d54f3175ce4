// The output head's softmax cross entropy (skewadam.h), from the products of skew_product.cu.
//
// The loss takes one product whose tiles of logits never leave the chip: of each row a tile keeps the largest logit and the sum of
// exponentials below it (8 bytes for 128 columns), k_join joins a row's. The gradients take the vocabulary in pieces: the logits' gradient of a
// piece in bf16, from its logits anew, then the piece's share of dh, added up in fp32 over the pieces, and its rows of dW.
#include <cmath>

#include "skew_ops.h"
#include "skew_product.h"

namespace skew {
namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 24, kMaxRows = int64_t(1) << 24;
constexpr int64_t kPieceBytes = int64_t(512) << 20;  // of the logits' gradient, at most
constexpr int64_t kPieceCols = 256;                  // but this many columns at least (more bytes then, from 2^20 tokens on: 8 GiB for 2^24), and a multiple

constexpr int kJoinWarps = 16;

struct JoinArgs {
    const float2 *part;
    const float *picked;
    const void *targets;
    float *loss, *lse;
    int64_t tokens, vocab;
    int32_t parts;
    bool wide;
};

// A lane to a token, every sixteenth part to a warp, eight parts at a time. Parts are in powers of two (skew_product.h). Bound by latency: 24 us for 6606 tokens
// of 313 parts while parts were added one by one in eight warps.
__global__ void __launch_bounds__(32 * kJoinWarps) k_join(const JoinArgs A) {
    __shared__ float2 of_warp[kJoinWarps][32];
    wait_launch_before();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = blockIdx.x * int64_t(32) + lane;
    const bool there = t < A.tokens;
    constexpr int kDeep = 8;
    const float2 none = make_float2(-INFINITY, 0.f);
    float top = -INFINITY, sum = 0.f;
    auto add = [&](const float2 (&p)[kDeep]) {
        float high = top;
#pragma unroll
        for (int j = 0; j < kDeep; ++j) high = fmaxf(high, p[j].x);
        const float from = fabsf(high) < INFINITY ? high : 0.f;  // (as the parts)
        sum *= exp2f(top - from);
#pragma unroll
        for (int j = 0; j < kDeep; ++j) sum = fmaf(p[j].y, exp2f(p[j].x - from), sum);
        top = high;
    };
    float2 p[kDeep];
    for (int i = warp; there && i < A.parts; i += kJoinWarps * kDeep) {
#pragma unroll
        for (int j = 0; j < kDeep; ++j) p[j] = i + j * kJoinWarps < A.parts ? A.part[int64_t(i + j * kJoinWarps) * A.tokens + t] : none;
        add(p);
    }
    of_warp[warp][lane] = make_float2(top, sum);
    __syncthreads();
    if (warp || !there) return;
    top = -INFINITY;
    sum = 0.f;
    for (int w = 0; w < kJoinWarps; w += kDeep) {
#pragma unroll
        for (int j = 0; j < kDeep; ++j) p[j] = of_warp[w + j][lane];
        add(p);
    }
    constexpr float kLn2 = 0.693147180559945309417f;
    const float rest = log2f(sum);
    const int64_t v = A.wide ? static_cast<const int64_t *>(A.targets)[t] : static_cast<const int32_t *>(A.targets)[t];
    A.lse[t] = (top + rest) * kLn2;
    A.loss[t] = v < 0 || v >= A.vocab ? 0.f : (top - A.picked[t] + rest) * kLn2;  // (the difference first: nothing is lost where the target is the largest)
}

// What the gradients read of the activations: rows of padded tokens as zeros (whatever they hold then enters no gradient), on 16-byte boundaries;
// and the largest dloss of each CTA. A logit's gradient is rounded to bf16 divided by the largest of all, so that where all are
// equal, as in a mean, the largest terms (at the targets, near -1) lose almost nothing.
constexpr int kTidyThreads = 256, kTidyCols = 1024;  // a warp's share of a row

struct TidyArgs {
    const uint16_t *h;
    uint16_t *out;
    const void *targets;
    const float *dloss;
    float *peaks;
    int64_t tokens, vocab, width, ld, ld_out;
    bool wide, vec;
    bool as_is;  // the loss: only the boundaries
};

__global__ void __launch_bounds__(kTidyThreads) k_tidy(const TidyArgs A) {
    __shared__ float of_warp[kTidyThreads / 32];
    release_launch_after();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float peak = 0.f;
    const int64_t shares = (A.ld_out + kTidyCols - 1) / kTidyCols;
    for (int64_t i = blockIdx.x * int64_t(kTidyThreads / 32) + warp; i < A.tokens * shares; i += int64_t(gridDim.x) * (kTidyThreads / 32)) {
        const int64_t t = i / shares, c0 = i % shares * kTidyCols + lane * 8;
        const int64_t v = A.as_is ? 0 : A.wide ? static_cast<const int64_t *>(A.targets)[t] : static_cast<const int32_t *>(A.targets)[t];
        const bool there = v >= 0 && v < A.vocab;
        if (there && c0 == 0 && !A.as_is) peak = fmaxf(peak, fabsf(A.dloss[t]));
        const uint16_t *from = A.h + t * A.ld;
        uint4 u[kTidyCols / 256];
#pragma unroll
        for (int j = 0; j < kTidyCols / 256; ++j) {
            const int64_t c = c0 + j * 256;
            u[j] = make_uint4(0, 0, 0, 0);
            if (!there || c >= A.ld_out) continue;
            if (A.vec) {
                u[j] = *reinterpret_cast<const uint4 *>(from + c);
            } else {
                uint32_t x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = c + k < A.width ? from[c + k] : 0;
                u[j] = make_uint4(x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16);
            }
        }
#pragma unroll
        for (int j = 0; j < kTidyCols / 256; ++j)
            if (c0 + j * 256 < A.ld_out) *reinterpret_cast<uint4 *>(A.out + t * A.ld_out + c0 + j * 256) = u[j];
    }
    if (A.as_is) return;
    if (!lane) of_warp[warp] = peak;
    __syncthreads();
    if (threadIdx.x) return;
    for (int w = 1; w < kTidyThreads / 32; ++w) peak = fmaxf(peak, of_warp[w]);
    A.peaks[blockIdx.x] = peak;
    if (!blockIdx.x)
        for (int i = gridDim.x; i < kPeaks; ++i) A.peaks[i] = 0.f;
}

int check(const skew_head_config_t *c, int64_t tokens) {
    if (!c) return ops_fail(SKEW_EINVAL, "config is NULL");
    if (c->rows < 1 || c->rows > kMaxRows) return ops_fail(SKEW_EINVAL, "rows must be in [1, 2^24]");
    if (c->width < 1 || c->width > int64_t(1) << 20) return ops_fail(SKEW_EINVAL, "width must be in [1, 2^20]");
    if (!std::isfinite(c->scale)) return ops_fail(SKEW_EINVAL, "scale must be finite");
    if (c->flags & ~SKEW_HEAD_IDS_64) return ops_fail(SKEW_EINVAL, "unknown flags");
    if (tokens < 0 || tokens > kMaxTokens) return ops_fail(SKEW_EINVAL, "tokens must be in [0, 2^24]");
    return SKEW_OK;
}

int check_ptr(const char *what, const void *p, uintptr_t es, bool needed) {
    if ((needed && !p) || ((uintptr_t)p & (es - 1))) return ops_fail(SKEW_EINVAL, "%s must be a device pointer aligned to its type", what);
    return SKEW_OK;
}

int check_workspace(const void *ws, size_t bytes, size_t need) {
    if (!ws || ((uintptr_t)ws & 255) || bytes < need) return ops_fail(SKEW_EINVAL, "workspace must be 256-byte aligned and at least %zu bytes", need);
    return SKEW_OK;
}

size_t whole(size_t bytes) { return (bytes + 255) / 256 * 256; }

struct Layout {
    int64_t parts, piece, pieces;
    size_t picked, copy, loss_bytes;  // parts, then the picked logits, and the activations' copy
    int64_t ld;                    // of the activations' copy
    size_t sums, tidy, peaks, shares, dh_parts, grad_bytes;  // a piece, dh's sums over the pieces, the copy, peaks, shares of tiles
};

Layout layout(const skew_head_config_t *c, int64_t tokens) {
    Layout L{};
    const int64_t T = tokens ? tokens : 1, wide = product_loss_columns();
    L.parts = (c->rows + wide - 1) / wide;
    L.picked = whole(size_t(T) * L.parts * 8);
    L.ld = (c->width + 7) / 8 * 8;
    L.copy = L.picked + whole(size_t(T) * 4);
    L.loss_bytes = L.copy + whole(size_t(T) * L.ld * 2);
    int64_t most = kPieceBytes / (2 * T) / kPieceCols * kPieceCols;
    if (most < kPieceCols) most = kPieceCols;
    L.pieces = (c->rows + most - 1) / most;
    L.piece = ((c->rows + L.pieces - 1) / L.pieces + kPieceCols - 1) / kPieceCols * kPieceCols;
    L.pieces = (c->rows + L.piece - 1) / L.piece;
    L.sums = whole(size_t(T) * L.piece * 2);
    L.tidy = L.sums + (L.pieces > 1 ? whole(size_t(T) * c->width * 4) : 0);
    L.peaks = L.tidy + whole(size_t(T) * L.ld * 2);
    L.shares = L.peaks + whole(kPeaks * 4);
    // the parts of dh, and of dW's rows of a piece (the last may be shorter)
    L.dh_parts = product_parts_bytes(1, T, c->width);
    const int64_t rest = c->rows - (L.pieces - 1) * L.piece;
    size_t parts = L.dh_parts;
    for (const int64_t n : {L.piece, rest})
        if (const size_t b = product_parts_bytes(1, n, c->width); b > parts) parts = b;
    L.grad_bytes = L.shares + whole(parts);
    return L;
}

cudaError_t launch_tidy(const TidyArgs &A, cudaStream_t s) {
    const int64_t blocks = (A.tokens * ((A.ld_out + kTidyCols - 1) / kTidyCols) + kTidyThreads / 32 - 1) / (kTidyThreads / 32);
    return ops_launch(false, k_tidy, uint32_t(blocks < kPeaks ? blocks : kPeaks), kTidyThreads, 0, s, A);
}

bool units(int64_t width, const void *p) { return width % 8 == 0 && ((uintptr_t)p & 15) == 0; }

}  // namespace
}  // namespace skew

using namespace skew;

extern "C" {

size_t skew_head_loss_workspace_bytes(const skew_head_config_t *c, int64_t tokens) { return check(c, tokens) == SKEW_OK ? layout(c, tokens).loss_bytes : 0; }
size_t skew_head_grad_workspace_bytes(const skew_head_config_t *c, int64_t tokens) { return check(c, tokens) == SKEW_OK ? layout(c, tokens).grad_bytes : 0; }

int skew_head_loss(const skew_head_config_t *c, const void *h, int64_t ld_h, const void *table, const void *targets, int64_t tokens, float *loss, float *lse,
                   void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check(c, tokens);
    if (rc) return rc;
    const bool wide = c->flags & SKEW_HEAD_IDS_64;
    if ((rc = check_ptr("h", h, 2, tokens > 0)) || (rc = check_ptr("table", table, 2, true)) || (rc = check_ptr("targets", targets, wide ? 8 : 4, tokens > 0)) ||
        (rc = check_ptr("loss", loss, 4, tokens > 0)) || (rc = check_ptr("lse", lse, 4, tokens > 0)))
        return rc;
    if (ld_h < c->width || ld_h > int64_t(1) << 31) return ops_fail(SKEW_EINVAL, "row stride must be in [width, 2^31]");
    const Layout L = layout(c, tokens);
    if ((rc = check_workspace(workspace, workspace_bytes, L.loss_bytes))) return rc;
    if (!tokens) return SKEW_OK;
    char *ws = (char *)workspace;
    cudaStream_t s = (cudaStream_t)stream;
    // Activations off 16-byte boundaries come from a copy: the table alone is then cut out of its lines (2314 tokens, 311 x 3149: 103 us without).
    const bool copy = !units(c->width, h) || ld_h % 8;
    if (copy && (rc = ops_cuda(launch_tidy({(const uint16_t *)h, (uint16_t *)(ws + L.copy), targets, nullptr, nullptr, tokens, c->rows, c->width, ld_h, L.ld, wide, false, true}, s),
                               "k_tidy")))
        return rc;
    ProductArgs A{};
    A.a = copy ? (const void *)(ws + L.copy) : h;
    A.b = table;
    A.lda = copy ? L.ld : ld_h;
    A.ldb = c->width;
    A.rows = tokens;
    A.groups = 1;
    A.inner = (int32_t)c->width;
    A.cols = (int32_t)c->rows;
    A.scale = c->scale;
    A.flags = (wide ? kIds64 : 0) | kRelease;
    A.targets = targets;
    A.vocab = c->rows;
    A.part = (float2 *)ws;
    A.picked = (float *)(ws + L.picked);
    if ((rc = ops_cuda(product_launch(kByCols, kLoss, A, s), "k_product"))) return rc;
    const JoinArgs J{A.part, A.picked, targets, loss, lse, tokens, c->rows, (int32_t)L.parts, wide};
    return ops_cuda(ops_launch(true, k_join, uint32_t((tokens + 31) / 32), 32 * kJoinWarps, 0, s, J), "k_join");
}

int skew_head_grad(const skew_head_config_t *c, const void *h, int64_t ld_h, const void *table, const void *targets, int64_t tokens, const float *lse,
                   const float *dloss, void *dh, const void *base, void *dtable, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check(c, tokens);
    if (rc) return rc;
    const bool wide = c->flags & SKEW_HEAD_IDS_64;
    if ((rc = check_ptr("h", h, 2, tokens > 0)) || (rc = check_ptr("table", table, 2, true)) || (rc = check_ptr("targets", targets, wide ? 8 : 4, tokens > 0)) ||
        (rc = check_ptr("lse", lse, 4, tokens > 0)) || (rc = check_ptr("dloss", dloss, 4, tokens > 0)) || (rc = check_ptr("dh", dh, 2, tokens > 0)) ||
        (rc = check_ptr("base", base, 2, false)) || (rc = check_ptr("dtable", dtable, 2, true)))
        return rc;
    if (ld_h < c->width || ld_h > int64_t(1) << 31) return ops_fail(SKEW_EINVAL, "row stride must be in [width, 2^31]");
    const Layout L = layout(c, tokens);
    if ((rc = check_workspace(workspace, workspace_bytes, L.grad_bytes))) return rc;
    char *ws = (char *)workspace;
    cudaStream_t s = (cudaStream_t)stream;
    const int32_t width = (int32_t)c->width;
    float *const peaks = (float *)(ws + L.peaks);
    const uint16_t *const tidy = (const uint16_t *)(ws + L.tidy);
    if (tokens) {
        const TidyArgs A{(const uint16_t *)h, (uint16_t *)(ws + L.tidy), targets, dloss, peaks, tokens, c->rows, c->width, ld_h, L.ld, wide,
                         units(c->width, h) && ld_h % 8 == 0, false};
        if ((rc = ops_cuda(launch_tidy(A, s), "k_tidy"))) return rc;
    }
    for (int64_t v0 = 0; v0 < c->rows; v0 += L.piece) {
        const int64_t n = c->rows - v0 < L.piece ? c->rows - v0 : L.piece;
        const uint16_t *w = (const uint16_t *)table + v0 * c->width;
        const bool first = v0 == 0, last = v0 + n == c->rows;
        if (tokens) {
            ProductArgs P{};  // the logits' gradient: (tokens, n)
            P.a = tidy;
            P.b = w;
            P.lda = L.ld;
            P.peaks = peaks;
            P.ldb = c->width;
            P.rows = tokens;
            P.groups = 1;
            P.inner = width;
            P.cols = (int32_t)n;
            P.scale = c->scale;
            P.flags = (wide ? kIds64 : 0) | kOutVec | kRelease;
            P.targets = targets;
            P.first = v0;
            P.vocab = c->rows;
            P.lse = lse;
            P.dloss = dloss;
            P.out = ws;
            P.ldo = L.piece;
            if ((rc = ops_cuda(product_launch(kByCols, kLogitsGrad, P, s), "k_product"))) return rc;
            ProductArgs H{};  // its share of dh
            H.a = ws;
            H.b = w;
            H.lda = L.piece;
            H.ldb = c->width;
            H.rows = tokens;
            H.groups = 1;
            H.inner = (int32_t)n;
            H.cols = width;
            H.scale = c->scale;
            H.peaks = peaks;
            H.parts = L.dh_parts ? (float *)(ws + L.shares) : nullptr;
            H.base = first ? nullptr : ws + L.sums;
            H.out = last ? dh : ws + L.sums;
            H.ldo = c->width;
            H.flags = kBase32 | (last ? 0 : kOut32) | (units(c->width, H.out) ? kOutVec : 0) | kRelease;
            if ((rc = ops_cuda(product_launch(kByRows, kStore, H, s), "k_product"))) return rc;
        }
        ProductArgs W{};  // its rows of dW
        W.a = ws;
        W.b = tidy;
        W.lda = L.piece;
        W.ldb = L.ld;
        W.peaks = tokens ? peaks : nullptr;
        W.parts = product_parts_bytes(1, n, c->width) ? (float *)(ws + L.shares) : nullptr;
        W.rows = tokens;
        W.groups = 1;
        W.inner = (int32_t)n;
        W.cols = width;
        W.scale = c->scale;
        W.base = base ? (const uint16_t *)base + v0 * c->width : nullptr;
        W.out = (uint16_t *)dtable + v0 * c->width;
        W.ldo = c->width;
        W.flags = (units(c->width, W.out) && units(c->width, base) ? kOutVec : 0) | (last ? 0u : uint32_t(kRelease));
        if ((rc = ops_cuda(product_launch(kOuter, kStore, W, s), "k_product"))) return rc;
    }
    return SKEW_OK;
}

}  // extern "C"
