// The experts' products (skewadam.h): checks, and the products of skew_product.cu that they are.
#include "skew_ops.h"
#include "skew_product.h"

namespace skew {
namespace {

constexpr int64_t kMaxRows = int64_t(1) << 30;
constexpr int kMaxExperts = 1024;

int check(const skew_experts_config_t *c, int64_t rows, const int32_t *offsets) {
    if (!c) return ops_fail(SKEW_EINVAL, "config is NULL");
    if (c->experts < 1 || c->experts > kMaxExperts) return ops_fail(SKEW_EINVAL, "experts must be in [1, %d]", kMaxExperts);
    if (c->n < 1 || c->n > 1 << 20 || c->m < 1 || c->m > 1 << 20) return ops_fail(SKEW_EINVAL, "n and m must be in [1, 2^20]");
    if (c->flags & ~(SKEW_EXPERTS_ROWS_FP32 | SKEW_EXPERTS_GRAD_FP32)) return ops_fail(SKEW_EINVAL, "unknown flags");
    if (rows < 0 || rows > kMaxRows) return ops_fail(SKEW_EINVAL, "rows must be in [0, 2^30]");
    if (!offsets || ((uintptr_t)offsets & 3)) return ops_fail(SKEW_EINVAL, "offsets must be a device pointer aligned to its type");
    return SKEW_OK;
}

int check_rows(const char *what, const void *p, int64_t rows, int64_t width, int64_t ld) {
    if ((rows && !p) || ((uintptr_t)p & 1)) return ops_fail(SKEW_EINVAL, "%s must be a device pointer aligned to its type", what);
    if (ld < width || ld > int64_t(1) << 31) return ops_fail(SKEW_EINVAL, "row stride must be in [width, 2^31]");
    return SKEW_OK;
}

int check_ptr(const char *what, const void *p, uintptr_t es, bool needed) {
    if ((needed && !p) || ((uintptr_t)p & (es - 1))) return ops_fail(SKEW_EINVAL, "%s must be a device pointer aligned to its type", what);
    return SKEW_OK;
}

// Rows of an expert, on average over all experts (those without rows too: what each has is known on the device alone), from which on `product` takes the rows as a
// tile's rows, 256 at a time, instead of its columns, 64 at a time. (The matrices, whose lines lie across the summed index, are the slower operand of a tile's rows; but half a
// tile is wasted, and a tile of few rows takes longer to write out. us straight / turned for 64, 128, 256, 384 and 512 rows each, uneven loads: 128 experts of 4096 x 4096
// 689 / 650, 729 / 691, 970 / 946, 1269 / 1358, 1592 / 1757; 256 of 2048 x 512 107 / 102, 124 / 122, 150 / 144, 195 / 189, 236 / 230; 64 of 4096 x 1024 105 / 107, 108 / 108,
// 130 / 130, 172 / 170, 214 / 216. Even loads of 384 differ the most: 1264 / 1539 at 4096 x 4096, 171 / 182 at 4096 x 1024, 195 / 190 at 2048 x 512. grad_rows, whose lines
// lie along the summed index, is turned always: 1774 straight, 1795 turned at 512 rows, and 46 against 23 for 17 rows of 164 experts of 1648 x 128.)
constexpr int64_t kStraightRows = 384;

// The two products by rows: of `inner` columns each, times one matrix a group, to `cols` columns.
int by_rows(ProductKind kind, const skew_experts_config_t *c, const void *x, int64_t ld, const void *w, const int32_t *offsets, int64_t rows, void *y, cudaStream_t s) {
    const bool wide = c->flags & SKEW_EXPERTS_ROWS_FP32;
    const int32_t inner = kind == kGroupRows ? c->n : c->m, cols = kind == kGroupRows ? c->m : c->n;
    int rc;
    if ((rc = check_rows("rows", x, rows, inner, ld)) || (rc = check_ptr("w", w, 2, true)) || (rc = check_ptr("result", y, wide ? 4 : 2, rows > 0))) return rc;
    if (!rows) return SKEW_OK;
    ProductArgs A{};
    const bool straight = kind == kGroupRows && rows >= kStraightRows * c->experts;
    A.a = straight ? x : w;
    A.b = straight ? w : x;
    A.lda = straight ? ld : c->m;
    A.ldb = straight ? c->m : ld;
    A.a_group = A.b_group = int64_t(c->n) * c->m;
    A.offsets = offsets;
    A.rows = rows;
    A.groups = c->experts;
    A.inner = inner;
    A.cols = cols;
    A.out = y;
    A.ldo = cols;
    A.scale = 1.f;
    A.flags = (wide ? kOut32 : 0) | (cols % 8 == 0 && ((uintptr_t)y & 15) == 0 ? kOutVec : 0);
    return ops_cuda(product_launch(straight ? kByRows : kind, kStore, A, s), "k_product");
}

}  // namespace
}  // namespace skew

using namespace skew;

extern "C" {

int skew_experts_product(const skew_experts_config_t *c, const void *x, int64_t ld_x, const void *w, const int32_t *offsets, int64_t rows, void *y, void *stream) {
    const int rc = check(c, rows, offsets);
    return rc ? rc : by_rows(kGroupRows, c, x, ld_x, w, offsets, rows, y, (cudaStream_t)stream);
}

int skew_experts_grad_rows(const skew_experts_config_t *c, const void *dy, int64_t ld_dy, const void *w, const int32_t *offsets, int64_t rows, void *dx,
                           void *stream) {
    const int rc = check(c, rows, offsets);
    return rc ? rc : by_rows(kGroupCols, c, dy, ld_dy, w, offsets, rows, dx, (cudaStream_t)stream);
}

size_t skew_experts_workspace_bytes(const skew_experts_config_t *c) {
    if (check(c, 0, (const int32_t *)4) != SKEW_OK) return 0;
    const size_t parts = product_parts_bytes(c->experts, c->n, c->m);
    return parts ? parts : 256;
}

int skew_experts_grad(const skew_experts_config_t *c, const void *x, int64_t ld_x, const void *dy, int64_t ld_dy, const int32_t *offsets, int64_t rows,
                      const void *base, void *dw, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check(c, rows, offsets);
    if (rc) return rc;
    const bool wide = c->flags & SKEW_EXPERTS_GRAD_FP32;
    if ((rc = check_rows("x", x, rows, c->n, ld_x)) || (rc = check_rows("dy", dy, rows, c->m, ld_dy)) || (rc = check_ptr("base", base, wide ? 4 : 2, false)) ||
        (rc = check_ptr("dw", dw, wide ? 4 : 2, true)))
        return rc;
    const size_t need = skew_experts_workspace_bytes(c);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)
        return ops_fail(SKEW_EINVAL, "workspace must be 256-byte aligned and at least %zu bytes", need);
    ProductArgs A{};
    A.parts = product_parts_bytes(c->experts, c->n, c->m) ? (float *)workspace : nullptr;
    A.a = x;
    A.b = dy;
    A.lda = ld_x;
    A.ldb = ld_dy;
    A.offsets = offsets;
    A.rows = rows;
    A.groups = c->experts;
    A.inner = c->n;
    A.cols = c->m;
    A.out = dw;
    A.base = base;
    A.ldo = c->m;
    A.o_group = int64_t(c->n) * c->m;
    A.scale = 1.f;
    A.flags = (wide ? kOut32 | kBase32 : 0) | (c->m % 8 == 0 && (((uintptr_t)dw | (uintptr_t)base) & 15) == 0 ? kOutVec : 0);
    return ops_cuda(product_launch(kOuter, kStore, A, (cudaStream_t)stream), "k_product");
}

}  // extern "C"
