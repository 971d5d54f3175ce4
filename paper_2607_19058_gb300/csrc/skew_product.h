// Matrix products on the tensor cores, of bf16 with sums in fp32, as the experts' products and the output head's
// loss need them (skew_product.cu). Not part of the public ABI.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace skew {

// What is multiplied. A "line" is a run of memory: 64 contiguous elements of it, at a time, come to shared memory.
//   BY_ROWS    : C[r, j] = sum_k A[r, k] B_e[k, j]   A: lines of k, one for each row r of the group e; B: lines of j  (STORE)
//   BY_COLS    : C[r, j] = sum_k A[r, k] B[j, k]     A: as above;                       B: lines of k    (LOSS, LOGITS_GRAD)
//   OUTER      : C_e[i, j] = sum_r A[r, i] B[r, j]   A: lines of i, B: lines of j, one for each row r of the group e
//   GROUP_ROWS : C[r, j] = sum_k B[r, k] A_e[k, j]   A: lines of j, B: lines of k, one for each row r, of the group e
//   GROUP_COLS : C[r, j] = sum_k B[r, k] A_e[j, k]   A: lines of k, B: as above
// The GROUP kinds turn the tile: its 256 rows are columns of the matrix, of which there are always enough, and its columns the group's rows, as few as 64.
enum ProductKind { kByRows, kByCols, kOuter, kGroupRows, kGroupCols };

// What becomes of a tile of sums.
//   STORE  : out = base + scale * peak * C
//   LOSS   : of x = scale * C, per row and tile, the largest and the sum of exponentials; the target's x
//   LOGITS_GRAD : out = (exp(x - lse) - [j is the target]) * dloss / peak, bf16
enum ProductEnd { kStore = 0, kLoss = 1, kLogitsGrad = 2 };

enum : uint32_t { kOut32 = 1, kBase32 = 2, kOutVec = 4 /* out and base: 16-byte accesses */, kIds64 = 8,
                kRelease = 16 /* a launch of the same call follows, which may start up while this one ends */ };

struct ProductArgs {
    const void *a, *b;          // bf16
    int64_t lda, ldb, a_group, b_group;  // elements between lines, and between A's groups (GROUP) or B's (BY_ROWS)
    const int32_t *offsets;     // groups + 1 row numbers on the device; NULL: one group of all rows
    int64_t rows;               // r in [0, rows)
    int32_t groups, cols;       // j in [0, cols)
    int32_t inner;              // k, or OUTER's i, in [0, inner)
    uint32_t flags;
    void *out;
    const void *base;           // strides as out; may be out
    int64_t ldo, o_group;
    float scale;
    float *parts;               // product_parts_bytes() for the sums of tiles that are cut along the summed index (STORE of OUTER or BY_ROWS); NULL: none is
    const float *peaks;         // kPeaks numbers that are not negative, or NULL. LOGITS_GRAD divides by the largest, STORE multiplies by it
    int32_t splits, chunk;      // set by product_launch: shares of the summed index; its steps between two additions outside of the tensor cores
    // LOSS, LOGITS_GRAD
    const void *targets;        // one for each row; not in [0, vocab): none
    int64_t first, vocab;       // the column j is the vocabulary's `first` + j
    const float *lse, *dloss;
    float2 *part;               // [part of a row][rows]: (largest, sum) in powers of two
    float *picked;              // [rows]: the target's x, in powers of two (x log2 e)
};

constexpr int kPeaks = 512;

// Bytes for the parts of a result of `groups` matrices of height x cols (BY_ROWS: one, of rows x cols); 0 where its tiles are too many to be cut.
size_t product_parts_bytes(int64_t groups, int64_t height, int64_t cols);
// Columns of a LOSS part.
int32_t product_loss_columns();
// Runs the product on `stream`; every pointer, size and stride has been checked.
cudaError_t product_launch(ProductKind kind, ProductEnd end, const ProductArgs &A, cudaStream_t stream);
// Synchronises, and reads and clears the word in which a wait on the device that gave up leaves its mark: a SKEW_* code.
int product_status(cudaStream_t stream);

}  // namespace skew
