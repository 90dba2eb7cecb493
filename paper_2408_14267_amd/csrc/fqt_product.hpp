// The products of a linear layer's backward pass for callers that have dz in bf16 already
// (fqt_linear.hip has them; fqt_loss.hip makes dz piece by piece).
#pragma once

#include "fqt_tile.hpp"

namespace fqt {
namespace dense {

// Plan of a product of operands of e bytes, and the bytes of its partial sums.
tile::Plan plan_of(int64_t M, int64_t N, int64_t K, size_t e, const tile::Costs &costs = tile::DENSE_COSTS);
size_t part_bytes(const tile::Plan &p, int64_t M, int64_t N);
// Up to this many rows fqt_linear_forward is a product on the vector units, one launch that takes no workspace (callers keep other
// things there).
constexpr int FEW_MOST = 4;
inline int64_t round_up(int64_t v, int64_t q) { return (v + q - 1) / q * q; }
// Whether rows of n elements of e bytes, ld apart, are whole 16-byte pieces.
inline bool whole_pieces(int64_t n, int64_t ld, size_t e) { return n * e % 16 == 0 && ld * e % 16 == 0; }

// Partial column sums [parts][N] of dz, added up to dbias (null: not asked for).
struct DbiasArgs {
  const float *part;
  float *dbias;
  int64_t N;
  int32_t parts;
};
// dx and dw in one launch of tiles of one shape, the longer contraction's first and perhaps split: the tiles that a last
// round of one leaves CUs idle with run beside those of the other.
struct Together {
  bool on;                 // (off: one after the other by their plans)
  int shape;
  tile::Tiles dx, dw;
};
// The cheapest of these by tile::STEP_COSTS, on if it takes less time than the two plans.
Together plan_together(int64_t M, int64_t N, int64_t K, const tile::Plan &dx, const tile::Plan &dw);
size_t part_bytes(const Together &t, int64_t M, int64_t N, int64_t K);

// dx = dz w + add and dw = dz^T x, each computed where its pointer is given.  dzx and dzw: dz as it goes into
// either, rows of M; w and x: operands along the features, their `rows` features.  add: float32 of row stride
// ldadd, may be dx itself; null for none.
struct Gradients {
  int64_t M, N, K;
  tile::Operand dzx, dzw, w, x;
  tile::Plan plan_dx, plan_dw;
  void *dx, *dw;
  const float *add;
  int64_t lddx, ldadd, lddw;
  int32_t dx_dtype, dw_dtype;
  float *part;             // part_bytes of either plan, or of both together
  DbiasArgs bias;
  Together together;
};
int launch_gradients(const Gradients &g, hipStream_t st);
// Rows of src (cols elements, stride ld) to rows of `pitch` elements, zero past cols.
struct Copy {
  const void *src;
  void *dst;
  int64_t rows, cols, ld, pitch;
  uint32_t blocks;         // workgroups of 256 threads (0: no copy)
};
// The copy of an operand into rows of `pitch` elements of e bytes.
Copy copy_of(const void *src, int64_t rows, int64_t cols, int64_t ld, void *dst, int64_t pitch, int64_t e);
// Both copies in one launch; widen: 8-bit codes to bf16 (exact).
int launch_copies(const Copy &x, const Copy &w, int32_t dtype, bool widen, hipStream_t st);

// Writes zeros to a matrix.
int zero_matrix(void *p, int64_t rows, int64_t cols, int64_t ld, size_t e, hipStream_t st);

}  // namespace dense
}  // namespace fqt
