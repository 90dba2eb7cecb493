// Newton-Schulz orthogonalisation and the optimizer step on it.
//
// X is kept on the short side of the matrix (m x n, m <= n), padded with zeros to multiples of 64, as
// float16 pairs hi + lo of X 2^15 (hi the nearest float16, lo the nearest to the rest): 22 bits and
// their rounding, as good as float32 where entries are not 2^-24 of the largest.  A product is the sum
// of hi hi, hi lo and lo hi on the 16-bit matrix cores with float32 sums; lo lo is below the rounding.
// That is three matrix instructions at 16 times the rate of the float32 ones.
//
// The powers of two keep every entry inside float16: the singular values of X stay below 1.21 (the
// quintic maps [0, 1.21] into itself), so |X| < 2^15 1.21, |P| = |X X^T| < 1.47 (2^14) and
// |b P + c P^2| < 2.81 (2^13) are below 65504 with the factors in brackets.
//
// A step is three products: P = X X^T and Q = b P + c P P, both symmetric, of which only the tiles on
// and above the diagonal are computed and stored twice; X' = a X + Q X, which reads X along m (PANEL_COLS).
// The last step's product stores the result, or updates the weights, instead of X'.
#include "fqt_tile.hpp"

namespace fqt {
namespace dense {
namespace {

#pragma clang fp contract(fast)

using tile::Operand;
using tile::PANEL_ROWS;
using tile::PANEL_COLS;

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
// Where |u| is small beside eps the first X_i are: |X_i| <= a^i |X_0|.  Step i then stores its X, P and Q with
// k_i more bits of scale (2^15+k, 2^14+2k, 2^13+2k; 2^-k_i the power of two above a^i |X_0|, k_i = 0 where that
// reaches 1/2), so that float16 holds the smallest gradients as well as any, whatever the number of
// steps.  The factors depend on |u|, so they stay on the device, one set a step:
struct Units {
  float down;            // 2^-2k, in the terms of Q and X' that have P once more
  float up;              // 2^(k' - k) to the next step's k' (1 after the last step)
  float out;             // 2^-k, from the stored X 2^-15 to X
};
constexpr int MAX_STEPS = 32;

struct Split { uint16_t hi, lo; };
__device__ __forceinline__ Split split(float v) {
  const _Float16 h = static_cast<_Float16>(v);
  const _Float16 l = static_cast<_Float16>(v - static_cast<float>(h));
  return {__builtin_bit_cast(uint16_t, h), __builtin_bit_cast(uint16_t, l)};
}
__device__ __forceinline__ float join(uint16_t hi, uint16_t lo) {
  return static_cast<float>(__builtin_bit_cast(_Float16, hi)) + static_cast<float>(__builtin_bit_cast(_Float16, lo));
}
// A matrix of pairs in panels of 32 columns (tile::SPLITK): row r of panel c is the 64 values
// at (c * rows + r) * 64.
struct Pairs {
  uint16_t *p;
  int64_t rows;
  __device__ __forceinline__ uint16_t *at(int64_t r, int64_t c) const {
    return p + (c / 32 * rows + r) * 64 + c % 32;
  }
};
// 8 columns from c (a multiple of 8) of row r.
__device__ __forceinline__ void store_split8(const Pairs &p, int64_t r, int64_t c, const float (&v)[8]) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const Split a = split(v[2 * i]), b = split(v[2 * i + 1]);
    h[i] = a.hi | uint32_t(b.hi) << 16;
    l[i] = a.lo | uint32_t(b.lo) << 16;
  }
  uint16_t *q = p.at(r, c);
  *reinterpret_cast<uint4 *>(q) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4 *>(q + 32) = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ void load_split8(const Pairs &p, int64_t r, int64_t c, float (&v)[8]) {
  const uint16_t *q = p.at(r, c);
  const uint4 h = *reinterpret_cast<const uint4 *>(q), l = *reinterpret_cast<const uint4 *>(q + 32);
  const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = join(uint16_t(hw[i]), uint16_t(lw[i]));
    v[2 * i + 1] = join(uint16_t(hw[i] >> 16), uint16_t(lw[i] >> 16));
  }
}

// ----------------------------------------------------------------------------- u and its norm

struct Source {
  const void *g;
  float *m;              // momentum, or null
  int64_t rows, cols, ldg, ldm;
  int32_t g_dtype, nesterov;
  float momentum;
};
// u of 8 columns from c of row r, 0 past the matrix.  UPDATE: the momentum takes its step first.
template <bool UPDATE>
__device__ __forceinline__ void load_u(const Source &s, int64_t r, int64_t c, float (&u)[8]) {
  const int n = int(min(s.cols - c, int64_t(8)));
  if (r >= s.rows || n <= 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = 0.0f;
    return;
  }
  if (!s.m || UPDATE || s.nesterov) {
    const int64_t at = r * s.ldg + c;
    if (s.g_dtype == FQT_BF16) load8f(static_cast<const bf16 *>(s.g) + at, n, u);
    else load8f(static_cast<const float *>(s.g) + at, n, u);
  }
  if (s.m) {
    float *p = s.m + r * s.ldm + c;
    float m[8];
    load8f(p, n, m);
    if constexpr (UPDATE) {
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = fmaf(s.momentum, m[i], u[i]);
      store8f(p, n, m);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = s.nesterov ? fmaf(s.momentum, m[i], u[i]) : m[i];
  }
}
constexpr int NORM_BLOCKS = 1024;

__device__ __forceinline__ double block_sum(double v, double *slots) {        // of 256 threads
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) slots[threadIdx.x / 64] = v;
  __syncthreads();
  return slots[0] + slots[1] + slots[2] + slots[3];
}

// Updates the momentum and adds up u^2 in float64 (no overflow, no underflow), a partial sum per
// workgroup; groups: 8-column groups of a row.
__global__ void __launch_bounds__(256) k_ns_norm(Source s, FastDiv groups, uint32_t all, double *part) {
  __shared__ double slots[4];
  double sum = 0.0;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += gridDim.x * 256) {
    const uint32_t r = fdiv(i, groups);
    float u[8];
    load_u<true>(s, r, int64_t(i - r * groups.d) * 8, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += double(u[j]) * double(u[j]);
  }
  sum = block_sum(sum, slots);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}
// 2^(15+k_0) / (|u| + eps) from the partial sums; one workgroup writes the units of the steps.
struct Start {
  const double *part;
  int32_t parts, steps;
  float eps;
  Units *units;
};
__device__ __forceinline__ double unit_scale(const Start &s, double *slots, bool write) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < s.parts; i += 256) sum += s.part[i];
  const double norm = sqrt(block_sum(sum, slots));
  double most = norm / (norm + double(s.eps));             // bound of |X_i|, i = 0 here
  // |X_i| < 2^-k: X below 2^15, P below 2^14, Q (|b| P at most) below 4.8 2^13.  (NaN: 0)
  auto bits = [](double v) { return v > 0.0 ? max(0, -ilogb(v) - 1) : 0; };
  const double inv = ldexp(1.0, 15 + bits(most)) / (norm + double(s.eps));
  if (const int i = threadIdx.x; write && i < s.steps) {   // a thread a step
    for (int j = 0; j < i; ++j) most = fmin(1.0, most * double(NS_A));
    const int k = bits(most), next = i + 1 < s.steps ? bits(fmin(1.0, most * double(NS_A))) : k;
    s.units[i] = {ldexpf(1.0f, -2 * k), ldexpf(1.0f, next - k), ldexpf(1.0f, -k)};
  }
  return inv;
}
// The 64 x 64 tile of X_0 2^15 at (x0, y0): put(row, column, 8 values) in the tile.  Tall matrices are
// transposed on the way, through t.
template <bool TALL, typename F>
__device__ __forceinline__ void start_tile(const Source &s, double inv, int64_t x0, int64_t y0, float (*t)[65], F &&put) {
  if constexpr (TALL) {
    for (int i = threadIdx.x; i < 512; i += 256) {
      float u[8];
      load_u<false>(s, y0 + i / 8, x0 + i % 8 * 8, u);
#pragma unroll
      for (int j = 0; j < 8; ++j) t[i % 8 * 8 + j][i / 8] = float(u[j] * inv);
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < 512; i += 256) {
    float v[8];
    if constexpr (TALL) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = t[i / 8][i % 8 * 8 + j];
    } else {
      load_u<false>(s, x0 + i / 8, y0 + i % 8 * 8, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = float(v[j] * inv);
    }
    put(i / 8, i % 8 * 8, v);
  }
}
// X_0 = u / (|u| + eps) as pairs, zeros in the padding.
template <bool TALL>
__global__ void __launch_bounds__(256) k_ns_start(Source s, Start b, Pairs x) {
  __shared__ double slots[4];
  __shared__ float t[TALL ? 64 : 1][65];
  const double inv = unit_scale(b, slots, blockIdx.x + blockIdx.y == 0);
  const int64_t x0 = int64_t(blockIdx.y) * 64, y0 = int64_t(blockIdx.x) * 64;
  start_tile<TALL>(s, inv, x0, y0, t, [&](int r, int c, const float (&v)[8]) { store_split8(x, x0 + r, y0 + c, v); });
}

// ----------------------------------------------------------------------------- products

enum Mode { GRAM, POLY, APPLY };
struct NsArgs {
  Pairs x, p, q, next;   // X [mp][np]; P, Q [mp][mp]; the next X
  int64_t mp, np;
  int64_t m, n;          // without padding
  tile::Tiles tiles;
  float *part;
  const Units *units;    // this step's
  // the last step's result
  void *out;             // o, or null
  float *w;              // weights, or null
  int64_t ldo;
  int32_t last, o_dtype, tall;
  float keep, rate;      // w = keep w - rate X
};

// The last step's X', 8 columns from n of row m: v is X' 2^(15+k).
__device__ __forceinline__ void store_result8(const NsArgs &a, int64_t m, int64_t n, const float (&v)[8]) {
  if (m >= a.m) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (n + i >= a.n) break;
    const int64_t at = a.tall ? (n + i) * a.ldo + m : m * a.ldo + n + i;
    const float o = v[i] * 0x1p-15f * a.units->out;
    if (a.w) a.w[at] = fmaf(a.keep, a.w[at], -a.rate * o);
    else if (a.o_dtype == FQT_BF16) static_cast<bf16 *>(a.out)[at] = from_f32<bf16>(o);
    else static_cast<float *>(a.out)[at] = o;
  }
}
// P 2^14 from sums 2^30; Q 2^13 from sums 2^28 and P 2^14; X' 2^15 from sums 2^28 and X 2^15 (and the k
// bits of each; down = 2^-2k, up = 2^(k'-k)).
__device__ __forceinline__ float gram_of(float sum) { return sum * 0x1p-16f; }
__device__ __forceinline__ float poly_of(float sum, float p, float down) {
  return fmaf(NS_B * 0.5f, p, sum * (NS_C * 0x1p-15f) * down);
}
__device__ __forceinline__ float apply_of(float sum, float x, const Units &u) { return fmaf(NS_A, x, sum * 0x1p-13f * u.down) * u.up; }

// The epilogue of 8 consecutive n (tile::run_epilogue).  diagonal: the tile holds its own mirror image.
template <int MODE>
struct Finish {
  static constexpr int DEPTH = MODE == GRAM ? 1 : 4;
  static constexpr bool MIRROR = MODE != APPLY, SUMS = false;
  struct Fetch { float x[MODE == GRAM ? 1 : 8]; };         // X, or P
  const NsArgs &a;
  bool diagonal;
  __device__ __forceinline__ bool in(int64_t m, int64_t n) const {
    return m < a.mp && n < (MODE == APPLY ? a.np : a.mp);
  }
  Units units;
  __device__ __forceinline__ void columns(int64_t) {
    if constexpr (MODE != GRAM) units = *a.units;
  }
  __device__ __forceinline__ Fetch fetch(int64_t m, int64_t n) {
    Fetch f;
    if constexpr (MODE != GRAM)
      if (in(m, n)) load_split8(MODE == APPLY ? a.x : a.p, m, n, f.x);
    return f;
  }
  __device__ __forceinline__ void finish(int64_t m, int64_t n, float (&v)[8], const Fetch &f) {
    if (!in(m, n)) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (MODE == GRAM) v[i] = gram_of(v[i]);
      else if constexpr (MODE == POLY) v[i] = poly_of(v[i], f.x[i], units.down);
      else v[i] = apply_of(v[i], f.x[i], units);
    }
    if (MODE == APPLY && a.last) store_result8(a, m, n, v);
    else store_split8(MODE == GRAM ? a.p : MODE == POLY ? a.q : a.next, m, n, v);
  }
  __device__ __forceinline__ void mirror(int64_t n, int64_t m, const float (&v)[8]) {
    if (!diagonal && in(m, n)) store_split8(MODE == GRAM ? a.p : a.q, n, m, v);
  }
};

template <int MODE, int SHAPE>
__global__ void __launch_bounds__(tile::ShapeOf<SHAPE>::type::THREADS, 2) k_ns(NsArgs a) {
  typedef typename tile::ShapeOf<SHAPE>::type S;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];
  const tile::Place at = tile::place<SHAPE>(a.tiles, blockIdx.x);
  const int64_t K = MODE == GRAM ? a.np : a.mp;
  if (at.m0 >= a.mp || at.n0 >= (MODE == APPLY ? a.np : a.mp)) return;       // (parts of an edge tile)
  // rows: of the result along the operand; a panel holds `rows of the matrix` x 128 bytes
  auto op = [&](const Pairs &p, int64_t rows) {
    return Operand{reinterpret_cast<const char *>(p.p), p.rows * tile::KB, rows};
  };
  typename tile::Acc<tile::SPLITK>::type acc[S::FM][S::FN];
  if constexpr (MODE == GRAM)
    tile::contract<tile::SPLITK, PANEL_ROWS, PANEL_ROWS, SHAPE, S>(op(a.x, a.mp), op(a.x, a.mp), K, at, a.tiles, lds, acc);
  else if constexpr (MODE == POLY)
    tile::contract<tile::SPLITK, PANEL_ROWS, PANEL_ROWS, SHAPE, S>(op(a.p, a.mp), op(a.p, a.mp), K, at, a.tiles, lds, acc);
  else
    tile::contract<tile::SPLITK, PANEL_ROWS, PANEL_COLS, SHAPE, S>(op(a.q, a.mp), op(a.x, a.np), K, at, a.tiles, lds, acc);
  if constexpr (MODE != APPLY)
    if (a.tiles.splits > 1) {
      tile::run_epilogue<tile::SPLITK, S>(acc, lds, at.m0, at.n0,
                                          tile::StorePart{a.part + at.split * a.mp * a.mp, a.mp, a.mp});
      return;
    }
  tile::run_epilogue<tile::SPLITK, S>(acc, lds, at.m0, at.n0, Finish<MODE>{a, at.diagonal});
}

// The partial sums of a split symmetric product, added in order: a workgroup per 64 x 64 tile on or above
// the diagonal of tiles of edge B, whose mirror image goes out through LDS.
template <int MODE, int B>
__global__ void __launch_bounds__(512) k_ns_join_symmetric(NsArgs a) {
  __shared__ float t[64][65];
  const int64_t m0 = int64_t(blockIdx.y) * 64, n0 = int64_t(blockIdx.x) * 64;
  if (m0 / B > n0 / B) return;
  Finish<MODE> f{a, m0 / B == n0 / B};
  f.columns(n0);
  const int r = threadIdx.x / 8, c = threadIdx.x % 8 * 8;
  const auto q = f.fetch(m0 + r, n0 + c);
  float v[8] = {};
#pragma unroll 8
  for (uint32_t s = 0; s < a.tiles.splits; ++s) {
    float u[8];
    load8f(a.part + (s * a.mp + m0 + r) * a.mp + n0 + c, 8, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += u[j];
  }
  f.finish(m0 + r, n0 + c, v, q);
  if (f.diagonal) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) t[r][c + j] = v[j];
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = t[c + j][r];
  f.mirror(n0 + r, m0 + c, v);
}

// ----------------------------------------------------------------------------- few rows
// Up to 64 rows: a launch or two per step instead of three or four.  Workgroup b keeps columns
// [b slice, (b + 1) slice) of X.  It adds up everyone's partial sums of P (in order), takes Q from it in
// LDS, and goes over its columns 64 at a time: X' = a X + Q X, and its part of the next P = X' X'^T.
// Past DIRECT workgroups the sums are joined by a launch of their own (64 x 25088: 10 + 5 instead of 32 us
// a step on 32 workgroups).  All operands are 64 rows of 128 bytes per 32 columns, swizzled as
// fqt_tile.hpp says.
struct SmallArgs {
  NsArgs n;
  const float *from;     // [workgroups][64][64] partial sums of P 2^30
  float *to;
  int64_t slice;         // columns of a workgroup, a multiple of 64
};
constexpr int PANEL = 64 * tile::KB;                       // bytes of 32 columns
constexpr int SMALL_BLOCKS = 256, DIRECT = 32;             // workgroups at most; reading all partial sums

// Byte offset of columns n ... (8-byte steps) of row m of a matrix of row panels, plane hi or lo.
__device__ __forceinline__ uint32_t panel_at(uint32_t m, uint32_t n, int lo) {
  return n / 32 * PANEL + m * tile::KB + (((n % 32 / 8 + 4 * lo) ^ (m & 7)) * 16) + (n & 7) * 2;
}
__device__ __forceinline__ void put4(char *lds, uint32_t m, uint32_t n, const float (&v)[4]) {
  Split s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = split(v[i]);
  *reinterpret_cast<uint2 *>(lds + panel_at(m, n, 0)) = make_uint2(s[0].hi | uint32_t(s[1].hi) << 16, s[2].hi | uint32_t(s[3].hi) << 16);
  *reinterpret_cast<uint2 *>(lds + panel_at(m, n, 1)) = make_uint2(s[0].lo | uint32_t(s[1].lo) << 16, s[2].lo | uint32_t(s[3].lo) << 16);
}
__device__ __forceinline__ void join4(const char *hi, const char *lo, float (&v)[4]) {
  const uint2 h = *reinterpret_cast<const uint2 *>(hi), l = *reinterpret_cast<const uint2 *>(lo);
  v[0] = join(uint16_t(h.x), uint16_t(l.x));
  v[1] = join(uint16_t(h.x >> 16), uint16_t(l.x >> 16));
  v[2] = join(uint16_t(h.y), uint16_t(l.y));
  v[3] = join(uint16_t(h.y >> 16), uint16_t(l.y >> 16));
}
typedef tile::f32x4 SmallAcc[2][2];
// acc += x w^T over 64 k's; LW: PANEL_ROWS (rows of w along k) or PANEL_COLS (two steps of 32 k's).
template <int LW>
__device__ __forceinline__ void small_product(const char *x, const char *w, uint32_t wm, uint32_t wn, SmallAcc &acc) {
  tile::Reader<PANEL_ROWS, 64, 2> rx;
  tile::Reader<LW, 64, 2> rw;
  rx.init(wm);
  rw.init(wn);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    tile::i32x4 fx[2][2], fw[2][2];
    rx.template read<true>(x + s * PANEL, 0, fx);
    rw.template read<true>(w + s * PANEL, 0, fw);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) tile::mma<tile::SPLITK>(acc[i][j], fw[j], fx[i]);
  }
}
__device__ __forceinline__ void store_small_part(const SmallAcc &acc, uint32_t wm, uint32_t wn, float *to) {
  const uint32_t l = __lane_id();
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
      *reinterpret_cast<tile::f32x4 *>(to + (wm + i * 16 + l % 16) * 64 + wn + j * 16 + 4 * (l / 16)) = acc[i][j];
}
// 64 columns of row panels between LDS and X (at column n).
__device__ __forceinline__ void panels_out(const char *lds, const Pairs &x, int64_t n) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t p = k * 256 + threadIdx.x, panel = p / 512, m = p / 8 % 64, piece = p % 8;
    const uint4 v = *reinterpret_cast<const uint4 *>(lds + panel * PANEL + m * tile::KB + ((piece ^ (m & 7)) * 16));
    *reinterpret_cast<uint4 *>(x.p + ((n / 32 + panel) * 64 + m) * 64 + piece * 8) = v;
  }
}

// out = the partial sums added up: 16 four-entry groups per workgroup, 16 threads each.
__global__ void __launch_bounds__(256) k_ns_small_join(const float *from, int32_t blocks, float *out) {
  __shared__ tile::f32x4 t[16][16];
  const uint32_t at = (blockIdx.x * 16 + threadIdx.x % 16) * 4, k = threadIdx.x / 16;
  tile::f32x4 v{};
#pragma unroll 16
  for (int b = k; b < blocks; b += 16) v += *reinterpret_cast<const tile::f32x4 *>(from + int64_t(b) * 4096 + at);
  t[k][threadIdx.x % 16] = v;
  __syncthreads();
  if (k) return;
#pragma unroll
  for (int j = 1; j < 16; ++j) v += t[j][threadIdx.x];
  *reinterpret_cast<tile::f32x4 *>(out + at) = v;
}

// X_0 and its partial sums of P.
template <bool TALL>
__global__ void __launch_bounds__(256) k_ns_small_start(Source s, Start b, SmallArgs a) {
  __shared__ double slots[4];
  __shared__ float t[TALL ? 64 : 1][65];
  __shared__ __attribute__((aligned(16))) char x[2 * PANEL];
  const double inv = unit_scale(b, slots, blockIdx.x == 0);
  const uint32_t wave = wave_id(), wm = wave / 2 * 32, wn = wave % 2 * 32;
  SmallAcc acc{};
  const int64_t end = min(a.n.np, (blockIdx.x + 1) * a.slice);
  for (int64_t n0 = blockIdx.x * a.slice; n0 < end; n0 += 64) {
    start_tile<TALL>(s, inv, 0, n0, t, [&](int r, int c, const float (&v)[8]) {
      const float lo[4] = {v[0], v[1], v[2], v[3]}, hi[4] = {v[4], v[5], v[6], v[7]};
      put4(x, r, c, lo);
      put4(x, r, c + 4, hi);
    });
    __syncthreads();
    panels_out(x, a.n.x, n0);
    small_product<PANEL_ROWS>(x, x, wm, wn, acc);
    __syncthreads();
  }
  store_small_part(acc, wm, wn, a.to + int64_t(blockIdx.x) * 4096);
}

__global__ void __launch_bounds__(256, 1) k_ns_small(SmallArgs a, int32_t blocks) {
  __shared__ __attribute__((aligned(16))) char p[2 * PANEL], q[2 * PANEL], x[2 * PANEL], y[2 * PANEL];
  const uint32_t wave = wave_id(), l = __lane_id(), wm = wave / 2 * 32, wn = wave % 2 * 32;
  const int64_t n_first = blockIdx.x * a.slice, end = min(a.n.np, n_first + a.slice);
  const Units units = *a.n.units;
  // X is read along its rows' order (m is the contraction)
  const Operand xo{reinterpret_cast<const char *>(a.n.x.p), 64 * tile::KB, a.n.np};
  auto load_x = [&](int64_t n0) {
    tile::Loader<PANEL_COLS, 64, 256> g;
    g.init(xo, n0);
    g.template load<0, 2>(x, 1);
    g.template load<0, 2>(x + PANEL, 1);
  };
  load_x(n_first);
  {
    float v[4][4] = {};
#pragma unroll 8
    for (int b = 0; b < blocks; ++b)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const tile::f32x4 u = *reinterpret_cast<const tile::f32x4 *>(a.from + b * 4096 + (k * 256 + threadIdx.x) * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[k][i] += u[i];
      }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t at = (k * 256 + threadIdx.x) * 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[k][i] = gram_of(v[k][i]);
      put4(p, at / 64, at % 64, v[k]);
    }
  }
  __syncthreads();
  {
    SmallAcc acc{};
    small_product<PANEL_ROWS>(p, p, wm, wn, acc);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t m = wm + i * 16 + l % 16, n = wn + j * 16 + 4 * (l / 16);
        float o[4], v[4];
        join4(p + panel_at(m, n, 0), p + panel_at(m, n, 1), o);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = poly_of(acc[i][j][k], o[k], units.down);
        put4(q, m, n, v);
      }
  }
  SmallAcc gram{};
  for (int64_t n0 = n_first; n0 < end; n0 += 64) {
    __builtin_amdgcn_s_waitcnt(0x0F70);                    // vmcnt(0): x has arrived
    __syncthreads();
    SmallAcc acc{};
    small_product<PANEL_COLS>(q, x, wm, wn, acc);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t m = wm + i * 16 + l % 16, n = wn + j * 16 + 4 * (l / 16);
        // X in the layout of its transposing reads: row m % 32 (hi), 32 + m % 32 (lo) of step m / 32
        const char *at = x + m / 32 * PANEL + m % 32 * tile::KB + ((n / 8 ^ tile::cols_swizzle<64>(m)) * 16) + (n & 7) * 2;
        float o[4], v[4];
        join4(at, at + 32 * tile::KB, o);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = apply_of(acc[i][j][k], o[k], units);
        if (a.n.last) {
          float r[8] = {v[0], v[1], v[2], v[3]};
          NsArgs cut = a.n;
          cut.n = min(a.n.n, n0 + n + 4);
          store_result8(cut, m, n0 + n, r);
        } else {
          put4(y, m, n, v);
        }
      }
    __syncthreads();
    if (n0 + 64 < end) load_x(n0 + 64);
    if (!a.n.last) {
      panels_out(y, a.n.next, n0);
      small_product<PANEL_ROWS>(y, y, wm, wn, gram);
    }
  }
  if (!a.n.last) store_small_part(gram, wm, wn, a.to + int64_t(blockIdx.x) * 4096);
}

// ----------------------------------------------------------------------------- host side

struct NsSizes { int64_t m, n, mp, np, ldg, ldo, ldm; bool tall; };
struct NsWs { size_t norm, x[2], p, q, part, total; tile::Plan gram, poly, apply; };

int check_ortho(const fqt_ortho_desc *d, NsSizes *s) {
  if (!d) return FQT_E_NULL;
  if (!float_type(d->g_dtype) || !float_type(d->o_dtype)) return FQT_E_DTYPE;
  if (d->rows < 0 || d->cols < 0 || d->rows > FQT_MAX_LD || d->cols > FQT_MAX_LD) return FQT_E_SHAPE;
  if (d->steps < 1 || d->steps > MAX_STEPS || !(d->eps > 0.0f) || !std::isfinite(d->eps)) return FQT_E_INVAL;
  s->tall = d->rows > d->cols;
  s->m = std::min(d->rows, d->cols);
  s->n = std::max(d->rows, d->cols);
  s->mp = (s->m + 63) / 64 * 64;
  s->np = (s->n + 63) / 64 * 64;
  s->ldg = row_stride(d->ldg, d->cols);
  s->ldo = row_stride(d->ldo, d->cols);
  s->ldm = row_stride(d->ldm, d->cols);
  // (the norm counts groups of 8 columns in 31 bits)
  if (!s->ldg || !s->ldo || !s->ldm || s->m > 65536 || d->rows * ((d->cols + 7) / 8) >= int64_t(1) << 31)
    return FQT_E_SHAPE;
  return FQT_OK;
}
NsWs ns_ws(const NsSizes &s) {
  NsWs w{};
  w.gram = tile::make_plan(s.mp, s.mp, s.np / 32, true, tile::SYMMETRIC_COSTS);
  w.poly = tile::make_plan(s.mp, s.mp, s.mp / 32, true, tile::SYMMETRIC_COSTS);
  // (X' has at least as many entries as its contraction is long: splitting it never pays)
  w.apply = tile::make_plan(s.mp, s.np, s.mp / 32, false, tile::PAIR_COSTS, 1);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
  w.norm = take(NORM_BLOCKS * sizeof(double) + MAX_STEPS * sizeof(Units));
  const size_t x = size_t(s.mp) * s.np * 4, p = size_t(s.mp) * s.mp * 4;       // two planes of 2 bytes
  w.x[0] = take(x);
  w.x[1] = take(x);
  w.p = take(p);
  w.q = take(p);
  if (s.mp == 64) {        // two sets of partial sums of P, and their sum
    w.part = take((2 * SMALL_BLOCKS + 1) * 4096 * sizeof(float));
    w.total = at;
    return w;
  }
  auto part = [&](const tile::Plan &pl, size_t entries) { return pl.splits > 1 ? size_t(pl.splits) * entries * 4 : 0; };
  w.part = take(std::max(part(w.gram, s.mp * s.mp), part(w.poly, s.mp * s.mp)));
  w.total = at;
  return w;
}

template <int MODE>
int launch_ns(const tile::Plan &plan, NsArgs a, hipStream_t st) {
  tile::for_launches(plan, [&]<int SHAPE>(const tile::Tiles &t) {
    a.tiles = t;
    k_ns<MODE, SHAPE><<<dim3(uint32_t(tile::blocks_of(t))), dim3(tile::ShapeOf<SHAPE>::type::THREADS), 0, st>>>(a);
    if constexpr (MODE != APPLY)
      if (t.splits > 1)
        k_ns_join_symmetric<MODE, tile::ShapeOf<SHAPE>::type::BM><<<dim3(a.mp / 64, a.mp / 64), dim3(512), 0, st>>>(a);
  });
  return last_launch_status();
}

int run_ortho(const fqt_ortho_desc *d, const NsSizes &s, Source src, NsArgs a, void *ws, size_t ws_bytes,
              hipStream_t st) {
  const NsWs w = ns_ws(s);
  if (ws_bytes < w.total) return FQT_E_WORKSPACE;
  char *base = static_cast<char *>(ws);
  auto pairs = [&](size_t at) { return Pairs{reinterpret_cast<uint16_t *>(base + at), s.mp}; };
  double *norm = reinterpret_cast<double *>(base + w.norm);
  Pairs x = pairs(w.x[0]), next = pairs(w.x[1]);
  const uint32_t groups = uint32_t((d->cols + 7) / 8), all = uint32_t(d->rows * groups);
  const int parts = int(std::min<uint32_t>((all + 255) / 256, NORM_BLOCKS));
  k_ns_norm<<<dim3(parts), dim3(256), 0, st>>>(src, make_fastdiv(groups), all, norm);
  FQT_TRY_(last_launch_status());
  a.mp = s.mp; a.np = s.np; a.m = s.m; a.n = s.n;
  a.p = pairs(w.p);
  a.q = pairs(w.q);
  a.part = reinterpret_cast<float *>(base + w.part);
  const Start start{norm, parts, d->steps, d->eps, reinterpret_cast<Units *>(norm + NORM_BLOCKS)};
  a.ldo = s.ldo;
  a.o_dtype = d->o_dtype;
  a.tall = s.tall;
  if (s.mp == 64) {
    const int64_t tiles = s.np / 64, per = (tiles + SMALL_BLOCKS - 1) / SMALL_BLOCKS;
    const int blocks = int((tiles + per - 1) / per);
    float *sums[2] = {a.part, a.part + SMALL_BLOCKS * 4096}, *joined = a.part + 2 * SMALL_BLOCKS * 4096;
    SmallArgs q{a, nullptr, sums[0], per * 64};
    q.n.x = x;
    if (s.tall) k_ns_small_start<true><<<dim3(blocks), dim3(256), 0, st>>>(src, start, q);
    else k_ns_small_start<false><<<dim3(blocks), dim3(256), 0, st>>>(src, start, q);
    FQT_TRY_(last_launch_status());
    for (int i = 0; i < d->steps; ++i) {
      q.n.units = start.units + i;
      q.n.x = x;
      q.n.next = next;
      q.n.last = i + 1 == d->steps;
      q.from = sums[i & 1];
      q.to = sums[~i & 1];
      if (blocks > DIRECT) {
        k_ns_small_join<<<dim3(64), dim3(256), 0, st>>>(q.from, blocks, joined);
        FQT_TRY_(last_launch_status());
        q.from = joined;
      }
      k_ns_small<<<dim3(blocks), dim3(256), 0, st>>>(q, blocks > DIRECT ? 1 : blocks);
      FQT_TRY_(last_launch_status());
      std::swap(x, next);
    }
    return FQT_OK;
  }
  const dim3 grid(s.np / 64, s.mp / 64);
  if (s.tall) k_ns_start<true><<<grid, dim3(256), 0, st>>>(src, start, x);
  else k_ns_start<false><<<grid, dim3(256), 0, st>>>(src, start, x);
  FQT_TRY_(last_launch_status());
  for (int i = 0; i < d->steps; ++i) {
    a.units = start.units + i;
    a.x = x;
    a.next = next;
    a.last = i + 1 == d->steps;
    FQT_TRY_(launch_ns<GRAM>(w.gram, a, st));
    FQT_TRY_(launch_ns<POLY>(w.poly, a, st));
    FQT_TRY_(launch_ns<APPLY>(w.apply, a, st));
    std::swap(x, next);
  }
  return FQT_OK;
}

}  // namespace
}  // namespace dense
}  // namespace fqt

using namespace fqt;
using namespace fqt::dense;

extern "C" int fqt_ortho_workspace_size(const fqt_ortho_desc *d, size_t *bytes) {
  NsSizes s;
  FQT_TRY_(check_ortho(d, &s));
  if (!bytes) return FQT_E_NULL;
  *bytes = s.m ? ns_ws(s).total : 256;
  return FQT_OK;
}

extern "C" int fqt_ortho_plan(const fqt_ortho_desc *d, int32_t product, fqt_product_plan *plan) {
  NsSizes s;
  FQT_TRY_(check_ortho(d, &s));
  if (!plan) return FQT_E_NULL;
  if (product < FQT_PRODUCT_GRAM || product > FQT_PRODUCT_APPLY) return FQT_E_INVAL;
  tile::Plan p{};
  if (s.mp > 64) {
    const NsWs w = ns_ws(s);
    p = product == FQT_PRODUCT_GRAM ? w.gram : product == FQT_PRODUCT_POLY ? w.poly : w.apply;
  }
  tile::describe(p, plan);
  return FQT_OK;
}

extern "C" int fqt_orthogonalize(const fqt_ortho_desc *d, const void *g, void *o, void *ws,
                                 size_t ws_bytes, void *hip_stream) {
  NsSizes s;
  FQT_TRY_(check_ortho(d, &s));
  if (s.m == 0) return FQT_OK;
  if (!g || !o || !ws) return FQT_E_NULL;
  if (!elem_aligned(g, d->g_dtype) || !elem_aligned(o, d->o_dtype) || !aligned(ws, 256)) return FQT_E_ALIGN;
  Source src{g, nullptr, d->rows, d->cols, s.ldg, 0, d->g_dtype, 0, 0.0f};
  NsArgs a{};
  a.out = o;
  return run_ortho(d, s, src, a, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
}

extern "C" int fqt_muon_step(const fqt_ortho_desc *d, const fqt_muon_cfg *cfg, const void *g, float *m,
                             float *w, void *ws, size_t ws_bytes, void *hip_stream) {
  NsSizes s;
  FQT_TRY_(check_ortho(d, &s));
  if (!cfg) return FQT_E_NULL;
  if (d->o_dtype != FQT_F32) return FQT_E_DTYPE;
  if (!std::isfinite(cfg->lr) || !std::isfinite(cfg->momentum) || !std::isfinite(cfg->weight_decay) ||
      !std::isfinite(cfg->scale))
    return FQT_E_INVAL;
  if (s.m == 0) return FQT_OK;
  if (!g || !m || !w || !ws) return FQT_E_NULL;
  if (!elem_aligned(g, d->g_dtype) || !aligned(m, 4) || !aligned(w, 4) || !aligned(ws, 256)) return FQT_E_ALIGN;
  Source src{g, m, d->rows, d->cols, s.ldg, s.ldm, d->g_dtype, cfg->nesterov ? 1 : 0, cfg->momentum};
  NsArgs a{};
  a.w = w;
  a.keep = 1.0f - cfg->lr * cfg->weight_decay;
  a.rate = cfg->lr * cfg->scale;
  return run_ortho(d, s, src, a, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
}
