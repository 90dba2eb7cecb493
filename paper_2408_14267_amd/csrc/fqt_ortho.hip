// Newton-Schulz orthogonalisation and the optimizer step on it.
//
// X is kept on the short side of the matrix (m x n, m <= n), padded with zeros to whole tiles, as
// two float16 planes hi + lo of X 2^15 (hi the nearest float16, lo the nearest to the rest): 22 bits
// and their rounding, as good as float32 where entries are not 2^-24 of the largest.  A product is
// the sum of hi hi, hi lo and lo hi on the 16-bit matrix cores with float32 sums; lo lo is below the
// rounding.  That is three passes of matrix instructions at many times the rate of float32 ones.
//
// The powers of two keep every entry inside float16: the singular values of X stay below 1.21 (the
// quintic maps [0, 1.21] into itself), so |X| < 2^15 1.21, |P| = |X X^T| < 1.47 (2^14) and
// |b P + c P^2| < 2.81 (2^13) are below 65504 with the factors in brackets.
//
// A step is three products: P = X X^T and Q = b P + c P P, both symmetric, of which only the tiles on
// and above the diagonal are computed and stored twice; X' = a X + Q X, which reads X along m (COLS).
// The last step's product stores the result, or updates the weights, instead of X'.
#include "fqt_tile.hpp"

namespace fqt {
namespace dense {
namespace {

#pragma clang fp contract(fast)

using tile::Operand;
using tile::ROWS;
using tile::COLS;

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float X_UNIT = 32768.0f;      // 2^15

struct Split { uint16_t hi, lo; };
__device__ __forceinline__ Split split(float v) {
  const _Float16 h = static_cast<_Float16>(v);
  const _Float16 l = static_cast<_Float16>(v - static_cast<float>(h));
  return {__builtin_bit_cast(uint16_t, h), __builtin_bit_cast(uint16_t, l)};
}
__device__ __forceinline__ float join(uint16_t hi, uint16_t lo) {
  return static_cast<float>(__builtin_bit_cast(_Float16, hi)) + static_cast<float>(__builtin_bit_cast(_Float16, lo));
}
struct Planes { uint16_t *hi, *lo; };
__device__ __forceinline__ void store_split8(const Planes &p, int64_t at, const float (&v)[8]) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const Split a = split(v[2 * i]), b = split(v[2 * i + 1]);
    h[i] = a.hi | uint32_t(b.hi) << 16;
    l[i] = a.lo | uint32_t(b.lo) << 16;
  }
  *reinterpret_cast<uint4 *>(p.hi + at) = make_uint4(h[0], h[1], h[2], h[3]);
  *reinterpret_cast<uint4 *>(p.lo + at) = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ void load_split8(const Planes &p, int64_t at, float (&v)[8]) {
  const uint4 h = *reinterpret_cast<const uint4 *>(p.hi + at), l = *reinterpret_cast<const uint4 *>(p.lo + at);
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
__device__ __forceinline__ float load_g(const Source &s, int64_t r, int64_t c) {
  const int64_t at = r * s.ldg + c;
  return s.g_dtype == FQT_BF16 ? to_f32(static_cast<const bf16 *>(s.g)[at]) : static_cast<const float *>(s.g)[at];
}
constexpr int NORM_BLOCKS = 512;

// Updates the momentum and adds up u^2 in float64, a partial sum per workgroup.
__global__ void __launch_bounds__(256) k_ns_norm(Source s, double *part) {
  __shared__ double sums[4];
  double sum = 0.0;
  const int64_t all = s.rows * s.cols;
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
    const int64_t r = i / s.cols, c = i % s.cols;
    float u = load_g(s, r, c);
    if (s.m) {
      float *m = s.m + r * s.ldm + c;
      const float v = fmaf(s.momentum, *m, u);
      *m = v;
      u = s.nesterov ? fmaf(s.momentum, v, u) : v;
    }
    sum += double(u) * double(u);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// X_0 = u / (|u| + eps) as planes [mp][np], zeros in the padding.  A workgroup takes a 64 x 64 tile of
// X; tall matrices are transposed on the way.
template <bool TALL>
__global__ void __launch_bounds__(256) k_ns_start(Source s, const double *part, int32_t parts, float eps,
                                                  Planes x, int64_t np) {
  __shared__ double sums[4];
  __shared__ float t[64][65];
  double sum = 0.0;
  for (int i = threadIdx.x; i < parts; i += 256) sum += part[i];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x / 64] = sum;
  __syncthreads();
  const double norm = sqrt(sums[0] + sums[1] + sums[2] + sums[3]);
  const float inv = float(double(X_UNIT) / (norm + double(eps)));
  const int64_t x0 = int64_t(blockIdx.y) * 64, y0 = int64_t(blockIdx.x) * 64;   // row and column of X
  for (int i = threadIdx.x; i < 64 * 64; i += 256) {
    const int a = i / 64, b = i % 64;                                          // b runs along u's columns
    const int64_t r = (TALL ? y0 : x0) + a, c = (TALL ? x0 : y0) + b;
    float u = 0.0f;
    if (r < s.rows && c < s.cols) {
      if (!s.m) {
        u = load_g(s, r, c);
      } else {
        const float v = s.m[r * s.ldm + c];
        u = s.nesterov ? fmaf(s.momentum, v, load_g(s, r, c)) : v;
      }
    }
    if constexpr (TALL) t[b][a] = u * inv;
    else t[a][b] = u * inv;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * 8; i += 256) {
    const int a = i / 8, b = i % 8 * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = t[a][b + j];
    store_split8(x, (x0 + a) * np + y0 + b, v);
  }
}

// ----------------------------------------------------------------------------- products

enum Mode { GRAM, POLY, APPLY };
struct NsArgs {
  Planes x, p, q, next;  // X [mp][np]; P, Q [mp][mp]; the next X
  int64_t mp, np;
  int64_t m, n;          // without padding
  uint32_t nm, nn, tiles, splits;
  int64_t steps;
  float *part;
  // the last step's result
  void *out;             // o, or null
  float *w;              // weights, or null
  int64_t ldo;
  int32_t last, o_dtype, tall;
  float keep, rate;      // w = keep w - rate X
};

template <int MODE>
__device__ __forceinline__ void ns_finish8(const NsArgs &a, int64_t m, int64_t n, bool mirror, float (&v)[8]) {
  if constexpr (MODE == APPLY) {
    if (m >= a.mp || n >= a.np) return;
    float x[8];
    load_split8(a.x, m * a.np + n, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf(NS_A, x[i], v[i] * 0x1p-13f);      // X' 2^15
    if (!a.last) {
      store_split8(a.next, m * a.np + n, v);
      return;
    }
    if (m >= a.m) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (n + i >= a.n) break;
      const int64_t at = a.tall ? (n + i) * a.ldo + m : m * a.ldo + n + i;
      const float o = v[i] * (1.0f / X_UNIT);
      if (a.w) a.w[at] = fmaf(a.keep, a.w[at], -a.rate * o);
      else if (a.o_dtype == FQT_BF16) static_cast<bf16 *>(a.out)[at] = from_f32<bf16>(o);
      else static_cast<float *>(a.out)[at] = o;
    }
  } else {
    if (m >= a.mp || n >= a.mp) return;
    const Planes &to = MODE == GRAM ? a.p : a.q;
    if constexpr (MODE == GRAM) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= 0x1p-16f;                            // P 2^14 of sums 2^30
    } else {
      float p[8];
      load_split8(a.p, m * a.mp + n, p);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = fmaf(NS_B * 0.5f, p[i], v[i] * (NS_C * 0x1p-15f));   // Q 2^13
    }
    store_split8(to, m * a.mp + n, v);
    if (mirror) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const Split s = split(v[i]);
        to.hi[(n + i) * a.mp + m] = s.hi;
        to.lo[(n + i) * a.mp + m] = s.lo;
      }
    }
  }
}

// Tile t of the tiles on and above the diagonal of k x k, by columns.
__device__ __forceinline__ tile::TileAt upper_tile(uint32_t t) {
  uint32_t c = uint32_t((sqrtf(8.0f * float(t) + 1.0f) - 1.0f) * 0.5f);
  while (c * (c + 1) / 2 > t) --c;
  while ((c + 1) * (c + 2) / 2 <= t) ++c;
  return {t - c * (c + 1) / 2, c};
}

template <int MODE, typename S>
__global__ void __launch_bounds__(S::THREADS) k_ns(NsArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];
  const uint32_t sp = blockIdx.x / a.tiles, b = blockIdx.x % a.tiles;
  const tile::TileAt at = MODE == APPLY ? tile::tile_at(b, a.nm, a.nn) : upper_tile(b);
  const int64_t m0 = int64_t(at.m) * S::BM, n0 = int64_t(at.n) * S::BN;
  const int64_t K = MODE == GRAM ? a.np : a.mp;
  const int64_t t0 = sp * a.steps, t1 = min(3 * (K / 64), t0 + a.steps);
  auto op = [&](const uint16_t *p, int64_t ld, int64_t rows) {
    return Operand{reinterpret_cast<const char *>(p), ld * 2, rows};
  };
  typename tile::Acc<tile::F16K>::type acc[S::FM][S::FN];
  if constexpr (MODE == GRAM) {
    const Operand h = op(a.x.hi, a.np, a.mp), l = op(a.x.lo, a.np, a.mp);
    const Operand x[3] = {h, h, l}, w[3] = {h, l, h};
    tile::run_tile<tile::F16K, ROWS, ROWS, S>(x, w, K, m0, n0, t0, t1, lds, acc);
  } else if constexpr (MODE == POLY) {
    const Operand h = op(a.p.hi, a.mp, a.mp), l = op(a.p.lo, a.mp, a.mp);
    const Operand x[3] = {h, h, l}, w[3] = {h, l, h};
    tile::run_tile<tile::F16K, ROWS, ROWS, S>(x, w, K, m0, n0, t0, t1, lds, acc);
  } else {
    const Operand qh = op(a.q.hi, a.mp, a.mp), ql = op(a.q.lo, a.mp, a.mp);
    const Operand xh = op(a.x.hi, a.np, a.np), xl = op(a.x.lo, a.np, a.np);
    const Operand x[3] = {qh, qh, ql}, w[3] = {xh, xl, xh};
    tile::run_tile<tile::F16K, ROWS, COLS, S>(x, w, K, m0, n0, t0, t1, lds, acc);
  }
  if (a.splits > 1) {
    const int64_t N = MODE == APPLY ? a.np : a.mp;
    float *part = a.part + sp * a.mp * N;
    tile::for_rows8<tile::F16K, S>(acc, lds, m0, n0, [&](int64_t m, int64_t n, float (&v)[8]) {
      if (m < a.mp && n < N) store8f(part + m * N + n, true, 8, v);
    });
  } else {
    tile::for_rows8<tile::F16K, S>(acc, lds, m0, n0, [&](int64_t m, int64_t n, float (&v)[8]) {
      ns_finish8<MODE>(a, m, n, at.m != at.n, v);
    });
  }
}

template <int MODE, typename S>
__global__ void __launch_bounds__(256) k_ns_join(NsArgs a) {
  const int64_t N = MODE == APPLY ? a.np : a.mp, groups = N / 8, all = a.mp * groups;
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
    const int64_t m = i / groups, n = i % groups * 8;
    if (MODE != APPLY && m / S::BM > n / S::BN) continue;                      // stored with its mirror image
    float v[8] = {}, t[8];
    for (uint32_t s = 0; s < a.splits; ++s) {
      load8f(a.part + (s * a.mp + m) * N + n, true, 8, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += t[j];
    }
    ns_finish8<MODE>(a, m, n, m / S::BM != n / S::BN, v);
  }
}

// ----------------------------------------------------------------------------- host side

using Large = tile::Shape<256, 256, 2, 4>;
using Middle = tile::Shape<128, 128, 2, 2>;
using Small = tile::Shape<64, 64, 2, 2>;

struct NsPlan { int shape; uint32_t nm, nn, tiles, splits; int64_t steps; };
NsPlan ns_plan(int64_t M, int64_t N, int64_t K, bool symmetric) {
  auto tiles = [&](int64_t b) {
    const int64_t r = (M + b - 1) / b, c = (N + b - 1) / b;
    return symmetric ? r * (r + 1) / 2 : r * c;
  };
  NsPlan p{};
  const int64_t b = tiles(256) >= 200 ? 256 : tiles(128) >= 200 ? 128 : 64;
  p.shape = b == 256 ? 0 : b == 128 ? 1 : 2;
  p.nm = uint32_t((M + b - 1) / b);
  p.nn = uint32_t((N + b - 1) / b);
  p.tiles = uint32_t(tiles(b));
  const int64_t total = 3 * (K / 64);
  int64_t splits = 1;
  if (b == 64) splits = std::max<int64_t>(1, std::min<int64_t>(1024 / p.tiles, total / 8));
  p.steps = (total + splits - 1) / splits;
  p.splits = uint32_t((total + p.steps - 1) / p.steps);
  return p;
}

struct NsSizes { int64_t m, n, mp, np, ldg, ldo, ldm; bool tall; };
struct NsWs { size_t norm, x[2], p, q, part, total; NsPlan gram, poly, apply; };

int check_ortho(const fqt_ortho_desc *d, NsSizes *s) {
  if (!d) return FQT_E_NULL;
  if (!float_type(d->g_dtype) || !float_type(d->o_dtype)) return FQT_E_DTYPE;
  if (d->rows < 0 || d->cols < 0 || d->rows > FQT_MAX_LD || d->cols > FQT_MAX_LD) return FQT_E_SHAPE;
  if (d->steps < 1 || d->steps > 32 || !(d->eps > 0.0f) || !std::isfinite(d->eps)) return FQT_E_INVAL;
  s->tall = d->rows > d->cols;
  s->m = std::min(d->rows, d->cols);
  s->n = std::max(d->rows, d->cols);
  s->mp = (s->m + 63) / 64 * 64;
  s->np = (s->n + 63) / 64 * 64;
  s->ldg = row_stride(d->ldg, d->cols);
  s->ldo = row_stride(d->ldo, d->cols);
  s->ldm = row_stride(d->ldm, d->cols);
  if (!s->ldg || !s->ldo || !s->ldm) return FQT_E_SHAPE;
  return FQT_OK;
}
NsWs ns_ws(const NsSizes &s) {
  NsWs w{};
  w.gram = ns_plan(s.mp, s.mp, s.np, true);
  w.poly = ns_plan(s.mp, s.mp, s.mp, true);
  w.apply = ns_plan(s.mp, s.np, s.mp, false);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
  w.norm = take(NORM_BLOCKS * sizeof(double));
  const size_t x = size_t(s.mp) * s.np * 4, p = size_t(s.mp) * s.mp * 4;       // two planes of 2 bytes
  w.x[0] = take(x);
  w.x[1] = take(x);
  w.p = take(p);
  w.q = take(p);
  auto part = [&](const NsPlan &pl, size_t entries) { return pl.splits > 1 ? size_t(pl.splits) * entries * 4 : 0; };
  w.part = take(std::max({part(w.gram, s.mp * s.mp), part(w.poly, s.mp * s.mp), part(w.apply, s.mp * s.np)}));
  w.total = at;
  return w;
}

template <int MODE>
int launch_ns(const NsPlan &pl, NsArgs a, hipStream_t st) {
  a.nm = pl.nm; a.nn = pl.nn; a.tiles = pl.tiles; a.splits = pl.splits; a.steps = pl.steps;
  auto go = [&]<typename S>(S) {
    k_ns<MODE, S><<<dim3(pl.tiles * pl.splits), dim3(S::THREADS), 0, st>>>(a);
    if (pl.splits > 1) {
      const int64_t all = a.mp * (MODE == APPLY ? a.np : a.mp) / 8;
      k_ns_join<MODE, S><<<dim3(std::min<int64_t>((all + 255) / 256, 4096)), dim3(256), 0, st>>>(a);
    }
  };
  if (pl.shape == 0) go(Large{});
  else if (pl.shape == 1) go(Middle{});
  else go(Small{});
  return last_launch_status();
}

int run_ortho(const fqt_ortho_desc *d, const NsSizes &s, Source src, NsArgs a, void *ws, size_t ws_bytes,
              hipStream_t st) {
  const NsWs w = ns_ws(s);
  if (ws_bytes < w.total) return FQT_E_WORKSPACE;
  char *base = static_cast<char *>(ws);
  auto planes = [&](size_t at, size_t entries) {
    uint16_t *p = reinterpret_cast<uint16_t *>(base + at);
    return Planes{p, p + entries};
  };
  double *norm = reinterpret_cast<double *>(base + w.norm);
  const size_t xe = size_t(s.mp) * s.np, pe = size_t(s.mp) * s.mp;
  Planes x = planes(w.x[0], xe), next = planes(w.x[1], xe);
  const int64_t all = d->rows * d->cols;
  const int parts = int(std::min<int64_t>((all + 1023) / 1024, NORM_BLOCKS));
  k_ns_norm<<<dim3(parts), dim3(256), 0, st>>>(src, norm);
  FQT_TRY_(last_launch_status());
  const dim3 grid(s.np / 64, s.mp / 64);
  if (s.tall) k_ns_start<true><<<grid, dim3(256), 0, st>>>(src, norm, parts, d->eps, x, s.np);
  else k_ns_start<false><<<grid, dim3(256), 0, st>>>(src, norm, parts, d->eps, x, s.np);
  FQT_TRY_(last_launch_status());
  a.mp = s.mp; a.np = s.np; a.m = s.m; a.n = s.n;
  a.p = planes(w.p, pe);
  a.q = planes(w.q, pe);
  a.part = reinterpret_cast<float *>(base + w.part);
  a.ldo = s.ldo;
  a.o_dtype = d->o_dtype;
  a.tall = s.tall;
  for (int i = 0; i < d->steps; ++i) {
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
