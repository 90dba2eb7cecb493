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

// X_0 = u / (|u| + eps) as pairs, zeros in the padding.  A workgroup takes a 64 x 64 tile of
// X; tall matrices are transposed on the way.
template <bool TALL>
__global__ void __launch_bounds__(256) k_ns_start(Source s, const double *part, int32_t parts, float eps,
                                                  Pairs x) {
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
    store_split8(x, x0 + a, y0 + b, v);
  }
}

// ----------------------------------------------------------------------------- products

enum Mode { GRAM, POLY, APPLY };
struct NsArgs {
  Pairs x, p, q, next;   // X [mp][np]; P, Q [mp][mp]; the next X
  int64_t mp, np;
  int64_t m, n;          // without padding
  tile::Tiles tiles;
  float *part;
  // the last step's result
  void *out;             // o, or null
  float *w;              // weights, or null
  int64_t ldo;
  int32_t last, o_dtype, tall;
  float keep, rate;      // w = keep w - rate X
};

// The epilogue of 8 consecutive n (tile::run_epilogue).  mirror: the group is stored transposed too.
template <int MODE>
struct Finish {
  static constexpr int DEPTH = MODE == GRAM ? 1 : 4;
  struct Fetch { float x[MODE == GRAM ? 1 : 8]; };         // X, or P
  const NsArgs &a;
  bool mirror;
  __device__ __forceinline__ bool in(int64_t m, int64_t n) const {
    return m < a.mp && n < (MODE == APPLY ? a.np : a.mp);
  }
  __device__ __forceinline__ void columns(int64_t) {}
  __device__ __forceinline__ Fetch fetch(int64_t m, int64_t n) {
    Fetch f;
    if constexpr (MODE != GRAM)
      if (in(m, n)) load_split8(MODE == APPLY ? a.x : a.p, m, n, f.x);
    return f;
  }
  __device__ __forceinline__ void finish(int64_t m, int64_t n, float (&v)[8], const Fetch &f) {
    if (!in(m, n)) return;
    if constexpr (MODE == APPLY) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = fmaf(NS_A, f.x[i], v[i] * 0x1p-13f);  // X' 2^15
      if (!a.last) {
        store_split8(a.next, m, n, v);
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
      const Pairs &to = MODE == GRAM ? a.p : a.q;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (MODE == GRAM) v[i] *= 0x1p-16f;                          // P 2^14 of sums 2^30
        else v[i] = fmaf(NS_B * 0.5f, f.x[i], v[i] * (NS_C * 0x1p-15f));       // Q 2^13
      }
      store_split8(to, m, n, v);
      if (mirror) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const Split s = split(v[i]);
          uint16_t *q = to.at(n + i, m);
          q[0] = s.hi;
          q[32] = s.lo;
        }
      }
    }
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
  if (a.tiles.splits > 1) {
    const int64_t N = MODE == APPLY ? a.np : a.mp;
    tile::run_epilogue<tile::SPLITK, S>(acc, lds, at.m0, at.n0, tile::StorePart{a.part + at.split * a.mp * N, a.mp, N});
  } else {
    tile::run_epilogue<tile::SPLITK, S>(acc, lds, at.m0, at.n0, Finish<MODE>{a, !at.diagonal});
  }
}

// The partial sums of a split contraction, added in order.  B: edge of the tiles, of which a symmetric
// product has those on and above the diagonal.
template <int MODE, int B>
__global__ void __launch_bounds__(256) k_ns_join(NsArgs a) {
  const int64_t N = MODE == APPLY ? a.np : a.mp, groups = N / 8, all = a.mp * groups;
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
    const int64_t m = i / groups, n = i % groups * 8;
    if (MODE != APPLY && m / B > n / B) continue;
    Finish<MODE> f{a, m / B != n / B};
    const auto q = f.fetch(m, n);
    float v[8] = {};
#pragma unroll 4
    for (uint32_t s = 0; s < a.tiles.splits; ++s) {
      float t[8];
      load8f(a.part + (s * a.mp + m) * N + n, true, 8, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += t[j];
    }
    f.finish(m, n, v, q);
  }
}

// ----------------------------------------------------------------------------- host side

struct NsSizes { int64_t m, n, mp, np, ldg, ldo, ldm; bool tall; };
struct NsWs { size_t norm, x[2], p, q, part, total; tile::Plan gram, poly, apply; };

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
  if (!s->ldg || !s->ldo || !s->ldm || s->m > 65536) return FQT_E_SHAPE;
  return FQT_OK;
}
NsWs ns_ws(const NsSizes &s) {
  NsWs w{};
  w.gram = tile::make_plan(s.mp, s.mp, s.np / 32, true);
  w.poly = tile::make_plan(s.mp, s.mp, s.mp / 32, true);
  w.apply = tile::make_plan(s.mp, s.np, s.mp / 32, false);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += align256(bytes); return o; };
  w.norm = take(NORM_BLOCKS * sizeof(double));
  const size_t x = size_t(s.mp) * s.np * 4, p = size_t(s.mp) * s.mp * 4;       // two planes of 2 bytes
  w.x[0] = take(x);
  w.x[1] = take(x);
  w.p = take(p);
  w.q = take(p);
  auto part = [&](const tile::Plan &pl, size_t entries) { return pl.splits > 1 ? size_t(pl.splits) * entries * 4 : 0; };
  w.part = take(std::max({part(w.gram, s.mp * s.mp), part(w.poly, s.mp * s.mp), part(w.apply, s.mp * s.np)}));
  w.total = at;
  return w;
}

template <int MODE>
int launch_ns(const tile::Plan &plan, NsArgs a, hipStream_t st) {
  tile::for_launches(plan, [&]<int SHAPE>(const tile::Tiles &t) {
    a.tiles = t;
    k_ns<MODE, SHAPE><<<dim3(tile::blocks_of(SHAPE, t)), dim3(tile::ShapeOf<SHAPE>::type::THREADS), 0, st>>>(a);
    if (t.splits > 1) {
      const int64_t all = a.mp * (MODE == APPLY ? a.np : a.mp) / 8;
      k_ns_join<MODE, tile::ShapeOf<SHAPE>::type::BM>
          <<<dim3(std::min<int64_t>((all + 255) / 256, 4096)), dim3(256), 0, st>>>(a);
    }
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
  const int64_t all = d->rows * d->cols;
  const int parts = int(std::min<int64_t>((all + 1023) / 1024, NORM_BLOCKS));
  k_ns_norm<<<dim3(parts), dim3(256), 0, st>>>(src, norm);
  FQT_TRY_(last_launch_status());
  const dim3 grid(s.np / 64, s.mp / 64);
  if (s.tall) k_ns_start<true><<<grid, dim3(256), 0, st>>>(src, norm, parts, d->eps, x);
  else k_ns_start<false><<<grid, dim3(256), 0, st>>>(src, norm, parts, d->eps, x);
  FQT_TRY_(last_launch_status());
  a.mp = s.mp; a.np = s.np; a.m = s.m; a.n = s.n;
  a.p = pairs(w.p);
  a.q = pairs(w.q);
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
