// Matrix product with bias, activation and residual in its epilogue, and its backward pass.
//
// The forward is one launch of matrix tiles (fqt_tile.hpp) whose epilogue scales, adds the bias,
// applies the activation and adds the residual to the float32 sums: no intermediate touches memory
// but the pre-activation, if asked for.  Contractions that are long for the number of output tiles
// are split over workgroups; their partial sums (float32, int32 of int8 operands) meet, in a fixed order, in a second launch
// with the same epilogue.
//
// The backward is one pass over dy (and z) that writes dz = dy act'(z) in bf16 and sums dbias, then
// the two products, which read dz and the operands as they are stored: dx = dz w reads w along n
// (COLS), dw = dz^T x reads both operands along m.
#include "fqt_tile.hpp"

namespace fqt {
namespace dense {
namespace {

#pragma clang fp contract(fast)

using tile::Operand;
using tile::ROWS;
using tile::COLS;

// ----------------------------------------------------------------------------- activations

// exp(-v).  WIDE: the rounding of the exponent, up to |v| 2^-24 of the result, is taken back (v is held
// where the result is neither 0 nor infinite already); for float32 outputs, since bf16's do not show it.
template <bool WIDE>
__device__ __forceinline__ float exp_neg(float v) {
  constexpr float LOG2E = 1.44269504088896341f, LOG2E_LOW = 1.92596299e-8f, LN2 = 0.69314718055994531f;
  if constexpr (WIDE) v = fminf(fmaxf(v, -150.0f), 150.0f);
  const float b = v * -LOG2E, e = __builtin_amdgcn_exp2f(b);
  if constexpr (!WIDE) return e;
  else return e * fmaf(fmaf(v, -LOG2E_LOW, fmaf(v, -LOG2E, -b)), LN2, 1.0f);
}
// Phi(-a) and exp(-a^2 / 2) for a >= 0, Phi the normal distribution function: exp(a^2 / 2) Phi(-a) (a + 3) is
// smooth in s = (a - 3) / (a + 3), and a sextic in it, fitted to the least largest error of a Phi(-a), is
// within 9e-9 of that; float32 roundings bring Phi to 2.5e-7 and a Phi(-a) to 9e-8.  The coefficients fall off, so
// nothing cancels.  About 23 issue slots; the library's erf costs four times that, and a 256 x 256 tile
// pays 0.4 us for each slot.
__device__ __forceinline__ float normal_tail(float a, float *e) {
  const float t = __builtin_amdgcn_rcpf(a + 3.0f), s = fmaf(t, -6.0f, 1.0f);
  float q = fmaf(s, 0.00200464337f, 0.00693698652f);
  q = fmaf(s, q, -0.0110280172f);
  q = fmaf(s, q, -0.0475851104f);
  q = fmaf(s, q, 0.229960269f);
  q = fmaf(s, q, -0.509330356f);
  q = fmaf(s, q, 0.729084549f);
  *e = __builtin_amdgcn_exp2f(a * (a * -0.72134752044448170f));
  return q * t * *e;
}
// (Phi(-30) is 0 in float32: a need not be larger, and an infinite one would meet it.)
__device__ __forceinline__ float tail_arg(float z) { return fminf(fabsf(z), 30.0f); }
template <int ACT, bool WIDE>
__device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == FQT_ACT_RELU) return z > 0.0f ? z : (z != z ? z : 0.0f);
  else if constexpr (ACT == FQT_ACT_GELU) {
    // z Phi(z) = max(z, 0) - |z| Phi(-|z|)
    const float a = tail_arg(z);
    float e;
    const float q = normal_tail(a, &e);
    return z != z ? z : fmaf(-a, q, fmaxf(z, 0.0f));
  } else if constexpr (ACT == FQT_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + exp_neg<WIDE>(z));
  else if constexpr (ACT == FQT_ACT_HARDTANH) return z != z ? z : fminf(fmaxf(z, -1.0f), 1.0f);
  else return z;
}
template <int ACT>
__device__ __forceinline__ float slope(float z) {
  if constexpr (ACT == FQT_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
  else if constexpr (ACT == FQT_ACT_GELU) {
    const float a = tail_arg(z);
    float e;
    const float q = normal_tail(a, &e), d = z > 0.0f ? 1.0f - q : q;
    return z != z ? z : fmaf(copysignf(a, z) * 0.39894228040143268f, e, d);
  } else if constexpr (ACT == FQT_ACT_SILU) {
    const float t = __builtin_amdgcn_rcpf(1.0f + exp_neg<false>(z));
    return t * fmaf(z, 1.0f - t, 1.0f);
  } else if constexpr (ACT == FQT_ACT_HARDTANH) return z > -1.0f && z < 1.0f ? 1.0f : 0.0f;
  else return 1.0f;
}
// Calls f.template operator()<ACT>() for the runtime code (uniform over the launch).
template <typename F>
__device__ __forceinline__ void with_act(int act, F &&f) {
  switch (act) {
    case FQT_ACT_RELU: f.template operator()<FQT_ACT_RELU>(); break;
    case FQT_ACT_GELU: f.template operator()<FQT_ACT_GELU>(); break;
    case FQT_ACT_SILU: f.template operator()<FQT_ACT_SILU>(); break;
    case FQT_ACT_HARDTANH: f.template operator()<FQT_ACT_HARDTANH>(); break;
    default: f.template operator()<FQT_ACT_NONE>();
  }
}

// ----------------------------------------------------------------------------- epilogue

struct Epilogue {
  const float *sx, *sw, *bias;
  const void *res;
  void *z, *y;
  int64_t M, N, ldr, ldz, ldy;
  int32_t y_dtype, act;
};

// Loads or stores of 8 elements whose type is known at run time (uniform).
__device__ __forceinline__ void load8(const void *p, int64_t at, int dt, int n, float (&o)[8]) {
  if (dt == FQT_BF16) load8f(static_cast<const bf16 *>(p) + at, n, o);
  else load8f(static_cast<const float *>(p) + at, n, o);
}
__device__ __forceinline__ void store8(void *p, int64_t at, int dt, int n, const float (&v)[8]) {
  if (dt == FQT_BF16) store8f(static_cast<bf16 *>(p) + at, n, v);
  else store8f(static_cast<float *>(p) + at, n, v);
}

// The epilogue of 8 consecutive n (tile::run_epilogue).
template <int ACT>
struct Finish {
  static constexpr int DEPTH = 4;
  static constexpr bool MIRROR = false, SUMS = false;
  struct Fetch {
    uint32_t res[8];       // the residual: 8 float32, or 8 bf16 in the first four
    float sx;
  };
  const Epilogue &e;
  float sw[8], bias[8];
  int cnt;                 // columns of the group that exist
  __device__ __forceinline__ Finish(const Epilogue &e_) : e(e_) {}
  __device__ __forceinline__ void columns(int64_t n) {
    cnt = int(max(int64_t(0), min(e.N - n, int64_t(8))));
    if (e.sw) load8f(e.sw + n, cnt, sw);
    if (e.bias) load8f(e.bias + n, cnt, bias);
  }
  __device__ __forceinline__ void column(int64_t n) {      // a single one
    cnt = 1;
    if (e.sw) sw[0] = e.sw[n];
    if (e.bias) bias[0] = e.bias[n];
  }
  __device__ __forceinline__ Fetch fetch(int64_t m, int64_t n) {
    Fetch f;
    if (m >= e.M || cnt == 0) return f;
    if (e.sx) f.sx = e.sx[m];
    if (e.res) {
      const int64_t at = m * e.ldr + n;
      if (e.y_dtype == FQT_BF16) {
        const bf16 *p = static_cast<const bf16 *>(e.res) + at;
        if (cnt == 8) {
          const u32x4 u = load_bytes16(p);
#pragma unroll
          for (int i = 0; i < 4; ++i) f.res[i] = u[i];
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t v = i < cnt ? p[i].v : 0;
            f.res[i / 2] = i & 1 ? f.res[i / 2] | v << 16 : v;
          }
        }
      } else {
        const float *p = static_cast<const float *>(e.res) + at;
        float t[8];
        load8f(p, cnt, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) f.res[i] = __float_as_uint(t[i]);
      }
    }
    return f;
  }
  __device__ __forceinline__ void finish(int64_t m, int64_t n, float (&v)[8], const Fetch &f) {
    if (m >= e.M || cnt == 0) return;
    if (e.sx) {            // (the sum times one and then the other: the scales' product may leave float32)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = v[i] * f.sx * sw[i];
    }
    if (e.bias) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += bias[i];
    }
    if (e.z) store8(e.z, m * e.ldz + n, e.y_dtype, cnt, v);
    const bool half = e.y_dtype == FQT_BF16;
    if (ACT != FQT_ACT_SILU || half) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = activate<ACT, false>(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = activate<ACT, true>(v[i]);
    }
    if (e.res) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t two = f.res[i / 2];
        v[i] += __uint_as_float(half ? (i & 1 ? two & 0xFFFF0000u : two << 16) : f.res[i]);
      }
    }
    store8(e.y, m * e.ldy + n, e.y_dtype, cnt, v);
  }
};

// ----------------------------------------------------------------------------- products

struct Product {
  Operand x, w;
  int64_t M, N, K;
  tile::Tiles tiles;
  float *part;           // [splits][M][ldp] partial sums (splits > 1), int32 words for int8 operands
  int64_t ldp;
};

template <int KIND, int LX, int LW, int SHAPE>
__global__ void __launch_bounds__(tile::ShapeOf<SHAPE>::type::THREADS, 2) k_product(Product p, Epilogue e) {
  typedef typename tile::ShapeOf<SHAPE>::type S;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];
  const tile::Place at = tile::place<SHAPE>(p.tiles, blockIdx.x);
  if (at.m0 >= p.M || at.n0 >= p.N) return;              // (parts of an edge tile)
  typename tile::Acc<KIND>::type acc[S::FM][S::FN];
  tile::contract<KIND, LX, LW, SHAPE, S>(p.x, p.w, p.K, at, p.tiles, lds, acc);
  if (p.tiles.splits > 1)
    tile::run_epilogue<KIND, S>(acc, lds, at.m0, at.n0, tile::StorePart{p.part + at.split * p.M * p.ldp, p.M, p.ldp});
  else
    with_act(e.act, [&]<int ACT>() { tile::run_epilogue<KIND, S>(acc, lds, at.m0, at.n0, Finish<ACT>(e)); });
}

// The partial sums of a split contraction, added in order, through the epilogue.  part: rows of ldp
// (a multiple of 8) words.
template <bool INTS>
__global__ void __launch_bounds__(256) k_product_finish(Product p, Epilogue e) {
  const int64_t groups = p.ldp / 8, all = p.M * groups;
  with_act(e.act, [&]<int ACT>() {
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
      const int64_t m = i / groups, n = i % groups * 8;
      Finish<ACT> f(e);
      f.columns(n);
      const auto q = f.fetch(m, n);
      std::conditional_t<INTS, int, float> sum[8] = {};
#pragma unroll 4
      for (uint32_t s = 0; s < p.tiles.splits; ++s) {
        float t[8];
        load8f(p.part + (s * p.M + m) * p.ldp + n, 8, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if constexpr (INTS) sum[j] += __float_as_int(t[j]);
          else sum[j] += t[j];
        }
      }
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = float(sum[j]);
      f.finish(m, n, v, q);
    }
  });
}

// ----------------------------------------------------------------------------- few rows
// Up to FEW_MOST rows of x the bound is one pass over w, and a matrix tile would compute 60 empty rows,
// want its contraction split to fill the chip, a second launch to join the parts and, for rows that
// are not whole 16-byte pieces, a copy of w.  Here a workgroup takes R rows of w, its threads a 16-byte piece
// each, on the vector units; the sums meet by shuffles and in LDS.  Four rows are where the vector units
// are as busy as the memory.  1 x 25088 -> 4096 e4m3 with the tiles and here 23.6 and 19.8 us (5.2 TB/s), bf16
// 41.0 and 37.2, four rows 23.8 and 22.9, 40.5 and 41.3; 1 x 4099 -> 2048 bf16 24.0 and 6.0 (the call).

// The elements of a 16-byte piece, and the sum of their products: bf16 as float32, int8 by fours, e4m3 by
// twos as float16, which holds them and their smallest exactly.
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
template <typename T> struct Piece;
template <>
struct Piece<bf16> {
  typedef float Sum;
  static constexpr int N = 8;
  float v[N];
  __device__ __forceinline__ explicit Piece(u32x4 u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ void add(const Piece &o, float &sum) const {
#pragma unroll
    for (int i = 0; i < N; ++i) sum = fmaf(v[i], o.v[i], sum);
  }
};
template <>
struct Piece<e4m3> {
  typedef float Sum;
  static constexpr int N = 16;
  f16x2 v[N / 2];
  __device__ __forceinline__ explicit Piece(u32x4 u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u[i], 1.0f, false));
      v[2 * i + 1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u[i], 1.0f, true));
    }
  }
  __device__ __forceinline__ void add(const Piece &o, float &sum) const {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) sum = __builtin_amdgcn_fdot2(v[i], o.v[i], sum, false);
  }
};
template <>
struct Piece<int8_t> {
  typedef int Sum;
  static constexpr int N = 16;
  u32x4 u;
  __device__ __forceinline__ explicit Piece(u32x4 v) : u(v) {}
  __device__ __forceinline__ void add(const Piece &o, int &sum) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_sdot4(int(u[i]), int(o.u[i]), sum, false);
  }
};
// Sums of V values over a wave, each step halving the values a lane still adds up: lane l returns that of
// value l / (64 / V).
template <int V, typename S>
__device__ __forceinline__ S fold(S (&v)[V]) {
  int o = 32;
#pragma unroll
  for (int n = V / 2; n > 0; n /= 2, o /= 2) {
    const bool up = __lane_id() & o;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const S lower = v[i], upper = v[i + n];              // (selected as values: v stays in registers)
      v[i] = (up ? upper : lower) + __shfl_xor(up ? lower : upper, o);
    }
  }
#pragma unroll
  for (; o > 0; o /= 2) v[0] += __shfl_xor(v[0], o);
  return v[0];
}

struct FewArgs {
  const void *x, *w;
  int64_t K, ldx, ldw;
};
constexpr int FEW_MOST = 4, FEW_WIDE = 2560, FEW_THREADS = 256;
// M: rows of x, or more (those past the last read it again and store nothing).
template <typename T, int M, int R>
__global__ void __launch_bounds__(FEW_THREADS) k_few_rows(FewArgs a, Epilogue e) {
  typedef typename Piece<T>::Sum Sum;
  typedef std::conditional_t<sizeof(T) == 2, uint16_t, uint8_t> Bits;
  constexpr int WAVES = FEW_THREADS / 64, V = M * R, AHEAD = R == 1 ? 4 : 2;
  __shared__ Sum slots[WAVES][V];
  const int64_t n0 = int64_t(blockIdx.x) * R;
  const T *x[M], *w[R];
#pragma unroll
  for (int m = 0; m < M; ++m) x[m] = static_cast<const T *>(a.x) + min(int64_t(m), e.M - 1) * a.ldx;
#pragma unroll
  for (int r = 0; r < R; ++r) w[r] = static_cast<const T *>(a.w) + min(n0 + r, e.N - 1) * a.ldw;
  Sum acc[V] = {};
  auto add = [&](const u32x4 (&ux)[M], const u32x4 (&uw)[R]) {
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const Piece<T> px(ux[m]);
#pragma unroll
      for (int r = 0; r < R; ++r) Piece<T>(uw[r]).add(px, acc[m * R + r]);
    }
  };
  const int pieces = int(a.K / Piece<T>::N);
  for (int p0 = threadIdx.x; p0 < pieces; p0 += AHEAD * FEW_THREADS) {
    u32x4 ux[AHEAD][M] = {}, uw[AHEAD][R] = {};
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int p = p0 + i * FEW_THREADS;
      if (p >= pieces) break;
#pragma unroll
      for (int r = 0; r < R; ++r) uw[i][r] = load_bytes16(w[r] + int64_t(p) * Piece<T>::N);
#pragma unroll
      for (int m = 0; m < M; ++m) ux[i][m] = load_bytes16(x[m] + int64_t(p) * Piece<T>::N);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) add(ux[i], uw[i]);
  }
  // the elements past the last whole piece, one a thread
  if (const int64_t k = int64_t(pieces) * Piece<T>::N + threadIdx.x; k < a.K) {
    u32x4 ux[M] = {}, uw[R] = {};
#pragma unroll
    for (int r = 0; r < R; ++r) uw[r][0] = reinterpret_cast<const Bits *>(w[r])[k];
#pragma unroll
    for (int m = 0; m < M; ++m) ux[m][0] = reinterpret_cast<const Bits *>(x[m])[k];
    add(ux, uw);
  }
  const Sum mine = fold<V>(acc);
  const int lane = threadIdx.x % 64;
  if (lane % (64 / V) == 0) slots[threadIdx.x / 64][lane / (64 / V)] = mine;
  __syncthreads();
  const int64_t m = threadIdx.x / R, n = n0 + threadIdx.x % R;
  if (threadIdx.x >= V || m >= e.M || n >= e.N) return;
  Sum sum = slots[0][threadIdx.x];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) sum += slots[i][threadIdx.x];
  with_act(e.act, [&]<int ACT>() {
    float v[8] = {float(sum)};
    Finish<ACT> f(e);
    f.column(n);
    f.finish(m, n, v, f.fetch(m, n));
  });
}

// ----------------------------------------------------------------------------- operand copies

// Rows of src (cols elements, stride ld) to rows of `pitch` elements, zero past cols, 8-bit codes
// widened to bf16 (exact) where ST is one and DT is bf16.
template <typename ST, typename DT>
__device__ __forceinline__ DT widen(ST v);
template <> __device__ __forceinline__ bf16 widen<bf16, bf16>(bf16 v) { return v; }
template <> __device__ __forceinline__ int8_t widen<int8_t, int8_t>(int8_t v) { return v; }
template <> __device__ __forceinline__ bf16 widen<int8_t, bf16>(int8_t v) { return from_f32<bf16>(float(v)); }
template <> __device__ __forceinline__ bf16 widen<e4m3, bf16>(e4m3 v) {
  return from_f32<bf16>(__builtin_amdgcn_cvt_f32_fp8(int(v.v), 0));
}
struct Copy {
  const void *src;
  void *dst;
  int64_t rows, cols, ld, pitch;
  uint32_t blocks;         // workgroups of 256 threads (0: no copy)
};
template <typename ST, typename DT>
__device__ __forceinline__ void repack_rows(const Copy &a, uint32_t block) {
  constexpr int V = 16 / sizeof(DT);
  const int64_t groups = a.pitch / V, all = a.rows * groups;
  for (int64_t i = int64_t(block) * 256 + threadIdx.x; i < all; i += int64_t(a.blocks) * 256) {
    const int64_t r = i / groups, c = i % groups * V;
    const ST *src = static_cast<const ST *>(a.src) + r * a.ld + c;
    DT o[V];
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = c + j < a.cols ? widen<ST, DT>(src[j]) : DT{};
    uint4 u;
    __builtin_memcpy(&u, o, 16);
    *reinterpret_cast<uint4 *>(static_cast<DT *>(a.dst) + r * a.pitch + c) = u;
  }
}
// Both operands' copies in one launch.
template <typename ST, typename DT>
__global__ void __launch_bounds__(256) k_repack(Copy x, Copy w) {
  if (blockIdx.x < x.blocks) repack_rows<ST, DT>(x, blockIdx.x);
  else repack_rows<ST, DT>(w, blockIdx.x - x.blocks);
}

// ----------------------------------------------------------------------------- dz

struct DzArgs {
  const void *z, *dy;
  const float *sx, *sw;
  bf16 *dzx, *dzw;       // dz sw (for dx) and dz sx (for dw), rows of `pitch`; may be one array
  float *part;           // [rows][N] partial column sums of dz, or null
  int64_t M, N, ldz, ldy, pitch;
  int32_t y_dtype, act;
  uint32_t rows, blocks; // row groups; workgroups (row groups times 512-column groups)
};
// A thread takes 8 columns, a wave every fourth row of the workgroup's; the waves' column sums meet in
// LDS.  About 35 issue slots per element with gelu, so that it takes 16 waves per CU to keep the memory
// busy behind them.
constexpr int DZ_WAVES = 4;
__device__ __forceinline__ void dz_pass(const DzArgs &a, uint32_t block) {
  __shared__ float sums[DZ_WAVES - 1][8][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint32_t row0 = block % a.rows;
  const int64_t n = (int64_t(block / a.rows) * 64 + lane) * 8;
  const int cnt = int(max(int64_t(0), min(a.N - n, int64_t(8))));
  float sum[8] = {};
  if (cnt) {
    float sw[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sw[i] = a.sw && i < cnt ? a.sw[n + i] : 1.0f;
    with_act(a.act, [&]<int ACT>() {
      for (int64_t m = int64_t(row0) * DZ_WAVES + wave; m < a.M; m += int64_t(a.rows) * DZ_WAVES) {
        float d[8], z[8], o[8];
        load8(a.dy, m * a.ldy + n, a.y_dtype, cnt, d);
        if constexpr (ACT != FQT_ACT_NONE) {
          load8(a.z, m * a.ldz + n, a.y_dtype, cnt, z);
#pragma unroll
          for (int i = 0; i < 8; ++i) d[i] *= slope<ACT>(z[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += d[i];
        if (a.dzx) {
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = d[i] * sw[i];
          store8f(a.dzx + m * a.pitch + n, 8, o);
        }
        if (a.dzw && a.dzw != a.dzx) {
          const float s = a.sx ? a.sx[m] : 1.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = d[i] * s;
          store8f(a.dzw + m * a.pitch + n, 8, o);
        }
      }
    });
  }
  if (!a.part) return;
  if (wave)
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave - 1][i][lane] = sum[i];
  __syncthreads();
  if (wave || !cnt) return;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int w = 0; w < DZ_WAVES - 1; ++w) sum[i] += sums[w][i][lane];
  store8f(a.part + int64_t(row0) * a.N + n, cnt, sum);
}

// What the products wait for, in one launch: the pass over dy and the copies of both operands.
template <typename ST>
__global__ void __launch_bounds__(256) k_prepare(DzArgs a, Copy x, Copy w) {
  static_assert(DZ_WAVES == 4, "256 threads");
  const uint32_t b = blockIdx.x;
  if (b < a.blocks) dz_pass(a, b);
  else if (b < a.blocks + x.blocks) repack_rows<ST, bf16>(x, b - a.blocks);
  else repack_rows<ST, bf16>(w, b - a.blocks - x.blocks);
}

// dbias[n] = sum of the partial rows: 32 columns per workgroup, 8 threads per column, fixed order.
struct DbiasArgs {
  const float *part;
  float *dbias;            // or null
  int64_t N;
  int32_t parts;
};
__device__ __forceinline__ void sum_dbias(const DbiasArgs &a, uint32_t block, float (*s)[32]) {
  const int64_t c = int64_t(block) * 32 + threadIdx.x % 32;
  const int k = threadIdx.x / 32;
  float v = 0.0f;
  if (c < a.N)
#pragma unroll 8
    for (int p = k; p < a.parts; p += 8) v += a.part[int64_t(p) * a.N + c];
  s[k][threadIdx.x % 32] = v;
  __syncthreads();
  if (k == 0 && c < a.N) {
#pragma unroll
    for (int j = 1; j < 8; ++j) v += s[j][threadIdx.x];
    a.dbias[c] = v;
  }
}
__global__ void __launch_bounds__(256) k_dbias(DbiasArgs a) {
  __shared__ float s[8][32];
  sum_dbias(a, blockIdx.x, s);
}

// Two products of small tiles side by side, and dbias: the backward's dx and dw where each alone leaves
// CUs idle (777 x 1000 x 513: 10 instead of 22 + 4 us).
__global__ void __launch_bounds__(tile::Small::THREADS, 2) k_product_pair(Product px, Epilogue ex, Product pw, Epilogue ew, DbiasArgs b) {
  typedef tile::Small S;
  static_assert(S::THREADS == 256, "dbias takes 256 threads");
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];
  tile::f32x4 acc[S::FM][S::FN];
  const uint32_t first = px.tiles.count, second = first + pw.tiles.count;
  if (blockIdx.x < first) {
    const tile::Place at = tile::place<tile::SMALL>(px.tiles, blockIdx.x);
    tile::contract<tile::BF16K, ROWS, COLS, tile::SMALL, S>(px.x, px.w, px.K, at, px.tiles, lds, acc);
    tile::run_epilogue<tile::BF16K, S>(acc, lds, at.m0, at.n0, Finish<FQT_ACT_NONE>(ex));
  } else if (blockIdx.x < second) {
    const tile::Place at = tile::place<tile::SMALL>(pw.tiles, blockIdx.x - first);
    tile::contract<tile::BF16K, COLS, COLS, tile::SMALL, S>(pw.x, pw.w, pw.K, at, pw.tiles, lds, acc);
    tile::run_epilogue<tile::BF16K, S>(acc, lds, at.m0, at.n0, Finish<FQT_ACT_NONE>(ew));
  } else {
    sum_dbias(b, blockIdx.x - second, reinterpret_cast<float (*)[32]>(lds));
  }
}
__global__ void __launch_bounds__(256) k_zero(char *p, int64_t rows, int64_t bytes, int64_t ld) {
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < rows * bytes; i += int64_t(gridDim.x) * 256)
    p[i / bytes * ld + i % bytes] = 0;
}

// ----------------------------------------------------------------------------- host side

struct Sizes {
  int64_t M, N, K;
  int64_t ldx, ldw, ldr, ldy, ldz, lddx, lddw;
  size_t xe;             // bytes of an operand element
};
int check_linear(const fqt_linear_desc *d, Sizes *s) {
  if (!d) return FQT_E_NULL;
  if (!(d->x_dtype == FQT_BF16 || code_type(d->x_dtype)) || !float_type(d->y_dtype) ||
      !float_type(d->dx_dtype) || !float_type(d->dw_dtype))
    return FQT_E_DTYPE;
  if (d->act < FQT_ACT_NONE || d->act > FQT_ACT_HARDTANH) return FQT_E_INVAL;
  if (d->M < 0 || d->N < 0 || d->K < 0 || d->M >= FQT_MAX_ROWS || d->N > FQT_MAX_LD || d->K > FQT_MAX_LD)
    return FQT_E_SHAPE;
  // (a launch counts its threads in 32 bits)
  for (const uint64_t tiles : {tile::large_tiles(d->M, d->N), tile::large_tiles(d->M, d->K), tile::large_tiles(d->N, d->K)})
    if (tiles >= tile::MOST_LARGE) return FQT_E_SHAPE;
  if (d->x_dtype == FQT_I8 && d->K > 133144) return FQT_E_SHAPE;   // 127^2 K < 2^31
  *s = {d->M, d->N, d->K, row_stride(d->ldx, d->K), row_stride(d->ldw, d->K), row_stride(d->ldr, d->N),
        row_stride(d->ldy, d->N), row_stride(d->ldz, d->N), row_stride(d->lddx, d->K),
        row_stride(d->lddw, d->K), elem_size(d->x_dtype)};
  if (!s->ldx || !s->ldw || !s->ldr || !s->ldy || !s->ldz || !s->lddx || !s->lddw) return FQT_E_SHAPE;
  return FQT_OK;
}

int64_t round_up(int64_t v, int64_t q) { return (v + q - 1) / q * q; }
// Whether rows of n elements, ld apart, are whole 16-byte pieces.
bool whole_pieces(int64_t n, int64_t ld, size_t e) { return n * e % 16 == 0 && ld * e % 16 == 0; }

tile::Plan plan_of(int64_t M, int64_t N, int64_t K, size_t e) {
  return tile::make_plan(M, N, (K * int64_t(e) + tile::KB - 1) / tile::KB, false, tile::DENSE_COSTS);
}
size_t part_bytes(const tile::Plan &p, int64_t M, int64_t N) {
  return p.splits > 1 ? align256(size_t(p.splits) * M * round_up(N, 8) * 4) : 0;
}

Epilogue sized(Epilogue e, int64_t M, int64_t N) {
  e.M = M;
  e.N = N;
  return e;
}
template <int KIND, int LX, int LW>
int launch_product(const tile::Plan &plan, Operand x, Operand w, int64_t M, int64_t N, int64_t K, Epilogue e,
                   float *part, hipStream_t st) {
  if (M == 0 || N == 0) return FQT_OK;
  Product p{x, w, M, N, K, plan.t[0], part, round_up(N, 8)};
  e = sized(e, M, N);
  tile::for_launches(plan, [&]<int SHAPE>(const tile::Tiles &t) {
    p.tiles = t;
    k_product<KIND, LX, LW, SHAPE><<<dim3(uint32_t(tile::blocks_of(t))), dim3(tile::ShapeOf<SHAPE>::type::THREADS), 0, st>>>(p, e);
  });
  FQT_TRY_(last_launch_status());
  if (plan.splits > 1) {
    const int64_t all = M * (p.ldp / 8);
    k_product_finish<KIND == tile::I8K><<<dim3(std::min<int64_t>((all + 255) / 256, 4096)), dim3(256), 0, st>>>(p, e);
    return last_launch_status();
  }
  return FQT_OK;
}

// Four rows of w a workgroup where they fill the chip all the same, since x is then read a quarter as often;
// one where they do not (us with four and one, bf16, K = 25088: 1 x 512 11.1 and 7.9, 1 x 2048 20.4 and 20.4, 4 x 512
// 15.1 and 12.2, 4 x 1000 16.5 and 20.6, 4 x 2048 23.3 and 36.4).
template <typename T>
int launch_few(const FewArgs &a, const Epilogue &e, hipStream_t st) {
  auto rows = [&]<int M>() {
    if (M * e.N >= FEW_WIDE) k_few_rows<T, M, 4><<<dim3(uint32_t((e.N + 3) / 4)), dim3(FEW_THREADS), 0, st>>>(a, e);
    else k_few_rows<T, M, 1><<<dim3(uint32_t(e.N)), dim3(FEW_THREADS), 0, st>>>(a, e);
  };
  if (e.M == 1) rows.template operator()<1>();
  else if (e.M == 2) rows.template operator()<2>();
  else rows.template operator()<4>();
  return last_launch_status();
}

// The copy of an operand into rows of `pitch` elements of e bytes.
Copy copy_of(const void *src, int64_t rows, int64_t cols, int64_t ld, void *dst, int64_t pitch, int64_t e) {
  const int64_t all = rows * (pitch * e / 16);
  return {src, dst, rows, cols, ld, pitch, uint32_t(std::min<int64_t>((all + 255) / 256, 4096))};
}

// Workspace of the forward: padded copies of operands whose rows are not whole 16-byte pieces, and
// the partial sums of a split contraction.
struct FwdWs { size_t x, w, part, total; int64_t pitch, e; tile::Plan plan; bool widen, copy_x, copy_w; };
FwdWs fwd_ws(const fqt_linear_desc &d, const Sizes &s) {
  FwdWs f{};
  if (s.M <= FEW_MOST) return f;
  // The e4m3 matrix instruction adds the products of a step in fewer bits than float32 has (sums off by
  // 1e-5 to 6e-5 of their norm): below the rounding of a bf16 output, not of a float32 one, for which the
  // codes go through bf16 copies (exact) and that type's instruction.
  f.widen = d.x_dtype == FQT_E4M3 && d.y_dtype == FQT_F32;
  f.e = f.widen ? 2 : int64_t(s.xe);
  f.pitch = round_up(s.K, 16 / f.e);
  f.copy_x = f.widen || !whole_pieces(s.K, s.ldx, s.xe);
  f.copy_w = f.widen || !whole_pieces(s.K, s.ldw, s.xe);
  f.plan = plan_of(s.M, s.N, s.K, f.e);
  f.x = 0;
  f.w = f.x + (f.copy_x ? align256(s.M * f.pitch * f.e) : 0);
  f.part = f.w + (f.copy_w ? align256(s.N * f.pitch * f.e) : 0);
  f.total = f.part + part_bytes(f.plan, s.M, s.N);
  return f;
}

// Workspace of the backward: dz in bf16 (twice for scaled operands), bf16 copies of operands that
// are codes or whose rows are not whole pieces, the partial sums of dbias, and those of the products
// (which run one after the other).
struct BwdWs { size_t dzx, dzw, x, w, bias, part, total; int64_t dz_pitch, pitch, rows; tile::Plan dx, dw; bool copy_x, copy_w; };
BwdWs bwd_ws(const Sizes &s) {
  BwdWs f{};
  const bool codes = s.xe == 1;
  f.dz_pitch = round_up(s.N, 8);
  f.pitch = round_up(s.K, 8);
  f.copy_x = codes || !whole_pieces(s.K, s.ldx, 2);
  f.copy_w = codes || !whole_pieces(s.K, s.ldw, 2);
  // row groups of the pass over dy: enough waves, few partial sums of dbias
  f.rows = std::max<int64_t>(1, std::min<int64_t>((s.M + 7) / 8, 128));
  f.dx = plan_of(s.M, s.K, s.N, 2);
  f.dw = plan_of(s.N, s.K, s.M, 2);
  const size_t dz = align256(size_t(s.M) * f.dz_pitch * 2);
  f.dzx = 0;
  f.dzw = codes ? dz : 0;
  f.x = f.dzw + dz;
  f.w = f.x + (f.copy_x ? align256(size_t(s.M) * f.pitch * 2) : 0);
  f.bias = f.w + (f.copy_w ? align256(size_t(s.N) * f.pitch * 2) : 0);
  f.part = f.bias + align256(size_t(f.rows) * s.N * 4);
  f.total = f.part + std::max(part_bytes(f.dx, s.M, s.K), part_bytes(f.dw, s.N, s.K));
  return f;
}

int zero_matrix(void *p, int64_t rows, int64_t cols, int64_t ld, size_t e, hipStream_t st) {
  if (rows == 0 || cols == 0) return FQT_OK;
  k_zero<<<dim3(std::min<int64_t>((rows * cols * int64_t(e) + 255) / 256, 4096)), dim3(256), 0, st>>>(
      static_cast<char *>(p), rows, cols * e, ld * e);
  return last_launch_status();
}

}  // namespace
}  // namespace dense
}  // namespace fqt

using namespace fqt;
using namespace fqt::dense;

extern "C" int fqt_linear_workspace_size(const fqt_linear_desc *d, int32_t backward, size_t *bytes) {
  Sizes s;
  FQT_TRY_(check_linear(d, &s));
  if (!bytes) return FQT_E_NULL;
  *bytes = std::max<size_t>(256, backward ? bwd_ws(s).total : fwd_ws(*d, s).total);
  return FQT_OK;
}

extern "C" int fqt_linear_plan(const fqt_linear_desc *d, int32_t product, fqt_product_plan *plan) {
  Sizes s;
  FQT_TRY_(check_linear(d, &s));
  if (!plan) return FQT_E_NULL;
  if (product < FQT_PRODUCT_FORWARD || product > FQT_PRODUCT_DW) return FQT_E_INVAL;
  tile::Plan p{};
  if (product == FQT_PRODUCT_FORWARD) p = fwd_ws(*d, s).plan;
  else p = product == FQT_PRODUCT_DX ? bwd_ws(s).dx : bwd_ws(s).dw;
  tile::describe(p, plan);
  return FQT_OK;
}

extern "C" int fqt_linear_forward(const fqt_linear_desc *d, const void *x, const void *w,
                                  const float *x_scale, const float *w_scale, const float *bias,
                                  const void *residual, void *z, void *y, void *ws, size_t ws_bytes,
                                  void *hip_stream) {
  Sizes s;
  FQT_TRY_(check_linear(d, &s));
  const bool codes = code_type(d->x_dtype);
  if (!codes && (x_scale || w_scale)) return FQT_E_DTYPE;
  if (s.M == 0 || s.N == 0) return FQT_OK;
  if (!y || !ws || (s.K && (!x || !w)) || (codes && (!x_scale || !w_scale))) return FQT_E_NULL;
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4) ||
      !aligned(bias, 4) || !elem_aligned(residual, d->y_dtype) || !elem_aligned(z, d->y_dtype) ||
      !elem_aligned(y, d->y_dtype) || !aligned(ws, 256))
    return FQT_E_ALIGN;
  const FwdWs f = fwd_ws(*d, s);
  if (ws_bytes < f.total) return FQT_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  Epilogue e{x_scale, w_scale, bias, residual, z, y, s.M, s.N, s.ldr, s.ldz, s.ldy, d->y_dtype, d->act};
  if (s.M <= FEW_MOST) {
    const FewArgs a{x, w, s.K, s.ldx, s.ldw};
    if (d->x_dtype == FQT_BF16) return launch_few<bf16>(a, e, st);
    return d->x_dtype == FQT_I8 ? launch_few<int8_t>(a, e, st) : launch_few<e4m3>(a, e, st);
  }
  char *base = static_cast<char *>(ws);
  auto operand = [&](const void *p, bool copy, size_t at, int64_t rows, int64_t ld, Copy *c) -> Operand {
    if (!copy) return {static_cast<const char *>(p), ld * f.e, rows};
    *c = copy_of(p, rows, s.K, ld, base + at, f.pitch, f.e);
    return {base + at, f.pitch * f.e, rows};
  };
  Copy cx{}, cw{};
  const Operand xo = operand(x, f.copy_x, f.x, s.M, s.ldx, &cx), wo = operand(w, f.copy_w, f.w, s.N, s.ldw, &cw);
  if (const dim3 grid(cx.blocks + cw.blocks); grid.x) {
    if (f.widen) k_repack<e4m3, bf16><<<grid, dim3(256), 0, st>>>(cx, cw);
    else if (codes) k_repack<int8_t, int8_t><<<grid, dim3(256), 0, st>>>(cx, cw);
    else k_repack<bf16, bf16><<<grid, dim3(256), 0, st>>>(cx, cw);
    FQT_TRY_(last_launch_status());
  }
  const int64_t K = f.copy_x || f.copy_w ? f.pitch : s.K;
  float *part = reinterpret_cast<float *>(base + f.part);
  if (d->x_dtype == FQT_BF16 || f.widen)
    return launch_product<tile::BF16K, ROWS, ROWS>(f.plan, xo, wo, s.M, s.N, K, e, part, st);
  if (d->x_dtype == FQT_I8)
    return launch_product<tile::I8K, ROWS, ROWS>(f.plan, xo, wo, s.M, s.N, K, e, part, st);
  return launch_product<tile::E4M3K, ROWS, ROWS>(f.plan, xo, wo, s.M, s.N, K, e, part, st);
}

extern "C" int fqt_linear_backward(const fqt_linear_desc *d, const void *x, const void *w,
                                   const float *x_scale, const float *w_scale, const void *z,
                                   const void *dy, void *dx, void *dw, float *dbias, void *ws,
                                   size_t ws_bytes, void *hip_stream) {
  Sizes s;
  FQT_TRY_(check_linear(d, &s));
  const bool codes = code_type(d->x_dtype);
  if (!codes && (x_scale || w_scale)) return FQT_E_DTYPE;
  if (!dx && !dw && !dbias) return FQT_OK;
  const bool any = s.M && s.N;
  if (!ws || (any && !dy) || (any && d->act != FQT_ACT_NONE && !z) || (dx && any && s.K && !w) ||
      (dw && any && s.K && !x) || (codes && any && ((dw && !x_scale) || (dx && !w_scale))))
    return FQT_E_NULL;
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(x_scale, 4) || !aligned(w_scale, 4) ||
      !elem_aligned(z, d->y_dtype) || !elem_aligned(dy, d->y_dtype) || !elem_aligned(dx, d->dx_dtype) ||
      !elem_aligned(dw, d->dw_dtype) || !aligned(dbias, 4) || !aligned(ws, 256))
    return FQT_E_ALIGN;
  const BwdWs f = bwd_ws(s);
  if (ws_bytes < f.total) return FQT_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (!any) {            // sums over nothing
    if (dx) FQT_TRY_(zero_matrix(dx, s.M, s.K, s.lddx, elem_size(d->dx_dtype), st));
    if (dw) FQT_TRY_(zero_matrix(dw, s.N, s.K, s.lddw, elem_size(d->dw_dtype), st));
    if (dbias) FQT_TRY_(zero_matrix(dbias, 1, s.N, s.N, 4, st));
    return FQT_OK;
  }
  char *base = static_cast<char *>(ws);
  // dy is dz itself where nothing changes it.
  const bool same = d->act == FQT_ACT_NONE && d->y_dtype == FQT_BF16 && !codes &&
                    whole_pieces(s.N, s.ldy, 2) && aligned(dy, 16);
  Operand dzx{base + f.dzx, f.dz_pitch * 2, s.M}, dzw{base + f.dzw, f.dz_pitch * 2, s.M};
  if (same) dzx = dzw = {static_cast<const char *>(dy), s.ldy * 2, s.M};
  auto operand = [&](const void *p, bool copy, size_t at, int64_t rows, int64_t ld, Copy *c) -> Operand {
    if (!copy) return {static_cast<const char *>(p), ld * 2, s.K};
    *c = copy_of(p, rows, s.K, ld, base + at, f.pitch, 2);
    return {base + at, f.pitch * 2, f.pitch};
  };
  Copy cx{}, cw{};
  Operand wo{}, xo{};
  if (dx) wo = operand(w, f.copy_w, f.w, s.N, s.ldw, &cw);
  if (dw) xo = operand(x, f.copy_x, f.x, s.M, s.ldx, &cx);
  DzArgs a{};
  if (!same || dbias) {
    a.z = z; a.dy = dy;
    a.sx = x_scale; a.sw = w_scale;
    if (!same && dx) a.dzx = reinterpret_cast<bf16 *>(base + f.dzx);
    if (!same && dw) a.dzw = reinterpret_cast<bf16 *>(base + f.dzw);
    a.part = dbias ? reinterpret_cast<float *>(base + f.bias) : nullptr;
    a.M = s.M; a.N = s.N; a.ldz = s.ldz; a.ldy = s.ldy; a.pitch = f.dz_pitch;
    a.y_dtype = d->y_dtype; a.act = d->act;
    a.rows = uint32_t(f.rows);
    a.blocks = uint32_t((f.dz_pitch + 511) / 512 * f.rows);
  }
  if (const dim3 grid(a.blocks + cx.blocks + cw.blocks); grid.x) {
    if (d->x_dtype == FQT_I8) k_prepare<int8_t><<<grid, dim3(256), 0, st>>>(a, cx, cw);
    else if (d->x_dtype == FQT_E4M3) k_prepare<e4m3><<<grid, dim3(256), 0, st>>>(a, cx, cw);
    else k_prepare<bf16><<<grid, dim3(256), 0, st>>>(a, cx, cw);
    FQT_TRY_(last_launch_status());
  }
  const DbiasArgs bias{a.part, dbias, s.N, int32_t(f.rows)};
  const uint32_t bias_blocks = dbias ? uint32_t((s.N + 31) / 32) : 0;
  float *part = reinterpret_cast<float *>(base + f.part);
  // dz rows are dz_pitch long in the workspace, zeros past N, so a contraction over n may end on a whole
  // piece; as a COLS operand dz has whole pieces of 8 columns.
  dzw.rows = same ? s.N : f.dz_pitch;
  const Epilogue ex{nullptr, nullptr, nullptr, nullptr, nullptr, dx, 0, 0, 0, 0, s.lddx, d->dx_dtype, FQT_ACT_NONE};
  const Epilogue ew{nullptr, nullptr, nullptr, nullptr, nullptr, dw, 0, 0, 0, 0, s.lddw, d->dw_dtype, FQT_ACT_NONE};
  auto small = [](const tile::Plan &p) { return p.shape[0] == tile::SMALL && p.launches == 1 && p.splits == 1; };
  if (dx && dw && s.K && small(f.dx) && small(f.dw)) {
    const Product px{dzx, wo, s.M, s.K, s.N, f.dx.t[0], nullptr, 0}, pw{dzw, xo, s.N, s.K, s.M, f.dw.t[0], nullptr, 0};
    k_product_pair<<<dim3(px.tiles.count + pw.tiles.count + bias_blocks), dim3(tile::Small::THREADS), 0, st>>>(
        px, sized(ex, s.M, s.K), pw, sized(ew, s.N, s.K), bias);
    return last_launch_status();
  }
  if (dbias) {
    k_dbias<<<dim3(bias_blocks), dim3(256), 0, st>>>(bias);
    FQT_TRY_(last_launch_status());
  }
  if (s.K == 0) return FQT_OK;
  if (dx) FQT_TRY_((launch_product<tile::BF16K, ROWS, COLS>(f.dx, dzx, wo, s.M, s.K, s.N, ex, part, st)));
  if (dw) FQT_TRY_((launch_product<tile::BF16K, COLS, COLS>(f.dw, dzw, xo, s.N, s.K, s.M, ew, part, st)));
  return FQT_OK;
}
