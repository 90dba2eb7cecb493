// Softmax cross entropy of a linear layer's outputs without keeping them, and its gradients.
//
// The forward is the product's tiles (fqt_tile.hpp) with an epilogue that takes each row of a wave's 64
// columns down to a pair (largest z, sum of the exponentials of the others over it); a second launch joins
// the pairs of a row.  8 bytes for 64 columns touch memory instead of 256.  The backward computes z again
// piece by piece of the classes, writes dz of a piece in bf16, and multiplies it into dx and dw
// (fqt_linear.hip's products) while it is still in the last-level cache.  All of it is bound by the matrix cores on
// large batches, by reading w on small ones.
#include "fqt_product.hpp"
#include "fqt_step.h"

namespace fqt {
namespace dense {
namespace {

#pragma clang fp contract(fast)

using tile::Operand;
using tile::ROWS;

constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.69314718055994531f;
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * LOG2E); }
// (NaN if either is one)
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float smaller(float a, float b) { return __builtin_elementwise_minimum(a, b); }

// A set of y = z log2(e): its largest, and the sum of 2^(y - top) over all others.  The largest's own 1 is left
// out, so that a loss near 0, the sum of the others, keeps its precision.  (In these units a value goes into the exponential
// without a product of its own; y and top are each off by half a unit in the last place, 2^-25 |y|.)
struct Soft {
  float top, rest;
};
constexpr float NOTHING = -__builtin_inff();
// What is subtracted: classes may all be out (minus infinity).
__device__ __forceinline__ float base_of(float top) { return top == NOTHING ? 0.0f : top; }
__device__ __forceinline__ Soft join(Soft a, Soft b) {
  const float hi = larger(a.top, b.top), e = __builtin_amdgcn_exp2f(smaller(a.top, b.top) - base_of(hi));
  const bool first = a.top >= b.top;
  return {hi, fmaf((first ? b.rest : a.rest) + 1.0f, e, first ? a.rest : b.rest)};
}
template <int X>
__device__ __forceinline__ Soft join_lanes(Soft a) {
  return join(a, Soft{lane_xor_f<X>(a.top), lane_xor_f<X>(a.rest)});
}
// N values: a pass of min and max leaves the largest and the others.
template <int N>
__device__ __forceinline__ Soft soft_of(const float (&v)[N]) {
  float top = v[0], low[N];
#pragma unroll
  for (int i = 1; i < N; ++i) {
    low[i] = smaller(top, v[i]);
    top = larger(top, v[i]);
  }
  const float base = base_of(top);
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 1; i < N; ++i) s[i % 2] += __builtin_amdgcn_exp2f(low[i] - base);
  return {top, s[0] + s[1]};
}

struct Out {
  const int64_t *target;
  float *loss, *lse;
  int64_t M, N, ignore;
  float smoothing;
  float *mean;             // for a launch of one workgroup that has all rows, or null
  float *logp;             // log p of the targets, or null
};
// Row m from its pair, the sum of its y and the target's y.
// Returns its loss, and in `counts` whether it counts.
__device__ __forceinline__ float finish_row(const Out &o, int64_t m, Soft s, float sum, float at, bool &counts) {
  const float rest = log1pf(s.rest);
  o.lse[m] = fmaf(s.top, LN2, rest);
  const int64_t t = o.target[m];
  const float gap = s.top - at;
  float loss = gap;
  if (o.smoothing > 0.0f) loss = (1.0f - o.smoothing) * loss + o.smoothing * (s.top - sum / float(o.N));
  loss = fmaf(loss, LN2, rest);
  counts = t != o.ignore;
  auto valid = [&](float v) { return !counts ? 0.0f : t < 0 || t >= o.N ? __builtin_nanf("") : v; };
  loss = valid(loss);
  o.loss[m] = loss;
  if (o.logp) o.logp[m] = valid(-fmaf(gap, LN2, rest));
  return loss;
}
// mean[0]: of the losses of the rows that count, mean[1]: 1 / their number.
__device__ __forceinline__ void store_mean(float *mean, double sum, int64_t count) {
  mean[0] = count ? float(sum / double(count)) : 0.0f;
  mean[1] = count ? float(1.0 / double(count)) : 0.0f;
}
// The sum and the count of a workgroup's threads to its mean.
__device__ __forceinline__ void mean_of(float *mean, double sum, int64_t count) {
  __shared__ double sums[16];
  __shared__ int64_t counts[16];
#pragma unroll
  for (int o = 32; o > 0; o /= 2) {
    sum += __shfl_xor(sum, o);
    count += __shfl_xor(count, o);
  }
  if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = sum, counts[threadIdx.x / 64] = count;
  __syncthreads();
  if (threadIdx.x) return;
  for (uint32_t i = 1; i < blockDim.x / 64; ++i) sum += sums[i], count += counts[i];
  store_mean(mean, sum, count);
}

// ----------------------------------------------------------------------------- forward by tiles

struct Logits {
  Operand x, w;
  int64_t M, N, K;
  tile::Tiles tiles;
  const float *sx, *sw, *bias;
  float *part;             // [splits][M][ldp] partial sums (splits > 1)
  int64_t ldp;
};
constexpr int SLOT = 64;   // columns of a pair
struct Pairs {
  Soft *pairs;             // [slots][M]
  float *sums;             // [slots][M] sums of y, or null
  float *at;               // [M] the target's y
  const int64_t *target;
  int64_t slots;
};

// Keeps what depends on v behind the branch it is in (the compiler moves cheap work before branches).
__device__ __forceinline__ void stay_here(float &v) { asm volatile("" : "+v"(v)); }

// A value of the lanes with bit X (16 or 32) clear and of those with it set, each to both.
template <int X>
__device__ __forceinline__ void halves(float v, float &clear, float &set) {
  const int i = __float_as_int(v);
  if constexpr (X == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(i, i, false, false);
    clear = __int_as_float(r[0]), set = __int_as_float(r[1]);
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(i, i, false, false);
    clear = __int_as_float(r[0]), set = __int_as_float(r[1]);
  }
}
// The pair of N values in each of four lanes (l, l ^ 16, l ^ 32, l ^ 48): the largest of all first, then one exponential
// of every other value; the losers among the four lanes' largest are two of the first exchange and one of the second.
template <int N>
__device__ __forceinline__ Soft soft_of_four(const float (&v)[N]) {
  float top = v[0], low[N + 1];
#pragma unroll
  for (int i = 1; i < N; ++i) {
    low[i - 1] = smaller(top, v[i]);
    top = larger(top, v[i]);
  }
  const uint32_t l = __lane_id();
  float a, b;
  halves<16>(top, a, b);
  low[N - 1] = l & 16 ? NOTHING : smaller(a, b);
  top = larger(a, b);
  halves<32>(top, a, b);
  low[N] = l & 48 ? NOTHING : smaller(a, b);
  top = larger(a, b);
  const float base = base_of(top);
  float s[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i <= N; ++i) s[i % 2] += __builtin_amdgcn_exp2f(low[i] - base);
  halves<16>(s[0] + s[1], a, b);
  halves<32>(a + b, a, b);
  return {top, a + b};
}

// The pairs of a tile, straight from the accumulators: lane l has row l % 16 of each 16 x 16 result and four
// columns from 4 (l / 16), so a row's 64 columns are in four lanes, 16 each.  SMOOTH: their sums too.  8192 x 100003 x 2304
// int8 (18 steps of 1.37 us a tile): of 19 us that a tile took beside its steps, 5 were this arithmetic, 3 the loads that
// are issued together here.
template <int KIND, bool SMOOTH, typename S>
__device__ __forceinline__ void store_pairs(const Logits &p, const Pairs &o, const tile::Place &at,
                                            const typename tile::Acc<KIND>::type (&acc)[S::FM][S::FN], char *lds) {
  constexpr int PER = S::FN * 4;
  const uint32_t wave = wave_id(), l = __lane_id(), q = l / 16;
  const int64_t m0 = at.m0 + (wave / S::WN) * S::TM, n0 = at.n0 + (wave % S::WN) * S::TN;
  const int64_t col = n0 + 4 * q;
  // (no branch between the loads: past the ends they read the last element again)
  float bias[PER], sw[PER], sx[S::FM];
  int64_t target[S::FM];
#pragma unroll
  for (int k = 0; k < S::FM; ++k) target[k] = o.target[min(m0 + k * 16 + l % 16, p.M - 1)];
  if constexpr (KIND != tile::BF16K) {
#pragma unroll
    for (int k = 0; k < S::FM; ++k) sx[k] = p.sx[min(m0 + k * 16 + l % 16, p.M - 1)];
#pragma unroll
    for (int j = 0; j < PER; ++j) sw[j] = p.sw[min(col + 16 * (j / 4) + j % 4, p.N - 1)];
  }
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < PER; ++j) bias[j] = p.bias[min(col + 16 * (j / 4) + j % 4, p.N - 1)] * LOG2E;
  } else {
#pragma unroll
    for (int j = 0; j < PER; ++j) bias[j] = 0.0f;
  }
  // columns past the last are out
  if (n0 + S::TN > p.N) {
#pragma unroll
    for (int j = 0; j < PER; ++j) bias[j] = col + 16 * (j / 4) + j % 4 < p.N ? bias[j] : NOTHING;
  }
  int where[S::FM];        // the target's place among the wave's columns
#pragma unroll
  for (int k = 0; k < S::FM; ++k) {
    const int64_t t = target[k] - n0;
    where[k] = m0 + k * 16 + l % 16 < p.M && t >= 0 && t < S::TN && t < p.N - n0 ? int(t) : -1;
  }
  Soft held{};
  float held_sum = 0.0f;
#pragma unroll
  for (int k = 0; k < S::FM; ++k) {
    float v[PER];
#pragma unroll
    for (int j = 0; j < S::FN; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (KIND == tile::BF16K) v[4 * j + i] = fmaf(acc[k][j][i], LOG2E, bias[4 * j + i]);
        else v[4 * j + i] = fmaf(float(acc[k][j][i]) * (sx[k] * LOG2E), sw[4 * j + i], bias[4 * j + i]);
      }
    if (const bool mine = where[k] >= 0 && uint32_t(where[k] / 4 % 4) == q; __any(mine)) {
      const int i = where[k] / 16 * 4 + where[k] % 4;
      float z = v[0];
      stay_here(z);
#pragma unroll
      for (int j = 1; j < PER; ++j) z = i == j ? v[j] : z;
      if (mine) o.at[m0 + k * 16 + l % 16] = z;
    }
    const Soft s = soft_of_four<PER>(v);
    float sum = 0.0f;
    if constexpr (SMOOTH) {
#pragma unroll
      for (int j = 0; j < PER; ++j) sum += col + 16 * (j / 4) + j % 4 < p.N ? v[j] : 0.0f;
      sum += lane_xor_f<16>(sum);
      sum += lane_xor_f<32>(sum);
    }
    if constexpr (S::TN == SLOT) {
      // each quarter of the lanes keeps one of four results, so that a store takes 64 rows
      if (k % 4 == int(q)) held = s, held_sum = sum;
      if (k % 4 == 3) {
        const int64_t r = m0 + (k / 4) * 64 + l;
        if (r < p.M && n0 < p.N) {
          o.pairs[n0 / SLOT * p.M + r] = held;
          if constexpr (SMOOTH) o.sums[n0 / SLOT * p.M + r] = held_sum;
        }
      }
    } else {
      static_assert(S::TN * 2 == SLOT && S::WN == 2 && S::BN == SLOT, "two waves make a slot");
      float4 *both = reinterpret_cast<float4 *>(lds);      // [2][BM]
      if (q == 0) both[wave % 2 * S::BM + (wave / 2) * S::TM + k * 16 + l] = make_float4(s.top, s.rest, sum, 0.0f);
    }
  }
  if constexpr (S::TN != SLOT) {
    const float4 *both = reinterpret_cast<const float4 *>(lds);
    __syncthreads();
    const int64_t r = at.m0 + threadIdx.x;
    if (threadIdx.x < S::BM && r < p.M) {
      const float4 a = both[threadIdx.x], b = both[S::BM + threadIdx.x];
      o.pairs[at.n0 / SLOT * p.M + r] = join(Soft{a.x, a.y}, Soft{b.x, b.y});
      if constexpr (SMOOTH) o.sums[at.n0 / SLOT * p.M + r] = a.z + b.z;
    }
  }
}

template <int KIND, bool SMOOTH, int SHAPE>
__global__ void __launch_bounds__(tile::ShapeOf<SHAPE>::type::THREADS, 2) k_loss_tiles(Logits p, Pairs o) {
  typedef typename tile::ShapeOf<SHAPE>::type S;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];
  const tile::Place at = tile::place<SHAPE>(p.tiles, blockIdx.x);
  if (at.m0 >= p.M || at.n0 >= p.N) return;              // (parts of an edge tile)
  typename tile::Acc<KIND>::type acc[S::FM][S::FN];
  tile::contract<KIND, ROWS, ROWS, SHAPE, S>(p.x, p.w, p.K, at, p.tiles, lds, acc);
  if (p.tiles.splits > 1)
    tile::run_epilogue<KIND, S>(acc, lds, at.m0, at.n0, tile::StorePart{p.part + at.split * p.M * p.ldp, p.M, p.ldp});
  else
    store_pairs<KIND, SMOOTH, S>(p, o, at, acc, lds);
}

// Joins the pairs of 16 rows by 16 threads each, which take every 16th slot; workgroups walk the rows.
__global__ void __launch_bounds__(256) k_loss_rows(Pairs p, Out o) {
  constexpr int AHEAD = 8;
  __shared__ float4 all[16][17];
  const int r = threadIdx.x % 16, g = threadIdx.x / 16;
  const int64_t slots = p.slots;
  for (int64_t m0 = int64_t(blockIdx.x) * 16; m0 < o.M; m0 += int64_t(gridDim.x) * 16) {
    const int64_t m = m0 + r;
    Soft s{NOTHING, 0.0f};
    float sum = 0.0f;
    if (m < o.M)
      for (int64_t i0 = g; i0 < slots; i0 += 16 * AHEAD) {
        Soft t[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
          t[i] = i0 + 16 * i < slots ? p.pairs[(i0 + 16 * i) * o.M + m] : Soft{NOTHING, 0.0f};
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) s = join(s, t[i]);
        if (p.sums)
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) sum += i0 + 16 * i < slots ? p.sums[(i0 + 16 * i) * o.M + m] : 0.0f;
      }
    all[g][r] = make_float4(s.top, s.rest, sum, 0.0f);
    __syncthreads();
    if (g == 0 && m < o.M) {
#pragma unroll
      for (int i = 1; i < 16; ++i) {
        const float4 b = all[i][r];
        s = join(s, Soft{b.x, b.y});
        sum += b.z;
      }
      const int64_t t = p.target[m];
      bool counts;
      finish_row(o, m, s, sum, t >= 0 && t < o.N ? p.at[m] : 0.0f, counts);
    }
    __syncthreads();
  }
}
// The same for up to 1024 rows by one workgroup, `rows` (a power of two) threads side by side, and their mean: a launch less
// (4 us of the 15 of a small call).
__global__ void __launch_bounds__(1024) k_loss_rows_mean(Pairs p, Out o, uint32_t rows) {
  constexpr int AHEAD = 8;
  __shared__ float4 all[1024];
  const uint32_t groups = 1024 / rows, g = threadIdx.x / rows;
  const int64_t m = threadIdx.x % rows;
  Soft s{NOTHING, 0.0f};
  float sum = 0.0f;
  if (m < o.M)
    for (int64_t i0 = g; i0 < p.slots; i0 += groups * AHEAD) {
      Soft t[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        t[i] = i0 + groups * i < p.slots ? p.pairs[(i0 + groups * i) * o.M + m] : Soft{NOTHING, 0.0f};
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) s = join(s, t[i]);
      if (p.sums)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) sum += i0 + groups * i < p.slots ? p.sums[(i0 + groups * i) * o.M + m] : 0.0f;
    }
  all[threadIdx.x] = make_float4(s.top, s.rest, sum, 0.0f);
  __syncthreads();
  float loss = 0.0f;
  bool counts = false;
  if (g == 0 && m < o.M) {
    for (uint32_t i = 1; i < groups; ++i) {
      const float4 b = all[i * rows + m];
      s = join(s, Soft{b.x, b.y});
      sum += b.z;
    }
    const int64_t t = p.target[m];
    loss = finish_row(o, m, s, sum, t >= 0 && t < o.N ? p.at[m] : 0.0f, counts);
  }
  mean_of(o.mean, double(loss), counts);
}

// ----------------------------------------------------------------------------- forward by rows
// Where z passes through the workspace (few rows, or a split contraction): a workgroup takes CHUNK columns of a
// row down to a pair, or the whole row to its loss if that is all (then every 256 threads of a workgroup take a row, and one
// with all rows their mean); z are sums of `splits` words.  One row of 65536 by one workgroup took 18 us.
struct RowArgs {
  const float *part;
  const float *sx, *sw, *bias;
  int64_t ldp;
  uint32_t splits;
};
constexpr int CHUNK = 4096;
template <bool INTS>
__global__ void __launch_bounds__(1024) k_loss_dense(RowArgs a, Pairs p, Out o) {
  __shared__ float4 waves[16];
  __shared__ float found_of[4];
  const uint32_t thread = threadIdx.x % 256, row = threadIdx.x / 256;
  const int64_t m = blockIdx.x / p.slots * (blockDim.x / 256) + row, slot = blockIdx.x % p.slots, t = o.target[m];
  const int64_t n0 = slot * CHUNK, end = min(o.N, n0 + CHUNK);
  const float sx = a.sx ? a.sx[m] : 1.0f;
  float &found = found_of[row];
  if (thread == 0) found = 0.0f;
  __syncthreads();
  Soft s{NOTHING, 0.0f};
  float sum = 0.0f;
#pragma unroll 4
  for (int64_t n = n0 + thread * 4; n < end; n += 1024) {
    const int cnt = int(min(end - n, int64_t(4)));
    std::conditional_t<INTS, int, float> w[4] = {};
    for (uint32_t i = 0; i < a.splits; ++i) {
      const float *at = a.part + (i * o.M + m) * a.ldp + n;
      uint32_t u[4] = {};
      if (cnt == 4) {
        const u32x4 q = load_bytes16(at);
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = q[j];
      } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < cnt) u[j] = __float_as_uint(at[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (INTS) w[j] += int(u[j]);
        else w[j] += __uint_as_float(u[j]);
      }
    }
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = float(w[i]);
      if (i >= cnt) {
        v[i] = NOTHING;
        continue;
      }
      if (a.sx) v[i] = v[i] * sx * a.sw[n + i];
      if (a.bias) v[i] += a.bias[n + i];
      v[i] *= LOG2E;
      sum += v[i];
      if (n + i == t) found = v[i];
    }
    s = join(s, soft_of<4>(v));
  }
  s = join_lanes<32>(join_lanes<16>(join_lanes<8>(join_lanes<4>(join_lanes<2>(join_lanes<1>(s))))));
  sum += lane_xor_f<1>(sum);
  sum += lane_xor_f<2>(sum);
  sum += lane_xor_f<4>(sum);
  sum += lane_xor_f<8>(sum);
  sum += lane_xor_f<16>(sum);
  sum += lane_xor_f<32>(sum);
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = make_float4(s.top, s.rest, sum, 0.0f);
  __syncthreads();
  if (thread == 0) {
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      const float4 b = waves[row * 4 + i];
      s = join(s, Soft{b.x, b.y});
      sum += b.z;
    }
  }
  if (p.slots == 1) {
    float loss = 0.0f;
    bool counts = false;
    if (thread == 0) loss = finish_row(o, m, s, sum, found, counts);
    if (o.mean) mean_of(o.mean, double(loss), counts);
    return;
  }
  if (thread) return;
  p.pairs[slot * o.M + m] = s;
  if (p.sums) p.sums[slot * o.M + m] = sum;
  if (t >= n0 && t < end) p.at[m] = found;
}

__global__ void __launch_bounds__(1024) k_loss_mean(const float *loss, const int64_t *target, int64_t ignore, int64_t M, float *mean) {
  double sum = 0.0;
  int64_t count = 0;
#pragma unroll 4
  for (int64_t m = threadIdx.x; m < M; m += 1024) {
    // (a row that is left out has loss 0)
    sum += loss[m];
    count += target[m] != ignore;
  }
  mean_of(mean, sum, count);
}

// ----------------------------------------------------------------------------- log p of the targets
// dz at a target that is nearly certain is p - 1: a float32 z is off by 2^-24 |z| a rounding, which is then left alone
// (10 classes, losses of 1e-5: wrong in the second digit).  The forward leaves log p; where it is not given, z of the targets, M
// of the M x N, is summed in float64, a wave a row, and its difference from lse rounded once.  Bound by reading x again and M
// rows of w: 4608 x 65536 x 4096 bf16 in 17 us of 5700, 777 x 10007 x 513 e4m3 in 4.7 (its launch) of 79; beside the tiles of a
// split contraction it takes 0.3 us (64 x 1000 x 4096: 20.3 a call without it, 20.6 with it).

struct Targets {
  const void *x, *w;
  const float *sx, *sw, *bias, *lse;
  const int64_t *target;
  int64_t M, N, K, ldx, ldw, ignore;
  float *logp;             // [M]
  int32_t dtype;
};
// The sum of the products that a lane has of two rows: of pieces of 16 bytes, and the elements behind them.  Exact for int8 (K
// <= 133144), float64 for the others, whose products float32 holds exactly.
template <int DTYPE>
__device__ __forceinline__ double dot_rows(const void *xp, const void *wp, int64_t K) {
  typedef std::conditional_t<DTYPE == FQT_BF16, uint16_t, uint8_t> Bits;
  constexpr int V = 16 / sizeof(Bits);
  const Bits *x = static_cast<const Bits *>(xp), *w = static_cast<const Bits *>(wp);
  std::conditional_t<DTYPE == FQT_I8, int, double> sum = 0;
  auto add = [&](uint32_t a, uint32_t b) {               // the elements of a word of each
    if constexpr (DTYPE == FQT_BF16) {
      sum += double(__uint_as_float(a << 16) * __uint_as_float(b << 16));
      sum += double(__uint_as_float(a & 0xFFFF0000u) * __uint_as_float(b & 0xFFFF0000u));
    } else if constexpr (DTYPE == FQT_I8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += int(int8_t(a >> (8 * i))) * int(int8_t(b >> (8 * i)));
    } else {
      sum += double(__builtin_amdgcn_cvt_f32_fp8(int(a), 0) * __builtin_amdgcn_cvt_f32_fp8(int(b), 0));
      sum += double(__builtin_amdgcn_cvt_f32_fp8(int(a), 1) * __builtin_amdgcn_cvt_f32_fp8(int(b), 1));
      sum += double(__builtin_amdgcn_cvt_f32_fp8(int(a), 2) * __builtin_amdgcn_cvt_f32_fp8(int(b), 2));
      sum += double(__builtin_amdgcn_cvt_f32_fp8(int(a), 3) * __builtin_amdgcn_cvt_f32_fp8(int(b), 3));
    }
  };
  const int64_t pieces = K / V;
#pragma unroll 4
  for (int64_t i = __lane_id(); i < pieces; i += 64) {
    const u32x4 a = load_bytes16(x + i * V), b = load_bytes16(w + i * V);
#pragma unroll
    for (int j = 0; j < 4; ++j) add(a[j], b[j]);
  }
  if (const int64_t k = pieces * V + __lane_id(); k < K) add(x[k], w[k]);      // (zeros above)
  return double(sum);
}
// The rows of wave `wave` of `waves`.
__device__ __forceinline__ void target_rows(const Targets &a, int64_t wave, int64_t waves) {
  const int64_t e = a.dtype == FQT_BF16 ? 2 : 1;
  for (int64_t m = wave; m < a.M; m += waves) {
    const int64_t t = a.target[m];
    double z = 0.0;
    const bool counts = t != a.ignore && t >= 0 && t < a.N;
    if (counts) {
      const void *x = static_cast<const char *>(a.x) + m * a.ldx * e, *w = static_cast<const char *>(a.w) + t * a.ldw * e;
      if (a.dtype == FQT_BF16) z = dot_rows<FQT_BF16>(x, w, a.K);
      else if (a.dtype == FQT_I8) z = dot_rows<FQT_I8>(x, w, a.K);
      else z = dot_rows<FQT_E4M3>(x, w, a.K);
#pragma unroll
      for (int o = 32; o > 0; o /= 2) z += __shfl_xor(z, o);
      if (a.sx) z *= double(a.sx[m]) * double(a.sw[t]);
      if (a.bias) z += double(a.bias[t]);
      z -= double(a.lse[m]);
    }
    if (__lane_id() == 0) a.logp[m] = float(z);
  }
}
__global__ void __launch_bounds__(256) k_loss_targets(Targets a) {
  target_rows(a, int64_t(blockIdx.x) * 4 + wave_id(), int64_t(gridDim.x) * 4);
}

// ----------------------------------------------------------------------------- dz

constexpr float LIKELY = -LN2;     // log p of a target from which on dz comes from expm1
struct DzOut {
  const float *lse, *logp, *dloss, *dmean, *mean;
  const int64_t *target;
  int64_t ignore, classes, first;  // all classes; the piece's first
  float keep, even;                // 1 - smoothing, smoothing / classes
  float rise;                      // smoothing - smoothing / classes
  bf16 *dzx, *dzw;                 // dz sw and dz sx, rows of `pitch` (one array for bf16 operands); or null
  int64_t pitch;
  float *part;                     // [ceil(M / unit)][N] partial column sums, or null
  int32_t unit;
};
// The epilogue of 8 consecutive classes (tile::run_epilogue).
struct StoreDz {
  static constexpr int DEPTH = 4;
  static constexpr bool MIRROR = false, SUMS = false;
  struct Fetch {
    float lse, logp, c, sx;
    int32_t t;             // the target's place from n on; -1: not there, -2: the row is left out
  };
  const Logits &p;
  const DzOut &o;
  float sw[8], bias[8], sum[8], each;
  int cnt;
  __device__ __forceinline__ StoreDz(const Logits &p_, const DzOut &o_) : p(p_), o(o_) {
    each = o.dmean ? o.dmean[0] * o.mean[1] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.0f;
  }
  __device__ __forceinline__ void columns(int64_t n) {
    cnt = int(max(int64_t(0), min(p.N - n, int64_t(8))));
#pragma unroll
    for (int i = 0; i < 8; ++i) sw[i] = 1.0f, bias[i] = 0.0f;
    if (p.sw) load8f(p.sw + n, cnt, sw);
    if (p.bias) load8f(p.bias + n, cnt, bias);
  }
  __device__ __forceinline__ Fetch fetch(int64_t m, int64_t n) {
    Fetch f{};
    if (m >= p.M || cnt == 0) return f;
    const int64_t t = o.target[m];
    f.lse = o.lse[m];
    f.logp = o.logp[m];
    f.c = o.dloss ? o.dloss[m] : each;
    f.sx = p.sx ? p.sx[m] : 1.0f;
    const int64_t d = t - o.first - n;
    if (t == o.ignore) f.t = -2;
    else if (t < 0 || t >= o.classes) f.t = -1, f.c = __builtin_nanf("");
    else f.t = d >= 0 && d < 8 ? int(d) : -1;
    return f;
  }
  __device__ __forceinline__ void finish(int64_t m, int64_t n, float (&v)[8], const Fetch &f) {
    if (m >= p.M || cnt == 0) return;
    // (what few rows or launches need stands behind branches: a group of 8 takes 100 issue slots of the 160 that
    // it took with selects for all of it)
    if (p.sx) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = v[i] * f.sx * sw[i];
    }
    if (p.bias) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += bias[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = exp_of(v[i] - f.lse);
    if (o.even != 0.0f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] -= o.even;
    }
    if (f.t >= 0) {
      // p - 1 of a likely target without cancellation (an unlikely one's p counts where labels are smoothed)
      const bool likely = f.logp > LIKELY;
      const float own = expm1f(f.logp) + o.rise;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = f.t != i ? v[i] : likely ? own : v[i] - o.keep;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= f.c;
    if (f.t == -2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.0f;
    }
    if (cnt < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < cnt ? v[i] : 0.0f;
    }
    if (o.part) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[i] += v[i];
    }
    if (!p.sx) {
      if (o.dzx) store8f(o.dzx + m * o.pitch + n, 8, v);
      return;
    }
    float u[8];
    if (o.dzx) {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = v[i] * sw[i];
      store8f(o.dzx + m * o.pitch + n, 8, u);
    }
    if (o.dzw) {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = v[i] * f.sx;
      store8f(o.dzw + m * o.pitch + n, 8, u);
    }
  }
};
// dz of a piece of the classes; its row pitch is a multiple of 8, zeros past the piece.
// With a split contraction, whose join makes dz, the workgroups behind the `tiles` that compute z take the targets.
template <int KIND, int SHAPE>
__global__ void __launch_bounds__(tile::ShapeOf<SHAPE>::type::THREADS, 2) k_loss_dz(Logits p, DzOut o, Targets a, uint32_t tiles) {
  typedef typename tile::ShapeOf<SHAPE>::type S;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];
  if (blockIdx.x >= tiles) {
    constexpr int WAVES = S::THREADS / 64;
    target_rows(a, int64_t(blockIdx.x - tiles) * WAVES + wave_id(), int64_t(gridDim.x - tiles) * WAVES);
    return;
  }
  const tile::Place at = tile::place<SHAPE>(p.tiles, blockIdx.x);
  if (at.m0 >= p.M || at.n0 >= p.N) return;              // (parts of an edge tile)
  typename tile::Acc<KIND>::type acc[S::FM][S::FN];
  tile::contract<KIND, ROWS, ROWS, SHAPE, S>(p.x, p.w, p.K, at, p.tiles, lds, acc);
  if (p.tiles.splits > 1) {
    tile::run_epilogue<KIND, S>(acc, lds, at.m0, at.n0, tile::StorePart{p.part + at.split * p.M * p.ldp, p.M, p.ldp});
    return;
  }
  StoreDz e(p, o);
  tile::run_epilogue<KIND, S>(acc, lds, at.m0, at.n0, e);
  if (!o.part) return;
  // A lane has the sums of its 8 columns over every (512 / TN)th row of the wave.
  constexpr int PER_ROW = S::TN / 8;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (PER_ROW == 4) e.sum[i] += lane_xor_f<4>(e.sum[i]);
    e.sum[i] += lane_xor_f<8>(e.sum[i]);
    e.sum[i] += lane_xor_f<16>(e.sum[i]);
    e.sum[i] += lane_xor_f<32>(e.sum[i]);
  }
  const uint32_t wave = wave_id(), l = __lane_id();
  const int64_t m = at.m0 + (wave / S::WN) * S::TM, n = at.n0 + (wave % S::WN) * S::TN + l * 8;
  if (l >= PER_ROW || m >= p.M) return;
  // (the launch's other tiles may be smaller: a part for each `unit` rows, the first of them has the sum)
  for (int64_t u = m / o.unit; u * o.unit < min(m + S::TM, p.M); ++u) {
    store8f(o.part + u * p.N + n, e.cnt, e.sum);
#pragma unroll
    for (int i = 0; i < 8; ++i) e.sum[i] = 0.0f;
  }
}

// dz from the partial sums of a split contraction: a thread takes 8 columns, a wave every fourth row of the
// workgroup's `unit`.
template <bool INTS>
__global__ void __launch_bounds__(256) k_loss_dz_join(Logits p, DzOut o, uint32_t groups) {
  __shared__ float sums[3][8][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t u = blockIdx.x % groups, n = (int64_t(blockIdx.x / groups) * 64 + lane) * 8;
  StoreDz e(p, o);
  e.columns(n);
  if (e.cnt)
    for (int64_t m = u * o.unit + wave; m < min(p.M, (u + 1) * o.unit); m += 4) {
      const auto f = e.fetch(m, n);
      std::conditional_t<INTS, int, float> w[8] = {};
#pragma unroll 4
      for (uint32_t s = 0; s < p.tiles.splits; ++s) {
        float t[8];
        load8f(p.part + (s * p.M + m) * p.ldp + n, 8, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (INTS) w[i] += __float_as_int(t[i]);
          else w[i] += t[i];
        }
      }
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = float(w[i]);
      e.finish(m, n, v, f);
    }
  if (!o.part) return;
  if (wave)
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[wave - 1][i][lane] = e.sum[i];
  __syncthreads();
  if (wave || !e.cnt) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) e.sum[i] = ((e.sum[i] + sums[0][i][lane]) + sums[1][i][lane]) + sums[2][i][lane];
  store8f(o.part + u * p.N + n, e.cnt, e.sum);
}

// ----------------------------------------------------------------------------- host side

struct Sizes {
  int64_t M, N, K;
  int64_t ldx, ldw, lddx, lddw;
  size_t xe;
  bool codes;
};
int check_loss(const fqt_loss_desc *d, Sizes *s) {
  if (!d) return FQT_E_NULL;
  if (!(d->x_dtype == FQT_BF16 || code_type(d->x_dtype)) || !float_type(d->dx_dtype) || !float_type(d->dw_dtype))
    return FQT_E_DTYPE;
  if (!(d->smoothing >= 0.0f && d->smoothing <= 1.0f)) return FQT_E_INVAL;
  if (d->M < 0 || d->N < 1 || d->K < 0 || d->M >= FQT_MAX_ROWS || d->N > FQT_MAX_LD || d->K > FQT_MAX_LD)
    return FQT_E_SHAPE;
  // (a launch counts its threads in 32 bits)
  for (const uint64_t tiles : {tile::large_tiles(d->M, d->N), tile::large_tiles(d->M, d->K), tile::large_tiles(d->N, d->K)})
    if (tiles >= tile::MOST_LARGE) return FQT_E_SHAPE;
  if (d->x_dtype == FQT_I8 && d->K > 133144) return FQT_E_SHAPE;   // 127^2 K < 2^31
  *s = {d->M, d->N, d->K, row_stride(d->ldx, d->K), row_stride(d->ldw, d->K), row_stride(d->lddx, d->K),
        row_stride(d->lddw, d->K), elem_size(d->x_dtype), code_type(d->x_dtype)};
  if (!s->ldx || !s->ldw || !s->lddx || !s->lddw) return FQT_E_SHAPE;
  return FQT_OK;
}
int check_pointers(const fqt_loss_desc &d, const Sizes &s, const void *x, const void *w, const float *sx,
                   const float *sw, const float *bias, const int64_t *target) {
  if (!s.codes && (sx || sw)) return FQT_E_DTYPE;
  if (s.M && (!target || (s.K && (!x || !w)) || (s.codes && (!sx || !sw)))) return FQT_E_NULL;
  if (!aligned(x, 16) || !aligned(w, 16) || !aligned(sx, 4) || !aligned(sw, 4) || !aligned(bias, 4) ||
      !aligned(target, 8))
    return FQT_E_ALIGN;
  return FQT_OK;
}

// us a step and before and after the steps of widened codes (as tile::STEP_COSTS).
constexpr tile::Costs WIDE_COSTS{{2.5}, {1.1, 1.6}, {0.35, 0.55, 0.85}, {6, 5, 4}};

// z's plan, from codes themselves (direct) or operands of 16 bits.
tile::Plan plan_z(int32_t dtype, bool direct, int64_t M, int64_t n, int64_t K) {
  if (direct && dtype == FQT_E4M3) return tile::make_plan(M, n, (K + tile::KB - 1) / tile::KB, false, WIDE_COSTS);
  return plan_of(M, n, K, direct ? 1 : 2, tile::STEP_COSTS);
}

// Workspace of the forward: copies of operands whose rows are not whole 16-byte pieces,
// z of few rows or partial sums, and pairs, sums and the targets' z.
struct FwdWs { size_t x, w, part, pairs, sums, at, total; int64_t pitch, e, slots; tile::Plan plan; bool few, copy_x, copy_w; };
FwdWs fwd_ws(const fqt_loss_desc &d, const Sizes &s) {
  FwdWs f{};
  // z of few rows is written to the workspace by fqt_linear_forward: its bytes are few beside those of w
  f.few = s.M <= FEW_MOST;
  auto pairs = [&](size_t from, int64_t slots) {
    f.slots = slots;
    f.pairs = from;
    f.sums = f.pairs + align256(size_t(slots) * s.M * sizeof(Soft));
    f.at = f.sums + (d.smoothing > 0.0f ? align256(size_t(slots) * s.M * 4) : 0);
    f.total = f.at + align256(size_t(s.M) * 4);
  };
  const int64_t chunks = (s.N + CHUNK - 1) / CHUNK;
  if (f.few) {
    pairs(align256(size_t(s.M) * s.N * 4), chunks);
    return f;
  }
  f.e = int64_t(s.xe);
  f.pitch = round_up(s.K, 16 / f.e);
  f.copy_x = !whole_pieces(s.K, s.ldx, s.xe);
  f.copy_w = !whole_pieces(s.K, s.ldw, s.xe);
  f.plan = plan_z(d.x_dtype, s.codes, s.M, s.N, s.K);
  f.w = f.x + (f.copy_x ? align256(size_t(s.M) * f.pitch * f.e) : 0);
  f.part = f.w + (f.copy_w ? align256(size_t(s.N) * f.pitch * f.e) : 0);
  if (f.plan.splits > 1) pairs(f.part + part_bytes(f.plan, s.M, s.N), chunks);
  else pairs(f.part, (s.N + SLOT - 1) / SLOT);
  return f;
}

// The classes of a piece of the backward: dz in bf16 of a piece takes about PIECE_BYTES, but a piece has PIECE_LEAST
// classes at least, up to a quarter more where these are all: past 32768 rows (16384 of codes, which have dz twice) dz grows with the
// rows, 131072 x 65536 takes 1.1 GB (2.2 GB of codes).  (Each
// piece reads and writes a float32 dx, 8 M K bytes, beside the 4 M n of its dz.)
constexpr int64_t PIECE_BYTES = int64_t(256) << 20, PIECE_LEAST = 4096;
int64_t piece_of(const Sizes &s) {
  const int64_t most = std::max(PIECE_LEAST, PIECE_BYTES / std::max<int64_t>(1, s.M * (s.codes ? 4 : 2)));
  if (s.N <= most + most / 4) return s.N;
  const int64_t pieces = (s.N + most - 1) / most;
  return std::min(s.N, round_up((s.N + pieces - 1) / pieces, 256));
}

int64_t dz_pitch_of(int64_t n) { return n <= 512 ? round_up(n, 8) : (round_up(n, 64) / 64 | 1) * 64; }

// Workspace of the backward: dz of a piece (twice for scaled operands), bf16 copies of operands that are codes
// or whose rows are not whole pieces (w: of a piece), dx in float32 where several pieces add up to it,
// the partial sums of dbias and those of the products.
struct PiecePlan { tile::Plan z, dx, dw; int64_t unit; Together together; };
struct BwdWs {
  size_t dzx, dzw, x, w, dx, logp, bias, part, total;
  int64_t piece, dz_pitch, pitch, K;
  bool copy_x, copy_w, direct, sum_dx;
  PiecePlan plan[2];       // of the pieces, of the last one
};
PiecePlan plan_piece(const fqt_loss_desc &d, const Sizes &s, int64_t n, const BwdWs &f) {
  PiecePlan p{};
  p.z = plan_z(d.x_dtype, f.direct, s.M, n, f.K);
  p.dx = plan_of(s.M, s.K, n, 2, tile::STEP_COSTS);
  p.dw = plan_of(n, s.K, s.M, 2, tile::STEP_COSTS);
  p.together = plan_together(s.M, n, s.K, p.dx, p.dw);
  p.unit = 128;            // rows of a wave's results: the fewest of the launches
  for (int i = 0; i < p.z.launches; ++i)
    p.unit = std::min<int64_t>(p.unit, p.z.shape[i] == tile::LARGE ? 128 : p.z.shape[i] == tile::MIDDLE ? 64 : 32);
  // (of a joining workgroup: enough of them, few partial sums)
  if (p.z.splits > 1) p.unit = std::max<int64_t>(4, (s.M + 127) / 128);
  return p;
}
BwdWs bwd_ws(const fqt_loss_desc &d, const Sizes &s) {
  BwdWs f{};
  f.piece = piece_of(s);
  f.dz_pitch = dz_pitch_of(f.piece);
  f.pitch = round_up(s.K, 8);
  f.copy_x = s.codes || !whole_pieces(s.K, s.ldx, 2);
  f.copy_w = s.codes || !whole_pieces(s.K, s.ldw, 2);
  // z comes from the codes themselves where their rows are whole pieces: half the bytes, and int8's matrix rate
  // (4608 x 32768 x 4096 int8: 2970 -> 2740 us)
  f.direct = s.codes && whole_pieces(s.K, s.ldx, 1) && whole_pieces(s.K, s.ldw, 1);
  f.K = !f.direct && (f.copy_x || f.copy_w) ? f.pitch : s.K;
  f.sum_dx = f.piece < s.N && d.dx_dtype != FQT_F32;
  const size_t dz = align256(size_t(s.M) * f.dz_pitch * 2);
  f.dzw = f.dzx + (s.codes ? dz : 0);
  f.x = f.dzw + dz;
  f.w = f.x + (f.copy_x ? align256(size_t(s.M) * f.pitch * 2) : 0);
  f.dx = f.w + (f.copy_w ? align256(size_t(f.piece) * f.pitch * 2) : 0);
  f.logp = f.dx + (f.sum_dx ? align256(size_t(s.M) * s.K * 4) : 0);
  f.bias = f.logp + align256(size_t(s.M) * 4);
  size_t part = 0, groups = 1;
  for (int i = 0; i < 2; ++i) {
    const int64_t n = i && s.N % f.piece ? s.N % f.piece : f.piece;
    // (a plan costs the host 2.5 us)
    const PiecePlan &p = f.plan[i] = i && n == f.piece ? f.plan[0] : plan_piece(d, s, n, f);
    part = std::max({part, part_bytes(p.z, s.M, n), part_bytes(p.dx, s.M, s.K), part_bytes(p.dw, n, s.K),
                     part_bytes(p.together, s.M, n, s.K)});
    groups = std::max(groups, size_t((s.M + p.unit - 1) / p.unit));
  }
  f.part = f.bias + align256(groups * f.piece * 4);
  f.total = f.part + part;
  return f;
}

template <int KIND>
int launch_logits(const tile::Plan &plan, Logits p, const Pairs &o, hipStream_t st) {
  tile::for_launches(plan, [&]<int SHAPE>(const tile::Tiles &t) {
    p.tiles = t;
    const dim3 grid(uint32_t(tile::blocks_of(t))), block(tile::ShapeOf<SHAPE>::type::THREADS);
    if (o.sums) k_loss_tiles<KIND, true, SHAPE><<<grid, block, 0, st>>>(p, o);
    else k_loss_tiles<KIND, false, SHAPE><<<grid, block, 0, st>>>(p, o);
  });
  return last_launch_status();
}
// Workgroups of `waves` waves for the targets of M rows; they walk where the rows are more.
uint32_t target_blocks(int64_t M, int64_t waves) { return uint32_t(std::min<int64_t>((M + waves - 1) / waves, 1 << 14)); }
// a: null where o.logp is there already.
template <int KIND>
int launch_dz(const PiecePlan &plan, Logits p, const DzOut &o, const Targets *a, hipStream_t st) {
  const bool beside = a && plan.z.splits > 1;
  if (a && !beside) k_loss_targets<<<dim3(target_blocks(a->M, 4)), dim3(256), 0, st>>>(*a);
  tile::for_launches(plan.z, [&]<int SHAPE>(const tile::Tiles &t) {
    p.tiles = t;
    constexpr int THREADS = tile::ShapeOf<SHAPE>::type::THREADS;
    const uint32_t tiles = uint32_t(tile::blocks_of(t)), more = beside ? target_blocks(a->M, THREADS / 64) : 0;
    k_loss_dz<KIND, SHAPE><<<dim3(tiles + more), dim3(THREADS), 0, st>>>(p, o, a ? *a : Targets{}, tiles);
  });
  if (plan.z.splits > 1) {
    const uint32_t groups = uint32_t((p.M + plan.unit - 1) / plan.unit);
    k_loss_dz_join<KIND == tile::I8K><<<dim3(groups * uint32_t((p.N + 511) / 512)), dim3(256), 0, st>>>(p, o, groups);
  }
  return last_launch_status();
}
// z in the workspace to pairs, or to the losses where a chunk is a row; few: all rows by one workgroup then, and the
// mean, if it is asked for.
int launch_dense(const RowArgs &a, const Pairs &p, Out o, bool ints, bool few, float *mean, hipStream_t st) {
  few = few && p.slots == 1;
  if (few) o.mean = mean;
  const dim3 grid(few ? 1u : uint32_t(o.M * p.slots)), block(few ? uint32_t(256 * o.M) : 256);
  if (ints) k_loss_dense<true><<<grid, block, 0, st>>>(a, p, o);
  else k_loss_dense<false><<<grid, block, 0, st>>>(a, p, o);
  return last_launch_status();
}
// Whether one workgroup takes all rows' pairs, 32 each at most.
bool one_group(const Pairs &p, int64_t M) { return M <= 1024 && M * p.slots <= 32768; }
// Pairs to the losses, and the mean where one workgroup has all rows.
int launch_rows(const Pairs &p, Out o, float *mean, hipStream_t st) {
  if (mean && one_group(p, o.M)) {
    uint32_t rows = 16;
    while (rows < o.M) rows *= 2;
    o.mean = mean;
    k_loss_rows_mean<<<dim3(1), dim3(1024), 0, st>>>(p, o, rows);
  } else {
    // (a launch counts its threads in 32 bits)
    k_loss_rows<<<dim3(uint32_t(std::min<int64_t>((o.M + 15) / 16, 1 << 16))), dim3(256), 0, st>>>(p, o);
  }
  return last_launch_status();
}

}  // namespace
}  // namespace dense
}  // namespace fqt

using namespace fqt;
using namespace fqt::dense;

extern "C" int fqt_loss_workspace_size(const fqt_loss_desc *d, int32_t backward, size_t *bytes) {
  Sizes s;
  FQT_TRY_(check_loss(d, &s));
  if (!bytes) return FQT_E_NULL;
  *bytes = std::max<size_t>(256, backward ? bwd_ws(*d, s).total : fwd_ws(*d, s).total);
  return FQT_OK;
}

extern "C" int fqt_loss_forward(const fqt_loss_desc *d, const void *x, const void *w, const float *x_scale,
                                const float *w_scale, const float *bias, const int64_t *target, float *loss,
                                float *lse, float *mean, void *ws, size_t ws_bytes, void *hip_stream) {
  return fqt_loss_forward_logp(d, x, w, x_scale, w_scale, bias, target, loss, lse, nullptr, mean, ws, ws_bytes, hip_stream);
}

extern "C" int fqt_loss_forward_logp(const fqt_loss_desc *d, const void *x, const void *w, const float *x_scale,
                                     const float *w_scale, const float *bias, const int64_t *target, float *loss,
                                     float *lse, float *logp, float *mean, void *ws, size_t ws_bytes,
                                     void *hip_stream) {
  Sizes s;
  FQT_TRY_(check_loss(d, &s));
  FQT_TRY_(check_pointers(*d, s, x, w, x_scale, w_scale, bias, target));
  if (!ws || (s.M && (!loss || !lse))) return FQT_E_NULL;
  if (!aligned(loss, 4) || !aligned(lse, 4) || !aligned(logp, 4) || !aligned(mean, 4) || !aligned(ws, 256))
    return FQT_E_ALIGN;
  const FwdWs f = fwd_ws(*d, s);
  if (ws_bytes < f.total) return FQT_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  char *base = static_cast<char *>(ws);
  const Out o{target, loss, lse, s.M, s.N, d->ignore, d->smoothing, nullptr, logp};
  bool averaged = false;
  const Pairs pairs{reinterpret_cast<Soft *>(base + f.pairs),
                    d->smoothing > 0.0f ? reinterpret_cast<float *>(base + f.sums) : nullptr,
                    reinterpret_cast<float *>(base + f.at), target, f.slots};
  if (s.M && f.few) {
    fqt_linear_desc l{};
    l.M = s.M; l.N = s.N; l.K = s.K;
    l.ldx = s.ldx; l.ldw = s.ldw;
    l.x_dtype = d->x_dtype;
    l.y_dtype = l.dx_dtype = l.dw_dtype = FQT_F32;
    float *z = reinterpret_cast<float *>(base);
    FQT_TRY_(fqt_linear_forward(&l, x, w, x_scale, w_scale, bias, nullptr, nullptr, z, ws, ws_bytes, hip_stream));
    FQT_TRY_(launch_dense({z, nullptr, nullptr, nullptr, s.N, 1}, pairs, o, false, true, mean, st));
    averaged = f.slots == 1 || one_group(pairs, s.M);
    if (f.slots > 1) FQT_TRY_(launch_rows(pairs, o, mean, st));
  } else if (s.M) {
    Copy cx{}, cw{};
    auto operand = [&](const void *p, bool copy, size_t at, int64_t rows, int64_t ld, Copy *c) -> Operand {
      if (!copy) return {static_cast<const char *>(p), ld * f.e, rows};
      *c = copy_of(p, rows, s.K, ld, base + at, f.pitch, f.e);
      return {base + at, f.pitch * f.e, rows};
    };
    const Operand xo = operand(x, f.copy_x, f.x, s.M, s.ldx, &cx), wo = operand(w, f.copy_w, f.w, s.N, s.ldw, &cw);
    FQT_TRY_(launch_copies(cx, cw, d->x_dtype, false, st));
    const Logits p{xo, wo, s.M, s.N, f.copy_x || f.copy_w ? f.pitch : s.K, f.plan.t[0], x_scale, w_scale, bias,
                   reinterpret_cast<float *>(base + f.part), round_up(s.N, 8)};
    const bool ints = d->x_dtype == FQT_I8;
    if (ints) FQT_TRY_(launch_logits<tile::I8K>(f.plan, p, pairs, st));
    else if (s.codes) FQT_TRY_(launch_logits<tile::WIDEK>(f.plan, p, pairs, st));
    else FQT_TRY_(launch_logits<tile::BF16K>(f.plan, p, pairs, st));
    if (f.plan.splits > 1) FQT_TRY_(launch_dense({p.part, x_scale, w_scale, bias, p.ldp, f.plan.splits}, pairs, o, ints, false, nullptr, st));
    if (f.plan.splits == 1 || f.slots > 1) {
      averaged = one_group(pairs, s.M);
      FQT_TRY_(launch_rows(pairs, o, mean, st));
    }
  }
  if (!mean || averaged) return FQT_OK;
  k_loss_mean<<<dim3(1), dim3(1024), 0, st>>>(loss, target, d->ignore, s.M, mean);
  return last_launch_status();
}

extern "C" int fqt_loss_backward(const fqt_loss_desc *d, const void *x, const void *w, const float *x_scale,
                                 const float *w_scale, const float *bias, const int64_t *target, const float *lse,
                                 const float *dloss, const float *dmean, const float *mean, void *dx, void *dw,
                                 float *dbias, void *ws, size_t ws_bytes, void *hip_stream) {
  return fqt_loss_backward_logp(d, x, w, x_scale, w_scale, bias, target, lse, nullptr, dloss, dmean, mean, dx, dw,
                                dbias, ws, ws_bytes, hip_stream);
}

extern "C" int fqt_loss_backward_logp(const fqt_loss_desc *d, const void *x, const void *w, const float *x_scale,
                                      const float *w_scale, const float *bias, const int64_t *target,
                                      const float *lse, const float *logp, const float *dloss, const float *dmean,
                                      const float *mean, void *dx, void *dw, float *dbias, void *ws, size_t ws_bytes,
                                      void *hip_stream) {
  Sizes s;
  FQT_TRY_(check_loss(d, &s));
  FQT_TRY_(check_pointers(*d, s, x, w, x_scale, w_scale, bias, target));
  if ((dloss && dmean) || (!dmean) != (!mean)) return FQT_E_INVAL;
  if (!dx && !dw && !dbias) return FQT_OK;
  if (!ws || (s.M && (!lse || (!dloss && !dmean)))) return FQT_E_NULL;
  if (!aligned(lse, 4) || !aligned(logp, 4) || !aligned(dloss, 4) || !aligned(dmean, 4) || !aligned(mean, 4) ||
      !elem_aligned(dx, d->dx_dtype) || !elem_aligned(dw, d->dw_dtype) || !aligned(dbias, 4) || !aligned(ws, 256))
    return FQT_E_ALIGN;
  const BwdWs f = bwd_ws(*d, s);
  if (ws_bytes < f.total) return FQT_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (s.M == 0) {          // sums over nothing
    if (dw) FQT_TRY_(zero_matrix(dw, s.N, s.K, s.lddw, elem_size(d->dw_dtype), st));
    if (dbias) FQT_TRY_(zero_matrix(dbias, 1, s.N, s.N, 4, st));
    return FQT_OK;
  }
  char *base = static_cast<char *>(ws);
  for (int64_t first = 0; first < s.N; first += f.piece) {
    const int64_t n = std::min(f.piece, s.N - first), dz_pitch = dz_pitch_of(n);
    const PiecePlan &plan = f.plan[n != f.piece];
    // The operands along k (for z) and along the features (for the gradients).
    Copy cx{}, cw{};
    Operand xr{static_cast<const char *>(x), s.ldx * 2, s.M};
    Operand wr{static_cast<const char *>(w) + first * s.ldw * int64_t(s.xe), s.ldw * 2, n};
    if (f.copy_x) {
      if (first == 0) cx = copy_of(x, s.M, s.K, s.ldx, base + f.x, f.pitch, 2);
      xr = {base + f.x, f.pitch * 2, s.M};
    }
    if (f.copy_w) {
      cw = copy_of(wr.p, n, s.K, s.ldw, base + f.w, f.pitch, 2);
      wr = {base + f.w, f.pitch * 2, n};
    }
    FQT_TRY_(launch_copies(cx, cw, d->x_dtype, s.codes, st));
    const Operand xz{static_cast<const char *>(x), s.ldx, s.M}, wz{static_cast<const char *>(w) + first * s.ldw, s.ldw, n};
    Logits p{f.direct ? xz : xr, f.direct ? wz : wr, s.M, n, f.K, {}, x_scale, w_scale ? w_scale + first : nullptr, bias ? bias + first : nullptr,
             reinterpret_cast<float *>(base + f.part), round_up(n, 8)};
    const Targets targets{x, w, x_scale, w_scale, bias, lse, target, s.M, s.N, s.K, s.ldx, s.ldw, d->ignore,
                          reinterpret_cast<float *>(base + f.logp), d->x_dtype};
    const Targets *const a = first || logp ? nullptr : &targets;
    DzOut o{lse, logp ? logp : targets.logp, dloss, dmean, mean, target, d->ignore, s.N, first, 1.0f - d->smoothing,
            d->smoothing / float(s.N), d->smoothing - d->smoothing / float(s.N),
            reinterpret_cast<bf16 *>(base + f.dzx), reinterpret_cast<bf16 *>(base + f.dzw), dz_pitch,
            dbias ? reinterpret_cast<float *>(base + f.bias) : nullptr, int32_t(plan.unit)};
    if (!dx && (s.codes || !dw)) o.dzx = nullptr;
    if (!dw) o.dzw = nullptr;
    if (f.direct && d->x_dtype == FQT_I8) FQT_TRY_(launch_dz<tile::I8K>(plan, p, o, a, st));
    else if (f.direct) FQT_TRY_(launch_dz<tile::WIDEK>(plan, p, o, a, st));
    else FQT_TRY_(launch_dz<tile::BF16K>(plan, p, o, a, st));
    Gradients g{};
    g.M = s.M; g.N = n; g.K = s.K;
    g.dzx = {base + f.dzx, dz_pitch * 2, s.M};
    g.dzw = {base + f.dzw, dz_pitch * 2, round_up(n, 8)};
    g.w = {wr.p, wr.ld, f.copy_w ? f.pitch : s.K};
    g.x = {xr.p, xr.ld, f.copy_x ? f.pitch : s.K};
    g.plan_dx = plan.dx; g.plan_dw = plan.dw;
    if (dx) {
      // dx adds up in float32: in place, or in the workspace until the last piece
      const bool last = first + n == s.N || !f.sum_dx;
      float *acc = f.sum_dx ? reinterpret_cast<float *>(base + f.dx) : static_cast<float *>(dx);
      const int64_t ldacc = f.sum_dx ? std::max<int64_t>(1, s.K) : s.lddx;
      g.dx = last ? dx : acc;
      g.lddx = last ? s.lddx : ldacc;
      g.dx_dtype = last ? d->dx_dtype : FQT_F32;
      if (first) g.add = acc, g.ldadd = ldacc;
    }
    if (dw) g.dw = static_cast<char *>(dw) + first * s.lddw * int64_t(elem_size(d->dw_dtype));
    g.lddw = s.lddw;
    g.dw_dtype = d->dw_dtype;
    g.part = reinterpret_cast<float *>(base + f.part);
    g.together = plan.together;
    if (dbias) g.bias = {o.part, dbias + first, n, int32_t((s.M + plan.unit - 1) / plan.unit)};
    FQT_TRY_(launch_gradients(g, st));
  }
  return FQT_OK;
}
