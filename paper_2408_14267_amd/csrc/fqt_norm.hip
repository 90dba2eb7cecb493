// RMS norm of a residual sum with 8-bit output, its backward pass, and the row quantiser.
//
// The forward reads each row once: the row stays in registers while the sum of its squares and the
// maximum of |h g| are reduced together (|y| = rstd |h g|, so the scale needs no second sweep).
// The backward keeps h and dy of a row in registers for its one reduction, and each thread adds
// dy t of its own columns over all rows of its workgroup, so that dg costs one partial row per
// workgroup.  Both are bound by memory traffic.
#include "fqt_dense.hpp"

namespace fqt {
namespace dense {
namespace {

#pragma clang fp contract(fast)

struct NormArgs {
  const void *x, *r;
  const float *g;
  void *h, *y;
  uint8_t *q;
  float *scale, *rstd;
  int64_t rows;
  int32_t cols;
  int64_t ldx, ldr, ldh, ldy, ldq;
  int32_t q_dtype;
  float eps;
  int32_t norm;        // 0: the row quantiser (y = x)
};

__device__ __forceinline__ float wave_sum(float v) {
  v += lane_xor_f<1>(v);
  v += lane_xor_f<2>(v);
  v += lane_xor_f<4>(v);
  v += lane_xor_f<8>(v);
  v += lane_xor_f<16>(v);
  return v + lane_xor_f<32>(v);
}
__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
  v = max(v, lane_xor<1>(v));
  v = max(v, lane_xor<2>(v));
  v = max(v, lane_xor<4>(v));
  v = max(v, lane_xor<8>(v));
  v = max(v, lane_xor<16>(v));
  return max(v, lane_xor<32>(v));
}
// The bits of |v|: their unsigned order is the order of the values, with NaN on top.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Sum and maximum over the TPR threads of a row.  One barrier: the slots alternate between two
// halves, and a wave can be at most one row ahead of the others.
template <int TPR>
__device__ __forceinline__ void reduce_row(float &ss, uint32_t &mx, float2 (*slots)[16], int &half) {
  ss = wave_sum(ss);
  mx = wave_umax(mx);
  if constexpr (TPR > 64) {
    constexpr int WAVES = TPR / 64;
    if ((threadIdx.x & 63) == 0) slots[half][threadIdx.x >> 6] = make_float2(ss, __uint_as_float(mx));
    __syncthreads();
    ss = 0.0f;
    mx = 0u;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float2 o = slots[half][w];
      ss += o.x;
      mx = max(mx, __float_as_uint(o.y));
    }
    half ^= 1;
  }
}

// Threads of a workgroup: four rows of a wave each, or one row of TPR threads.
template <int TPR> constexpr int block_of = TPR == 64 ? 256 : TPR;

// What a row's codes are multiplied by: T / max, in two factors so that a maximum near the smallest
// float32 values does not overflow it, and 0 where the row's scale is 0 (also of a row that is not: its
// maximum may be so small, or its norm so large, that the scale has no float32).
struct CodeScale { float pre, inv; };
__device__ __forceinline__ CodeScale code_scale(uint32_t mx, float scale, float top) {
  const float m = __uint_as_float(mx);
  CodeScale c;
  c.pre = m < 1e-30f ? 0x1p100f : 1.0f;
  c.inv = scale != 0.0f ? top / (m * c.pre) : 0.0f;
  return c;
}

// 8 columns of a row as they are stored: loaded early, widened where they are used.  Columns past the
// row's end are 0.
template <typename T>
struct Raw8 {
  uint32_t w[sizeof(T) * 2];
  __device__ __forceinline__ void load(const T *p, int n) {
    if (n >= 8) {
#pragma unroll
      for (int j = 0; j < int(sizeof(T)) / 2; ++j) {
        const u32x4 u = load_bytes16(p + 16 / sizeof(T) * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[4 * j + i] = u[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        T e{};
        if (i < n) e = p[i];
        if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(e);
        else w[i / 2] = i & 1 ? w[i / 2] | uint32_t(e.v) << 16 : e.v;
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
  }
};
__device__ __forceinline__ void store_codes(uint8_t *q, int q_dtype, int n, const float (&v)[8]) {
  u32x2 o;
  if (q_dtype == FQT_I8) {
    o[0] = codes4<FQT_I8>(v[0], v[1], v[2], v[3]);
    o[1] = codes4<FQT_I8>(v[4], v[5], v[6], v[7]);
  } else {
    o[0] = codes4<FQT_E4M3>(v[0], v[1], v[2], v[3]);
    o[1] = codes4<FQT_E4M3>(v[4], v[5], v[6], v[7]);
  }
  if (n >= 8) {
    *reinterpret_cast<u32x2_at1 *>(q) = o;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) q[i] = uint8_t(o[i / 4] >> (8 * (i & 3)));
  }
}

// One row per TPR threads, VPT groups of 8 columns per thread.  Workgroups walk the rows with g in
// registers and the next row's loads under way.  4608 x 4096 bf16 with residual, sum, norm and codes
// (170 MB): 36 us a call on fresh inputs, 4.7 TB/s (a large copy reaches 5.1); a launch over the same inputs
// again takes 27, half of its reads from the last-level cache.
template <typename XT, typename YT, int TPR, int VPT>
__global__ void __launch_bounds__(block_of<TPR>) k_norm_fwd(NormArgs a) {
  constexpr int ROWS = block_of<TPR> / TPR;
  __shared__ float2 slots[2][16];
  const int t = threadIdx.x % TPR;
  int half = 0;
  // the thread's groups of 8 columns, and how many columns are left there
  auto col = [&](int v) { return (v * TPR + t) * 8; };
  auto left = [&](int v) { return a.cols - col(v); };
  float g[VPT][8];
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    if (a.g) {
      load8f(a.g + col(v), left(v), g[v]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[v][i] = 1.0f;
    }
  }
  const int64_t stride = int64_t(gridDim.x) * ROWS;
  int64_t row = int64_t(blockIdx.x) * ROWS + threadIdx.x / TPR;
  Raw8<XT> nx[VPT], nr[VPT];
  auto fetch = [&](int64_t at) {
    if (at >= a.rows) return;
#pragma unroll
    for (int v = 0; v < VPT; ++v) nx[v].load(static_cast<const XT *>(a.x) + at * a.ldx + col(v), left(v));
    if (a.r)
#pragma unroll
      for (int v = 0; v < VPT; ++v) nr[v].load(static_cast<const XT *>(a.r) + at * a.ldr + col(v), left(v));
  };
  fetch(row);
  for (; row < a.rows; row += stride) {
    float h[VPT][8];
    float ss = 0.0f;
    uint32_t mx = 0;
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[v][i] = nx[v].get(i);
        if (a.r) h[v][i] += nr[v].get(i);
        ss = fmaf(h[v][i], h[v][i], ss);
        mx = max(mx, abs_bits(h[v][i] * g[v][i]));
      }
    fetch(row + stride);
    reduce_row<TPR>(ss, mx, slots, half);
    const float rstd = a.norm ? 1.0f / sqrtf(ss / float(a.cols) + a.eps) : 1.0f;
    const float scale = rstd * __uint_as_float(mx) / code_top(a.q_dtype);
    if (t == 0) {
      if (a.rstd) a.rstd[row] = rstd;
      if (a.scale) a.scale[row] = scale;
    }
    const CodeScale cs = code_scale(mx, scale, code_top(a.q_dtype));
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      if (left(v) <= 0) continue;
      if (a.h) store8f(static_cast<XT *>(a.h) + row * a.ldh + col(v), left(v), h[v]);
      if (a.q) {
        float u[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = h[v][i] * g[v][i] * cs.pre * cs.inv;
        store_codes(a.q + row * a.ldq + col(v), a.q_dtype, left(v), u);
      }
      if (a.y) {
#pragma unroll
        for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * rstd * g[v][i];
        store8f(static_cast<YT *>(a.y) + row * a.ldy + col(v), left(v), h[v]);
      }
    }
  }
}

// Rows too long for registers: a workgroup per row reads it twice (statistics, then outputs; the
// second sweep comes from L2 up to some megabytes).  An element is read again before its own place
// in h is written, so h may be x or the residual here too.
constexpr int LONG_TPR = 1024;
template <typename XT, typename YT>
__global__ void __launch_bounds__(LONG_TPR) k_norm_fwd_long(NormArgs a) {
  __shared__ float2 slots[2][16];
  int half = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const XT *x = static_cast<const XT *>(a.x) + row * a.ldx;
    const XT *r = static_cast<const XT *>(a.r) + row * a.ldr;
    auto load_h = [&](int c, int n, float (&h)[8], float (&g)[8]) {
      load8f(x + c, n, h);
      if (a.r) {
        float u[8];
        load8f(r + c, n, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] += u[i];
      }
      if (a.g) {
        load8f(a.g + c, n, g);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.0f;
      }
    };
    float ss = 0.0f;
    uint32_t mx = 0;
    for (int c = threadIdx.x * 8; c < a.cols; c += LONG_TPR * 8) {
      float h[8], g[8];
      load_h(c, a.cols - c, h, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ss = fmaf(h[i], h[i], ss);
        mx = max(mx, abs_bits(h[i] * g[i]));
      }
    }
    reduce_row<LONG_TPR>(ss, mx, slots, half);
    const float rstd = a.norm ? 1.0f / sqrtf(ss / float(a.cols) + a.eps) : 1.0f;
    const float scale = rstd * __uint_as_float(mx) / code_top(a.q_dtype);
    if (threadIdx.x == 0) {
      if (a.rstd) a.rstd[row] = rstd;
      if (a.scale) a.scale[row] = scale;
    }
    const CodeScale cs = code_scale(mx, scale, code_top(a.q_dtype));
    for (int c = threadIdx.x * 8; c < a.cols; c += LONG_TPR * 8) {
      const int n = a.cols - c;
      float h[8], g[8], u[8];
      load_h(c, n, h, g);
      if (a.h) store8f(static_cast<XT *>(a.h) + row * a.ldh + c, n, h);
      if (a.q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = h[i] * g[i] * cs.pre * cs.inv;
        store_codes(a.q + row * a.ldq + c, a.q_dtype, n, u);
      }
      if (a.y) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = h[i] * rstd * g[i];
        store8f(static_cast<YT *>(a.y) + row * a.ldy + c, n, u);
      }
    }
  }
}

// ----------------------------------------------------------------------------- backward

struct NormBwdArgs {
  const void *h, *dy, *dres;
  const float *g, *rstd;
  void *dx;
  float *part;         // [workgroups][cols] partial sums of dg
  int64_t rows;
  int32_t cols;
  int64_t ldh, ldy, ldr, ldx;
};

// 8192 x 4096 bf16 with dres (269 MB): 54 us a call on fresh inputs with the launch that adds up dg, 4.9 TB/s;
// launches over the same inputs again take 41 + 5.
template <typename XT, typename YT, int TPR, int VPT>
__global__ void __launch_bounds__(block_of<TPR>) k_norm_bwd(NormBwdArgs a) {
  constexpr int ROWS = block_of<TPR> / TPR;
  __shared__ float2 slots[2][16];
  __shared__ float merge[ROWS > 1 ? ROWS - 1 : 1][ROWS > 1 ? TPR * VPT * 8 : 1];
  const int t = threadIdx.x % TPR;
  int half = 0;
  auto col = [&](int v) { return (v * TPR + t) * 8; };
  auto left = [&](int v) { return a.cols - col(v); };
  float dg[VPT][8] = {}, g[VPT][8];
#pragma unroll
  for (int v = 0; v < VPT; ++v) load8f(a.g + col(v), left(v), g[v]);
  const int64_t stride = int64_t(gridDim.x) * ROWS;
  int64_t row = int64_t(blockIdx.x) * ROWS + threadIdx.x / TPR;
  Raw8<XT> nh[VPT], nr[VPT];
  Raw8<YT> ny[VPT];
  float nrstd = 0.0f;
  auto fetch = [&](int64_t at) {
    if (at >= a.rows) return;
    nrstd = a.rstd[at];
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      nh[v].load(static_cast<const XT *>(a.h) + at * a.ldh + col(v), left(v));
      ny[v].load(static_cast<const YT *>(a.dy) + at * a.ldy + col(v), left(v));
    }
    if (a.dres)
#pragma unroll
      for (int v = 0; v < VPT; ++v) nr[v].load(static_cast<const XT *>(a.dres) + at * a.ldr + col(v), left(v));
  };
  fetch(row);
  for (; row < a.rows; row += stride) {
    const float rstd = nrstd;
    float h[VPT][8], u[VPT][8];
    Raw8<XT> r[VPT];
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      r[v] = nr[v];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[v][i] = nh[v].get(i) * rstd;                      // t
        const float d = ny[v].get(i);
        dg[v][i] = fmaf(d, h[v][i], dg[v][i]);
        u[v][i] = d * g[v][i];
        dot = fmaf(u[v][i], h[v][i], dot);
      }
    }
    fetch(row + stride);
    uint32_t none = 0;
    reduce_row<TPR>(dot, none, slots, half);
    const float m = dot / float(a.cols);
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
      if (left(v) <= 0) continue;
      float d[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        d[i] = rstd * (u[v][i] - h[v][i] * m);
        if (a.dres) d[i] += r[v].get(i);
      }
      store8f(static_cast<XT *>(a.dx) + row * a.ldx + col(v), left(v), d);
    }
  }
  if constexpr (ROWS > 1) {            // the rows' waves meet in LDS
    const int w = threadIdx.x / TPR;
    if (w > 0)
#pragma unroll
      for (int v = 0; v < VPT; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) merge[w - 1][(v * 8 + i) * TPR + t] = dg[v][i];
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int v = 0; v < VPT; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int k = 0; k < ROWS - 1; ++k) dg[v][i] += merge[k][(v * 8 + i) * TPR + t];
  }
  float *out = a.part + int64_t(blockIdx.x) * a.cols;
#pragma unroll
  for (int v = 0; v < VPT; ++v) {
    if (left(v) > 0) store8f(out + col(v), left(v), dg[v]);
  }
}

// Rows of up to 32768 columns: the row stays in registers as it is stored, 32 columns a thread, and is
// widened twice; 16 waves on a CU hide the loads, so nothing is loaded ahead.  1024 x 25088 bf16: 67 us
// a call on fresh inputs; over the same inputs again 56, and 68 with the row read twice.
constexpr int WIDE_TPR = 1024, WIDE_VPT = 4;
template <typename XT, typename YT>
__global__ void __launch_bounds__(WIDE_TPR) k_norm_bwd_wide(NormBwdArgs a) {
  __shared__ float2 slots[2][16];
  int half = 0;
  auto col = [&](int v) { return (v * WIDE_TPR + int(threadIdx.x)) * 8; };
  auto left = [&](int v) { return a.cols - col(v); };
  float dg[WIDE_VPT][8] = {};
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const float rstd = a.rstd[row];
    Raw8<XT> h[WIDE_VPT];
    Raw8<YT> y[WIDE_VPT];
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < WIDE_VPT; ++v) {
      h[v].load(static_cast<const XT *>(a.h) + row * a.ldh + col(v), left(v));
      y[v].load(static_cast<const YT *>(a.dy) + row * a.ldy + col(v), left(v));
    }
#pragma unroll
    for (int v = 0; v < WIDE_VPT; ++v) {
      float g[8];
      load8f(a.g + col(v), left(v), g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float t = h[v].get(i) * rstd, d = y[v].get(i);
        dg[v][i] = fmaf(d, t, dg[v][i]);
        dot = fmaf(d * g[i], t, dot);
      }
    }
    uint32_t none = 0;
    reduce_row<WIDE_TPR>(dot, none, slots, half);
    const float m = dot / float(a.cols);
#pragma unroll
    for (int v = 0; v < WIDE_VPT; ++v) {
      if (left(v) <= 0) continue;
      float g[8], d[8];
      load8f(a.g + col(v), left(v), g);
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = rstd * (y[v].get(i) * g[i] - h[v].get(i) * rstd * m);
      if (a.dres) {
        float e[8];
        load8f(static_cast<const XT *>(a.dres) + row * a.ldr + col(v), left(v), e);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] += e[i];
      }
      store8f(static_cast<XT *>(a.dx) + row * a.ldx + col(v), left(v), d);
    }
  }
  float *out = a.part + int64_t(blockIdx.x) * a.cols;
#pragma unroll
  for (int v = 0; v < WIDE_VPT; ++v)
    if (left(v) > 0) store8f(out + col(v), left(v), dg[v]);
}

// dx of rows too long for registers: h and dy are read twice.
template <typename XT, typename YT>
__global__ void __launch_bounds__(LONG_TPR) k_norm_bwd_long(NormBwdArgs a) {
  __shared__ float2 slots[2][16];
  int half = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const XT *hp = static_cast<const XT *>(a.h) + row * a.ldh;
    const YT *dyp = static_cast<const YT *>(a.dy) + row * a.ldy;
    const XT *rp = static_cast<const XT *>(a.dres) + row * a.ldr;
    const float rstd = a.rstd[row];
    float dot = 0.0f;
    auto load = [&](int c, int n, float (&t)[8], float (&u)[8]) {
      float g[8];
      load8f(hp + c, n, t);
      load8f(dyp + c, n, u);
      load8f(a.g + c, n, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] *= rstd, u[i] *= g[i];
    };
    for (int c = threadIdx.x * 8; c < a.cols; c += LONG_TPR * 8) {
      float t[8], u[8];
      load(c, a.cols - c, t, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) dot = fmaf(u[i], t[i], dot);
    }
    uint32_t none = 0;
    reduce_row<LONG_TPR>(dot, none, slots, half);
    const float m = dot / float(a.cols);
    for (int c = threadIdx.x * 8; c < a.cols; c += LONG_TPR * 8) {
      const int n = a.cols - c;
      float t[8], u[8], d[8];
      load(c, n, t, u);
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = rstd * (u[i] - t[i] * m);
      if (a.dres) {
        load8f(rp + c, n, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] += t[i];
      }
      store8f(static_cast<XT *>(a.dx) + row * a.ldx + c, n, d);
    }
  }
}
// Partial sums of dg of those rows: a thread per 8 columns, gridDim.y row groups.
template <typename XT, typename YT>
__global__ void __launch_bounds__(64) k_norm_dg_long(NormBwdArgs a) {
  const int c = (blockIdx.x * 64 + threadIdx.x) * 8, n = a.cols - c;
  if (n <= 0) return;
  float dg[8] = {};
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    float h[8], u[8];
    load8f(static_cast<const XT *>(a.h) + row * a.ldh + c, n, h);
    load8f(static_cast<const YT *>(a.dy) + row * a.ldy + c, n, u);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[i] = fmaf(u[i], h[i] * rstd, dg[i]);
  }
  store8f(a.part + int64_t(blockIdx.y) * a.cols + c, n, dg);
}

// dg[c] = sum of the partial rows: 32 columns per workgroup, 8 threads per column, in a fixed order.
__global__ void __launch_bounds__(256) k_norm_dg(const float *part, int32_t parts, int32_t cols, float *dg) {
  __shared__ float s[8][32];
  const int c = blockIdx.x * 32 + threadIdx.x % 32, k = threadIdx.x / 32;
  float v = 0.0f;
  if (c < cols)
#pragma unroll 8
    for (int p = k; p < parts; p += 8) v += part[int64_t(p) * cols + c];
  s[k][threadIdx.x % 32] = v;
  __syncthreads();
  if (k == 0 && c < cols) {
#pragma unroll
    for (int j = 1; j < 8; ++j) v += s[j][threadIdx.x];
    dg[c] = v;
  }
}

// ----------------------------------------------------------------------------- host side

// Calls f.template operator()<TPR, VPT>() with the smallest row shape that holds `cols`; false when
// the row does not fit registers.  A wave per row up to 1024 columns (no barrier), then a workgroup; 16
// columns a thread leave registers for the next row's loads (32 a thread spill them).
constexpr int FWD_MAX_COLS = 16384, BWD_MAX_COLS = 8192;
template <int MAX_COLS, typename F>
bool dispatch_row(int64_t cols, F &&f) {
  if (cols > MAX_COLS) return false;
  if (cols <= 512) f.template operator()<64, 1>();
  else if (cols <= 1024) f.template operator()<64, 2>();
  else if (cols <= 2048) f.template operator()<128, 2>();
  else if (cols <= 4096) f.template operator()<256, 2>();
  else if (cols <= 8192) f.template operator()<512, 2>();
  else if constexpr (MAX_COLS > 8192) f.template operator()<1024, 2>();
  return true;
}

template <typename F>
void dispatch_xy(int xt, int yt, F &&f) {
  if (xt == FQT_BF16) {
    if (yt == FQT_BF16) f.template operator()<bf16, bf16>();
    else f.template operator()<bf16, float>();
  } else {
    if (yt == FQT_BF16) f.template operator()<float, bf16>();
    else f.template operator()<float, float>();
  }
}

struct Strides { int64_t x, r, h, y, q; };
int check_norm(const fqt_norm_desc *d, Strides *s) {
  if (!d) return FQT_E_NULL;
  if (!float_type(d->x_dtype) || !float_type(d->y_dtype) ||
      !(code_type(d->q_dtype) || d->q_dtype == FQT_NO_CODES))
    return FQT_E_DTYPE;
  if (d->rows < 0 || d->cols < 0 || d->rows >= FQT_MAX_ROWS || d->cols > FQT_MAX_LD) return FQT_E_SHAPE;
  if (!(d->eps > 0.0f) || !std::isfinite(d->eps)) return FQT_E_INVAL;
  *s = {row_stride(d->ldx, d->cols), row_stride(d->ldr, d->cols), row_stride(d->ldh, d->cols),
        row_stride(d->ldy, d->cols), row_stride(d->ldq, d->cols)};
  if (!s->x || !s->r || !s->h || !s->y || !s->q) return FQT_E_SHAPE;
  return FQT_OK;
}

int run_norm(const fqt_norm_desc *d, NormArgs a, hipStream_t st) {
  if (d->rows == 0 || d->cols == 0) return FQT_OK;
  a.rows = d->rows;
  a.cols = int32_t(d->cols);
  a.q_dtype = d->q_dtype;
  a.eps = d->eps;
  dispatch_xy(d->x_dtype, d->y_dtype, [&]<typename XT, typename YT>() {
    if (!dispatch_row<FWD_MAX_COLS>(d->cols, [&]<int TPR, int VPT>() {
          constexpr int ROWS = block_of<TPR> / TPR;
          // as many workgroups as are resident at once, with equal numbers of rows
          const int64_t sets = (d->rows + ROWS - 1) / ROWS, most = 1024 * 256 / block_of<TPR>;
          const int64_t each = (sets + most - 1) / most, blocks = (sets + each - 1) / each;
          k_norm_fwd<XT, YT, TPR, VPT><<<dim3(blocks), dim3(block_of<TPR>), 0, st>>>(a);
        }))
      k_norm_fwd_long<XT, YT><<<dim3(std::min<int64_t>(d->rows, 512)), dim3(LONG_TPR), 0, st>>>(a);
  });
  return last_launch_status();
}

// Workgroups of the backward = rows of partial sums.
int64_t bwd_parts(int64_t rows, int64_t cols) {
  if (cols > WIDE_TPR * WIDE_VPT * 8) return std::min<int64_t>(std::max<int64_t>(rows, 1), 64);
  if (cols > BWD_MAX_COLS) return std::min<int64_t>(std::max<int64_t>(rows, 1), 256);
  const int64_t per = cols <= 1024 ? 4 : 1;     // rows of a workgroup at a time
  return std::min<int64_t>(std::max<int64_t>((rows + per - 1) / per, 1), 512);
}

}  // namespace
}  // namespace dense
}  // namespace fqt

using namespace fqt;
using namespace fqt::dense;

extern "C" int fqt_rmsnorm_forward(const fqt_norm_desc *d, const void *x, const void *residual,
                                   const float *g, void *h, void *y, void *q, float *scale,
                                   float *rstd, void *hip_stream) {
  Strides s;
  FQT_TRY_(check_norm(d, &s));
  if (q && d->q_dtype == FQT_NO_CODES) return FQT_E_DTYPE;
  if (d->rows == 0 || d->cols == 0) return FQT_OK;
  if (!x || !g || (q && !scale) || (scale && !q)) return FQT_E_NULL;
  if (!elem_aligned(x, d->x_dtype) || !elem_aligned(residual, d->x_dtype) || !aligned(g, 4) ||
      !elem_aligned(h, d->x_dtype) || !elem_aligned(y, d->y_dtype) || !aligned(scale, 4) ||
      !aligned(rstd, 4))
    return FQT_E_ALIGN;
  NormArgs a{};
  a.x = x; a.r = residual; a.g = g; a.h = h; a.y = y;
  a.q = static_cast<uint8_t *>(q);
  a.scale = scale; a.rstd = rstd;
  a.ldx = s.x; a.ldr = s.r; a.ldh = s.h; a.ldy = s.y; a.ldq = s.q;
  a.norm = 1;
  return run_norm(d, a, static_cast<hipStream_t>(hip_stream));
}

extern "C" int fqt_quantize_rows(const fqt_norm_desc *d, const void *x, void *q, float *scale,
                                 void *hip_stream) {
  Strides s;
  FQT_TRY_(check_norm(d, &s));
  if (!code_type(d->q_dtype)) return FQT_E_DTYPE;
  if (d->rows == 0 || d->cols == 0) return FQT_OK;
  if (!x || !q || !scale) return FQT_E_NULL;
  if (!elem_aligned(x, d->x_dtype) || !aligned(scale, 4)) return FQT_E_ALIGN;
  NormArgs a{};
  a.x = x;
  a.q = static_cast<uint8_t *>(q);
  a.scale = scale;
  a.ldx = s.x; a.ldq = s.q;
  return run_norm(d, a, static_cast<hipStream_t>(hip_stream));
}

extern "C" int fqt_norm_workspace_size(const fqt_norm_desc *d, size_t *bytes) {
  Strides s;
  FQT_TRY_(check_norm(d, &s));
  if (!bytes) return FQT_E_NULL;
  *bytes = align256(size_t(bwd_parts(d->rows, d->cols)) * size_t(d->cols) * sizeof(float));
  return FQT_OK;
}

extern "C" int fqt_rmsnorm_backward(const fqt_norm_desc *d, const void *h, const float *g,
                                    const float *rstd, const void *dy, const void *dres, void *dx,
                                    float *dg, void *ws, size_t ws_bytes, void *hip_stream) {
  Strides s;
  FQT_TRY_(check_norm(d, &s));
  size_t need = 0;
  FQT_TRY_(fqt_norm_workspace_size(d, &need));
  if (d->cols == 0) return FQT_OK;
  if (!g || !dg || !ws || (d->rows && (!h || !rstd || !dy || !dx))) return FQT_E_NULL;
  if (!elem_aligned(h, d->x_dtype) || !aligned(g, 4) || !aligned(rstd, 4) ||
      !elem_aligned(dy, d->y_dtype) || !elem_aligned(dres, d->x_dtype) ||
      !elem_aligned(dx, d->x_dtype) || !aligned(dg, 4) || !aligned(ws, 256))
    return FQT_E_ALIGN;
  if (ws_bytes < need) return FQT_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  NormBwdArgs a{};
  a.h = h; a.dy = dy; a.dres = dres; a.g = g; a.rstd = rstd; a.dx = dx;
  a.part = static_cast<float *>(ws);
  a.rows = d->rows;
  a.cols = int32_t(d->cols);
  a.ldh = s.h; a.ldy = s.y; a.ldr = s.r; a.ldx = s.x;
  const int64_t parts = bwd_parts(d->rows, d->cols);
  dispatch_xy(d->x_dtype, d->y_dtype, [&]<typename XT, typename YT>() {
    if (dispatch_row<BWD_MAX_COLS>(d->cols, [&]<int TPR, int VPT>() {
          k_norm_bwd<XT, YT, TPR, VPT><<<dim3(parts), dim3(block_of<TPR>), 0, st>>>(a);
        }))
      return;
    if (d->cols <= WIDE_TPR * WIDE_VPT * 8) {
      k_norm_bwd_wide<XT, YT><<<dim3(parts), dim3(WIDE_TPR), 0, st>>>(a);
      return;
    }
    if (d->rows)
      k_norm_bwd_long<XT, YT><<<dim3(std::min<int64_t>(d->rows, 512)), dim3(LONG_TPR), 0, st>>>(a);
    k_norm_dg_long<XT, YT><<<dim3((d->cols + 511) / 512, parts), dim3(64), 0, st>>>(a);
  });
  FQT_TRY_(last_launch_status());
  k_norm_dg<<<dim3((d->cols + 31) / 32), dim3(256), 0, st>>>(a.part, int32_t(parts),
                                                             int32_t(d->cols), dg);
  return last_launch_status();
}
