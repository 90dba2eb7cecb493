// Operators over a list of tensors: AdamW with states in float32 or 8 bits, and the norm of all gradients.
//
// A launch takes up to LIST tensors by value, as kernel arguments: nothing has to be copied to the device or
// kept for a captured graph, and gradients may move from step to step.  Workgroups take chunks; a search
// over the chunk counts (scalar, in the arguments) finds a workgroup's tensor.  Both are bound by memory
// traffic on large models and by their launches on small ones.
#include "fqt_dense.hpp"
#include "fqt_step.h"

namespace fqt {
namespace dense {
namespace {

// Products and sums are rounded one by one as they are written, so that codes can be computed again elsewhere
// bit for bit (fmaf where one rounding does).
#pragma clang fp contract(off)

constexpr int BLOCK = FQT_STATE_BLOCK;

// The tensors of a launch; chunk c of the launch belongs to the last entry whose `begin` is <= c.  Launches have
// 4 KB of arguments, so entries hold what their kernel needs: 62 tensors with 8-bit states are one launch of 51
// us, as two launches of 48 and 14 they took 57.
struct NormEntry {
  const void *g;
  uint32_t n;                         // elements (a longer tensor has several entries)
};
struct AdamEntry {
  const void *g;
  float *p, *m, *v;
  uint32_t n;
};
struct CodesEntry {
  const void *g;
  float *p;
  char *m, *v;
  float *m_scale, *v_scale;
  uint32_t n;
  uint32_t quad;                      // (place in the random sequence) / 4 from the list's `quad` on
};
template <typename E>
struct List {
  static constexpr int MOST = (4096 - 192) / (sizeof(E) + 4);
  E e[MOST];
  uint32_t begin[MOST];               // first chunks
  uint32_t half[(MOST + 31) / 32];    // bit i: the gradient of entry i is bf16
  int32_t count;
  uint64_t quad;
};
static_assert(sizeof(List<NormEntry>) <= 3968 && sizeof(List<AdamEntry>) <= 3968 && sizeof(List<CodesEntry>) <= 3968, "kernel arguments");
template <typename E>
__device__ __forceinline__ bool is_half(const List<E> &l, int i) { return l.half[i / 32] >> (i % 32) & 1; }
template <typename E>
__device__ __forceinline__ int entry_of(const List<E> &l, uint32_t chunk) {
  int lo = 0, hi = l.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (l.begin[mid] <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Four elements from p, at most n of them.
__device__ __forceinline__ void load4(const float *p, int64_t n, float (&o)[4]) {
  if (n >= 4) {
    const u32x4 u = load_bytes16(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(u[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = i < n ? p[i] : 0.0f;
  }
}
typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void load4(const bf16 *p, int64_t n, float (&o)[4]) {
  if (n >= 4) {
    const u32x2_at2 u = *reinterpret_cast<const u32x2_at2 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __uint_as_float(i & 1 ? u[i / 2] & 0xFFFF0000u : u[i / 2] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = i < n ? to_f32(p[i]) : 0.0f;
  }
}
__device__ __forceinline__ void load4(const void *p, int64_t at, bool half, int64_t n, float (&o)[4]) {
  if (half) load4(static_cast<const bf16 *>(p) + at, n, o);
  else load4(static_cast<const float *>(p) + at, n, o);
}
__device__ __forceinline__ void store4(float *p, int64_t n, const float (&v)[4]) {
  if (n >= 4) {
    store_bytes16(p, u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])});
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = v[i];
  }
}
typedef uint32_t u32_at1 __attribute__((aligned(1)));
__device__ __forceinline__ uint32_t load_codes(const char *p, int64_t n) {
  if (n >= 4) return *reinterpret_cast<const u32_at1 *>(p);
  uint32_t u = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < n) u |= uint32_t(uint8_t(p[i])) << (8 * i);
  return u;
}
__device__ __forceinline__ void store_codes(char *p, int64_t n, uint32_t u) {
  if (n >= 4) {
    *reinterpret_cast<u32_at1 *>(p) = u;
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < n) p[i] = char(u >> (8 * i));
  }
}

// ----------------------------------------------------------------------------- AdamW

struct Adam {
  float beta1, rest1, beta2, rest2;   // beta and 1 - beta
  float rate, even;                   // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  float decay, eps;                   // lr weight_decay
  uint32_t t;
  uint64_t seed;
  double lr, b1, b2;                  // for t from the device
  const int64_t *step;
  const float *scale;
};
// b^t by squaring.
__host__ __device__ inline double power(double b, uint64_t t) {
  double r = 1.0;
  for (; t; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}
__host__ __device__ inline void at_step(Adam &a, int64_t t) {
  a.t = uint32_t(t);
  a.rate = float(a.lr / (1.0 - power(a.b1, uint64_t(t))));
  a.even = float(1.0 / sqrt(1.0 - power(a.b2, uint64_t(t))));
}

__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
  v = max(v, lane_xor<1>(v));
  v = max(v, lane_xor<2>(v));
  v = max(v, lane_xor<4>(v));
  v = max(v, lane_xor<8>(v));
  v = max(v, lane_xor<16>(v));
  return max(v, lane_xor<32>(v));
}

// The codes of four values of a wave's block, and its scale.  A positive e4m3 is the upper bits of the
// float32 of its value times 2^-120 (the exponents' biases differ by that much, subnormals included), so that adding
// 16 random bits right below the code rounds up with the probability of the 20 bits that are cut off, to 2^-16.
// The largest value gets code 0x7E exactly; min takes the quotient's last rounding.
template <bool ROOT>
__device__ __forceinline__ uint32_t encode(const float (&x)[4], const uint32_t (&random)[4], float *scale, bool store) {
  uint32_t mx = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) mx = max(mx, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  mx = wave_umax(mx);
  const float top = __uint_as_float(mx);
  const bool none = top < 0x1p-100f;                       // (false for NaN)
  const float inv = none ? 0.0f : 1.0f / top * 448.0f;
  if (store) *scale = none ? 0.0f : top * (1.0f / 448.0f);
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t bits = __float_as_uint(fabsf(x[i]) * inv * 0x1p-120f);
    uint32_t c = min((bits + (ROOT ? random[i] >> 16 << 4 : (random[i] & 0xFFFFu) << 4)) >> 20, 0x7Eu);
    if constexpr (ROOT) c = x[i] > 0.0f && !none ? max(c, 1u) : c;
    else c |= __float_as_uint(x[i]) >> 24 & 0x80u;
    codes |= c << (8 * i);
  }
  return codes;
}
__device__ __forceinline__ void decode(uint32_t u, float scale, float (&o)[4]) {
  o[0] = __builtin_amdgcn_cvt_f32_fp8(int(u), 0) * scale;
  o[1] = __builtin_amdgcn_cvt_f32_fp8(int(u), 1) * scale;
  o[2] = __builtin_amdgcn_cvt_f32_fp8(int(u), 2) * scale;
  o[3] = __builtin_amdgcn_cvt_f32_fp8(int(u), 3) * scale;
}

// A wave takes BLOCKS blocks of 256 elements, four consecutive elements a lane, all loads first: four of them with
// 8-bit states, one with float32 (VGG-16, us with one, two and four blocks: 8-bit states, bf16 gradients 404, 390, 383: 5.1
// TB/s; float32 686, 730, 725: 5.6 TB/s).
template <typename E> constexpr int adam_blocks = std::is_same_v<E, CodesEntry> ? 4 : 1;
template <typename E> constexpr int adam_chunk = 4 * adam_blocks<E> * BLOCK;
template <typename E>
__global__ void __launch_bounds__(256) k_adamw(List<E> list, Adam a) {
  constexpr bool CODES = std::is_same_v<E, CodesEntry>;
  constexpr int BLOCKS = adam_blocks<E>;
  const int at = entry_of(list, blockIdx.x);
  const E &e = list.e[at];
  const bool half = is_half(list, at);
  if (a.step) at_step(a, max(*a.step, int64_t(1)));
  const float s = a.scale ? *a.scale : 1.0f;
  const int lane = threadIdx.x % 64;
  const int64_t b0 = (int64_t(blockIdx.x - list.begin[at]) * 4 + wave_id()) * BLOCKS;
  float g[BLOCKS][4], p[BLOCKS][4], m[BLOCKS][4], v[BLOCKS][4];
  uint32_t cm[BLOCKS], cv[BLOCKS];
  float sm[BLOCKS], sv[BLOCKS];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const int64_t i = (b0 + b) * BLOCK + lane * 4, left = int64_t(e.n) - i;
    load4(e.g, i, half, left, g[b]);
    load4(e.p + i, left, p[b]);
    if constexpr (CODES) {
      cm[b] = load_codes(e.m + i, left);
      cv[b] = load_codes(e.v + i, left);
      const bool any = (b0 + b) * BLOCK < e.n;
      sm[b] = any ? e.m_scale[b0 + b] : 0.0f;
      sv[b] = any ? e.v_scale[b0 + b] : 0.0f;
    } else {
      load4(e.m + i, left, m[b]);
      load4(e.v + i, left, v[b]);
    }
  }
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const int64_t i = (b0 + b) * BLOCK + lane * 4, left = int64_t(e.n) - i;
    if ((b0 + b) * BLOCK >= e.n) break;
    float root[4];
    if constexpr (CODES) {
      decode(cm[b], sm[b], m[b]);
      decode(cv[b], sv[b], v[b]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float d = g[b][j] * s;
      if constexpr (CODES) v[b][j] *= v[b][j];
      m[b][j] = a.beta1 * m[b][j] + a.rest1 * d;
      v[b][j] = a.beta2 * v[b][j] + a.rest2 * d * d;
      root[j] = sqrtf(v[b][j]);
      p[b][j] -= fmaf(a.decay, p[b][j], a.rate * m[b][j] / fmaf(root[j], a.even, a.eps));
    }
    store4(e.p + i, left, p[b]);
    if constexpr (CODES) {
      const Ctr4 r = philox_block(list.quad + e.quad + (uint64_t(i) >> 2), 3, a.seed, a.t, 0);
      store_codes(e.m + i, left, encode<false>(m[b], r.v, e.m_scale + b0 + b, lane == 0));
      store_codes(e.v + i, left, encode<true>(root, r.v, e.v_scale + b0 + b, lane == 0));
    } else {
      store4(e.m + i, left, m[b]);
      store4(e.v + i, left, v[b]);
    }
  }
}

// ----------------------------------------------------------------------------- norm

// The sum of squares of a chunk, in float64 (float32 squares leave its range past 1.8e19, and a sum over 10^8
// terms its precision).
constexpr int NORM_QUADS = 8, NORM_CHUNK = 256 * 4 * NORM_QUADS;
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o > 0; o /= 2) v += __shfl_xor(v, o);
  return v;
}
__global__ void __launch_bounds__(256) k_sum_squares(List<NormEntry> list, double *part) {
  __shared__ double waves[4];
  const int at = entry_of(list, blockIdx.x);
  const NormEntry &e = list.e[at];
  const bool half = is_half(list, at);
  const int64_t i0 = int64_t(blockIdx.x - list.begin[at]) * NORM_CHUNK + threadIdx.x * 4;
  float g[NORM_QUADS][4];
#pragma unroll
  for (int q = 0; q < NORM_QUADS; ++q) load4(e.g, i0 + q * 1024, half, int64_t(e.n) - i0 - q * 1024, g[q]);
  double sum = 0.0;
#pragma unroll
  for (int q = 0; q < NORM_QUADS; ++q)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = fma(double(g[q][j]), double(g[q][j]), sum);
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.x] = (waves[0] + waves[1]) + (waves[2] + waves[3]);
}
__global__ void __launch_bounds__(1024) k_norm(const double *part, int64_t parts, float max_norm, float *out) {
  __shared__ double waves[16];
  double sum = 0.0;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < parts; i += 1024) sum += part[i];
  sum = wave_sum(sum);
  if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = sum;
  __syncthreads();
  if (threadIdx.x) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) sum += waves[i];
  const double norm = sqrt(sum), f = double(max_norm) / (norm + 1e-6);
  out[0] = float(norm);
  out[1] = norm != norm ? float(norm) : f < 1.0 ? float(f) : 1.0f;
}

// ----------------------------------------------------------------------------- host side

// Calls f(list, chunks) for each launch of up to List::MOST entries and MOST_CHUNKS chunks; longer tensors have
// several entries of SPAN elements.
constexpr int64_t MOST_CHUNKS = 1 << 23, SPAN = 1 << 30;   // (a launch counts its threads in 32 bits)
template <typename E, typename F>
int for_lists(const fqt_param *t, int32_t count, int64_t chunk, F &&f) {
  List<E> l{};
  int64_t chunks = 0;
  auto flush = [&]() -> int {
    if (!l.count) return FQT_OK;
    const int st = f(l, uint32_t(chunks));
    l.count = 0;
    std::fill(std::begin(l.half), std::end(l.half), 0u);
    chunks = 0;
    return st;
  };
  for (int32_t i = 0; i < count; ++i) {
    for (int64_t at = 0; at < t[i].n; at += SPAN) {
      const int64_t n = std::min(t[i].n - at, SPAN), c = (n + chunk - 1) / chunk;
      if (l.count == List<E>::MOST || chunks + c > MOST_CHUNKS) FQT_TRY_(flush());
      if constexpr (std::is_same_v<E, CodesEntry>) {
        const uint64_t quad = uint64_t(t[i].first + at) / 4;
        if (l.count && (quad < l.quad || quad - l.quad > UINT32_MAX)) FQT_TRY_(flush());
        if (!l.count) l.quad = quad;
      }
      E &e = l.e[l.count];
      e.g = static_cast<const char *>(t[i].g) + at * elem_size(t[i].g_dtype);
      if constexpr (std::is_same_v<E, AdamEntry>) {
        e.p = t[i].p + at;
        e.m = static_cast<float *>(t[i].m) + at;
        e.v = static_cast<float *>(t[i].v) + at;
      } else if constexpr (std::is_same_v<E, CodesEntry>) {
        e.p = t[i].p + at;
        e.m = static_cast<char *>(t[i].m) + at;
        e.v = static_cast<char *>(t[i].v) + at;
        e.m_scale = t[i].m_scale + at / BLOCK;
        e.v_scale = t[i].v_scale + at / BLOCK;
        e.quad = uint32_t(uint64_t(t[i].first + at) / 4 - l.quad);
      }
      e.n = uint32_t(n);
      l.begin[l.count] = uint32_t(chunks);
      if (t[i].g_dtype == FQT_BF16) l.half[l.count / 32] |= 1u << l.count % 32;
      ++l.count;
      chunks += c;
    }
  }
  return flush();
}

int check_list(const fqt_param *t, int32_t count) {
  if (count < 0 || count > FQT_MAX_PARAMS) return FQT_E_SHAPE;
  if (count && !t) return FQT_E_NULL;
  for (int32_t i = 0; i < count; ++i) {
    if (!float_type(t[i].g_dtype)) return FQT_E_DTYPE;
    if (t[i].n < 0 || t[i].n > int64_t(1) << 40) return FQT_E_SHAPE;
  }
  return FQT_OK;
}
int64_t chunks_of(const fqt_param *t, int32_t count, int64_t chunk) {
  int64_t c = 0;
  for (int32_t i = 0; i < count; ++i) c += (t[i].n + chunk - 1) / chunk;
  return c;
}

}  // namespace
}  // namespace dense
}  // namespace fqt

using namespace fqt;
using namespace fqt::dense;

extern "C" int fqt_grad_norm_workspace_size(const fqt_param *params, int32_t count, size_t *bytes) {
  FQT_TRY_(check_list(params, count));
  if (!bytes) return FQT_E_NULL;
  *bytes = std::max<size_t>(256, align256(size_t(chunks_of(params, count, NORM_CHUNK)) * sizeof(double)));
  return FQT_OK;
}

extern "C" int fqt_grad_norm(const fqt_param *params, int32_t count, float max_norm, float *out, void *ws,
                             size_t ws_bytes, void *hip_stream) {
  size_t need = 0;
  FQT_TRY_(fqt_grad_norm_workspace_size(params, count, &need));
  if (!(max_norm > 0.0f)) return FQT_E_INVAL;
  if (!out || !ws) return FQT_E_NULL;
  if (!aligned(out, 4) || !aligned(ws, 256)) return FQT_E_ALIGN;
  for (int32_t i = 0; i < count; ++i) {
    if (params[i].n && !params[i].g) return FQT_E_NULL;
    if (!elem_aligned(params[i].g, params[i].g_dtype)) return FQT_E_ALIGN;
  }
  if (ws_bytes < need) return FQT_E_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  double *part = static_cast<double *>(ws);
  int64_t done = 0;
  FQT_TRY_(for_lists<NormEntry>(params, count, NORM_CHUNK, [&](const List<NormEntry> &l, uint32_t chunks) {
    k_sum_squares<<<dim3(chunks), dim3(256), 0, st>>>(l, part + done);
    done += chunks;
    return last_launch_status();
  }));
  k_norm<<<dim3(1), dim3(1024), 0, st>>>(part, done, max_norm, out);
  return last_launch_status();
}

extern "C" int fqt_adamw_step(const fqt_adamw_cfg *cfg, const fqt_param *params, int32_t count, int64_t step,
                              const int64_t *step_dev, const float *grad_scale, void *hip_stream) {
  if (!cfg) return FQT_E_NULL;
  const bool codes = cfg->state_dtype == FQT_E4M3;
  if (!codes && cfg->state_dtype != FQT_F32) return FQT_E_DTYPE;
  auto rate = [](double v) { return v >= 0.0 && v <= 1e30; };
  if (!rate(cfg->lr) || !rate(cfg->eps) || !rate(cfg->weight_decay) || !rate(cfg->lr * cfg->weight_decay) ||
      !(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0))
    return FQT_E_INVAL;
  if (!step_dev && step < 1) return FQT_E_INVAL;
  FQT_TRY_(check_list(params, count));
  if (!aligned(step_dev, 8) || !aligned(grad_scale, 4)) return FQT_E_ALIGN;
  for (int32_t i = 0; i < count; ++i) {
    const fqt_param &t = params[i];
    if (t.first < 0 || t.first % 4 || t.first > int64_t(1) << 60) return FQT_E_INVAL;
    if (!t.n) continue;
    if (!t.g || !t.p || !t.m || !t.v || (codes && (!t.m_scale || !t.v_scale))) return FQT_E_NULL;
    if (!elem_aligned(t.g, t.g_dtype) || !aligned(t.p, 4) || (!codes && (!aligned(t.m, 4) || !aligned(t.v, 4))) ||
        (codes && (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))))
      return FQT_E_ALIGN;
  }
  Adam a{};
  a.beta1 = float(cfg->beta1);
  a.rest1 = float(1.0 - cfg->beta1);
  a.beta2 = float(cfg->beta2);
  a.rest2 = float(1.0 - cfg->beta2);
  a.decay = float(cfg->lr * cfg->weight_decay);
  a.eps = float(cfg->eps);
  a.seed = cfg->seed;
  a.lr = cfg->lr;
  a.b1 = cfg->beta1;
  a.b2 = cfg->beta2;
  a.step = step_dev;
  a.scale = grad_scale;
  if (!step_dev) at_step(a, step);
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  auto run = [&]<typename E>() {
    return for_lists<E>(params, count, adam_chunk<E>, [&](const List<E> &l, uint32_t chunks) {
      k_adamw<E><<<dim3(chunks), dim3(256), 0, st>>>(l, a);
      return last_launch_status();
    });
  };
  return codes ? run.template operator()<CodesEntry>() : run.template operator()<AdamEntry>();
}
