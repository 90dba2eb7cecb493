// Matrix-product tile of the dense operators: D[m][n] = sum over k of x[m][k] w[n][k].
//
// A workgroup computes BM x BN outputs, each of its WM x WN waves (BM / WM) x (BN / WN) of them as
// 16 x 16 MFMA tiles.  The contraction runs in steps of 128 bytes per row through two LDS buffers:
// the loads of step t + 1 go from memory into LDS without passing registers (buffer_load ... lds)
// while the matrix cores work on step t, with one barrier per step.
//
// Operand layouts.  ROWS: the operand's rows run along k (x as [M][K], w as [N][K]).  COLS (16-bit
// types only): it is stored [K][rows], and the transposing LDS read gathers the k's of a fragment.
// The order of the k's inside a fragment does not matter as long as both operands use the same, so
// 8-bit fragments are simply the 16-byte pieces l / 16 and 4 + l / 16 of a 128-byte row.
//
// LDS swizzle (in 16-byte pieces, on the source side of the load, since a load to LDS writes the
// 64 lanes' pieces in a row).  ROWS: piece c of row r at c ^ (r & 7), so that the 16 rows of a
// fragment, 128 bytes apart, meet all banks.  COLS: piece c of row k at c ^ 2 f(k), f = k's low two
// bits and bits 3-4, so that the 16 rows that one transposing read touches lie in different banks.
#pragma once

#include "fqt_dense.hpp"

namespace fqt {
namespace tile {

enum Kind { BF16K, F16K, I8K, E4M3K };
enum Layout { ROWS, COLS };

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int KB = 128;             // bytes of a row per contraction step

template <int KIND> struct Acc { typedef f32x4 type; };
template <> struct Acc<I8K> { typedef i32x4 type; };
template <int KIND> constexpr int elem_bytes = KIND == I8K || KIND == E4M3K ? 1 : 2;

// acc += w-fragment (rows of the result tile) x x-fragment (columns) over one 128-byte step, from
// the two 16-byte pieces of each.  Lane l of the result holds n = 4 (l / 16) + i, m = l % 16.
template <int KIND>
__device__ __forceinline__ void mma(typename Acc<KIND>::type &acc, const i32x4 (&w)[2], const i32x4 (&x)[2]) {
  if constexpr (KIND == BF16K) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[s]),
                                                    __builtin_bit_cast(bf16x8, x[s]), acc, 0, 0, 0);
  } else if constexpr (KIND == F16K) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w[s]),
                                                   __builtin_bit_cast(f16x8, x[s]), acc, 0, 0, 0);
  } else if constexpr (KIND == I8K) {
#pragma unroll
    for (int s = 0; s < 2; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[s], x[s], acc, 0, 0, 0);
  } else {
    // unit scales (exponent 127) and e4m3 on both sides
    const i32x8 a = __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7);
    const i32x8 b = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 0, 0, 0, 0x7F7F7F7F, 0, 0x7F7F7F7F);
  }
}

// One operand as a kernel argument: `rows` x K elements, row stride ld bytes (of a k row in COLS).
struct Operand {
  const char *p;
  int64_t ld;
  int64_t rows;
};

typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ lds_char *lds_ptr(const char *p) {
  return (lds_char *)(uint32_t)(uintptr_t)p;
}

// The loads of one operand's step: LINES rows of the tile, THREADS threads.
template <int LAYOUT, int LINES, int THREADS>
struct Loader {
  static constexpr int PIECES = LINES * KB / 16;          // 16-byte pieces of a step
  static constexpr int PER = PIECES / THREADS;
  static constexpr int ROW_PIECES = LAYOUT == ROWS ? KB / 16 : LINES / 8;
  static_assert(PIECES % THREADS == 0, "whole pieces per thread");
  const char *base;      // first byte of the next step
  int64_t step;          // bytes from one step to the next
  uint32_t off[PER];     // byte offset of each piece from base, BUF_NONE past the operand
  uint32_t kpos[PER];    // its position along k: bytes (ROWS) or rows (COLS)

  // line0: the tile's first row.
  __device__ __forceinline__ void init(const Operand &o, int64_t line0) {
    if constexpr (LAYOUT == ROWS) {
      base = o.p + line0 * o.ld;
      step = KB;
    } else {
      base = o.p + line0 * 2;
      step = (KB / 2) * o.ld;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const uint32_t p = j * THREADS + threadIdx.x;
      const uint32_t row = p / ROW_PIECES, slot = p % ROW_PIECES;
      if constexpr (LAYOUT == ROWS) {
        const uint32_t piece = slot ^ (row & 7);
        // rows past the operand read its last one: their results are not stored
        const int64_t r = min(int64_t(row), o.rows - 1 - line0);
        off[j] = uint32_t(r * o.ld) + piece * 16;
        kpos[j] = piece * 16;
      } else {
        const uint32_t f = (row & 3) | ((row >> 1) & 12);
        const uint32_t piece = slot ^ ((2 * f) & (ROW_PIECES - 1));
        off[j] = line0 + int64_t(piece) * 8 < o.rows ? uint32_t(row * o.ld) + piece * 16 : BUF_NONE;
        kpos[j] = row;
      }
    }
  }
  // left: bytes (ROWS) or rows (COLS) of the contraction that are left from here.  Pieces past it
  // are written as zeros.
  __device__ __forceinline__ void load(char *lds, int64_t left) {
    const uint32_t lim = uint32_t(min(left, int64_t(KB)));
    const __amdgpu_buffer_rsrc_t r = buffer_of(base, 0x7FFFFFFFu);
    char *at = lds + wave_id() * 1024;
#pragma unroll
    for (int j = 0; j < PER; ++j)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds_ptr(at + j * THREADS * 16), 16,
                                               kpos[j] < lim ? off[j] : BUF_NONE, 0, 0, 0);
    base += step;
  }
};

// Fragment reads of one operand's step by a wave: FRAGS tiles of 16 lines from line0.
template <int LAYOUT, int LINES, int FRAGS>
struct Reader {
  uint32_t at[LAYOUT == ROWS ? 2 : FRAGS];
  __device__ __forceinline__ void init(uint32_t line0) {
    const uint32_t l = __lane_id();
    if constexpr (LAYOUT == ROWS) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
        at[s] = (line0 + l % 16) * KB + ((s * 4 + l / 16) ^ (l & 7)) * 16;
    } else {
      // lane l points at row k = 8 (l / 16) + (l % 16) / 4, four columns from 4 (l % 4)
      const uint32_t k = 8 * (l / 16) + (l % 16) / 4, f = (k & 3) | ((k >> 1) & 12);
#pragma unroll
      for (int i = 0; i < FRAGS; ++i) {
        const uint32_t piece = (line0 / 8 + 2 * i + (l % 4) / 2) ^ ((2 * f) & (LINES / 8 - 1));
        at[i] = k * (LINES * 2) + piece * 16 + (l & 1) * 8;
      }
    }
  }
  __device__ __forceinline__ void read(const char *lds, int i, i32x4 (&o)[2]) const {
    if constexpr (LAYOUT == ROWS) {
#pragma unroll
      for (int s = 0; s < 2; ++s) o[s] = *reinterpret_cast<const i32x4 *>(lds + at[s] + i * 16 * KB);
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        typedef __attribute__((address_space(3))) i16x4 lds_v4;
        const char *p = lds + at[i] + s * 32 * LINES * 2;
        const i16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)(uint32_t)(uintptr_t)p);
        const i16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4 *)(uint32_t)(uintptr_t)(p + 4 * LINES * 2));
        typedef short i16x8 __attribute__((ext_vector_type(8)));
        const i16x8 c = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        o[s] = __builtin_bit_cast(i32x4, c);
      }
    }
  }
};

template <int BM_, int BN_, int WM_, int WN_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
  static constexpr int THREADS = 64 * WM * WN;
  static constexpr int TM = BM / WM, TN = BN / WN;        // outputs of a wave
  static constexpr int FM = TM / 16, FN = TN / 16;
  static constexpr int BUF = (BM + BN) * KB;              // bytes of one step
  static constexpr int LDS = 2 * BUF;
};

// The accumulators of the tile at (m0, n0) over the steps [t0, t1) of the contraction (K: elements
// of a row in all).  SEGS products are summed, product s from operands x[s] and w[s]: its steps
// follow those of product s - 1.
template <int KIND, int LX, int LW, typename S, int SEGS>
__device__ __forceinline__ void run_tile(const Operand (&x)[SEGS], const Operand (&w)[SEGS], int64_t K,
                                         int64_t m0, int64_t n0, int64_t t0, int64_t t1, char *lds,
                                         typename Acc<KIND>::type (&acc)[S::FM][S::FN]) {
  constexpr int64_t STEP = KB / elem_bytes<KIND>;          // elements of a step
  const int64_t steps = (K + STEP - 1) / STEP;             // of one product
  const uint32_t wave = wave_id();
  const uint32_t wm = (wave / S::WN) * S::TM, wn = (wave % S::WN) * S::TN;
  Reader<LX, S::BM, S::FM> rx;
  Reader<LW, S::BN, S::FN> rw;
  rx.init(wm);
  rw.init(wn);
#pragma unroll
  for (int i = 0; i < S::FM; ++i)
#pragma unroll
    for (int j = 0; j < S::FN; ++j) acc[i][j] = typename Acc<KIND>::type{};
  if (t0 >= t1) return;

  Loader<LX, S::BM, S::THREADS> gx;
  Loader<LW, S::BN, S::THREADS> gw;
  int seg = 0;
  int64_t t = t0;
  if constexpr (SEGS > 1) {
    seg = int(t / steps);
    t -= seg * steps;
  }
  auto start = [&](int s, int64_t at) {
    gx.init(x[s], m0);
    gw.init(w[s], n0);
    gx.base += at * gx.step;
    gw.base += at * gw.step;
  };
  auto stage = [&](int buf) {
    const int64_t left = K - t * STEP;                     // elements
    char *p = lds + buf * S::BUF;
    gx.load(p, LX == ROWS ? left * elem_bytes<KIND> : left);
    gw.load(p + S::BM * KB, LW == ROWS ? left * elem_bytes<KIND> : left);
    ++t;
    if constexpr (SEGS > 1) {
      if (t == steps && seg + 1 < SEGS) {
        t = 0;
        ++seg;
        // (the operands of one product differ from the last one's in their addresses only)
        gx.base = x[seg].p + (LX == ROWS ? m0 * x[0].ld : m0 * 2);
        gw.base = w[seg].p + (LW == ROWS ? n0 * w[0].ld : n0 * 2);
      }
    }
  };
  start(seg, t);
  stage(0);
  int buf = 0;
  for (int64_t i = t0; i < t1; ++i) {
    __builtin_amdgcn_s_waitcnt(0x0F70);                    // vmcnt(0): this step is in LDS
    __syncthreads();                                       // ... everyone's, and the other buffer is free
    if (i + 1 < t1) stage(buf ^ 1);
    const char *p = lds + buf * S::BUF;
    i32x4 fw[S::FN][2];
#pragma unroll
    for (int j = 0; j < S::FN; ++j) rw.read(p + S::BM * KB, j, fw[j]);
#pragma unroll
    for (int k = 0; k < S::FM; ++k) {
      i32x4 fx[2];
      rx.read(p, k, fx);
#pragma unroll
      for (int j = 0; j < S::FN; ++j) mma<KIND>(acc[k][j], fw[j], fx);
    }
    buf ^= 1;
  }
  __syncthreads();                                         // LDS is free for the epilogue
}

// Hands the wave's results to f(m, n, v): 8 consecutive n of one row m each, through the wave's own
// 16 x TN patch of LDS, so that a row's stores cover whole lines.
template <int KIND, typename S, typename F>
__device__ __forceinline__ void for_rows8(const typename Acc<KIND>::type (&acc)[S::FM][S::FN], char *lds,
                                          int64_t m0, int64_t n0, F &&f) {
  constexpr int PITCH = S::TN + 4;                         // floats; rows shifted against the banks
  static_assert(S::WM * S::WN * 16 * PITCH * 4 <= S::LDS, "patches fit");
  const uint32_t wave = wave_id(), l = __lane_id();
  float *patch = reinterpret_cast<float *>(lds) + wave * 16 * PITCH;
  const int64_t mw = m0 + (wave / S::WN) * S::TM, nw = n0 + (wave % S::WN) * S::TN;
  constexpr int GROUPS = 16 * S::TN / 8;                   // 8-element groups of the patch
#pragma unroll
  for (int k = 0; k < S::FM; ++k) {
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
      const typename Acc<KIND>::type a = acc[k][j];
      *reinterpret_cast<float4 *>(patch + (l % 16) * PITCH + j * 16 + 4 * (l / 16)) =
          make_float4(float(a[0]), float(a[1]), float(a[2]), float(a[3]));
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int g = 0; g < (GROUPS + 63) / 64; ++g) {
      const uint32_t q = g * 64 + l;
      if (GROUPS % 64 && q >= GROUPS) break;
      const uint32_t r = q / (S::TN / 8), c = q % (S::TN / 8) * 8;
      float v[8];
      const float4 a = *reinterpret_cast<const float4 *>(patch + r * PITCH + c);
      const float4 b = *reinterpret_cast<const float4 *>(patch + r * PITCH + c + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
      f(mw + k * 16 + r, nw + c, v);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Tile of workgroup b of nm x nn tiles.  Each XCD (b % 8) walks a contiguous run of the order below,
// which goes down GROUP tiles of m before the next n, so that the tiles an XCD has in flight share
// operand rows in its L2.
struct TileAt { uint32_t m, n; };
__device__ __forceinline__ TileAt tile_at(uint32_t b, uint32_t nm, uint32_t nn) {
  constexpr uint32_t GROUP = 8;
  const uint32_t total = nm * nn, q = total / XCDS, r = total % XCDS, x = b % XCDS;
  const uint32_t s = x * q + min(x, r) + b / XCDS;
  const uint32_t per = GROUP * nn, g = s / per, in = s % per;
  const uint32_t rows = min(GROUP, nm - g * GROUP);
  return {g * GROUP + in % rows, in / rows};
}

}  // namespace tile
}  // namespace fqt
