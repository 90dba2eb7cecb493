// Matrix-product tile of the dense operators: D[m][n] = sum over k of x[m][k] w[n][k].
//
// A workgroup computes BM x BN outputs, each of its WM x WN waves (BM / WM) x (BN / WN) of them as
// 16 x 16 MFMA tiles.  The contraction runs in steps of 128 bytes per row through two or three LDS buffers:
// the loads of later steps go from memory into LDS without passing registers (buffer_load ... lds)
// while the matrix cores work on step t.
//
// Operand layouts.  ROWS: the operand's rows run along k (x as [M][K], w as [N][K]).  COLS (16-bit
// types only): it is stored [K][rows], and the transposing LDS read gathers the k's of a fragment.
// The order of the k's inside a fragment does not matter as long as both operands use the same, so
// 8-bit fragments are simply the 16-byte pieces l / 16 and 4 + l / 16 of a 128-byte row.
//
// WIDE operands are e4m3 codes, widened to bf16 (exact) between LDS and the matrix cores, for sums in float32: half the
// bytes of bf16 copies, which are not written.
//
// SPLIT operands hold float16 pairs hi + lo in panels: panel c has the columns 32 c ... 32 c + 31 of
// all rows, 128 bytes a row, the 32 hi before the 32 lo.  A step is 32 columns; the two pieces of a
// fragment are its hi and its lo, and three matrix instructions (hi hi, hi lo, lo hi) feed on them: half
// the reads and loads of three products one after the other.  Panels make every load of a step
// contiguous, along k (PANEL_ROWS) as well as across it (PANEL_COLS: LDS rows 0-31 are the hi, 32-63 the
// lo of 32 k's).
//
// LDS swizzle (in 16-byte pieces, on the source side of the load, since a load to LDS writes the
// 64 lanes' pieces in a row).  ROWS: piece c of row r at c ^ (r & 7), so that the 16 rows of a
// fragment, 128 bytes apart, meet all banks.  COLS: piece c of row k at c ^ swizzle(k), so that the
// eight 32-byte rows that half a transposing read touches lie in different banks.
#pragma once

#include "fqt_dense.hpp"

namespace fqt {
namespace tile {

enum Kind { BF16K, SPLITK, I8K, E4M3K, WIDEK };
enum Layout { ROWS, COLS, PANEL_ROWS, PANEL_COLS };

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int KB = 128;             // bytes of a row per contraction step
constexpr bool by_rows(int layout) { return layout == ROWS || layout == PANEL_ROWS; }

template <int KIND> struct Acc { typedef f32x4 type; };
template <> struct Acc<I8K> { typedef i32x4 type; };
template <int KIND> constexpr int elem_bytes = KIND == I8K || KIND == E4M3K || KIND == WIDEK ? 1 : KIND == SPLITK ? 4 : 2;

// acc += w-fragment (rows of the result tile) x x-fragment (columns) over one 128-byte step, from
// the two 16-byte pieces of each, in mma_parts instructions.  Lane l of the result holds n = 4 (l / 16) + i, m = l % 16.
template <int KIND> constexpr int mma_parts = KIND == E4M3K ? 1 : KIND == SPLITK ? 3 : KIND == WIDEK ? 4 : 2;
// Eight codes as bf16.
__device__ __forceinline__ bf16x8 widen8(int lo, int hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(uint32_t(lo), 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(uint32_t(lo), 1.0f, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(uint32_t(hi), 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(uint32_t(hi), 1.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
template <int KIND, int PART>
__device__ __forceinline__ void mma_part(typename Acc<KIND>::type &acc, const i32x4 (&w)[2], const i32x4 (&x)[2]) {
  if constexpr (KIND == BF16K) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[PART]),
                                                  __builtin_bit_cast(bf16x8, x[PART]), acc, 0, 0, 0);
  } else if constexpr (KIND == SPLITK) {               // hi lo, lo hi, hi hi
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w[PART == 1]),
                                                 __builtin_bit_cast(f16x8, x[PART == 0]), acc, 0, 0, 0);
  } else if constexpr (KIND == WIDEK) {
    constexpr int H = PART % 2 * 2;
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8(w[PART / 2][H], w[PART / 2][H + 1]),
                                                  widen8(x[PART / 2][H], x[PART / 2][H + 1]), acc, 0, 0, 0);
  } else if constexpr (KIND == I8K) {
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[PART], x[PART], acc, 0, 0, 0);
  } else {
    // unit scales (exponent 127) and e4m3 on both sides
    const i32x8 a = __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7);
    const i32x8 b = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 0, 0, 0, 0x7F7F7F7F, 0, 0x7F7F7F7F);
  }
}
template <int KIND>
__device__ __forceinline__ void mma(typename Acc<KIND>::type &acc, const i32x4 (&w)[2], const i32x4 (&x)[2]) {
  mma_part<KIND, 0>(acc, w, x);
  if constexpr (mma_parts<KIND> > 1) mma_part<KIND, 1>(acc, w, x);
  if constexpr (mma_parts<KIND> > 2) mma_part<KIND, 2>(acc, w, x);
  if constexpr (mma_parts<KIND> > 3) mma_part<KIND, 3>(acc, w, x);
}

// One operand as a kernel argument: `rows` x K elements, row stride ld bytes (of a k row in COLS, of a
// panel in PANEL_*).
struct Operand {
  const char *p;
  int64_t ld;
  int64_t rows;
};

typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ lds_char *lds_ptr(const char *p) {
  return (lds_char *)(uint32_t)(uintptr_t)p;
}

// Swizzle of row k of a COLS step, in pieces.  Half a wave's transposing read touches 32 bytes of each of
// rows 0-3 and 8-11 (plus 16, plus 4) of 2 LINES bytes; the banks repeat after 256 bytes.  The row's
// bits 2 and 5 must not count: a lane reads rows 4 and 32 further from one address.
template <int LINES>
__device__ __forceinline__ uint32_t cols_swizzle(uint32_t k) {
  if constexpr (LINES == 64) return 2 * (((k >> 1) & 1) | ((k >> 2) & 2));     // (odd rows start mid-way)
  else return 2 * ((k & 3) | ((k >> 1) & 4));
}

// 16 bytes per lane from r at `off` to lds + 16 lane (lds wave-uniform).
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, char *lds, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, lds_ptr(lds), 16, off, 0, 0, 0);
}

// The loads of one operand's step: LINES rows of the tile, THREADS threads.
template <int LAYOUT, int LINES, int THREADS>
struct Loader {
  static constexpr int PIECES = LINES * KB / 16;          // 16-byte pieces of a step
  static constexpr int PER = PIECES / THREADS;
  static constexpr int ROW_PIECES = by_rows(LAYOUT) ? KB / 16 : LINES / 8;
  static_assert(PIECES % THREADS == 0, "whole pieces per thread");
  const char *base;      // first byte of the next step
  int64_t step;          // bytes from one step to the next
  uint32_t off[PER];     // byte offset of each piece from base, BUF_NONE past the operand
  uint32_t kpos[PER];    // its position along k: bytes (ROWS), rows (COLS); panels are whole steps

  // line0: the tile's first row.
  __device__ __forceinline__ void init(const Operand &o, int64_t line0) {
    if constexpr (LAYOUT == ROWS) {
      base = o.p + line0 * o.ld;
      step = KB;
    } else if constexpr (LAYOUT == COLS) {
      base = o.p + line0 * 2;
      step = (KB / 2) * o.ld;
    } else if constexpr (LAYOUT == PANEL_ROWS) {
      base = o.p + line0 * KB;
      step = o.ld;
    } else {
      base = o.p + line0 / 32 * o.ld;
      step = 32 * KB;
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const uint32_t p = j * THREADS + threadIdx.x;
      const uint32_t row = p / ROW_PIECES, slot = p % ROW_PIECES;
      if constexpr (by_rows(LAYOUT)) {
        const uint32_t piece = slot ^ (row & 7);
        // rows past the operand read its last one: their results are not stored
        const int64_t r = min(int64_t(row), o.rows - 1 - line0);
        off[j] = uint32_t(r * (LAYOUT == ROWS ? o.ld : KB)) + piece * 16;
        kpos[j] = LAYOUT == ROWS ? piece * 16 : 0;
      } else {
        const uint32_t piece = slot ^ cols_swizzle<LINES>(row);
        const bool in = line0 + int64_t(piece) * 8 < o.rows;
        if constexpr (LAYOUT == COLS) {
          off[j] = in ? uint32_t(row * o.ld) + piece * 16 : BUF_NONE;
          kpos[j] = row;
        } else {
          off[j] = in ? piece / 4 * uint32_t(o.ld) + row % 32 * KB + row / 32 * (KB / 2) + piece % 4 * 16 : BUF_NONE;
          kpos[j] = 0;
        }
      }
    }
  }
  // left: bytes (ROWS) or rows (COLS) of the contraction that are left from here.  Pieces past it
  // are written as zeros.
  template <int FROM, int TO>
  __device__ __forceinline__ void load(char *lds, int64_t left) {
    const uint32_t lim = uint32_t(max(int64_t(0), min(left, int64_t(KB))));
    const __amdgpu_buffer_rsrc_t r = buffer_of(base, 0x7FFFFFFFu);
    char *at = lds + wave_id() * 1024;
#pragma unroll
    for (int j = FROM; j < TO; ++j)
      load_to_lds(r, at + j * THREADS * 16, kpos[j] < lim ? off[j] : BUF_NONE);
    if (TO == PER) base += step;
  }
};

// Two fragments of a COLS operand by transposing reads, from the lane's addresses a and b, as one block
// of assembly with its own wait.  For its own reads of this kind the compiler waits until every load to LDS in flight
// has arrived, though those fill other buffers; where one tile's step has to hide the next one's loads
// (run_tile) that costs more than the closer wait: 128 x 128 tiles of 8192 x 8192 x 4096 in 501 instead
// of 566 us.
template <int LINES>
__device__ __forceinline__ void read_cols(const char *a, const char *b, i32x4 (&x)[2], i32x4 (&y)[2]) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  i32x2 r[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n"
      "ds_read_b64_tr_b16 %1, %8 offset:%10\n"
      "ds_read_b64_tr_b16 %2, %8 offset:%11\n"
      "ds_read_b64_tr_b16 %3, %8 offset:%12\n"
      "ds_read_b64_tr_b16 %4, %9\n"
      "ds_read_b64_tr_b16 %5, %9 offset:%10\n"
      "ds_read_b64_tr_b16 %6, %9 offset:%11\n"
      "ds_read_b64_tr_b16 %7, %9 offset:%12\n"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"((uint32_t)(uintptr_t)a), "v"((uint32_t)(uintptr_t)b), "i"(4 * LINES * 2), "i"(32 * LINES * 2),
        "i"(36 * LINES * 2)
      : "memory");
  x[0] = __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3);
  x[1] = __builtin_shufflevector(r[2], r[3], 0, 1, 2, 3);
  y[0] = __builtin_shufflevector(r[4], r[5], 0, 1, 2, 3);
  y[1] = __builtin_shufflevector(r[6], r[7], 0, 1, 2, 3);
}

// The same for four fragments, from the lane's addresses a[0 ... 3].
template <int LINES>
__device__ __forceinline__ void read_cols4(const char *lds, const uint32_t *a, i32x4 (&o)[4][2]) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  i32x2 r[16];
  const uint32_t at = (uint32_t)(uintptr_t)lds;
  asm volatile(
      "ds_read_b64_tr_b16 %0, %16\n"
      "ds_read_b64_tr_b16 %1, %16 offset:%20\n"
      "ds_read_b64_tr_b16 %2, %16 offset:%21\n"
      "ds_read_b64_tr_b16 %3, %16 offset:%22\n"
      "ds_read_b64_tr_b16 %4, %17\n"
      "ds_read_b64_tr_b16 %5, %17 offset:%20\n"
      "ds_read_b64_tr_b16 %6, %17 offset:%21\n"
      "ds_read_b64_tr_b16 %7, %17 offset:%22\n"
      "ds_read_b64_tr_b16 %8, %18\n"
      "ds_read_b64_tr_b16 %9, %18 offset:%20\n"
      "ds_read_b64_tr_b16 %10, %18 offset:%21\n"
      "ds_read_b64_tr_b16 %11, %18 offset:%22\n"
      "ds_read_b64_tr_b16 %12, %19\n"
      "ds_read_b64_tr_b16 %13, %19 offset:%20\n"
      "ds_read_b64_tr_b16 %14, %19 offset:%21\n"
      "ds_read_b64_tr_b16 %15, %19 offset:%22\n"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]),
        "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
      : "v"(at + a[0]), "v"(at + a[1]), "v"(at + a[2]), "v"(at + a[3]), "i"(4 * LINES * 2), "i"(32 * LINES * 2),
        "i"(36 * LINES * 2)
      : "memory");
#pragma unroll
  for (int f = 0; f < 4; ++f) {
    o[f][0] = __builtin_shufflevector(r[4 * f], r[4 * f + 1], 0, 1, 2, 3);
    o[f][1] = __builtin_shufflevector(r[4 * f + 2], r[4 * f + 3], 0, 1, 2, 3);
  }
}

// Fragment reads of one operand's step by a wave: FRAGS tiles of 16 lines from line0.
template <int LAYOUT, int LINES, int FRAGS>
struct Reader {
  uint32_t at[by_rows(LAYOUT) ? 2 : FRAGS];
  __device__ __forceinline__ void init(uint32_t line0) {
    const uint32_t l = __lane_id();
    if constexpr (by_rows(LAYOUT)) {
#pragma unroll
      for (int s = 0; s < 2; ++s)
        at[s] = (line0 + l % 16) * KB + ((s * 4 + l / 16) ^ (l & 7)) * 16;
    } else {
      // lane l points at row k = 8 (l / 16) + (l % 16) / 4, four columns from 4 (l % 4)
      const uint32_t k = 8 * (l / 16) + (l % 16) / 4;
#pragma unroll
      for (int i = 0; i < FRAGS; ++i) {
        const uint32_t piece = (line0 / 8 + 2 * i + (l % 4) / 2) ^ cols_swizzle<LINES>(k);
        at[i] = k * (LINES * 2) + piece * 16 + (l & 1) * 8;
      }
    }
  }
  // Fragments i ... i + 3, COLS ones with their own wait.
  __device__ __forceinline__ void read4(const char *lds, int i, i32x4 (&o)[4][2]) const {
    if constexpr (by_rows(LAYOUT)) read(lds, i, o);
    else read_cols4<LINES>(lds, at + i, o);
  }
  // Fragments i ... i + N - 1, COLS ones in pairs with their own wait.
  template <int N>
  __device__ __forceinline__ void read(const char *lds, int i, i32x4 (&o)[N][2]) const {
    if constexpr (by_rows(LAYOUT)) {
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int s = 0; s < 2; ++s)
          o[j][s] = *reinterpret_cast<const i32x4 *>(lds + at[s] + (i + j) * 16 * KB);
    } else {
      static_assert(N % 2 == 0, "fragments in pairs");
#pragma unroll
      for (int j = 0; j < N; j += 2) read_cols<LINES>(lds + at[i + j], lds + at[i + j + 1], o[j], o[j + 1]);
    }
  }
};

// The steps [t0, t1) of one operand.  Steps past the last are loaded as zeros without touching memory,
// so that the count of loads in flight is the same in every step.
template <int KIND, int LAYOUT, int LINES, int THREADS>
struct Feed {
  typedef Loader<LAYOUT, LINES, THREADS> L;
  static constexpr int64_t STEP = KB / elem_bytes<KIND>;   // elements of a step
  static constexpr int UNIT = LAYOUT == ROWS ? elem_bytes<KIND> : 1;
  L g;
  int64_t left, todo;      // elements from here on, steps to load
  __device__ __forceinline__ void init(const Operand &o, int64_t K, int64_t line0, int64_t t0, int64_t t1) {
    g.init(o, line0);
    g.base += t0 * g.step;
    left = K - t0 * STEP;
    todo = t1 - t0;
  }
  __device__ __forceinline__ void load(char *lds) {
    g.template load<0, L::PER>(lds, todo > 0 ? left * UNIT : 0);
    --todo;
    left -= STEP;
  }
};

// BM x BN outputs by WM x WN waves, through BUFS step buffers (XBUFS of x).
template <int BM_, int BN_, int WM_, int WN_, int BUFS_ = 2, int XBUFS_ = BUFS_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, BUFS = BUFS_;
  static constexpr int THREADS = 64 * WM * WN;
  static constexpr int TM = BM / WM, TN = BN / WN;        // outputs of a wave
  static constexpr int FM = TM / 16, FN = TN / 16;
  static constexpr int BUF = (BM + BN) * KB;              // bytes of one step
  static constexpr int LDS = (XBUFS_ * BM + BUFS * BN) * KB;
};

// A barrier of the workgroup that waits for nothing else: what has to be complete is waited for by
// name.
__device__ __forceinline__ void barrier_only() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
template <int N>
__device__ __forceinline__ void wait_loads() {             // all but the last N loads are complete
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0F70);
}
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }

template <int KIND, typename S>
__device__ __forceinline__ void clear_acc(typename Acc<KIND>::type (&acc)[S::FM][S::FN]) {
#pragma unroll
  for (int i = 0; i < S::FM; ++i)
#pragma unroll
    for (int j = 0; j < S::FN; ++j) acc[i][j] = typename Acc<KIND>::type{};
}

// The accumulators of the tile at (m0, n0) over the steps [t0, t1) of the contraction.  BUFS - 1
// steps are in flight; one barrier per step, after which the step is in LDS for everyone and the
// buffer of the step before it is free.
template <int KIND, int LX, int LW, typename S>
__device__ __forceinline__ void run_tile(const Operand &x, const Operand &w, int64_t K,
                                         int64_t m0, int64_t n0, int64_t t0, int64_t t1, char *lds,
                                         typename Acc<KIND>::type (&acc)[S::FM][S::FN]) {
  const uint32_t wave = wave_id();
  Reader<LX, S::BM, S::FM> rx;
  Reader<LW, S::BN, S::FN> rw;
  rx.init((wave / S::WN) * S::TM);
  rw.init((wave % S::WN) * S::TN);
  clear_acc<KIND, S>(acc);
  if (t0 >= t1) return;
  Feed<KIND, LX, S::BM, S::THREADS> gx;
  Feed<KIND, LW, S::BN, S::THREADS> gw;
  gx.init(x, K, m0, t0, t1);
  gw.init(w, K, n0, t0, t1);
  constexpr int AHEAD = S::BUFS - 1, LOADS = gx.g.PER + gw.g.PER;
#pragma unroll
  for (int b = 0; b < AHEAD; ++b) {
    gx.load(lds + b * S::BUF);
    gw.load(lds + b * S::BUF + S::BM * KB);
  }
  char *at = lds, *to = lds + AHEAD * S::BUF;
  auto next = [&](char *p) { return p == lds + (S::BUFS - 1) * S::BUF ? lds : p + S::BUF; };
  for (int64_t i = t0; i < t1; ++i) {
    wait_lds();                                            // the step before is read
    wait_loads<(AHEAD - 1) * LOADS>();
    // (not barrier_only: matrix instructions of the last step may be issued behind the barrier)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    gx.load(to);
    gw.load(to + S::BM * KB);
    i32x4 fw[S::FN][2];
    rw.read(at + S::BM * KB, 0, fw);
    constexpr int XS = by_rows(LX) ? 1 : 2;                // x fragments read at a time
#pragma unroll
    for (int k = 0; k < S::FM; k += XS) {
      i32x4 fx[XS][2];
      rx.read(at, k, fx);
#pragma unroll
      for (int i = 0; i < XS; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) mma<KIND>(acc[k + i][j], fw[j], fx[i]);
    }
    at = next(at);
    to = next(to);
  }
  wait_loads<0>();
  __syncthreads();                                         // LDS is free for the epilogue
}

// The same for workgroups of eight waves, two per SIMD, with 256 or so outputs a side: while one wave
// of a SIMD issues matrix instructions, the other one reads fragments and starts loads.  Waves 4-7
// run one barrier behind waves 0-3 for that.  A step is two halves of a wave's tile, each a
// reading phase and a matrix phase of 512 cycles with a barrier after it:
//   half   fragments read          step loaded
//   0      x, first half; w        x of step t + 2, into the third buffer
//   1      x, second half          w of step t + 2, into this buffer (w is read by now)
// so that x has eight, w six phases to arrive.  A wave waits for its own loads at the end of the reading
// phase before the one that needs them, and the barrier between makes them everyone's.  A step takes 1.37 us (2048
// cycles of matrix instructions, at the 1.8 to 1.9 GHz that the power limit leaves; 76 % busy in long products).  Quarters
// (phases of 256 cycles, shorter than a reading phase) took 1.58, and 1.9 with operands across the contraction.
template <int KIND, int LX, int LW, typename S>
__device__ __forceinline__ void run_tile8(const Operand &x, const Operand &w, int64_t K,
                                          int64_t m0, int64_t n0, int64_t t0, int64_t t1, char *lds,
                                          typename Acc<KIND>::type (&acc)[S::FM][S::FN]) {
  static_assert(S::THREADS == 512 && S::FM == 8 && S::FN == 4 && S::LDS == (3 * S::BM + 2 * S::BN) * KB, "tiles in halves");
  const uint32_t wave = wave_id();
  Reader<LX, S::BM, S::FM> rx;
  Reader<LW, S::BN, S::FN> rw;
  rx.init((wave / S::WN) * S::TM);
  rw.init((wave % S::WN) * S::TN);
  clear_acc<KIND, S>(acc);
  if (t0 >= t1) return;
  Feed<KIND, LX, S::BM, S::THREADS> gx;
  Feed<KIND, LW, S::BN, S::THREADS> gw;
  gx.init(x, K, m0, t0, t1);
  gw.init(w, K, n0, t0, t1);
  constexpr int NX = gx.g.PER, NW = gw.g.PER;
  constexpr uint32_t XBUF = S::BM * KB, WBUF = S::BN * KB;
  char *const xs = lds, *const ws = lds + 3 * XBUF;
  gw.load(ws);
  gx.load(xs);
  gw.load(ws + WBUF);
  gx.load(xs + XBUF);
  wait_loads<NX + NW>();
  barrier_only();
  if (wave >= 4) barrier_only();
  i32x4 fx[4][2], fw[4][2];
  auto half = [&](int m) {
    wait_lds();
    barrier_only();
    __builtin_amdgcn_s_setprio(1);
    auto part = [&]<int P>() {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) mma_part<KIND, P>(acc[m + i][j], fw[j], fx[i]);
    };
    part.template operator()<0>();
    if constexpr (mma_parts<KIND> > 1) part.template operator()<1>();
    if constexpr (mma_parts<KIND> > 2) part.template operator()<2>();
    if constexpr (mma_parts<KIND> > 3) part.template operator()<3>();
    __builtin_amdgcn_s_setprio(0);
    barrier_only();
  };
  char *xat = xs, *xto = xs + 2 * XBUF, *wat = ws;
  for (int64_t t = t0; t < t1; ++t) {
    rx.read4(xat, 0, fx);
    rw.read4(wat, 0, fw);
    gx.load(xto);
    half(0);
    rx.read4(xat, 4, fx);
    gw.load(wat);
    wait_loads<NX + NW>();                                 // both of step t + 1
    half(4);
    xto = xat;
    xat = xat == xs + 2 * XBUF ? xs : xat + XBUF;
    wat = wat == ws ? ws + WBUF : ws;
  }
  if (wave < 4) barrier_only();
  wait_loads<0>();
  __syncthreads();                                         // LDS is free for the epilogue
}

// Orders the LDS accesses of a wave's lanes for the compiler (the hardware keeps a wave's in order).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Takes a wave's results through the epilogue e, 8 consecutive n of one row m at a time, by way of the
// wave's own 16 x TN patch of LDS, so that a row's stores cover whole lines.  A lane keeps its columns:
//   e.columns(n)              called first: what depends on the columns alone
//   e.fetch(m, n)             what the epilogue reads for a group; DEPTH groups are under way, since
//                             the latency of one after the other would cost as much as a third of a
//                             product over 64 steps
//   e.finish(m, n, v, f)      the group's sums v and its fetch f
//   e.mirror(n, m, v)         E::MIRROR only: 8 finished values of column n from row m on
// E::SUMS takes the accumulators' words as they are (int32 sums of 8-bit products stay exact); the others
// get them as float32.
template <int KIND, typename S, typename E>
__device__ __forceinline__ void run_epilogue(const typename Acc<KIND>::type (&acc)[S::FM][S::FN], char *lds,
                                             int64_t m0, int64_t n0, E &&e) {
  constexpr int PITCH = S::TN + 4;                         // floats; rows shifted against the banks
  static_assert(S::WM * S::WN * 16 * PITCH * 4 <= S::LDS, "patches fit");
  constexpr int PER_ROW = S::TN / 8, ROWS_AT_ONCE = 64 / PER_ROW, G = 16 / ROWS_AT_ONCE;
  static_assert(PER_ROW * ROWS_AT_ONCE == 64 && G >= 1, "a lane keeps its columns");
  typedef typename std::remove_reference_t<E>::Fetch Fetch;
  constexpr int ALL = S::FM * G, DEPTH = ALL < std::remove_reference_t<E>::DEPTH ? ALL : std::remove_reference_t<E>::DEPTH;
  const uint32_t wave = wave_id(), l = __lane_id();
  float *patch = reinterpret_cast<float *>(lds) + wave * 16 * PITCH;
  const uint32_t r = l / PER_ROW, c = l % PER_ROW * 8;
  const int64_t m = m0 + (wave / S::WN) * S::TM + r, n = n0 + (wave % S::WN) * S::TN + c;
  e.columns(n);
  Fetch q[DEPTH];
#pragma unroll
  for (int i = 0; i < DEPTH; ++i) q[i] = e.fetch(m + i * ROWS_AT_ONCE, n);
#pragma unroll
  for (int k = 0; k < S::FM; ++k) {
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
      f32x4 a;
      if constexpr (std::remove_reference_t<E>::SUMS) a = __builtin_bit_cast(f32x4, acc[k][j]);
      else a = __builtin_convertvector(acc[k][j], f32x4);
      *reinterpret_cast<f32x4 *>(patch + (l % 16) * PITCH + j * 16 + 4 * (l / 16)) = a;
    }
    wave_fence();
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int i = k * G + g;
      float v[8];
      const float4 a = *reinterpret_cast<const float4 *>(patch + (g * ROWS_AT_ONCE + r) * PITCH + c);
      const float4 b = *reinterpret_cast<const float4 *>(patch + (g * ROWS_AT_ONCE + r) * PITCH + c + 4);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
      v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
      const Fetch f = q[i % DEPTH];
      if (i + DEPTH < ALL) q[i % DEPTH] = e.fetch(m + (i + DEPTH) * ROWS_AT_ONCE, n);
      e.finish(m + i * ROWS_AT_ONCE, n, v, f);
      if constexpr (std::remove_reference_t<E>::MIRROR) {
        float *p = patch + (g * ROWS_AT_ONCE + r) * PITCH + c;
        *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
      }
    }
    wave_fence();
    if constexpr (std::remove_reference_t<E>::MIRROR) {
#pragma unroll
      for (int h = 0; h < S::TN / 32; ++h) {
        const uint32_t i = h * 64 + l, col = i % S::TN, half = i / S::TN * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = patch[(half + j) * PITCH + col];
        e.mirror(n - c + col, m - r + k * 16 + half, v);
      }
      wave_fence();
    }
  }
}
// Partial sums of a split contraction: rows of ld (a multiple of 8) words, int32 or float32.
struct StorePart {
  static constexpr int DEPTH = 1;
  static constexpr bool MIRROR = false, SUMS = true;
  struct Fetch {};
  float *part;
  int64_t M, ld;
  __device__ __forceinline__ void columns(int64_t) {}
  __device__ __forceinline__ Fetch fetch(int64_t, int64_t) { return {}; }
  __device__ __forceinline__ void finish(int64_t m, int64_t n, float (&v)[8], const Fetch &) {
    if (m < M && n < ld) dense::store8f(part + m * ld + n, 8, v);
  }
};

// ----------------------------------------------------------------------------- plans
// The shapes of a workgroup's tile.
using Large = Shape<256, 256, 2, 4, 2, 3>;
using Middle = Shape<128, 128, 2, 2>;
using Small = Shape<64, 64, 2, 2, 3>;
enum ShapeId { LARGE, MIDDLE, SMALL };
template <int SHAPE> struct ShapeOf;
template <> struct ShapeOf<LARGE> { typedef Large type; };
template <> struct ShapeOf<MIDDLE> { typedef Middle type; };
template <> struct ShapeOf<SMALL> { typedef Small type; };
constexpr int EDGES[] = {Large::BM, Middle::BM, Small::BM}, SHAPE_THREADS[] = {Large::THREADS, Middle::THREADS, Small::THREADS};

// One launch of a product: `count` tiles from tile `first` on, of an order over nm x nn tiles or,
// symmetric, over the tiles on and above the diagonal.  parts: workgroups take sixteenths (Small) of
// the tiles of a Large grid, for the tiles that a last round of workgroups would leave most CUs idle
// with: 32 Large tiles over 64 steps take 104 us, their 512 parts 26 (30-35 in a call, after the Large ones).
struct Tiles {
  uint32_t nm, nn, first, count;
  uint32_t splits;         // pieces of the contraction, each `steps` long
  uint32_t steps;
  int32_t symmetric, parts;
};
struct Plan {
  int shape[2];
  Tiles t[2];
  int launches;
  uint32_t splits;
  double us;               // what the costs below make of it
};

// us a step of a workgroup with one, two or three of them on a CU, and us before the first and after the last
// step with Large, Middle and Small tiles: measured on bf16 operands, on pairs as PANEL_ROWS x PANEL_COLS
// (512 and 1024 rows) and on symmetric products of pairs (512 to 4096 rows).  (DENSE_COSTS of
// Large tiles with the loop in quarters: kept, so that the plans of the linear products, and with them the order of sums, stay
// as they were.)  8-bit operands and the backward's
// layouts are planned with the bf16 costs, not measured apart: a step is the same bytes, but 8-bit matrix
// instructions run faster and reads across the contraction slower (6 to 11 %).
struct Costs { double large[1], middle[2], small[3], start[3]; };
constexpr Costs DENSE_COSTS{{1.58}, {0.60, 0.90}, {0.25, 0.40, 0.58}, {6, 5, 4}},
    // with the loop as it is: 2000 x 20000 x 2000 bf16 in 157 us, with DENSE_COSTS' choice of tiles in 197
    STEP_COSTS{{1.45}, {0.60, 0.90}, {0.25, 0.40, 0.58}, {6, 5, 4}},
    PAIR_COSTS{{2.0}, {0.81, 1.26}, {0.28, 0.39, 0.62}, {18, 8, 5}},
    SYMMETRIC_COSTS{{2.0}, {0.81, 1.15}, {0.28, 0.40, 0.75}, {10, 8, 4}};

// Workgroups of a launch.
inline uint64_t blocks_of(const Tiles &t) { return uint64_t(t.count) * t.splits * (t.parts ? 16 : 1); }
// Whether a launch counts its threads in 32 bits.
inline bool launchable(const Plan &p) {
  for (int i = 0; i < p.launches; ++i)
    if (blocks_of(p.t[i]) * SHAPE_THREADS[p.shape[i]] >> 32) return false;
  return true;
}
// Large tiles that cover M x N.
inline uint64_t large_tiles(int64_t M, int64_t N) {
  return uint64_t((M + Large::BM - 1) / Large::BM) * uint64_t((N + Large::BN - 1) / Large::BN);
}
constexpr uint64_t MOST_LARGE = 1ull << 23;                // fewer than this are one launch

inline void describe(const Plan &p, fqt_product_plan *o) {
  *o = {};
  o->launches = p.launches;
  o->splits = int32_t(p.splits);
  for (int i = 0; i < p.launches; ++i) {
    o->tile[i] = p.t[i].parts ? Small::BM : EDGES[p.shape[i]];
    o->threads[i] = SHAPE_THREADS[p.shape[i]];
    o->workgroups[i] = int64_t(blocks_of(p.t[i]));
  }
}

// The cheapest plan that can be launched; products of fewer than MOST_LARGE tiles have one.  most: the most pieces
// of the contraction.
inline Plan make_plan(int64_t M, int64_t N, int64_t steps, bool symmetric, const Costs &costs, int64_t most = 64) {
  auto grid = [&](int64_t b) {
    Tiles t{};
    t.nm = uint32_t((M + b - 1) / b);
    t.nn = uint32_t((N + b - 1) / b);
    t.count = symmetric ? t.nm * (t.nm + 1) / 2 : t.nm * t.nn;
    t.splits = 1;
    t.steps = uint32_t(steps);
    t.symmetric = symmetric;
    return t;
  };
  Plan best{};
  double cost = 1e30;
  auto take = [&](double c, const Plan &p) {
    if (c < cost && launchable(p)) cost = c, best = p, best.us = c;
  };
  const double s = double(steps);
  const double entries = double(M) * double(N) * (symmetric ? 0.5 : 1.0);
  // us of `blocks` workgroups of `n` steps, `cu` of which fit a CU
  auto run = [](uint64_t blocks, double n, int cu, const double *step, double start) {
    const uint64_t full = 256 * cu, rest = blocks % full;
    double c = double(blocks / full) * (step[cu - 1] * n + start);
    if (rest) c += step[(rest - 1) / 256] * n + start;
    return c;
  };
  const double launch = 3;
  {
    const Tiles t = grid(256);
    const uint32_t tail = t.count % 256;
    if (tail && t.count > 256) {
      Plan p{{LARGE, SMALL}, {t, t}, 2, 1};
      p.t[0].count = t.count - tail;
      p.t[1].first = t.count - tail;
      p.t[1].count = tail;
      p.t[1].parts = 1;
      take(run(p.t[0].count, s, 1, costs.large, costs.start[0]) + run(16 * tail, s, 3, costs.small, costs.start[2]) + 2 * launch, p);
    }
  }
  auto split = [&](int shape, int64_t b, int cu, const double *step, double start) {
    const Tiles g = grid(b);
    for (int64_t n = 1; n <= most && (n == 1 || steps / n >= 4); n += n < 16 ? 1 : 8) {
      Tiles t = g;
      t.steps = uint32_t(std::max<int64_t>(1, (steps + n - 1) / n));
      t.splits = uint32_t(std::max<int64_t>(1, (steps + t.steps - 1) / t.steps));
      double c = run(blocks_of(t), t.steps, cu, step, start) + launch;
      // the partial sums, written and read at 4 TB/s one split after the other, and their launch
      if (t.splits > 1) c += 4 + 0.2 * t.splits + t.splits * entries * 8 / 4e6;
      take(c, Plan{{shape, shape}, {t, t}, 1, t.splits});
    }
  };
  split(LARGE, 256, 1, costs.large, costs.start[0]);
  split(MIDDLE, 128, 2, costs.middle, costs.start[1]);
  split(SMALL, 64, 3, costs.small, costs.start[2]);
  return best;
}

// Where workgroup b of a launch works.
struct Place {
  int64_t m0, n0;
  uint32_t split;
  bool diagonal;           // of a symmetric product: the tile is its own mirror image
};
// Each XCD (b % 8) walks a contiguous run of the order below, which goes down GROUP tiles of m before
// the next n, one split after the other, so that the tiles an XCD has in flight share operand rows and
// their piece of the contraction in its L2 (512 x 512 x 25088 bf16: 26 us; each split over all XCDs 40).
template <int SHAPE>
__device__ __forceinline__ Place place(const Tiles &t, uint32_t b) {
  typedef typename ShapeOf<SHAPE>::type S;
  const uint32_t parts = SHAPE == SMALL && t.parts ? 16 : 1;
  const uint32_t total = t.count * parts, all = total * t.splits;
  const uint32_t q = all / XCDS, r = all % XCDS, x = b % XCDS;
  uint32_t s = x * q + min(x, r) + b / XCDS;
  const uint32_t split = s / total;
  s %= total;
  const uint32_t part = s % parts;
  s = s / parts + t.first;
  uint32_t m, n;
  if (t.symmetric) {       // by columns of the upper triangle
    n = uint32_t((sqrtf(8.0f * float(s) + 1.0f) - 1.0f) * 0.5f);
    while (n * (n + 1) / 2 > s) --n;
    while ((n + 1) * (n + 2) / 2 <= s) ++n;
    m = s - n * (n + 1) / 2;
  } else {
    constexpr uint32_t GROUP = 8;
    const uint32_t per = GROUP * t.nn, g = s / per, in = s % per;
    const uint32_t rows = min(GROUP, t.nm - g * GROUP);
    m = g * GROUP + in % rows;
    n = in / rows;
  }
  if (parts > 1) return {int64_t(m) * 256 + part / 4 * 64, int64_t(n) * 256 + part % 4 * 64, split, m == n};
  return {int64_t(m) * S::BM, int64_t(n) * S::BN, split, m == n};
}

// The accumulators of a placed tile, by the loop that suits the shape.
template <int KIND, int LX, int LW, int SHAPE, typename S>
__device__ __forceinline__ void contract(const Operand &x, const Operand &w, int64_t K,
                                         const Place &at, const Tiles &t, char *lds,
                                         typename Acc<KIND>::type (&acc)[S::FM][S::FN]) {
  constexpr int64_t STEP = KB / elem_bytes<KIND>;
  const int64_t total = (K + STEP - 1) / STEP;
  const int64_t t0 = int64_t(at.split) * t.steps, t1 = min(total, t0 + t.steps);
  if constexpr (SHAPE == LARGE) run_tile8<KIND, LX, LW, S>(x, w, K, at.m0, at.n0, t0, t1, lds, acc);
  else run_tile<KIND, LX, LW, S>(x, w, K, at.m0, at.n0, t0, t1, lds, acc);
}
// Calls f.template operator()<SHAPE>(tiles) for each launch of a plan.
template <typename F>
inline void for_launches(const Plan &p, F &&f) {
  for (int i = 0; i < p.launches; ++i) {
    if (p.t[i].count == 0) continue;
    switch (p.shape[i]) {
      case LARGE: f.template operator()<LARGE>(p.t[i]); break;
      case MIDDLE: f.template operator()<MIDDLE>(p.t[i]); break;
      default: f.template operator()<SMALL>(p.t[i]);
    }
  }
}

}  // namespace tile
}  // namespace fqt
