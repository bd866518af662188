// Rows to 8-bit integers (k_quant_rows) and the seam between two blocks (k_norm_residual): the operands of the 8-bit
// linear layers.
//
// A row v becomes q = nearest-even(v / s) with one scale s = max(max |v| / 127, 2^-126), rounded once to fp32.  The
// nearest integer is decided exactly: for rows that come as numbers (k_quant_rows) on the quotient itself, for rows
// that are computed (k_norm_residual) on values held in 64 bits.  A row's sums are added in one order, however many rows
// a launch has, so that a row's bits do not depend on the other rows.
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace fb {
namespace {

// 16 and 8 bytes on any address: rows of odd length start anywhere.
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(1)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(1)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

constexpr float kTinyScale = 1.17549435e-38f;   // 2^-126
constexpr uint32_t kInf = 0x7f800000u;

// Elements c .. c + 7 of a row of n, zero past its end (TAIL: n % 8 != 0, so that a piece may end early).  A piece that
// ends early comes from the row's last eight elements, moved down: one load in the place of up to seven, which a whole
// wave would wait for.  Nothing outside the row is read (but the other half of a word that holds one of its elements).
template <bool TAIL>
__device__ __forceinline__ void load8(const float *p, int c, int n, float (&v)[8]) {
  if (TAIL && n < 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[min(c + i, n - 1)];   // all on their way at once
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < n ? v[i] : 0.f;
    return;
  }
  const float *at = p + (TAIL ? min(c, n - 8) : c);
  const f32x4u a = *reinterpret_cast<const f32x4u *>(at), b = *reinterpret_cast<const f32x4u *>(at + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
  if (TAIL && c + 8 > n) {
    const int by = c + 8 - n;
#pragma unroll
    for (int s = 4; s > 0; s >>= 1)
      if (by & s) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i + s < 8 ? v[i + s] : 0.f;
      }
  }
}
// The same of a row of bf16, as it is stored.  Rows of odd length start off 4 bytes, which a load of 16 bytes pays for several
// times over: those come from the five words around them.
template <bool TAIL>
__device__ __forceinline__ u32x4 raw8(const bf16 *p, int c, int n) {
  if constexpr (!TAIL) return *reinterpret_cast<const u32x4u *>(p + c);
  if (n < 8) {
    u32x4 v = {0, 0, 0, 0};
    uint32_t e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = __builtin_bit_cast(uint16_t, p[min(c + j, n - 1)]);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j >> 1] |= c + j < n ? e[j] << (16 * (j & 1)) : 0u;
    return v;
  }
  typedef uint32_t words __attribute__((ext_vector_type(4), aligned(4)));
  const uintptr_t at = (uintptr_t)(p + min(c, n - 8));
  const u32x4 w = *reinterpret_cast<const words *>(at & ~(uintptr_t)3);
  const uint32_t last = *reinterpret_cast<const uint32_t *>((at + 15) & ~(uintptr_t)3), by = (uint32_t)at & 3;
  u32x4 v = {__builtin_amdgcn_alignbyte(w[1], w[0], by), __builtin_amdgcn_alignbyte(w[2], w[1], by),
             __builtin_amdgcn_alignbyte(w[3], w[2], by), __builtin_amdgcn_alignbyte(last, w[3], by)};
  if (c + 8 > n) {
    const int s = 16 * (c + 8 - n);   // 16 .. 112
    typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
    const u64x2 d = __builtin_bit_cast(u64x2, v);
    const uint64_t far = d[1] >> (s & 63);
    v = __builtin_bit_cast(u32x4, s >= 64 ? u64x2{far, 0} : u64x2{d[0] >> s | d[1] << (64 - s), far});
  }
  return v;
}
__device__ __forceinline__ float half_of(u32x4 v, int j) {
  return __builtin_bit_cast(float, j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16);
}
template <bool TAIL>
__device__ __forceinline__ void load8(const bf16 *p, int c, int n, float (&v)[8]) {
  const u32x4 a = raw8<TAIL>(p, c, n);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = half_of(a, i);
}
// Eight elements as they are stored.
template <typename T> struct Piece;
template <> struct Piece<float> {
  float v[8];
  template <bool TAIL> __device__ __forceinline__ void load(const float *p, int c, int n) { load8<TAIL>(p, c, n, v); }
  __device__ __forceinline__ float operator[](int j) const { return v[j]; }
};
template <> struct Piece<bf16> {
  u32x4 v;
  template <bool TAIL> __device__ __forceinline__ void load(const bf16 *p, int c, int n) { v = raw8<TAIL>(p, c, n); }
  __device__ __forceinline__ float operator[](int j) const { return half_of(v, j); }
};
template <bool TAIL, bool NT = false>
__device__ __forceinline__ void store8(float *p, int c, int n, const float (&v)[8]) {
  if (!TAIL || c + 8 <= n) {
    const f32x4u a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
    if constexpr (NT) {   // past the caches
      __builtin_nontemporal_store(a, reinterpret_cast<f32x4u *>(p + c));
      __builtin_nontemporal_store(b, reinterpret_cast<f32x4u *>(p + c + 4));
    } else {
      *reinterpret_cast<f32x4u *>(p + c) = a;
      *reinterpret_cast<f32x4u *>(p + c + 4) = b;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) p[c + i] = v[i];
  }
}
template <bool TAIL>
__device__ __forceinline__ void store8(bf16 *p, int c, int n, const float (&v)[8]) {
  if (!TAIL || c + 8 <= n) {
    const bf16x8 w = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3], (bf16)v[4], (bf16)v[5], (bf16)v[6], (bf16)v[7]};
    *reinterpret_cast<u32x4u *>(p + c) = __builtin_bit_cast(u32x4, w);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) p[c + i] = (bf16)v[i];
  }
}
// Eight codes, each in byte AT of a word; zeros for a row without a scale.
template <bool TAIL, int AT>
__device__ __forceinline__ void store_codes(int8_t *p, int c, int n, const uint32_t (&q)[8], bool bad) {
  if (!TAIL || c + 8 <= n) {
    u32x2u w;
    constexpr uint32_t two = 0x0c0c0400 + 0x0101 * AT;
#pragma unroll
    for (int i = 0; i < 2; ++i) {   // the bytes of a pair, then the two halves
      const uint32_t lo = __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], two), hi = __builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], two);
      w[i] = bad ? 0u : __builtin_amdgcn_perm(hi, lo, 0x05040100);
    }
    *reinterpret_cast<u32x2u *>(p + c) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) p[c + i] = bad ? (int8_t)0 : (int8_t)(q[i] >> (8 * AT));
  }
}

// Reductions over the 16, 32 or 64 lanes that share a row, by moves between lanes rather than through LDS (a step of
// which waits some hundred cycles: with the vectors read early one token of 1536 takes 3.9 us in place of 4.8).  In a group of
// 2, 4 and 8 lanes that already hold their result the mirrored lane belongs to the other half of the next larger one; rows
// of 16 and halves of 32 lanes come together by gfx950's swaps.  Both sides of an exchange add the same two numbers.
template <int CTRL> __device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL> __device__ __forceinline__ double moved(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)moved<CTRL>((uint32_t)(u >> 32)) << 32 | moved<CTRL>((uint32_t)u));
}
template <bool WIDE> __device__ __forceinline__ void both(uint32_t v, uint32_t &a, uint32_t &b) {
  const auto r = WIDE ? __builtin_amdgcn_permlane32_swap(v, v, false, false) : __builtin_amdgcn_permlane16_swap(v, v, false, false);
  a = r[0];
  b = r[1];
}
template <bool WIDE> __device__ __forceinline__ void both(double v, double &a, double &b) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  uint32_t al, ah, bl, bh;
  both<WIDE>((uint32_t)u, al, bl);
  both<WIDE>((uint32_t)(u >> 32), ah, bh);
  a = __builtin_bit_cast(double, (uint64_t)ah << 32 | al);
  b = __builtin_bit_cast(double, (uint64_t)bh << 32 | bl);
}
template <int LANES, typename V, typename Op> __device__ __forceinline__ V reduced(V v, Op op) {
  v = op(v, moved<0xb1>(v));    // lanes 1 0 3 2
  v = op(v, moved<0x4e>(v));    // 2 3 0 1
  v = op(v, moved<0x141>(v));   // mirrored within 8
  v = op(v, moved<0x140>(v));   // within 16
  V a, b;
  if constexpr (LANES >= 32) {
    both<false>(v, a, b);
    v = op(a, b);
  }
  if constexpr (LANES >= 64) {
    both<true>(v, a, b);
    v = op(a, b);
  }
  return v;
}

// Threads that share a row: 16, 32 or 64 lanes of a wave, or the TR threads of a workgroup of its own.
template <int TR> struct Row {
  static constexpr int WAVES = TR <= 64 ? 1 : TR / 64, BLOCK = TR <= 64 ? 256 : TR, ROWS = BLOCK / TR;
  static __device__ __forceinline__ int64_t index() { return (int64_t)blockIdx.x * ROWS + threadIdx.x / TR; }
  static __device__ __forceinline__ int lane() { return threadIdx.x % TR; }
  static unsigned blocks(int M) { return (unsigned)(((int64_t)M + ROWS - 1) / ROWS); }
  static constexpr int LANES = TR < 64 ? TR : 64;
};

}  // namespace

// ------------------------------------------------------------------------------------- rows to codes
// TR threads a row, NV pieces of eight elements each, held in registers between the maximum and the codes, so that
// a row is read once.  Bound by HBM (M K (2 or 4 + 1) bytes): 24960 x 8960 bf16 130 us, 5.2 TB/s (what a large copy reaches);
// 13824 x 5120 fp32 65 us, 5.5 TB/s; 1 x 1536 3.0 us, a launch's latency.  With five operations an element the codes hide
// behind the loads; the threads of a row are one wave's or less up to four pieces each, four waves' up to eight, then sixteen's, in steps that
// leave little of the last pass idle (8960 on 256 x 8 pieces 150 us, on 256 x 5 129).
template <typename T, int TR, int NV, bool TAIL>
__global__ __launch_bounds__(Row<TR>::BLOCK) void k_quant_rows(int M, int K, const T *__restrict__ x, int64_t xs,
                                                               int8_t *__restrict__ q, float *__restrict__ scale) {
  using R = Row<TR>;
  const int64_t row = R::index();
  if (row >= M) return;
  const T *xr = x + row * xs;
  float v[NV][8];
  uint32_t top = 0;   // of the magnitudes' bit patterns, which are ordered as the magnitudes; infinities and NaN above all
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = 8 * (R::lane() + TR * i);
    if (c < K) {
      load8<TAIL>(xr, c, K, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __builtin_bit_cast(uint32_t, v[i][j]) & 0x7fffffffu);
  }
  top = reduced<R::LANES>(top, [](uint32_t a, uint32_t b) { return max(a, b); });
  if constexpr (R::WAVES > 1) {
    __shared__ uint32_t part[R::WAVES];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < R::WAVES; ++w) top = max(top, part[w]);
  }
  const bool bad = top >= kInf;
  const float s = fmaxf(__builtin_bit_cast(float, top) / 127.0f, kTinyScale), inv = 1.0f / s;
  if (R::lane() == 0) scale[row] = bad ? __builtin_nanf("") : s;
  int8_t *qr = q + row * K;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = 8 * (R::lane() + TR * i);
    if (c >= K) break;
    // v inv, rounded once, to the nearest integer: added to 1.5 2^23 the integer is what the low bits hold.  It is off v / s
    // by less than 127 2^-24 < 8e-6: further than that from a border it decides.
    constexpr float kRound = 12582912.0f;
    uint32_t code[8];
    float far = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float r = fmaf(v[i][j], inv, kRound);
      far = fmaxf(far, fabsf(fmaf(v[i][j], inv, kRound - r)));
      code[j] = __builtin_bit_cast(uint32_t, r);
    }
    if (far > 0.49998f) {
      // two numbers of 24 bits whose quotient is no border are further from one than 64 bits round
#pragma unroll
      for (int j = 0; j < 8; ++j) code[j] = (uint32_t)(int)__builtin_rint((double)v[i][j] / (double)s);
    }
    store_codes<TAIL, 0>(qr, c, K, code, bad);
  }
}

template <typename T, int TR, int NV>
static hipError_t quant_rows(int M, int K, const T *x, int64_t xs, int8_t *q, float *scale, hipStream_t s) {
  const dim3 grid(Row<TR>::blocks(M)), block(Row<TR>::BLOCK);
  if (K % 8) hipLaunchKernelGGL((k_quant_rows<T, TR, NV, true>), grid, block, 0, s, M, K, x, xs, q, scale);
  else hipLaunchKernelGGL((k_quant_rows<T, TR, NV, false>), grid, block, 0, s, M, K, x, xs, q, scale);
  return hipGetLastError();
}

template <typename T>
static hipError_t quant_rows_of(int M, int K, const T *x, int64_t xs, int8_t *q, float *scale, hipStream_t s) {
  const int pieces = (K + 7) / 8;
#define FB_ROWS(TR, NV) if (pieces <= TR * NV) return quant_rows<T, TR, NV>(M, K, x, xs, q, scale, s);
  FB_ROWS(16, 1) FB_ROWS(32, 1) FB_ROWS(64, 1) FB_ROWS(32, 3) FB_ROWS(64, 2) FB_ROWS(64, 3) FB_ROWS(64, 4)
  FB_ROWS(256, 2) FB_ROWS(256, 3) FB_ROWS(256, 4) FB_ROWS(256, 5) FB_ROWS(256, 6) FB_ROWS(256, 8)
  FB_ROWS(1024, 3) FB_ROWS(1024, 4) FB_ROWS(1024, 6) FB_ROWS(1024, 8)
#undef FB_ROWS
  return hipErrorInvalidValue;
}

// Launches take less than 2^32 threads: rows in parts.
constexpr int kRowsPerLaunch = 1 << 20;

hipError_t launch_quant_rows(ActType t, int M, int K, const void *x, int64_t x_row_stride, int8_t *q, float *scale,
                             hipStream_t s) {
  for (int64_t m = 0; m < M; m += kRowsPerLaunch) {
    const int rows = (int)(M - m < kRowsPerLaunch ? M - m : kRowsPerLaunch);
    const hipError_t e =
        t == ACT_BF16 ? quant_rows_of(rows, K, (const bf16 *)x + m * x_row_stride, x_row_stride, q + m * K, scale + m, s)
                      : quant_rows_of(rows, K, (const float *)x + m * x_row_stride, x_row_stride, q + m * K, scale + m, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------- the seam between two blocks
// h = alpha x + gate (post_norm(y) gain), the stream as it is stored (fp32), then pre_norm(h) (1 + scale) + shift as
// activations or as codes.  A row of x and y is read once and stays in registers through both norms.  Mean and variance
// come from one pass of sums in 64 bits over the row less its first element (the pivot), so that a large common offset
// costs no digits: the variance is off by about 2^-53 (1 + (mean - pivot)^2 / variance) of itself.  Codes are decided on
// values in 64 bits as well.
// Bound by HBM: (4 + e) M D bytes read, 4 M D + (e or 1) M D written: 24960 x 1536 bf16 to codes 98 us (4.3 TB/s) and to
// activations 98 (4.7), 16384 x 5120 to activations 215 (4.7), one token of 1536 4.0 us; without a branch 24960 x 1536 45 us.
// The 64-bit arithmetic, some 35 instructions an element at the rate of 32-bit ones, hides behind that for the most part, as
// long as registers leave four waves a SIMD: y stays as it is stored.  The stream in fp32 where activations follow would save
// 1 to 6% (1560 x 1536 9.8 us against 10.4), and sums without the pivot for RMS norm nothing.  Pieces of four
// elements, which make a wave's accesses to fp32 whole ranges, bring the vectors in twice as many waits: measured on the fp32
// stream, (16384, 5120) to activations 191 in place of 212, but (24960, 1536) 102 in place of 96 and (8192, 6144) 152 in
// place of 131.
namespace {

// Rows of 513 to 2048 elements are on one wave, two or four, by the number of rows.  So that a row's bits are those it has among
// few rows and among many, their sums are added in one order: chunks of 64 pieces one after another in each lane, then lanes.
template <int TR, int NV> struct Sums {
  static constexpr int CHUNKS = Row<TR>::WAVES * NV;
  static constexpr bool BY_LANE = Row<TR>::WAVES > 1 && CHUNKS <= 4;
  static constexpr int PARTS = BY_LANE ? 64 * CHUNKS : Row<TR>::WAVES;
};
// The row's two sums, for all its threads, from its pieces'.  part: LDS that this call alone uses, so that one barrier does.
template <int TR, int NV>
__device__ __forceinline__ void row_sums(const double (&sum)[NV], const double (&sq)[NV], double &a, double &b, double (*part)[2]) {
  using R = Row<TR>;
  using S = Sums<TR, NV>;
  const auto add = [](double p, double q) { return p + q; };
  a = sum[0];
  b = sq[0];
  if constexpr (S::BY_LANE) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      part[64 * (R::WAVES * i + wave) + lane][0] = sum[i];
      part[64 * (R::WAVES * i + wave) + lane][1] = sq[i];
    }
    __syncthreads();
    a = part[lane][0];
    b = part[lane][1];
#pragma unroll
    for (int c = 1; c < S::CHUNKS; ++c) {
      a += part[64 * c + lane][0];
      b += part[64 * c + lane][1];
    }
  } else {
#pragma unroll
    for (int i = 1; i < NV; ++i) {
      a += sum[i];
      b += sq[i];
    }
  }
  a = reduced<R::LANES>(a, add);
  b = reduced<R::LANES>(b, add);
  if constexpr (R::WAVES > 1 && !S::BY_LANE) {
    if ((threadIdx.x & 63) == 0) {
      part[threadIdx.x >> 6][0] = a;
      part[threadIdx.x >> 6][1] = b;
    }
    __syncthreads();
    a = b = 0;
#pragma unroll
    for (int w = 0; w < R::WAVES; ++w) {
      a += part[w][0];
      b += part[w][1];
    }
  }
}

// A row's norm, (v - mean) by, in type V; from the sums of v - pivot and of its square over D elements (pivot 0 but for
// LayerNorm's, whose mean is pivot + sum / D).
template <typename V> struct Norm;
template <> struct Norm<double> {   // the pivot comes off first: what equals it in a row of one value leaves no digits
  double by = 1.0, pivot = 0.0, plus = 0.0;
  __device__ __forceinline__ Norm(int kind, double first, double sum, double sq, int D, double eps) {
    if (kind == NORM_NONE) return;
    const double n = D, m = kind == NORM_LAYER ? sum / n : 0.0, var = sq / n - m * m;
    by = 1.0 / sqrt((var < 0 ? 0 : var) + eps);   // NaN stays
    pivot = first;
    plus = -m * by;
  }
  __device__ __forceinline__ double operator()(float v) const { return fma((double)v - pivot, by, plus); }
};
template <> struct Norm<float> {
  // The mean in two parts, so that it costs no digits of v - mean.  Where the deviation is past 2^64, all in units of 2^64:
  // v - mean may be past fp32's range there, and the reciprocal below it.
  float by, unit = 1.f, mean, rest;
  __device__ __forceinline__ Norm(int kind, double pivot, double sum, double sq, int D, double eps) {
    const Norm<double> n(kind, pivot, sum, sq, D, eps);
    const bool wide = n.by < 0x1p-64;
    const double m = (kind == NORM_LAYER ? pivot + sum / (double)D : 0.0) * (wide ? 0x1p-64 : 1.0);
    if (wide) unit = 0x1p-64f;
    by = (float)(wide ? n.by * 0x1p64 : n.by);
    mean = (float)m;
    rest = (float)(m - (double)mean);
  }
  __device__ __forceinline__ float operator()(float v) const { return (fmaf(v, unit, -mean) - rest) * by; }
};

// Elements c .. c + 7 of a vector, or eight times `otherwise` for none.
template <bool TAIL>
__device__ __forceinline__ void load8_or(const float *p, float otherwise, int c, int n, float (&v)[8]) {
  if (p) {
    load8<TAIL>(p, c, n, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = otherwise;
  }
}

}  // namespace

enum { SEAM_NONE = 0, SEAM_ACT = 1, SEAM_I8 = 2 };

// FULL: the row fills its threads' pieces, so that no load waits behind a branch: (1560, 1536) to codes 10.4 us against 11.9,
// (24960, 1536) 98 and 100, (1560, 2048) to activations 12.3 and 13.2.
template <typename T, int TR, int NV, bool TAIL, int OUT, bool NT, bool FULL>
__global__ __launch_bounds__(Row<TR>::BLOCK) void k_norm_residual(int M, SeamArgs a) {
  using R = Row<TR>;
  using V = std::conditional_t<OUT == SEAM_I8, double, float>;   // of the outputs
  constexpr int PARTS = Sums<TR, NV>::PARTS;
  __shared__ __attribute__((aligned(16))) double part[2 * PARTS][2], tops[R::WAVES];
  const int64_t row = R::index();
  if (row >= M) return;
  const int D = a.D;   // elements past it (TAIL) take no branches: they stand at the pivot in the sums, and at zero in the end
  const float *xr = a.x + row * D;
  const T *yr = (const T *)a.y + row * D;
  float h[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = 8 * (R::lane() + TR * i);
    if (FULL || c < D) load8<TAIL>(xr, c, D, h[i]);
  }
  // one piece a thread: what it needs of the vectors is on its way before the sums
  constexpr bool EARLY = NV == 1;
  float gain[8], gate[8], scale[8], shift[8];
  if (EARLY && 8 * R::lane() < D) {
    load8_or<TAIL>(a.gain, 1.f, 8 * R::lane(), D, gain);
    load8_or<TAIL>(a.gate, 1.f, 8 * R::lane(), D, gate);
    load8_or<TAIL>(a.scale, 0.f, 8 * R::lane(), D, scale);
    load8_or<TAIL>(a.shift, 0.f, 8 * R::lane(), D, shift);
  }
  if (a.y) {
    Piece<T> y[NV];
    const double pivot = a.post == NORM_LAYER ? (double)to_f32(yr[0]) : 0.0;
    double sums[NV] = {}, sqs[NV] = {}, sum = 0, sq = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (!FULL && c >= D) break;
      y[i].template load<TAIL>(yr, c, D);
      if (a.post == NORM_NONE) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double d = (double)(TAIL && c + j >= D ? (float)pivot : y[i][j]) - pivot;
        sums[i] += d;
        sqs[i] = fma(d, d, sqs[i]);
      }
    }
    if (a.post != NORM_NONE) row_sums<TR, NV>(sums, sqs, sum, sq, part);
    const Norm<double> norm(a.post, pivot, sum, sq, D, a.eps);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (!FULL && c >= D) break;
      if constexpr (!EARLY) {
        load8_or<TAIL>(a.gain, 1.f, c, D, gain);
        load8_or<TAIL>(a.gate, 1.f, c, D, gate);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // in 64 bits whatever comes of h, so that the stream does not depend on that: the first and the last product are exact
        h[i][j] = (float)fma((double)gate[j] * (double)gain[j], norm(y[i][j]), (double)a.alpha * (double)h[i][j]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] = a.alpha * h[i][j];
  }
  if (a.x_out) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (FULL || c < D) store8<TAIL, NT>(a.x_out + row * D, c, D, h[i]);
    }
  }
  if constexpr (OUT != SEAM_NONE) {
    double pivot = 0, sums[NV] = {}, sqs[NV] = {}, sum = 0, sq = 0;
    V v[NV][8], top = 0;
    if (a.pre == NORM_LAYER) {
      // the row's first element: of its first lane, for rows of several waves through LDS (read by all at the sums' barrier)
      float first = __shfl(h[0][0], TR < 64 ? (int)(threadIdx.x & 63 & ~(TR - 1)) : 0, 64);
      if constexpr (R::WAVES > 1) {
        if (threadIdx.x == 0) tops[0] = first;
        __syncthreads();
        first = (float)tops[0];
      }
      pivot = (double)first;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (!FULL && c >= D) break;
      if (a.pre == NORM_NONE) continue;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const double d = (double)(TAIL && c + j >= D ? (float)pivot : h[i][j]) - pivot;
        sums[i] += d;
        sqs[i] = fma(d, d, sqs[i]);
      }
    }
    if (a.pre != NORM_NONE) row_sums<TR, NV>(sums, sqs, sum, sq, part + PARTS);
    const Norm<V> norm(a.pre, pivot, sum, sq, D, a.eps);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (!FULL && c >= D) break;
      if constexpr (!EARLY) {
        load8_or<TAIL>(a.scale, 0.f, c, D, scale);
        load8_or<TAIL>(a.shift, 0.f, c, D, shift);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[i][j] = TAIL && c + j >= D ? (V)0 : fma(norm(h[i][j]), (V)1 + (V)scale[j], (V)shift[j]);
        if constexpr (OUT == SEAM_I8) {
          top = fmax(top, fabs(v[i][j]));
          bad |= v[i][j] != v[i][j];   // the maximum leaves NaN out
        }
      }
      if constexpr (OUT == SEAM_ACT) store8<TAIL>((T *)a.out + row * D, c, D, v[i]);
    }
    if constexpr (OUT == SEAM_I8) {
      top = bad ? (double)INFINITY : top;
      top = reduced<R::LANES>(top, [](double p, double q) { return fmax(p, q); });
      if constexpr (R::WAVES > 1) {
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < R::WAVES; ++w) top = fmax(top, tops[w]);
      }
      const float s = fmaxf((float)(top / 127.0), kTinyScale);
      bad = !(s < INFINITY);
      const double inv = 1.0 / (double)s;
      if (R::lane() == 0) a.q_scale[row] = bad ? __builtin_nanf("") : s;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = 8 * (R::lane() + TR * i);
        if (!FULL && c >= D) break;
        // v / s + 1/2 to 24 bits behind the point, the integer in the low word's last byte: off by less than a step of those
        // it decides, but where it comes out as a whole number
        uint32_t code[8], least = ~0u;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          code[j] = (uint32_t)__builtin_bit_cast(uint64_t, fma(v[i][j], inv, 402653184.5));   // 1.5 2^28 + 1/2
          least = min(least, code[j] << 8);
        }
        if (least == 0) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            // the border, a number of 8 bits times s, is exact, and so is the sign of its distance
            const int up = (int)code[j] >> 24;
            const double over = fma(up - 0.5, (double)s, -v[i][j]);
            if (code[j] << 8 == 0 && (over > 0 || (over == 0 && up % 2))) code[j] -= 1;
          }
        }
        store_codes<TAIL, 3>(a.q + row * D, c, D, code, bad);
      }
    }
  }
}

template <typename T, int TR, int NV, int OUT>
static hipError_t norm_rows(int M, const SeamArgs &a, hipStream_t s) {
  const dim3 grid(Row<TR>::blocks(M)), block(Row<TR>::BLOCK);
  // a stream of 64 MiB and more is stored non-temporally: nothing reads it soon ((24960, 1536) to codes 102 -> 98 us,
  // (16384, 5120) to activations 219 -> 215); a smaller one the next kernel may still find in the caches
  const bool nt = a.x_out && (size_t)M * a.D * 4 >= (size_t)64 << 20;
  // on 256 threads it lost as often as it gained: (1560, 4096) to codes 21.3 us in place of 22.3, to activations 19.5 of 19.2,
  // (9000, 4096) 99 of 98 and 97 of 98, (16384, 4096) fp32 192 of 188 and 215 of 218
  constexpr bool FULL = NV > 1 && TR <= 128;
  const bool full = FULL && a.D == 8 * TR * NV;
  const auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, block, 0, s, M, a); };
  if (a.D % 8) go(k_norm_residual<T, TR, NV, true, OUT, false, false>);
  else if (nt) full ? go(k_norm_residual<T, TR, NV, false, OUT, true, FULL>) : go(k_norm_residual<T, TR, NV, false, OUT, true, false>);
  else full ? go(k_norm_residual<T, TR, NV, false, OUT, false, FULL>) : go(k_norm_residual<T, TR, NV, false, OUT, false, false>);
  return hipGetLastError();
}

template <typename T, int OUT>
static hipError_t norm_rows_of(int M, const SeamArgs &a, hipStream_t s) {
  const int pieces = (a.D + 7) / 8;
#define FB_ROWS(TR, NV) if (pieces <= TR * NV) return norm_rows<T, TR, NV, OUT>(M, a, s);
  FB_ROWS(16, 1) FB_ROWS(32, 1) FB_ROWS(64, 1)   // several rows a wave: 24960 x 64 10 us, on whole waves 34
  // few rows wait on a row's own chain, which more threads shorten, many on the waves' arithmetic: on 256 threads and on one
  // wave 1 x 1536 to codes 4.0 us and 4.6, 512 rows 5.8 and 6.1, 650 rows 7.2 and 6.4, 1560 rows 12.3 and 10.4; to activations
  // 512 rows 5.4 and 6.2, 780 rows 7.2 and 6.7
  if (M <= 2 * cu_count()) { FB_ROWS(256, 1) }
  FB_ROWS(64, 2) FB_ROWS(64, 3) FB_ROWS(128, 2) FB_ROWS(192, 2) FB_ROWS(256, 2) FB_ROWS(256, 3)
#undef FB_ROWS
  return hipErrorInvalidValue;
}

hipError_t launch_norm_residual(ActType t, int M, const SeamArgs &a, hipStream_t s) {
  const size_t e = t == ACT_BF16 ? 2 : 4;
  for (int64_t m = 0; m < M; m += kRowsPerLaunch) {
    const int rows = (int)(M - m < kRowsPerLaunch ? M - m : kRowsPerLaunch);
    SeamArgs p = a;
    p.x += m * a.D;
    if (p.y) p.y = (const char *)a.y + (size_t)m * a.D * e;
    if (p.x_out) p.x_out += m * a.D;
    if (p.out) p.out = (char *)a.out + (size_t)m * a.D * e;
    if (p.q) { p.q += m * a.D; p.q_scale += m; }
    const int out = p.out ? SEAM_ACT : p.q ? SEAM_I8 : SEAM_NONE;
    hipError_t err;
    if (t == ACT_BF16)
      err = out == SEAM_I8 ? norm_rows_of<bf16, SEAM_I8>(rows, p, s)
            : out == SEAM_ACT ? norm_rows_of<bf16, SEAM_ACT>(rows, p, s) : norm_rows_of<bf16, SEAM_NONE>(rows, p, s);
    else
      err = out == SEAM_I8 ? norm_rows_of<float, SEAM_I8>(rows, p, s)
            : out == SEAM_ACT ? norm_rows_of<float, SEAM_ACT>(rows, p, s) : norm_rows_of<float, SEAM_NONE>(rows, p, s);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace fb
