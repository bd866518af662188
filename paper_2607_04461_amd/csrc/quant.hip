// Rows to 8-bit integers (k_quant_rows) and the seam between two blocks (k_norm_residual): the operands of the 8-bit
// linear layers.
//
// A row v becomes q = nearest-even(v / s) with one scale s = max(max |v| / 127, 2^-126), rounded once to fp32.  The
// nearest integer is decided exactly: for rows that come as numbers (k_quant_rows) on the quotient itself, for rows
// that are computed (k_norm_residual) on values held in 64 bits.  So a code depends neither on the order in which a
// row's sums were added nor on how many threads shared the row, and two launches that form the same row agree to the
// bit.
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

// Elements c .. c + 7 of a row of n, zero past its end (TAIL: n % 8 != 0, so that a piece may end early).
template <bool TAIL>
__device__ __forceinline__ void load8(const float *p, int c, int n, float (&v)[8]) {
  if (!TAIL || c + 8 <= n) {
    const f32x4u a = *reinterpret_cast<const f32x4u *>(p + c), b = *reinterpret_cast<const f32x4u *>(p + c + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = a[i];
      v[4 + i] = b[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < n ? p[c + i] : 0.f;
  }
}
template <bool TAIL>
__device__ __forceinline__ void load8(const bf16 *p, int c, int n, float (&v)[8]) {
  if (!TAIL || c + 8 <= n) {
    const u32x4u a = *reinterpret_cast<const u32x4u *>(p + c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __builtin_bit_cast(float, a[i] << 16);
      v[2 * i + 1] = __builtin_bit_cast(float, a[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < n ? (float)p[c + i] : 0.f;
  }
}
template <bool TAIL>
__device__ __forceinline__ void store8(float *p, int c, int n, const float (&v)[8]) {
  if (!TAIL || c + 8 <= n) {
    *reinterpret_cast<f32x4u *>(p + c) = f32x4u{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4u *>(p + c + 4) = f32x4u{v[4], v[5], v[6], v[7]};
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
template <bool TAIL>
__device__ __forceinline__ void store_codes(int8_t *p, int c, int n, const int (&q)[8]) {
  if (!TAIL || c + 8 <= n) {
    u32x2u w;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w[i] = (uint32_t)(q[4 * i] & 255) | (uint32_t)(q[4 * i + 1] & 255) << 8 | (uint32_t)(q[4 * i + 2] & 255) << 16 |
             (uint32_t)q[4 * i + 3] << 24;
    *reinterpret_cast<u32x2u *>(p + c) = w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < n) p[c + i] = (int8_t)q[i];
  }
}

// Threads that share a row: one wave, or a workgroup of its own.
template <int TR> struct Row {
  static constexpr int WAVES = TR / 64, BLOCK = TR == 64 ? 256 : TR;
  static __device__ __forceinline__ int64_t index() {
    return TR == 64 ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : (int64_t)blockIdx.x;
  }
  static __device__ __forceinline__ int lane() { return TR == 64 ? threadIdx.x & 63 : threadIdx.x; }
};

}  // namespace

// ------------------------------------------------------------------------------------- rows to codes
// TR threads a row, NV pieces of eight elements each, held in registers between the maximum and the codes, so that
// a row is read once.  Bound by HBM (M K (2 or 4 + 1) bytes).
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
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
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
    int code[8];
    bool near = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // v inv is off v / s by less than 127 (2^-23 + 2^-24) < 3e-5: further than that from a border it decides
      const float t = v[i][j] * inv, r = __builtin_rintf(t);
      near |= fabsf(t - r) > 0.49995f;
      code[j] = (int)r;
    }
    if (near) {
      // two numbers of 24 bits whose quotient is no border are further from one than 64 bits round
#pragma unroll
      for (int j = 0; j < 8; ++j) code[j] = (int)__builtin_rint((double)v[i][j] / (double)s);
    }
    if (bad) {
#pragma unroll
      for (int j = 0; j < 8; ++j) code[j] = 0;
    }
    store_codes<TAIL>(qr, c, K, code);
  }
}

template <typename T, int TR, int NV>
static hipError_t quant_rows(int M, int K, const T *x, int64_t xs, int8_t *q, float *scale, hipStream_t s) {
  const unsigned blocks = TR == 64 ? (unsigned)(((int64_t)M + 3) / 4) : (unsigned)M;
  if (K % 8)
    hipLaunchKernelGGL((k_quant_rows<T, TR, NV, true>), dim3(blocks), dim3(Row<TR>::BLOCK), 0, s, M, K, x, xs, q, scale);
  else
    hipLaunchKernelGGL((k_quant_rows<T, TR, NV, false>), dim3(blocks), dim3(Row<TR>::BLOCK), 0, s, M, K, x, xs, q, scale);
  return hipGetLastError();
}

template <typename T>
static hipError_t quant_rows_of(int M, int K, const T *x, int64_t xs, int8_t *q, float *scale, hipStream_t s) {
  const int pieces = (K + 7) / 8;
  if (pieces <= 64) return quant_rows<T, 64, 1>(M, K, x, xs, q, scale, s);
  if (pieces <= 128) return quant_rows<T, 64, 2>(M, K, x, xs, q, scale, s);
  if (pieces <= 256) return quant_rows<T, 64, 4>(M, K, x, xs, q, scale, s);
  if (pieces <= 512) return quant_rows<T, 256, 2>(M, K, x, xs, q, scale, s);
  if (pieces <= 1024) return quant_rows<T, 256, 4>(M, K, x, xs, q, scale, s);
  if (pieces <= 2048) return quant_rows<T, 256, 8>(M, K, x, xs, q, scale, s);
  if (pieces <= 4096) return quant_rows<T, 1024, 4>(M, K, x, xs, q, scale, s);
  return quant_rows<T, 1024, 8>(M, K, x, xs, q, scale, s);
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
// Bound by HBM: (4 + e) M D bytes read, 4 M D + (e or 1) M D written.
namespace {

// Sums over the row of two numbers and, for codes, a maximum.  Every call has LDS of its own, so that one barrier does.
template <int TR> __device__ __forceinline__ void row_sums(double &a, double &b) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    a += __shfl_xor(a, o, 64);
    b += __shfl_xor(b, o, 64);
  }
}
template <int TR> __device__ __forceinline__ void join_sums(double &a, double &b, double (*part)[2]) {
  if constexpr (Row<TR>::WAVES > 1) {
    if ((threadIdx.x & 63) == 0) {
      part[threadIdx.x >> 6][0] = a;
      part[threadIdx.x >> 6][1] = b;
    }
    __syncthreads();
    a = b = 0;
#pragma unroll
    for (int w = 0; w < Row<TR>::WAVES; ++w) {
      a += part[w][0];
      b += part[w][1];
    }
  }
}

struct Norm {
  double mean, rstd;
};
// From the sums of (v - pivot) and its square over D elements.
__device__ __forceinline__ Norm norm_of(int kind, double pivot, double sum, double sq, int D, double eps) {
  const double n = D, m = kind == NORM_LAYER ? sum / n : 0.0;
  double var = sq / n - m * m;
  var = var < 0 ? 0 : var;   // NaN stays
  return {kind == NORM_LAYER ? pivot + m : 0.0, 1.0 / sqrt(var + eps)};
}

}  // namespace

enum { SEAM_NONE = 0, SEAM_ACT = 1, SEAM_I8 = 2 };

template <typename T, int TR, int NV, bool TAIL, int OUT>
__global__ __launch_bounds__(Row<TR>::BLOCK) void k_norm_residual(int M, SeamArgs a) {
  using R = Row<TR>;
  using V = std::conditional_t<OUT == SEAM_I8, double, float>;   // of the elements
  __shared__ double part[R::WAVES > 1 ? 2 * R::WAVES : 1][2], tops[R::WAVES];
  const int64_t row = R::index();
  if (row >= M) return;
  const int D = a.D;
  const float *xr = a.x + row * D;
  const T *yr = (const T *)a.y + row * D;
  float h[NV][8];
  if (a.y) {
    float y[NV][8];
    Norm n = {0.0, 1.0};
    const double pivot = a.post == NORM_LAYER ? (double)to_f32(yr[0]) : 0.0;
    double sum = 0, sq = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (c < D) {
        load8<TAIL>(yr, c, D, y[i]);
        load8<TAIL>(xr, c, D, h[i]);
        if (a.post != NORM_NONE) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (TAIL && c + j >= D) break;
            const double d = (double)y[i][j] - pivot;
            sum += d;
            sq = fma(d, d, sq);
          }
        }
      }
    }
    if (a.post != NORM_NONE) {
      row_sums<TR>(sum, sq);
      join_sums<TR>(sum, sq, part);
      n = norm_of(a.post, pivot, sum, sq, D, a.eps);
    }
    const V mean = (V)n.mean, rstd = (V)n.rstd, alpha = (V)a.alpha;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (c >= D) break;
      float gain[8], gate[8];
      if (a.gain) load8<TAIL>(a.gain, c, D, gain);
      if (a.gate) load8<TAIL>(a.gate, c, D, gate);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        V u = ((V)y[i][j] - mean) * rstd;
        if (a.gain) u *= (V)gain[j];
        h[i][j] = (float)(a.gate ? fma((V)gate[j], u, alpha * (V)h[i][j]) : alpha * (V)h[i][j] + u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (c >= D) break;
      load8<TAIL>(xr, c, D, h[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i][j] = a.alpha * h[i][j];
    }
  }
  if (a.x_out) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (c < D) store8<TAIL>(a.x_out + row * D, c, D, h[i]);
    }
  }
  if constexpr (OUT != SEAM_NONE) {
    Norm n = {0.0, 1.0};
    if (a.pre != NORM_NONE) {
      // the row's first element: of lane 0, for rows of several waves through LDS (read by all at the sums' barrier)
      double pivot = 0, sum = 0, sq = 0;
      if (a.pre == NORM_LAYER) {
        float first = h[0][0];
        if constexpr (R::WAVES > 1) {
          if (threadIdx.x == 0) tops[0] = first;
          __syncthreads();
          first = (float)tops[0];
        }
        pivot = (double)__builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, first)));
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = 8 * (R::lane() + TR * i);
        if (c < D) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (TAIL && c + j >= D) break;
            const double d = (double)h[i][j] - pivot;
            sum += d;
            sq = fma(d, d, sq);
          }
        }
      }
      row_sums<TR>(sum, sq);
      join_sums<TR>(sum, sq, part + (R::WAVES > 1 ? R::WAVES : 0));
      n = norm_of(a.pre, pivot, sum, sq, D, a.eps);
    }
    const V mean = (V)n.mean, rstd = (V)n.rstd;
    V v[NV][8], top = 0;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = 8 * (R::lane() + TR * i);
      if (c >= D) break;
      float scale[8], shift[8];
      if (a.scale) load8<TAIL>(a.scale, c, D, scale);
      if (a.shift) load8<TAIL>(a.shift, c, D, shift);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (TAIL && c + j >= D) break;
        V w = ((V)h[i][j] - mean) * rstd;
        if (a.scale) w *= (V)1 + (V)scale[j];
        if (a.shift) w += (V)shift[j];
        v[i][j] = w;
        if constexpr (OUT == SEAM_I8) {
          top = fmax(top, fabs(w));
          bad |= w != w;   // the maximum leaves NaN out
        }
      }
      if constexpr (OUT == SEAM_ACT) store8<TAIL>((T *)a.out + row * D, c, D, v[i]);
    }
    if constexpr (OUT == SEAM_I8) {
      top = bad ? (double)INFINITY : top;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) top = fmax(top, __shfl_xor(top, o, 64));
      if constexpr (R::WAVES > 1) {
        if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < R::WAVES; ++w) top = fmax(top, tops[w]);
      }
      float s = fmaxf((float)(top / 127.0), kTinyScale);
      bad = !(s < INFINITY);
      const double inv = 1.0 / (double)s;
      if (R::lane() == 0) a.q_scale[row] = bad ? __builtin_nanf("") : s;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = 8 * (R::lane() + TR * i);
        if (c >= D) break;
        int code[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) code[j] = bad || (TAIL && c + j >= D) ? 0 : (int)__builtin_rint(v[i][j] * inv);
        store_codes<TAIL>(a.q + row * D, c, D, code);
      }
    }
  }
}

template <typename T, int TR, int NV, int OUT>
static hipError_t norm_rows(int M, const SeamArgs &a, hipStream_t s) {
  const unsigned blocks = TR == 64 ? (unsigned)(((int64_t)M + 3) / 4) : (unsigned)M;
  if (a.D % 8) hipLaunchKernelGGL((k_norm_residual<T, TR, NV, true, OUT>), dim3(blocks), dim3(Row<TR>::BLOCK), 0, s, M, a);
  else hipLaunchKernelGGL((k_norm_residual<T, TR, NV, false, OUT>), dim3(blocks), dim3(Row<TR>::BLOCK), 0, s, M, a);
  return hipGetLastError();
}

template <typename T, int OUT>
static hipError_t norm_rows_of(int M, const SeamArgs &a, hipStream_t s) {
  const int pieces = (a.D + 7) / 8;
  if (pieces <= 64) return norm_rows<T, 64, 1, OUT>(M, a, s);
  if (pieces <= 128) return norm_rows<T, 64, 2, OUT>(M, a, s);
  if (pieces <= 192) return norm_rows<T, 64, 3, OUT>(M, a, s);
  if (pieces <= 512) return norm_rows<T, 256, 2, OUT>(M, a, s);
  return norm_rows<T, 256, 3, OUT>(M, a, s);
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
