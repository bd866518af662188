// LayerNorm of the fp32 residual stream with the rows' statistics, and its gradient.
//   xhat = (x - mean) rstd,   y = xhat f + b,   f = weight or 1 + weight (adaLN)
//   g = dy f,   dx = residual + rstd (g - mean(g) - xhat mean(g xhat))
//   dweight = sum_m dy xhat,   dbias = sum_m dy over the rows of a group (they share a weight and a bias)
// Both are bound by HBM: every row is read once and held in registers between its reductions, by one wave up to
// 2048 elements and by four beyond (16384 x 5120 to bf16 98 us, 5.2 TB/s; the gradient of 24960 x 1536 with the residual
// stream's 113 us and 5 for the vectors' sums, 4.7 TB/s).  The mean is summed in 64 bits (a few per cent of the time a
// row's bytes take) and taken off in two parts, so that rows far from zero keep their digits; the other sums are fp32.  Where the variance
// and eps leave fp32's normal numbers (a deviation past 2^64, or eps below 2^-126), the row is formed anew in 64 bits.
// The gradient of the vectors is a sum over thousands of rows: a workgroup adds up a chunk of rows of one group in
// registers, and a second launch adds the chunks' sums in order, in 64 bits.  No atomics: a call's bits are always
// the same.  A chunk is what gives four workgroups a CU (more rows: fewer partial sums, but an uneven last round).
#include <algorithm>
#include <initializer_list>

#include "common.h"
#include "kernels.h"

namespace fb {
namespace {

constexpr int THREADS = 256;

// The elements of a row of D that a lane of L holds, 4 NC at most: pieces of four, or one every L where D or an address
// is no multiple of four elements.
template <int L, int NC, bool VEC>
struct Row {
  template <typename F> __device__ static __forceinline__ void each(int t, int D, F f) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = VEC ? 4 * (c * L + t) + i : (4 * c + i) * L + t;
        f(4 * c + i, e, e < D);
      }
  }
  // elements past D read as zero; at null: all `none`
  template <typename T> __device__ static __forceinline__ void load(float (&v)[4 * NC], const T *at, int t, int D, float none = 0.f) {
    if (!at) {
#pragma unroll
      for (int i = 0; i < 4 * NC; ++i) v[i] = none;
      return;
    }
    if constexpr (VEC) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int e = 4 * (c * L + t);
        if constexpr (sizeof(T) == 4) {
          const f32x4 p = e < D ? *reinterpret_cast<const f32x4 *>(at + e) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * c + i] = p[i];
        } else {
          const u32x2 p = e < D ? *reinterpret_cast<const u32x2 *>(at + e) : u32x2{0, 0};
          const bf16x4 q = __builtin_bit_cast(bf16x4, p);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * c + i] = (float)q[i];
        }
      }
    } else {
      each(t, D, [&](int i, int e, bool in) { v[i] = in ? to_f32(at[e]) : 0.f; });
    }
  }
  template <typename T> __device__ static __forceinline__ void store(T *at, const float (&v)[4 * NC], int t, int D) {
    if constexpr (VEC) {
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int e = 4 * (c * L + t);
        if (e >= D) continue;
        if constexpr (sizeof(T) == 4)
          *reinterpret_cast<f32x4 *>(at + e) = f32x4{v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]};
        else
          *reinterpret_cast<bf16x4 *>(at + e) = bf16x4{(bf16)v[4 * c], (bf16)v[4 * c + 1], (bf16)v[4 * c + 2], (bf16)v[4 * c + 3]};
      }
    } else {
      each(t, D, [&](int i, int e, bool in) { if (in) at[e] = from_f32<T>(v[i]); });
    }
  }
};

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

template <typename T, int WPR, int NC, bool VEC>
__global__ __launch_bounds__(THREADS) void k_layer_norm(LayerNormArgs a) {
  using R = Row<64 * WPR, NC, VEC>;
  __shared__ double s_sum[4], s_wide[4];
  __shared__ float s_sq[4];
  const int w = threadIdx.x >> 6, t = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
  constexpr int ROWS = 4 / WPR;
  // four waves a row meet at barriers: the row is then the workgroup's, and so is the number of turns
  for (int64_t m = (int64_t)blockIdx.x * ROWS + (WPR == 1 ? w : 0); m < a.M; m += (int64_t)gridDim.x * ROWS) {
    float v[4 * NC];
    R::load(v, a.x + m * a.D, t, a.D);
    double sum = 0;
#pragma unroll
    for (int i = 0; i < 4 * NC; ++i) sum += (double)v[i];
    sum = wave_sum64(sum);
    if constexpr (WPR > 1) {
      if ((threadIdx.x & 63) == 0) s_sum[w] = sum;
      __syncthreads();
      sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
    }
    const double mean = sum / a.D;
    const float hi = (float)mean, lo = (float)(mean - (double)hi);
    float sq = 0;
    R::each(t, a.D, [&](int i, int, bool in) {
      v[i] = in ? (v[i] - hi) - lo : 0.f;
      sq = fmaf(v[i], v[i], sq);
    });
    sq = wave_sum(sq);
    if constexpr (WPR > 1) {
      if ((threadIdx.x & 63) == 0) s_sq[w] = sq;
      __syncthreads();
      sq = (s_sq[0] + s_sq[1]) + (s_sq[2] + s_sq[3]);
    }
    const float var = sq / (float)a.D + a.eps;
    float rstd = 1.0f / sqrtf(var), by = rstd;
    if (!(var >= 0x1p-126f && var < INFINITY)) {      // every wave of the row alike
      R::load(v, a.x + m * a.D, t, a.D);
      double wide = 0;
      R::each(t, a.D, [&](int i, int, bool in) {
        const double c = in ? (double)v[i] - mean : 0.0;
        wide = fma(c, c, wide);
      });
      wide = wave_sum64(wide);
      if constexpr (WPR > 1) {      // apart from s_sum: the next row writes that before a barrier
        if ((threadIdx.x & 63) == 0) s_wide[w] = wide;
        __syncthreads();
        wide = (s_wide[0] + s_wide[1]) + (s_wide[2] + s_wide[3]);
      }
      const double r = 1.0 / sqrt(wide / a.D + (double)a.eps);
      R::each(t, a.D, [&](int i, int, bool in) { v[i] = in ? (float)(((double)v[i] - mean) * r) : 0.f; });
      rstd = (float)r;
      by = 1.f;
    }
    const int64_t group = m / a.per;
    float f[4 * NC], b[4 * NC];
    R::load(f, a.weight ? a.weight + group * a.D : nullptr, t, a.D, 1.f - a.offset);
    R::load(b, a.bias ? a.bias + group * a.D : nullptr, t, a.D);
#pragma unroll
    for (int i = 0; i < 4 * NC; ++i) v[i] = fmaf(v[i] * by, f[i] + a.offset, b[i]);
    R::store((T *)a.out + m * a.D, v, t, a.D);
    if (t == 0) {
      if (a.mean) a.mean[m] = hi;
      if (a.rstd) a.rstd[m] = rstd;
    }
  }
}

// A saved mean is off by half a step of fp32, a shift that the whole row's xhat would share.  Up to 4096 deviations from zero it
// stays below 2^-12 of one, and the statistics are taken as they are given; rows farther away take off what the mean left
// (24960 x 1536: 118 us, 119 with every row's).  Rows of a deviation past 2^120 are taken in units of 2^16, since x - mean may
// be past fp32's range.
// One chunk of rows of one group: dx of its rows, and its share of dweight and dbias, to the chunk's row of `partial`
// ([chunks][2][D]), or straight to the group's where a group is one chunk.
// Two waves a SIMD: without asking, rows of 1537 to 2048 took 258 to 278 registers and one wave (8192 x 2048, bf16: 62 us for 58).
template <typename T, int WPR, int NC, bool VEC>
__global__ __launch_bounds__(THREADS, 2) void k_layer_norm_grad(LayerNormGradArgs a) {
  using R = Row<64 * WPR, NC, VEC>;
  extern __shared__ float s_acc[];       // WPR 1: [2][256 NC] for the four waves' sums
  __shared__ float s_red[2][4][2];
  __shared__ double s_rest[4];
  const int w = threadIdx.x >> 6, t = WPR == 1 ? threadIdx.x & 63 : threadIdx.x, D = a.D;
  const int64_t group = blockIdx.x / a.chunks;
  const int64_t first = group * a.per + (int64_t)(blockIdx.x % a.chunks) * a.rows;
  const int64_t end = min(min(first + a.rows, (group + 1) * (int64_t)a.per), (int64_t)a.M);
  float f[4 * NC], dw[4 * NC], db[4 * NC];
  R::load(f, a.weight ? a.weight + group * D : nullptr, t, D, 1.f - a.offset);
#pragma unroll
  for (int i = 0; i < 4 * NC; ++i) {
    f[i] += a.offset;
    dw[i] = db[i] = 0.f;
  }
  int turn = 0;
  for (int64_t m = first + (WPR == 1 ? w : 0); m < end; m += 4 / WPR, turn ^= 1) {
    float x[4 * NC], g[4 * NC];
    R::load(x, a.x + m * D, t, D);
    R::load(g, (const T *)a.dy + m * D, t, D);
    const float rstd = a.rstd[m];
    float mean = a.mean[m], by = rstd, off = 0.f;
    if (rstd < 0x1p-120f || fabsf(mean) * rstd > 4096.f) {      // every wave of the row alike
      const float unit = rstd < 0x1p-120f ? 0x1p-16f : 1.f;
      mean *= unit;
      by /= unit;
      double rest = 0;
      R::each(t, D, [&](int i, int, bool in) {
        x[i] *= unit;
        rest += in ? (double)(x[i] - mean) : 0.0;
      });
      rest = wave_sum64(rest);
      if constexpr (WPR > 1) {
        if ((threadIdx.x & 63) == 0) s_rest[w] = rest;
        __syncthreads();
        rest = (s_rest[0] + s_rest[1]) + (s_rest[2] + s_rest[3]);
      }
      off = (float)(rest / D) * by;
    }
    float s1 = 0, s2 = 0;
    R::each(t, D, [&](int i, int, bool in) {
      x[i] = in ? fmaf(x[i] - mean, by, -off) : 0.f;
      dw[i] = fmaf(g[i], x[i], dw[i]);
      db[i] += g[i];
      g[i] *= f[i];
      s1 += g[i];
      s2 = fmaf(g[i], x[i], s2);
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      s1 += __shfl_xor(s1, o, 64);
      s2 += __shfl_xor(s2, o, 64);
    }
    if constexpr (WPR > 1) {
      if ((threadIdx.x & 63) == 0) {
        s_red[turn][w][0] = s1;
        s_red[turn][w][1] = s2;
      }
      __syncthreads();
      s1 = (s_red[turn][0][0] + s_red[turn][1][0]) + (s_red[turn][2][0] + s_red[turn][3][0]);
      s2 = (s_red[turn][0][1] + s_red[turn][1][1]) + (s_red[turn][2][1] + s_red[turn][3][1]);
    }
    if (a.dx) {
      const float m1 = s1 / (float)D, m2 = s2 / (float)D;
      float r[4 * NC];
      R::load(r, a.residual ? a.residual + m * D : nullptr, t, D);
#pragma unroll
      for (int i = 0; i < 4 * NC; ++i) r[i] = fmaf(rstd, (g[i] - m1) - x[i] * m2, r[i]);
      R::store(a.dx + m * D, r, t, D);
    }
  }
  if (!a.dweight && !a.dbias) return;
  float *ow, *ob;
  if (a.chunks == 1) {
    ow = a.dweight ? a.dweight + group * D : nullptr;
    ob = a.dbias ? a.dbias + group * D : nullptr;
  } else {
    ow = a.partial + (int64_t)blockIdx.x * 2 * D;
    ob = ow + D;
  }
  if constexpr (WPR == 1) {
    constexpr int HALF = 256 * NC;
    for (int k = 0; k < 4; ++k) {
      if (w == k) {
#pragma unroll
        for (int i = 0; i < 4 * NC; ++i) {
          float *p = s_acc + 64 * i + t, *q = p + HALF;
          dw[i] += k ? *p : 0.f;
          db[i] += k ? *q : 0.f;
          *p = dw[i];
          *q = db[i];
        }
      }
      __syncthreads();
    }
    if (w != 3) return;
  }
  if (ow) R::store(ow, dw, t, D);
  if (ob) R::store(ob, db, t, D);
}

// dweight and dbias of a group: the sums of its chunks, in order.  16 threads a column take every 16th chunk each.
__global__ __launch_bounds__(1024) void k_layer_norm_sum(int D, int chunks, int64_t groups, const float *partial, float *dweight, float *dbias) {
  __shared__ double part[16][64];
  const int col = blockIdx.x * 64 + (threadIdx.x & 63), slice = threadIdx.x >> 6;
  const int which = blockIdx.y;                       // 0: dweight, 1: dbias
  float *dst = which ? dbias : dweight;
  if (!dst) return;                                   // the whole workgroup
  for (int64_t group = blockIdx.z; group < groups; group += gridDim.z) {
    double s = 0;
    if (col < D) {
      const float *p = partial + (group * chunks * 2 + which) * (int64_t)D + col;
#pragma unroll 4
      for (int c = slice; c < chunks; c += 16) s += (double)p[(int64_t)c * 2 * D];
    }
    part[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice == 0 && col < D) {
      for (int i = 1; i < 16; ++i) s += part[i][threadIdx.x];
      dst[group * D + col] = (float)s;
    }
    __syncthreads();
  }
}

bool on16(std::initializer_list<const void *> all) {
  for (const void *p : all)
    if ((uintptr_t)p % 16) return false;
  return true;
}

template <typename T, int WPR, int NC>
hipError_t launch_norm(const LayerNormArgs &a, bool vec, hipStream_t s) {
  const int64_t want = (a.M + 4 / WPR - 1) / (4 / WPR);
  const dim3 grid((unsigned)std::min<int64_t>(want, 1 << 20));
  if (vec) hipLaunchKernelGGL((k_layer_norm<T, WPR, NC, true>), grid, dim3(THREADS), 0, s, a);
  else hipLaunchKernelGGL((k_layer_norm<T, WPR, NC, false>), grid, dim3(THREADS), 0, s, a);
  return hipGetLastError();
}

template <typename T, int WPR, int NC>
hipError_t launch_grad(const LayerNormGradArgs &a, int64_t blocks, bool vec, hipStream_t s) {
  const size_t lds = WPR == 1 ? 2 * 256 * NC * sizeof(float) : 0;
  if (vec) hipLaunchKernelGGL((k_layer_norm_grad<T, WPR, NC, true>), dim3((unsigned)blocks), dim3(THREADS), lds, s, a);
  else hipLaunchKernelGGL((k_layer_norm_grad<T, WPR, NC, false>), dim3((unsigned)blocks), dim3(THREADS), lds, s, a);
  return hipGetLastError();
}

// Pieces a lane of one or of four waves holds, few enough to hold the row.  What the edges are worth, beside the next class (us,
// bf16 unless fp32 is named): 24960 x 512 two pieces 16, its gradient 37, six 23 and 47; 24960 x 1536 six 42 and 121 (fp32 54 and
// 137), eight 45 and 124 (52 and 141); 8192 x 2048 one wave 23 and 51, four 22 and 54; 16384 x 5120 five 98 and 265 (fp32 122 and
// 287), six 102 and 250 (118 and 284).  Rows of 513 to 1024 would need a class of their own: 1037 x 701 takes 24 single loads a
// lane where 11 hold the row.
#define FB_BY_WIDTH(call)                          \
  do {                                             \
    if (D <= 512) { return call(1, 2); }           \
    if (D <= 1536) { return call(1, 6); }          \
    if (D <= 2048) { return call(1, 8); }          \
    if (D <= 4096) { return call(4, 4); }          \
    if (D <= 5120) { return call(4, 5); }          \
    return call(4, 6);                             \
  } while (0)

template <typename T>
hipError_t norm_by_width(const LayerNormArgs &a, bool vec, hipStream_t s) {
  const int D = a.D;
#define FB_CALL(WPR, NC) launch_norm<T, WPR, NC>(a, vec, s)
  FB_BY_WIDTH(FB_CALL);
#undef FB_CALL
}

template <typename T>
hipError_t grad_by_width(const LayerNormGradArgs &a, int64_t blocks, bool vec, hipStream_t s) {
  const int D = a.D;
#define FB_CALL(WPR, NC) launch_grad<T, WPR, NC>(a, blocks, vec, s)
  FB_BY_WIDTH(FB_CALL);
#undef FB_CALL
}

// Rows of a chunk: four workgroups a CU (by the 256 of the card, not those seen: the order of the sums goes by it), and not
// fewer than a row a wave (1037 x 701, fp32: 17 us in chunks of 16 rows, 10 of 4).
int chunk_rows(int64_t M, int per) {
  return (int)std::min<int64_t>(per, std::max<int64_t>(4, (M + 1023) / 1024));
}

}  // namespace

hipError_t launch_layer_norm(ActType t, const LayerNormArgs &a, hipStream_t s) {
  const bool vec = a.D % 4 == 0 && on16({a.x, a.weight, a.bias, a.out});
  return t == ACT_BF16 ? norm_by_width<bf16>(a, vec, s) : norm_by_width<float>(a, vec, s);
}

size_t layer_norm_grad_workspace(int64_t M, int D, int per) {
  const int rows = chunk_rows(M, per);
  const int64_t groups = (M + per - 1) / per, chunks = (per + rows - 1) / rows;
  return chunks == 1 ? 0 : (size_t)(groups * chunks * 2) * D * sizeof(float);
}

int64_t layer_norm_grad_blocks(int64_t M, int per) {
  const int rows = chunk_rows(M, per);
  return (M + per - 1) / per * ((per + rows - 1) / rows);
}

hipError_t launch_layer_norm_grad(ActType t, LayerNormGradArgs a, hipStream_t s) {
  a.rows = chunk_rows(a.M, a.per);
  a.chunks = (a.per + a.rows - 1) / a.rows;
  const int64_t groups = (a.M + a.per - 1) / a.per;
  const bool vec = a.D % 4 == 0 && on16({a.x, a.weight, a.dy, a.residual, a.dx, a.dweight, a.dbias, a.partial});
  const hipError_t e = t == ACT_BF16 ? grad_by_width<bf16>(a, groups * a.chunks, vec, s)
                                     : grad_by_width<float>(a, groups * a.chunks, vec, s);
  if (e != hipSuccess || a.chunks == 1 || (!a.dweight && !a.dbias)) return e;
  hipLaunchKernelGGL(k_layer_norm_sum, dim3((unsigned)((a.D + 63) / 64), 2, (unsigned)std::min<int64_t>(groups, 65535)), dim3(1024), 0, s,
                     a.D, a.chunks, groups, a.partial, a.dweight, a.dbias);
  return hipGetLastError();
}

}  // namespace fb
