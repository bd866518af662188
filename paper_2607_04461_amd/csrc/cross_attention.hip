// Cross-attention to prompts of their own lengths, and its gradient.  Candidate b attends with its tq queries to the first
// len keys of its prompt; query heads may share a key head.  With scores S = q k^T / sqrt(dh):
//   P = exp(S - lse),  out = P v,  lse = log sum exp S;   an empty prompt: out = 0, lse = -inf
//   delta = sum_d dout out,  dS = P (dout v^T - delta) / sqrt(dh),  dq = dS k,  dk = dS^T q,  dv = P^T dout
// dk and dv are summed over the prompt's candidates and the heads that share the key head, in their order; no atomics.
//
// All kernels keep one side in registers and take the other in tiles through LDS, and form the scores so that a lane's
// values belong to one row of the side it keeps: the products of two tiles then are the right operand of the next product as
// they stand, with its k in an order that the left operand follows.  P and dS are rounded to the operands' type for that
// product (bf16: 8 bits, as the values they meet; in two parts where that is free: forward with 16 queries a wave or heads of
// at most 32, in the gradient everywhere but in x32 with more than 64 keys and queries).
//   * k_cross: a wave keeps 16 or 32 queries.  One pass over the keys with the running maximum and sum.
//   * k_cross_dq: the same with dout, lse and delta, which it forms: two products give P and dP, the third dq.
//   * k_cross_dkv: a wave keeps keys and values; the queries and dout of all candidates of the prompt pass by.
//   * x32::k_dq, x32::k_dkv: the same for bf16 and head dims 64 and 128, on 32 x 32 x 16 products.
// bf16 of head dim 128 with more than 64 queries runs forward on k_attn_fa (attention.hip).
// Bound by the matrix cores for many queries, by the reading of k and v for few: then ranges of keys go to several
// workgroups and k_cross_join joins them (one query of 40 heads to 4001 keys: 18 us and 4, 82 MB at 4.5 TB/s).  fp32, 4 x 12
// heads of 1560 x 512, head dim 128: forward 193 us (102 TFLOP/s of 154), gradient 635.
#include <algorithm>

#include "fragments.h"
#include "kernels.h"

namespace fb {
namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct CrossP {
  CrossArgs a;
  int nqb;                // blocks of queries
  int splits;             // ranges of keys (k_cross) or of queries (k_cross_dkv)
  float qscale, scale;    // log2(e) / sqrt(dh), 1 / sqrt(dh)
  float *part;            // workspace: partial results
  const void *dout;
  void *dq, *dk, *dv;
  float *delta;           // [batch][heads][tq]
};

__device__ __forceinline__ int prompt_of(const CrossArgs &a, int b) {
  if (!a.kv_index) return min(b, a.n_kv - 1);
  return max(0, min(a.kv_index[b], a.n_kv - 1));
}
__device__ __forceinline__ int keys_of(const CrossArgs &a, int c) { return a.kv_len ? max(0, min(a.kv_len[c], a.tk)) : a.tk; }

// A tile of ROWS rows of dh elements on their way through 256 registers' threads into LDS: rows at or past `valid` and
// columns at or past dh are zero, whatever memory holds there.
template <typename T, int ROWS, int DH, int THREADS>
struct Stage {
  static constexpr int PIECE = 16 / sizeof(T), PITCH = DH + PIECE, PER_ROW = DH / PIECE;
  static constexpr int N = (ROWS * PER_ROW + THREADS - 1) / THREADS;
  u32x4 v[N];
  __device__ __forceinline__ void load(const T *base, int64_t stride, int valid, int dh) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = threadIdx.x + THREADS * i, row = p / PER_ROW, c = p % PER_ROW * PIECE;
      v[i] = row < valid && c < dh && row < ROWS ? *reinterpret_cast<const u32x4 *>(base + row * stride + c) : u32x4{0, 0, 0, 0};
    }
  }
  __device__ __forceinline__ void land(T *lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int p = threadIdx.x + THREADS * i, row = p / PER_ROW, c = p % PER_ROW * PIECE;
      if (row < ROWS) *reinterpret_cast<u32x4 *>(lds + row * PITCH + c) = v[i];
    }
  }
};

// fragments of a row of dh elements, zero past dh; `ok` false: zero
template <typename T, int DH>
__device__ __forceinline__ void row_frags(Frag<T> (&f)[DH / 32], const T *row, int dh, bool ok) {
  const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
  for (int c = 0; c < DH / 32; ++c) f[c] = ok && 32 * c + 8 * g < dh ? load_frag(row + 32 * c + 8 * g) : zero_frag<T>();
}

// right operand of the next product out of two tiles of scores
template <typename T>
__device__ __forceinline__ Frag<T> pair_frag(f32x4 lo, f32x4 hi) {
  Frag<T> f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = from_f32<T>(lo[i]);
    f[4 + i] = from_f32<T>(hi[i]);
  }
  return f;
}

// What rounding two tiles to f left.  A second product with it gives a sum the digits of fp32 operands: P and dS rounded to
// bf16 are off by 2^-8 each, which counts as much in a result as its own rounding.
template <typename T>
__device__ __forceinline__ Frag<T> rest_frag(f32x4 lo, f32x4 hi, Frag<T> f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    lo[e] -= to_f32(f[e]);
    hi[e] -= to_f32(f[4 + e]);
  }
  return pair_frag<T>(lo, hi);
}

__device__ __forceinline__ float across(float v, bool maximum) {   // over the four lanes of a column
#pragma unroll
  for (int o = 16; o < 64; o <<= 1) {
    const float w = __shfl_xor(v, o, 64);
    v = maximum ? fmaxf(v, w) : v + w;
  }
  return v;
}

// workgroup -> (unit, query block): the query blocks of a unit stay on one XCD (ids go round the eight)
__device__ __forceinline__ bool unit_of(const CrossP &p, int id, int &b, int &h, int &qb) {
  const int rest = id >> 3, u = rest / p.nqb * 8 + (id & 7);
  if (u >= p.a.batch * p.a.heads) return false;
  h = u / p.a.batch;
  b = u % p.a.batch;
  qb = rest % p.nqb;
  return true;
}

// Scores whose exponents (base 2) pass 2^30 differ by 2^8 or not at all, and the rounding of a product with the scale would pass
// any power's range: their differences are taken as they are.
__device__ __forceinline__ bool far(float exponent) { return fabsf(exponent) > 0x1p30f; }

template <typename T> constexpr int TILE = sizeof(T) == 2 ? 64 : 32;    // rows of a tile in LDS

// Two waves a SIMD are asked for in all three kernels, which also keeps their accumulators out of the accumulation registers:
// fp32, the sizes above, forward 211 -> 189 us, gradient 747 -> 635 (k_cross_dkv had 307 registers, one wave a SIMD).
// k_cross_dkv for bf16 of head dim 128 keeps one: 487 registers would spill.
template <typename T, int DH, int NQ, bool SPLIT>
__global__ __launch_bounds__(256, 2) void k_cross(CrossP p) {
  constexpr int KT = TILE<T>, NS = KT / 16, NC = DH / 32, ND = DH / 16;
  // 16 queries a wave are bound by the reading of k and v, and small heads by the scores: there P goes in two parts
  constexpr int PARTS = sizeof(T) == 2 && (NQ == 1 || DH == 32) ? 2 : 1;
  typedef Stage<T, KT, DH, 256> St;
  extern __shared__ __attribute__((aligned(16))) char s_mem[];
  T *sk = reinterpret_cast<T *>(s_mem), *sv = sk + KT * St::PITCH;
  int b, h, qb;
  if (!unit_of(p, blockIdx.x, b, h, qb)) return;
  const CrossArgs &a = p.a;
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4, w = threadIdx.x >> 6;
  const int q0 = (qb * 4 + w) * 16 * NQ, c = prompt_of(a, b), len = keys_of(a, c), kh = h / (a.heads / a.kv_heads);
  const bool idle = q0 >= a.tq;
  const int tiles = (len + KT - 1) / KT;
  const int t0 = SPLIT ? (int)((int64_t)tiles * blockIdx.y / p.splits) : 0;
  const int t1 = SPLIT ? (int)((int64_t)tiles * (blockIdx.y + 1) / p.splits) : tiles;
  const T *K = (const T *)a.k + c * a.kv_bs + kh * a.head_dim, *V = (const T *)a.v + c * a.kv_bs + kh * a.head_dim;
  Frag<T> qf[NQ][NC];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int i = q0 + 16 * n + li;
    row_frags<T, DH>(qf[n], (const T *)a.q + b * a.q_bs + (int64_t)min(i, a.tq - 1) * a.q_rs + h * a.head_dim, a.head_dim, i < a.tq);
  }
  f32x4 o[NQ][ND];
  float top[NQ], off[NQ], sum[NQ];        // the running maximum, what exponents are taken less (base 2), and the sum
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    top[n] = -INFINITY;
    off[n] = -3.4028235e38f;
    sum[n] = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  St ks, vs;
  auto load = [&](int t) __attribute__((always_inline)) {
    ks.load(K + (int64_t)t * KT * a.kv_rs, a.kv_rs, len - t * KT, a.head_dim);
    vs.load(V + (int64_t)t * KT * a.kv_rs, a.kv_rs, len - t * KT, a.head_dim);
  };
  if (t0 < t1) load(t0);
  for (int t = t0; t < t1; ++t) {
    __syncthreads();          // the last tile has been read
    ks.land(sk);
    vs.land(sv);
    __syncthreads();
    if (t + 1 < t1) load(t + 1);
    if (idle) continue;
    f32x4 s[NQ][NS];
#pragma unroll
    for (int j = 0; j < NS; ++j) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) s[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        const Frag<T> kf = load_frag(sk + (16 * j + li) * St::PITCH + 32 * k + 8 * g);
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][j] = mma(kf, qf[n][k], s[n][j]);
      }
    }
    if ((t + 1) * KT > len) {
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (t * KT + 16 * j + 4 * g + e >= len) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) s[n][j][e] = -INFINITY;
          }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float m = top[n];
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, s[n][j][e]);
      m = across(m, true);
      // as the exponents have it, rounding and all: a maximum that stays leaves the sums as they are
      float next = m == -INFINITY ? off[n] : rounded_product(m, p.qscale), scale = p.qscale;     // a row of -inf only: all of it 0
      if (far(next)) {
        next = m == -INFINITY ? off[n] : m;
        scale = 1.f;
      }
      const float shrink = __builtin_amdgcn_exp2f(off[n] - next);
      top[n] = m;
      off[n] = next;
      sum[n] *= shrink;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][d][e] *= shrink;
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][j][e] = __builtin_amdgcn_exp2f(fmaf(s[n][j][e], scale, -next));
          sum[n] += s[n][j][e];
        }
    }
#pragma unroll
    for (int j = 0; j < NS; j += 2) {
      Frag<T> pf[NQ], rest[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        pf[n] = pair_frag<T>(s[n][j], s[n][j + 1]);
        if constexpr (PARTS == 2) rest[n] = rest_frag<T>(s[n][j], s[n][j + 1], pf[n]);
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const Frag<T> vf = load_column_frag(sv, St::PITCH, 16 * d, 16 * j + 4 * g, 16 * j + 16 + 4 * g);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          o[n][d] = mma(vf, pf[n], o[n][d]);
          if constexpr (PARTS == 2) o[n][d] = mma(vf, rest[n], o[n][d]);
        }
      }
    }
  }
  if (idle) return;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int i = q0 + 16 * n + li;
    const float l = across(sum[n], false);
    if (i >= a.tq) continue;
    if constexpr (SPLIT) {
      // [row][split][dh + 4]: the sums as they stand, what their exponents were taken less, the sum and the maximum
      float *dst = p.part + ((((int64_t)b * a.heads + h) * a.tq + i) * p.splits + blockIdx.y) * (a.head_dim + 4);
#pragma unroll
      for (int d = 0; d < ND; ++d)
        if (16 * d + 4 * g < a.head_dim) *reinterpret_cast<f32x4 *>(dst + 16 * d + 4 * g) = o[n][d];
      if (g == 0) {
        dst[a.head_dim] = off[n];
        dst[a.head_dim + 1] = l;
        dst[a.head_dim + 2] = top[n];
      }
    } else {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      T *O = (T *)a.out + b * a.o_bs + (int64_t)i * a.o_rs + h * a.head_dim;
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const int at = 16 * d + 4 * g;
        if (at >= a.head_dim) continue;
        if constexpr (sizeof(T) == 4)
          *reinterpret_cast<f32x4 *>(O + at) = f32x4{o[n][d][0] * inv, o[n][d][1] * inv, o[n][d][2] * inv, o[n][d][3] * inv};
        else
          *reinterpret_cast<bf16x4 *>(O + at) = bf16x4{(bf16)(o[n][d][0] * inv), (bf16)(o[n][d][1] * inv),
                                                       (bf16)(o[n][d][2] * inv), (bf16)(o[n][d][3] * inv)};
      }
      if (a.lse && g == 0)
        a.lse[((int64_t)b * a.heads + h) * a.tq + i] = l == 0.f ? -INFINITY : ((far(off[n]) ? top[n] * p.qscale : off[n]) + log2f(l)) * LN2;
    }
  }
}

// A row of the output out of its ranges of keys: one wave a row.
template <typename T>
__global__ __launch_bounds__(256) void k_cross_join(CrossP p) {
  const CrossArgs &a = p.a;
  const int64_t rows = (int64_t)a.batch * a.heads * a.tq;
  const int lane = threadIdx.x & 63;
  for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += (int64_t)gridDim.x * 4) {
    const int i = (int)(r % a.tq), h = (int)(r / a.tq % a.heads), b = (int)(r / a.tq / a.heads);
    const int pitch = a.head_dim + 4;
    const float *src = p.part + r * p.splits * pitch;
    // lane s: the maximum and sum of range s (at most 64), then its factor and the row's sum
    const float ls = lane < p.splits ? src[lane * pitch + a.head_dim + 1] : 0.f;
    float ms = lane < p.splits ? src[lane * pitch + a.head_dim] : -INFINITY;
    const float raw = lane < p.splits ? src[lane * pitch + a.head_dim + 2] : -INFINITY;
    float v[16][2];        // the first ranges' sums, on their way meanwhile
    auto load = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
      for (int s = 0; s < 16; ++s)
#pragma unroll
        for (int e = 0; e < 2; ++e) v[s][e] = s0 + s < p.splits && lane + 64 * e < a.head_dim ? src[(s0 + s) * pitch + lane + 64 * e] : 0.f;
    };
    load(0);
    // far scores' ranges are told apart by their maxima themselves
    const float most = wave_max(ls != 0.f ? raw : -INFINITY);
    const bool apart = far(most * p.qscale);
    if (apart) ms = raw;
    const float top = wave_max(ls != 0.f ? ms : -INFINITY);
    const float mine = ls != 0.f ? __builtin_amdgcn_exp2f(ms - (top == -INFINITY ? 0.f : top)) : 0.f;
    const float l = wave_sum(mine * ls);
    float o[2] = {0.f, 0.f};
    for (int s0 = 0; s0 < p.splits; s0 += 16) {
      if (s0) load(s0);
#pragma unroll
      for (int s = 0; s < 16; ++s) {
        const float f = __shfl(mine, s0 + s, 64);      // splits <= 64; 0 past them and for an empty range
#pragma unroll
        for (int e = 0; e < 2; ++e) o[e] = fmaf(f, f != 0.f ? v[s][e] : 0.f, o[e]);
      }
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    T *O = (T *)a.out + b * a.o_bs + (int64_t)i * a.o_rs + h * a.head_dim;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (lane + 64 * e < a.head_dim) O[lane + 64 * e] = from_f32<T>(o[e] * inv);
    if (a.lse && lane == 0) a.lse[r] = l == 0.f ? -INFINITY : ((apart ? top * p.qscale : top) + log2f(l)) * LN2;
  }
}

// The keys that dq sums over: one key alone has P = 1 whatever its score, and dP - delta would be the rounding of both.
__device__ __forceinline__ int scored_keys(int len) { return len == 1 ? 0 : len; }

// delta of a row: the sums of eight products each, added in pairs 8, 4, 2 and 1 eights apart.  The same in k_cross_delta and
// in the kernels of dq, so that dk and dv do not depend on whether dq is asked for.
template <typename T>
__device__ __forceinline__ float eight_products(Frag<T> x, Frag<T> y) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(to_f32(x[e]), to_f32(y[e]), s);
  return s;
}
template <typename T>
__device__ __forceinline__ float row_delta(Frag<T> x, Frag<T> y, int lanes) {
  float s = eight_products<T>(x, y);
  for (int o = lanes >> 1; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  return s;
}

// delta[b][h][i] = sum_d dout out
template <typename T>
__global__ __launch_bounds__(256) void k_cross_delta(CrossP p) {
  const CrossArgs &a = p.a;
  const int lanes = a.head_dim / 8, at = threadIdx.x % lanes;
  const int64_t rows = (int64_t)a.batch * a.tq * a.heads, step = (int64_t)gridDim.x * (256 / lanes);
  for (int64_t r = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes; r < rows; r += step) {   // a row's lanes together
    const int h = (int)(r % a.heads), i = (int)(r / a.heads % a.tq), b = (int)(r / a.heads / a.tq);
    const int64_t from = b * a.o_bs + (int64_t)i * a.o_rs + h * a.head_dim + 8 * at;
    const float s = row_delta<T>(load_frag((const T *)a.out + from), load_frag((const T *)p.dout + from), lanes);
    if (at == 0) p.delta[((int64_t)b * a.heads + h) * a.tq + i] = s;
  }
}

template <typename T, int DH, int NQ>
__global__ __launch_bounds__(256, 2) void k_cross_dq(CrossP p) {
  constexpr int KT = TILE<T>, NS = KT / 16, NC = DH / 32, ND = DH / 16;
  typedef Stage<T, KT, DH, 256> St;
  extern __shared__ __attribute__((aligned(16))) char s_mem[];
  T *sk = reinterpret_cast<T *>(s_mem), *sv = sk + KT * St::PITCH;
  int b, h, qb;
  if (!unit_of(p, blockIdx.x, b, h, qb)) return;
  const CrossArgs &a = p.a;
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4, w = threadIdx.x >> 6;
  const int q0 = (qb * 4 + w) * 16 * NQ, c = prompt_of(a, b), len = keys_of(a, c), kh = h / (a.heads / a.kv_heads);
  const bool idle = q0 >= a.tq;
  const int tiles = (scored_keys(len) + KT - 1) / KT;
  const T *K = (const T *)a.k + c * a.kv_bs + kh * a.head_dim, *V = (const T *)a.v + c * a.kv_bs + kh * a.head_dim;
  Frag<T> qf[NQ][NC], df[NQ][NC];
  float lse[NQ], delta[NQ];       // base 2; +inf: the row's probabilities are 0
  f32x4 o[NQ][ND];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int i = q0 + 16 * n + li, at = min(i, a.tq - 1);
    row_frags<T, DH>(qf[n], (const T *)a.q + b * a.q_bs + (int64_t)at * a.q_rs + h * a.head_dim, a.head_dim, i < a.tq);
    row_frags<T, DH>(df[n], (const T *)p.dout + b * a.o_bs + (int64_t)at * a.o_rs + h * a.head_dim, a.head_dim, i < a.tq);
    const int64_t r = ((int64_t)b * a.heads + h) * a.tq + at;
    lse[n] = i < a.tq && a.lse[r] != -INFINITY ? a.lse[r] * LOG2E : INFINITY;
    {   // delta in k_cross_delta's order: a lane has eights g, 4 + g, 8 + g, 12 + g of the row
      Frag<T> of[NC];
      row_frags<T, DH>(of, (const T *)a.out + b * a.o_bs + (int64_t)at * a.o_rs + h * a.head_dim, a.head_dim, i < a.tq);
      float e[NC];
#pragma unroll
      for (int k = 0; k < NC; ++k) e[k] = eight_products<T>(of[k], df[n][k]);
      float s = NC == 4 ? (e[0] + e[NC / 2]) + (e[NC > 1 ? 1 : 0] + e[NC - 1]) : NC == 2 ? e[0] + e[NC - 1] : e[0];
      s += __shfl_xor(s, 32, 64);
      s += __shfl_xor(s, 16, 64);
      delta[n] = s;
      if (g == 0 && i < a.tq) p.delta[r] = s;
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  St ks, vs;
  auto load = [&](int t) __attribute__((always_inline)) {
    ks.load(K + (int64_t)t * KT * a.kv_rs, a.kv_rs, len - t * KT, a.head_dim);
    vs.load(V + (int64_t)t * KT * a.kv_rs, a.kv_rs, len - t * KT, a.head_dim);
  };
  if (tiles) load(0);
  for (int t = 0; t < tiles; ++t) {
    __syncthreads();          // the last tile has been read
    ks.land(sk);
    vs.land(sv);
    __syncthreads();
    if (t + 1 < tiles) load(t + 1);
    if (idle) continue;
#pragma unroll
    for (int j = 0; j < NS; j += 2) {
      f32x4 s[NQ][2], dp[NQ][2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) s[n][x] = dp[n][x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          const Frag<T> kf = load_frag(sk + (16 * (j + x) + li) * St::PITCH + 32 * k + 8 * g);
          const Frag<T> vf = load_frag(sv + (16 * (j + x) + li) * St::PITCH + 32 * k + 8 * g);
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            s[n][x] = mma(kf, qf[n][k], s[n][x]);
            dp[n][x] = mma(vf, df[n][k], dp[n][x]);
          }
        }
      }
      Frag<T> pf[NQ], rest[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // keys past the end meet rows of zeros in k, which take nothing of them; their scores are 0, not masked
            const float pr = __builtin_amdgcn_exp2f(fmaf(s[n][x][e], p.qscale, -lse[n]));
            const bool in = t * KT + 16 * (j + x) + 4 * g + e < len;
            s[n][x][e] = in ? pr * (dp[n][x][e] - delta[n]) : 0.f;
          }
        pf[n] = pair_frag<T>(s[n][0], s[n][1]);
        if constexpr (sizeof(T) == 2) rest[n] = rest_frag<T>(s[n][0], s[n][1], pf[n]);
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const Frag<T> kf = load_column_frag(sk, St::PITCH, 16 * d, 16 * j + 4 * g, 16 * j + 16 + 4 * g);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          o[n][d] = mma(kf, pf[n], o[n][d]);
          if constexpr (sizeof(T) == 2) o[n][d] = mma(kf, rest[n], o[n][d]);
        }
      }
    }
  }
  if (idle) return;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int i = q0 + 16 * n + li;
    if (i >= a.tq) continue;
    T *O = (T *)p.dq + b * a.q_bs + (int64_t)i * a.q_rs + h * a.head_dim;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const int at = 16 * d + 4 * g;
      if (at >= a.head_dim) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[n][d][e] *= p.scale;
      if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4 *>(O + at) = o[n][d];
      else *reinterpret_cast<bf16x4 *>(O + at) = bf16x4{(bf16)o[n][d][0], (bf16)o[n][d][1], (bf16)o[n][d][2], (bf16)o[n][d][3]};
    }
  }
}

// The prompt's candidates in order into list, by the first wave; their number.
__device__ __forceinline__ void list_candidates(const CrossArgs &a, int c, int *list, int *count) {
  if (threadIdx.x < 64) {
    int n = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
      const bool mine = b0 + (int)threadIdx.x < a.batch && prompt_of(a, b0 + threadIdx.x) == c;
      const uint64_t votes = __ballot(mine);
      if (mine) list[n + __popcll(votes & ((1ull << threadIdx.x) - 1))] = b0 + threadIdx.x;
      n += __popcll(votes);
    }
    if (threadIdx.x == 0) *count = n;
  }
  __syncthreads();
}

// Keys [128 kb ...) of a prompt's key head against a range of the (candidate, head, query tile) triples that read them.
template <typename T, int DH, int NK>
__global__ __launch_bounds__(256, sizeof(T) == 2 && DH == 128 ? 1 : 2) void k_cross_dkv(CrossP p) {
  constexpr int QT = TILE<T>, NS = QT / 16, NC = DH / 32, ND = DH / 16, KB = 64 * NK;
  typedef Stage<T, QT, DH, 256> St;
  extern __shared__ __attribute__((aligned(16))) char s_mem[];
  T *sq = reinterpret_cast<T *>(s_mem), *sd = sq + QT * St::PITCH;
  float *s_lse = reinterpret_cast<float *>(sd + QT * St::PITCH), *s_delta = s_lse + QT;
  int *s_list = reinterpret_cast<int *>(s_delta + QT), *s_count = s_list + p.a.batch;
  const CrossArgs &a = p.a;
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4, w = threadIdx.x >> 6;
  const int kb = blockIdx.x, c = blockIdx.y / a.kv_heads, kh = blockIdx.y % a.kv_heads, split = blockIdx.z;
  const int len = keys_of(a, c), shared = a.heads / a.kv_heads;
  if (p.splits > 1 && kb * KB >= len) return;       // k_cross_sum writes those rows
  list_candidates(a, c, s_list, s_count);
  const int key0 = kb * KB + w * 16 * NK;
  const T *K = (const T *)a.k + c * a.kv_bs + kh * a.head_dim, *V = (const T *)a.v + c * a.kv_bs + kh * a.head_dim;
  Frag<T> kf[NK][NC], vf[NK][NC];
  f32x4 dk[NK][ND], dv[NK][ND];
#pragma unroll
  for (int n = 0; n < NK; ++n) {
    const int i = key0 + 16 * n + li;
    const int64_t at = (int64_t)min(i, a.tk - 1) * a.kv_rs;
    row_frags<T, DH>(kf[n], K + at, a.head_dim, i < len);
    row_frags<T, DH>(vf[n], V + at, a.head_dim, i < len);
#pragma unroll
    for (int d = 0; d < ND; ++d) dk[n][d] = dv[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int nqt = (a.tq + QT - 1) / QT;
  const int64_t all = kb * KB < len ? (int64_t)*s_count * shared * nqt : 0;
  const int64_t u0 = all * split / p.splits, u1 = all * (split + 1) / p.splits;
  St qs, ds;
  float ls = 0.f, de = 0.f;
  int left = 0;               // queries of the tile loaded last, and what lies past it
  auto load = [&](int64_t u) __attribute__((always_inline)) {
    const int qt = (int)(u % nqt), h = kh * shared + (int)(u / nqt % shared), b = s_list[u / nqt / shared];
    const int64_t i0 = (int64_t)qt * QT;
    left = a.tq - qt * QT;
    qs.load((const T *)a.q + b * a.q_bs + i0 * a.q_rs + h * a.head_dim, a.q_rs, a.tq - qt * QT, a.head_dim);
    ds.load((const T *)p.dout + b * a.o_bs + i0 * a.o_rs + h * a.head_dim, a.o_rs, a.tq - qt * QT, a.head_dim);
    if (threadIdx.x < QT) {
      const bool ok = i0 + threadIdx.x < a.tq;
      const int64_t r = ((int64_t)b * a.heads + h) * a.tq + (ok ? i0 + threadIdx.x : 0);
      ls = ok && a.lse[r] != -INFINITY ? a.lse[r] * LOG2E : INFINITY;
      de = ok ? p.delta[r] : 0.f;
    }
  };
  if (u0 < u1) load(u0);
  for (int64_t u = u0; u < u1; ++u) {
    __syncthreads();          // the last tile has been read
    qs.land(sq);
    ds.land(sd);
    if (threadIdx.x < QT) {
      s_lse[threadIdx.x] = ls;
      s_delta[threadIdx.x] = de;
    }
    __syncthreads();
    if (left < QT) {          // the last query again in place of rows of zeros, which would meet an infinite key with a NaN
      for (int e = threadIdx.x; e < (QT - left) * DH; e += 256) sq[(left + e / DH) * St::PITCH + e % DH] = sq[(left - 1) * St::PITCH + e % DH];
      __syncthreads();
    }
    if (u + 1 < u1) load(u + 1);
    if (key0 >= len) continue;
#pragma unroll
    for (int j = 0; j < NS; j += 2) {
      f32x4 s[NK][2], dp[NK][2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int n = 0; n < NK; ++n) s[n][x] = dp[n][x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NC; ++k) {
          const Frag<T> qf = load_frag(sq + (16 * (j + x) + li) * St::PITCH + 32 * k + 8 * g);
          const Frag<T> df = load_frag(sd + (16 * (j + x) + li) * St::PITCH + 32 * k + 8 * g);
#pragma unroll
          for (int n = 0; n < NK; ++n) {
            s[n][x] = mma(qf, kf[n][k], s[n][x]);
            dp[n][x] = mma(df, vf[n][k], dp[n][x]);
          }
        }
        const f32x4 l4 = *reinterpret_cast<const f32x4 *>(s_lse + 16 * (j + x) + 4 * g);
        const f32x4 d4 = *reinterpret_cast<const f32x4 *>(s_delta + 16 * (j + x) + 4 * g);
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[n][x][e] = __builtin_amdgcn_exp2f(fmaf(s[n][x][e], p.qscale, -l4[e]));
            dp[n][x][e] = s[n][x][e] * (dp[n][x][e] - d4[e]);
          }
      }
      Frag<T> pf[NK], sf[NK], pr[NK], sr[NK];
#pragma unroll
      for (int n = 0; n < NK; ++n) {
        pf[n] = pair_frag<T>(s[n][0], s[n][1]);
        sf[n] = pair_frag<T>(dp[n][0], dp[n][1]);
        if constexpr (sizeof(T) == 2) {
          pr[n] = rest_frag<T>(s[n][0], s[n][1], pf[n]);
          sr[n] = rest_frag<T>(dp[n][0], dp[n][1], sf[n]);
        }
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const Frag<T> qf = load_column_frag(sq, St::PITCH, 16 * d, 16 * j + 4 * g, 16 * j + 16 + 4 * g);
        const Frag<T> df = load_column_frag(sd, St::PITCH, 16 * d, 16 * j + 4 * g, 16 * j + 16 + 4 * g);
#pragma unroll
        for (int n = 0; n < NK; ++n) {
          dk[n][d] = mma(qf, sf[n], dk[n][d]);
          dv[n][d] = mma(df, pf[n], dv[n][d]);
          if constexpr (sizeof(T) == 2) {
            dk[n][d] = mma(qf, sr[n], dk[n][d]);
            dv[n][d] = mma(df, pr[n], dv[n][d]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NK; ++n) {
    const int i = key0 + 16 * n + li;
    if (i >= a.tk || (p.splits > 1 && i >= len)) continue;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const int at = 16 * d + 4 * g;
      if (at >= a.head_dim) continue;
      f32x4 x = dk[n][d], y = dv[n][d];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = i < scored_keys(len) ? x[e] * p.scale : 0.f;      // also rows past the prompt's end
        y[e] = i < len ? y[e] : 0.f;
      }
      if (p.splits > 1) {       // [split][prompt][tk][key head][2][dh]
        float *dst = p.part + (((((int64_t)split * a.n_kv + c) * a.tk + i) * a.kv_heads + kh) * 2) * a.head_dim + at;
        *reinterpret_cast<f32x4 *>(dst) = x;
        *reinterpret_cast<f32x4 *>(dst + a.head_dim) = y;
      } else {
        const int64_t to = c * a.kv_bs + (int64_t)i * a.kv_rs + kh * a.head_dim + at;
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<f32x4 *>((T *)p.dk + to) = x;
          *reinterpret_cast<f32x4 *>((T *)p.dv + to) = y;
        } else {
          *reinterpret_cast<bf16x4 *>((T *)p.dk + to) = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
          *reinterpret_cast<bf16x4 *>((T *)p.dv + to) = bf16x4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
        }
      }
    }
  }
}

// ---- bf16, head dims 64 and 128: 32 x 32 x 16 products, a wave's 32 queries (or keys) in registers.
// A product's lane holds rows 8 (r >> 2) + 4 g + (r & 3) of column lane & 31 (g = lane >> 5, r < 16), so registers 8 c ..
// 8 c + 7 are the right operand of the next product's 16 k of chunk c, in the order 4 g + 0..3, 8 + 4 g + 0..3.  Its left
// operand comes out of a transposed copy of the tile in LDS whose groups of four are kept in that order, so that it is one
// 16-byte read (gfx950's transposing reads pass 71 bytes a clock and CU here, 16-byte reads 190, and the products of one
// candidate's tile need 128).  The copy costs each thread a few 8-byte reads, byte permutations and writes a tile.
// 4 x 40 heads of 4096 queries, head dim 128, prompts of 512 and 300 keys (341 GFLOP as five products, 478 as the seven that
// two kernels form): k_dq 320 us, 140 of them its rows in and out at HBM's rate, k_dkv 355, k_cross_sum 23; with every prompt
// of 512 keys 715 us in all.  On 16 x 16 products k_cross_dq took 533, k_cross_dkv 670 and delta, now formed by k_dq, 65.
// Both corrections enter as the accumulators' first values: S starts at -lse, dP at -delta, so that a pair of exponent and
// product is all that is left to do for an element.
namespace x32 {

constexpr int QT = 64;               // rows of a tile
constexpr int TP = QT * 2 + 16;      // bytes of a row of the transposed copy
// 16-byte chunk c of row r of a tile without padding is kept at c ^ swz(r): the 16 rows of a read phase at one chunk fall
// into 16 different places of the banks' 256 bytes
template <int DH> __device__ __forceinline__ int swz(int r) { return DH == 128 ? r & 15 : (r >> 1) & 7; }
template <int DH> __device__ __forceinline__ int row_at(int r, int c) { return r * DH * 2 + ((c ^ swz<DH>(r)) << 4); }
// place of the four rows 4 qg .. 4 qg + 3 of column d
__device__ __forceinline__ int column_at(int d, int qg) {
  const int gi = qg & 3, place = (gi & 1) << 1 | gi >> 1, slot = (qg >> 2) * 2 + (place >> 1);
  return d * TP + ((slot ^ (d >> 4 & 7)) << 4) + (place & 1) * 8;
}
// Left operands.  Of a tile: row 32 x + li, chunk 2 k + g, at row_base ^ 32 k; of the copy: column 32 d + li, the rows of
// chunk c and lane half g, whose place (2 c + g) ^ (2 d + li / 16) is 2 (c ^ d) + (g ^ li / 16).
// A barrier for what is written to and read from LDS by instructions of its own: loads that write LDS stay in flight, which
// __syncthreads would wait for.
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// v as a new value: what is computed from it inside a loop is not kept in registers across the loop
__device__ __forceinline__ int fresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}
template <int DH> __device__ __forceinline__ int row_base(int li, int g) { return row_at<DH>(li, g); }
template <int DH> __device__ __forceinline__ bf16x8 row_frag(const char *t, int base, int x, int k) {
  return *reinterpret_cast<const bf16x8 *>(t + 32 * x * DH * 2 + (base ^ (k << 5)));
}
__device__ __forceinline__ int column_base(int li, int g) { return li * TP + ((g ^ (li >> 4)) << 4); }
__device__ __forceinline__ bf16x8 column_frag(const char *t, int base, int d, int c) {
  return *reinterpret_cast<const bf16x8 *>(t + base + d * 32 * TP + ((c ^ d) << 5));
}
// Rows 4 qg .. + 3 of columns 4 dg .. + 3, a register pair a row.  In a tile: row e at (place ^ 16 e) + e rows; in the copy:
// column e at place + e TP, with the rows of a column beside each other.
template <int DH> __device__ __forceinline__ int block_rows(int dg, int qg) { return row_at<DH>(4 * qg, dg >> 1) + (dg & 1) * 8; }
template <int DH> __device__ __forceinline__ int block_row(int place, int e) {
  return (place ^ (DH == 128 ? e << 4 : (e >> 1) << 4)) + e * DH * 2;
}
__device__ __forceinline__ int block_columns(int dg, int qg) { return column_at(4 * dg, qg); }
__device__ __forceinline__ void store_columns(char *t, const u32x2 (&r)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
    const int x = e >> 1;
    *reinterpret_cast<u32x2 *>(t + e * TP) =
        u32x2{__builtin_amdgcn_perm(r[1][x], r[0][x], sel), __builtin_amdgcn_perm(r[3][x], r[2][x], sel)};
  }
}
// `valid` rows of dh elements at stride as a buffer: what lies past it reads as zero.  off(row): a row's offset, or past it
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const bf16 *at, int stride, int valid, int dh) {
  const uint64_t x = (uint64_t)at;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  const uint32_t bytes = __builtin_amdgcn_readfirstlane((uint32_t)((valid - 1) * stride + dh) * 2u);
  return __builtin_amdgcn_make_buffer_rsrc((void *)(((uint64_t)hi << 32) | lo), (short)0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ uint32_t off(int row, int stride, int col, int valid) {
  return row < valid ? (uint32_t)(row * stride + col) * 2u : 0x80000000u;
}
// 64 lanes' 16 bytes each to LDS, one behind the other from `to` on
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t r, char *to, uint32_t offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)to, 16, offset, 0, 0, 0);
}
__device__ __forceinline__ u32x2 load_pair(__amdgpu_buffer_rsrc_t r, uint32_t offset) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, offset, 0, 0));
}
__device__ __forceinline__ f32x16 mma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
// registers 8 c .. 8 c + 7 as an operand
__device__ __forceinline__ bf16x8 chunk_frag(const f32x16 &v, int c) {
  bf16x8 f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (bf16)v[8 * c + i];
  return f;
}

__device__ __forceinline__ bf16x8 chunk_rest(const f32x16 &v, int c, bf16x8 f) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (bf16)(v[8 * c + i] - (float)f[i]);
  return r;
}

// dq of 128 queries, 32 a wave; also delta, for k_dkv.  TWO: dS in two parts (see two_parts).
template <int DH, bool TWO>
__global__ __launch_bounds__(256, 2) void k_dq(CrossP p) {
  constexpr int NC = DH / 16, ND = DH / 32, DG = DH / 4, BLOCKS = 16 * DG / 256, TILE_B = QT * DH * 2;
  constexpr int CH = DH / 8, RPI = 64 / CH, N = 32 / RPI;      // chunks of a row; rows of a 64-lane load; loads of 32 rows
  extern __shared__ __attribute__((aligned(16))) char s_mem[];
  char *sk = s_mem, *sv = sk + TILE_B, *st = sv + 2 * TILE_B;     // k; v of odd and even tiles; k transposed
  int b, h, qb;
  if (!unit_of(p, blockIdx.x, b, h, qb)) return;
  const CrossArgs &a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, g = lane >> 5, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int q0 = (qb * 4 + w) * 32, c = prompt_of(a, b), len = keys_of(a, c), kh = h / (a.heads / a.kv_heads);
  const bool idle = q0 >= a.tq;
  const int tiles = (scored_keys(len) + QT - 1) / QT, i = q0 + li, at = min(i, a.tq - 1);
  const bf16 *K = (const bf16 *)a.k + c * a.kv_bs + kh * DH, *V = (const bf16 *)a.v + c * a.kv_bs + kh * DH;
  u32x2 kr[BLOCKS][4];
  const int rs = (int)a.kv_rs, cb = column_base(li, g);
  const int dg = tid % DG, qg = tid / DG;
  auto load = [&](int t) __attribute__((always_inline)) {
    const int valid = min(QT, len - t * QT);
    const __amdgpu_buffer_rsrc_t kt = rows_rsrc(K + (int64_t)t * QT * a.kv_rs, rs, valid, DH), vt = rows_rsrc(V + (int64_t)t * QT * a.kv_rs, rs, valid, DH);
    const int kf = fresh(4 * qg), at = fresh(lane);      // offsets are made anew for each tile: they would be spilled
#pragma unroll
    for (int x = 0; x < BLOCKS; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        kr[x][e] = load_pair(kt, off(kf + 1024 / DG * x + e, rs, 4 * dg, valid));
#pragma unroll
    for (int x = 0; x < QT / RPI / 4; ++x) {
      const int first = (w * (QT / RPI / 4) + x) * RPI, row = first + at / CH;
      load_to_lds(vt, sv + ((t & 1) ^ 1) * TILE_B + first * DH * 2, off(row, rs, 8 * (at % CH ^ swz<DH>(row)), valid));
    }
  };
  auto land = [&]() __attribute__((always_inline)) {
    const int br = fresh(block_rows<DH>(dg, qg));
#pragma unroll
    for (int x = 0; x < BLOCKS; ++x) {      // 1024 / DG rows further: the same chunk, and a place 1024 / DG / 16 pairs on
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<u32x2 *>(sk + block_row<DH>(br, e) + x * (1024 / DG) * DH * 2) = kr[x][e];
      store_columns(st + fresh(block_columns(dg, qg + 256 / DG * x)), kr[x]);
    }
  };
  if (tiles) load(0);
  // The wave's rows come and go as whole rows, through LDS: a lane's own pieces of one row would take each line of memory
  // in several parts, and the loads and stores of a workgroup's queries half of its time.
  char *mine = s_mem + w * 32 * DH * 2;
  const int lrow = lane / CH, lch = lane % CH;
  bf16x8 qf[NC], df[NC];
  float lse = 0.f, delta = 0.f;
  if (!idle) {
    float *s_delta = reinterpret_cast<float *>(st) + 32 * w;
    bf16x8 qv[N], dv[N], ov[N];
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const int row = min(q0 + RPI * x + lrow, a.tq - 1);
      const int64_t from = b * a.o_bs + (int64_t)row * a.o_rs + h * DH + 8 * lch;
      qv[x] = load_frag((const bf16 *)a.q + b * a.q_bs + (int64_t)row * a.q_rs + h * DH + 8 * lch);
      dv[x] = load_frag((const bf16 *)p.dout + from);
      ov[x] = load_frag((const bf16 *)a.out + from);
    }
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const float s = row_delta<bf16>(ov[x], dv[x], CH);
      if (lch == 0) s_delta[RPI * x + lrow] = s;
      *reinterpret_cast<bf16x8 *>(mine + row_at<DH>(RPI * x + lrow, lch)) = qv[x];
    }
    const int rb = row_base<DH>(li, g);
    own_lds();
#pragma unroll
    for (int k = 0; k < NC; ++k) qf[k] = row_frag<DH>(mine, rb, 0, k);
    own_lds();
#pragma unroll
    for (int x = 0; x < N; ++x) *reinterpret_cast<bf16x8 *>(mine + row_at<DH>(RPI * x + lrow, lch)) = dv[x];
    own_lds();
#pragma unroll
    for (int k = 0; k < NC; ++k) df[k] = row_frag<DH>(mine, rb, 0, k);
    delta = s_delta[li];
    const int64_t r = ((int64_t)b * a.heads + h) * a.tq + at;
    lse = a.lse[r] == -INFINITY ? INFINITY : a.lse[r] * LOG2E / p.qscale;
    if (g == 0 && i < a.tq) p.delta[r] = delta;
  }
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  for (int t = 0; t < tiles; ++t) {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this tile's v
    __syncthreads();                      // ... of every wave; the last tile has been read
    land();
    lds_barrier();
    if (t + 1 < tiles) load(t + 1);
    const char *vt = sv + ((t & 1) ^ 1) * TILE_B;
    if (idle) continue;
#pragma unroll 1
    for (int x = 0; x < 2; ++x) {
      const int rx = fresh(row_base<DH>(li, g)) + 32 * x * DH * 2;
      // place 2 x + y of column tile d: (2 x + y) ^ d is (y ^ d) + 2 x, or less 2 x where y ^ d has that bit
      const int up = fresh(cb) + 64 * x, down = up - 128 * x;
      auto column = [&](int n) __attribute__((always_inline)) { return column_frag(st, (n / ND ^ n % ND) & 2 ? down : up, n % ND, n / ND); };
      f32x16 s, dp;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = -lse;
        dp[e] = -delta;
      }
      bf16x8 f[3][2], cf[3];            // operands, read two steps ahead
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        f[k][0] = row_frag<DH>(sk, rx, 0, k);
        f[k][1] = row_frag<DH>(vt, rx, 0, k);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        if (k + 2 < NC) {
          f[(k + 2) % 3][0] = row_frag<DH>(sk, rx, 0, k + 2);
          f[(k + 2) % 3][1] = row_frag<DH>(vt, rx, 0, k + 2);
        } else {
          cf[k + 2 - NC] = column(k + 2 - NC);
        }
        s = mma32(f[k % 3][0], qf[k], s);
        dp = mma32(f[k % 3][1], df[k], dp);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) dp[e] *= __builtin_amdgcn_exp2f(s[e] * p.qscale);
      if ((t + 1) * QT > len) {        // keys past the end: exp(-lse) may be anything, and infinity times their zeros a NaN
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (t * QT + 32 * x + 8 * (e >> 2) + 4 * g + (e & 3) >= len) dp[e] = 0.f;
      }
      const bf16x8 df2[2] = {chunk_frag(dp, 0), chunk_frag(dp, 1)};
      bf16x8 dr2[2];
      if constexpr (TWO) {
        dr2[0] = chunk_rest(dp, 0, df2[0]);
        dr2[1] = chunk_rest(dp, 1, df2[1]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int y = 0; y < 2 * ND; ++y) {
        if (y + 2 < 2 * ND) cf[(y + 2) % 3] = column(y + 2);
        o[y % ND] = mma32(cf[y % 3], df2[y / ND], o[y % ND]);
        if constexpr (TWO) o[y % ND] = mma32(cf[y % 3], dr2[y / ND], o[y % ND]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  __syncthreads();            // the last tile has been read
  if (idle) return;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<bf16x4 *>(mine + row_at<DH>(li, 4 * d + e) + 8 * g) =
          bf16x4{(bf16)(o[d][4 * e] * p.scale), (bf16)(o[d][4 * e + 1] * p.scale), (bf16)(o[d][4 * e + 2] * p.scale), (bf16)(o[d][4 * e + 3] * p.scale)};
  own_lds();
  bf16 *O = (bf16 *)p.dq + b * a.q_bs + h * DH + 8 * lch;
#pragma unroll
  for (int x = 0; x < N; ++x) {
    const int row = q0 + RPI * x + lrow;
    const bf16x8 v = *reinterpret_cast<const bf16x8 *>(mine + row_at<DH>(RPI * x + lrow, lch));
    if (row < a.tq) store_frag(O + (int64_t)row * a.q_rs, v);
  }
}

constexpr int KEYS = 256;            // keys of a workgroup of k_dkv, 32 a wave

// Measured and not kept: 64 keys a wave on one wave a SIMD, half the LDS reads: 320 accumulators are more than the 256
// accumulation registers, and moving them took 860 us; operands read two steps ahead: they spill.
// dk and dv of 256 keys of a prompt's key head against a range of the (candidate, head, query tile) triples that read them.
// The tiles of q and dout reach LDS by loads that write it themselves, one tile ahead in two buffers; rows past tq are past
// the buffer's range and read as zero.
template <int DH, bool TWO>
__global__ __launch_bounds__(512) void k_dkv(CrossP p) {
  constexpr int NC = DH / 16, ND = DH / 32, RB = DH * 2, TILE_B = QT * RB, NCH = RB / 16, ROWS = 64 / NCH;
  extern __shared__ __attribute__((aligned(16))) char s_mem[];
  char *rows = s_mem, *tq = rows + 4 * TILE_B, *td = tq + DH * TP;      // [2][q, dout], then their transposed copies
  float *s_lse = reinterpret_cast<float *>(td + DH * TP), *s_delta = s_lse + 2 * QT;
  int *s_list = reinterpret_cast<int *>(s_delta + 2 * QT), *s_count = s_list + p.a.batch;
  const CrossArgs &a = p.a;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, g = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the key blocks of one range of queries follow each other on one XCD, whose L2 then holds its q and dout
  const int nkb = (a.tk + KEYS - 1) / KEYS, units = a.n_kv * a.kv_heads, rest = blockIdx.x >> 3;
  const int kb = rest % nkb, uu = rest / nkb * 8 + (blockIdx.x & 7);
  if (uu >= units * p.splits) return;
  const int c = uu % units / a.kv_heads, kh = uu % a.kv_heads, split = uu / units;
  const int len = keys_of(a, c), shared = a.heads / a.kv_heads;
  if (p.splits > 1 && kb * KEYS >= len) return;       // k_cross_sum writes those rows
  list_candidates(a, c, s_list, s_count);
  const int key0 = kb * KEYS + w * 32, key = key0 + li;
  const bf16 *K = (const bf16 *)a.k + c * a.kv_bs + (int64_t)min(key, a.tk - 1) * a.kv_rs + kh * DH;
  const bf16 *V = (const bf16 *)a.v + c * a.kv_bs + (int64_t)min(key, a.tk - 1) * a.kv_rs + kh * DH;
  bf16x8 kf[NC], vf[NC];
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    kf[k] = key < len ? load_frag(K + 16 * k + 8 * g) : zero_frag<bf16>();
    vf[k] = key < len ? load_frag(V + 16 * k + 8 * g) : zero_frag<bf16>();
  }
  f32x16 dk[ND], dv[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) dk[d][e] = dv[d][e] = 0.f;
  const int nqt = (a.tq + QT - 1) / QT;
  const int64_t all = kb * KEYS < len ? (int64_t)*s_count * shared * nqt : 0;
  const int64_t u0 = all * split / p.splits, u1 = all * (split + 1) / p.splits;
  constexpr int COPIES = 2 * 16 * (DH / 4) / 512;
  const int cb = column_base(li, g), which = COPIES == 2 ? 0 : tid / 256, dg = tid % (DH / 4), qg = tid / (DH / 4) % 16;
  const int q_rs = (int)a.q_rs, o_rs = (int)a.o_rs;
  int qt = (int)(u0 % nqt), hs = (int)(u0 / nqt % shared), bi = (int)(u0 / nqt / shared);   // the triple to load next
  float ls = 0.f, de = 0.f;
  int left = 0;             // queries of the tile loaded last
  auto load = [&](int buf) __attribute__((always_inline)) {
    const int h = kh * shared + hs, b = __builtin_amdgcn_readfirstlane(s_list[bi]), valid = min(QT, a.tq - qt * QT);
    left = valid;
    const __amdgpu_buffer_rsrc_t rq = rows_rsrc((const bf16 *)a.q + b * a.q_bs + (int64_t)qt * QT * a.q_rs + h * DH, q_rs, valid, DH);
    const __amdgpu_buffer_rsrc_t rd = rows_rsrc((const bf16 *)p.dout + b * a.o_bs + (int64_t)qt * QT * a.o_rs + h * DH, o_rs, valid, DH);
    const int at = fresh(lane);       // offsets are made anew for each tile: spilled ones would come back behind the loads
#pragma unroll
    for (int x = 0; x < QT / ROWS / 8; ++x) {       // a load fills ROWS rows, 64 chunks; each wave takes its share of them
      const int first = (w * (QT / ROWS / 8) + x) * ROWS, row = first + at / NCH, ch = at % NCH ^ swz<DH>(row);
      char *to = rows + buf * 2 * TILE_B + first * RB;
      load_to_lds(rq, to, off(row, q_rs, 8 * ch, valid));
      load_to_lds(rd, to + TILE_B, off(row, o_rs, 8 * ch, valid));
    }
    if (tid < QT) {
      const bool ok = tid < valid;
      const int64_t r = ((int64_t)b * a.heads + h) * a.tq + (ok ? qt * QT + tid : 0);
      ls = ok ? a.lse[r] : INFINITY;       // as they are: to use them here would wait for the tile
      de = ok ? p.delta[r] : 0.f;
    }
    if (++qt == nqt) {       // the next triple
      qt = 0;
      if (++hs == shared) {
        hs = 0;
        ++bi;
      }
    }
  };
  const int steps = (int)(u1 - u0);
  if (steps) load(0);
  for (int u = 0; u < steps; ++u) {
    const int buf = u & 1;
    const char *rq = rows + buf * 2 * TILE_B, *rd = rq + TILE_B;
    if (tid < QT) {
      s_lse[buf * QT + tid] = ls == -INFINITY ? ls : -ls * LOG2E / p.qscale;
      s_delta[buf * QT + tid] = -de;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this tile's rows
    __syncthreads();                      // ... of every wave; the last tile's copies have been read
    if (left < QT) {          // the last query again in place of rows of zeros, which would meet an infinite key with a NaN
      char *q = rows + buf * 2 * TILE_B;
      for (int e = left * NCH + tid; e < QT * NCH; e += 512)
        *reinterpret_cast<u32x4 *>(q + row_at<DH>(e / NCH, e % NCH)) = *reinterpret_cast<const u32x4 *>(q + row_at<DH>(left - 1, e % NCH));
      lds_barrier();
    }
    if (u + 1 < steps) load(buf ^ 1);
    {
      const int br = fresh(block_rows<DH>(dg, qg)), bc = fresh(block_columns(dg, qg));
#pragma unroll
      for (int x = 0; x < COPIES; ++x) {       // head dim 128: a block of each tile a thread; 64: of one of them
        const bool second = COPIES == 2 ? x : which;
        u32x2 r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = *reinterpret_cast<const u32x2 *>((second ? rd : rq) + block_row<DH>(br, e));
        store_columns((second ? td : tq) + bc, r);
      }
    }
    lds_barrier();
    if (key0 >= len) continue;
    const int rb = row_base<DH>(li, g);
#pragma unroll 1
    for (int x = 0; x < 2; ++x) {
      const int rx = fresh(rb) + buf * 2 * TILE_B + 32 * x * RB;
      // place 2 x + y of column tile d: (2 x + y) ^ d is (y ^ d) + 2 x, or less 2 x where y ^ d has that bit
      const int up = fresh(cb) + 64 * x, down = up - 128 * x;
      auto column = [&](const char *t, int d, int y) __attribute__((always_inline)) { return column_frag(t, (y ^ d) & 2 ? down : up, d, y); };
      f32x16 s, dp;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const f32x4 l4 = *reinterpret_cast<const f32x4 *>(s_lse + buf * QT + 32 * x + 8 * e + 4 * g);
        const f32x4 d4 = *reinterpret_cast<const f32x4 *>(s_delta + buf * QT + 32 * x + 8 * e + 4 * g);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          s[4 * e + k] = l4[k];
          dp[4 * e + k] = d4[k];
        }
      }
      bf16x8 f[2][2], cf[2];       // operands, read a step ahead
      f[0][0] = row_frag<DH>(rows, rx, 0, 0);
      f[0][1] = row_frag<DH>(rows + TILE_B, rx, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < NC; ++k) {
        if (k + 1 < NC) {
          f[(k + 1) & 1][0] = row_frag<DH>(rows, rx, 0, k + 1);
          f[(k + 1) & 1][1] = row_frag<DH>(rows + TILE_B, rx, 0, k + 1);
        } else {
          cf[0] = column(td, 0, 0);
          cf[1] = column(tq, 0, 0);
        }
        s = mma32(f[k & 1][0], kf[k], s);
        dp = mma32(f[k & 1][1], vf[k], dp);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = __builtin_amdgcn_exp2f(s[e] * p.qscale);
        dp[e] *= s[e];
      }
      const bf16x8 pf[2] = {chunk_frag(s, 0), chunk_frag(s, 1)}, sf[2] = {chunk_frag(dp, 0), chunk_frag(dp, 1)};
      bf16x8 pr[2], sr[2];
      if constexpr (TWO)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          pr[y] = chunk_rest(s, y, pf[y]);
          sr[y] = chunk_rest(dp, y, sf[y]);
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int y = 0; y < 2 * ND; ++y) {
        const bf16x8 c0 = cf[0], c1 = cf[1];
        if (y + 1 < 2 * ND) {
          cf[0] = column(td, (y + 1) % ND, (y + 1) / ND);
          cf[1] = column(tq, (y + 1) % ND, (y + 1) / ND);
        }
        dv[y % ND] = mma32(c0, pf[y / ND], dv[y % ND]);
        dk[y % ND] = mma32(c1, sf[y / ND], dk[y % ND]);
        if constexpr (TWO) {
          dv[y % ND] = mma32(c0, pr[y / ND], dv[y % ND]);
          dk[y % ND] = mma32(c1, sr[y / ND], dk[y % ND]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  if (key >= a.tk || (p.splits > 1 && key >= len)) return;
  const bool live = key < len;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int at = 32 * d + 8 * e + 4 * g;
      f32x4 x, y;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        x[k] = live && len > 1 ? dk[d][4 * e + k] * p.scale : 0.f;
        y[k] = live ? dv[d][4 * e + k] : 0.f;
      }
      if (p.splits > 1) {       // [split][prompt][tk][key head][2][dh]
        float *dst = p.part + (((((int64_t)split * a.n_kv + c) * a.tk + key) * a.kv_heads + kh) * 2) * DH + at;
        *reinterpret_cast<f32x4 *>(dst) = x;
        *reinterpret_cast<f32x4 *>(dst + DH) = y;
      } else {
        const int64_t to = c * a.kv_bs + (int64_t)key * a.kv_rs + kh * DH + at;
        *reinterpret_cast<bf16x4 *>((bf16 *)p.dk + to) = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
        *reinterpret_cast<bf16x4 *>((bf16 *)p.dv + to) = bf16x4{(bf16)y[0], (bf16)y[1], (bf16)y[2], (bf16)y[3]};
      }
    }
}

// P and dS go in two parts where that costs next to nothing: few keys, or few queries, which are bound by the reading of the
// other side.
bool two_parts(const CrossArgs &a) { return a.tk <= QT || a.tq <= QT; }
template <int DH> constexpr size_t dq_lds() { return (size_t)3 * QT * DH * 2 + DH * TP; }
template <int DH> constexpr size_t dkv_lds() { return (size_t)4 * QT * DH * 2 + 2 * DH * TP + 4 * QT * 4; }
// Offsets of a tile's rows are 31 bits.
bool takes(const CrossArgs &a) { return (a.head_dim == 64 || a.head_dim == 128) && a.q_rs < 1 << 23 && a.o_rs < 1 << 23 && a.kv_rs < 1 << 23; }

}  // namespace x32

// dk and dv out of the ranges' sums, in order, four elements a thread; rows past a prompt's end: 0
template <typename T>
__global__ __launch_bounds__(256) void k_cross_sum(CrossP p) {
  const CrossArgs &a = p.a;
  const int64_t row = (int64_t)a.kv_heads * 2 * a.head_dim, total = (int64_t)a.n_kv * a.tk * row;
  for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e < total; e += (int64_t)gridDim.x * 1024) {
    const int c = (int)(e / (a.tk * row)), i = (int)(e / row % a.tk), x = (int)(e % row);
    const int kh = x / (2 * a.head_dim), which = x / a.head_dim & 1, d = x % a.head_dim;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (i < keys_of(a, c))
#pragma unroll 8
      for (int k = 0; k < p.splits; ++k) s += *reinterpret_cast<const f32x4 *>(p.part + k * total + e);
    T *dst = (T *)(which ? p.dv : p.dk) + c * a.kv_bs + (int64_t)i * a.kv_rs + kh * a.head_dim + d;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4 *>(dst) = s;
    else *reinterpret_cast<bf16x4 *>(dst) = bf16x4{(bf16)s[0], (bf16)s[1], (bf16)s[2], (bf16)s[3]};
  }
}

template <typename T, int DH> constexpr size_t tile_bytes() { return (size_t)2 * TILE<T> * (DH * sizeof(T) + 16); }

CrossP params(const CrossArgs &a) {
  CrossP p{};
  p.a = a;
  p.splits = 1;
  p.qscale = (float)(1.4426950408889634 / sqrt((double)a.head_dim));
  p.scale = (float)(1.0 / sqrt((double)a.head_dim));
  return p;
}
unsigned unit_grid(const CrossP &p) { return (unsigned)(((int64_t)p.a.batch * p.a.heads + 7) / 8 * 8 * p.nqb); }

// queries of a wave: 32 where a candidate has more than a workgroup of 16s
template <typename T> int wave_queries(const CrossArgs &a) { return sizeof(T) == 2 && a.tq > 64 ? 32 : 16; }

// Into how many ranges the keys are cut: two workgroups a CU out of one candidate's (so that its bits do not depend on the
// pool), four tiles of keys each at least, and none for more than 64 queries, which fill the card by themselves.
template <typename T> int key_splits(const CrossArgs &a) {
  const int64_t wgs = (int64_t)a.heads * ((a.tq + 4 * wave_queries<T>(a) - 1) / (4 * wave_queries<T>(a)));
  const int64_t tiles = (a.tk + TILE<T> - 1) / TILE<T>;
  if (a.tq > 64) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(64, std::min(512 / wgs, tiles / 4)));
}

template <typename T> constexpr int BLOCK_KEYS = sizeof(T) == 2 ? 128 : 64;

// Into how many ranges the queries of k_cross_dkv and k_dkv are cut, for the least estimate of whole rounds of workgroups
// (one a CU) at 2 us a tile of queries, and of the ranges' sums, written and read at 5 bytes a ps; a tile each at least.
// By the sizes alone, not by the kernel that takes the strides, since the workspace goes by it.
template <typename T> int query_splits(const CrossArgs &a) {
  const int keys = sizeof(T) == 2 && a.head_dim >= 64 ? x32::KEYS : BLOCK_KEYS<T>;
  const int64_t wgs = (int64_t)a.n_kv * a.kv_heads * ((a.tk + keys - 1) / keys);
  const double tiles = (double)a.batch * (a.heads / a.kv_heads) * ((a.tq + TILE<T> - 1) / TILE<T>) / a.n_kv;
  const double bytes = 16.0 * a.n_kv * a.tk * a.kv_heads * a.head_dim;
  int best = 1;
  double least = 0;
  for (int s = 1; s <= 64 && (s == 1 || tiles >= s); ++s) {
    const double cost = (double)((wgs * s + 255) / 256) * tiles / s * 2.0 + (s > 1 ? s * bytes / 5e6 + 4 : 0);
    if (s == 1 || cost < least) {
      best = s;
      least = cost;
    }
  }
  return best;
}

template <typename T, int DH, int NQ>
hipError_t forward(CrossP p, void *workspace, size_t bytes, hipStream_t s) {
  p.nqb = (p.a.tq + 64 * NQ - 1) / (64 * NQ);
  if constexpr (NQ == 1) {        // 32 queries a wave are more than key_splits cuts
    const int splits = key_splits<T>(p.a);
    if (splits > 1 && workspace && bytes >= cross_attention_workspace(sizeof(T) == 2 ? ACT_BF16 : ACT_F32, p.a)) {
      p.splits = splits;
      p.part = (float *)workspace;
      hipLaunchKernelGGL((k_cross<T, DH, NQ, true>), dim3(unit_grid(p), splits), dim3(256), (tile_bytes<T, DH>()), s, p);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      const int64_t rows = (int64_t)p.a.batch * p.a.heads * p.a.tq;
      hipLaunchKernelGGL((k_cross_join<T>), dim3((unsigned)std::min<int64_t>((rows + 3) / 4, 1 << 16)), dim3(256), 0, s, p);
      return hipGetLastError();
    }
  }
  if (NQ == 2 && attention_own_takes(p.a)) return launch_attention_own(p.a, s);
  hipLaunchKernelGGL((k_cross<T, DH, NQ, false>), dim3(unit_grid(p)), dim3(256), (tile_bytes<T, DH>()), s, p);
  return hipGetLastError();
}

template <typename T, int DH>
hipError_t forward_by_queries(const CrossP &p, void *workspace, size_t bytes, hipStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (wave_queries<T>(p.a) == 32) return forward<T, DH, 2>(p, workspace, bytes, s);
  return forward<T, DH, 1>(p, workspace, bytes, s);
}

template <typename T, int DH>
hipError_t gradient(CrossP p, const CrossGradArgs &b, hipStream_t s) {
  const CrossArgs &a = p.a;
  p.dout = b.dout;
  p.dq = b.dq; p.dk = b.dk; p.dv = b.dv;
  p.delta = (float *)b.workspace;
  const int64_t rows = (int64_t)a.batch * a.heads * a.tq;
  p.part = p.delta + (rows + 63) / 64 * 64;
  hipError_t e = hipSuccess;
  constexpr size_t lds = tile_bytes<T, DH>();
  const bool wide = sizeof(T) == 2 && x32::takes(a);
  if (!b.dq) {
    hipLaunchKernelGGL((k_cross_delta<T>), dim3((unsigned)std::min<int64_t>((rows * (a.head_dim / 8) + 255) / 256, 1 << 16)), dim3(256), 0, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (b.dq) {
    if constexpr (sizeof(T) == 2 && DH >= 64) {
      if (wide) {
        p.nqb = (a.tq + 127) / 128;
        auto kern = x32::two_parts(a) ? x32::k_dq<DH, true> : x32::k_dq<DH, false>;
        if ((e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)x32::dq_lds<DH>())) != hipSuccess) return e;
        hipLaunchKernelGGL(kern, dim3(unit_grid(p)), dim3(256), (x32::dq_lds<DH>()), s, p);
      }
    }
    if (!wide) {
      constexpr int NQ = sizeof(T) == 2 ? 2 : 1;
      p.nqb = (a.tq + 64 * NQ - 1) / (64 * NQ);
      hipLaunchKernelGGL((k_cross_dq<T, DH, NQ>), dim3(unit_grid(p)), dim3(256), lds, s, p);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (b.dk) {
    p.splits = query_splits<T>(a);
    if constexpr (sizeof(T) == 2 && DH >= 64) {
      if (wide) {
        const int64_t sets = ((int64_t)a.n_kv * a.kv_heads * p.splits + 7) / 8 * 8 * ((a.tk + x32::KEYS - 1) / x32::KEYS);
        const size_t bytes = x32::dkv_lds<DH>() + (a.batch + 1) * 4;
        auto kern = x32::two_parts(a) ? x32::k_dkv<DH, true> : x32::k_dkv<DH, false>;
        // the most that any call asks for: the attribute is the process's, and calls of other batches may run beside this one
        constexpr int most = (int)x32::dkv_lds<DH>() + (CROSS_GRAD_BATCH + 1) * 4;
        if ((e = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, most)) != hipSuccess) return e;
        hipLaunchKernelGGL(kern, dim3((unsigned)sets), dim3(512), bytes, s, p);
      }
    }
    if (!wide) {
      constexpr int NK = BLOCK_KEYS<T> / 64;
      const size_t more = (2 * TILE<T> + a.batch + 1) * 4;
      hipLaunchKernelGGL((k_cross_dkv<T, DH, NK>), dim3((a.tk + BLOCK_KEYS<T> - 1) / BLOCK_KEYS<T>, a.n_kv * a.kv_heads, p.splits),
                         dim3(256), lds + more, s, p);
    }
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (p.splits > 1) {
      const int64_t fours = (int64_t)a.n_kv * a.tk * a.kv_heads * a.head_dim / 2;
      hipLaunchKernelGGL((k_cross_sum<T>), dim3((unsigned)std::min<int64_t>((fours + 255) / 256, 1 << 16)), dim3(256), 0, s, p);
      e = hipGetLastError();
    }
  }
  return e;
}

template <typename T>
size_t grad_bytes(const CrossArgs &a) {
  const int64_t rows = ((int64_t)a.batch * a.heads * a.tq + 63) / 64 * 64;
  const int splits = query_splits<T>(a);
  return (size_t)(rows + (splits > 1 ? (int64_t)splits * a.n_kv * a.tk * a.kv_heads * 2 * a.head_dim : 0)) * 4;
}

}  // namespace

size_t cross_attention_workspace(ActType t, const CrossArgs &a) {
  const int splits = t == ACT_BF16 ? key_splits<bf16>(a) : key_splits<float>(a);
  return splits > 1 ? (size_t)a.batch * a.heads * a.tq * splits * (a.head_dim + 4) * 4 : 0;
}

hipError_t launch_cross_attention(ActType t, const CrossArgs &a, void *workspace, size_t bytes, hipStream_t s) {
  const CrossP p = params(a);
  if (t == ACT_BF16)
    return a.head_dim <= 32 ? forward_by_queries<bf16, 32>(p, workspace, bytes, s)
           : a.head_dim == 64 ? forward_by_queries<bf16, 64>(p, workspace, bytes, s) : forward_by_queries<bf16, 128>(p, workspace, bytes, s);
  return a.head_dim <= 32 ? forward_by_queries<float, 32>(p, workspace, bytes, s)
         : a.head_dim == 64 ? forward_by_queries<float, 64>(p, workspace, bytes, s) : forward_by_queries<float, 128>(p, workspace, bytes, s);
}

size_t cross_attention_grad_workspace(ActType t, const CrossArgs &a) {
  return t == ACT_BF16 ? grad_bytes<bf16>(a) : grad_bytes<float>(a);
}

hipError_t launch_cross_attention_grad(ActType t, const CrossArgs &a, const CrossGradArgs &b, hipStream_t s) {
  const CrossP p = params(a);
  if (t == ACT_BF16)
    return a.head_dim <= 32 ? gradient<bf16, 32>(p, b, s) : a.head_dim == 64 ? gradient<bf16, 64>(p, b, s) : gradient<bf16, 128>(p, b, s);
  return a.head_dim <= 32 ? gradient<float, 32>(p, b, s) : a.head_dim == 64 ? gradient<float, 64>(p, b, s) : gradient<float, 128>(p, b, s);
}

}  // namespace fb
