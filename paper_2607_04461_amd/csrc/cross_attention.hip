// Cross-attention to prompts of their own lengths, and its gradient.  Candidate b attends with its tq queries to the first
// len keys of its prompt; query heads may share a key head.  With scores S = q k^T / sqrt(dh):
//   P = exp(S - lse),  out = P v,  lse = log sum exp S;   an empty prompt: out = 0, lse = -inf
//   delta = sum_d dout out,  dS = P (dout v^T - delta) / sqrt(dh),  dq = dS k,  dk = dS^T q,  dv = P^T dout
// dk and dv are summed over the prompt's candidates and the heads that share the key head, in their order; no atomics.
//
// All kernels keep one side in registers and take the other in tiles through LDS, and form the scores so that a lane's
// values belong to one row of the side it keeps: the 16 x 16 products of two tiles then are the right operand of the next
// product as they stand, with its k in the order 4 g + 0..3, 16 + 4 g + 0..3, which the left operand's transposing LDS
// reads follow.  P and dS are rounded to the operands' type for that product (bf16: 8 bits, as the values they meet).
//   * k_cross: a wave keeps 16 or 32 queries.  One pass over the keys with the running maximum and sum.
//   * k_cross_dq: the same with dout and lse: two products give P and dP, the third dq.
//   * k_cross_dkv: a wave keeps keys and values; the queries and dout of all candidates of the prompt pass by.
// Bound by the matrix cores for many queries, by the reading of k and v for few: then ranges of keys go to several
// workgroups and k_cross_join joins them.
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

template <typename T> constexpr int TILE = sizeof(T) == 2 ? 64 : 32;    // rows of a tile in LDS

template <typename T, int DH, int NQ, bool SPLIT>
__global__ __launch_bounds__(256) void k_cross(CrossP p) {
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
  float top[NQ], sum[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    top[n] = -INFINITY;
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
      const float off = m == -INFINITY ? 0.f : m * p.qscale;     // a row of -inf only: all of it 0
      const float shrink = __builtin_amdgcn_exp2f(fmaf(top[n], p.qscale, -off));
      top[n] = m;
      sum[n] *= shrink;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][d][e] *= shrink;
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][j][e] = __builtin_amdgcn_exp2f(fmaf(s[n][j][e], p.qscale, -off));
          sum[n] += s[n][j][e];
        }
    }
#pragma unroll
    for (int j = 0; j < NS; j += 2) {
      Frag<T> pf[NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) pf[n] = pair_frag<T>(s[n][j], s[n][j + 1]);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const Frag<T> vf = load_column_frag(sv, St::PITCH, 16 * d, 16 * j + 4 * g, 16 * j + 16 + 4 * g);
#pragma unroll
        for (int n = 0; n < NQ; ++n) o[n][d] = mma(vf, pf[n], o[n][d]);
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
      // [row][split][dh + 2]: the sums as they stand, the maximum (base 2) and the sum
      float *dst = p.part + ((((int64_t)b * a.heads + h) * a.tq + i) * p.splits + blockIdx.y) * (a.head_dim + 4);
#pragma unroll
      for (int d = 0; d < ND; ++d)
        if (16 * d + 4 * g < a.head_dim) *reinterpret_cast<f32x4 *>(dst + 16 * d + 4 * g) = o[n][d];
      if (g == 0) {
        dst[a.head_dim] = top[n] * p.qscale;
        dst[a.head_dim + 1] = l;
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
        a.lse[((int64_t)b * a.heads + h) * a.tq + i] = l == 0.f ? -INFINITY : (top[n] * p.qscale + log2f(l)) * LN2;
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
    float top = -INFINITY;
    for (int s = 0; s < p.splits; ++s)
      if (src[s * pitch + a.head_dim + 1] != 0.f) top = fmaxf(top, src[s * pitch + a.head_dim]);
    const float off = top == -INFINITY ? 0.f : top;
    float l = 0.f, o[2] = {0.f, 0.f};
    for (int s = 0; s < p.splits; ++s) {
      const float ls = src[s * pitch + a.head_dim + 1];
      if (ls == 0.f) continue;
      const float f = __builtin_amdgcn_exp2f(src[s * pitch + a.head_dim] - off);
      l = fmaf(f, ls, l);
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (lane + 64 * e < a.head_dim) o[e] = fmaf(f, src[s * pitch + lane + 64 * e], o[e]);
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    T *O = (T *)a.out + b * a.o_bs + (int64_t)i * a.o_rs + h * a.head_dim;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (lane + 64 * e < a.head_dim) O[lane + 64 * e] = from_f32<T>(o[e] * inv);
    if (a.lse && lane == 0) a.lse[r] = l == 0.f ? -INFINITY : (top + log2f(l)) * LN2;
  }
}

// delta[b][h][i] = sum_d dout out: head_dim / 8 lanes a row
template <typename T>
__global__ __launch_bounds__(256) void k_cross_delta(CrossP p) {
  const CrossArgs &a = p.a;
  const int lanes = a.head_dim / 8, at = threadIdx.x % lanes;
  const int64_t rows = (int64_t)a.batch * a.tq * a.heads, step = (int64_t)gridDim.x * 256 / lanes;
  // a wave's lanes leave the loop together: the exchange below needs all of a row's lanes, which share r
  for (int64_t r = ((int64_t)blockIdx.x * 256 + threadIdx.x) / lanes; r < rows; r += step) {
    const int h = (int)(r % a.heads), i = (int)(r / a.heads % a.tq), b = (int)(r / a.heads / a.tq);
    const int64_t from = b * a.o_bs + (int64_t)i * a.o_rs + h * a.head_dim + 8 * at;
    const Frag<T> x = load_frag((const T *)a.out + from), y = load_frag((const T *)p.dout + from);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(to_f32(x[e]), to_f32(y[e]), s);
    for (int o = lanes >> 1; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (at == 0) p.delta[((int64_t)b * a.heads + h) * a.tq + i] = s;
  }
}

template <typename T, int DH, int NQ>
__global__ __launch_bounds__(256) void k_cross_dq(CrossP p) {
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
  const int tiles = (len + KT - 1) / KT;
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
    delta[n] = p.delta[r];
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
      Frag<T> pf[NQ];
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
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const Frag<T> kf = load_column_frag(sk, St::PITCH, 16 * d, 16 * j + 4 * g, 16 * j + 16 + 4 * g);
#pragma unroll
        for (int n = 0; n < NQ; ++n) o[n][d] = mma(kf, pf[n], o[n][d]);
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

constexpr int MOST_BATCH = 4096;

// Keys [128 kb ...) of a prompt's key head against a range of the (candidate, head, query tile) triples that read them.
template <typename T, int DH, int NK>
__global__ __launch_bounds__(256, 1) void k_cross_dkv(CrossP p) {
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
  if (threadIdx.x < 64) {                           // the prompt's candidates
    int n = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
      const bool mine = b0 + lane < a.batch && prompt_of(a, b0 + lane) == c;
      const uint64_t votes = __ballot(mine);
      if (mine) s_list[n + __popcll(votes & ((1ull << lane) - 1))] = b0 + lane;
      n += __popcll(votes);
    }
    if (lane == 0) *s_count = n;
  }
  __syncthreads();
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
  auto load = [&](int64_t u) __attribute__((always_inline)) {
    const int qt = (int)(u % nqt), h = kh * shared + (int)(u / nqt % shared), b = s_list[u / nqt / shared];
    const int64_t i0 = (int64_t)qt * QT;
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
      Frag<T> pf[NK], sf[NK];
#pragma unroll
      for (int n = 0; n < NK; ++n) {
        pf[n] = pair_frag<T>(s[n][0], s[n][1]);
        sf[n] = pair_frag<T>(dp[n][0], dp[n][1]);
      }
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const Frag<T> qf = load_column_frag(sq, St::PITCH, 16 * d, 16 * j + 4 * g, 16 * j + 16 + 4 * g);
        const Frag<T> df = load_column_frag(sd, St::PITCH, 16 * d, 16 * j + 4 * g, 16 * j + 16 + 4 * g);
#pragma unroll
        for (int n = 0; n < NK; ++n) {
          dk[n][d] = mma(qf, sf[n], dk[n][d]);
          dv[n][d] = mma(df, pf[n], dv[n][d]);
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
        x[e] = i < len ? x[e] * p.scale : 0.f;      // rows past the prompt's end
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

// Into how many ranges the keys are cut: a workgroup a CU out of one candidate's (so that its bits do not depend on the
// pool), four tiles of keys each at least.
template <typename T> int key_splits(const CrossArgs &a) {
  const int64_t wgs = (int64_t)a.heads * ((a.tq + 4 * wave_queries<T>(a) - 1) / (4 * wave_queries<T>(a)));
  const int64_t tiles = (a.tk + TILE<T> - 1) / TILE<T>;
  return (int)std::max<int64_t>(1, std::min(256 / wgs, tiles / 4));
}

// Into how many ranges the queries of k_cross_dkv are cut: four workgroups a CU, four tiles of queries each at least
template <typename T> int query_splits(const CrossArgs &a, int keys) {
  const int64_t wgs = (int64_t)a.n_kv * a.kv_heads * ((a.tk + keys - 1) / keys);
  const int64_t tiles = (int64_t)a.batch * (a.heads / a.kv_heads) * ((a.tq + TILE<T> - 1) / TILE<T>) / a.n_kv;
  return (int)std::max<int64_t>(1, std::min<int64_t>((1024 + wgs - 1) / wgs, tiles / 4));
}
template <typename T> constexpr int BLOCK_KEYS = sizeof(T) == 2 ? 128 : 64;

template <typename T, int DH, int NQ>
hipError_t forward(CrossP p, void *workspace, size_t bytes, hipStream_t s) {
  p.nqb = (p.a.tq + 64 * NQ - 1) / (64 * NQ);
  const int splits = key_splits<T>(p.a);
  if (splits > 1 && workspace && bytes >= cross_attention_workspace(sizeof(T) == 2 ? ACT_BF16 : ACT_F32, p.a)) {
    p.splits = splits;
    p.part = (float *)workspace;
    hipLaunchKernelGGL((k_cross<T, DH, NQ, true>), dim3(unit_grid(p), splits), dim3(256), (tile_bytes<T, DH>()), s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t rows = (int64_t)p.a.batch * p.a.heads * p.a.tq;
    hipLaunchKernelGGL((k_cross_join<T>), dim3((unsigned)std::min<int64_t>((rows + 3) / 4, 1 << 16)), dim3(256), 0, s, p);
  } else {
    hipLaunchKernelGGL((k_cross<T, DH, NQ, false>), dim3(unit_grid(p)), dim3(256), (tile_bytes<T, DH>()), s, p);
  }
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
  hipLaunchKernelGGL((k_cross_delta<T>), dim3((unsigned)std::min<int64_t>((rows * (a.head_dim / 8) + 255) / 256, 1 << 16)), dim3(256), 0,
                     s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  constexpr size_t lds = tile_bytes<T, DH>();
  if (b.dq) {
    constexpr int NQ = sizeof(T) == 2 ? 2 : 1;
    p.nqb = (a.tq + 64 * NQ - 1) / (64 * NQ);
    hipLaunchKernelGGL((k_cross_dq<T, DH, NQ>), dim3(unit_grid(p)), dim3(256), lds, s, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (b.dk) {
    constexpr int NK = BLOCK_KEYS<T> / 64;
    p.splits = query_splits<T>(a, BLOCK_KEYS<T>);
    const size_t more = (2 * TILE<T> + a.batch + 1) * 4;
    hipLaunchKernelGGL((k_cross_dkv<T, DH, NK>), dim3((a.tk + BLOCK_KEYS<T> - 1) / BLOCK_KEYS<T>, a.n_kv * a.kv_heads, p.splits),
                       dim3(256), lds + more, s, p);
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
  const int splits = query_splits<T>(a, BLOCK_KEYS<T>);
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
