// Linear layers on 8-bit integers: C[m][n] = a_scale[m] w_scale[n] sum_k A[m][k] W[n][k] with the epilogues of the other
// linear layers.  The sum is exact in 32 bits (K <= 65536: at most 2^14 2^16 = 2^30), so every tiling and every order of
// K gives the same bits, and the choice of kernel changes no output.
#include "common.h"
#include "kernels.h"

namespace fb {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(1)));

// (acc w_scale) a_scale + bias: the roundings of every kernel here.
__device__ __forceinline__ float scaled(int acc, float ws, float as, float bias) { return fmaf((float)acc * ws, as, bias); }

// One output from its scaled value.
template <int EPI, typename TO>
__device__ __forceinline__ void put(const EpiArgs &e, int64_t at, int n, float v) {
  if constexpr (EPI == EPI_STORE || EPI == EPI_GELU) {
    ((TO *)e.out)[at] = from_f32<TO>(EPI == EPI_GELU ? gelu_tanh(v) : v);
  } else if constexpr (EPI == EPI_STORE_F32) {
    ((float *)e.out)[at] = v;
  } else {
    const float h = (e.res_in ? e.res_in : (const float *)e.out)[at];
    const float r = e.gate ? fmaf(e.gate[n], v, h) : h + v;
    ((float *)e.out)[at] = r;
    if (e.cache) e.cache[at] = r;
  }
}

}  // namespace

// ------------------------------------------------------------------------------ any size and alignment
// 64x64 tiles, four waves of 32x32, K tiles of 128 through registers into LDS.
namespace any8 {
constexpr int BM = 64, BN = 64, BK = 128;
// 16-byte chunk c of row r at c ^ swz(r): the 16 lanes that read one chunk of 16 rows at once meet 16 places
__device__ __forceinline__ int swz(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int at(int r, int c) { return r * BK + ((c ^ swz(r)) << 4); }
// bytes k .. k + 15 of a row of K, zero past its end
__device__ __forceinline__ u32x4 chunk(const int8_t *p, int k, int K) {
  if (k + 16 <= K) return *reinterpret_cast<const u32x4u *>(p + k);
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (k + i < K) v[i >> 2] |= (uint32_t)(uint8_t)p[k + i] << (8 * (i & 3));
  return v;
}
}  // namespace any8

template <int EPI, typename TO>
__global__ __launch_bounds__(256) void k_linear_i8_any(int M, int N, int K, I8Args g, EpiArgs e, int NT) {
  using namespace any8;
  __shared__ __attribute__((aligned(16))) char lds[2][(BM + BN) * BK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, fr = lane & 15, fq = lane >> 4;
  const int mt = blockIdx.x / NT, m0 = mt * BM, n0 = (blockIdx.x - mt * NT) * BN;
  const int wm = 32 * (wave >> 1), wn = 32 * (wave & 1);
  const int lr = tid >> 3, lc = tid & 7;
  // rows past the end: the last one again, never stored
  const int8_t *ar[2], *wr[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    ar[i] = g.A + (int64_t)min(m0 + lr + 32 * i, M - 1) * K;
    wr[i] = g.W + (int64_t)min(n0 + lr + 32 * i, N - 1) * K;
  }
  u32x4 ra[2], rw[2];
  auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ra[i] = chunk(ar[i], k0 + 16 * lc, K);
      rw[i] = chunk(wr[i], k0 + 16 * lc, K);
    }
  };
  auto store = [&](char *s) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      *reinterpret_cast<u32x4 *>(s + at(lr + 32 * i, lc)) = ra[i];
      *reinterpret_cast<u32x4 *>(s + BM * BK + at(lr + 32 * i, lc)) = rw[i];
    }
  };
  i32x4 acc[2][2] = {};
  const int KT = (K + BK - 1) / BK;
  load(0);
  store(lds[0]);
  __syncthreads();
  for (int kt = 0; kt < KT; ++kt) {
    const char *s = lds[kt & 1];
    if (kt + 1 < KT) load((kt + 1) * BK);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      i32x4 fa[2], fw[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = *reinterpret_cast<const i32x4 *>(s + at(wm + 16 * i + fr, 4 * ks + fq));
        fw[i] = *reinterpret_cast<const i32x4 *>(s + BM * BK + at(wn + 16 * i + fr, 4 * ks + fq));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[i], fa[j], acc[i][j], 0, 0, 0);
    }
    if (kt + 1 < KT) store(lds[(kt + 1) & 1]);
    __syncthreads();
  }
  // lane: columns 4 fq .. + 3 of row fr
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int m = m0 + wm + 16 * j + fr;
    if (m >= M) continue;
    const float as = g.a_scale[m];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + wn + 16 * i + 4 * fq + q;
        if (n < N) put<EPI, TO>(e, (int64_t)m * e.ldo + n, n, scaled(acc[i][j][q], g.w_scale[n], as, e.bias ? e.bias[n] : 0.f));
      }
  }
}

// ------------------------------------------------------------------------------------------- dispatch
namespace {

constexpr int kRowsPerLaunch = 1 << 15;   // any8's grid within 2^32 threads at N <= 2^20

template <int EPI, typename TO>
hipError_t launch_any(int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s) {
  const int NT = (N + any8::BN - 1) / any8::BN, MT = (M + any8::BM - 1) / any8::BM;
  hipLaunchKernelGGL((k_linear_i8_any<EPI, TO>), dim3(MT * NT), dim3(256), 0, s, M, N, K, g, e, NT);
  return hipGetLastError();
}

template <int EPI, typename TO>
hipError_t launch_epi(int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s) {
  for (int64_t m = 0; m < M; m += kRowsPerLaunch) {
    I8Args p = g;
    p.A += m * K;
    p.a_scale += m;
    EpiArgs r = e;
    const size_t es = EPI == EPI_STORE || EPI == EPI_GELU ? sizeof(TO) : sizeof(float);
    r.out = (char *)e.out + (size_t)m * e.ldo * es;
    if (r.res_in) r.res_in += m * e.ldo;
    if (r.cache) r.cache += m * e.ldo;
    const hipError_t err = launch_any<EPI, TO>((int)(M - m < kRowsPerLaunch ? M - m : kRowsPerLaunch), N, K, p, r, s);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_linear_i8(ActType t, int epi, int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s) {
  const bool bf = t == ACT_BF16;
  switch (epi) {
    case EPI_STORE: return bf ? launch_epi<EPI_STORE, bf16>(M, N, K, g, e, s) : launch_epi<EPI_STORE_F32, float>(M, N, K, g, e, s);
    case EPI_GELU: return bf ? launch_epi<EPI_GELU, bf16>(M, N, K, g, e, s) : launch_epi<EPI_GELU, float>(M, N, K, g, e, s);
    case EPI_STORE_F32: return launch_epi<EPI_STORE_F32, float>(M, N, K, g, e, s);
    case EPI_RESIDUAL: return launch_epi<EPI_RESIDUAL, float>(M, N, K, g, e, s);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace fb
