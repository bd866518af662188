// Linear layers on 8-bit integers: C[m][n] = a_scale[m] w_scale[n] sum_k A[m][k] W[n][k] with the epilogues of the other
// linear layers.  The sum is exact in 32 bits (K <= 65536: at most 2^14 2^16 = 2^30), so every tiling and every order of
// K gives the same bits, and the choice of kernel changes no output.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace fb {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(1)));

// (acc w_scale) a_scale + bias: the roundings of every kernel here.
__device__ __forceinline__ float scaled(int acc, float ws, float as, float bias) { return fmaf((float)acc * ws, as, bias); }

// One output from its scaled value (RESIDUAL: and its column's gate and what it is added to).
template <int EPI, typename TO>
__device__ __forceinline__ void put(const EpiArgs &e, int64_t at, float v, float gate, float h) {
  if constexpr (EPI == EPI_STORE || EPI == EPI_GELU) {
    ((TO *)e.out)[at] = from_f32<TO>(EPI == EPI_GELU ? gelu_tanh(v) : v);
  } else if constexpr (EPI == EPI_STORE_F32) {
    ((float *)e.out)[at] = v;
  } else {
    const float r = fmaf(gate, v, h);   // a gate of one adds v
    ((float *)e.out)[at] = r;
    if (e.cache) e.cache[at] = r;
  }
}

// The workgroup's barrier for LDS accesses of the waves, not for loads that are still on their way (__syncthreads waits for
// those too).
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// 16 bytes on any address.  BYTES: where it may be off 4 bytes, which a load pays for with three to five times its time
// (20 x 24 x 11073 28 us, x 11076 8.8): from the five words around them, each of which holds one of the bytes at least.
template <bool BYTES = false> __device__ __forceinline__ i32x4 whole_piece(const int8_t *p) {
  if constexpr (!BYTES) return __builtin_bit_cast(i32x4, *reinterpret_cast<const u32x4u *>(p));
  typedef uint32_t words __attribute__((ext_vector_type(4), aligned(4)));
  const uintptr_t at = (uintptr_t)p;
  const u32x4 w = *reinterpret_cast<const words *>(at & ~(uintptr_t)3);
  const uint32_t last = *reinterpret_cast<const uint32_t *>((at + 15) & ~(uintptr_t)3), by = (uint32_t)at & 3;
  // an address on 4 bytes has `last` in w already, and shifts by nothing
  return i32x4{(int)__builtin_amdgcn_alignbyte(w[1], w[0], by), (int)__builtin_amdgcn_alignbyte(w[2], w[1], by),
               (int)__builtin_amdgcn_alignbyte(w[3], w[2], by), (int)__builtin_amdgcn_alignbyte(last, w[3], by)};
}
// Bytes k .. k + 15 of a row of K >= 16, zero past its end, from the 16 bytes at min(k, K - 16).
__device__ __forceinline__ i32x4 cut_piece(i32x4 v, int k, int K) {
  typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
  const int s = 8 * min(max(k + 16 - K, 0), 16);
  const u64x2 w = __builtin_bit_cast(u64x2, v);
  const uint64_t far = w[1] >> (s & 63);   // by s, or by s - 64
  const u64x2 r = s >= 128 ? u64x2{0, 0} : s >= 64 ? u64x2{far, 0} : s ? u64x2{w[0] >> s | w[1] << (64 - s), far} : w;
  return __builtin_bit_cast(i32x4, r);
}
// The same for any K, from the row itself; nothing outside it is read.
__device__ __forceinline__ i32x4 piece(const int8_t *p, int k, int K) {
  if (K >= 16) return cut_piece(whole_piece(p + min(k, K - 16)), k, K);
  i32x4 v = {0, 0, 0, 0};
  for (int i = k; i < K; ++i) v[(i - k) >> 2] |= (int)((uint32_t)(uint8_t)p[i] << (8 * ((i - k) & 3)));
  return v;
}

}  // namespace

// ------------------------------------------------------------------------- few rows: K shared by the waves
// (16 MF) x (16 NF) outputs a workgroup, K dealt to its eight waves in pieces of 128 bytes, operands from memory straight
// into the products' registers: for layers whose larger tiles would leave most CUs idle, of any size and alignment.  U
// pieces of a wave's K, all loaded before their products, are on their way at once.  The waves' sums are added in LDS.
// Bound by the loads, 16 rows of 64 bytes each (25 bytes a ns and CU, 16 where rows start off words), below a few us by
// latency: (20, 24, 11076) 8.8 us, (20, 24, 11073) 15.3, (389, 701, 253) fp32 4.8.  Sixteen waves were no faster, and four
// pieces at once slower where K is short.
template <int EPI, typename TO, int MF, int NF, int WAVES, int U, bool BYTES>
__global__ __launch_bounds__(64 * WAVES) void k_linear_i8_split(int M, int N, int K, I8Args g, EpiArgs e) {
  constexpr int T = 64 * WAVES;
  __shared__ __attribute__((aligned(16))) int sums[WAVES][MF * NF * 256];
  const int tid = threadIdx.x, lane = tid & 63, fr = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m0 = blockIdx.y * (16 * MF), n0 = blockIdx.x * (16 * NF);
  // rows past the end: the last one again, never stored
  const int8_t *ar[MF], *wr[NF];
#pragma unroll
  for (int j = 0; j < MF; ++j) ar[j] = g.A + (int64_t)min(m0 + 16 * j + fr, M - 1) * K;
#pragma unroll
  for (int i = 0; i < NF; ++i) wr[i] = g.W + (int64_t)min(n0 + 16 * i + fr, N - 1) * K;
  i32x4 acc[NF][MF] = {};
  auto products = [&](const i32x4 (&fw)[2][NF], const i32x4 (&fa)[2][MF]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < NF; ++i)
#pragma unroll
        for (int j = 0; j < MF; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[h][i], fa[h][j], acc[i][j], 0, 0, 0);
  };
  // U whole pieces at a time, then what is left of them, then the one that K ends in
  const int whole = K / 128;
  int p = wave;
  auto batch = [&](auto ALL) {
    i32x4 fw[U][2][NF], fa[U][2][MF];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!decltype(ALL)::value && p + u * WAVES >= whole) break;
      const int k = 128 * (p + u * WAVES) + 16 * fq;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < NF; ++i) fw[u][h][i] = whole_piece<BYTES>(wr[i] + k + 64 * h);
#pragma unroll
        for (int j = 0; j < MF; ++j) fa[u][h][j] = whole_piece<BYTES>(ar[j] + k + 64 * h);
      }
    }
    __builtin_amdgcn_sched_barrier(0);   // no load sinks to its use
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!decltype(ALL)::value && p + u * WAVES >= whole) break;
      products(fw[u], fa[u]);
    }
  };
  for (; p + (U - 1) * WAVES < whole; p += U * WAVES) batch(std::true_type{});
  if (p < whole) batch(std::false_type{});
  if (K % 128 && whole % WAVES == wave) {
    const int k = 128 * whole + 16 * fq;
    i32x4 fw[2][NF], fa[2][MF];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < NF; ++i) fw[h][i] = piece(wr[i], k + 64 * h, K);
#pragma unroll
      for (int j = 0; j < MF; ++j) fa[h][j] = piece(ar[j], k + 64 * h, K);
    }
    products(fw, fa);
  }
  const int busy = min(WAVES, (K + 127) / 128);   // waves with a share of K
  if (wave < busy) {
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
      for (int j = 0; j < MF; ++j)   // lane: columns 4 fq .. + 3 of row fr
        *reinterpret_cast<i32x4 *>(&sums[wave][(j * NF + i) * 256 + fr * 16 + 4 * fq]) = acc[i][j];
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < (MF * NF * 256 + T - 1) / T; ++x) {
    const int o = tid + T * x, ml = o / (16 * NF), nl = o % (16 * NF), m = m0 + ml, n = n0 + nl;
    if (o >= MF * NF * 256 || m >= M || n >= N) continue;
    const int at = ((ml >> 4) * NF + (nl >> 4)) * 256 + (ml & 15) * 16 + (nl & 15);
    const int64_t to = (int64_t)m * e.ldo + n;
    float h = 0.f;
    if constexpr (EPI == EPI_RESIDUAL) h = (e.res_in ? e.res_in : (const float *)e.out)[to];
    int sum = 0;
    for (int w = 0; w < busy; ++w) sum += sums[w][at];
    put<EPI, TO>(e, to, scaled(sum, g.w_scale[n], g.a_scale[m], e.bias ? e.bias[n] : 0.f),
                 EPI == EPI_RESIDUAL && e.gate ? e.gate[n] : 1.f, h);
  }
}

// ------------------------------------------------------------------------------ any size and alignment
// 128x128 tiles, four waves of 64x64, two workgroups a CU.  K tiles of 128 bytes go through registers into two LDS
// stages, loaded two K tiles ahead: rows that start on any byte are not loaded into LDS directly.  K >= 16.  Bound by those
// loads and stores: (3000, 2504, 3004) 43 us, on bytes that start off words 52, on ring tiles with K = 3008 28.
namespace any8 {
constexpr int BM = 128, BN = 128, BK = 128, STAGE = (BM + BN) * BK, PER = (BM + BN) / 32;
// 16-byte piece c of row r at c ^ swz(r): the 16 lanes that read one piece of 16 rows at once meet 16 places
__device__ __forceinline__ int swz(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int at(int r, int c) { return r * BK + ((c ^ swz(r)) << 4); }
}  // namespace any8

template <int EPI, typename TO>
__global__ __launch_bounds__(256, 2) void k_linear_i8_any(int M, int N, int K, I8Args g, EpiArgs e, int NT) {
  using namespace any8;
  extern __shared__ __attribute__((aligned(16))) char smem_any[];
  const int tid = threadIdx.x, lane = tid & 63, fr = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mt = blockIdx.x / NT, m0 = mt * BM, n0 = (blockIdx.x - mt * NT) * BN;
  const int wm = 64 * (wave >> 1), wn = 64 * (wave & 1);
  const int lr = tid >> 3, lc = tid & 7;
  // rows past the end: the last one again, never stored
  const int8_t *const A0 = g.A + (int64_t)m0 * K, *const W0 = g.W + (int64_t)n0 * K;
  uint32_t row[PER];
#pragma unroll
  for (int x = 0; x < PER; ++x)
    row[x] = (uint32_t)K * (uint32_t)(x < PER / 2 ? min(lr + 32 * x, M - 1 - m0) : min(lr + 32 * (x - PER / 2), N - 1 - n0));
  i32x4 r[2][PER];   // K tile kt + 2 is loaded into one set while kt + 1 waits in the other
  auto load = [&](auto S, int kt) {
    const uint32_t k = (uint32_t)min(kt * BK + 16 * lc, K - 16);   // past the last K tile: loaded and not used
#pragma unroll
    for (int x = 0; x < PER; ++x) r[decltype(S)::value][x] = whole_piece((x < PER / 2 ? A0 : W0) + row[x] + k);
  };
  auto store = [&](auto S) {
    constexpr int st = decltype(S)::value;
#pragma unroll
    for (int x = 0; x < PER; ++x) *reinterpret_cast<i32x4 *>(smem_any + st * STAGE + at(lr + 32 * x, lc)) = r[st][x];
  };
  auto store_last = [&](auto S, int kt) {   // the K tile that K ends in
    constexpr int st = decltype(S)::value;
#pragma unroll
    for (int x = 0; x < PER; ++x) r[st][x] = cut_piece(r[st][x], kt * BK + 16 * lc, K);
    store(S);
  };
  i32x4 acc[4][4] = {};
  auto products = [&](auto S) {
    const char *s = smem_any + decltype(S)::value * STAGE;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      i32x4 fa[4], fw[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        fw[i] = *reinterpret_cast<const i32x4 *>(s + BM * BK + at(wn + 16 * i + fr, 4 * ks + fq));
        fa[i] = *reinterpret_cast<const i32x4 *>(s + at(wm + 16 * i + fr, 4 * ks + fq));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[i], fa[j], acc[i][j], 0, 0, 0);
    }
  };
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  const int KT = (K + BK - 1) / BK;
  load(S0{}, 0);
  load(S1{}, 1);
  if (KT > 1) store(S0{});
  else store_last(S0{}, 0);
  barrier();
  int kt = 0;
  for (; kt + 3 < KT; kt += 2) {
    load(S0{}, kt + 2);
    products(S0{});
    store(S1{});
    barrier();
    load(S1{}, kt + 3);
    products(S1{});
    store(S0{});
    barrier();
  }
  if (KT - kt == 3) load(S0{}, kt + 2);
  products(S0{});
  if (KT - kt == 2) {
    store_last(S1{}, kt + 1);
    barrier();
    products(S1{});
  } else if (KT - kt == 3) {
    store(S1{});
    barrier();
    products(S1{});
    store_last(S0{}, kt + 2);
    barrier();
    products(S0{});
  }
  barrier();   // every wave has read its last fragments
  // The wave's 64x64 sums through the freed stages, so that a store covers 64 columns of a row; 16-byte piece c of row r
  // at c ^ (r & 15).
  int *wl = reinterpret_cast<int *>(smem_any) + wave * (64 * 64);
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)   // lane: columns 4 fq .. + 3 of row fr
      *reinterpret_cast<i32x4 *>(wl + (16 * j + fr) * 64 + (((4 * i + fq) ^ fr) << 2)) = acc[i][j];
  // Lane l has column l, and the scale of row l, which the others take from it: every lane stays in the loop.
  const int mb = m0 + wm;
  const bool live = n0 + wn + lane < N;
  const int n = min(n0 + wn + lane, N - 1);
  const float as = g.a_scale[min(mb + lane, M - 1)];
  const float ws = g.w_scale[n], bias = e.bias ? e.bias[n] : 0.f, gate = EPI == EPI_RESIDUAL && e.gate ? e.gate[n] : 1.f;
  constexpr int B = 8;   // rows at a time, what is read of them before what is written
  const int rows = min(64, M - mb);
  for (int i0 = 0; i0 < rows; i0 += B) {
    float h[B];
    if constexpr (EPI == EPI_RESIDUAL) {
#pragma unroll
      for (int i = 0; i < B; ++i)
        if (i0 + i < rows) h[i] = (e.res_in ? e.res_in : (const float *)e.out)[(int64_t)(mb + i0 + i) * e.ldo + n];
    }
#pragma unroll
    for (int i = 0; i < B; ++i) {
      const int r = i0 + i;
      if (r >= rows) break;
      const float a = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, as), r));
      const float v = scaled(wl[r * 64 + (((lane >> 2) ^ (r & 15)) << 2) + (lane & 3)], ws, a, bias);
      if (live) put<EPI, TO>(e, (int64_t)(mb + r) * e.ldo + n, v, gate, EPI == EPI_RESIDUAL ? h[i] : 0.f);
    }
  }
}

// --------------------------------------------------------------------------------- tiles through an LDS ring
// (32 WTA) x (64 WT) tiles on eight waves, two of a SIMD, in a 2 (m) x 4 (n) grid of (16 WTA) x (16 WT) wave tiles, for
// K % 16 == 0, N % 8 == 0 and operands on 16 bytes.  K tiles of 128 bytes, the rows of the bf16 kernels' LDS, reach an
// LDS ring of NST stages by buffer loads that write LDS themselves (waves 0-3 the A rows, 4-7 the W rows), each K
// tile's loads issued NST - 1 tiles ahead or more; the fragments of a 64-byte substep are read between the
// products of the one before, and one barrier a K tile keeps the waves together.  The weights are the products' row
// operand, their rows permuted within groups of 32 so that a lane ends with eight consecutive columns of one row.
// On 256x256 tiles (16384, 5120, 13824) residual takes 975 us, 2.38 POP/s (an 8192^3 library product reaches 2.1), at 1.5
// GHz with the matrix cores busy 63% of the cycles: power bounds it.  With the loads, the LDS reads or the epilogue left
// out it takes 0.81, 0.96 and 0.83 of its time, the products alone 0.61.  (24960, 8960, 1536) GELU takes 370, 1.86 POP/s,
// at 2.0 GHz and 42%: 0.89, 0.92, 0.67 and 0.51, so there the epilogue costs most, 12 K tiles and 447 MB of output a launch.
// Two workgroups of four waves a CU on smaller tiles, so that one's epilogue runs under the other's products, took 388 at
// best where these took 398, and 1219 where these took 1033.
// The tiles for one round of workgroups are bound by the bytes a CU brings into LDS, 70 to 85 a ns: (1560, 1536, 8960) 31
// us, 204 tiles of 96x128.  With half of each K tile for four waves in place of eight, three quarters of the LDS reads
// and half the steps, they were slower (33, and 20 for 17 of (1560, 4608, 1536) on 128x128).
namespace ring {

constexpr int BK = 128;
constexpr uint32_t OUT_OF_RANGE = 0x80000000u;   // past every buffer below: reads give zero, writes are dropped

// 16-byte piece c of row r lies at c ^ swz(r): the 16 lanes that read one piece each of 16 rows (consecutive ones, or a
// permuted group's) meet 16 places of the 256 bytes that the banks span.
__device__ __forceinline__ int swz(int r) { return ((r >> 1) & 5) | (((r >> 1) ^ (r >> 3)) & 2); }
__device__ __forceinline__ int at(int r, int c) { return r * BK + ((c ^ swz(r)) << 4); }

// A buffer of wave-uniform address and size, in scalar registers.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *base, uint32_t bytes) {
  const uint64_t p = (uint64_t)base;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)p), hi = __builtin_amdgcn_readfirstlane((uint32_t)(p >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void *)(((uint64_t)hi << 32) | lo), (short)0,
                                           (int)__builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
__device__ __forceinline__ f32x4 ld4(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
}
template <int POL> __device__ __forceinline__ void st4(__amdgpu_buffer_rsrc_t r, uint32_t off, f32x4 v) {
  __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, off, 0, POL);
}

// Wait until at most n vector memory operations of this wave are in flight.
template <int N> __device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "the counter has six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x70 | 0xF00);
}
template <int PER> __device__ __forceinline__ void wait_tiles(int n) {   // but n K tiles of PER loads
  switch (n) {
    case 0: wait_loads<0>(); break;
    case 1: wait_loads<PER>(); break;
    default: wait_loads<2 * PER>(); break;
  }
}
// Workgroup -> tile: contiguous ranges of tiles for each of the 8 XCDs (dispatch is round-robin over them), in groups of
// `group` row blocks that sweep all column tiles, so that an XCD's workgroups share rows of A and W in its L2.
__device__ __forceinline__ void tile_of(int bid, int MT, int NT, int group, int &mt, int &nt) {
  const int total = MT * NT, xcd = bid & 7, t = xcd * (total >> 3) + min(xcd, total & 7) + (bid >> 3);
  const int per = group * NT, first = t / per * group, gm = min(MT - first, group), r = t - t / per * per;
  mt = first + r % gm;
  nt = r / gm;
}

// A wave's accumulators acc[i][j] hold row mbase + 16 j + fr and columns nbase + 32 (i / 2) + 8 fq + 4 (i % 2) .. + 3.
// They leave through the freed ring, so that every global access covers whole rows of the wave's tile: bf16 outputs as
// bf16 rows of 16 WT columns, fp32 ones as rows of 32 columns, one column group after another.  A wave has a region of its
// own there, in which its accesses are in order.
template <int EPI, typename TO, int WTA, int WT, int POL>
__device__ __forceinline__ void epilogue(const I8Args &g, const EpiArgs &e, const i32x4 (&acc)[WT][WTA], int M, int N,
                                         int mbase, int nbase, int fr, int fq, int lane, int wave, char *lds) {
  constexpr int R = 16 * WTA, CG = WT / 2;
  constexpr bool NARROW = (EPI == EPI_STORE || EPI == EPI_GELU) && sizeof(TO) == 2;
  constexpr uint32_t ES = NARROW ? 2u : 4u;
  char *wl = lds + wave * (NARROW ? R * 32 * WT : R * 128);
  const int rows = max(0, min(M - mbase, 16 * WTA));
  const uint32_t bytes = (uint32_t)rows * (uint32_t)e.ldo * ES;
  const int64_t base = (int64_t)mbase * e.ldo;
  const __amdgpu_buffer_rsrc_t rsO = buffer((char *)e.out + base * ES, bytes);
  const __amdgpu_buffer_rsrc_t rsS = buffer(g.w_scale, (uint32_t)N * 4u), rsB = buffer(e.bias, e.bias ? (uint32_t)N * 4u : 0u);
  float as[WTA];
#pragma unroll
  for (int j = 0; j < WTA; ++j) as[j] = g.a_scale[min(mbase + 16 * j + fr, M - 1)];
  barrier();   // every wave is past its last fragment reads
  if constexpr (NARROW) {
    constexpr int NC = 2 * WT;   // pieces of eight columns a row
    auto place = [&](int r, int k) { return r * (32 * WT) + ((k ^ (WT == 4 ? (r >> 1) & 7 : (r >> 2) & 3)) << 4); };
    f32x4 ws[CG][2], bias[CG][2];
#pragma unroll
    for (int cg = 0; cg < CG; ++cg) {
      const int n = nbase + 32 * cg + 8 * fq;
      const uint32_t cn = n < N ? (uint32_t)n * 4u : OUT_OF_RANGE;   // N % 8 == 0
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        ws[cg][hf] = ld4(rsS, cn + 16 * hf);
        bias[cg][hf] = ld4(rsB, cn + 16 * hf);
      }
    }
    constexpr int RI = 64 / NC;   // rows an instruction covers
    const int k = lane % NC, rr = lane / NC, n = nbase + 8 * k;
    // a buffer is below 2^30 bytes: an offset out of range stays there with a row's offset added
    const uint32_t o0 = n < N ? (uint32_t)rr * (uint32_t)e.ldo * 2u + (uint32_t)n * 2u : OUT_OF_RANGE;
#pragma unroll
    for (int cg = 0; cg < CG; ++cg)
#pragma unroll
      for (int j = 0; j < WTA; ++j) {
        auto value = [&](int q) {
          const float v = scaled(acc[2 * cg + (q >> 2)][j][q & 3], ws[cg][q >> 2][q & 3], as[j], bias[cg][q >> 2][q & 3]);
          return EPI == EPI_GELU ? gelu_tanh(v) : v;
        };
        typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
        u32x4 w;   // by pairs: one conversion each, and no moves between them
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float lo = value(2 * q), hi = value(2 * q + 1);
          w[q] = __builtin_bit_cast(uint32_t, bf16x2{(bf16)lo, (bf16)hi});
        }
        *reinterpret_cast<u32x4 *>(wl + place(16 * j + fr, 4 * cg + fq)) = w;
      }
#pragma unroll
    for (int t = 0; t < R / RI; ++t) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(wl + place(RI * t + rr, k));
      __builtin_amdgcn_raw_buffer_store_b128(v, rsO, o0 + (uint32_t)(RI * t) * (uint32_t)e.ldo * 2u, 0, POL);
    }
  } else {
    constexpr int NTR = R / 8, B = NTR % 4 == 0 ? 4 : 2, NB = NTR / B;   // read-back instructions a column group, in batches of B
    static_assert(NTR % B == 0, "batches");
    const __amdgpu_buffer_rsrc_t rsI = buffer((const char *)(e.res_in ? e.res_in : (const float *)e.out) + base * 4, bytes);
    const __amdgpu_buffer_rsrc_t rsC = buffer(e.cache ? e.cache + base : nullptr, e.cache ? bytes : 0u);
    const __amdgpu_buffer_rsrc_t rsG = buffer(e.gate, e.gate ? (uint32_t)N * 4u : 0u);
    const int k = lane & 7, rr = lane >> 3;
    const uint32_t step = 8u * (uint32_t)e.ldo * 4u;
#pragma unroll
    for (int cg = 0; cg < CG; ++cg) {
      const int nw = nbase + 32 * cg + 8 * fq, n = nbase + 32 * cg + 4 * k;
      const uint32_t cw = nw < N ? (uint32_t)nw * 4u : OUT_OF_RANGE;
      const f32x4 ws[2] = {ld4(rsS, cw), ld4(rsS, cw + 16)}, bias[2] = {ld4(rsB, cw), ld4(rsB, cw + 16)};
      const uint32_t o0 = n < N ? (uint32_t)rr * (uint32_t)e.ldo * 4u + (uint32_t)n * 4u : OUT_OF_RANGE;
      f32x4 gate = {1.f, 1.f, 1.f, 1.f}, h[2][B];
      if (EPI == EPI_RESIDUAL && e.gate) gate = ld4(rsG, n < N ? (uint32_t)n * 4u : OUT_OF_RANGE);
      auto fetch = [&](int bt) {
        if constexpr (EPI == EPI_RESIDUAL) {
#pragma unroll
          for (int i = 0; i < B; ++i) h[bt & 1][i] = ld4(rsI, o0 + (uint32_t)(B * bt + i) * step);
        }
      };
      fetch(0);
#pragma unroll
      for (int j = 0; j < WTA; ++j)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          f32x4 v;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            v[q] = scaled(acc[2 * cg + hf][j][q], ws[hf][q], as[j], bias[hf][q]);
            if constexpr (EPI == EPI_GELU) v[q] = gelu_tanh(v[q]);
          }
          const int r = 16 * j + fr, kk = 2 * fq + hf;
          *reinterpret_cast<f32x4 *>(wl + r * 128 + ((kk ^ ((r >> 1) & 7)) << 4)) = v;
        }
#pragma unroll
      for (int bt = 0; bt < NB; ++bt) {
        if (bt + 1 < NB) fetch(bt + 1);
#pragma unroll
        for (int i = 0; i < B; ++i) {
          const int t = B * bt + i, r = 8 * t + rr;
          f32x4 v = *reinterpret_cast<const f32x4 *>(wl + r * 128 + ((k ^ ((r >> 1) & 7)) << 4));
          if constexpr (EPI == EPI_RESIDUAL) {
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = fmaf(gate[q], v[q], h[bt & 1][i][q]);
          }
          st4<POL>(rsO, o0 + (uint32_t)t * step, v);
          if (EPI == EPI_RESIDUAL && e.cache) st4<POL>(rsC, o0 + (uint32_t)t * step, v);
        }
      }
    }
  }
}

template <int EPI, typename TO, int WTA, int WT, int NST, int POL>
__device__ __forceinline__ void tile(int M, int N, int K, const I8Args &g, const EpiArgs &e, int m0, int n0, char *smem) {
  static_assert(WTA >= 2 && WTA <= 8 && (WT == 2 || WT == 4), "tile");
  constexpr int BM = 32 * WTA, BN = 64 * WT, STAGE = (BM + BN) * BK;
  static_assert(NST >= 2 && NST <= 3 && NST * STAGE <= 160 * 1024, "wait_tiles counts two tiles ahead; LDS");
  constexpr int NA = WTA, NW = 2 * WT, NL = NA > NW ? NA : NW;   // loads a K tile of an A wave and of a W wave
  constexpr int NR = WT + WTA;                                   // fragments a substep
  const int tid = threadIdx.x, lane = tid & 63, fr = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;
  const bool loads_a = wave < 4;
  const __amdgpu_buffer_rsrc_t rs = loads_a ? buffer(g.A + (int64_t)m0 * K, (uint32_t)min(M - m0, BM) * (uint32_t)K)
                                            : buffer(g.W + (int64_t)n0 * K, (uint32_t)min(N - n0, BN) * (uint32_t)K);
  // load x: rows row0 + 8 x .. + 7, lane l the piece that belongs in slot l & 7 of row l >> 3
  const int row0 = loads_a ? 8 * NA * wave : 8 * NW * (wave - 4);
  uint32_t voff[8];
#pragma unroll
  for (int x = 0; x < NL; ++x) {
    const int r = row0 + 8 * x + (lane >> 3);
    voff[x] = (uint32_t)(r * K + (((lane & 7) ^ swz(r)) << 4));
  }
  char *const dst0 = smem + ((loads_a ? 0 : BM) + row0) * BK;
  const int KT = (K + BK - 1) / BK;
  // LAST: the last K tile, whose pieces past K (the next row's bytes, or past the last row) read as zero
  auto load_one = [&](auto LAST, int kt, int st, int x) {
    if (loads_a ? x >= NA : x >= NW) return;
    uint32_t off = voff[x];
    if (decltype(LAST)::value && kt * BK + (((lane & 7) ^ swz(row0 + 8 * x + (lane >> 3))) << 4) >= K) off = OUT_OF_RANGE;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void *)(dst0 + st * STAGE + x * (8 * BK)), 16,
                                             off, kt * BK, 0, 0);
  };
  uint32_t offW[2][2], offA[2][2];   // of fragments 0 and 1 of each substep; those 32 rows on share their swizzle
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      offW[ks][q] = BM * BK + at(16 * WT * wn + 8 * (fr >> 2) + 4 * q + (fr & 3), fq + 4 * ks);
      offA[ks][q] = at(16 * WTA * wm + 16 * q + fr, fq + 4 * ks);
    }
  i32x4 acc[WT][WTA];
  i32x4 fw0[WT], fa0[WTA], fw1[WT], fa1[WTA];
  auto rd = [&](int st, int ks, i32x4 *fw, i32x4 *fa, int x) {
    const char *base = smem + st * STAGE;
    if (x < WT) fw[x] = *reinterpret_cast<const i32x4 *>(base + offW[ks][x & 1] + 32 * BK * (x >> 1));
    else fa[x - WT] = *reinterpret_cast<const i32x4 *>(base + offA[ks][x & 1] + 32 * BK * ((x - WT) >> 1));
  };
  // the products of one substep; between them the reads of the next and the loads of K tile `kt`
  auto substep = [&](auto READ, auto LOAD, auto LAST, const i32x4 *fw, const i32x4 *fa, int nst, int nks, i32x4 *nfw, i32x4 *nfa, int kt,
                     int st) {
#pragma unroll
    for (int j = 0; j < WTA; ++j) {
#pragma unroll
      for (int i = 0; i < WT; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[i], fa[j], acc[i][j], 0, 0, 0);
      if constexpr (decltype(READ)::value) {
#pragma unroll
        for (int x = j * NR / WTA; x < (j + 1) * NR / WTA; ++x) rd(nst, nks, nfw, nfa, x);
      }
      if constexpr (decltype(LOAD)::value) {
#pragma unroll
        for (int x = j * NL / WTA; x < (j + 1) * NL / WTA; ++x) load_one(LAST, kt, st, x);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  using T_ = std::true_type;
  using F_ = std::false_type;
#pragma unroll
  for (int t = 0; t < NST; ++t)
    if (t < KT) {
#pragma unroll
      for (int x = 0; x < NL; ++x) load_one(T_{}, t, t, x);
    }
  auto landed = [&](int ahead) {   // but `ahead` K tiles
    if (loads_a) wait_tiles<NA>(ahead);
    else wait_tiles<NW>(ahead);
  };
  landed(min(NST, KT) - 1);
  barrier();
#pragma unroll
  for (int x = 0; x < NR; ++x) rd(0, 0, fw0, fa0, x);
#pragma unroll
  for (int i = 0; i < WT; ++i)
#pragma unroll
    for (int j = 0; j < WTA; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  int kt = 0, st = 0;
  auto full = [&](auto LAST) {
    const int nx = st + 1 == NST ? 0 : st + 1;
    substep(T_{}, F_{}, F_{}, fw0, fa0, st, 1, fw1, fa1, 0, 0);
    landed(NST - 2);   // K tile kt + 1
    barrier();         // for every wave; and nobody reads stage st any more
    substep(T_{}, T_{}, LAST, fw1, fa1, nx, 0, fw0, fa0, kt + NST, st);
    st = nx;
  };
  for (; kt + NST + 1 < KT; ++kt) full(F_{});
  if (kt + NST < KT) {
    full(T_{});
    ++kt;
  }
  for (; kt + 1 < KT; ++kt) {   // nothing left to load
    const int nx = st + 1 == NST ? 0 : st + 1;
    substep(T_{}, F_{}, F_{}, fw0, fa0, st, 1, fw1, fa1, 0, 0);
    landed(KT - 2 - kt);
    barrier();
    substep(T_{}, F_{}, F_{}, fw1, fa1, nx, 0, fw0, fa0, 0, 0);
    st = nx;
  }
  substep(T_{}, F_{}, F_{}, fw0, fa0, st, 1, fw1, fa1, 0, 0);
  substep(F_{}, F_{}, F_{}, fw1, fa1, 0, 0, fw0, fa0, 0, 0);
  static_assert(8 * 16 * WTA * 128 <= NST * STAGE, "the ring holds the waves' rows");
  epilogue<EPI, TO, WTA, WT, POL>(g, e, acc, M, N, m0 + 16 * WTA * wm, n0 + 16 * WT * wn, fr, fq, lane, wave, smem);
}

}  // namespace ring

// ------------------------------------------------------------ few rows, aligned: K shared by the waves, each with a ring
// (16 MF) x (16 NF) outputs a workgroup and K dealt to its waves in pieces of 128 bytes as in k_linear_i8_split, but each
// wave brings its pieces through an LDS ring of its own by loads that write LDS, rows of 128 bytes whole, NST pieces
// ahead: nobody waits for another wave until the sums are added, and a CU reads two to three times the bytes a ns.  For K
// in whole pieces of 16 bytes and rows on 16 bytes.  (130, 1536, 8960) 9.5 us against 18.9 of k_linear_i8_split, (37, 1536,
// 8960) 6.7 and 14.0, (1, 5120, 13824) 12.6 and 19.5 (5.6 TB/s, W from the cache behind L2): the bytes a CU has on its way
// bound it, below some 5 us latency.  Four stages for four waves or for a 16x16 tile were no faster.
template <int EPI, typename TO, int MF, int NF, int WAVES, int NST>
__global__ __launch_bounds__(64 * WAVES) void k_linear_i8_few(int M, int N, int K, I8Args g, EpiArgs e) {
  using namespace ring;
  constexpr int T = 64 * WAVES, ROWS = 16 * (MF + NF), STAGE = ROWS * BK, LA = 2 * MF, LW = 2 * NF, PER = LA + LW;
  static_assert(NST <= 3 && (NST - 1) * PER < 64 && NST * STAGE >= MF * NF * 1024, "a wave's ring holds its sums");
  extern __shared__ __attribute__((aligned(16))) char smem_few[];
  const int tid = threadIdx.x, lane = tid & 63, fr = lane & 15, fq = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m0 = blockIdx.y * (16 * MF), n0 = blockIdx.x * (16 * NF);
  char *const mine = smem_few + wave * (NST * STAGE);
  const __amdgpu_buffer_rsrc_t rsA = buffer(g.A + (int64_t)m0 * K, (uint32_t)min(M - m0, 16 * MF) * (uint32_t)K);
  const __amdgpu_buffer_rsrc_t rsW = buffer(g.W + (int64_t)n0 * K, (uint32_t)min(N - n0, 16 * NF) * (uint32_t)K);
  // load x: rows 8 x .. + 7 of A (x < LA), then of W; lane l the piece that belongs in slot l & 7 of row l >> 3
  const int lr = lane >> 3, ls = lane & 7;
  const int pieces = (K + BK - 1) / BK, count = wave < pieces ? (pieces - wave + WAVES - 1) / WAVES : 0;
  auto load = [&](int i) {   // this wave's piece i
    const int k0 = (wave + i * WAVES) * BK;
    char *to = mine + (i % NST) * STAGE;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      const int r = 8 * (x < LA ? x : x - LA) + lr, slot = (ls ^ swz(8 * x + lr)) << 4;
      // past K (the next row's bytes, or past the last row): zero
      const uint32_t off = k0 + slot < K ? (uint32_t)(r * K + slot) : OUT_OF_RANGE;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(x < LA ? rsA : rsW, (__attribute__((address_space(3))) void *)(to + x * (8 * BK)), 16,
                                               off, k0, 0, 0);
    }
  };
  i32x4 acc[NF][MF] = {};
#pragma unroll
  for (int i = 0; i < NST; ++i)
    if (i < count) load(i);
  for (int i = 0; i < count; ++i) {
    wait_tiles<PER>(min(NST - 1, count - 1 - i));   // all but the pieces after this one
    asm volatile("" ::: "memory");
    const char *from = mine + (i % NST) * STAGE;
    i32x4 fw[2][NF], fa[2][MF];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < MF; ++j) fa[h][j] = *reinterpret_cast<const i32x4 *>(from + at(16 * j + fr, 4 * h + fq));
#pragma unroll
      for (int n = 0; n < NF; ++n) fw[h][n] = *reinterpret_cast<const i32x4 *>(from + at(16 * (MF + n) + fr, 4 * h + fq));
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0): the stage has been read
    __builtin_amdgcn_sched_barrier(0);
    if (i + NST < count) load(i + NST);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < NF; ++n)
#pragma unroll
        for (int j = 0; j < MF; ++j) acc[n][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[h][n], fa[h][j], acc[n][j], 0, 0, 0);
  }
  if (count) {
#pragma unroll
    for (int n = 0; n < NF; ++n)
#pragma unroll
      for (int j = 0; j < MF; ++j)   // lane: columns 4 fq .. + 3 of row fr
        *reinterpret_cast<i32x4 *>(mine + ((j * NF + n) * 256 + fr * 16 + 4 * fq) * 4) = acc[n][j];
  }
  __syncthreads();
  const int busy = min(WAVES, pieces);
#pragma unroll
  for (int x = 0; x < (MF * NF * 256 + T - 1) / T; ++x) {
    const int o = tid + T * x, ml = o / (16 * NF), nl = o % (16 * NF), m = m0 + ml, n = n0 + nl;
    if (o >= MF * NF * 256 || m >= M || n >= N) continue;
    const int64_t to = (int64_t)m * e.ldo + n;
    float h = 0.f;
    if constexpr (EPI == EPI_RESIDUAL) h = (e.res_in ? e.res_in : (const float *)e.out)[to];
    const char *from = smem_few + (((ml >> 4) * NF + (nl >> 4)) * 256 + (ml & 15) * 16 + (nl & 15)) * 4;
    int sum = 0;
    for (int w = 0; w < busy; ++w) sum += *reinterpret_cast<const int *>(from + w * (NST * STAGE));
    put<EPI, TO>(e, to, scaled(sum, g.w_scale[n], g.a_scale[m], e.bias ? e.bias[n] : 0.f),
                 EPI == EPI_RESIDUAL && e.gate ? e.gate[n] : 1.f, h);
  }
}

template <int EPI, typename TO, int WTA, int WT, int NST, int POL>
__global__ __launch_bounds__(512, 1) void k_linear_i8_ring(int M, int N, int K, I8Args g, EpiArgs e, int MT, int NT, int group) {
  extern __shared__ __attribute__((aligned(16))) char smem_ring[];
  int mt, nt;
  ring::tile_of(blockIdx.x, MT, NT, group, mt, nt);
  ring::tile<EPI, TO, WTA, WT, NST, POL>(M, N, K, g, e, 32 * WTA * mt, 64 * WT * nt, smem_ring);
}

// The same on MT row blocks of two heights, `tall` of 32 WTA rows and the others of 32 (WTA - 1), spread evenly over the
// block index (block i is tall where floor((i + 1) tall / MT) > floor(i tall / MT)), 256 columns wide: so that a launch fills
// whole rounds of the chip.
template <int EPI, typename TO, int WTA, int POL>
__global__ __launch_bounds__(512, 1) void k_linear_i8_mix(int M, int N, int K, I8Args g, EpiArgs e, int MT, int NT, int group,
                                                          int tall) {
  extern __shared__ __attribute__((aligned(16))) char smem_mix[];
  int mt, nt;
  ring::tile_of(blockIdx.x, MT, NT, group, mt, nt);
  const int before = (int)((int64_t)mt * tall / MT), upto = (int)((int64_t)(mt + 1) * tall / MT);
  const int m0 = 32 * ((WTA - 1) * mt + before), n0 = 256 * nt;
  if (m0 >= M) return;   // a forced plan of more blocks than M has
  if (upto > before) ring::tile<EPI, TO, WTA, 4, 2, POL>(M, N, K, g, e, m0, n0, smem_mix);
  else ring::tile<EPI, TO, WTA - 1, 4, 2, POL>(M, N, K, g, e, m0, n0, smem_mix);
}

// ------------------------------------------------------------------------------------------- dispatch
namespace {

// Outputs of 64 MiB and more are stored non-temporally (the nt bit of a buffer store): a round's burst of output lines
// then leaves the next tiles' operands in L2.  (24960, 8960, 1536) GELU 383 -> 372 us, (16384, 5120, 13824) residual
// 1000 -> 968, (24960, 4608, 1536) 169 -> 159.  Smaller ones stay where the next kernel finds them.
constexpr int kStoreNT = 2;
constexpr size_t kNTBytes = (size_t)64 << 20;
// Rows of a launch: a grid of 512 threads for 256 outputs, the most a kernel takes, is within 2^32 threads and 2^16 rows
// of workgroups.  Larger tiles would take more; past 32768 rows they run as several launches all the same.
int rows_per_launch(int N) { return std::min(1 << 15, (1 << 30) / N); }

// Choice of kernel: estimates of a launch's device time in us, whole rounds of workgroups at a time, which stay within
// 10% of the fastest over the shapes they were fitted to (us below: 256x256, 128x256, 128x128 two a CU, 128x128 with three
// stages; MI355X; every kernel gives the same bits).
//   * Ring tiles: a round costs its K tiles and a fixed part, the epilogue, larger where it reads and writes the
//     residual stream.  (24960, 8960, 1536) GELU 377, 425, 406, 483; (16384, 5120, 13824) residual 968, 1158, 1315, 1443;
//     (24960, 1536, 1536) residual 148, 140, 136, 149; (24960, 1536, 8960) residual 394, 381, 410, 480; (4680, 1536,
//     8960) 117, 75, 81, 97; (1560, 4608, 1536) 22, 16.4, 15.4, 18; (900, 7168, 512) 128x256 9.1, 128x128 8.3; (3120, 2304,
//     768) GELU 12.8 and 11.5; (1560, 4608, 2048) 18.4 and 17.8, (3000, 2504, 3008) 27.6 and 30.3.
//   * Row blocks of two heights, where they save a round: beside 256x256, 128x256 and two 128x128, (24960, 8960, 1536) GELU
//     370, 374, 422, 401; (6240, 8960, 1536) GELU 97, 105, 112, 105; (3120, 8960, 1536) GELU 52, 54, 66, 58; (24960, 1536,
//     8960) residual 364, 395, 382, 411; (12480, 1536, 8960) residual 212, 225, 211, 230; (24960, 1536, 1536) residual 138,
//     149, 140, 136, where the estimate misses the fastest by 2%.
//   * What fits one round of 128x128 tiles waits on the latency of each K tile, which a third stage hides best, and less on
//     smaller tiles as long as those fit a round too.  (1560, 1536, 8960) residual 84, 54, 50, and with three stages 128x128
//     35, 96x128 33, 64x128 45 (two rounds); (1560, 1536, 1536) 9.3, 8.6, 10.5; (512, 1536, 4096) 15.4, 14.1, 13.3; (851,
//     1536, 8960) 29, 27, 25; (200, 5120, 5120) 18.7, 18.5, 16.5.
//   * k_linear_i8_few by the bytes a CU reads, 85 a ns, and a part a round: (130, 1536, 8960) 32x32 9.5, 64x32 13.9, 64x128
//     ring tiles 22.6; (64, 5120, 5120) 64x32 11.2, 32x32 12.4, ring 15.8; (37, 1536, 8960) 32x16 6.7, 16x16 7.6, ring 21;
//     (200, 5120, 5120) 26 and 16.5; (325, 1536, 1536) 8.5 and 6.7.
//   * k_linear_i8_split the same way, 25 a ns, 16 on rows off 4 bytes: it has what few does not take, and small layers, for
//     which it needs no more LDS than its sums: (390, 704, 256) 3.4 against 3.9 of few and 3.8 of ring tiles.
//   * k_linear_i8_any for the larger layers off 16 bytes: (3000, 2501, 3001) 52 (64x32 split 176), (777, 1111, 999) 16
//     and 12, (389, 701, 253) 10 and 4.8, (5000, 333, 2222) 24 and 40.
enum Kernel { SPLIT11, SPLIT21, SPLIT22, SPLIT42, ANY, FEW11, FEW21, FEW22, FEW42,
              RING_256x256, RING_128x256, RING_128x128_TWO, RING_128x128, RING_96x128, RING_64x128, MIX };
struct Plan {
  Kernel kernel;
  int wta = 0, blocks = 0, tall = 0;   // MIX
};
constexpr const char *kNames[] = {"split:16x16", "split:32x16", "split:32x32", "split:64x32", "any", "few:16x16",
                                  "few:32x16", "few:32x32", "few:64x32", "256x256", "128x256", "128x128:two", "128x128",
                                  "96x128", "64x128"};

// A round of 32 w rows, of one of 256.
constexpr double kHeight[9] = {0, 0, 0, 0, 0, 0.75, 0.82, 0.9, 1.0};
// Whether rows start off 4 bytes.
bool off_words(const I8Args &g, int K) { return ((uintptr_t)g.A | (uintptr_t)g.W | (uintptr_t)K) % 4; }

// aligned: what the ring tiles take; pieces: rows of whole 16-byte pieces; words: rows on 4 bytes.
Plan pick(int M, int N, int K, bool aligned, bool pieces, bool words, int epi) {
  // FLASHBON_I8_TILE (tests and tuning) forces a kernel by its name; one that does not take the layer is passed over
  // ("mix:<w>:<blocks>:<tall>": two heights of 32 w and 32 (w - 1) rows, w in 6..8, covering M)
  if (const char *force = getenv("FLASHBON_I8_TILE")) {
    for (int k = 0; k < MIX; ++k)
      if (!strcmp(force, kNames[k]) && (k <= SPLIT42 || (k == ANY ? K >= 16 : k <= FEW42 ? pieces : aligned))) return {(Kernel)k};
    Plan p = {MIX};
    if (aligned && sscanf(force, "mix:%d:%d:%d", &p.wta, &p.blocks, &p.tall) == 3 && p.wta >= 6 && p.wta <= 8 && p.tall >= 0 &&
        p.tall <= p.blocks && p.blocks <= M && 32 * ((int64_t)(p.wta - 1) * p.blocks + p.tall) >= M)
      return p;
  }
  const double cus = cu_count(), kt = (K + 127) / 128;
  Plan best = {SPLIT11};
  double t_best = 1e30;
  // rounds of `slots` workgroups of bm x bn outputs, each `per_round`
  auto offer = [&](Kernel k, int bm, int bn, double slots, double once, double per_round) {
    const double tiles = (double)((M + bm - 1) / bm) * ((N + bn - 1) / bn), t = once + ceil(tiles / slots) * per_round;
    if (t < t_best) {
      t_best = t;
      best = {k};
    }
  };
  const double rate = words ? 25e3 : 16e3;   // bytes a us and CU
  offer(SPLIT11, 16, 16, cus, 2.1, (16 + fmin(16, M)) * K / rate);
  offer(SPLIT21, 32, 16, cus, 2.1, (16 + fmin(32, M)) * K / rate);
  offer(SPLIT22, 32, 32, cus, 2.1, (32 + fmin(32, M)) * K / rate);
  offer(SPLIT42, 64, 32, cus, 2.8, (32 + fmin(64, M)) * K / rate);
  if (pieces) {
    const double ring = 85e3;
    offer(FEW11, 16, 16, cus, 2.5, 0.5 + (16 + fmin(16, M)) * K / ring);
    offer(FEW21, 32, 16, cus, 2.5, 0.7 + (16 + fmin(32, M)) * K / ring);
    offer(FEW22, 32, 32, cus, 2.5, 1.0 + (32 + fmin(32, M)) * K / ring);
    offer(FEW42, 64, 32, cus, 2.5, 2.3 + (32 + fmin(64, M)) * K / ring);
  }
  if (!aligned) {
    if (K >= 16) offer(ANY, 128, 128, 2 * cus, 5.0, 1.2 * kt);
    return best;
  }
  if ((double)((M + 127) / 128) * ((N + 127) / 128) <= cus) {
    offer(RING_64x128, 64, 128, cus, 3.3, 0.3 * kt);
    offer(RING_96x128, 96, 128, cus, 3.3, 0.345 * kt);
    offer(RING_128x128, 128, 128, cus, 3.3, 0.37 * kt);
    return best;
  }
  const bool res = epi == EPI_RESIDUAL;
  offer(RING_256x256, 256, 256, cus, 0, 1.75 * kt + (res ? 27 : 9));
  offer(RING_128x256, 128, 256, cus, 0, 1.03 * kt + (res ? 15 : 6));
  const bool alone = (double)((M + 127) / 128) * ((N + 127) / 128) <= 2 * cus;   // one round, nothing stored before it
  offer(RING_128x128_TWO, 128, 128, 2 * cus, 0, 1.2 * kt + (res ? 12 : alone ? 2.9 : 5.5));
  // as many blocks of two heights as fill whole rounds
  const int NT = (N + 255) / 256;
  for (int w = 8; w >= 6; --w) {
    const int lo = 32 * (w - 1), least = (M + lo + 31) / (lo + 32), most = (M + lo - 1) / lo;
    for (int r = (int)((least * NT + cus - 1) / cus); r * cus < (double)(most + 1) * NT; ++r) {
      const int blocks = std::min(most, (int)(r * cus / NT)), tall = std::max(0, (M - lo * blocks + 31) / 32);
      if (blocks < least || tall > blocks) continue;
      const double t = r * ((1.75 * kt + (res ? 27 : 9)) * (kHeight[w - 1] + (kHeight[w] - kHeight[w - 1]) * tall / blocks));
      if (t < 0.98 * t_best) {
        t_best = t;
        best = {MIX, w, blocks, tall};
      }
    }
  }
  return best;
}

template <int EPI, typename TO>
hipError_t launch_any(int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s) {
  const int NT = (N + any8::BN - 1) / any8::BN, MT = (M + any8::BM - 1) / any8::BM;
  hipLaunchKernelGGL((k_linear_i8_any<EPI, TO>), dim3(MT * NT), dim3(256), 2 * any8::STAGE, s, M, N, K, g, e, NT);
  return hipGetLastError();
}

template <int EPI, typename TO, int MF, int NF, int U>
hipError_t launch_split(int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s) {
  const dim3 grid((N + 16 * NF - 1) / (16 * NF), (M + 16 * MF - 1) / (16 * MF));
  if (off_words(g, K))
    hipLaunchKernelGGL((k_linear_i8_split<EPI, TO, MF, NF, 8, U, true>), grid, dim3(512), 0, s, M, N, K, g, e);
  else
    hipLaunchKernelGGL((k_linear_i8_split<EPI, TO, MF, NF, 8, U, false>), grid, dim3(512), 0, s, M, N, K, g, e);
  return hipGetLastError();
}

// Gives a kernel its LDS on the current device, once; ready: the devices that have it.
template <typename F> hipError_t with_lds(F kern, int lds, std::atomic<uint64_t> &ready) {
  int dev = 0;
  hipError_t err = hipGetDevice(&dev);
  if (err != hipSuccess) return err;
  const uint64_t bit = (uint64_t)1 << (dev & 63);
  if (dev <= 63 && (ready & bit)) return hipSuccess;
  err = hipFuncSetAttribute((const void *)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (err == hipSuccess) ready |= bit;
  return err;
}

template <int EPI, typename TO> bool stores_past_caches(int M, int N, const EpiArgs &e) {
  return (size_t)M * N * (EPI == EPI_STORE || EPI == EPI_GELU ? sizeof(TO) : EPI == EPI_RESIDUAL && e.cache ? 8 : 4) >= kNTBytes;
}

// Row blocks of a tile group, a compromise over what was measured at 1, 2, 4 and 8: (24960, 8960, 1536) 403, 370, 364, 362 us;
// (24960, 4608, 1536) 164, 164, 166, 168; (16384, 13824, 5120) 967, 931, 915, 958; (16384, 5120, 13824) 992, 974, 988, 1011;
// (16384, 5120, 5120) 486, 476, 482, 491; (24960, 1536, 8960) 357, 356, 351, 363; (24960, 1536, 1536) 135, 134, 133, 133.
int group_of(int N, int K) { return N <= 2048 ? 1 : K >= 4096 ? 2 : 8; }

template <int EPI, typename TO, int MF, int NF, int WAVES, int NST>
hipError_t launch_few(int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s) {
  constexpr int LDS = WAVES * NST * 16 * (MF + NF) * ring::BK;
  const auto kern = k_linear_i8_few<EPI, TO, MF, NF, WAVES, NST>;
  static std::atomic<uint64_t> ready;
  const hipError_t err = with_lds(kern, LDS, ready);
  if (err != hipSuccess) return err;
  hipLaunchKernelGGL(kern, dim3((N + 16 * NF - 1) / (16 * NF), (M + 16 * MF - 1) / (16 * MF)), dim3(64 * WAVES), LDS, s, M, N, K, g, e);
  return hipGetLastError();
}

template <int EPI, typename TO, int WTA>
hipError_t launch_mix(int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s, const Plan &p) {
  constexpr int LDS = 2 * (32 * WTA + 256) * ring::BK;
  const bool nt = stores_past_caches<EPI, TO>(M, N, e);
  const auto kern = nt ? k_linear_i8_mix<EPI, TO, WTA, kStoreNT> : k_linear_i8_mix<EPI, TO, WTA, 0>;
  static std::atomic<uint64_t> ready[2];
  const hipError_t err = with_lds(kern, LDS, ready[nt]);
  if (err != hipSuccess) return err;
  const int NT = (N + 255) / 256;
  hipLaunchKernelGGL(kern, dim3(p.blocks * NT), dim3(512), LDS, s, M, N, K, g, e, p.blocks, NT, group_of(N, K), p.tall);
  return hipGetLastError();
}

template <int EPI, typename TO, int WTA, int WT, int NST>
hipError_t launch_ring(int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s) {
  constexpr int BM = 32 * WTA, BN = 64 * WT, LDS = NST * (BM + BN) * ring::BK;
  const bool nt = stores_past_caches<EPI, TO>(M, N, e);
  const auto kern = nt ? k_linear_i8_ring<EPI, TO, WTA, WT, NST, kStoreNT> : k_linear_i8_ring<EPI, TO, WTA, WT, NST, 0>;
  static std::atomic<uint64_t> ready[2];
  const hipError_t err = with_lds(kern, LDS, ready[nt]);
  if (err != hipSuccess) return err;
  const int MT = (M + BM - 1) / BM, NT = (N + BN - 1) / BN;
  hipLaunchKernelGGL(kern, dim3(MT * NT), dim3(512), LDS, s, M, N, K, g, e, MT, NT, group_of(N, K));
  return hipGetLastError();
}

template <int EPI, typename TO>
hipError_t launch_rows(int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s) {
  const uintptr_t at = (uintptr_t)g.A | (uintptr_t)g.W | (uintptr_t)g.w_scale | (uintptr_t)e.bias | (uintptr_t)e.out |
                       (uintptr_t)e.res_in | (uintptr_t)e.cache | (uintptr_t)e.gate;
  const bool pieces = K % 16 == 0 && ((uintptr_t)g.A | (uintptr_t)g.W) % 16 == 0;
  const Plan p = pick(M, N, K, pieces && N % 8 == 0 && at % 16 == 0, pieces, !off_words(g, K), EPI);
  switch (p.kernel) {
    case SPLIT11: return launch_split<EPI, TO, 1, 1, 2>(M, N, K, g, e, s);
    case SPLIT21: return launch_split<EPI, TO, 2, 1, 2>(M, N, K, g, e, s);
    case SPLIT22: return launch_split<EPI, TO, 2, 2, 2>(M, N, K, g, e, s);
    case SPLIT42: return launch_split<EPI, TO, 4, 2, 1>(M, N, K, g, e, s);
    case ANY: return launch_any<EPI, TO>(M, N, K, g, e, s);
    case FEW11: return launch_few<EPI, TO, 1, 1, 8, 2>(M, N, K, g, e, s);
    case FEW21: return launch_few<EPI, TO, 2, 1, 8, 2>(M, N, K, g, e, s);
    case FEW22: return launch_few<EPI, TO, 2, 2, 8, 2>(M, N, K, g, e, s);
    case FEW42: return launch_few<EPI, TO, 4, 2, 6, 2>(M, N, K, g, e, s);
    case RING_256x256: return launch_ring<EPI, TO, 8, 4, 2>(M, N, K, g, e, s);
    case RING_128x256: return launch_ring<EPI, TO, 4, 4, 3>(M, N, K, g, e, s);
    case RING_128x128: return launch_ring<EPI, TO, 4, 2, 3>(M, N, K, g, e, s);
    case RING_128x128_TWO: return launch_ring<EPI, TO, 4, 2, 2>(M, N, K, g, e, s);
    case RING_96x128: return launch_ring<EPI, TO, 3, 2, 3>(M, N, K, g, e, s);
    case RING_64x128: return launch_ring<EPI, TO, 2, 2, 3>(M, N, K, g, e, s);
    case MIX:
      return p.wta == 8   ? launch_mix<EPI, TO, 8>(M, N, K, g, e, s, p)
             : p.wta == 7 ? launch_mix<EPI, TO, 7>(M, N, K, g, e, s, p)
                          : launch_mix<EPI, TO, 6>(M, N, K, g, e, s, p);
  }
  return hipErrorInvalidValue;
}

template <int EPI, typename TO>
hipError_t launch_epi(int M, int N, int K, const I8Args &g, const EpiArgs &e, hipStream_t s) {
  const int most = rows_per_launch(N);
  for (int64_t m = 0; m < M; m += most) {
    I8Args p = g;
    p.A += m * K;
    p.a_scale += m;
    EpiArgs r = e;
    const size_t es = EPI == EPI_STORE || EPI == EPI_GELU ? sizeof(TO) : sizeof(float);
    r.out = (char *)e.out + (size_t)m * e.ldo * es;
    if (r.res_in) r.res_in += m * e.ldo;
    if (r.cache) r.cache += m * e.ldo;
    const hipError_t err = launch_rows<EPI, TO>((int)std::min<int64_t>(M - m, most), N, K, p, r, s);
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
