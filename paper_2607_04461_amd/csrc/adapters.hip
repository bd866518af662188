// Low-rank adapters of many requests beside a shared projection, and their gradient.  Rows come in groups (a request's
// tokens, `per` of them), each group with an adapter a of its own or none:
//   u = x down_a^T,   out = base + gate s_a u up_a^T
//   du = s_a dy up_a,   dx = base + du down_a,   d_down_a = sum_m du^T x,   d_up_a = s_a sum_m dy^T u
// A projection adds 2 r flops to each element it reads and writes, so all of it is bound by memory: by HBM for many rows (at
// r = 128 by the weights' way out of L2), by the latency of its launches for few.  The kernels carry both directions:
//   * k_both: a tile of rows of one adapter through both products.  x goes straight from memory to the matrix cores, every
//     eighth block of columns on each of eight waves, whose sums meet in LDS; u's tile stays there for the second product.
//     24960 rows, 1536 to 1536, rank 32, bf16: 59 us, 3.7 TB/s (as k_down and k_up 75, most of it rows in 64-byte pieces).
//   * k_down, k_up: the same in two launches, for few rows on large weights, whose ranks and columns then go to many
//     workgroups.
//   * k_outer: the sum over rows of an outer product, both operands through LDS, the activations' columns by transposing
//     reads: 39 us for both gradients of the case above, x and dy at 3.9 TB/s.  Rows reach it through lists sorted by
//     adapter, in chunks; k_outer_sum adds the chunks' sums in order.
//   * k_prepare: those lists, and up and down the other way round for the gradient's two products.
// u and du are fp32 and stay so: next to bf16 weights each is split into bf16 parts that are multiplied one by one, three
// where the result is fp32 (24 bits) and two where it is bf16 (16 bits of it, against the 8 that are kept).
#include <algorithm>

#include "fragments.h"
#include "kernels.h"

namespace fb {
namespace {

__device__ __forceinline__ int adapter_of(const int32_t *index, int64_t group, int count) {
  const int a = index ? index[group] : 0;
  return a >= 0 && a < count ? a : -1;
}

// what rounding v to `part` left; nothing where v was not finite or rounded to infinity
__device__ __forceinline__ float rest(float v, float part) {
  const float r = v - part;
  return fabsf(r) <= fabsf(v) ? r : 0.f;
}

// parts of v: v ~ p[0] + p[1] + ...
template <typename T, int P>
__device__ __forceinline__ void split(f32x8 v, Frag<T> (&p)[P]) {
#pragma unroll
  for (int k = 0; k < P; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[k][i] = from_f32<T>(v[i]);
      v[i] = rest(v[i], to_f32(p[k][i]));
    }
}

// Rows of a workgroup, all of one adapter (-1: none): [row0, row0 + rows) of one group, or those in a list in LDS.
struct Tile {
  int64_t row0;
  const int *list;
  int rows, ad;
  __device__ __forceinline__ int64_t row(int i) const { return list ? list[i] : row0 + i; }
};
__device__ __forceinline__ Tile group_tile(int64_t id, int size, int64_t M, int per, const int32_t *index, int count) {
  const int tiles = (per + size - 1) / size;
  const int64_t group = id / tiles, from = (id % tiles) * size;
  Tile t;
  t.row0 = group * per + from;
  t.list = nullptr;
  t.rows = (int)max((int64_t)0, min(min((int64_t)size, per - from), M - t.row0));
  t.ad = t.rows > 0 ? adapter_of(index, group, count) : -1;
  return t;
}
// Rows 16 j .. 16 j + 15 of those with adapter id % (count + 1), the last of which is none, j = id / (count + 1): where groups
// are shorter than a tile, so that the rows of an adapter share a reading of its weights.  Each workgroup searches the index.
__device__ __forceinline__ Tile gathered_tile(int id, int64_t M, int per, const int32_t *index, int count, int *s_list, int *s_wave) {
  const int me = id % (count + 1), from = id / (count + 1) * 16, lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int waves = blockDim.x >> 6, rows = (int)M;
  int seen = 0;
  for (int m0 = 0; m0 < rows && seen < from + 16; m0 += blockDim.x) {
    const int m = m0 + threadIdx.x, ad = m < rows ? adapter_of(index, m / per, count) : -2;
    const bool match = ad == (me == count ? -1 : me);
    const uint64_t votes = __ballot(match);
    if (lane == 0) s_wave[w] = __popcll(votes);
    __syncthreads();
    int slot = seen + __popcll(votes & ((1ull << lane) - 1)) - from;
    for (int i = 0; i < waves; ++i) {
      if (i < w) slot += s_wave[i];
      seen += s_wave[i];
    }
    if (match && slot >= 0 && slot < 16) s_list[slot] = m;
    __syncthreads();
  }
  Tile t;
  t.row0 = 0;
  t.list = s_list;
  t.rows = max(0, min(16, seen - from));
  t.ad = me == count ? -1 : me;
  return t;
}
template <int SIZE, bool GATHER>
__device__ __forceinline__ Tile tile_of(int64_t id, int64_t M, int per, const int32_t *index, int count) {
  if constexpr (GATHER) {
    __shared__ int s_list[16], s_wave[8];
    return gathered_tile((int)id, M, per, index, count, s_list, s_wave);
  } else {
    return group_tile(id, SIZE, M, per, index, count);
  }
}

struct DownArgs {
  int64_t M;
  int per, K, rank, count;
  const void *x, *w;            // [M][K], [count][rank][K]
  const int32_t *index;
  const float *scales;          // [count] or null
  float *u;                     // [M][rank]
};

constexpr int WAVES = 8;        // each sums every eighth block of columns; their shares are added in order

// The waves' shares of x down^T for a tile's rows, to s_part [WAVES][MT RT][256]; a barrier must follow.
template <typename T, int MT, int RT>
__device__ __forceinline__ void down_shares(const DownArgs &a, const Tile &t, int rank0, float *s_part) {
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  f32x4 acc[MT][RT];
  const T *xr[MT], *wr[RT];
#pragma unroll
  for (int i = 0; i < MT; ++i) xr[i] = (const T *)a.x + t.row(min(16 * i + li, t.rows - 1)) * a.K;
#pragma unroll
  for (int j = 0; j < RT; ++j) wr[j] = (const T *)a.w + ((int64_t)t.ad * a.rank + min(rank0 + 16 * j + li, a.rank - 1)) * a.K;
  constexpr int SUB = 4 / sizeof(T), BLOCK = 32 * SUB;       // a wave takes whole lines of 128 bytes
  // blocks in flight: as many as their registers allow, since the few rows of a small tile wait on nothing else
  constexpr int DEPTH = MT == 1 && RT * sizeof(T) <= 4 ? 4 : 2;
  Frag<T> xf[DEPTH][SUB][MT], wf[DEPTH][SUB][RT];
  auto load = [&](int b, int block) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < SUB; ++c) {
      const int k = BLOCK * block + 32 * c + 8 * g;
      const bool in = k < a.K;      // K % 8 == 0
#pragma unroll
      for (int i = 0; i < MT; ++i) xf[b][c][i] = in ? load_frag(xr[i] + k) : zero_frag<T>();
#pragma unroll
      for (int j = 0; j < RT; ++j) wf[b][c][j] = in ? load_frag(wr[j] + k) : zero_frag<T>();
    }
  };
  auto multiply = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < SUB; ++c)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[i][j] = mma(xf[b][c][i], wf[b][c][j], acc[i][j]);
  };
  const int blocks = (a.K + BLOCK - 1) / BLOCK;
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (w + d * WAVES < blocks) load(d, w + d * WAVES);
  for (int s0 = w; s0 < blocks; s0 += DEPTH * WAVES) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int s = s0 + d * WAVES;
      if (s < blocks) {
        multiply(d);
        if (s + DEPTH * WAVES < blocks) load(d, s + DEPTH * WAVES);
      }
    }
  }
  // element (row 4 g + e, rank li) of tile (i, j)
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) s_part[(w * MT * RT + i * RT + j) * 256 + (4 * g + e) * 16 + li] = acc[i][j][e];
}
// Element p of [MT RT][256] out of the shares, in order: row and rank of it, and its sum
template <int MT, int RT>
__device__ __forceinline__ float down_sum(const float *s_part, int p, int &row, int &r) {
  float v = 0.f;
#pragma unroll
  for (int k = 0; k < WAVES; ++k) v += s_part[k * MT * RT * 256 + p];
  row = p / (RT * 256) * 16 + (p & 255) / 16;
  r = p / 256 % RT * 16 + (p & 15);
  return v;
}

template <typename T, int MT, int RT, bool GATHER>
__global__ __launch_bounds__(64 * WAVES) void k_down(DownArgs a) {
  extern __shared__ __attribute__((aligned(16))) float s_part[];
  const Tile t = tile_of<16 * MT, GATHER>(blockIdx.x, a.M, a.per, a.index, a.count);
  if (t.rows <= 0) return;
  const int rank0 = blockIdx.y * 16 * RT, ranks = min(16 * RT, a.rank - rank0);
  if (t.ad < 0) {
    for (int i = threadIdx.x; i < t.rows * ranks; i += 64 * WAVES) a.u[t.row(i / ranks) * a.rank + rank0 + i % ranks] = 0.f;
    return;
  }
  down_shares<T, MT, RT>(a, t, rank0, s_part);
  __syncthreads();
  const float scale = a.scales ? a.scales[t.ad] : 1.f;
  for (int p = threadIdx.x; p < MT * RT * 256; p += 64 * WAVES) {
    int row, r;
    const float v = down_sum<MT, RT>(s_part, p, row, r) * scale;
    if (row < t.rows && r < ranks) a.u[t.row(row) * a.rank + rank0 + r] = v;
  }
}

struct UpArgs {
  int64_t M;
  int per, N, rank, count, cols, parts;      // cols: columns of a workgroup, whole turns; workgroups a row
  const float *u;                     // [M][rank]
  const void *w;                      // [count][N][rank]
  const int32_t *index;
  const float *scales, *gate;         // [count], [N] or null
  const void *base;                   // [M][N] of the output's type, or null: zeros
  void *out;
};

template <typename T, typename O> constexpr int PARTS = sizeof(T) == 4 ? 1 : sizeof(O) == 4 ? 3 : 2;

// out = base + f u up^T for a tile's rows and the columns [from, to), 256 bytes of a row a turn from wave `first` of `waves` on.
// u(i, c, p): part p of u, row li of sixteen i, ranks 32 c + 8 g and on.  The products cross s_out, which only this wave uses, so that base and out pass
// as 256 bytes of four rows at a time: in the products' own layout, 64 bytes of sixteen, 24960 x 1536 took 50 us for 38.
template <typename O> constexpr int TURN = 256 / sizeof(O);
template <typename O> constexpr int OUT_PITCH = TURN<O> + 4;
template <typename O> constexpr size_t OUT_BYTES = 16 * OUT_PITCH<O> * 4;      // of a wave
template <typename T, typename O, int MT, int RK, typename U>
__device__ __forceinline__ void up_columns(const UpArgs &a, const Tile &t, const U &u, float *s_out, int from, int to, int first, int waves) {
  constexpr int E = 16 / sizeof(O), Q = TURN<O> / 32;        // elements of a lane's piece; groups of 32 columns
  typedef O Piece __attribute__((ext_vector_type(E)));
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4;
  const int ad = t.ad;
  const float scale = ad < 0 ? 0.f : a.scales ? a.scales[ad] : 1.f;
  const T *W = (const T *)a.w + (int64_t)max(ad, 0) * a.N * a.rank;
  // column of row li of tile h: four of each eight
  const int col = 8 * (li >> 2) + (li & 3);
  for (int n0 = from + TURN<O> * first; n0 < to; n0 += TURN<O> * waves) {
    const int n = n0 + E * li;                               // this lane's columns of rows 4 x + g; N % 8 == 0
    Piece b[MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int row = 16 * i + 4 * x + g;
        if (a.base && n < to && row < t.rows) b[i][x] = *reinterpret_cast<const Piece *>((const O *)a.base + t.row(row) * a.N + n);
        else b[i][x] = (Piece)((O)0.f);
      }
    Frag<T> wf[Q][2][RK];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < RK; ++c) {
          const int r = 32 * c + 8 * g;
          wf[q][h][c] = r < a.rank && ad >= 0 ? load_frag(W + (int64_t)min(n0 + 32 * q + col + 4 * h, a.N - 1) * a.rank + r) : zero_frag<T>();
        }
    float f[E];
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = a.gate && n < to ? scale * a.gate[n + e] : scale;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      if (ad >= 0) {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int p = PARTS<T, O> - 1; p >= 0; --p)     // the small parts first
#pragma unroll
            for (int c = 0; c < RK; ++c) {
              const Frag<T> uf = u(i, c, p);
#pragma unroll
              for (int h = 0; h < 2; ++h) acc[h] = mma(wf[q][h][c], uf, acc[h]);
            }
#pragma unroll
          for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4 *>(s_out + li * OUT_PITCH<O> + 32 * q + 8 * g + 4 * h) = acc[h];
        }
        own_lds();
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int row = 16 * i + 4 * x + g;
        Piece o = b[i][x];
        if (ad >= 0) {
#pragma unroll
          for (int y = 0; y < E / 4; ++y) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(s_out + (4 * x + g) * OUT_PITCH<O> + E * li + 4 * y);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[4 * y + e] = from_f32<O>(fmaf(f[4 * y + e], v[e], to_f32(o[4 * y + e])));
          }
        }
        if (n < to && row < t.rows) *reinterpret_cast<Piece *>((O *)a.out + t.row(row) * a.N + n) = o;
      }
      own_lds();
    }
  }
}

// Two waves a SIMD (919 rows, 1536 to 8960, rank 128, bf16 with an fp32 result: the call 38 us, without asking 41), but for 32
// rows of 128 ranks, which would spill (24960 rows, 1536 to 1536, fp32: 452 us for 432).
template <typename T, typename O, int MT, int RK, bool GATHER>
__global__ __launch_bounds__(256, MT * RK < 8 ? 2 : 1) void k_up(UpArgs a) {
  extern __shared__ __attribute__((aligned(16))) float s_part[];
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Tile t = tile_of<16 * MT, GATHER>(blockIdx.x / a.parts, a.M, a.per, a.index, a.count);      // a row's workgroups follow each other
  if (t.rows <= 0 || (t.ad < 0 && a.base == a.out)) return;
  Frag<T> uf[MT][RK][PARTS<T, O>];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int c = 0; c < RK; ++c) {
      const int r = 32 * c + 8 * g;
      split<T, PARTS<T, O>>(r < a.rank ? load_frag(a.u + t.row(min(16 * i + li, t.rows - 1)) * a.rank + r) : zero_frag<float>(), uf[i][c]);
    }
  const int from = blockIdx.x % a.parts * a.cols;
  auto u = [&](int i, int c, int p) __attribute__((always_inline)) { return uf[i][c][p]; };
  up_columns<T, O, MT, RK>(a, t, u, s_part + w * (OUT_BYTES<O> / 4), from, min(from + a.cols, a.N), w, 4);
}

// Whether u's parts stay in LDS for the second product: 32 rows of 128 ranks leave no registers for them beside the weights'.
// 24960 rows, rank 128, bf16: 8960 to 1536 435 us and 1536 to 8960 462; with the parts in registers 487 and 659 (spilled), in
// tiles of 16 rows 650 and 638.
template <int MT, int RT> constexpr bool LDS_PARTS = MT * RT > 8;
constexpr int PART_PITCH = 128 + 8;
template <typename T, typename O, int MT, int RT> constexpr size_t u_bytes() {
  return LDS_PARTS<MT, RT> ? PARTS<T, O> * 16 * MT * PART_PITCH * sizeof(T) : 16 * MT * ((RT < 2 ? 32 : 16 * RT) + 4) * 4;
}
template <typename T, typename O, int MT, int RT> constexpr size_t both_lds() {
  const size_t shares = WAVES * MT * RT * 1024, outs = WAVES * OUT_BYTES<O>;
  return (shares > outs ? shares : outs) + u_bytes<T, O, MT, RT>();
}

// Both in one launch: u's tile stays in LDS.  d.u, its scales and the sums' order as in k_down, so the bits are the same.
template <typename T, typename O, int MT, int RT, bool GATHER>
__global__ __launch_bounds__(64 * WAVES) void k_both(DownArgs d, UpArgs a) {
  constexpr int RK = RT < 2 ? 1 : RT / 2, PITCH = 32 * RK + 4;
  extern __shared__ __attribute__((aligned(16))) float s_part[];
  // u's tile [16 MT][PITCH], zero past the rank, behind the larger of the shares and the waves' products
  float *su = s_part + (both_lds<T, O, MT, RT>() - u_bytes<T, O, MT, RT>()) / 4;
  T *sp = reinterpret_cast<T *>(su);       // or its parts [PARTS][16 MT][PART_PITCH]
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4;
  const Tile t = tile_of<16 * MT, GATHER>(blockIdx.x, a.M, a.per, a.index, a.count);
  if (t.rows <= 0) return;
  const int ad = t.ad;
  constexpr bool LDS = LDS_PARTS<MT, RT>;
  Frag<T> uf[LDS ? 1 : MT][RK][PARTS<T, O>];
  if (ad < 0) {
    for (int i = threadIdx.x; i < t.rows * a.rank; i += 64 * WAVES) d.u[t.row(i / a.rank) * a.rank + i % a.rank] = 0.f;
    if (a.base == a.out) return;
#pragma unroll
    for (int i = 0; i < (LDS ? 1 : MT); ++i)
#pragma unroll
      for (int c = 0; c < RK; ++c)
#pragma unroll
        for (int p = 0; p < PARTS<T, O>; ++p) uf[i][c][p] = zero_frag<T>();
  } else {
    down_shares<T, MT, RT>(d, t, 0, s_part);
    __syncthreads();
    const float scale = d.scales ? d.scales[ad] : 1.f;
    for (int p = threadIdx.x; p < MT * RT * 256; p += 64 * WAVES) {
      int row, r;
      const float v = down_sum<MT, RT>(s_part, p, row, r) * scale;
      if (row < t.rows && r < a.rank) d.u[t.row(row) * a.rank + r] = v;
      if constexpr (LDS) {
        float left = r < a.rank ? v : 0.f;
#pragma unroll
        for (int k = 0; k < PARTS<T, O>; ++k) {
          const T part = from_f32<T>(left);
          sp[(k * 16 * MT + row) * PART_PITCH + r] = part;
          left = rest(left, to_f32(part));
        }
      } else {
        su[row * PITCH + r] = r < a.rank ? v : 0.f;
        if (RT == 1) su[row * PITCH + r + 16] = 0.f;
      }
    }
    __syncthreads();
    if constexpr (!LDS) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < RK; ++c) split<T, PARTS<T, O>>(load_frag(su + (16 * i + li) * PITCH + 32 * c + 8 * g), uf[i][c]);
    }
  }
  // u's tile has been read; the shares' place serves the products
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto u = [&](int i, int c, int p) __attribute__((always_inline)) {
    if constexpr (LDS) return load_frag(sp + (p * 16 * MT + 16 * i + li) * PART_PITCH + 32 * c + 8 * g);
    else return uf[i][c][p];
  };
  up_columns<T, O, MT, RK>(a, t, u, s_part + w * (OUT_BYTES<O> / 4), 0, a.N, w, WAVES);
}

// What the gradient needs first, in one launch of [blocks][2 count + count]: the transposed weights, out[z][c][r] =
// in[z][r][c] for `count` matrices of each of two shapes, and the lists of rows (k_prepare's last planes).
struct PrepareArgs {
  const void *in[2];
  void *out[2];
  int rows[2], cols[2], count;
  int64_t M;
  int per, chunk, chunks;
  const int32_t *index;
  int32_t *list, *chunk_adapter, *first;     // null: no lists
};

// The rows of adapter `me`, in order, as a list that starts at a multiple of `chunk` and is filled up with -1:
// `list`; chunk_adapter[c]: the adapter of a chunk, -1 past the last; first[a], first[count + a]: an adapter's chunks.
// Workgroup `slice` of `slices` writes its share of the list.  The counts are integers, so the order of their additions
// changes nothing.
__device__ __forceinline__ void list_rows(const PrepareArgs &a, int me, int slice, int slices) {
  __shared__ int s_rows[1024], s_group[256], s_wave[4], s_sum[2];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, M = (int)a.M, groups = (M + a.per - 1) / a.per;
  for (int i = tid; i < 1024; i += 256) s_rows[i] = 0;
  if (tid < 2) s_sum[tid] = 0;
  __syncthreads();
  for (int i = tid; i < groups; i += 256) {
    const int ad = adapter_of(a.index, i, a.count);
    if (ad >= 0) atomicAdd(&s_rows[ad], min(a.per, M - i * a.per));
  }
  __syncthreads();
  for (int i = tid; i < a.count; i += 256) {
    const int n = (s_rows[i] + a.chunk - 1) / a.chunk;
    if (n && i < me) atomicAdd(&s_sum[0], n);
    if (n) atomicAdd(&s_sum[1], n);
  }
  __syncthreads();
  const int before = s_sum[0], total = s_sum[1], mine = s_rows[me], own = (mine + a.chunk - 1) / a.chunk;
  if (slice == 0) {
    if (tid == 0) {
      a.first[me] = before;
      a.first[a.count + me] = own;
    }
    for (int i = tid; i < own; i += 256) a.chunk_adapter[before + i] = me;
    if (me == 0)
      for (int i = total + tid; i < a.chunks; i += 256) a.chunk_adapter[i] = -1;
  }
  int32_t *at = a.list + (int64_t)before * a.chunk;
  if (slice == 0)
    for (int i = mine + tid; i < own * a.chunk; i += 256) at[i] = -1;
  for (int g0 = 0; g0 < groups; g0 += 256) {
    const bool match = g0 + tid < groups && adapter_of(a.index, g0 + tid, a.count) == me;
    const uint64_t votes = __ballot(match);
    if (lane == 0) s_wave[w] = __popcll(votes);
    __syncthreads();
    int slot = __popcll(votes & ((1ull << lane) - 1)), all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i < w) slot += s_wave[i];
      all += s_wave[i];
    }
    if (match) s_group[slot] = g0 + tid;
    __syncthreads();
    // every group but the last of all is whole, so an adapter's rows are dense; fewer than M + per of them
    const uint32_t items = (uint32_t)all * a.per;
    for (uint32_t i = slice * 256 + tid; i < items; i += slices * 256) {
      const uint32_t k = i / (uint32_t)a.per, row = (uint32_t)s_group[k] * a.per + (i - k * a.per);
      if (row < (uint32_t)M) at[i] = (int32_t)row;
    }
    at += items;
    __syncthreads();
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_prepare(PrepareArgs a) {
  __shared__ T s[32][33];
  if ((int)blockIdx.y >= 2 * a.count) {
    const int slices = min((int)gridDim.x, 16);
    if (a.list && (int)blockIdx.x < slices) list_rows(a, blockIdx.y - 2 * a.count, blockIdx.x, slices);
    return;
  }
  const int job = (int)blockIdx.y >= a.count, z = blockIdx.y - job * a.count;
  const int rows = a.rows[job], cols = a.cols[job], tc = (cols + 31) / 32;
  if ((int64_t)blockIdx.x >= (int64_t)tc * ((rows + 31) / 32)) return;
  const int r0 = blockIdx.x / tc * 32, c0 = blockIdx.x % tc * 32, x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const T *in = (const T *)a.in[job] + (int64_t)z * rows * cols;
  T *out = (T *)a.out[job] + (int64_t)z * rows * cols;
  for (int i = y; i < 32; i += 8)
    if (r0 + i < rows && c0 + x < cols) s[i][x] = in[(int64_t)(r0 + i) * cols + c0 + x];
  __syncthreads();
  for (int i = y; i < 32; i += 8)
    if (c0 + i < cols && r0 + x < rows) out[(int64_t)(c0 + i) * rows + r0 + x] = s[x][i];
}

struct OuterArgs {
  int rank, chunk;
  int cols[2];                        // K and N
  const void *x[2];                   // x [M][K] and dy [M][N]
  const float *u[2];                  // du and u [M][rank]
  const int32_t *list, *chunk_adapter;
  float *partial;                     // [chunks][rank K + N rank]: d_down as [rank][K], then d_up as [N][rank]
};

constexpr int OUTER_COLS = 256, OUTER_CHUNK = 1024;   // columns of a workgroup; most rows of a chunk

template <typename T, int RT>
__global__ __launch_bounds__(256, 2) void k_outer(OuterArgs a) {
  constexpr int PARTS = sizeof(T) == 4 ? 1 : 3;
  constexpr int XP = OUTER_COLS + 16 / sizeof(T), UP = 32 + 16 / sizeof(T);   // pitches, elements
  constexpr int PIECE = 16 / sizeof(T);                                       // elements of a 16-byte load
  // u's rows go to LDS the other way round, two rows of a rank a write and sixteen lanes beside each other, so that a write
  // meets no bank twice (a row of u across the lanes: 24960 rows, 1536 to 1536, rank 128, bf16: the call 407 us for 330)
  typedef T Two __attribute__((ext_vector_type(2)));
  constexpr int XN = 32 * OUTER_COLS / PIECE / 256, UN = (64 * RT + 255) / 256;
  extern __shared__ __attribute__((aligned(16))) char s_mem[];
  T *sx = reinterpret_cast<T *>(s_mem), *su = sx + 32 * XP;                   // [32][XP], [PARTS][16 RT][UP]
  int32_t *rows = reinterpret_cast<int32_t *>(su + PARTS * 16 * RT * UP);     // [chunk]
  const int chunk = blockIdx.y;
  if (a.chunk_adapter[chunk] < 0) return;
  const int blocks0 = (a.cols[0] + OUTER_COLS - 1) / OUTER_COLS;
  const int job = (int)blockIdx.x >= blocks0, c0 = ((int)blockIdx.x - job * blocks0) * OUTER_COLS, C = a.cols[job];
  const T *X = (const T *)a.x[job];
  const float *U = a.u[job];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, g = lane >> 4, w = tid >> 6;
  for (int i = tid; i < a.chunk; i += 256) rows[i] = a.list[(int64_t)chunk * a.chunk + i];
  __syncthreads();
  int steps = a.chunk / 32;
  while (steps > 1 && rows[32 * (steps - 1)] < 0) --steps;     // lists end within a chunk
  u32x4 xv[XN];
  f32x4 uv[UN][2];
  auto load = [&](int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < XN; ++i) {
      const int p = tid + 256 * i, m = rows[32 * s + p / (OUTER_COLS / PIECE)], c = c0 + p % (OUTER_COLS / PIECE) * PIECE;
      xv[i] = m >= 0 && c < C ? *reinterpret_cast<const u32x4 *>(X + (int64_t)m * C + c) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int p = tid + 256 * i, r = 4 * (p / 16);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int m = r < a.rank ? rows[32 * s + 2 * (p % 16) + y] : -1;
        uv[i][y] = m >= 0 ? *reinterpret_cast<const f32x4 *>(U + (int64_t)m * a.rank + r) : f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
  };
  auto land = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < XN; ++i) {
      const int p = tid + 256 * i;
      *reinterpret_cast<u32x4 *>(sx + p / (OUTER_COLS / PIECE) * XP + p % (OUTER_COLS / PIECE) * PIECE) = xv[i];
    }
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int p = tid + 256 * i, m = 2 * (p % 16), r = 4 * (p / 16);
      if (p >= 64 * RT) break;
#pragma unroll
      for (int k = 0; k < PARTS; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const Two v = {from_f32<T>(uv[i][0][e]), from_f32<T>(uv[i][1][e])};
          *reinterpret_cast<Two *>(su + (k * 16 * RT + r + e) * UP + m) = v;
#pragma unroll
          for (int y = 0; y < 2; ++y) uv[i][y][e] = rest(uv[i][y][e], to_f32(v[y]));
        }
    }
  };
  f32x4 acc[4][RT];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  load(0);
  for (int s = 0; s < steps; ++s) {
    __syncthreads();          // the last step's tiles have been read
    land();
    __syncthreads();
    if (s + 1 < steps) load(s + 1);
    Frag<T> xf[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) xf[i] = load_column_frag(sx, XP, 64 * w + 16 * i, 8 * g, 8 * g + 4);
#pragma unroll
    for (int k = PARTS - 1; k >= 0; --k)
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        const Frag<T> uf = load_frag(su + (k * 16 * RT + 16 * j + li) * UP + 8 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][j] = mma(xf[i], uf, acc[i][j]);
      }
  }
  float *out = a.partial + (int64_t)chunk * a.rank * ((int64_t)a.cols[0] + a.cols[1]) + (job ? (int64_t)a.rank * a.cols[0] : 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = c0 + 64 * w + 16 * i + 4 * g;      // C % 8 == 0: all four or none
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const int r = 16 * j + li;
      if (c >= C || r >= a.rank) continue;
      if (job) {
#pragma unroll
        for (int e = 0; e < 4; ++e) out[(int64_t)(c + e) * a.rank + r] = acc[i][j][e];
      } else {
        *reinterpret_cast<f32x4 *>(out + (int64_t)r * C + c) = acc[i][j];
      }
    }
  }
}

// An adapter's gradients out of its chunks' sums: 64 lanes of four elements, every fourth chunk to each of four waves, whose
// sums are added in order.
__global__ __launch_bounds__(256) void k_outer_sum(int count, int64_t down, int64_t up, const int32_t *first, const float *scales,
                                                   const float *partial, float *d_down, float *d_up) {
  __shared__ double s_part[3][64][4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t e = ((int64_t)blockIdx.x * 64 + lane) * 4, all = down + up;      // multiples of eight
  for (int a = blockIdx.y; a < count; a += gridDim.y) {
    const int n = first[count + a];
    const float *p = partial + first[a] * all + e;
    double s[4] = {0, 0, 0, 0};
    if (e < all) {
#pragma unroll 4
      for (int c = w; c < n; c += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(p + c * all);
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] += (double)v[k];
      }
    }
    if (w)
#pragma unroll
      for (int k = 0; k < 4; ++k) s_part[w - 1][lane][k] = s[k];
    __syncthreads();
    if (w == 0 && e < all) {
      const double scale = e < down || !scales || n == 0 ? 1.0 : (double)scales[a];      // 0 without rows, whatever the scale
      f32x4 v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = (float)((((s[k] + s_part[0][lane][k]) + s_part[1][lane][k]) + s_part[2][lane][k]) * scale);
      float *dst = e < down ? d_down : d_up;
      if (dst) *reinterpret_cast<f32x4 *>(dst + (e < down ? a * down + e : a * up + e - down)) = v;
    }
    __syncthreads();
  }
}

// Rows of a tile: as many as leave a tile a CU at least, and no more than a group has.  More rows read the weights less often,
// fewer leave more workgroups in flight: 24960 x 1536 x 1536, rank 32, both products 69 us on 32 rows, 71 on 64, 78 on 16.
int tile_rows(int64_t M, int per, int most) {
  int mt = most;
  while (mt > 1 && (16 * (mt / 2) >= per || (M + 16 * mt - 1) / (16 * mt) < 256)) mt /= 2;
  return mt;
}
int64_t tiles_of(int64_t M, int per, int rows) { return (M + per - 1) / per * ((per + rows - 1) / rows); }

// Whether rows are gathered by their adapters: groups shorter than a tile, where that takes not many more workgroups and the
// search of the index stays short.  254 fp32 rows of 11 adapters, rank 128, 13824 to 5120: 118 us, in a tile a row 386.
bool gathers(int64_t M, int per, int count) {
  return per < 16 && M <= 8192 && (M + 15) / 16 * (count + 1) <= 2 * ((M + per - 1) / per);
}
template <bool GATHER> int64_t tiles_for(int64_t M, int per, int count, int rows) {
  return GATHER ? (M + 15) / 16 * (count + 1) : tiles_of(M, per, rows);
}

template <typename T, int MT, int RT, bool GATHER = false>
hipError_t down_tile(const DownArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((k_down<T, MT, RT, GATHER>), dim3((unsigned)tiles_for<GATHER>(a.M, a.per, a.count, 16 * MT), (a.rank + 16 * RT - 1) / (16 * RT)),
                     dim3(64 * WAVES), WAVES * MT * RT * 1024, s, a);
  return hipGetLastError();
}
// The waves' sums take MT RT 8 KB of LDS: 64 KB at most, two workgroups a CU.  Few tiles share the ranks among workgroups:
// two rows, 64 ranks of 8960 to 1536, took 41 us on one CU each and take 18.
template <typename T>
hipError_t launch_down(const DownArgs &a, hipStream_t s) {
  if (gathers(a.M, a.per, a.count)) return down_tile<T, 1, 1, true>(a, s);
  const int mt = tile_rows(a.M, a.per, 4);
  if (mt == 1 && tiles_of(a.M, a.per, 16) < 256) return down_tile<T, 1, 1>(a, s);
  if (a.rank <= 16) return mt == 4 ? down_tile<T, 4, 1>(a, s) : mt == 2 ? down_tile<T, 2, 1>(a, s) : down_tile<T, 1, 1>(a, s);
  if (a.rank <= 32) return mt == 4 ? down_tile<T, 4, 2>(a, s) : mt == 2 ? down_tile<T, 2, 2>(a, s) : down_tile<T, 1, 2>(a, s);
  if (a.rank <= 64) return mt >= 2 ? down_tile<T, 2, 4>(a, s) : down_tile<T, 1, 4>(a, s);
  return down_tile<T, 1, 8>(a, s);
}

template <typename T, typename O, int MT, int RK, bool GATHER = false>
hipError_t up_tile(UpArgs a, hipStream_t s) {
  const int64_t tiles = tiles_for<GATHER>(a.M, a.per, a.count, 16 * MT);
  // columns of a workgroup: enough workgroups for eight a CU, a turn of its four waves at least
  constexpr int turn = 4 * TURN<O>;
  const int64_t turns = (a.N + turn - 1) / turn, parts = std::min<int64_t>(turns, std::max<int64_t>(1, 2048 / tiles));
  a.cols = (int)((turns + parts - 1) / parts * turn);
  a.parts = (a.N + a.cols - 1) / a.cols;
  hipLaunchKernelGGL((k_up<T, O, MT, RK, GATHER>), dim3((unsigned)(tiles * a.parts)), dim3(256), 4 * OUT_BYTES<O>, s, a);
  return hipGetLastError();
}
template <typename T, typename O>
hipError_t launch_up(const UpArgs &a, hipStream_t s) {
  if (gathers(a.M, a.per, a.count))
    return a.rank <= 32 ? up_tile<T, O, 1, 1, true>(a, s) : a.rank <= 64 ? up_tile<T, O, 1, 2, true>(a, s) : up_tile<T, O, 1, 4, true>(a, s);
  // As many rows as 256 tiles come here in fp32 of rank above 64 alone (launch_both), fewer have tiles of 16.
  if (a.rank <= 32) return up_tile<T, O, 1, 1>(a, s);
  if (a.rank <= 64) return up_tile<T, O, 1, 2>(a, s);
  if constexpr (sizeof(T) == 4)
    if (tile_rows(a.M, a.per, 2) == 2) return up_tile<T, O, 2, 4>(a, s);
  return up_tile<T, O, 1, 4>(a, s);
}

template <typename T, typename O, int MT, int RT, bool GATHER = false>
hipError_t both_tile(const DownArgs &d, const UpArgs &a, hipStream_t s) {
  constexpr size_t lds = both_lds<T, O, MT, RT>();
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute((const void *)k_both<T, O, MT, RT, GATHER>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_both<T, O, MT, RT, GATHER>), dim3((unsigned)tiles_for<GATHER>(a.M, a.per, a.count, 16 * MT)), dim3(64 * WAVES), lds, s, d, a);
  return hipGetLastError();
}

// u = d.scales x down^T, then out = base + a.gate a.scales u up^T.  In one launch where the rows fill the card, or the weights
// are so small that one CU passes them in the time of a second launch; else the columns and ranks of few rows go to several
// workgroups.
template <typename T, typename O>
hipError_t launch_both(const DownArgs &d, const UpArgs &a, hipStream_t s) {
  const bool wide = sizeof(T) == 4 && a.rank > 32;       // fp32 operands of many ranks: no registers for two tiles of rows
  const int mt = tile_rows(a.M, a.per, wide ? 1 : 2);
  const bool gather = gathers(a.M, a.per, a.count), small = a.rank <= 32 && a.N <= 2048 && d.K <= 2048;
  if ((gather || tiles_of(a.M, a.per, 16 * mt) < 256 ? !small : false) || (sizeof(T) == 4 && a.rank > 64)) {
    const hipError_t e = launch_down<T>(d, s);
    return e != hipSuccess ? e : launch_up<T, O>(a, s);
  }
  if (gather) return a.rank <= 16 ? both_tile<T, O, 1, 1, true>(d, a, s) : both_tile<T, O, 1, 2, true>(d, a, s);
  if (a.rank <= 16) return mt == 2 ? both_tile<T, O, 2, 1>(d, a, s) : both_tile<T, O, 1, 1>(d, a, s);
  if (a.rank <= 32) return mt == 2 ? both_tile<T, O, 2, 2>(d, a, s) : both_tile<T, O, 1, 2>(d, a, s);
  if constexpr (sizeof(T) == 4) {
    return both_tile<T, O, 1, 4>(d, a, s);
  } else {
    if (a.rank <= 64) return mt == 2 ? both_tile<T, O, 2, 4>(d, a, s) : both_tile<T, O, 1, 4>(d, a, s);
    return mt == 2 ? both_tile<T, O, 2, 8>(d, a, s) : both_tile<T, O, 1, 8>(d, a, s);
  }
}

template <typename T, int RT>
hipError_t outer_rank(const OuterArgs &a, dim3 grid, hipStream_t s) {
  const size_t lds = (32 * (OUTER_COLS + 16 / sizeof(T)) + (sizeof(T) == 4 ? 1 : 3) * 16 * RT * (32 + 16 / sizeof(T))) * sizeof(T) +
                     a.chunk * 4;
  hipLaunchKernelGGL((k_outer<T, RT>), grid, dim3(256), lds, s, a);
  return hipGetLastError();
}

// Rows of a chunk: what gives the outer products about a thousand workgroups, in steps of 32
int outer_chunk(int64_t M, int N, int K) {
  const int64_t blocks = (N + OUTER_COLS - 1) / OUTER_COLS + (K + OUTER_COLS - 1) / OUTER_COLS;
  const int64_t rows = (M * blocks / 1024 + 31) / 32 * 32;
  return (int)std::min<int64_t>(OUTER_CHUNK, std::max<int64_t>(64, rows));
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// the gradient's workspace: parts in order, each on 256 bytes
struct GradSpace {
  int chunk;
  int64_t chunks;
  size_t up_t, down_t, du, list, chunk_adapter, first, partial, bytes;
  GradSpace(ActType t, const AdapterArgs &a) {
    const size_t es = t == ACT_BF16 ? 2 : 4;
    chunk = outer_chunk(a.M, a.N, a.K);
    const int64_t groups = (a.M + a.per - 1) / a.per;
    chunks = (a.M + chunk - 1) / chunk + std::min<int64_t>(a.count, groups);
    size_t at = 0;
    auto take = [&](size_t n) { const size_t p = at; at += up256(n); return p; };
    up_t = take((size_t)a.count * a.N * a.rank * es);
    down_t = take((size_t)a.count * a.K * a.rank * es);
    du = take((size_t)a.M * a.rank * 4);
    list = take((size_t)chunks * chunk * 4);
    chunk_adapter = take((size_t)chunks * 4);
    first = take((size_t)a.count * 8);
    partial = take((size_t)chunks * a.rank * ((size_t)a.N + a.K) * 4);
    bytes = at;
  }
};

template <typename T>
hipError_t adapters(const AdapterArgs &a, bool out_f32, hipStream_t s) {
  DownArgs d;
  d.M = a.M; d.per = a.per; d.K = a.K; d.rank = a.rank; d.count = a.count;
  d.x = a.x; d.w = a.down; d.index = a.index; d.scales = nullptr; d.u = a.u;
  UpArgs p;
  p.M = a.M; p.per = a.per; p.N = a.N; p.rank = a.rank; p.count = a.count; p.cols = p.parts = 0;
  p.u = a.u; p.w = a.up; p.index = a.index; p.scales = a.scales; p.gate = a.gate; p.base = a.base; p.out = a.out;
  return out_f32 ? launch_both<T, float>(d, p, s) : launch_both<T, T>(d, p, s);
}

template <typename T>
hipError_t adapters_grad(const AdapterArgs &a, const AdapterGradArgs &b, bool dx_f32, hipStream_t s) {
  const GradSpace g(sizeof(T) == 2 ? ACT_BF16 : ACT_F32, a);
  char *ws = (char *)b.workspace;
  float *du = (float *)(ws + g.du);
  int32_t *list = (int32_t *)(ws + g.list), *chunk_adapter = (int32_t *)(ws + g.chunk_adapter), *first = (int32_t *)(ws + g.first);
  PrepareArgs t;
  t.in[0] = a.up; t.out[0] = ws + g.up_t; t.rows[0] = a.N; t.cols[0] = a.rank;
  t.in[1] = a.down; t.out[1] = ws + g.down_t; t.rows[1] = a.rank; t.cols[1] = a.K;
  t.count = a.count; t.M = a.M; t.per = a.per; t.chunk = g.chunk; t.chunks = (int)g.chunks; t.index = a.index;
  t.list = b.d_down || b.d_up ? list : nullptr; t.chunk_adapter = chunk_adapter; t.first = first;
  const int across = std::max(a.N, a.K);
  hipLaunchKernelGGL((k_prepare<T>), dim3((across + 31) / 32 * ((a.rank + 31) / 32), 3 * a.count), dim3(256), 0, s, t);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  DownArgs d;
  d.M = a.M; d.per = a.per; d.K = a.N; d.rank = a.rank; d.count = a.count;
  d.x = b.dy; d.w = ws + g.up_t; d.index = a.index; d.scales = a.scales; d.u = du;
  if (!b.dx) {
    if ((e = launch_down<T>(d, s)) != hipSuccess) return e;
  } else {
    UpArgs p;
    p.M = a.M; p.per = a.per; p.N = a.K; p.rank = a.rank; p.count = a.count; p.cols = p.parts = 0;
    p.u = du; p.w = ws + g.down_t; p.index = a.index; p.scales = nullptr; p.gate = nullptr; p.base = b.base; p.out = b.dx;
    if ((e = dx_f32 ? launch_both<T, float>(d, p, s) : launch_both<T, T>(d, p, s)) != hipSuccess) return e;
  }
  if (!b.d_down && !b.d_up) return hipSuccess;
  OuterArgs o;
  o.rank = a.rank; o.chunk = g.chunk;
  o.cols[0] = a.K; o.cols[1] = a.N; o.x[0] = a.x; o.x[1] = b.dy; o.u[0] = du; o.u[1] = a.u;
  o.list = list; o.chunk_adapter = chunk_adapter; o.partial = (float *)(ws + g.partial);
  const dim3 grid((a.K + OUTER_COLS - 1) / OUTER_COLS + (a.N + OUTER_COLS - 1) / OUTER_COLS, (unsigned)g.chunks);
  e = a.rank <= 16 ? outer_rank<T, 1>(o, grid, s) : a.rank <= 32 ? outer_rank<T, 2>(o, grid, s)
      : a.rank <= 64 ? outer_rank<T, 4>(o, grid, s) : outer_rank<T, 8>(o, grid, s);
  if (e != hipSuccess) return e;
  const int64_t down = (int64_t)a.rank * a.K, up = (int64_t)a.rank * a.N;
  hipLaunchKernelGGL(k_outer_sum, dim3((unsigned)((down + up + 255) / 256), std::min(a.count, 65535)), dim3(256), 0, s, a.count, down, up, first,
                     a.scales, o.partial, b.d_down, b.d_up);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adapters(ActType t, const AdapterArgs &a, bool out_f32, hipStream_t s) {
  return t == ACT_BF16 ? adapters<bf16>(a, out_f32, s) : adapters<float>(a, out_f32, s);
}

size_t adapters_grad_workspace(ActType t, const AdapterArgs &a) { return GradSpace(t, a).bytes; }

hipError_t launch_adapters_grad(ActType t, const AdapterArgs &a, const AdapterGradArgs &b, bool dx_f32, hipStream_t s) {
  return t == ACT_BF16 ? adapters_grad<bf16>(a, b, dx_f32, s) : adapters_grad<float>(a, b, dx_f32, s);
}

}  // namespace fb
