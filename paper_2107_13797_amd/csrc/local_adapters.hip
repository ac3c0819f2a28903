// A projection that all parties share with each row's own low-rank adapter beside it, and its gradients.
//
//   forward   h[t] = scale A[a] drop(x[t]),      y[t] = W x[t] + B[a] h[t]           a = the row's adapter
//   backward  g[t] = scale B[a]^T dy[t],         dx[t] = W^T dy[t] + drop'(A[a]^T g[t])
//             dA[a] = sum_t g[t] drop(x[t])^T,   dB[a] = sum_t dy[t] h[t]^T
//
// h and g, the rows' short vectors ("z" where a kernel serves both directions), come from k_shrink; k_project forms the
// large product with the adapters' part as its first summand; k_grad sums over the rows of one adapter, which k_group
// lists. W^T and B^T for the backward pass are laid out by k_transpose, so that every product reduces along rows.
#include "local_common.hpp"

using namespace haflo::local;

namespace {

constexpr int kThreads = 256;

// An adapter matrix of every party, element (party, out, r) at party * party_step + out * out_step + r * r_step.
struct Low {
  size_t party_step, out_step, r_step;
};

__device__ __forceinline__ int party_of(const int* index, u32 t, u32 parties) {
  const int a = index[t];
  return (u32)a < parties ? a : -1;
}

// eight elements at (row, k) of a matrix, zeros past its edges
template <class T, bool WIDE>
__device__ __forceinline__ Vec8<T> load_tile(const T* m, size_t ld, u32 row, u32 rows, u32 k, u32 cols) {
  if (row >= rows || k >= cols) return Vec8<T>{};
  const T* p = m + (size_t)row * ld + k;
  if (WIDE && k + 8 <= cols) return load_wide(p);
  return load_some(p, cols - k < 8 ? (int)(cols - k) : 8);
}
template <class T>
__device__ __forceinline__ void apply_drop(Vec8<T>& v, const Drop& d, u32 row, u32 k) {
  const u32x4 draws = philox(d, k >> 3, row);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (!kept(d, draws, j)) v.v[j] = (T)0.0f;
}

// z[t, r] = scale[a] s sum_k drop(x[t, k]) F[a][r, k], F rows of length `inner`. A block takes 16 rows and one part of
// the reduction, its wavefronts a quarter of that each; once for every party among the rows.
template <class T, bool WIDE, int RT>
__global__ __launch_bounds__(kThreads) void k_shrink(const T* x, size_t ldx, const T* f, const float* scale, const int* index, u32 rows,
                                                     u32 inner, u32 rank, u32 parties, Drop d, u32 parts, float* z, u32* status) {
  __shared__ float sum[kThreads / kWave][RT][16][16];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const u32 t0 = blockIdx.x / parts * 16, part = blockIdx.x % parts;
  const u32 mine = t0 + lane % 16;
  const int raw = mine < rows ? index[mine] : -1;
  const int a = (u32)raw < parties ? raw : -1;
  if (status && part == 0 && threadIdx.x < 16 && raw != a && raw != -1) atomicOr(status, HAFLO_ST_RANGE);
  // this wavefront's share of the reduction, in steps of 32
  const u32 steps = (inner + 31) / 32, units = parts * (kThreads / kWave), unit = part * (kThreads / kWave) + wave;
  const u32 first = (u32)((u64)steps * unit / units), end = (u32)((u64)steps * (unit + 1) / units);
  float own[RT];  // of element (row lane / 16 * 4 + wave, r = lane % 16)
#pragma unroll
  for (int i = 0; i < RT; ++i) own[i] = 0.0f;
  const u32 out_t = t0 + lane / 16 * 4 + wave;
  const int out_a = out_t < rows ? party_of(index, out_t, parties) : -1;
  u64 left = __builtin_amdgcn_ballot_w64(a >= 0) & 0xFFFF;
  while (left) {
    const int who = __builtin_amdgcn_readlane(a, __builtin_ctzll(left));
    left &= ~__builtin_amdgcn_ballot_w64(a == who);
    const T* fa = f + (size_t)who * rank * inner;
    f32x4 acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (u32 s = first; s < end; ++s) {
      const u32 k = s * 32 + lane / 16 * 8;
      Vec8<T> xv = load_tile<T, WIDE>(x, ldx, mine, rows, k, inner);
      if (d.threshold) apply_drop(xv, d, mine, k);
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const Vec8<T> fv = load_tile<T, WIDE>(fa, inner, i * 16 + lane % 16, rank, k, inner);
        acc[i] = mma32(fv, xv, acc[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[wave][i][lane % 16][lane / 16 * 4 + j] = acc[i][j];
    __syncthreads();
    if (out_a == who) {
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const u32 t = lane / 16 * 4 + wave, r = lane % 16;
        own[i] = (sum[0][i][t][r] + sum[1][i][t][r]) + (sum[2][i][t][r] + sum[3][i][t][r]);
      }
    }
    __syncthreads();
  }
  if (out_t < rows) {
    const float by = out_a < 0 ? 0.0f : scale[out_a] * (d.threshold ? d.scale : 1.0f);
#pragma unroll
    for (int i = 0; i < RT; ++i)
      if (i * 16 + lane % 16 < rank) z[((size_t)part * rows + out_t) * rank + i * 16 + lane % 16] = own[i] * by;
  }
}

// z[i] = sum over parts
__global__ __launch_bounds__(kThreads) void k_join(const float* in, u32 parts, size_t count, float* z) {
  const size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= count) return;
  float s = 0.0f;
  for (u32 p = 0; p < parts; ++p) s += in[p * count + i];
  z[i] = s;
}

// out[c, r] = in[r, c], `count` matrices of rows x cols one behind the other
template <class T>
__global__ __launch_bounds__(kThreads) void k_transpose(const T* in, size_t ld, size_t in_step, u32 rows, u32 cols, T* out, size_t out_step) {
  __shared__ T tile[64][66];
  const u32 tiles_c = (cols + 63) / 64, tiles = tiles_c * ((rows + 63) / 64);
  const u32 which = blockIdx.x / tiles, at = blockIdx.x % tiles, r0 = at / tiles_c * 64, c0 = at % tiles_c * 64;
  in += which * in_step;
  out += which * out_step;
  for (u32 i = threadIdx.x; i < 64 * 64; i += kThreads) {
    const u32 r = r0 + i / 64, c = c0 + i % 64;
    if (r < rows && c < cols) tile[i / 64][i % 64] = in[(size_t)r * ld + c];
  }
  __syncthreads();
  for (u32 i = threadIdx.x; i < 64 * 64; i += kThreads) {
    const u32 c = c0 + i / 64, r = r0 + i % 64;
    if (r < rows && c < cols) out[(size_t)c * rows + r] = tile[i % 64][i / 64];
  }
}

// y[t, o] = drop'(sum_r z[t, r] F[a][o, r]) + sum_k x[t, k] W[o, k]. A block of four wavefronts takes 128 rows by 128
// outputs, a wavefront 64 x 64 as 4 x 4 products of 16 x 16; 128 bytes of the reduction at a time go through LDS.
template <class T, bool WIDE, bool DROP>
__global__ __launch_bounds__(kThreads) void k_project(const T* x, size_t ldx, const T* w, size_t ldw, const T* f, Low low, const float* z,
                                                      const int* index, u32 rows, u32 inner, u32 outer, u32 parties, u32 rank, Drop d,
                                                      T* y, size_t ldy) {
  constexpr int KE = 128 / sizeof(T), kPitch = KE + 16 / sizeof(T), kVecs = KE / 8;  // elements of a step, of a row in LDS
  constexpr int kLoads = 128 * kVecs / kThreads;
  __shared__ __align__(16) T lx[128 * kPitch];
  __shared__ __align__(16) T lw[128 * kPitch];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const u32 tiles_o = (outer + 127) / 128;
  const u32 t0 = blockIdx.x / tiles_o * 128, o0 = blockIdx.x % tiles_o * 128;
  const u32 wt = t0 + (wave & 1) * 64, wo = o0 + (wave >> 1) * 64;  // this wavefront's corner
  f32x4 acc[4][4];  // [outputs / 16][rows / 16]
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // the adapters' part, in 32 bits: once for every party among the 64 rows
  int a[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const u32 t = wt + j * 16 + lane % 16;
    a[j] = t < rows ? party_of(index, t, parties) : -1;
  }
  const int a_of_lane = wt + lane < rows ? party_of(index, wt + lane, parties) : -1;
  u64 left = __builtin_amdgcn_ballot_w64(a_of_lane >= 0);
  while (left) {
    const int who = __builtin_amdgcn_readlane(a_of_lane, __builtin_ctzll(left));
    left &= ~__builtin_amdgcn_ballot_w64(a_of_lane == who);
    const T* fa = f + (size_t)who * low.party_step;
    // rows of other parties are left as they are, not added to with zeros: an adapter may hold infinities
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f32x4 own[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) own[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      const u32 o = wo + i * 16 + lane % 16;
      for (u32 r0 = 0; r0 < rank; r0 += 16) {
        const u32 r = r0 + lane / 16 * 4;
        float zv[4][4], fv[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          fv[e] = o < outer && r + e < rank ? (float)fa[o * low.out_step + (r + e) * low.r_step] : 0.0f;
#pragma unroll
          for (int j = 0; j < 4; ++j) zv[j][e] = a[j] == who && r + e < rank ? z[(size_t)(wt + j * 16 + lane % 16) * rank + r + e] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j) own[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fv[e], zv[j][e], own[j], 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (a[j] == who) acc[i][j] = own[j];
    }
  }
  if (DROP) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32 o = wo + i * 16 + lane / 16 * 4;
        const u32x4 draws = philox(d, o >> 3, wt + j * 16 + lane % 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][e] = kept(d, draws, (o & 4) + e) ? acc[i][j][e] * d.scale : 0.0f;
      }
  }

  Vec8<T> gx[kLoads], gw[kLoads];
  const auto fetch = [&](u32 k0) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const u32 c = threadIdx.x + i * kThreads, r = c / kVecs, k = k0 + c % kVecs * 8;
      gx[i] = load_tile<T, WIDE>(x, ldx, t0 + r, rows, k, inner);
      gw[i] = load_tile<T, WIDE>(w, ldw, o0 + r, outer, k, inner);
    }
  };
  fetch(0);
  for (u32 k0 = 0; k0 < inner; k0 += KE) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const u32 c = threadIdx.x + i * kThreads, r = c / kVecs, k = c % kVecs * 8;
      store_wide(lx + r * kPitch + k, gx[i]);
      store_wide(lw + r * kPitch + k, gw[i]);
    }
    __syncthreads();
    if (k0 + KE < inner) fetch(k0 + KE);
#pragma unroll
    for (int s = 0; s < KE / 32; ++s) {
      Vec8<T> xv[4], wv[4];
      const u32 k = s * 32 + lane / 16 * 8;
#pragma unroll
      for (int j = 0; j < 4; ++j) xv[j] = load_wide(lx + (wt - t0 + j * 16 + lane % 16) * kPitch + k);
#pragma unroll
      for (int i = 0; i < 4; ++i) wv[i] = load_wide(lw + (wo - o0 + i * 16 + lane % 16) * kPitch + k);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = mma32(wv[i], xv[j], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const u32 t = wt + j * 16 + lane % 16, o = wo + i * 16 + lane / 16 * 4;
      if (t >= rows) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (o + e < outer) y[(size_t)t * ldy + o + e] = (T)acc[i][j][e];
    }
}

constexpr u32 kGradRows = 128;  // rows of one chunk of a party's list
constexpr u32 kGroupCounts = 16384;
inline u32 group_waves(size_t parties) { return parties <= 1024 ? 16 : 4; }  // whose counts fit LDS

// Groups the rows by adapter: `list` holds the rows of party 0 in ascending order, then those of party 1, ...;
// begin[p] where p's start; chunk_begin[p] the first of p's chunks of kGradRows rows; chunk[c] = p. One block; its
// wavefronts take a range of rows each, count them, and list them from where their counts say.
__global__ __launch_bounds__(1024) void k_group(const int* index, u32 rows, u32 parties, u32* begin, u32* chunk_begin, u32* chunk, u32* list,
                                                u32* status) {
  __shared__ u32 counts[kGroupCounts];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id(), waves = blockDim.x / kWave;
  const u32 per = (rows + waves - 1) / waves, first = wave * per < rows ? wave * per : rows, end = rows - first < per ? rows : first + per;
  for (u32 i = threadIdx.x; i < waves * parties; i += blockDim.x) counts[i] = 0;
  __syncthreads();
  for (int pass = 0; pass < 2; ++pass) {
    for (u32 t0 = first; t0 < end; t0 += kWave) {
      const u32 t = t0 + lane;
      const int raw = t < end ? index[t] : -1;
      const int a = (u32)raw < parties ? raw : -1;
      if (pass == 0 && raw != a && raw != -1 && status) atomicOr(status, HAFLO_ST_RANGE);
      u64 left = __builtin_amdgcn_ballot_w64(a >= 0);
      while (left) {
        const int leader = __builtin_ctzll(left), who = __builtin_amdgcn_readlane(a, leader);
        const u64 same = __builtin_amdgcn_ballot_w64(a == who);
        left &= ~same;
        u32 at = 0;
        if ((int)lane == leader) at = atomicAdd(&counts[wave * parties + who], (u32)__builtin_popcountll(same));
        at = (u32)__builtin_amdgcn_readlane((int)at, leader);
        if (pass == 1 && a == who) list[at + (u32)__builtin_popcountll(same & ((1ull << lane) - 1))] = t;
      }
    }
    __syncthreads();
    if (pass == 0 && threadIdx.x == 0) {  // counts to places
      u32 at = 0, chunks = 0;
      for (u32 p = 0; p < parties; ++p) {
        begin[p] = at;
        chunk_begin[p] = chunks;
        u32 n = 0;
        for (u32 w = 0; w < waves; ++w) {
          const u32 c = counts[w * parties + p];
          counts[w * parties + p] = at + n;
          n += c;
        }
        at += n;
        for (u32 i = 0; i < n; i += kGradRows) chunk[chunks++] = p;
      }
      begin[parties] = at;
      chunk_begin[parties] = chunks;
    }
    __syncthreads();
  }
}

// out[chunk][r][col] = sum over the chunk's rows t of z[t, r] drop(m[t, col]): a block takes 512 columns and sixteen r,
// its wavefronts a quarter of the rows each, a lane eight columns.
template <class T, bool WIDE>
__global__ __launch_bounds__(kThreads) void k_grad(const T* m, size_t ld, u32 cols, const float* z, u32 rank, u32 parties, const u32* begin,
                                                   const u32* chunk_begin, const u32* chunk, const u32* list, Drop d, float* out) {
  constexpr int kR = 16;
  __shared__ float sum[kR / 2][kWave * 8];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const u32 tiles_c = (cols + 511) / 512, tiles_r = (rank + kR - 1) / kR;
  const u32 c = blockIdx.x / (tiles_c * tiles_r), at = blockIdx.x % (tiles_c * tiles_r);
  if (c >= chunk_begin[parties]) return;
  const u32 col = at / tiles_r * 512 + lane * 8, r0 = at % tiles_r * kR;
  const u32 p = chunk[c], first = begin[p] + (c - chunk_begin[p]) * kGradRows;
  const u32 end = first + kGradRows < begin[p + 1] ? first + kGradRows : begin[p + 1];
  float acc[kR][8];
#pragma unroll
  for (int r = 0; r < kR; ++r)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[r][j] = 0.0f;
  for (u32 i = first + wave; i < end; i += kThreads / kWave) {
    const u32 t = (u32)__builtin_amdgcn_readfirstlane((int)list[i]);
    Vec8<T> v = load_tile<T, WIDE>(m + (size_t)t * ld, ld, 0, 1, col, cols);
    if (d.threshold) apply_drop(v, d, t, col);
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (float)v.v[j];
#pragma unroll
    for (int r = 0; r < kR; ++r) {
      const float zr = r0 + r < rank ? z[(size_t)t * rank + r0 + r] : 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[r][j] += zr * f[j];
    }
  }
  const float by = d.threshold ? d.scale : 1.0f;
  // the wavefronts' sums one after the other, in their order, half of the r at a time
  for (int half = 0; half < 2; ++half) {
    for (u32 w = 0; w < (u32)(kThreads / kWave); ++w) {
      if (wave == w) {
#pragma unroll
        for (int r = 0; r < kR; ++r)
          if (r / (kR / 2) == half) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              float* const s = &sum[r % (kR / 2)][lane * 8 + j];
              *s = w == 0 ? acc[r][j] : *s + acc[r][j];
            }
          }
      }
      __syncthreads();
    }
    for (u32 i = threadIdx.x; i < (u32)(kR / 2) * 512; i += kThreads) {
      const u32 r = r0 + half * (kR / 2) + i / 512, cc = at / tiles_r * 512 + i % 512;
      if (r < rank && cc < cols) out[((size_t)c * rank + r) * cols + cc] = sum[i / 512][i % 512] * by;
    }
    __syncthreads();
  }
}

// grad[p] = sum of the party's chunks, in their order; laid out as r_step and col_step say
__global__ __launch_bounds__(kThreads) void k_grad_join(const float* in, const u32* chunk_begin, u32 rank, u32 cols, size_t r_step,
                                                        size_t col_step, float* grad) {
  const size_t n = (size_t)rank * cols;
  const u32 blocks = (u32)((n + kThreads - 1) / kThreads), p = blockIdx.x / blocks;
  const size_t i = (size_t)(blockIdx.x % blocks) * kThreads + threadIdx.x;
  if (i >= n) return;
  float s = 0.0f;
  for (u32 c = chunk_begin[p]; c < chunk_begin[p + 1]; ++c) s += in[c * n + i];
  grad[p * n + i / cols * r_step + i % cols * col_step] = s;
}

struct Sizes {
  size_t rows, inner, outer, parties, rank;
};
bool adapter_sizes(int type, const Sizes& s) {
  return valid_type(type) && s.rows <= kMostCount && s.inner >= 1 && s.inner <= kMostCount - 512 && s.outer >= 1 &&
         s.outer <= kMostCount - 512 && s.parties >= 1 && s.parties <= HAFLO_ADAPTER_MAX_PARTIES && s.rank >= 1 &&
         s.rank <= HAFLO_ADAPTER_MAX_RANK;
}
// parts of k_shrink's reduction: enough blocks to fill the chip, at least 512 columns each
u32 shrink_parts(size_t rows, size_t k) {
  if (rows == 0) return 1;
  const size_t tiles = ceil_div(rows, 16), want = tiles < 512 ? ceil_div(512, tiles) : 1, most = ceil_div(k, 512);
  return (u32)(want < most ? want : most);
}
struct Plan {
  size_t z_parts, z, w_t, b_t, begin, chunk_begin, chunk, list, sums, total;
  size_t chunks;  // at most
};
Plan adapter_plan(int type, bool backward, const Sizes& s) {
  Plan p = {};
  size_t b = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = b;
    b += align256(bytes);
    return at;
  };
  const size_t e = type_size(type), k = backward ? s.outer : s.inner, parts = shrink_parts(s.rows, k);
  p.z_parts = take(parts > 1 ? parts * s.rows * s.rank * 4 : 0);
  if (backward) {
    p.z = take(s.rows * s.rank * 4);
    p.w_t = take(s.inner * s.outer * e);
    p.b_t = take(s.parties * s.outer * s.rank * e);
    p.chunks = s.rows / kGradRows + s.parties;
    p.begin = take((s.parties + 1) * 4);
    p.chunk_begin = take((s.parties + 1) * 4);
    p.chunk = take(p.chunks * 4);
    p.list = take(s.rows * 4);
    p.sums = take(p.chunks * s.rank * (s.inner > s.outer ? s.inner : s.outer) * 4);
  }
  p.total = b;
  return p;
}

template <class T>
void shrink(const T* x, size_t ldx, const T* f, const float* scale, const int* index, size_t rows, size_t inner, size_t rank,
            size_t parties, const Drop& d, float* z_parts, float* z, u32* status, hipStream_t st) {
  const u32 parts = shrink_parts(rows, inner);
  const dim3 grid((unsigned)(ceil_div(rows, 16) * parts)), block(kThreads);
  const bool wide = wide_rows<T>(x, ldx) && wide_rows<T>(f, inner);
  float* const to = parts > 1 ? z_parts : z;
#define HAFLO_LOCAL_RUN(WIDE, RT)                                                                                                     \
  hipLaunchKernelGGL((k_shrink<T, WIDE, RT>), grid, block, 0, st, x, ldx, f, scale, index, (u32)rows, (u32)inner, (u32)rank, (u32)parties, d, \
                     parts, to, status)
#define HAFLO_LOCAL_RANK(WIDE)                  \
  do {                                          \
    if (rank <= 16) HAFLO_LOCAL_RUN(WIDE, 1);   \
    else if (rank <= 64) HAFLO_LOCAL_RUN(WIDE, 4); \
    else HAFLO_LOCAL_RUN(WIDE, 8);              \
  } while (0)
  if (wide) HAFLO_LOCAL_RANK(true);
  else HAFLO_LOCAL_RANK(false);
#undef HAFLO_LOCAL_RANK
#undef HAFLO_LOCAL_RUN
  if (parts > 1)
    hipLaunchKernelGGL(k_join, dim3((unsigned)ceil_div(rows * rank, kThreads)), block, 0, st, z_parts, parts, rows * rank, z);
}

template <class T>
void project(const T* x, size_t ldx, const T* w, size_t ldw, const T* f, const Low& low, const float* z, const int* index, size_t rows,
             size_t inner, size_t outer, size_t parties, size_t rank, const Drop& d, T* y, size_t ldy, hipStream_t st) {
  const dim3 grid((unsigned)(ceil_div(rows, 128) * ceil_div(outer, 128))), block(kThreads);
  const bool wide = wide_rows<T>(x, ldx) && wide_rows<T>(w, ldw);
#define HAFLO_LOCAL_RUN(WIDE, DROP)                                                                                                       \
  hipLaunchKernelGGL((k_project<T, WIDE, DROP>), grid, block, 0, st, x, ldx, w, ldw, f, low, z, index, (u32)rows, (u32)inner, (u32)outer, \
                     (u32)parties, (u32)rank, d, y, ldy)
  if (d.threshold) {
    if (wide) HAFLO_LOCAL_RUN(true, true);
    else HAFLO_LOCAL_RUN(false, true);
  } else {
    if (wide) HAFLO_LOCAL_RUN(true, false);
    else HAFLO_LOCAL_RUN(false, false);
  }
#undef HAFLO_LOCAL_RUN
}

template <class T>
void grad(const T* m, size_t ld, size_t cols, const float* z, const Sizes& s, const Plan& p, char* ws, const Drop& d, size_t r_step,
          size_t col_step, float* out, hipStream_t st) {
  const dim3 block(kThreads);
  const dim3 grid((unsigned)(p.chunks * ceil_div(cols, 512) * ceil_div(s.rank, 16)));
  const u32* begin = (const u32*)(ws + p.begin);
  const u32* chunk_begin = (const u32*)(ws + p.chunk_begin);
  float* const sums = (float*)(ws + p.sums);
#define HAFLO_LOCAL_RUN(WIDE)                                                                                                          \
  hipLaunchKernelGGL((k_grad<T, WIDE>), grid, block, 0, st, m, ld, (u32)cols, z, (u32)s.rank, (u32)s.parties, begin, chunk_begin,      \
                     (const u32*)(ws + p.chunk), (const u32*)(ws + p.list), d, sums)
  if (wide_rows<T>(m, ld)) HAFLO_LOCAL_RUN(true);
  else HAFLO_LOCAL_RUN(false);
#undef HAFLO_LOCAL_RUN
  hipLaunchKernelGGL(k_grad_join, dim3((unsigned)(s.parties * ceil_div(s.rank * cols, kThreads))), block, 0, st, (const float*)sums, chunk_begin,
                     (u32)s.rank, (u32)cols, r_step, col_step, out);
}

template <class T>
void transpose(const T* in, size_t ld, size_t in_step, size_t rows, size_t cols, size_t count, T* out, size_t out_step, hipStream_t st) {
  const size_t tiles = ceil_div(rows, 64) * ceil_div(cols, 64);
  hipLaunchKernelGGL((k_transpose<T>), dim3((unsigned)(tiles * count)), dim3(kThreads), 0, st, in, ld, in_step, (u32)rows, (u32)cols, out, out_step);
}

}  // namespace

extern "C" {

size_t haflo_adapter_workspace_bytes(int type, int backward, size_t rows, size_t inner, size_t outer, size_t parties, size_t rank) {
  const Sizes s = {rows, inner, outer, parties, rank};
  return adapter_sizes(type, s) ? adapter_plan(type, backward != 0, s).total : (size_t)-1;
}

int haflo_adapter_forward(int type, const void* d_x, size_t ldx, const void* d_w, size_t ldw, const void* d_a, const void* d_b,
                          const float* d_scale, const int32_t* d_index, size_t rows, size_t inner, size_t outer, size_t parties,
                          size_t rank, double p, uint64_t seed, uint64_t offset, void* d_y, size_t ldy, float* d_h,
                          uint32_t* d_status, void* d_workspace, size_t workspace_bytes, void* stream) {
  const Sizes s = {rows, inner, outer, parties, rank};
  if (!adapter_sizes(type, s) || !(p >= 0.0 && p <= 1.0)) return HAFLO_EINVAL;
  if (rows == 0) return HAFLO_OK;
  if (!d_x || ldx < inner || !d_w || ldw < inner || !d_a || !d_b || !d_scale || !d_index || !d_y || ldy < outer || !d_h) return HAFLO_EINVAL;
  const Plan plan = adapter_plan(type, false, s);
  if (plan.total && (!d_workspace || workspace_bytes < plan.total)) return HAFLO_EINVAL;
  char* const ws = (char*)d_workspace;
  const hipStream_t st = (hipStream_t)stream;
  const Drop d = make_drop(p, seed, offset);
  Drop none = d;
  none.threshold = 0;
  HAFLO_LOCAL_TYPES(type, {
    shrink<T>((const T*)d_x, ldx, (const T*)d_a, d_scale, d_index, rows, inner, rank, parties, d, (float*)(ws + plan.z_parts), d_h, d_status, st);
    const Low low = {outer * rank, rank, 1};
    project<T>((const T*)d_x, ldx, (const T*)d_w, ldw, (const T*)d_b, low, d_h, d_index, rows, inner, outer, parties, rank, none, (T*)d_y, ldy, st);
  });
  return launched();
}

int haflo_adapter_backward(int type, const void* d_dy, size_t lddy, const void* d_x, size_t ldx, const void* d_w, size_t ldw,
                           const void* d_a, const void* d_b, const float* d_scale, const int32_t* d_index, const float* d_h,
                           size_t rows, size_t inner, size_t outer, size_t parties, size_t rank, double p, uint64_t seed,
                           uint64_t offset, void* d_dx, size_t lddx, float* d_da, float* d_db, uint32_t* d_status,
                           void* d_workspace, size_t workspace_bytes, void* stream) {
  const Sizes s = {rows, inner, outer, parties, rank};
  if (!adapter_sizes(type, s) || !(p >= 0.0 && p <= 1.0)) return HAFLO_EINVAL;
  if (!d_w || ldw < inner || !d_a || !d_b || !d_scale || !d_da || !d_db) return HAFLO_EINVAL;
  if (rows && (!d_dy || lddy < outer || !d_x || ldx < inner || !d_index || !d_h || (d_dx && lddx < inner))) return HAFLO_EINVAL;
  const Plan plan = adapter_plan(type, true, s);
  if (!d_workspace || workspace_bytes < plan.total) return HAFLO_EINVAL;
  char* const ws = (char*)d_workspace;
  const hipStream_t st = (hipStream_t)stream;
  const Drop d = make_drop(p, seed, offset);
  Drop none = d;
  none.threshold = 0;
  HAFLO_LOCAL_TYPES(type, {
    float* const g = (float*)(ws + plan.z);
    hipLaunchKernelGGL(k_group, dim3(1), dim3(group_waves(parties) * kWave), 0, st, d_index, (u32)rows, (u32)parties, (u32*)(ws + plan.begin),
                       (u32*)(ws + plan.chunk_begin), (u32*)(ws + plan.chunk), (u32*)(ws + plan.list), d_status);
    if (rows) {
      T* const b_t = (T*)(ws + plan.b_t);
      transpose<T>((const T*)d_b, rank, outer * rank, outer, rank, parties, b_t, outer * rank, st);
      shrink<T>((const T*)d_dy, lddy, b_t, d_scale, d_index, rows, outer, rank, parties, none, (float*)(ws + plan.z_parts), g, nullptr, st);
      if (d_dx) {
        T* const w_t = (T*)(ws + plan.w_t);
        transpose<T>((const T*)d_w, ldw, 0, outer, inner, 1, w_t, 0, st);
        const Low low = {rank * inner, 1, inner};
        project<T>((const T*)d_dy, lddy, w_t, outer, (const T*)d_a, low, g, d_index, rows, outer, inner, parties, rank, d, (T*)d_dx, lddx, st);
      }
    }
    grad<T>((const T*)d_x, ldx, inner, g, s, plan, ws, d, inner, 1, d_da, st);
    grad<T>((const T*)d_dy, lddy, outer, d_h, s, plan, ws, none, 1, rank, d_db, st);
  });
  return launched();
}

}  // extern "C"
