// Newton-Schulz orthogonalisation of a batch of matrices with a short side, as adapters' gradients are.
//
//   X_0 = G / (|G|_F + eps),   X_j+1 = (a_j + b_j K_j + c_j K_j^2) X_j,   K_j = X_j X_j^T,   out = keep base + scale X_n
//
// X_j is P_j X_0 with a polynomial P_j of K_0, which is k x k for a short side of k, and K_j, P_j and all factors commute. So G
// is read twice however many steps there are: k_gram forms K_0, k_steps the polynomial from it (of more than 64 rows
// k_products does, product by product), and k_apply multiplies.
// All of it is in 64 bits. A quintic of slope a at zero raises weak directions by a in each step, to 485 in five of 3.4445, and takes
// that back where they have grown; an error d of K_0 then changes a weak direction by some 28000 d of itself, which 32 bits
// do not bear. The matrix instructions of 64 bits take 64 cycles for 16 x 16 x 4, half the rate of those of 32.
#include "local_common.hpp"

using namespace haflo::local;

namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));

constexpr u32 kThreads = 256, kWaves = kThreads / kWave;
constexpr size_t kMostShort = HAFLO_ADAPTER_MAX_RANK;
constexpr size_t kMostDistance = (size_t)1 << 32;  // between rows of the result
constexpr size_t kMostLength = (size_t)1 << 38;    // of all matrices' long sides together, whose pieces 32 bits count
constexpr u32 kChunk = 32;  // of the long side in one step of k_gram

// acc += a b on 16 x 16 by 4: lane l holds row l % 16 of both operands at element l / 16, and in acc[r] row 4 r + l / 16 of the
// first operand against row l % 16 of the second.
__device__ __forceinline__ f64x4 mma4(double a, double b, f64x4 acc) { return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, acc, 0, 0, 0); }

// Matrices of one shape, `step` apart, rows `ld` apart.
template <class T>
struct Batch {
  T* p;
  size_t ld, step;
};

template <bool V>
struct Flag {
  static constexpr bool value = V;
};

// The short side is covered by KT tiles of sixteen. Row `place` of tile i is the short side's 16 i + place where its rows are the
// matrix's; where they are its columns, it is KT place + i, so that a lane's rows of all tiles lie beside each other in memory.
template <int KT, bool TALL>
__device__ __forceinline__ u32 short_of(u32 tile, u32 place) {
  return TALL ? KT * place + tile : 16 * tile + place;
}

// `N` elements from `s` on of a row of `k`, zeros behind it
template <class T, int N>
__device__ __forceinline__ void load_few(const T* row, u32 s, u32 k, T (&out)[N]) {
  if (s + N <= k) {
    __builtin_memcpy(out, row + s, sizeof(out));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = s + i < k ? row[s + i] : (T)0.0f;
  }
}

// What a lane holds of 32 places of the long side: row (lane % 16) of every tile at places at + 8 (lane / 16) .. + 7. Where rows are
// the matrix's columns, each place is one load of KT elements; WHOLE: KT divides k, so that a lane's are all there or none is.
template <class T, int KT, bool TALL>
struct Chunk;
template <class T, int KT>
struct Chunk<T, KT, false> {
  Vec8<T> v[KT];
  template <bool WHOLE>
  __device__ __forceinline__ void load(const T* m, size_t ld, u32 k, u32 length, u32 at) {
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      const u32 s = 16 * i + lane_id() % 16;
      v[i] = load_cols(m + (size_t)(s < k ? s : k - 1) * ld, at + lane_id() / 16 * 8, length);
    }
  }
  __device__ __forceinline__ double get(int i, int e, u32, u32, u32) const { return (double)(float)v[i].get(e); }
};
template <class T, int KT>
struct Chunk<T, KT, true> {
  T v[8][KT];
  template <bool WHOLE>
  __device__ __forceinline__ void load(const T* m, size_t ld, u32 k, u32 length, u32 at) {
    const u32 s = KT * (lane_id() % 16), l = at + lane_id() / 16 * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const T* const row = m + (size_t)(l + e < length ? l + e : length - 1) * ld;
      if (WHOLE) {
        __builtin_memcpy(v[e], row + (s < k ? s : 0), sizeof(v[e]));
      } else {
#pragma unroll
        for (int i = 0; i < KT; ++i) v[e][i] = row[s + i < k ? s + i : k - 1];
      }
    }
  }
  // (what lies past the matrix is another of its elements, and zero here)
  __device__ __forceinline__ double get(int i, int e, u32 k, u32 length, u32 at) const {
    return KT * (lane_id() % 16) + i < k && at + lane_id() / 16 * 8 + e < length ? (double)(float)v[e][i] : 0.0;
  }
};

// Rows W and 7 - W of eight rows of tiles, on and under the diagonal: nine products whichever.
template <int W>
__device__ __forceinline__ void two_rows(const double (&d)[8], f64x4 (&acc)[9]) {
#pragma unroll
  for (int j = 0; j <= W; ++j) acc[j] = mma4(d[W], d[j], acc[j]);
#pragma unroll
  for (int j = 0; j <= 7 - W; ++j) acc[W + 1 + j] = mma4(d[7 - W], d[j], acc[W + 1 + j]);
}

// One part of K_0, unscaled: a block takes `parts`-th pieces of the long side. Up to four tiles each wavefront forms all products of tiles,
// of its own chunks; of eight a wavefront forms two rows of tiles, of all chunks.
template <class T, int KT, bool TALL>
__global__ __launch_bounds__(kThreads) void k_gram(Batch<const T> g, u32 k, u32 length, u32 parts, double* out, u32 first_block) {
  constexpr u32 N = 16 * KT;
  constexpr bool kSplit = KT == 8;
  constexpr int kPairs = kSplit ? 9 : KT * (KT + 1) / 2;
  __shared__ double sum[kSplit ? 1 : kWaves][256];
  const u32 block = first_block + blockIdx.x, party = block / parts, part = block % parts;
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const T* const m = g.p + party * g.step;
  const u32 chunks = (length + kChunk - 1) / kChunk, first = (u32)((u64)chunks * part / parts), end = (u32)((u64)chunks * (part + 1) / parts);
  f64x4 acc[kPairs];
#pragma unroll
  for (int n = 0; n < kPairs; ++n) acc[n] = f64x4{0.0, 0.0, 0.0, 0.0};
  const auto add = [&](auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    constexpr u32 kStride = kSplit ? 1 : kWaves;
    Chunk<T, KT, TALL> now, next;
    u32 c = kSplit ? first : first + wave;
    if (c < end) next.template load<kWhole>(m, g.ld, k, length, c * kChunk);
    for (; c < end; c += kStride) {
      now = next;
      if (c + kStride < end) next.template load<kWhole>(m, g.ld, k, length, (c + kStride) * kChunk);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        double d[KT];
#pragma unroll
        for (int i = 0; i < KT; ++i) d[i] = now.get(i, e, k, length, c * kChunk);
        if constexpr (kSplit) {
          if (wave == 0) two_rows<0>(d, acc);
          else if (wave == 1) two_rows<1>(d, acc);
          else if (wave == 2) two_rows<2>(d, acc);
          else two_rows<3>(d, acc);
        } else {
          int n = 0;
#pragma unroll
          for (int i = 0; i < KT; ++i)
#pragma unroll
            for (int j = 0; j <= i; ++j, ++n) acc[n] = mma4(d[i], d[j], acc[n]);
        }
      }
    }
  };
  if (k % KT == 0) add(Flag<true>());
  else add(Flag<false>());
  double* const to = out + (size_t)block * N * N;
  const auto put = [&](u32 i, u32 j, u32 row, u32 col, double v) {  // both halves of the symmetric matrix, zeros past the short side
    const u32 s = short_of<KT, TALL>(i, row), t = short_of<KT, TALL>(j, col);
    const double w = s < k && t < k ? v : 0.0;
    to[s * N + t] = w;
    if (i != j) to[t * N + s] = w;
  };
  if constexpr (kSplit) {
#pragma unroll
    for (int n = 0; n < 9; ++n) {
      const bool up = (u32)n <= wave;
#pragma unroll
      for (int r = 0; r < 4; ++r) put(up ? wave : 7 - wave, up ? n : n - wave - 1, 4 * r + lane / 16, lane % 16, acc[n][r]);
    }
  } else {
    int n = 0;
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int j = 0; j <= i; ++j, ++n) {
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[wave][(4 * r + lane / 16) * 16 + lane % 16] = acc[n][r];
        __syncthreads();
        double s = 0.0;
#pragma unroll
        for (u32 w = 0; w < kWaves; ++w) s += sum[w][threadIdx.x];
        put(i, j, threadIdx.x / 16, threadIdx.x % 16, s);
        __syncthreads();
      }
  }
}

struct Steps {
  double c[HAFLO_UPDATE_MAX_STEPS][3];
  int count;
};
// The sum over a block's threads.
template <u32 THREADS>
__device__ __forceinline__ double block_sum(double v, double* room) {
  v = lanes_join(v, kWave, [](double a, double b) { return a + b; });
  if (THREADS == kWave) return v;
  if (lane_id() == 0) room[threadIdx.x / kWave] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (u32 w = 0; w < THREADS / kWave; ++w) v += room[w];
  return v;
}
// element i of the parts' sum, eight loads on their way at a time
__device__ __forceinline__ double sum_parts(const double* parts, u32 count, size_t each, u32 i) {
  double s = 0.0;
  u32 p = 0;
  for (; p + 8 <= count; p += 8) {
    double v[8];
#pragma unroll
    for (u32 j = 0; j < 8; ++j) v[j] = parts[(p + j) * each + i];
    s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  }
#pragma unroll 4
  for (; p < count; ++p) s += parts[p * each + i];
  return s;
}
__device__ __forceinline__ double factor_of(double squares, double eps) { return 1.0 / (sqrt(squares) + eps); }

// One tile of x y, N elements each of rows i of x and j of y: lane l takes elements 8 t + 2 (l / 16) and the next of row l % 16 of both.
template <u32 N>
__device__ __forceinline__ f64x4 tile_product(const double* x, const double* y, u32 i, u32 j, u32 ld) {
  const u32 at = lane_id() % 16 * ld + lane_id() / 16 * 2;
  const double *const a = x + 16 * i * ld + at, *const b = y + 16 * j * ld + at;
  double u[N / 8][2], v[N / 8][2];
#pragma unroll
  for (u32 t = 0; t < N / 8; ++t) {
    __builtin_memcpy(u[t], __builtin_assume_aligned(a + 8 * t, 16), 16);
    __builtin_memcpy(v[t], __builtin_assume_aligned(b + 8 * t, 16), 16);
  }
  f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (u32 t = 0; t < N / 8; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e) acc = mma4(u[t][e], v[t][e], acc);
  return acc;
}
// tile -> its row and column among those on and under the diagonal
__device__ __forceinline__ u32 tile_row(u32 tile) {
  u32 i = 0;
  while ((i + 1) * (i + 2) / 2 <= tile) ++i;
  return i;
}

// The polynomial of up to 64 rows, by one block in LDS: to = scale P / (|G|_F + eps). Products are of symmetric matrices that commute: the
// tiles on and under the diagonal are formed and mirrored, and the second operand's rows are read for its columns. Results
// stay in registers until all have read the operands, and then take an operand's place. The matrix instructions in turn bound it.
template <int KT>
constexpr u32 step_threads() {
  return KT == 1 ? kWave : KT == 2 ? 4 * kWave : 8 * kWave;
}
template <int KT>
__global__ __launch_bounds__(step_threads<KT>()) void k_steps(const double* parts, u32 count, Steps steps, double scale, double eps, double* to) {
  constexpr u32 N = 16 * KT, S = N + 2, THREADS = step_threads<KT>(), WAVES = THREADS / kWave, TILES = KT * (KT + 1) / 2;
  __shared__ __align__(16) double lds[3][N * S];
  __shared__ double room[WAVES];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  parts += (size_t)blockIdx.x * count * N * N;
  to += (size_t)blockIdx.x * N * N;
  double *const K = lds[0], *const Q = lds[1], *const P = lds[2];
  double squares = 0.0;
  for (u32 i = threadIdx.x; i < N * N; i += THREADS) {
    const double s = sum_parts(parts, count, N * N, i);
    K[i / N * S + i % N] = s;
    if (i / N == i % N) squares += s;
  }
  const double by = factor_of(block_sum<THREADS>(squares, room), eps);
  for (u32 i = threadIdx.x; i < N * N; i += THREADS) K[i / N * S + i % N] *= by * by;  // (each thread its own)
  __syncthreads();
  // out = one I + self x + both x y, of x0 and, with two jobs, of x1
  const auto products = [&](auto jobs, double* out0, double* out1, const double* x0, const double* x1, const double* y, double one, double self, double both) {
    constexpr u32 TOTAL = decltype(jobs)::value ? 2 * TILES : TILES, PER = (TOTAL + WAVES - 1) / WAVES;
    f64x4 acc[PER];
#pragma unroll
    for (u32 n = 0; n < PER; ++n) {
      const u32 id = wave + n * WAVES, tile = id % TILES, i = tile_row(tile), j = tile - i * (i + 1) / 2;
      if (id >= TOTAL) continue;
      const double* const from = id < TILES ? x0 : x1;
      acc[n] = tile_product<N>(from, y, i, j, S);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u32 row = 16 * i + 4 * r + lane / 16, col = 16 * j + lane % 16;
        acc[n][r] = both * acc[n][r] + (self != 0.0 ? self * from[row * S + col] : 0.0) + (row == col ? one : 0.0);
      }
    }
    __syncthreads();
#pragma unroll
    for (u32 n = 0; n < PER; ++n) {
      const u32 id = wave + n * WAVES, tile = id % TILES, i = tile_row(tile), j = tile - i * (i + 1) / 2;
      if (id >= TOTAL) continue;
      double* const o = id < TILES ? out0 : out1;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u32 row = 16 * i + 4 * r + lane / 16, col = 16 * j + lane % 16;
        o[row * S + col] = acc[n][r];
        if (i != j) o[col * S + row] = acc[n][r];
      }
    }
    __syncthreads();
  };
  const Flag<false> one_job;
  const Flag<true> two_jobs;
  for (int s = 0; s < steps.count; ++s) {
    const bool last = s + 1 == steps.count;
    double* const first = s == 0 ? P : Q;
    products(one_job, first, first, K, K, K, steps.c[s][0], steps.c[s][1], steps.c[s][2]);
    if (s == 0 && !last) {
      products(one_job, Q, Q, K, K, P, 0.0, 0.0, 1.0);  // (Q for what is between)
      products(one_job, K, K, Q, Q, P, 0.0, 0.0, 1.0);
    } else if (s > 0 && last) {
      products(one_job, P, P, P, P, Q, 0.0, 0.0, 1.0);
    } else if (s > 0) {
      products(two_jobs, K, P, K, P, Q, 0.0, 0.0, 1.0);
      products(one_job, K, K, K, K, Q, 0.0, 0.0, 1.0);
    }
  }
  for (u32 i = threadIdx.x; i < N * N; i += THREADS) to[i] = P[i / N * S + i % N] * (by * scale);
}

// More than 64 rows: K_0 and G's factor, from the parts.
constexpr u32 kLarge = 128;
__global__ __launch_bounds__(1024) void k_gram_join(const double* parts, u32 count, double eps, double* K, double* factor) {
  __shared__ double room[16];
  constexpr u32 kEach = kLarge * kLarge / 1024;
  parts += (size_t)blockIdx.x * count * kLarge * kLarge;
  double s[kEach], squares = 0.0;
#pragma unroll
  for (u32 n = 0; n < kEach; ++n) {
    const u32 i = n * 1024 + threadIdx.x;
    s[n] = sum_parts(parts, count, kLarge * kLarge, i);
    if (i / kLarge == i % kLarge) squares += s[n];
  }
  const double by = factor_of(block_sum<1024>(squares, room), eps);
#pragma unroll
  for (u32 n = 0; n < kEach; ++n) K[(size_t)blockIdx.x * kLarge * kLarge + n * 1024 + threadIdx.x] = s[n] * by * by;
  if (threadIdx.x == 0) factor[blockIdx.x] = by;
}
// out = one I + self x + both x y, times the party's factor where there is one
struct Product {
  const double *x, *y, *factor;
  double *out;
  double one, self, both;
};
struct Products {
  Product job[2];
};
// A wavefront forms one tile on or under the diagonal.
constexpr u32 kLargeTiles = 36;
__global__ __launch_bounds__(kWave) void k_products(Products p, u32 jobs, u32 first_block) {
  const u32 block = first_block + blockIdx.x, lane = lane_id(), tile = block % kLargeTiles, of = block / kLargeTiles;
  const Product q = p.job[of % jobs];
  const u32 party = of / jobs;
  const u32 i = tile_row(tile), j = tile - i * (i + 1) / 2;
  const size_t at = (size_t)party * kLarge * kLarge;
  const double* const x = q.x + at;
  const f64x4 acc = tile_product<kLarge>(x, q.y + at, i, j, kLarge);
  const double by = q.factor ? q.factor[party] : 1.0;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const u32 row = 16 * i + 4 * r + lane / 16, col = 16 * j + lane % 16;
    const double v = (q.both * acc[r] + (q.self != 0.0 ? q.self * x[row * kLarge + col] : 0.0) + (row == col ? q.one : 0.0)) * by;
    q.out[at + row * kLarge + col] = v;
    if (i != j) q.out[at + col * kLarge + row] = v;
  }
}

// out = keep base + P G. P lies in LDS; a wavefront takes `kPlaces` places of the long side by the whole short side at a time, and asks
// for the next ones before it multiplies.
template <int KT, bool TALL>
struct Apply {
  static constexpr int kVec = KT == 8 ? 2 : 4;  // along the long side, of rows
  static constexpr u32 kPlaces = TALL ? 16 : 16 * kVec;
  static constexpr u32 N = 16 * KT, S = N + 2;
};
template <class T, int KT, bool TALL>
__global__ __launch_bounds__(kThreads) void k_apply(Batch<const T> g, Batch<const T> base, Batch<T> out, const double* poly, u32 k, u32 length, double keep,
                                                    u32 blocks, u32 first_block) {
  using A = Apply<KT, TALL>;
  constexpr u32 N = A::N, S = A::S;
  __shared__ __align__(16) double P[N * S];
  const u32 block = first_block + blockIdx.x, party = block / blocks;
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id(), place = lane % 16, group = lane / 16;
  poly += (size_t)party * N * N;
  const T* const m = g.p + party * g.step;
  const T* const b = base.p ? base.p + party * base.step : nullptr;
  T* const o = out.p + party * out.step;
  const u32 pieces = (length + A::kPlaces - 1) / A::kPlaces, stride = blocks * kWaves;
  u32 piece = block % blocks * kWaves + wave;
  if constexpr (TALL) {
    // rows of the result are places of the long side; tile j holds the short side's KT (lane % 16) + j
    T next[KT][4], x[KT][4];
    const auto ask = [&](u32 at) {  // sixteen of the reduction, four to a lane, KT times
      const u32 l = at + place;
#pragma unroll
      for (u32 t = 0; t < KT; ++t) load_few<T, 4>(m + (size_t)(l < length ? l : length - 1) * g.ld, 16 * t + 4 * group, k, next[t]);
    };
    if (piece < pieces) ask(piece * A::kPlaces);
    for (u32 i = threadIdx.x; i < N * N; i += kThreads) P[i / N * S + i % N] = poly[i];
    __syncthreads();
    for (; piece < pieces; piece += stride) {
      const u32 at = piece * A::kPlaces, s = KT * place;
      __builtin_memcpy(x, next, sizeof(x));
      T was[4][KT] = {};
      if (b) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const u32 l = at + 4 * r + group;
          load_few<T, KT>(b + (size_t)(l < length ? l : length - 1) * base.ld, s, k, was[r]);
        }
      }
      if (piece + stride < pieces) ask((piece + stride) * A::kPlaces);
      f64x4 acc[KT];
#pragma unroll
      for (int j = 0; j < KT; ++j) acc[j] = f64x4{0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (u32 t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          double d[KT];
          __builtin_memcpy(d, &P[(16 * t + 4 * group + e) * S + s], sizeof(d));
          const double v = (double)(float)x[t][e];
#pragma unroll
          for (int j = 0; j < KT; ++j) acc[j] = mma4(v, d[j], acc[j]);
          if (KT == 8) __builtin_amdgcn_sched_barrier(0);  // (P's elements not all at once: there are registers for two steps')
        }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u32 l = at + 4 * r + group;
        if (l >= length) continue;
        T now[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j) now[j] = (T)(float)(b ? keep * (double)(float)was[r][j] + acc[j][r] : acc[j][r]);
        T* const to = o + (size_t)l * out.ld + s;
        if (s + KT <= k) {
          __builtin_memcpy(to, now, sizeof(now));
        } else {
#pragma unroll
          for (int j = 0; j < KT; ++j)
            if (s + j < k) to[j] = now[j];
        }
      }
    }
  } else {
    // tile j of the result's columns holds places at + kVec (lane % 16) + j
    constexpr int V = A::kVec;
    for (u32 i = threadIdx.x; i < N * N; i += kThreads) P[i / N * S + i % N] = poly[i];
    __syncthreads();
    for (; piece < pieces; piece += stride) {
      f64x4 acc[KT][V];
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[i][j] = f64x4{0.0, 0.0, 0.0, 0.0};
      const u32 l = piece * A::kPlaces + V * place;
      const auto ask = [&](u32 s, T (&x)[V]) { load_few<T, V>(m + (size_t)(s < k ? s : k - 1) * g.ld, l < length ? l : length, length, x); };
      constexpr u32 kAhead = N / 4 < 8 ? N / 4 : 8;  // loads on their way together, of one row of each lane group
      T x[kAhead][V];
#pragma unroll
      for (u32 n = 0; n < kAhead; ++n) ask(4 * n + group, x[n]);
      for (u32 t0 = 0; t0 < N; t0 += 4 * kAhead) {
        T now[kAhead][V];
        __builtin_memcpy(now, x, sizeof(x));
        if (t0 + 4 * kAhead < N) {
#pragma unroll
          for (u32 n = 0; n < kAhead; ++n) ask(t0 + 4 * (kAhead + n) + group, x[n]);
        }
#pragma unroll
        for (u32 n = 0; n < kAhead; ++n) {
          const u32 s = t0 + 4 * n + group;
#pragma unroll
          for (int i = 0; i < KT; ++i) {
            const double d = P[(16 * i + place) * S + s];
#pragma unroll
            for (int j = 0; j < V; ++j) acc[i][j] = mma4(d, s < k ? (double)(float)now[n][j] : 0.0, acc[i][j]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const u32 s = 16 * i + 4 * r + group;
          if (s >= k) continue;
          T was[V] = {}, now[V];
          if (b) load_few<T, V>(b + (size_t)s * base.ld, l < length ? l : length, length, was);
#pragma unroll
          for (int j = 0; j < V; ++j) now[j] = (T)(float)(b ? keep * (double)(float)was[j] + acc[i][j][r] : acc[i][j][r]);
          T* const to = o + (size_t)s * out.ld + l;
          if (l + V <= length) {
            __builtin_memcpy(to, now, sizeof(now));
          } else {
#pragma unroll
            for (int j = 0; j < V; ++j)
              if (l + j < length) to[j] = now[j];
          }
        }
    }
  }
}

struct Shape {
  size_t parties, k, length;
  bool tall;
  u32 tiles() const { return k <= 16 ? 1 : k <= 32 ? 2 : k <= 48 ? 3 : k <= 64 ? 4 : 8; }
  size_t side() const { return 16 * tiles(); }
};
struct Plan {
  size_t parts, gram, poly, factor, extra, total;
};
bool update_sizes(int type, size_t parties, size_t rows, size_t cols, Shape& s) {
  if (!valid_type(type) || parties > HAFLO_ADAPTER_MAX_PARTIES || rows < 1 || cols < 1 || rows > kMostCount || cols > kMostCount) return false;
  s = {parties, rows < cols ? rows : cols, rows < cols ? cols : rows, rows > cols};
  return s.k <= kMostShort && parties * s.length <= kMostLength;
}
Plan update_plan(const Shape& s) {
  Plan p;
  const size_t chunks = ceil_div(s.length, kChunk), want = ceil_div((size_t)512, s.parties ? s.parties : 1), most = ceil_div(chunks, 8);
  p.parts = want < most ? want : most;
  const size_t each = s.side() * s.side() * 8;
  p.gram = 0;
  p.poly = p.gram + s.parties * p.parts * each;
  p.factor = p.poly + s.parties * each;
  p.extra = p.factor + align256(s.parties * 8);
  p.total = s.k > 64 ? p.extra + 5 * s.parties * each : p.factor;
  return p;
}

// scale P / (|G|_F + eps) of more than 64 rows, product by product
void large_steps(const Shape& s, const Plan& plan, const Steps& steps, double scale, double eps, char* ws, hipStream_t st) {
  const size_t each = s.parties * kLarge * kLarge * 8;
  const auto place = [&](int i) { return (double*)(ws + plan.extra + i * each); };
  double *const K = place(0), *const Q = place(1), *P = place(2), *const M = place(3), *spare = place(4);
  double *const factor = (double*)(ws + plan.factor), *const to = (double*)(ws + plan.poly);
  hipLaunchKernelGGL(k_gram_join, dim3((unsigned)s.parties), dim3(1024), 0, st, (const double*)(ws + plan.gram), (u32)plan.parts, eps, K, factor);
  const auto run = [&](Products p, u32 jobs) {
    in_turns(s.parties * jobs * kLargeTiles, kWave, [&](u32 first, dim3 grid, dim3 block) { hipLaunchKernelGGL(k_products, grid, block, 0, st, p, jobs, first); });
  };
  for (int i = 0; i < steps.count; ++i) {
    const double a = steps.c[i][0], b = steps.c[i][1], c = steps.c[i][2];
    if (steps.count == 1) {
      run({{{K, K, factor, to, a * scale, b * scale, c * scale}, {}}}, 1);
      break;
    }
    double* const q = i == 0 ? P : Q;
    run({{{K, K, nullptr, q, a, b, c}, {}}}, 1);
    if (i + 1 == steps.count) {
      run({{{P, Q, factor, to, 0.0, 0.0, scale}, {}}}, 1);
      break;
    }
    run({{{K, q, nullptr, M, 0.0, 0.0, 1.0}, {P, Q, nullptr, spare, 0.0, 0.0, 1.0}}}, i == 0 ? 1 : 2);
    run({{{M, q, nullptr, K, 0.0, 0.0, 1.0}, {}}}, 1);
    if (i > 0) {
      double* const was = P;
      P = spare;
      spare = was;
    }
  }
}

// Blocks of one matrix in k_apply: each brings P to LDS once, and there are enough for all compute units.
u32 apply_blocks(const Shape& s, u32 places) {
  const size_t need = ceil_div(s.length, places), want = ceil_div((size_t)1024, s.parties);
  return (u32)(need < want ? need : want);
}

template <class T, bool TALL>
void update(const Batch<const T>& g, const Batch<const T>& base, const Batch<T>& out, const Shape& s, const Plan& plan, const Steps& steps, double keep,
            double scale, double eps, char* ws, hipStream_t st) {
  double* const poly = (double*)(ws + plan.poly);
#define HAFLO_LOCAL_RUN(KT)                                                                                                                     \
  do {                                                                                                                                          \
    in_turns(s.parties * plan.parts, kThreads, [&](u32 first, dim3 grid, dim3 block) {                                                          \
      hipLaunchKernelGGL((k_gram<T, KT, TALL>), grid, block, 0, st, g, (u32)s.k, (u32)s.length, (u32)plan.parts, (double*)(ws + plan.gram), first); \
    });                                                                                                                                         \
    if constexpr (KT <= 4)                                                                                                                      \
      hipLaunchKernelGGL((k_steps<KT>), dim3((unsigned)s.parties), dim3(step_threads<KT>()), 0, st, (const double*)(ws + plan.gram),             \
                         (u32)plan.parts, steps, scale, eps, poly);                                                                             \
    else                                                                                                                                        \
      large_steps(s, plan, steps, scale, eps, ws, st);                                                                                          \
    const u32 blocks = apply_blocks(s, kWaves * Apply<KT, TALL>::kPlaces);                                                                      \
    in_turns(s.parties * blocks, kThreads, [&](u32 first, dim3 grid, dim3 block) {                                                              \
      hipLaunchKernelGGL((k_apply<T, KT, TALL>), grid, block, 0, st, g, base, out, (const double*)poly, (u32)s.k, (u32)s.length, keep, blocks,  \
                         first);                                                                                                                \
    });                                                                                                                                         \
  } while (0)
  switch (s.tiles()) {
    case 1: HAFLO_LOCAL_RUN(1); break;
    case 2: HAFLO_LOCAL_RUN(2); break;
    case 3: HAFLO_LOCAL_RUN(3); break;
    case 4: HAFLO_LOCAL_RUN(4); break;
    default: HAFLO_LOCAL_RUN(8); break;
  }
#undef HAFLO_LOCAL_RUN
}

// Whether an output may lie where an input does: matrix over matrix, row over row.
bool over(const void* in, size_t ld_in, size_t step_in, const void* out, size_t ld_out, size_t step_out, size_t parties, size_t rows) {
  return in != out || ((ld_in == ld_out || rows <= 1) && (step_in == step_out || parties <= 1));
}

}  // namespace

extern "C" {

size_t haflo_update_workspace_bytes(int type, size_t parties, size_t rows, size_t cols) {
  Shape s;
  return update_sizes(type, parties, rows, cols, s) ? update_plan(s).total : (size_t)-1;
}

int haflo_orthogonal_update(int type, const void* d_g, size_t ldg, size_t step_g, const void* d_base, size_t ldb, size_t step_b, size_t parties, size_t rows,
                            size_t cols, const double* coefficients, int steps, double keep, double scale, double eps, void* d_out, size_t ldo,
                            size_t step_o, void* d_workspace, size_t workspace_bytes, void* stream) {
  Shape s;
  if (!update_sizes(type, parties, rows, cols, s) || !coefficients || steps < 1 || steps > HAFLO_UPDATE_MAX_STEPS || !(eps > 0.0 && eps < HUGE_VAL) ||
      !(fabs(scale) < HUGE_VAL) || !(fabs(keep) < HUGE_VAL))
    return HAFLO_EINVAL;
  Steps list = {};
  list.count = steps;
  for (int i = 0; i < 3 * steps; ++i) {
    if (!(fabs(coefficients[i]) < HUGE_VAL)) return HAFLO_EINVAL;
    list.c[i / 3][i % 3] = coefficients[i];
  }
  if (parties == 0) return HAFLO_OK;
  if (!d_g || ldg < cols || !d_out || ldo < cols || (d_base && ldb < cols) || ldo > kMostDistance) return HAFLO_EINVAL;
  if (parties > 1 && step_o < (rows - 1) * ldo + cols) return HAFLO_EINVAL;  // matrices of the result over each other
  if (!over(d_g, ldg, step_g, d_out, ldo, step_o, parties, rows) || !over(d_base, ldb, step_b, d_out, ldo, step_o, parties, rows)) return HAFLO_EINVAL;
  const Plan plan = update_plan(s);
  if (!enough(d_workspace, workspace_bytes, plan.total)) return HAFLO_EINVAL;
  HAFLO_LOCAL_TYPES(type, {
    const Batch<const T> g = {(const T*)d_g, ldg, step_g}, base = {(const T*)d_base, ldb, step_b};
    const Batch<T> out = {(T*)d_out, ldo, step_o};
    if (s.tall) update<T, true>(g, base, out, s, plan, list, keep, scale, eps, (char*)d_workspace, (hipStream_t)stream);
    else update<T, false>(g, base, out, s, plan, list, keep, scale, eps, (char*)d_workspace, (hipStream_t)stream);
  });
  return launched();
}

}  // extern "C"
