// Newton-Schulz orthogonalisation of a batch of matrices with a short side, as adapters' gradients are.
//
//   X_0 = G / (|G|_F + eps),   X_j+1 = (a_j + b_j K_j + c_j K_j^2) X_j,   K_j = X_j X_j^T,   out = keep base + scale X_n
//
// X_j is P_j X_0 with a polynomial P_j of K_0, which is k x k for a short side of k, and K_j, P_j and all factors commute. So G
// is read twice by most lists of steps: k_gram forms K_0, k_steps the polynomial from it (of more than 64 rows
// k_products does, product by product), and k_apply multiplies.
// All of it is in 64 bits. A quintic of slope a at zero raises weak directions by a in each step, to 485 in five of 3.4445, and takes
// that back where they have grown; an error d of K_0 then changes a weak direction by some 28000 d of itself, which 32 bits
// do not bear. The matrix instructions of 64 bits take 64 cycles for 16 x 16 x 4, half the rate of those of 32.
// What is rounded on the way from K_0 does not commute, and grows with the cube of what the steps raise, where X's own roundings
// grow with that itself. So a list that raises by more is cut (cuts_of): behind each part K is formed again from X = P G (k_gram_again), and
// the parts' polynomials are multiplied (k_chain). Against products one by one in 80 bits, as parts of what is greatest, 64 x 256 of equal rows: 5 steps
// of 3.4445 in one part 8e-10, 8 uncut 1e-5, 16 uncut 4e6; 8 in three parts 3.4e-11, 16 in six 3.2e-7 (one by one in 64 bits an error is
// some 2^-53 of what the steps raise by, of the greatest singular value: 4.4e-8, which is 50 times as much of what is greatest here).
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

// Blocks are dealt to the eight dies in turn, and a matrix's blocks go to one of them, whose cache then holds what they all read: its
// K, factors and P come from memory once in each launch (k_products of 64 matrices of 128 rows 14 us where each die reads them all).
// `each` blocks a matrix; a block past the last matrix has none.
constexpr u32 kDies = 8;
struct Place {
  u32 party, part;
};
__device__ __forceinline__ Place place_of_block(u32 block, u32 each, u32 parties) {
  if (parties < kDies) return {block / each, block % each};
  const u32 at = block / kDies;
  return {at / each * kDies + block % kDies, at % each};
}
inline size_t blocks_of(size_t each, size_t parties) { return (parties < kDies ? parties : ceil_div(parties, kDies) * kDies) * each; }

template <int V>
struct Number {
  static constexpr int value = V;
};

// The short side is covered by KT tiles of sixteen. Row `place` of tile i is the short side's 16 i + place where its rows are the
// matrix's; where they are its columns, it is KT place + i, so that a lane's rows of all tiles lie beside each other in memory.
template <int KT, bool TALL>
__device__ __forceinline__ u32 short_of(u32 tile, u32 place) {
  return TALL ? KT * place + tile : 16 * tile + place;
}

// `N` elements from `s` on of a row of `k`; past its end any of the row's
template <class T, int N>
__device__ __forceinline__ void load_few(const T* row, u32 s, u32 k, T (&out)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = row[s + i < k ? s + i : k - 1];
}
// the same where N divides k and no element is taken by itself
template <class T, int N>
__device__ __forceinline__ void load_whole(const T* row, u32 s, u32 k, T (&out)[N]) {
  __builtin_memcpy(out, row + (s < k ? s : 0), sizeof(out));
}
template <class T, int N>
__device__ __forceinline__ void store_few(T* row, u32 s, u32 k, const T (&in)[N]) {
  if (s + N <= k) {
    __builtin_memcpy(row + s, in, sizeof(in));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (s + i < k) row[s + i] = in[i];
  }
}

// What a lane holds of 32 places of the long side: row (lane % 16) of every tile at places at + 8 (lane / 16) .. + 7, zeros past the long
// side. Rows past the short side are other ones of the matrix: what they give is left aside. Loads stand in no branch that lanes
// take apart, as they would be waited for at its end. WHOLE: KT divides k.
template <class T, int KT, bool TALL>
struct Chunk {
  Vec8<T> v[KT];      // of rows
  T t[TALL ? 8 : 1][KT];  // of columns: each place is one load of KT elements
  template <bool WHOLE>
  __device__ __forceinline__ void load(const T* m, size_t ld, u32 k, u32 length, u32 at) {
    const u32 place = lane_id() % 16, l = at + lane_id() / 16 * 8;
    if constexpr (TALL) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const T* const row = m + (size_t)(l + e < length ? l + e : length - 1) * ld;
        if (WHOLE) load_whole<T, KT>(row, KT * place, k, t[e]);
        else load_few<T, KT>(row, KT * place, k, t[e]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        const u32 s = 16 * i + place;
        const T* const row = m + (size_t)(s < k ? s : k - 1) * ld;
        if (at + kChunk <= length) v[i] = load_wide(row + l);
        else v[i] = load_cols(row, l, length);
      }
    }
  }
  __device__ __forceinline__ void end(u32 length, u32 at) {  // (rows' ends are zeros already)
    if (!TALL || at + kChunk <= length) return;
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int i = 0; i < KT; ++i)
        if (at + lane_id() / 16 * 8 + e >= length) t[TALL ? e : 0][i] = (T)0.0f;
  }
  __device__ __forceinline__ double get(int i, int e) const { return TALL ? (double)(float)t[TALL ? e : 0][i] : (double)(float)v[i].get(e); }
};

// Rows W and 7 - W of eight rows of tiles, on and under the diagonal: nine products whichever.
template <int W>
__device__ __forceinline__ void two_rows(const double (&d)[8], f64x4 (&acc)[9]) {
#pragma unroll
  for (int j = 0; j <= W; ++j) acc[j] = mma4(d[W], d[j], acc[j]);
#pragma unroll
  for (int j = 0; j <= 7 - W; ++j) acc[W + 1 + j] = mma4(d[7 - W], d[j], acc[W + 1 + j]);
}

// The products of tiles of chunks first, first + stride .. below end. Up to six tiles a wavefront forms all products, of eight two
// rows' (`wave` 0 .. 3).
template <int KT>
constexpr int pairs_of() {
  return KT == 8 ? 9 : KT * (KT + 1) / 2;
}
template <class T, int KT, bool TALL>
__device__ __forceinline__ void gram(const T* m, size_t ld, u32 k, u32 length, u32 first, u32 end, u32 stride, u32 wave, f64x4 (&acc)[pairs_of<KT>()]) {
#pragma unroll
  for (int n = 0; n < pairs_of<KT>(); ++n) acc[n] = f64x4{0.0, 0.0, 0.0, 0.0};
  const auto add = [&](auto whole, auto rows) {
    constexpr bool kWhole = decltype(whole)::value;
    Chunk<T, KT, TALL> now, next;
    u32 c = first;
    if (c < end) next.template load<kWhole>(m, ld, k, length, c * kChunk);
    for (; c < end; c += stride) {
      now = next;
      if (c + stride < end) next.template load<kWhole>(m, ld, k, length, (c + stride) * kChunk);
      now.end(length, c * kChunk);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        double d[KT];
#pragma unroll
        for (int i = 0; i < KT; ++i) d[i] = now.get(i, e);
        if constexpr (KT == 8) {
          two_rows<decltype(rows)::value>(d, acc);
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
  const auto by_rows = [&](auto whole) {
    if (KT < 8 || wave == 0) add(whole, Number<0>());
    else if (wave == 1) add(whole, Number<KT < 8 ? 0 : 1>());
    else if (wave == 2) add(whole, Number<KT < 8 ? 0 : 2>());
    else add(whole, Number<KT < 8 ? 0 : 3>());
  };
  if (!TALL || k % KT == 0) by_rows(Number<1>());
  else by_rows(Number<0>());
}
// the row of a tile among those on and under the diagonal, counted row by row
__device__ __forceinline__ u32 tile_row(u32 tile) {
  u32 i = 0;
  while ((i + 1) * (i + 2) / 2 <= tile) ++i;
  return i;
}
// A block's sums of up to six rows of tiles, some tiles at a time: put(row, column, sum) for both halves, zeros past the short side.
template <int KT>
constexpr int tiles_at_once() {
  return pairs_of<KT>() < 5 ? pairs_of<KT>() : KT == 3 ? 3 : KT == 6 ? 7 : 5;
}
template <int KT, bool TALL, u32 WAVES, class Put>
__device__ __forceinline__ void gram_sums(const f64x4 (&acc)[pairs_of<KT>()], u32 wave, u32 k, double (*sum)[tiles_at_once<KT>()][256], const Put& put) {
  constexpr int kOnce = tiles_at_once<KT>();
  const u32 lane = lane_id();
#pragma unroll
  for (int n0 = 0; n0 < pairs_of<KT>(); n0 += kOnce) {
    if (n0) __syncthreads();
#pragma unroll
    for (int n = 0; n < kOnce; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[wave][n][(4 * r + lane / 16) * 16 + lane % 16] = acc[n0 + n][r];
    __syncthreads();
    for (u32 at = threadIdx.x; at < kOnce * 256; at += WAVES * kWave) {
      const u32 n = at / 256, of = at % 256, i = tile_row(n0 + n), j = n0 + n - i * (i + 1) / 2;
      double v = 0.0;
#pragma unroll
      for (u32 w = 0; w < WAVES; ++w) v += sum[w][n][of];
      const u32 s = short_of<KT, TALL>(i, of / 16), t = short_of<KT, TALL>(j, of % 16);
      v = s < k && t < k ? v : 0.0;
      put(s, t, v);
      if (i != j) put(t, s, v);
    }
  }
}

// One part of K_0, unscaled: a block takes `parts`-th pieces of the long side. Its matrix instructions bound it where the short side is long (64
// matrices of 4096 x 64 float32 34 us, in 57 % of whose cycles they are busy: 20 us at their rate, 14 of memory), a launch and the loads'
// latency otherwise (8 of 16 x 4096 3.7 us).
template <class T, int KT, bool TALL>
__global__ __launch_bounds__(kThreads) void k_gram(Batch<const T> g, u32 k, u32 length, u32 parts, u32 parties, double* out, u32 first_block) {
  constexpr u32 N = 16 * KT;
  constexpr bool kSplit = KT == 8;
  __shared__ double sum[kSplit ? 1 : kWaves][tiles_at_once<KT>()][256];
  const auto [party, part] = place_of_block(first_block + blockIdx.x, parts, parties);
  if (party >= parties) return;
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const u32 chunks = (length + kChunk - 1) / kChunk, first = (u32)((u64)chunks * part / parts), end = (u32)((u64)chunks * (part + 1) / parts);
  f64x4 acc[pairs_of<KT>()];
  gram<T, KT, TALL>(g.p + party * g.step, g.ld, k, length, kSplit ? first : first + wave, end, kSplit ? 1 : kWaves, wave, acc);
  double* const to = out + ((size_t)party * parts + part) * N * N;
  if constexpr (kSplit) {
#pragma unroll
    for (int n = 0; n < 9; ++n) {
      const bool up = (u32)n <= wave;
      const u32 i = up ? wave : 7 - wave, j = up ? n : n - wave - 1;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u32 s = short_of<KT, TALL>(i, 4 * r + lane / 16), t = short_of<KT, TALL>(j, lane % 16);
        const double v = s < k && t < k ? acc[n][r] : 0.0;
        to[s * N + t] = v;
        if (i != j) to[t * N + s] = v;
      }
    }
  } else {
    gram_sums<KT, TALL, kWaves>(acc, wave, k, sum, [&](u32 s, u32 t, double v) { to[s * N + t] = v; });
  }
}

struct Steps {
  double c[HAFLO_UPDATE_MAX_STEPS][3];
  int count;
  u32 cuts;  // bit i: behind step i K is formed again
  // the end of the part that begins with step `first`
  __host__ __device__ __forceinline__ int end(int first) const {
    while (first + 1 < count && !(cuts >> first & 1)) ++first;
    return first + 1;
  }
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
// Elements at, at + apart .. of the parts' sums, many loads on their way at a time.
template <u32 E>
__device__ __forceinline__ void sum_parts(const double* parts, u32 count, size_t each, u32 at, u32 apart, double (&s)[E]) {
  constexpr u32 kAhead = E >= 8 ? 2 : 16 / E;
#pragma unroll
  for (u32 e = 0; e < E; ++e) s[e] = 0.0;
  u32 p = 0;
  for (; p + kAhead <= count; p += kAhead) {
    double v[kAhead][E];
#pragma unroll
    for (u32 j = 0; j < kAhead; ++j)
#pragma unroll
      for (u32 e = 0; e < E; ++e) v[j][e] = parts[(p + j) * each + at + e * apart];
#pragma unroll
    for (u32 e = 0; e < E; ++e)
#pragma unroll
      for (u32 j = 0; j < kAhead; ++j) s[e] += v[j][e];
  }
  for (; p < count; ++p)
#pragma unroll
    for (u32 e = 0; e < E; ++e) s[e] += parts[p * each + at + e * apart];
}
// (of a matrix of zeros 0: 1 / eps may be infinite)
__device__ __forceinline__ double factor_of(double squares, double eps) { return squares == 0.0 ? 0.0 : 1.0 / (sqrt(squares) + eps); }

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
  __builtin_amdgcn_sched_barrier(0);  // all are asked for before the first is waited for
  f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (u32 t = 0; t < N / 8; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e) acc = mma4(u[t][e], v[t][e], acc);
  return acc;
}

// The polynomial of K where it lies in LDS with Q and P, rows N + 2 apart, by a block of WAVES wavefronts; it is left in P. Products are of
// symmetric matrices that commute: the tiles on and under the diagonal are formed and mirrored, and the second operand's rows are
// read for its columns. Results stay in registers until all have read the operands, and then take an operand's place. A chain of products
// bounds it, of each step three, which wait for each other: of 64 rows 6.7 us a step, 4.7 of them matrix instructions (17 products of ten tiles in
// five steps, 64 cycles a tile and four elements, on the four vector units of one compute unit).
template <int KT, u32 WAVES>
__device__ __forceinline__ void polynomial(double* K, double* Q, double* P, const Steps& steps, u32 wave) {
  constexpr u32 N = 16 * KT, S = N + 2, TILES = KT * (KT + 1) / 2;
  const u32 lane = lane_id();
  // this wavefront's tiles, of two jobs at most (the row of a tile is found once: the search takes as long as some matrix instructions)
  constexpr u32 MOST = (2 * TILES + WAVES - 1) / WAVES;
  u32 row_of[MOST], col_of[MOST];
#pragma unroll
  for (u32 n = 0; n < MOST; ++n) {
    const u32 tile = (wave + n * WAVES) % TILES;
    row_of[n] = tile_row(tile);
    col_of[n] = tile - row_of[n] * (row_of[n] + 1) / 2;
  }
  // out = one I + self x + both x y, of x0 and, with two jobs, of x1
  const auto products = [&](auto jobs, double* out0, double* out1, const double* x0, const double* x1, const double* y, double one, double self, double both) {
    constexpr u32 TOTAL = decltype(jobs)::value * TILES, PER = (TOTAL + WAVES - 1) / WAVES;
    f64x4 acc[PER];
#pragma unroll
    for (u32 n = 0; n < PER; ++n) {
      const u32 id = wave + n * WAVES, i = row_of[n], j = col_of[n];
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
      const u32 id = wave + n * WAVES, i = row_of[n], j = col_of[n];
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
  const Number<1> one_job;
  const Number<2> two_jobs;
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
}
// The same of one tile by one wavefront, in registers: lane l's results are elements 4 r + l / 16 of row l % 16, as the matrix is symmetric,
// which is what the lane brings to the next product. 256 cycles each, one after the other.
__device__ __forceinline__ f64x4 tile_squared(const f64x4& x, const f64x4& y) {
  f64x4 acc = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (int r = 0; r < 4; ++r) acc = mma4(x[r], y[r], acc);
  return acc;
}
__device__ __forceinline__ f64x4 polynomial(f64x4 K, const Steps& steps, int first, int end) {
  f64x4 P = {};
  for (int s = first; s < end; ++s) {
    const f64x4 square = tile_squared(K, K);
    f64x4 Q;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      Q[r] = steps.c[s][2] * square[r] + (steps.c[s][1] * K[r] + (4 * r + lane_id() / 16 == lane_id() % 16 ? steps.c[s][0] : 0.0));
    if (s + 1 < end) K = tile_squared(tile_squared(K, Q), Q);
    P = s == first ? Q : tile_squared(P, Q);
  }
  return P;
}

// From K's sums, element threadIdx.x + e THREADS of it in `sums`, to scale P / (|G|_F + eps), which put(row, column, value) takes: by a block,
// of one tile by a wavefront. `again`: they are sums of X, and the factor of G is in it. Of one tile steps first .. end - 1.
template <int KT>
struct StepRoom {
  double m[KT == 1 ? 1 : 3][KT == 1 ? 1 : 16 * KT * (16 * KT + 2)];
};
template <int KT>
constexpr u32 step_threads() {
  return KT == 1 ? kWave : KT == 2 ? 8 * kWave : KT == 3 ? 12 * kWave : 16 * kWave;
}
template <int KT>
constexpr u32 step_elements() {
  return 256 * KT * KT / step_threads<KT>();
}
template <int KT, class Put>
__device__ __forceinline__ void steps_of(const Steps& steps, int first, int end, double scale, double eps, bool again, StepRoom<KT>& held, double* room,
                                         const double (&sums)[step_elements<KT>()], const Put& put) {
  constexpr u32 N = 16 * KT, S = N + 2, THREADS = step_threads<KT>(), E = step_elements<KT>();
  double squares = 0.0;
#pragma unroll
  for (u32 e = 0; e < E; ++e) {
    const u32 i = threadIdx.x + e * THREADS;
    if (i / N == i % N) squares += sums[e];
  }
  const double by = again ? 1.0 : factor_of(block_sum<THREADS>(squares, room), eps);
  if constexpr (KT == 1) {
    // (element lane + 64 r is of row 4 r + lane / 16 and column lane % 16: as the products have it)
    f64x4 K;
#pragma unroll
    for (int r = 0; r < 4; ++r) K[r] = sums[r] * by * by;
    const f64x4 P = polynomial(K, steps, first, end);
#pragma unroll
    for (int r = 0; r < 4; ++r) put(4 * r + threadIdx.x / 16, threadIdx.x % 16, P[r] * (by * scale));
  } else {
    double *const K = held.m[0], *const P = held.m[2];
#pragma unroll
    for (u32 e = 0; e < E; ++e) {
      const u32 i = threadIdx.x + e * THREADS;
      K[i / N * S + i % N] = sums[e] * by * by;
    }
    __syncthreads();
    polynomial<KT, THREADS / kWave>(K, held.m[1], P, steps, (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)));
#pragma unroll
    for (u32 e = 0; e < E; ++e) {
      const u32 i = threadIdx.x + e * THREADS;
      put(i / N, i % N, P[i / N * S + i % N] * (by * scale));
    }
  }
}

// The polynomial of 17 to 64 rows, and of up to 16 where the list is cut, from the parts' sums, by a block (five steps of 32 rows 13 us, of
// 48 21, of 64 36).
template <int KT>
__global__ __launch_bounds__(step_threads<KT>()) void k_steps(const double* parts, u32 count, Steps steps, double scale, double eps, u32 again, double* to) {
  constexpr u32 N = 16 * KT;
  __shared__ __align__(16) StepRoom<KT> held;
  __shared__ double room[16];
  parts += (size_t)blockIdx.x * count * N * N;
  to += (size_t)blockIdx.x * N * N;
  double sums[step_elements<KT>()];
  sum_parts(parts, count, N * N, threadIdx.x, step_threads<KT>(), sums);
  steps_of<KT>(steps, 0, steps.count, scale, eps, again, held, room, sums, [&](u32 i, u32 j, double v) { to[i * N + j] = v; });
}

// K of X = P G: a wavefront forms X on sixteen places of the long side, as the transpose, whose results lie in registers as the products by
// themselves take them, and rows FROM .. TO - 1 of tiles of X X^T from it. R is P transposed, rows N + 2 apart in LDS. Pieces piece, piece + stride ..
// below end. It is a part of lists that most calls do not have, and is kept simple: its loads are waited for (64 matrices of 4096 x 64 float32
// 90 us a part, of 128 x 4096 615, of which matrix instructions are 44 and 250).
constexpr int tiles_below(int rows) { return rows * (rows + 1) / 2; }
template <class T, int KT, bool TALL, int FROM, int TO, int COUNT>
__device__ __forceinline__ void gram_again(const T* m, size_t ld, const double* R, u32 k, u32 length, u32 piece, u32 end, u32 stride, f64x4 (&acc)[COUNT]) {
  static_assert(tiles_below(TO) - tiles_below(FROM) <= COUNT, "");
  constexpr u32 S = 16 * KT + 2;
  const u32 place = lane_id() % 16, group = lane_id() / 16;
#pragma unroll
  for (int n = 0; n < COUNT; ++n) acc[n] = f64x4{0.0, 0.0, 0.0, 0.0};
  for (; piece < end; piece += stride) {
    const u32 l = piece * 16 + place, at = l < length ? l : length - 1;
    f64x4 x[TO];
#pragma unroll
    for (int i = 0; i < TO; ++i) x[i] = f64x4{0.0, 0.0, 0.0, 0.0};
#pragma unroll 4
    for (u32 t = 0; t < 4 * KT; ++t) {
      const u32 s = 4 * t + group, row = s < k ? s : k - 1;
      const T v = TALL ? m[at * ld + row] : m[row * ld + at];
      const double d = s < k && l < length ? (double)(float)v : 0.0;
#pragma unroll
      for (int i = 0; i < TO; ++i) x[i] = mma4(d, R[s * S + 16 * i + place], x[i]);
    }
    // x[i][r]: place 4 r + group of row 16 i + place
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      int n = 0;
#pragma unroll
      for (int i = FROM; i < TO; ++i)
#pragma unroll
        for (int j = 0; j <= i; ++j, ++n) acc[n] = mma4(x[i][r], x[j][r], acc[n]);
    }
  }
}
// A block's sums of them in `room`: wavefronts in turn put, and from the one behind `from` on add, `count` tiles from the `first` on.
template <u32 WAVES, int COUNT>
__device__ __forceinline__ void join_waves(const f64x4 (&acc)[COUNT], u32 wave, u32 from, u32 first, int count, double* room) {
  const u32 lane = lane_id();
  for (u32 w = 0; w < WAVES; ++w) {
    if (wave == w) {
#pragma unroll
      for (int n = 0; n < COUNT; ++n) {
        if (n >= count) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          double& sum = room[256 * (first + n) + 64 * r + lane];
          sum = w > from ? sum + acc[n][r] : acc[n][r];
        }
      }
    }
    __syncthreads();
  }
}
template <class T, int KT, bool TALL>
__global__ __launch_bounds__(kThreads) void k_gram_again(Batch<const T> g, const double* R, u32 k, u32 length, u32 parts, u32 parties, double* out) {
  constexpr u32 N = 16 * KT, S = N + 2, TILES = KT * (KT + 1) / 2;
  __shared__ __align__(16) double held[N * S];
  static_assert(N * S >= 256 * TILES, "");
  const auto [party, part] = place_of_block(blockIdx.x, parts, parties);
  if (party >= parties) return;
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const u32 pieces = (length + 15) / 16, first = (u32)((u64)pieces * part / parts), end = (u32)((u64)pieces * (part + 1) / parts);
  R += (size_t)party * N * N;
  for (u32 i = threadIdx.x; i < N * N; i += kThreads) held[i / N * S + i % N] = R[i];
  __syncthreads();
  // (the sums of eight rows of tiles are too many for one wavefront's registers: a pair of them shares its pieces)
  constexpr bool kPairs = KT == 8;
  constexpr int kRows = kPairs ? 6 : KT, kCount = tiles_below(kRows);
  const T* const m = g.p + party * g.step;
  f64x4 acc[kCount];
  const bool second = kPairs && wave % 2;
  if (second) gram_again<T, KT, TALL, kPairs ? kRows : 0, KT>(m, g.ld, held, k, length, first + wave / 2, end, kWaves / 2, acc);
  else gram_again<T, KT, TALL, 0, kRows>(m, g.ld, held, k, length, kPairs ? first + wave / 2 : first + wave, end, kPairs ? kWaves / 2 : kWaves, acc);
  __syncthreads();  // R's place is free
  join_waves<kWaves>(acc, wave, second, second ? kCount : 0, second ? (int)TILES - kCount : kCount, held);
  double* const to = out + ((size_t)party * parts + part) * N * N;
  for (u32 at = threadIdx.x; at < 256 * TILES; at += kThreads) {
    const u32 n = at / 256, i = tile_row(n), j = n - i * (i + 1) / 2, s = 16 * i + at % 256 / 16, t = 16 * j + at % 16;
    to[s * N + t] = held[at];
    if (i != j) to[t * N + s] = held[at];
  }
}
// R P, of the polynomial so far, transposed, and the next part's, which is symmetric: the transpose of their product in its order. All of its
// tiles: what is rounded on the way is not symmetric. `turned`: the product itself.
template <u32 N>
__global__ __launch_bounds__(kWave) void k_chain(const double* R, const double* P, u32 parties, u32 turned, double* out) {
  constexpr u32 KT = N / 16;
  const auto [party, tile] = place_of_block(blockIdx.x, KT * KT, parties);
  if (party >= parties) return;
  const u32 lane = lane_id(), i = tile / KT, j = tile % KT;
  const size_t at = (size_t)party * N * N;
  const f64x4 acc = tile_product<N>(R + at, P + at, i, j, N);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const u32 row = 16 * i + 4 * r + lane / 16, col = 16 * j + lane % 16;
    out[at + (turned ? col * N + row : row * N + col)] = acc[r];
  }
}

// More than 64 rows: K_0 and G's factor, from the parts; a block takes an eighth of a matrix, and each the parts' diagonals (16 parts of 8
// matrices 7.6 us, by a block each 34).
constexpr u32 kSlices = 8;
template <u32 N>
constexpr u32 join_threads() {
  return 4 * N;
}
template <u32 N>
__global__ __launch_bounds__(join_threads<N>()) void k_gram_join(const double* parts, u32 count, u32 parties, double eps, u32 again, double* K, double* factor) {
  __shared__ double room[join_threads<N>() / kWave];
  constexpr u32 kEach = N * N / kSlices / join_threads<N>();
  const auto [party, slice] = place_of_block(blockIdx.x, kSlices, parties);
  if (party >= parties) return;
  parts += (size_t)party * count * N * N;
  double s[kEach], squares = 0.0;
  sum_parts(parts, count, N * N, slice * kEach * join_threads<N>() + threadIdx.x, join_threads<N>(), s);
  if (threadIdx.x < N) {
    double d[1];
    sum_parts(parts, count, N * N, threadIdx.x * (N + 1), 0, d);
    squares = d[0];
  }
  const double by = again ? 1.0 : factor_of(block_sum<join_threads<N>()>(squares, room), eps);
#pragma unroll
  for (u32 n = 0; n < kEach; ++n) K[(size_t)party * N * N + (slice * kEach + n) * join_threads<N>() + threadIdx.x] = s[n] * by * by;
  if (slice == 0 && threadIdx.x == 0) factor[party] = by;
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
// A wavefront forms one tile on or under the diagonal. Five steps are fourteen launches: of 8 matrices 4.8 us each, most of it the launch and the
// operands' way from the last one's results; of 64 12.7, in which operands are read 32 KiB a tile. Up to 96 rows are taken as 96 (39
// matrices of 87 x 3927 float32 268 us, 419 as 128).
template <u32 N>
constexpr u32 large_tiles() {
  return (N / 16) * (N / 16 + 1) / 2;
}
template <u32 N>
__global__ __launch_bounds__(kWave) void k_products(Products p, u32 jobs, u32 parties, u32 first_block) {
  const auto [party, part] = place_of_block(first_block + blockIdx.x, jobs * large_tiles<N>(), parties);
  if (party >= parties) return;
  const u32 lane = lane_id(), tile = part % large_tiles<N>();
  const Product q = p.job[part / large_tiles<N>()];
  const u32 i = tile_row(tile), j = tile - i * (i + 1) / 2;
  const size_t at = (size_t)party * N * N;
  const double* const x = q.x + at;
  const f64x4 acc = tile_product<N>(x, q.y + at, i, j, N);
  const double by = q.factor ? q.factor[party] : 1.0;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const u32 row = 16 * i + 4 * r + lane / 16, col = 16 * j + lane % 16;
    const double v = (q.both * acc[r] + (q.self != 0.0 ? q.self * x[row * N + col] : 0.0) + (row == col ? q.one : 0.0)) * by;
    q.out[at + row * N + col] = v;
    if (i != j) q.out[at + col * N + row] = v;
  }
}

// A result rounded once. On the way to 16 bits float32 takes it towards zero, and its last bit says whether anything was cut off: with more than two
// bits behind those of the type the second rounding is then as one of the whole number.
template <class T>
__device__ __forceinline__ T once(double v) {
  const float near = (float)v;
  if (sizeof(T) == 4) return (T)near;
  const double back = (double)near;
  u32 bits = __builtin_bit_cast(u32, near);
  if (back != v) bits = (bits - (fabs(back) > fabs(v) ? 1u : 0u)) | 1u;
  return (T)__builtin_bit_cast(float, bits);
}

// out = keep base + P G, P in LDS with rows N + 2 apart: a wavefront takes `kPlaces` places of the long side by the whole short side at a
// time, pieces piece, piece + stride .., and asks for the next ones before it multiplies. Past the short side P is 0 against
// everything before it, so that any numbers may stand there. WHOLE: no load or store is cut by the short side's end. 64 matrices of
// 4096 x 64 float32 onto a base: 53 us, 3.8 TB/s, matrix instructions busy in 62 % of the cycles.
template <int KT, bool TALL>
struct Apply {
  static constexpr int kVec = KT > 2 ? 2 : 4;  // along the long side, of rows
  static constexpr u32 kPlaces = TALL ? 16 : 16 * kVec;
  static constexpr u32 N = 16 * KT, S = N + 2;
  static bool whole(size_t k) { return !TALL || (k % 4 == 0 && k % KT == 0); }
};
template <class T>
struct Matrices {
  const T *g, *base;
  T* out;
  size_t ldg, ldb, ldo;
};
template <class T, int KT, bool TALL, bool WHOLE>
__device__ __forceinline__ void apply(const Matrices<T>& m, const double* P, u32 k, u32 length, double keep, u32 piece, u32 stride) {
  using A = Apply<KT, TALL>;
  constexpr u32 N = A::N, S = A::S;
  const u32 place = lane_id() % 16, group = lane_id() / 16, pieces = (length + A::kPlaces - 1) / A::kPlaces;
  const auto row = [&](u32 i, u32 n) { return (size_t)(i < n ? i : n - 1); };
  if constexpr (TALL) {
    // rows of the result are places of the long side; tile j holds the short side's KT (lane % 16) + j
    const u32 s = KT * place;
    T next[KT][4], x[KT][4];
    const auto ask = [&](u32 at) {  // sixteen of the reduction, four to a lane, KT times
      const T* const from = m.g + row(at + place, length) * m.ldg;
#pragma unroll
      for (u32 t = 0; t < KT; ++t) {
        if (WHOLE) load_whole<T, 4>(from, 16 * t + 4 * group, k, next[t]);
        else load_few<T, 4>(from, 16 * t + 4 * group, k, next[t]);
      }
    };
    if (piece < pieces) ask(piece * A::kPlaces);
    for (; piece < pieces; piece += stride) {
      const u32 at = piece * A::kPlaces;
      __builtin_memcpy(x, next, sizeof(x));
      T was[4][KT] = {};
      if (m.base) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const T* const from = m.base + row(at + 4 * r + group, length) * m.ldb;
          if (WHOLE) load_whole<T, KT>(from, s, k, was[r]);
          else load_few<T, KT>(from, s, k, was[r]);
        }
      }
      if (piece + stride < pieces) ask((piece + stride) * A::kPlaces);
      f64x4 acc[KT];
#pragma unroll
      for (int j = 0; j < KT; ++j) acc[j] = f64x4{0.0, 0.0, 0.0, 0.0};
      // a step's elements of P are read under the products of the step before (and not earlier: there are registers for two steps')
      double d[2][KT];
      const auto read = [&](int n) { __builtin_memcpy(d[n & 1], &P[(16 * (n / 4) + 4 * group + n % 4) * S + s], sizeof(d[0])); };
      read(0);
#pragma unroll
      for (int n = 0; n < 4 * KT; ++n) {
        if (n + 1 < 4 * KT) read(n + 1);
        const double v = (double)(float)x[n / 4][n % 4];
#pragma unroll
        for (int j = 0; j < KT; ++j) acc[j] = mma4(v, d[n & 1][j], acc[j]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u32 l = at + 4 * r + group;
        T now[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j) now[j] = once<T>(m.base ? keep * (double)(float)was[r][j] + acc[j][r] : acc[j][r]);
        if (l < length) store_few<T, KT>(m.out + (size_t)l * m.ldo, s, k, now);
      }
    }
  } else {
    // tile j of the result's columns holds places at + kVec (lane % 16) + j
    constexpr int V = A::kVec;
    constexpr u32 kAhead = KT == 1 ? 4 : KT == 3 ? 6 : 8;  // loads on their way together, of one row of each lane group
    static_assert(N % (4 * kAhead) == 0, "");
    for (; piece < pieces; piece += stride) {
      f64x4 acc[KT][V];
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[i][j] = f64x4{0.0, 0.0, 0.0, 0.0};
      const u32 l = piece * A::kPlaces + V * place;
      const bool full = (piece + 1) * A::kPlaces <= length;
      const auto load = [&](const T* from, T (&x)[V]) {
        if (full) load_whole<T, V>(from, l, length, x);
        else load_few<T, V>(from, l, length, x);
      };
      T x[kAhead][V];
#pragma unroll
      for (u32 n = 0; n < kAhead; ++n) load(m.g + row(4 * n + group, k) * m.ldg, x[n]);
      for (u32 t0 = 0; t0 < N; t0 += 4 * kAhead) {
        T now[kAhead][V];
        __builtin_memcpy(now, x, sizeof(x));
        if (t0 + 4 * kAhead < N) {
#pragma unroll
          for (u32 n = 0; n < kAhead; ++n) load(m.g + row(t0 + 4 * (kAhead + n) + group, k) * m.ldg, x[n]);
        }
        double d[2][KT];
        const auto read = [&](u32 n) {
#pragma unroll
          for (int i = 0; i < KT; ++i) d[n & 1][i] = P[(16 * i + place) * S + t0 + 4 * n + group];
        };
        read(0);
#pragma unroll
        for (u32 n = 0; n < kAhead; ++n) {
          if (n + 1 < kAhead) read(n + 1);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const double v = (double)(float)now[n][j];
#pragma unroll
            for (int i = 0; i < KT; ++i) acc[i][j] = mma4(d[n & 1][i], v, acc[i][j]);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int i = 0; i < KT; ++i) {
        T was[4][V] = {};
        if (m.base) {
#pragma unroll
          for (int r = 0; r < 4; ++r) load(m.base + row(16 * i + 4 * r + group, k) * m.ldb, was[r]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const u32 s = 16 * i + 4 * r + group;
          T now[V];
#pragma unroll
          for (int j = 0; j < V; ++j) now[j] = once<T>(m.base ? keep * (double)(float)was[r][j] + acc[i][j][r] : acc[i][j][r]);
          if (s < k) store_few<T, V>(m.out + (size_t)s * m.ldo, l, length, now);
        }
      }
    }
  }
}
template <class T>
__device__ __forceinline__ Matrices<T> matrices_of(const Batch<const T>& g, const Batch<const T>& base, const Batch<T>& out, u32 party) {
  return {g.p + party * g.step, base.p ? base.p + party * base.step : nullptr, out.p + party * out.step, g.ld, base.ld, out.ld};
}
// `from`: P; of one tile and with steps the parts' sums, from which each block's first wavefront forms the polynomial itself, which takes it no
// longer than a launch (8 matrices of 16 x 4096 float32 13.5 us by three launches and 12.3 by two).
struct Polynomial {
  const double* from;
  u32 count;
  Steps steps;
  double scale, eps;
};
template <class T, int KT, bool TALL, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_apply(Batch<const T> g, Batch<const T> base, Batch<T> out, Polynomial poly, u32 k, u32 length, double keep,
                                                    u32 blocks, u32 parties, u32 first_block) {
  using A = Apply<KT, TALL>;
  __shared__ __align__(16) double P[A::N * A::S];
  const auto [party, part] = place_of_block(first_block + blockIdx.x, blocks, parties);
  if (party >= parties) return;
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const double* const from = poly.from + (size_t)party * poly.count * A::N * A::N;
  if (KT == 1 && poly.steps.count) {
    __shared__ StepRoom<1> held;
    __shared__ double room[1];
    if (wave == 0) {
      double sums[4];
      sum_parts(from, poly.count, 256, threadIdx.x, kWave, sums);
      steps_of<1>(poly.steps, 0, poly.steps.count, poly.scale, poly.eps, false, held, room, sums, [&](u32 i, u32 j, double v) { P[i * A::S + j] = v; });
    }
  } else {
#pragma unroll 8
    for (u32 i = threadIdx.x; i < A::N * A::N; i += kThreads) P[i / A::N * A::S + i % A::N] = from[i];
  }
  __syncthreads();
  apply<T, KT, TALL, WHOLE>(matrices_of(g, base, out, party), P, k, length, keep, part * kWaves + wave, blocks * kWaves);
}

// All of it for small matrices of one tile, by a block each and without a workspace. us a call by one launch and by three: 8 matrices of 4 x 256 float32
// 8 and 12, of 16 x 1024 16 and 13 (where the host waits for neither; its own part is 7 us less for one).
constexpr u32 kOneThreads = 512, kOneWaves = kOneThreads / kWave;
template <class T, bool TALL, bool WHOLE>
__global__ __launch_bounds__(kOneThreads) void k_update(Batch<const T> g, Batch<const T> base, Batch<T> out, u32 k, u32 length, Steps steps, double keep,
                                                        double scale, double eps) {
  constexpr int KT = 1;
  constexpr u32 N = 16 * KT, S = N + 2;
  __shared__ __align__(16) StepRoom<KT> held;
  __shared__ __align__(16) double sums[N * S];  // K's, and then P
  __shared__ double part[kOneWaves][1][256], room[16];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const Matrices<T> m = matrices_of(g, base, out, blockIdx.x);
  f64x4 acc[pairs_of<KT>()];
  gram<T, KT, TALL>(m.g, m.ldg, k, length, wave, (length + kChunk - 1) / kChunk, kOneWaves, wave, acc);
  gram_sums<KT, TALL, kOneWaves>(acc, wave, k, part, [&](u32 s, u32 t, double v) { sums[s * S + t] = v; });
  __syncthreads();
  int end = steps.end(0);
  if (wave == 0) {
    double own[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) own[e] = sums[(4 * e + threadIdx.x / 16) * S + threadIdx.x % 16];
    steps_of<KT>(steps, 0, end, end == steps.count ? scale : 1.0, eps, false, held, room, own, [&](u32 i, u32 j, double v) { sums[i * S + j] = v; });
  }
  __syncthreads();
  while (end < steps.count) {  // k_gram_again, k_steps and k_chain of the next part
    const int first = end;
    end = steps.end(first);
    gram_again<T, KT, TALL, 0, KT>(m.g, m.ldg, sums, k, length, wave, (length + 15) / 16, kOneWaves, acc);
    join_waves<kOneWaves>(acc, wave, 0, 0, 1, part[0][0]);
    if (wave == 0) {
      const u32 place = threadIdx.x % 16, group = threadIdx.x / 16;
      double own[4], R[4], next[4];
      int n = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        own[e] = part[0][0][64 * e + threadIdx.x];
        R[e] = sums[place * S + 4 * e + group];
      }
      steps_of<KT>(steps, first, end, end == steps.count ? scale : 1.0, eps, true, held, room, own, [&](u32, u32, double v) { next[n++] = v; });
      f64x4 chain = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int e = 0; e < 4; ++e) chain = mma4(R[e], next[e], chain);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u32 row = 4 * r + group;
        sums[end == steps.count && !TALL ? place * S + row : row * S + place] = chain[r];
      }
    }
    __syncthreads();
  }
  apply<T, KT, TALL, WHOLE>(m, sums, k, length, keep, wave, kOneWaves);
}

struct Shape {
  size_t parties, k, length;
  bool tall;
  u32 tiles() const { return k <= 16 ? 1 : k <= 32 ? 2 : k <= 48 ? 3 : k <= 64 ? 4 : k <= 96 ? 6 : 8; }
  size_t side() const { return 16 * tiles(); }
};
constexpr size_t kOneLength = 768;
struct Plan {  // parts 0: a block a matrix, and no workspace
  size_t parts, gram, poly, factor, chain, extra, total;
};
bool update_sizes(int type, size_t parties, size_t rows, size_t cols, Shape& s) {
  if (!valid_type(type) || parties > HAFLO_ADAPTER_MAX_PARTIES || rows < 1 || cols < 1 || rows > kMostCount || cols > kMostCount) return false;
  s = {parties, rows < cols ? rows : cols, rows < cols ? cols : rows, rows > cols};
  return s.k <= kMostShort && parties * s.length <= kMostLength;
}
Plan update_plan(const Shape& s) {
  Plan p = {};
  if (s.k <= 16 && s.length <= kOneLength) return p;
  // Parts of K_0's sums: enough for all compute units, and no more chunks to one than hide the first loads; but whoever joins the parts reads them
  // all. Calls, us, with at most an 8th / a 4th / a 16th of the chunks' number: 7 of 1001 x 37 float32 35.3 / 34.5 / 38.5, 8 of 64 x 4096 (parts of
  // 4 chunks and more: 32) 64.3 / 69.1 / 65.9, 2 of 64 x 10000 76.6 / 93.1 / 72.8 (40, 79 and 20 parts), 3001 x 100 121 / 109 / 153, 8 of
  // 4096 x 32 22.4 / 23.1 / 23.4. All matrices' parts: of 64 of 16 x 4096 28 with 1024, 23 with 512; 300 of them 67 and 72, with 256 77. Of more than 32 rows with 256 / 512 /
  // 1024: 16 of 64 x 4096 74 / 81 / 81, 64 of them 118 / 120 / 132, of 128 x 4096 506 / 525 / 553, of 48 x 2000 54 / 56 / 62; but 300 of 64 x 4096
  // 510 / 495 / 491, of 128 x 4096 2690 / 2500 / 2420.
  const u32 tiles = s.tiles();
  const size_t chunks = ceil_div(s.length, kChunk), want = ceil_div((size_t)(tiles <= 2 ? 512 : 256), s.parties ? s.parties : 1);
  size_t most = ceil_div(chunks, tiles <= 2 ? 8 : 4);
  if (tiles > 2 && tiles <= 4 && most > 20) most = 20;
  p.parts = want < most ? want : most;
  const size_t each = s.side() * s.side() * 8;
  p.gram = 0;
  p.poly = p.gram + s.parties * p.parts * each;
  p.chain = p.poly + s.parties * each;  // two, of lists that are cut
  p.factor = p.chain + 2 * s.parties * each;
  p.extra = p.factor + align256(s.parties * 8);
  p.total = s.k > 64 ? p.extra + 5 * s.parties * each : p.factor;
  return p;
}

// Where a list is cut: it may raise a direction by kMostWhole in one part (five steps of 3.4445 are 485, whose roundings are then below 2e-9 of what
// is greatest, a thirtieth of a rounding to float32), and each part of a longer one by kMostEach (three are 41). Steps' factors a + b x + c x^2 are taken at their
// greatest over what K's eigenvalues x can be: 0 .. `most`, and x (a + b x + c x^2)^2 after the step, whose slope is 0 where the factor
// or a + 3 b x + 5 c x^2 is.
constexpr double kMostWhole = 512.0, kMostEach = 48.0;
u32 cuts_of(const Steps& steps) {
  double grow[HAFLO_UPDATE_MAX_STEPS], most = 1.0;
  for (int i = 0; i < steps.count; ++i) {
    const double a = steps.c[i][0], b = steps.c[i][1], c = steps.c[i][2], last = most;
    const auto factor = [&](double x) { return a + x * (b + c * x); };
    double after = 0.0;
    grow[i] = 1.0;
    const auto look = [&](double x) {
      if (!(x >= 0.0 && x <= last)) return;
      const double f = fabs(factor(x));
      if (!(f <= grow[i])) grow[i] = f;
      if (!(x * f * f <= after)) after = x * f * f;
    };
    look(0.0);
    look(last);
    if (c != 0.0) {
      const double root = sqrt(9.0 * b * b - 20.0 * a * c);
      look(-b / (2.0 * c));
      look((-3.0 * b + root) / (10.0 * c));
      look((-3.0 * b - root) / (10.0 * c));
    } else if (b != 0.0) {
      look(-a / (3.0 * b));
    }
    most = after;
    if (!(grow[i] < HUGE_VAL && most < HUGE_VAL)) grow[i] = most = HUGE_VAL;
  }
  double whole = 1.0, part = 1.0;
  for (int i = 0; i < steps.count; ++i) whole *= grow[i];
  u32 cuts = 0;
  for (int i = 0; i < steps.count && !(whole <= kMostWhole); ++i) {
    part *= grow[i];
    if (i == 0 || part <= kMostEach) continue;
    cuts |= 1u << (i - 1);
    part = grow[i];
  }
  return cuts;
}

// scale P / (|G|_F + eps) of more than 64 rows, product by product
template <u32 N>
void large_steps(const Shape& s, const Plan& plan, const Steps& steps, double scale, double eps, bool again, double* to, char* ws, hipStream_t st) {
  const size_t each = s.parties * N * N * 8;
  const auto place = [&](int i) { return (double*)(ws + plan.extra + i * each); };
  double *const K = place(0), *const Q = place(1), *P = place(2), *const M = place(3), *spare = place(4);
  double* const factor = (double*)(ws + plan.factor);
  hipLaunchKernelGGL((k_gram_join<N>), dim3((unsigned)blocks_of(kSlices, s.parties)), dim3(join_threads<N>()), 0, st, (const double*)(ws + plan.gram), (u32)plan.parts,
                     (u32)s.parties, eps, (u32)again, K, factor);
  const auto run = [&](Products p, u32 jobs) {
    in_turns(blocks_of(jobs * large_tiles<N>(), s.parties), kWave,
             [&](u32 first, dim3 grid, dim3 block) { hipLaunchKernelGGL((k_products<N>), grid, block, 0, st, p, jobs, (u32)s.parties, first); });
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
  // (us a call with 512 / 768 / 1024 for all matrices: 64 of 16 x 4096 float32 22.5 / 23.3 / 27.6, 300 of them 77 / 72 / 71, 300 of 2000 x 32
  // 98 / 92 / 93, 64 of 64 x 4096 124 / 142 / 124)
  const size_t need = ceil_div(s.length, places), want = ceil_div((size_t)(s.tiles() <= 2 ? 768 : 512), s.parties);
  return (u32)(need < want ? need : want);
}

template <class T, int KT, bool TALL>
void update(const Batch<const T>& g, const Batch<const T>& base, const Batch<T>& out, const Shape& s, const Plan& plan, const Steps& steps, double keep,
            double scale, double eps, char* ws, hipStream_t st) {
  const u32 k = (u32)s.k, length = (u32)s.length;
  const bool whole = Apply<KT, TALL>::whole(k);
  if constexpr (KT == 1) {
    if (plan.parts == 0) {
      const dim3 grid((unsigned)s.parties), block(kOneThreads);
      if (whole) hipLaunchKernelGGL((k_update<T, TALL, true>), grid, block, 0, st, g, base, out, k, length, steps, keep, scale, eps);
      else hipLaunchKernelGGL((k_update<T, TALL, !TALL>), grid, block, 0, st, g, base, out, k, length, steps, keep, scale, eps);
      return;
    }
  }
  double *const sums = (double*)(ws + plan.gram), *const poly = (double*)(ws + plan.poly);
  in_turns(blocks_of(plan.parts, s.parties), kThreads, [&](u32 first, dim3 grid, dim3 block) {
    hipLaunchKernelGGL((k_gram<T, KT, TALL>), grid, block, 0, st, g, k, length, (u32)plan.parts, (u32)s.parties, sums, first);
  });
  const auto form = [&](const Steps& part, double by, bool again, double* to) {
    if constexpr (KT <= 4)
      hipLaunchKernelGGL((k_steps<KT>), dim3((unsigned)s.parties), dim3(step_threads<KT>()), 0, st, (const double*)sums, (u32)plan.parts, part, by, eps, (u32)again, to);
    else
      large_steps<16 * KT>(s, plan, part, by, eps, again, to, ws, st);
  };
  Polynomial from = {poly, 1, {}, scale, eps};
  if (steps.cuts) {
    constexpr u32 N = 16 * KT;
    double *R = (double*)(ws + plan.chain), *next = R + s.parties * N * N;
    for (int first = 0, end; first < steps.count; first = end) {
      end = steps.end(first);
      const bool last = end == steps.count;
      Steps part = {};
      for (; part.count < end - first; ++part.count)
        for (int j = 0; j < 3; ++j) part.c[part.count][j] = steps.c[first + part.count][j];
      if (first == 0) {
        form(part, 1.0, false, R);
        continue;
      }
      // (few enough lanes for one launch each, as in k_gram_join)
      hipLaunchKernelGGL((k_gram_again<T, KT, TALL>), dim3((unsigned)blocks_of(plan.parts, s.parties)), dim3(kThreads), 0, st, g, (const double*)R, k, length,
                         (u32)plan.parts, (u32)s.parties, sums);
      form(part, last ? scale : 1.0, true, poly);
      hipLaunchKernelGGL((k_chain<N>), dim3((unsigned)blocks_of(KT * KT, s.parties)), dim3(kWave), 0, st, (const double*)R, (const double*)poly, (u32)s.parties,
                         (u32)(last && !TALL), next);
      double* const was = R;
      R = next;
      next = was;
    }
    from.from = R;
  } else if constexpr (KT == 1) {
    from = {sums, (u32)plan.parts, steps, scale, eps};
  } else {
    form(steps, scale, false, poly);
  }
  const u32 blocks = apply_blocks(s, kWaves * Apply<KT, TALL>::kPlaces);
  in_turns(blocks_of(blocks, s.parties), kThreads, [&](u32 first, dim3 grid, dim3 block) {
    if (whole) hipLaunchKernelGGL((k_apply<T, KT, TALL, true>), grid, block, 0, st, g, base, out, from, k, length, keep, blocks, (u32)s.parties, first);
    else hipLaunchKernelGGL((k_apply<T, KT, TALL, !TALL>), grid, block, 0, st, g, base, out, from, k, length, keep, blocks, (u32)s.parties, first);
  });
}
template <class T, bool TALL>
void update(const Batch<const T>& g, const Batch<const T>& base, const Batch<T>& out, const Shape& s, const Plan& plan, const Steps& steps, double keep,
            double scale, double eps, char* ws, hipStream_t st) {
  switch (s.tiles()) {
    case 1: return update<T, 1, TALL>(g, base, out, s, plan, steps, keep, scale, eps, ws, st);
    case 2: return update<T, 2, TALL>(g, base, out, s, plan, steps, keep, scale, eps, ws, st);
    case 3: return update<T, 3, TALL>(g, base, out, s, plan, steps, keep, scale, eps, ws, st);
    case 4: return update<T, 4, TALL>(g, base, out, s, plan, steps, keep, scale, eps, ws, st);
    case 6: return update<T, 6, TALL>(g, base, out, s, plan, steps, keep, scale, eps, ws, st);
    default: return update<T, 8, TALL>(g, base, out, s, plan, steps, keep, scale, eps, ws, st);
  }
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
  list.cuts = cuts_of(list);
  if (parties == 0) return HAFLO_OK;
  if (!d_g || ldg < cols || !d_out || ldo < cols || (d_base && ldb < cols) || ldo > kMostDistance) return HAFLO_EINVAL;
  // matrices of the result over each other: neither behind one another nor with rows between each other's
  if (parties > 1 && step_o < (rows - 1) * ldo + cols && !(step_o >= cols && step_o <= ldo && (parties - 1) * step_o + cols <= ldo)) return HAFLO_EINVAL;
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
