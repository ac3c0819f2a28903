// The norms around a block of a model, with the gate and the residual stream between them, and their gradients.
//
//   forward   p = f q post (q = 1 / sqrt(mean f^2 + eps); p = f without a norm behind the block)
//             r = scale x + gate p,   h = r t pre,   t = 1 / sqrt(mean r^2 + eps)
//   backward  a = dh pre,  D = dr + t (a - r^ mean(a r^)),  r^ = r t          dx = scale D,  dpre = sum over rows of dh r^
//             b = D gate post,  df = q (b - f^ mean(b f^)),  f^ = f q         dgate = D p,  dpost = sum over rows of D gate f^
//
// A lane holds eight columns of a row and a group of lanes the row, so that each matrix is read once. Means of squares are
// taken in 64 bits: every float32 has a square there. The way back forms p and r again from x, f and both roots, which is
// fewer bytes than reading them, and keeps its columns' sums over all rows that a block takes.
#include "local_common.hpp"

using namespace haflo::local;

namespace {

constexpr u32 kThreads = 256;
constexpr u32 kBlockLanes = 512;                      // of a block, of rows that take no more
constexpr u32 kMostLanes = 1024;                      // of one row
constexpr size_t kRowCols = (size_t)kMostLanes * 8;   // columns of a row that lanes hold; longer rows are read again
constexpr size_t kNormBlocks = 1024, kBackBlocks = 512;
constexpr u32 kTileCols = kThreads * 8;               // of the long rows' way back

enum Mode { kStream = 0, kGated = 1, kFullGate = 2 };  // r = x; a block's f with a gate by columns or none; a gate for every element

template <class T>
struct Norm {
  const T *x, *f, *gate;
  size_t ldx, ldf, ldg;
  const float *gate_cols, *post, *pre;
  u32 rows, cols;
  float scale;
  double eps, per_col;  // 1 / cols
  bool apart;           // no result lies over an operand, and rows have eight elements

  // a vector of a row, on its way and as it is
  __device__ __forceinline__ Vec8<T> ask(const T* row, u32 col) const { return apart ? load_clamped(row, col, cols) : load_cols(row, col, cols); }
  __device__ __forceinline__ void have(Vec8<T>& v, u32 col) const {
    if (apart) settle(v, col, cols);
  }
};

struct Eight {
  float v[8];
};
template <class T>
__device__ __forceinline__ Eight floats(const Vec8<T>& a) {
  Eight e;
#pragma unroll
  for (int j = 0; j < 8; ++j) e.v[j] = (float)a.get(j);
  return e;
}
template <class T>
__device__ __forceinline__ Vec8<T> rounded(const Eight& e) {
  Vec8<T> a = {};
#pragma unroll
  for (int j = 0; j < 8; ++j) a.set(j, (T)e.v[j]);
  return a;
}
__device__ __forceinline__ Eight gains(const float* g, u32 col, u32 cols) {  // ones without any
  if (g) return floats(load_cols(g, col, cols));
  Eight e;
#pragma unroll
  for (int j = 0; j < 8; ++j) e.v[j] = 1.0f;
  return e;
}
__device__ __forceinline__ double squares(const Eight& e) {
  double s = 0.0;
#pragma unroll
  for (int j = 0; j < 8; ++j) s += (double)e.v[j] * (double)e.v[j];
  return s;
}
// The sum over a row's group of `lanes` lanes, a power of two, the same bits in each. Groups of more than a wavefront take turns at two
// places in LDS: a wavefront is at most one sum ahead. All of a block's groups call it together.
template <class S>
struct GroupSum {
  S (*parts)[kMostLanes / kWave];
  u32 lanes, turn;
  __device__ __forceinline__ S operator()(S v) {
    v = lanes_join(v, lanes, [](S a, S b) { return a + b; });
    if (lanes > kWave) {
      turn ^= 1;
      const u32 wave = threadIdx.x / kWave, waves = lanes / kWave, first = wave & ~(waves - 1);
      if (lane_id() == 0) parts[turn][wave] = v;
      __syncthreads();
      v = parts[turn][first];
      for (u32 w = 1; w < waves; ++w) v += parts[turn][first + w];
    }
    return v;
  }
};
__device__ __forceinline__ float root(double sum, double per_col, double eps) { return (float)(1.0 / sqrt(sum * per_col + eps)); }

// f^ and r of eight columns; f^ is f where q is 1
template <int MODE>
__device__ __forceinline__ void join_stream(const Eight& x, Eight& f, const Eight& post, const Eight& gate, float q, float scale, Eight& p, Eight& r) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    f.v[j] *= q;
    p.v[j] = f.v[j] * post.v[j];
    r.v[j] = MODE == kStream ? x.v[j] : scale * x.v[j] + gate.v[j] * p.v[j];
  }
}

// A block takes every gridDim.x-th set of rows, so that the gains are read once, and asks for the next rows before it forms the means.
// Memory bounds it: 16384 x 4096 bfloat16 call after call 114 to 122 us, 4.4 to 4.7 TB/s (a copy of 4 GiB 4.9); float32 8192 x 4096 105 us, 5.1;
// 3001 x 1001 float16 with a gate for every element 11 us, 2.7 TB/s, where a launch and two dependent means are half of it; one row 4 us.
template <class T, int MODE, int MOST>
__global__ __launch_bounds__(MOST) void k_norm(Norm<T> n, u32 lanes, T* r_out, size_t ldr, T* h_out, size_t ldh, float* rstd) {
  __shared__ double parts[2][kMostLanes / kWave];
  GroupSum<double> sum = {parts, lanes, 0};
  const u32 groups = blockDim.x / lanes, col = threadIdx.x % lanes * 8;
  const Eight post = gains(n.post, col, n.cols), pre = gains(n.pre, col, n.cols), by_cols = gains(n.gate_cols, col, n.cols);
  const u64 step = (u64)gridDim.x * groups;
  u64 mine = (u64)blockIdx.x * groups + threadIdx.x / lanes;
  Vec8<T> xn, fn, gn;
  const auto ask = [&](u64 row) {
    row = row < n.rows ? row : n.rows - 1;
    xn = n.ask(n.x + row * n.ldx, col);
    if (MODE != kStream) fn = n.ask(n.f + row * n.ldf, col);
    if (MODE == kFullGate) gn = n.ask(n.gate + row * n.ldg, col);
  };
  ask(mine);
  for (u64 base = (u64)blockIdx.x * groups; base < n.rows; base += step, mine += step) {
    const bool live = mine < n.rows;
    const u64 row = mine;
    Vec8<T> xv = xn, fv = fn, gv = gn;
    if (base + step < n.rows) ask(mine + step);
    n.have(xv, col);
    if (MODE != kStream) n.have(fv, col);
    if (MODE == kFullGate) n.have(gv, col);
    Eight f = floats(fv), p, r;
    float q = 1.0f, t = 1.0f;
    if (MODE != kStream && n.post) q = root(sum(squares(f)), n.per_col, n.eps);
    join_stream<MODE>(floats(xv), f, post, MODE == kFullGate ? floats(gv) : by_cols, q, n.scale, p, r);
    if (n.pre) t = root(sum(squares(r)), n.per_col, n.eps);
    if (!live) continue;
    if (MODE != kStream) store_cols(r_out + row * ldr, col, n.cols, rounded<T>(r));
    if (n.pre) {
#pragma unroll
      for (int j = 0; j < 8; ++j) r.v[j] = r.v[j] * t * pre.v[j];  // (t pre may be below the normal numbers)
      store_cols(h_out + row * ldh, col, n.cols, rounded<T>(r));
    }
    if (col == 0) {
      rstd[row] = q;
      rstd[n.rows + row] = t;
    }
  }
}

// The same for rows that the lanes do not hold: a block takes a row, and reads it once for each mean and once for the results
// (4096 x 20000 bfloat16 228 us, 2.9 TB/s of what has to be read and written).
template <class T, int MODE>
__global__ __launch_bounds__(kMostLanes) void k_norm_long(Norm<T> n, T* r_out, size_t ldr, T* h_out, size_t ldh, float* rstd) {
  __shared__ double parts[2][kMostLanes / kWave];
  GroupSum<double> sum = {parts, kMostLanes, 0};
  for (u64 row = blockIdx.x; row < n.rows; row += gridDim.x) {
    float q = 1.0f, t = 1.0f;
    const auto stream = [&](u32 col) {
      Eight f = {}, gate = {}, p, r;
      if (MODE != kStream) f = floats(load_cols(n.f + row * n.ldf, col, n.cols));
      if (MODE != kStream) gate = MODE == kFullGate ? floats(load_cols(n.gate + row * n.ldg, col, n.cols)) : gains(n.gate_cols, col, n.cols);
      join_stream<MODE>(floats(load_cols(n.x + row * n.ldx, col, n.cols)), f, gains(n.post, col, n.cols), gate, q, n.scale, p, r);
      return r;
    };
    if (MODE != kStream && n.post) {
      double s = 0.0;
      for (u32 col = threadIdx.x * 8; col < n.cols; col += kRowCols) s += squares(floats(load_cols(n.f + row * n.ldf, col, n.cols)));
      q = root(sum(s), n.per_col, n.eps);
    }
    if (n.pre) {
      double s = 0.0;
      for (u32 col = threadIdx.x * 8; col < n.cols; col += kRowCols) s += squares(stream(col));
      t = root(sum(s), n.per_col, n.eps);
    }
    for (u32 col = threadIdx.x * 8; col < n.cols; col += kRowCols) {
      Eight r = stream(col);
      if (MODE != kStream) store_cols(r_out + row * ldr, col, n.cols, rounded<T>(r));
      if (n.pre) {
        const Eight pre = gains(n.pre, col, n.cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) r.v[j] = r.v[j] * t * pre.v[j];
        store_cols(h_out + row * ldh, col, n.cols, rounded<T>(r));
      }
    }
    if (threadIdx.x == 0) {
      rstd[row] = q;
      rstd[n.rows + row] = t;
    }
  }
}

template <class T>
struct Back {
  const T *dh, *dr;
  size_t lddh, lddr;
  const float* rstd;
  T *dx, *df, *dgate;
  size_t lddx, lddf, lddg;
  float* sums;   // of the block's gains and of dpre: blocks x width each
  u32 width;     // of a row of them
};
// Eight columns of a row on the way back: as they are loaded, and up to the means.
template <class T, int MODE>
struct BackIn {
  Vec8<T> x, f, gate, dh, dr;
  float q, t;
  __device__ __forceinline__ void load(const Norm<T>& n, const Back<T>& b, u64 row, u32 col) {
    row = row < n.rows ? row : n.rows - 1;
    x = n.ask(n.x + row * n.ldx, col);
    if (MODE != kStream) f = n.ask(n.f + row * n.ldf, col);
    if (MODE == kFullGate) gate = n.ask(n.gate + row * n.ldg, col);
    dh = dr = Vec8<T>{};
    if (n.pre) dh = n.ask(b.dh + row * b.lddh, col);
    if (b.dr) dr = n.ask(b.dr + row * b.lddr, col);
    q = b.rstd[row];
    t = b.rstd[n.rows + row];
  }
};
struct BackRow {
  Eight f, unit, gate, dh, dr;  // f^ (f without a norm), r^
  float q, t;
};
template <int MODE, class T>
__device__ __forceinline__ BackRow back_row(BackIn<T, MODE> in, const Norm<T>& n, u32 col, const Eight& post, const Eight& by_cols) {
  BackRow v;
  n.have(in.x, col);
  if (MODE != kStream) n.have(in.f, col);
  if (MODE == kFullGate) n.have(in.gate, col);
  n.have(in.dh, col);
  n.have(in.dr, col);
  v.f = MODE == kStream ? Eight{} : floats(in.f);
  v.gate = MODE == kFullGate ? floats(in.gate) : by_cols;
  v.q = in.q;
  v.t = in.t;
  Eight p;
  join_stream<MODE>(floats(in.x), v.f, post, v.gate, v.q, n.scale, p, v.unit);
#pragma unroll
  for (int j = 0; j < 8; ++j) v.unit.v[j] *= v.t;
  v.dh = floats(in.dh);
  v.dr = floats(in.dr);
  return v;
}
// the first mean's terms, and from it to D: v.dr
__device__ __forceinline__ float stream_terms(const BackRow& v, const Eight& pre) {
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) s += v.dh.v[j] * pre.v[j] * v.unit.v[j];
  return s;
}
__device__ __forceinline__ void stream_grad(BackRow& v, const Eight& pre, float mean) {
#pragma unroll
  for (int j = 0; j < 8; ++j) v.dr.v[j] += v.t * (v.dh.v[j] * pre.v[j] - v.unit.v[j] * mean);
}
// the second mean's terms
__device__ __forceinline__ float block_terms(const BackRow& v, const Eight& post) {
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) s += v.dr.v[j] * v.gate.v[j] * post.v[j] * v.f.v[j];
  return s;
}
// Sums over rows: of D f^, or of D gate f^ with a gate for every element, and of dh r^. A gate by columns and the gain behind the block
// are the same for all rows, so that both their gradients are the first sum's.
struct Sums {
  Eight block, pre;
};
template <class T, int MODE>
__device__ __forceinline__ void back_store(const Norm<T>& n, const Back<T>& b, u64 row, u32 col, const BackRow& v, const Eight& post, float mean, Sums& s) {
  Eight e;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    s.pre.v[j] += v.dh.v[j] * v.unit.v[j];
    if (MODE != kStream) s.block.v[j] += (MODE == kFullGate ? v.dr.v[j] * v.gate.v[j] : v.dr.v[j]) * v.f.v[j];
    e.v[j] = MODE == kStream ? v.dr.v[j] : n.scale * v.dr.v[j];
  }
  if (b.dx) store_cols(b.dx + row * b.lddx, col, n.cols, rounded<T>(e));
  if (MODE != kStream && b.df) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float dp = v.dr.v[j] * v.gate.v[j];
      e.v[j] = n.post ? v.q * (dp * post.v[j] - v.f.v[j] * mean) : dp;
    }
    store_cols(b.df + row * b.lddf, col, n.cols, rounded<T>(e));
  }
  if (MODE == kFullGate && b.dgate) {
#pragma unroll
    for (int j = 0; j < 8; ++j) e.v[j] = v.dr.v[j] * (v.f.v[j] * post.v[j]);
    store_cols(b.dgate + row * b.lddg, col, n.cols, rounded<T>(e));
  }
}

// The gains lie in LDS, as registers are for the row and for the next one, which is asked for before the means are formed (with the gains in
// registers 140 of them left a compute unit one block of 512 lanes: 16384 x 4096 bfloat16 233 us). Memory bounds it: that case 165 us, 4.9 TB/s.
template <class T, int MODE, int MOST>
__global__ __launch_bounds__(MOST, 4) void k_norm_back(Norm<T> n, Back<T> b, u32 lanes) {
  __shared__ float parts[2][kMostLanes / kWave];
  __shared__ __align__(16) float held[3][MOST * 8];
  GroupSum<float> sum = {parts, lanes, 0};
  const u32 groups = blockDim.x / lanes, group = threadIdx.x / lanes, col = threadIdx.x % lanes * 8;
  if (group == 0) {
    store_wide(held[0] + col, rounded<float>(gains(n.post, col, n.cols)));
    store_wide(held[1] + col, rounded<float>(gains(n.pre, col, n.cols)));
    store_wide(held[2] + col, rounded<float>(gains(n.gate_cols, col, n.cols)));
  }
  const auto gain = [&](int which) { return floats(*(const Vec8<float>*)(held[which] + col)); };
  const u64 step = (u64)gridDim.x * groups;
  u64 mine = (u64)blockIdx.x * groups + group;
  Sums s = {};
  constexpr bool kEarly = sizeof(T) == 2 && MODE != kFullGate;  // (where the next row's registers are there)
  BackIn<T, MODE> next;
  if (kEarly) next.load(n, b, mine, col);
  __syncthreads();
  for (u64 base = (u64)blockIdx.x * groups; base < n.rows; base += step, mine += step) {
    if (!kEarly) next.load(n, b, mine, col);
    BackRow v = back_row(next, n, col, gain(0), MODE == kFullGate ? Eight{} : gain(2));
    if (kEarly && base + step < n.rows) next.load(n, b, mine + step, col);
    if (n.pre) {
      const float mean = sum(stream_terms(v, gain(1))) * (float)n.per_col;
      stream_grad(v, gain(1), mean);
    }
    const float mean = MODE != kStream && n.post ? sum(block_terms(v, gain(0))) * (float)n.per_col : 0.0f;
    if (mine < n.rows) back_store<T, MODE>(n, b, mine, col, v, gain(0), mean, s);
  }
  // the groups' sums of the same columns, in their order
  Eight* const mine_of[2] = {&s.block, &s.pre};
  if (groups > 1) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) store_wide(held[i] + threadIdx.x * 8, rounded<float>(*mine_of[i]));
    __syncthreads();
    if (group != 0) return;
    for (u32 g = 1; g < groups; ++g)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const Eight other = floats(*(const Vec8<float>*)(held[i] + (g * lanes + threadIdx.x) * 8));
#pragma unroll
        for (int j = 0; j < 8; ++j) mine_of[i]->v[j] += other.v[j];
      }
  }
  if (col < b.width)
#pragma unroll
    for (int i = 0; i < 2; ++i) store_wide(b.sums + ((size_t)i * gridDim.x + blockIdx.x) * b.width + col, rounded<float>(*mine_of[i]));
}

// Long rows: both means of a row, by one block, which reads the row once for each (with k_norm_back_long, 4096 x 20000 bfloat16, 460 us: the
// row is read three times, at 2.1 TB/s of what has to be moved once).
template <class T, int MODE>
__global__ __launch_bounds__(kMostLanes) void k_norm_means(Norm<T> n, Back<T> b, float* means) {
  __shared__ float parts[2][kMostLanes / kWave];
  GroupSum<float> sum = {parts, kMostLanes, 0};
  for (u64 row = blockIdx.x; row < n.rows; row += gridDim.x) {
    float first = 0.0f, second = 0.0f;
    // `step` 0: the first mean's terms of eight columns; 1: the second's, with the first mean
    const auto terms = [&](u32 col, int step) {
      const Eight post = gains(n.post, col, n.cols), pre = gains(n.pre, col, n.cols);
      BackIn<T, MODE> in;
      in.load(n, b, row, col);
      BackRow v = back_row(in, n, col, post, gains(n.gate_cols, col, n.cols));
      if (step == 0) return stream_terms(v, pre);
      if (n.pre) stream_grad(v, pre, first);
      return block_terms(v, post);
    };
    if (n.pre) {
      float s = 0.0f;
      for (u32 col = threadIdx.x * 8; col < n.cols; col += kRowCols) s += terms(col, 0);
      first = sum(s) * (float)n.per_col;
    }
    if (MODE != kStream && n.post) {
      float s = 0.0f;
      for (u32 col = threadIdx.x * 8; col < n.cols; col += kRowCols) s += terms(col, 1);
      second = sum(s) * (float)n.per_col;
    }
    if (threadIdx.x == 0) {
      means[row] = first;
      means[n.rows + row] = second;
    }
  }
}
// Long rows with their means: a block takes eight columns a lane of every `blocks`-th row.
template <class T, int MODE>
__global__ __launch_bounds__(kThreads) void k_norm_back_long(Norm<T> n, Back<T> b, const float* means, u32 blocks, u32 first_block) {
  const u32 block = first_block + blockIdx.x, part = block % blocks, col = block / blocks * kTileCols + threadIdx.x * 8;
  if (col >= n.cols) return;
  const Eight post = gains(n.post, col, n.cols), pre = gains(n.pre, col, n.cols), by_cols = gains(n.gate_cols, col, n.cols);
  Sums s = {};
  for (u64 row = part; row < n.rows; row += blocks) {
    BackIn<T, MODE> in;
    in.load(n, b, row, col);
    BackRow v = back_row(in, n, col, post, by_cols);
    if (n.pre) stream_grad(v, pre, means[row]);
    back_store<T, MODE>(n, b, row, col, v, post, means[n.rows + row], s);
  }
  const Eight* const held[2] = {&s.block, &s.pre};
#pragma unroll
  for (int i = 0; i < 2; ++i) store_wide(b.sums + ((size_t)i * blocks + part) * b.width + col, rounded<float>(*held[i]));
}

// The blocks' sums of 64 columns: sixteen wavefronts take a part of the blocks each, eight loads on their way at a time (512 blocks' sums of
// 4096 columns 5 us; by four wavefronts, load after load, 42).
constexpr u32 kJoinWaves = 16;
struct Joined {
  float *post, *gate, *pre;
  const float *of_post, *of_gate;  // what the first sum is multiplied by for them, or NULL
};
__global__ __launch_bounds__(kJoinWaves * kWave) void k_norm_join(const float* sums, u32 blocks, u32 width, u32 cols, Joined to, u32 first_block) {
  __shared__ float parts[kJoinWaves][kWave];
  const u32 tiles = (cols + kWave - 1) / kWave, block = first_block + blockIdx.x, which = block / tiles, lane = lane_id(), wave = threadIdx.x / kWave;
  const u32 col = block % tiles * kWave + lane;
  if (which == 0 ? !to.post && !to.gate : !to.pre) return;
  const u32 first = (u32)((u64)blocks * wave / kJoinWaves), end = (u32)((u64)blocks * (wave + 1) / kJoinWaves);
  const float* const from = sums + (size_t)which * blocks * width + (col < cols ? col : cols - 1);
  float s = 0.0f;
  u32 i = first;
  for (; i + 8 <= end; i += 8) {
    float v[8];
#pragma unroll
    for (u32 j = 0; j < 8; ++j) v[j] = from[(size_t)(i + j) * width];
    s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  }
  for (; i < end; ++i) s += from[(size_t)i * width];
  parts[wave][lane] = s;
  __syncthreads();
  if (wave != 0 || col >= cols) return;
  s = 0.0f;
#pragma unroll
  for (u32 w = 0; w < kJoinWaves; ++w) s += parts[w][lane];
  if (which == 1) {
    to.pre[col] = s;
  } else {
    if (to.post) to.post[col] = to.of_post ? s * to.of_post[col] : s;
    if (to.gate) to.gate[col] = to.of_gate ? s * to.of_gate[col] : s;
  }
}

u32 lanes_of(size_t cols) {
  u32 lanes = 1;
  while ((size_t)lanes * 8 < cols) lanes *= 2;
  return lanes;
}
// Several rows to a block where there are many: their columns' sums are joined in LDS before k_norm_join reads them (3001 x 1001 float16, a row
// to a block of 128 lanes 29 us, four rows to one of 512 lanes 22). Few rows get a block each.
u32 threads_of(u32 lanes, size_t rows) {
  u32 threads = lanes < (u32)kWave ? (u32)kWave : lanes;
  while (threads < kBlockLanes && ceil_div(rows, threads / lanes) > kBackBlocks) threads *= 2;
  return threads;
}
size_t row_blocks(size_t rows, size_t cols, size_t most) {
  const u32 lanes = lanes_of(cols);
  const size_t need = ceil_div(rows, threads_of(lanes, rows) / lanes);
  return need < most ? need : most;
}
struct Plan {
  size_t blocks, width, means, total;
};
Plan back_plan(size_t rows, size_t cols) {
  Plan p;
  p.width = ceil_div(cols, 8) * 8;
  p.blocks = cols <= kRowCols ? row_blocks(rows, cols, kBackBlocks) : rows < 64 ? rows : 64;
  p.means = align256(2 * p.blocks * p.width * 4);
  p.total = p.means + (cols <= kRowCols ? 0 : align256(2 * rows * 4));
  return p;
}
constexpr double kLeastEps = 0x1p-254;  // a row of zeros has the root's reciprocal 2^127
bool finite_scale(double scale) { return fabs((float)scale) < HUGE_VAL; }
bool norm_sizes(int type, size_t rows, size_t cols) { return valid_type(type) && rows <= kMostCount && cols >= 1 && cols <= kMostCount; }

template <class T, int MODE>
void norm(const Norm<T>& n, T* r, size_t ldr, T* h, size_t ldh, float* rstd, hipStream_t st) {
  if (n.cols > kRowCols) {
    hipLaunchKernelGGL((k_norm_long<T, MODE>), dim3((unsigned)(n.rows < kNormBlocks ? n.rows : kNormBlocks)), dim3(kMostLanes), 0, st, n, r, ldr, h, ldh,
                       rstd);
    return;
  }
  const u32 lanes = lanes_of(n.cols), threads = threads_of(lanes, n.rows);
  const dim3 grid((unsigned)row_blocks(n.rows, n.cols, kNormBlocks)), block(threads);
  if (threads > kBlockLanes) hipLaunchKernelGGL((k_norm<T, MODE, kMostLanes>), grid, block, 0, st, n, lanes, r, ldr, h, ldh, rstd);
  else hipLaunchKernelGGL((k_norm<T, MODE, kBlockLanes>), grid, block, 0, st, n, lanes, r, ldr, h, ldh, rstd);
}
template <class T, int MODE>
void norm_back(const Norm<T>& n, const Back<T>& b, const Plan& plan, char* ws, hipStream_t st) {
  if (n.cols > kRowCols) {
    float* const means = (float*)(ws + plan.means);
    hipLaunchKernelGGL((k_norm_means<T, MODE>), dim3((unsigned)(n.rows < kNormBlocks ? n.rows : kNormBlocks)), dim3(kMostLanes), 0, st, n, b, means);
    in_turns(plan.blocks * ceil_div(n.cols, kTileCols), kThreads, [&](u32 first, dim3 grid, dim3 block) {
      hipLaunchKernelGGL((k_norm_back_long<T, MODE>), grid, block, 0, st, n, b, (const float*)means, (u32)plan.blocks, first);
    });
    return;
  }
  const u32 lanes = lanes_of(n.cols), threads = threads_of(lanes, n.rows);
  const dim3 grid((unsigned)plan.blocks), block(threads);
  if (threads > kBlockLanes) hipLaunchKernelGGL((k_norm_back<T, MODE, kMostLanes>), grid, block, 0, st, n, b, lanes);
  else hipLaunchKernelGGL((k_norm_back<T, MODE, kBlockLanes>), grid, block, 0, st, n, b, lanes);
}

}  // namespace

extern "C" {

int haflo_residual_norm(int type, const void* d_x, size_t ldx, const void* d_f, size_t ldf, const float* d_post, const void* d_gate, size_t ldg,
                        const float* d_gate_cols, const float* d_pre, size_t rows, size_t cols, double scale, double eps, void* d_r, size_t ldr,
                        void* d_h, size_t ldh, float* d_rstd, void* stream) {
  if (!norm_sizes(type, rows, cols) || !(eps >= kLeastEps && eps < HUGE_VAL) || !finite_scale(scale)) return HAFLO_EINVAL;
  if (rows == 0) return HAFLO_OK;
  if ((!d_f && (!d_pre || d_post || d_gate || d_gate_cols || scale != 1.0)) || (d_gate && d_gate_cols)) return HAFLO_EINVAL;
  if (!d_x || ldx < cols || (d_f && (ldf < cols || !d_r || ldr < cols)) || (d_gate && ldg < cols) || (d_pre && (!d_h || ldh < cols)) || !d_rstd)
    return HAFLO_EINVAL;
  const struct {
    const void* p;
    size_t ld;
  } in[3] = {{d_x, ldx}, {d_f, ldf}, {d_gate, ldg}}, out[2] = {{d_f ? d_r : nullptr, ldr}, {d_pre ? d_h : nullptr, ldh}};
  bool apart = cols >= 8;
  for (const auto& o : out)
    for (const auto& i : in) {
      if (o.p && !in_place(i.p, i.ld, o.p, o.ld, rows)) return HAFLO_EINVAL;
      apart = apart && !(o.p && o.p == i.p);
    }
  if (out[0].p && out[0].p == out[1].p) return HAFLO_EINVAL;
  const hipStream_t st = (hipStream_t)stream;
  HAFLO_LOCAL_TYPES(type, {
    const Norm<T> n = {(const T*)d_x, (const T*)d_f, (const T*)d_gate, ldx, ldf, ldg, d_gate_cols, d_post, d_pre, (u32)rows, (u32)cols, (float)scale,
                       eps, 1.0 / (double)cols, apart};
    if (!d_f) norm<T, kStream>(n, (T*)d_r, ldr, (T*)d_h, ldh, d_rstd, st);
    else if (d_gate) norm<T, kFullGate>(n, (T*)d_r, ldr, (T*)d_h, ldh, d_rstd, st);
    else norm<T, kGated>(n, (T*)d_r, ldr, (T*)d_h, ldh, d_rstd, st);
  });
  return launched();
}

size_t haflo_residual_norm_workspace_bytes(int type, size_t rows, size_t cols) {
  return norm_sizes(type, rows, cols) ? back_plan(rows, cols).total : (size_t)-1;
}

int haflo_residual_norm_backward(int type, const void* d_dh, size_t lddh, const void* d_dr, size_t lddr, const void* d_x, size_t ldx, const void* d_f,
                                 size_t ldf, const float* d_post, const void* d_gate, size_t ldg, const float* d_gate_cols, const float* d_pre,
                                 const float* d_rstd, size_t rows, size_t cols, double scale, void* d_dx, size_t lddx, void* d_df, size_t lddf,
                                 void* d_dgate, size_t lddg, float* d_dgate_cols, float* d_dpost, float* d_dpre, void* d_workspace,
                                 size_t workspace_bytes, void* stream) {
  if (!norm_sizes(type, rows, cols) || !finite_scale(scale)) return HAFLO_EINVAL;
  if ((d_dpost && !d_post) || (d_dpre && !d_pre) || (d_dgate_cols && !d_gate_cols)) return HAFLO_EINVAL;  // gradients of what is not there
  // (matrices of no rows may have no address)
  if (rows && ((!d_f && (!d_pre || d_post || d_gate || d_gate_cols || scale != 1.0)) || (d_gate && d_gate_cols) || (d_dgate && !d_gate) || (d_df && !d_f)))
    return HAFLO_EINVAL;
  if (rows && (!d_x || ldx < cols || (d_f && ldf < cols) || (d_gate && ldg < cols) || (d_pre && (!d_dh || lddh < cols)) || (d_dr && lddr < cols) || !d_rstd ||
               (d_dx && lddx < cols) || (d_df && lddf < cols) || (d_dgate && lddg < cols)))
    return HAFLO_EINVAL;
  const struct {
    const void* p;
    size_t ld;
  } in[5] = {{d_x, ldx}, {d_f, ldf}, {d_gate, ldg}, {d_pre ? d_dh : nullptr, lddh}, {d_dr, lddr}}, out[3] = {{d_dx, lddx}, {d_df, lddf}, {d_dgate, lddg}};
  bool apart = cols >= 8;
  for (int o = 0; o < 3; ++o) {
    for (const auto& i : in) {
      if (out[o].p && !in_place(i.p, i.ld, out[o].p, out[o].ld, rows)) return HAFLO_EINVAL;
      apart = apart && !(out[o].p && out[o].p == i.p);
    }
    if (out[o].p && (out[o].p == out[(o + 1) % 3].p)) return HAFLO_EINVAL;
  }
  const Plan plan = back_plan(rows, cols);
  if (!enough(d_workspace, workspace_bytes, plan.total)) return HAFLO_EINVAL;
  char* const ws = (char*)d_workspace;
  const hipStream_t st = (hipStream_t)stream;
  if (rows) HAFLO_LOCAL_TYPES(type, {
    const Norm<T> n = {(const T*)d_x, (const T*)d_f, (const T*)d_gate, ldx, ldf, ldg, d_gate_cols, d_post, d_pre, (u32)rows, (u32)cols, (float)scale,
                       0.0, 1.0 / (double)cols, apart};
    const Back<T> b = {(const T*)d_dh, (const T*)d_dr, lddh, lddr, d_rstd, (T*)d_dx, (T*)d_df, (T*)d_dgate, lddx, lddf, lddg, (float*)ws, (u32)plan.width};
    if (!d_f) norm_back<T, kStream>(n, b, plan, ws, st);
    else if (d_gate) norm_back<T, kFullGate>(n, b, plan, ws, st);
    else norm_back<T, kGated>(n, b, plan, ws, st);
  });
  if (d_dpost || d_dgate_cols || d_dpre)
    in_turns(2 * ceil_div(cols, kWave), kJoinWaves * kWave, [&](u32 first, dim3 grid, dim3 block) {
      hipLaunchKernelGGL(k_norm_join, grid, block, 0, st, (const float*)ws, (u32)(rows ? plan.blocks : 0), (u32)plan.width, (u32)cols,
                         Joined{d_dpost, d_dgate_cols, d_dpre, rows ? d_gate_cols : nullptr, rows ? d_post : nullptr}, first);
    });
  return launched();
}

}  // extern "C"
