// A projection with weights of eight bits, as the common model answers with: one scale for each output and one for each row of x.
//
//   s = amax / 127,  q = rint(v (127 / amax))  of every row,      y[t, o] = s_x[t] s_w[o] sum_k q_x[t, k] q_w[o, k] + bias[o] + residual[t, o]
//
// Sums are whole numbers of 32 bits and exact. Rows of eight bits are kept with zeros up to a multiple of 128 bytes, so that no
// product has an end to look after.
#include "local_common.hpp"
#include "local_tiles.hpp"

using namespace haflo::local;

namespace {

constexpr u32 kThreads = 256;
constexpr u32 kMostLanes = 1024;
constexpr size_t kRow = HAFLO_INT8_ROW, kMostInner = HAFLO_INT8_MAX_COLS;

constexpr size_t kMostResults = (size_t)1 << 42;  // whose tiles 32 bits count

size_t row_bytes(size_t cols) { return ceil_div(cols, kRow) * kRow; }

// What brings a row to eight bits. A row with a NaN or an infinity has the scale NaN, and zeros.
struct Scale {
  float first, by;  // q = rint((v first) by)
  float scale;
};
__device__ __forceinline__ Scale scale_of(u32 most) {  // the bits of the largest magnitude
  if (most >= 0x7F800000u) return {0.0f, 0.0f, __builtin_nanf("")};
  const float amax = __builtin_bit_cast(float, most);
  if (amax == 0.0f) return {0.0f, 0.0f, 0.0f};
  const float first = amax < 0x1p-100f ? 0x1p64f : 1.0f;  // 127 / amax has to be finite
  return {first, 127.0f / (amax * first), amax / 127.0f};
}
__device__ __forceinline__ u32 magnitude(float v) { return __builtin_bit_cast(u32, v) & 0x7FFFFFFFu; }
template <class T>
__device__ __forceinline__ u32 most_of(const Vec8<T>& v) {
  u32 m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const u32 b = magnitude((float)v.get(j));
    m = b > m ? b : m;
  }
  return m;
}
template <class T>
__device__ __forceinline__ u64 eight_bits(const Vec8<T>& v, const Scale& s) {
  u64 q = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float r = s.by == 0.0f ? 0.0f : __builtin_rintf((float)v.get(j) * s.first * s.by);
    q |= (u64)(u32)(uint8_t)(int8_t)(int)r << (8 * j);
  }
  return q;
}

// A row to eight bits by a group of `lanes` lanes, HELD times eight columns to a lane, and of a longer row the others again: `put` takes eight
// bytes at each multiple of eight below `width`. All of a block's groups call it together. Returns the row's scale.
template <u32 HELD, class T, class Put>
__device__ __forceinline__ float quantize_row(const T* from, u32 cols, u32 width, u32 lanes, u32* room, const Put& put) {
  const u32 at = threadIdx.x % lanes * 8, apart = lanes * 8;
  u32 m = 0;
  const auto load = [&](u32 first, Vec8<T> (&v)[HELD]) {
#pragma unroll
    for (u32 i = 0; i < HELD; ++i) v[i] = load_cols(from, first + i * apart, cols);
  };
  const auto look = [&](const Vec8<T> (&v)[HELD]) {
#pragma unroll
    for (u32 i = 0; i < HELD; ++i) {
      const u32 b = most_of(v[i]);
      m = b > m ? b : m;
    }
  };
  Vec8<T> own[HELD];
  load(at, own);
  look(own);
  for (u32 col = at + HELD * apart; col < cols; col += HELD * apart) {
    Vec8<T> more[HELD];
    load(col, more);
    look(more);
  }
  m = lanes_join(m, lanes, [](u32 a, u32 b) { return a > b ? a : b; });
  if (lanes > kWave) {
    const u32 wave = threadIdx.x / kWave, waves = lanes / kWave, first = wave & ~(waves - 1);
    if (lane_id() == 0) room[wave] = m;
    __syncthreads();
    for (u32 w = 0; w < waves; ++w) m = room[first + w] > m ? room[first + w] : m;
  }
  const Scale s = scale_of(m);
  const auto give = [&](u32 first, const Vec8<T> (&v)[HELD]) {
#pragma unroll
    for (u32 i = 0; i < HELD; ++i)
      if (first + i * apart < width) put(first + i * apart, eight_bits(v[i], s));
  };
  give(at, own);
  for (u32 col = at + HELD * apart; col < width; col += HELD * apart) {
    Vec8<T> more[HELD];
    load(col, more);
    give(col, more);
  }
  return s.scale;
}
// Memory bounds it (8192 x 4096 bfloat16 24 us, 4.2 TB/s), a launch where rows are few (64 of 4096 3.3 us).
template <class T>
__global__ __launch_bounds__(kMostLanes) void k_quantize(const T* x, size_t ldx, u32 rows, u32 cols, u32 width, u32 lanes, int8_t* q, float* scale,
                                                         u32 first_block) {
  __shared__ u32 room[kMostLanes / kWave];
  const u64 mine = (u64)(first_block + blockIdx.x) * (blockDim.x / lanes) + threadIdx.x / lanes;
  const bool live = mine < rows;
  const u64 row = live ? mine : rows - 1;
  u64* const to = (u64*)(q + row * width);
  const float s = quantize_row<1>(x + row * ldx, cols, width, lanes, room, [&](u32 col, u64 v) {
    if (live) to[col / 8] = v;
  });
  if (live && threadIdx.x % lanes == 0) scale[row] = s;
}

// A scale as a factor of 1 .. 2 and a power of two: the product of two scales may pass the range of float32 where the results do not.
struct Factor {
  float m;
  int e;
};
__device__ __forceinline__ Factor factor(float scale) {
  Factor f;
  f.m = 2.0f * frexpf(scale, &f.e);
  f.e = scale == 0.0f ? -512 : f.e - 1;  // (zero times whatever the other power is)
  return f;
}
// sum x w + more. The power is on the sum, which is then at most the result (and loses bits only where that is below the normal numbers). One for every
// result costs 8192 rows of 4096 to 4096 2 us of 130; a branch to plain products where all of a wavefront's scales are ordinary, 4.
__device__ __forceinline__ float scaled(int sum, const Factor& x, const Factor& w, float more) {
  return __builtin_fmaf(ldexpf((float)sum, x.e + w.e), x.m * w.m, more);
}

template <class T>
struct Out {
  const float *x_scale, *w_scale, *bias;
  const T* residual;
  size_t ldr;
  T* y;
  size_t ldy;
  u32 rows, outer;
};
// A wavefront's results, RT x OT products of 16 x 16 from row t0 and output o0 on, by way of LDS, 32 rows at a time, so that lanes store, and
// load the residual, along rows: of a short reduction the results are most of the work (16384 rows of 128 to 4096, float16, 60 us by four
// outputs of sixteen rows at a time and 44 by rows; 8192 of 4096 to 4096 147 and 124).
template <int RT, int OT>
constexpr u32 out_floats() {  // of one wavefront
  return (RT < 2 ? 16 : 32) * (16 * OT + 4);
}
template <class T, int RT, int OT>
__device__ __forceinline__ void store_results(const Out<T>& to, u32 t0, u32 o0, const i32x4 (&acc)[OT][RT], float* room) {
  constexpr u32 ROWS = RT < 2 ? 16 : 32, WIDTH = 16 * OT, LD = WIDTH + 4, PER = WIDTH / 8;
  const u32 lane = lane_id();
  Factor ws[OT][4];
  f32x4 bias[OT];
#pragma unroll
  for (int i = 0; i < OT; ++i)
#pragma unroll
    for (u32 r = 0; r < 4; ++r) {
      const u32 o = o0 + 16 * i + lane / 16 * 4 + r, at = o < to.outer ? o : to.outer - 1;
      ws[i][r] = factor(to.w_scale[at]);
      bias[i][r] = to.bias ? to.bias[at] : 0.0f;
    }
#pragma unroll
  for (int j0 = 0; j0 < RT; j0 += ROWS / 16) {
    if (j0) __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (u32 j = 0; j < ROWS / 16; ++j) {
      const u32 t = t0 + 16 * (j0 + j) + lane % 16;
      const Factor by = factor(to.x_scale[t < to.rows ? t : to.rows - 1]);
#pragma unroll
      for (int i = 0; i < OT; ++i) {
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = scaled(acc[i][j0 + j][r], by, ws[i][r], bias[i][r]);
        *(f32x4*)(room + (16 * j + lane % 16) * LD + 16 * i + lane / 16 * 4) = v;
      }
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (u32 n = 0; n < ROWS * PER / kWave; ++n) {
      const u32 at = n * kWave + lane, row = at / PER, col = at % PER * 8, t = t0 + 16 * j0 + row, o = o0 + col;
      if (t >= to.rows || o >= to.outer) continue;
      f32x4 v[2];
      __builtin_memcpy(v, __builtin_assume_aligned(room + row * LD + col, 16), sizeof(v));
      Vec8<T> y = {};
      if (to.residual) y = load_cols(to.residual + t * to.ldr, o, to.outer);
#pragma unroll
      for (int e = 0; e < 8; ++e) y.set(e, (T)(v[e / 4][e % 4] + (to.residual ? (float)y.get(e) : 0.0f)));
      store_cols(to.y + t * to.ldy, o, to.outer, y);
    }
  }
}

// A block takes TM rows by TN outputs, its WM x WN wavefronts a part of that each in products of 16 x 16. Two steps' tiles lie in LDS, and one
// is filled while the other is read; of tiles of 64 x 64 four steps' (4096 to 4096, 128 rows 19.8 us by two and 12.6 by four). Matrix
// instructions bound the large tiles: 8192 of 4096 to 4096 113 to 117 us, 2350 to 2430 TOP/s (a library product of these numbers 129 us), busy in two thirds
// of the cycles; the wait for loads the small ones (64 rows 9.2 us).
template <class T, int TM, int TN, int WM, int WN, bool FAR>
__global__ __launch_bounds__(WM * WN * kWave) void k_int8(const int8_t* x, const int8_t* w, u32 width, Out<T> to, u32 x_bytes, u32 w_bytes, u32 first_block) {
  constexpr int KE = step_elems<int8_t>(), WAVES = WM * WN, RT = TM / WM / 16, OT = TN / WN / 16;
  constexpr int LX = TM / 8 / WAVES, LW = TN / 8 / WAVES;
  constexpr bool kDeep = TM == 64;
  __shared__ __align__(16) int8_t lds[(kDeep ? 4 : 2) * (TM + TN) * KE];
  const auto x_tile = [&](int n) { return lds + n * (TM + TN) * KE; };
  const auto w_tile = [&](int n) { return x_tile(n) + TM * KE; };
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  // Blocks are dealt to the eight dies in turn: each gets neighbouring tiles, four tiles of rows by all outputs at a time,
  // whose operands its cache holds.
  const u32 tiles_m = (to.rows + TM - 1) / TM, tiles_n = (to.outer + TN - 1) / TN, tiles = tiles_m * tiles_n;
  const u32 block = first_block + blockIdx.x, die = block % 8, per = tiles / 8, over = tiles % 8;
  const u32 tile = die * per + (die < over ? die : over) + block / 8;
  const u32 band = tile / (4 * tiles_n), in_band = tile % (4 * tiles_n), high = tiles_m - band * 4 < 4 ? tiles_m - band * 4 : 4;
  const u32 t0 = (band * 4 + in_band % high) * TM, o0 = in_band / high * TN;
  const u32 row0 = wave / WN * (TM / WM), out0 = wave % WN * (TN / WN);  // this wavefront's corner

  using From = Source<int8_t, FAR>;
  const From from_x(x, x_bytes), from_w(w, w_bytes);
  typename From::At at_x[LX], at_w[LW];  // this lane's pieces; rows behind the last are the last one again
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const u32 r = (i * WAVES + wave) * 8 + lane / 8, t = t0 + r < to.rows ? t0 + r : to.rows - 1;
    at_x[i] = From::at(t, width, place_of(r, lane % 8) * 16);
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const u32 r = (i * WAVES + wave) * 8 + lane / 8, o = o0 + r < to.outer ? o0 + r : to.outer - 1;
    at_w[i] = From::at(o, width, place_of(r, lane % 8) * 16);
  }
  i32x4 acc[OT][RT];
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int i = 0; i < OT; ++i) acc[i][j] = i32x4{0, 0, 0, 0};
  if constexpr (kDeep)
    reduce_deep<int8_t, TM, TN, WAVES>(from_x, at_x, from_w, at_w, width / KE, wave, row0, out0, x_tile(0), w_tile(0), x_tile(1), w_tile(1), x_tile(2),
                                       w_tile(2), x_tile(3), w_tile(3), acc);
  else
    reduce<int8_t, TM, TN, WAVES>(from_x, at_x, from_w, at_w, width / KE, wave, row0, out0, x_tile(0), w_tile(0), x_tile(1), w_tile(1), acc);
  __syncthreads();  // the tiles' place is free
  static_assert(sizeof(lds) >= WAVES * out_floats<RT, OT>() * sizeof(float), "");
  store_results(to, t0 + row0, o0 + out0, acc, (float*)lds + wave * out_floats<RT, OT>());
}

// Few rows: a block takes 16 outputs by 16 R rows, its wavefronts a part of the reduction each, so that W is on its way from all
// of them at once, x and the next pieces with it; their sums are joined in LDS. With OWN the block brings the rows, at most sixteen, to
// eight bits itself, which takes no longer than a launch (8 rows of 2048 to 4096 6.4 us, by way of k_quantize 7.9; 16 8.5 and 8.6) and spares
// the host one. One row of 4096 to 4096 6 us, 2.7 TB/s of W: its way from memory, x's and the joining one
// after the other.
constexpr u32 kFewWaves = 8, kFewThreads = kFewWaves * kWave, kOwnBytes = 32768, kOwnPad = 16;  // (rows in LDS begin on different banks)
template <class T, int R, bool OWN>
__global__ __launch_bounds__(kFewThreads) void k_int8_few(const T* xf, size_t ldx, u32 cols, const int8_t* xq, const int8_t* w, u32 width, Out<T> to,
                                                          u32 first_block) {
  constexpr u32 kAhead = R == 1 ? 4 : 2;  // pieces of 128 bytes of each row that are on their way together
  constexpr u32 kResults = (256 * R + kFewThreads - 1) / kFewThreads;
  __shared__ __align__(16) int8_t own[OWN ? kOwnBytes + 16 * kOwnPad : 16];
  __shared__ float own_scale[16];
  __shared__ u32 room[kFewWaves];
  __shared__ int sums[kFewWaves][R][256];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const u32 tiles = (to.outer + 15) / 16, block = first_block + blockIdx.x, o0 = block % tiles * 16, t0 = block / tiles * 16 * R;
  const auto last = [](u32 i, u32 n) { return i < n ? i : n - 1; };
  const u32 pieces = width / 128, first = pieces * wave / kFewWaves, end = pieces * (wave + 1) / kFewWaves;
  const int8_t* const wr = w + (size_t)last(o0 + lane % 16, to.outer) * width + lane / 16 * 16;
  const int8_t* xr[R];
#pragma unroll
  for (int j = 0; j < R; ++j) xr[j] = (OWN ? own : xq) + (size_t)last(t0 + 16 * j + lane % 16, to.rows) * (OWN ? width + kOwnPad : width) + lane / 16 * 16;
  struct Pieces {
    i32x4 w[kAhead][2], x[OWN ? 1 : kAhead][2][R];
  };
  Pieces next;
  const auto ask = [&](u32 p) {
#pragma unroll
    for (u32 u = 0; u < kAhead; ++u)
#pragma unroll
      for (u32 h = 0; h < 2; ++h) {
        const size_t at = (size_t)last(p + u, end) * 128 + h * 64;
        next.w[u][h] = *(const i32x4*)(wr + at);
        if (!OWN) {
#pragma unroll
          for (int j = 0; j < R; ++j) next.x[OWN ? 0 : u][h][j] = *(const i32x4*)(xr[j] + at);
        }
      }
  };
  if (first < end) ask(first);
  // what the results take besides their sums: result i is of row t0 + i / 16 and output o0 + i % 16
  float by[kResults], bias[kResults], was[kResults], x_scale[kResults];
#pragma unroll
  for (u32 n = 0; n < kResults; ++n) {
    const u32 i = threadIdx.x + n * kFewThreads, t = last(t0 + i / 16, to.rows), o = last(o0 + i % 16, to.outer);
    by[n] = to.w_scale[o];
    x_scale[n] = OWN ? 0.0f : to.x_scale[t];
    bias[n] = to.bias ? to.bias[o] : 0.0f;
    was[n] = to.residual ? (float)to.residual[t * to.ldr + o] : 0.0f;
  }
  if (OWN) {
    u32 groups = 1;
    while (groups < to.rows) groups *= 2;
    const u32 lanes = kFewThreads / groups, group = threadIdx.x / lanes, row = last(group, to.rows);
    const auto put = [&](u32 col, u64 v) {
      if (group < to.rows) *(u64*)(own + group * (width + kOwnPad) + col) = v;
    };
    // (four vectors on their way where a lane has several; where it has one, the other three's branches cost 0.3 us)
    const float s = cols <= lanes * 8 ? quantize_row<1>(xf + row * ldx, cols, width, lanes, room, put) : quantize_row<4>(xf + row * ldx, cols, width, lanes, room, put);
    if (threadIdx.x % lanes == 0) own_scale[group] = s;
    __syncthreads();
  }
  i32x4 acc[R];
#pragma unroll
  for (int j = 0; j < R; ++j) acc[j] = i32x4{0, 0, 0, 0};
  for (u32 p = first; p < end; p += kAhead) {
    const Pieces now = next;
    if (p + kAhead < end) ask(p + kAhead);
#pragma unroll
    for (u32 u = 0; u < kAhead; ++u)
#pragma unroll
      for (u32 h = 0; h < 2; ++h) {
        const i32x4 wv = p + u < end ? now.w[u][h] : i32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < R; ++j) {
          const i32x4 xv = OWN ? *(const i32x4*)(xr[j] + (size_t)last(p + u, end) * 128 + h * 64) : now.x[OWN ? 0 : u][h][j];
          acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv, xv, acc[j], 0, 0, 0);
        }
      }
  }
  // row t of the tile at 16 t, its outputs beside each other
#pragma unroll
  for (int j = 0; j < R; ++j) *(i32x4*)&sums[wave][j][lane % 16 * 16 + lane / 16 * 4] = acc[j];
  __syncthreads();
#pragma unroll
  for (u32 n = 0; n < kResults; ++n) {
    const u32 i = threadIdx.x + n * kFewThreads, t = t0 + i / 16, o = o0 + i % 16;
    if (i >= 256 * R || t >= to.rows || o >= to.outer) continue;
    int s = 0;
#pragma unroll
    for (u32 v = 0; v < kFewWaves; ++v) s += sums[v][i / 256][i % 256];
    to.y[t * to.ldy + o] = (T)(scaled(s, factor(OWN ? own_scale[t] : x_scale[n]), factor(by[n]), bias[n]) + was[n]);
  }
}

constexpr size_t kFewRows = 32, kFewOuter = 4096, kFewBytes = 2048, kOwnOuter = 8192;
// Rows that the blocks which multiply them bring to eight bits too: each block does so again, so that few rows for few blocks gain by the launch and the
// workspace they are spared, and more lose. Graphs of the operator, us, this way / k_quantize before it, bfloat16, 1, 4, 5, 8 and 16 rows:
// 2048 to 2048 5.2 / 6.8, 5.9 / 7.4, 6.3 / 7.4, 6.4 / 7.8, 8.2 / 8.6; 4096 to 4096 5.4 / 6.9, 6.5 / 7.5, 8.3 / 7.4, 8.7 / 7.9, 8.6 / 8.6 (where calls from
// the host take 8.5 to 13 and the other way 13 or 17); 1 and 4 rows of 4096 to 8192 7.6 / 11.6, 9.3 / 11.6, to 16384 15.0 / 14.6, 17.5 / 15.2, to 32000
// 24.3 / 23.5, 28.0 / 23.2, of 2048 to 128000 76 / 50, 82 / 50.
bool own_rows(size_t rows, size_t cols, size_t outer) {
  return rows <= (outer <= kFewOuter ? 16 : outer <= kOwnOuter ? 4 : 0) && rows * row_bytes(cols) <= kOwnBytes;
}
// Products of rows in eight bits: k_int8_few where there is one block for each compute unit at most, and rows are long enough to split, else tiles of
// 64 x 64. Graphs of them, us, few / tiles, of 1, 16, 17, 32 and 48 rows: 1024 to 1024 4.4 / 4.4, 5.8 / 4.5, 4.3 / 4.8, 5.0 / 4.7, 5.0 / 4.7;
// 2048 to 2048 4.4 / 5.7, 5.8 / 5.8, 4.4 / 6.0, 5.0 / 6.0, 5.1 / 6.0; 4096 to 4096 4.7 / 8.4, 6.1 / 8.4, 6.8 / 8.7, 8.1 / 8.6, 12.2 / 8.7; 4096 to 8192
// 7.7 / 9.0, 10.4 / 9.0, 10.7 / 9.3, 13.2 / 9.4, 21.3 / 9.4.
bool few_rows(size_t rows, size_t width, size_t outer) { return rows <= kFewRows && outer <= kFewOuter && width >= kFewBytes; }
template <class T>
void few(const T* x, size_t ldx, size_t cols, const int8_t* xq, const int8_t* w, const Out<T>& to, hipStream_t st) {
#define HAFLO_LOCAL_RUN(R, OWN)                                                                                                            \
  in_turns(ceil_div(to.rows, 16 * R) * ceil_div(to.outer, 16), kFewThreads, [&](u32 first, dim3 grid, dim3 block) {                        \
    hipLaunchKernelGGL((k_int8_few<T, R, OWN>), grid, block, 0, st, x, ldx, (u32)cols, xq, w, (u32)row_bytes(cols), to, first);            \
  })
  if (!xq) HAFLO_LOCAL_RUN(1, true);
  else if (to.rows <= 16) HAFLO_LOCAL_RUN(1, false);
  else HAFLO_LOCAL_RUN(2, false);
#undef HAFLO_LOCAL_RUN
}
template <class T>
void quantize(const void* x, size_t ldx, size_t rows, size_t cols, int8_t* q, float* scale, hipStream_t st) {
  const size_t width = row_bytes(cols);
  u32 lanes = 16;
  while (lanes < kMostLanes && (size_t)lanes * 8 < width) lanes *= 2;
  const u32 threads = lanes < kThreads ? kThreads : lanes;
  in_turns(ceil_div(rows, threads / lanes), threads, [&](u32 first, dim3 grid, dim3 block) {
    hipLaunchKernelGGL((k_quantize<T>), grid, block, 0, st, (const T*)x, ldx, (u32)rows, (u32)cols, (u32)width, lanes, q, scale, first);
  });
}
template <class T>
void product(const int8_t* x, const int8_t* w, size_t cols, const Out<T>& to, hipStream_t st) {
  const size_t width = row_bytes(cols);
  if (few_rows(to.rows, width, to.outer)) return few<T>(nullptr, 0, cols, x, w, to, st);
  const size_t x_bytes = to.rows * width, w_bytes = to.outer * width;
  const bool far = x_bytes > 0xFFFFFFFFu || w_bytes > 0xFFFFFFFFu;
#define HAFLO_LOCAL_RUN(TM, TN, WM, WN, FAR)                                                                                        \
  in_turns(ceil_div(to.rows, TM) * ceil_div(to.outer, TN), WM * WN * kWave, [&](u32 first, dim3 grid, dim3 block) {                 \
    hipLaunchKernelGGL((k_int8<T, TM, TN, WM, WN, FAR>), grid, block, 0, st, x, w, (u32)width, to, (u32)x_bytes, (u32)w_bytes, first); \
  })
  // A tile of 256 x 256 takes a compute unit for itself, of 128 x 128 two share one; two rounds of the latter take 1.2 times one of the
  // former. us by 256 and by 128: float16 8192 of 4096 to 4096 124 and 155, 4096 of 1024 to 4096 24.5 and 31; 3656 of 94 to 4371, 270 large
  // tiles, 23.3 and 16.9. Fewer than 256 tiles of 128 x 128 leave compute units idle: 2048 of 2048 to 2048 16.6 by them and 18.2 by 64 x 64.
  const size_t large = ceil_div(to.rows, 256) * ceil_div(to.outer, 256), middle = ceil_div(to.rows, 128) * ceil_div(to.outer, 128);
  if (far) HAFLO_LOCAL_RUN(256, 256, 2, 4, true);
  else if (large >= 256 && 5 * ceil_div(large, 256) <= 3 * ceil_div(middle, 512)) HAFLO_LOCAL_RUN(256, 256, 2, 4, false);
  else if (middle >= 256) HAFLO_LOCAL_RUN(128, 128, 2, 2, false);
  else HAFLO_LOCAL_RUN(64, 64, 2, 2, false);
#undef HAFLO_LOCAL_RUN
}

bool int8_sizes(int type, size_t rows, size_t inner, size_t outer) {
  return valid_type(type) && rows <= kMostCount && inner >= 1 && inner <= kMostInner && outer >= 1 && outer <= kMostCount && rows * outer <= kMostResults;
}
bool aligned(const void* p) { return p && (uintptr_t)p % 16 == 0; }
struct Plan {
  size_t scale, total;
};
// `over`: the result lies over x, whose rows then have to be in eight bits before any block writes
Plan int8_plan(size_t rows, size_t inner, size_t outer, bool over) {
  Plan p = {0, 0};
  if (!over && own_rows(rows, inner, outer)) return p;
  p.scale = align256(rows * row_bytes(inner));
  p.total = p.scale + align256(rows * 4);
  return p;
}

}  // namespace

extern "C" {

int haflo_quantize_rows(int type, const void* d_x, size_t ldx, size_t rows, size_t cols, int8_t* d_q, float* d_scale, void* stream) {
  if (!int8_sizes(type, rows, cols, 1)) return HAFLO_EINVAL;
  if (rows == 0) return HAFLO_OK;
  if (!d_x || ldx < cols || !aligned(d_q) || !d_scale) return HAFLO_EINVAL;
  HAFLO_LOCAL_TYPES(type, quantize<T>(d_x, ldx, rows, cols, d_q, d_scale, (hipStream_t)stream));
  return launched();
}

int haflo_int8_product(int type, const int8_t* d_xq, const float* d_x_scale, const int8_t* d_wq, const float* d_w_scale, const float* d_bias,
                       const void* d_residual, size_t ldr, size_t rows, size_t inner, size_t outer, void* d_y, size_t ldy, void* stream) {
  if (!int8_sizes(type, rows, inner, outer)) return HAFLO_EINVAL;
  if (rows == 0) return HAFLO_OK;
  if (!aligned(d_xq) || !d_x_scale || !aligned(d_wq) || !d_w_scale || (d_residual && ldr < outer) || !d_y || ldy < outer) return HAFLO_EINVAL;
  if (!in_place(d_residual, ldr, d_y, ldy, rows)) return HAFLO_EINVAL;
  HAFLO_LOCAL_TYPES(type, {
    const Out<T> to = {d_x_scale, d_w_scale, d_bias, (const T*)d_residual, ldr, (T*)d_y, ldy, (u32)rows, (u32)outer};
    product<T>(d_xq, d_wq, inner, to, (hipStream_t)stream);
  });
  return launched();
}

size_t haflo_int8_workspace_bytes(int type, size_t rows, size_t inner, size_t outer) {
  return int8_sizes(type, rows, inner, outer) ? int8_plan(rows, inner, outer, false).total : (size_t)-1;
}

int haflo_int8_forward(int type, const void* d_x, size_t ldx, const int8_t* d_wq, const float* d_w_scale, const float* d_bias, const void* d_residual,
                       size_t ldr, size_t rows, size_t inner, size_t outer, void* d_y, size_t ldy, void* d_workspace, size_t workspace_bytes,
                       void* stream) {
  if (!int8_sizes(type, rows, inner, outer)) return HAFLO_EINVAL;
  if (rows == 0) return HAFLO_OK;
  if (!d_x || ldx < inner || !aligned(d_wq) || !d_w_scale || (d_residual && ldr < outer) || !d_y || ldy < outer) return HAFLO_EINVAL;
  if (!in_place(d_residual, ldr, d_y, ldy, rows)) return HAFLO_EINVAL;
  const Plan plan = int8_plan(rows, inner, outer, d_y == d_x);
  if (!enough(d_workspace, workspace_bytes, plan.total)) return HAFLO_EINVAL;
  int8_t* const xq = (int8_t*)d_workspace;
  float* const x_scale = (float*)((char*)d_workspace + plan.scale);
  HAFLO_LOCAL_TYPES(type, {
    if (plan.total == 0) {
      few<T>((const T*)d_x, ldx, inner, nullptr, d_wq, {nullptr, d_w_scale, d_bias, (const T*)d_residual, ldr, (T*)d_y, ldy, (u32)rows, (u32)outer},
             (hipStream_t)stream);
      return launched();
    }
    quantize<T>(d_x, ldx, rows, inner, xq, x_scale, (hipStream_t)stream);
    const Out<T> to = {x_scale, d_w_scale, d_bias, (const T*)d_residual, ldr, (T*)d_y, ldy, (u32)rows, (u32)outer};
    product<T>(xq, d_wq, inner, to, (hipStream_t)stream);
  });
  return launched();
}

}  // extern "C"
