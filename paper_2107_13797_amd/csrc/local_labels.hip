// Log-probabilities of labels with entropy and top alternatives, and their gradient by the logits.
//
// One pass over a row keeps, per lane, the running maximum m, s = sum e^(x - m) and t = sum e^(x - m) (x - m); then
// lse = m + ln s and the entropy is ln s - t / s. Two such states join by rescaling the one with the smaller maximum.
// The greatest elements are kept as one descending list per wavefront, entry j in lane j; an element is the 64-bit key
// (value in an order-preserving form, complement of its column), so that the larger key is the greater value or, of equal
// ones, the lower column, and the list does not depend on the order in which elements come.
#include "local_common.hpp"

using namespace haflo::local;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
// Up to here a lane takes a row by itself. 262144 rows, us, and by wavefronts: float32 24 columns 37 and 119, 33 columns 99 and 134, 48 columns 164
// and 127; bfloat16 33 columns 39 and 136, 48 columns 70 and 129, 64 columns 123 and 133; with 16 alternatives 33 columns 342 and 445, 48 661 and
// 488; 64 rows of 33 columns 9 and 10.
constexpr size_t kSmallCols = 32;
// Up to here a wavefront does (16384 rows, us, and by blocks: 1000 columns 16 and 35, 2000 columns 25 and 43), and of longer rows
// where there are many. By wavefronts and by blocks: 2048 rows of 2049 bfloat16 10 and 10, of 16384 23 and 21; 3000 rows 10 and 12, 28 and 27; 4096
// rows of 2049 10 and 14, of 16384 33 and 33, of 32768 61 and 55; 16384 rows of 4000 34 and 52, of 16000 110 and 126. float32: 2048 rows of
// 16384 28 and 27, 4096 rows of 2049 10 and 14, of 16384 48 and 47, of 65536 191 and 188. With alternatives the wavefronts gain more.
constexpr size_t kWaveCols = 2048, kManyWaveCols = 16384, kManyRows = 3000;
constexpr size_t kSplitCols = 2048;  // columns of one part of a row, at least
constexpr size_t kSplitBlocks = 1024;
constexpr int kAhead = 4;            // vectors on their way at a time
constexpr size_t kGradBlocks = 1 << 21;  // blocks of a launch at most, which loop over the rows
constexpr float kLog2e = 1.44269504088896341f, kLog2eRest = (float)(1.44269504088896341 - (double)kLog2e), kLn2 = 0.693147180559945309f;

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

struct Soft {
  float m, s, t;
};
__device__ __forceinline__ float shift_of(float m) { return m == neg_inf() ? 0.0f : m; }  // what exponents are taken relative to
__device__ __forceinline__ void raise_to(Soft& a, float m) {                              // m >= a.m
  const float by = a.m - shift_of(m), c = __builtin_amdgcn_exp2f(by * kLog2e);
  if (a.s != 0.0f) {
    a.t = c == 0.0f ? 0.0f : c * (a.t + by * a.s);
    a.s *= c;
  }
  a.m = m;
}
__device__ __forceinline__ void join(Soft& a, Soft b) {
  const float m = __builtin_fmaxf(a.m, b.m);
  if (a.m < m) raise_to(a, m);
  if (b.m < m) raise_to(b, m);
  a.s += b.s;
  a.t += b.t;
}
__device__ __forceinline__ Soft wave_join(Soft a) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int from = (int)(lane_id() ^ d);
    Soft b;
    b.m = lane_read(a.m, from);
    b.s = lane_read(a.s, from);
    b.t = lane_read(a.t, from);
    // both lanes of a pair join in the same order, so that they hold the same bits
    if (lane_id() & d) {
      join(b, a);
      a = b;
    } else {
      join(a, b);
    }
  }
  return a;
}

__device__ __forceinline__ u64 key_of(float x, u32 col) {
  u32 b = __builtin_bit_cast(u32, x);
  if (x == 0.0f) b = 0;  // zeros of both signs are equal
  u32 k = b & 0x80000000u ? ~b : b | 0x80000000u;
  if (x != x) k = 0xFFFFFFFFu;
  return (u64)k << 32 | (u32)~col;
}
__device__ __forceinline__ float value_of(u64 key) {
  const u32 k = (u32)(key >> 32);
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

struct TopList {
  u64 mine;   // this lane's entry, 0: none
  u64 last;   // entry top - 1, the same in all lanes, or the floor where that is higher
  u64 floor;  // no element up to it belongs into the list
};
// key_lane's `key` into the list, which it belongs into
__device__ __forceinline__ void top_insert(TopList& l, u64 key, int key_lane, int top) {
  const u32 lo = (u32)__builtin_amdgcn_readlane((int)(u32)key, key_lane);
  const u32 hi = (u32)__builtin_amdgcn_readlane((int)(u32)(key >> 32), key_lane);
  const u64 k = (u64)hi << 32 | lo;
  const int place = __builtin_popcountll(__builtin_amdgcn_ballot_w64(l.mine > k));
  // every lane's entry to the next lane
  const u32 plo = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)l.mine, 0x138, 0xF, 0xF, false);
  const u32 phi = (u32)__builtin_amdgcn_update_dpp(0, (int)(u32)(l.mine >> 32), 0x138, 0xF, 0xF, false);
  const int lane = (int)lane_id();
  if (lane > place) l.mine = (u64)phi << 32 | plo;
  if (lane == place) l.mine = k;
  const u64 last = (u64)(u32)__builtin_amdgcn_readlane((int)(u32)(l.mine >> 32), top - 1) << 32 |
                   (u32)__builtin_amdgcn_readlane((int)(u32)l.mine, top - 1);
  l.last = last > l.floor ? last : l.floor;
}
// Two descending lists to the 64 greatest of both: the larger of each entry and the other list's mirrored one is a
// bitonic sequence, which six exchanges sort.
__device__ __forceinline__ u64 top_merge(u64 mine, u64 mirrored) {
  u64 v = mine > mirrored ? mine : mirrored;
#pragma unroll
  for (int d = kWave / 2; d >= 1; d >>= 1) {
    const u64 o = lane_read(v, (int)(lane_id() ^ d));
    const bool upper = (lane_id() & d) != 0;
    v = (o > v) != upper ? o : v;
  }
  return v;
}

template <class T>
__device__ __forceinline__ void take(Soft& a, const Vec8<T>& v) {
  float x[8], most = neg_inf();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    x[j] = (float)v.get(j);
    most = __builtin_fmaxf(most, x[j]);
  }
  if (most > a.m) raise_to(a, most);
  const float m = shift_of(a.m);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float d = x[j] - m, e = __builtin_amdgcn_exp2f(d * kLog2e);
    a.s += e;
    a.t += e == 0.0f ? 0.0f : e * d;
  }
}

// the elements of `v` that belong into the list; all lanes of a wavefront call this together
template <class T>
__device__ __forceinline__ void take_top(TopList& l, const Vec8<T>& v, u32 col, u32 cols, bool live, int top) {
  u64 k[8], most = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    k[j] = live && col + j < cols ? key_of((float)v.get(j), col + j) : 0;
    most = k[j] > most ? k[j] : most;
  }
  if (__builtin_amdgcn_ballot_w64(most > l.last) == 0) return;
  if (l.last == 0) {
    // The first elements: `top` lanes have one that is no less than the top-th of the lanes' greatest, which is found bit by
    // bit; what is less need not be inserted only to be pushed out again (20 of 512: 25 insertions instead of 85).
    const u32 key = (u32)(most >> 32);
    u32 least = 0;
#pragma unroll 1
    for (u32 bit = 0x80000000u; bit; bit >>= 1)
      if (__builtin_popcountll(__builtin_amdgcn_ballot_w64(key >= (least | bit))) >= top) least |= bit;
    if (least) l.last = l.floor = ((u64)least << 32) - 1;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    u64 who = __builtin_amdgcn_ballot_w64(k[j] > l.last);
    while (who) {
      const int lane = __builtin_ctzll(who);
      top_insert(l, k[j], lane, top);
      who &= who - 1;
      who &= __builtin_amdgcn_ballot_w64(k[j] > l.last);
    }
  }
}

// eight elements of a row from column `col` on; -inf past its end
template <class T>
__device__ __forceinline__ Vec8<T> load_row(const T* row, u32 col, u32 cols) {
  return col + 8 <= cols ? load_wide(row + col) : load_some(row + col, (int)(cols - col), (T)neg_inf());
}

struct LabelOut {
  const int* label;
  float *logp, *entropy, *lse, *top_logp;
  int* top_index;
  u32* status;
};
// what a row's state and list say, written by one wavefront
template <class T>
__device__ __forceinline__ void finish_row(const LabelOut& o, const T* row, u32 r, u32 cols, Soft a, u64 mine, int top) {
  const float m = shift_of(a.m), log_s = logf(a.s);
  const bool empty = a.s == 0.0f;
  const u32 lane = lane_id();
  if (lane == 0) {
    const int label = o.label[r];
    const bool has = (u32)label < cols;
    if (!has && label != -1 && o.status) atomicOr(o.status, HAFLO_ST_RANGE);
    const float x = has ? (float)row[label] : 0.0f;
    o.logp[r] = !has ? 0.0f : empty ? neg_inf() : x - m - log_s;
    o.entropy[r] = empty ? 0.0f : log_s - a.t / a.s;
    o.lse[r] = empty ? neg_inf() : m + log_s;
  }
  if ((int)lane < top) {
    o.top_logp[(size_t)r * top + lane] = empty ? neg_inf() : value_of(mine) - m - log_s;
    o.top_index[(size_t)r * top + lane] = (int)~(u32)mine;
  }
}

struct Part {  // of a row, joined by k_label_join
  float m, s, t, unused;
};

// W wavefronts to a row or, with `parts` > 1, to one of its parts. Reading the row bounds it (8192 x 32768 bfloat16: 112 us call after call, 4.8 TB/s);
// one long row the length of a part and its list (131072 columns, 20 greatest: 11 us).
template <class T, int W, bool TOP>
__global__ __launch_bounds__(kThreads) void k_labels(const T* x, size_t ld, u32 rows, u32 cols, int top, u32 parts, LabelOut o,
                                                     Part* part, u64* lists, u32 first_block) {
  __shared__ Soft soft[kWaves];
  __shared__ u64 list[TOP ? kWaves : 1][kWave];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const u32 block = first_block + blockIdx.x, unit = W == 1 ? block * kWaves + wave : block;
  const u32 r = unit / parts, p = unit % parts;
  if (W == 1 && r >= rows) return;
  const T* row = x + (size_t)r * ld;
  const u32 vectors = (cols + 7) / 8;
  const u32 first = (u32)((u64)vectors * p / parts), end = (u32)((u64)vectors * (p + 1) / parts);
  constexpr u32 kStep = W * kWave;
  Soft a = {neg_inf(), 0.0f, 0.0f};
  TopList l = {0, 0, 0};
  for (u32 base = first; base < end; base += kStep * kAhead) {
    Vec8<T> v[kAhead];
    const u32 at = base + threadIdx.x % kStep;
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (at + i * kStep < end) v[i] = load_row(row, (at + i * kStep) * 8, cols);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const bool live = at + i * kStep < end;
      const u32 col = (at + i * kStep) * 8;
      if (live) take(a, v[i]);
      if (TOP && base + i * kStep < end) take_top(l, v[i], col, cols, live, top);
    }
  }
  a = wave_join(a);
  u64 mine = l.mine;
  if (W > 1) {
    if (lane_id() == 0) soft[wave] = a;
    if (TOP) list[wave][lane_id()] = mine;
    __syncthreads();
    if (wave != 0) return;
    for (int w = 1; w < W; ++w) {
      join(a, soft[w]);
      if (TOP) mine = top_merge(mine, list[w][kWave - 1 - lane_id()]);
    }
  }
  if (parts == 1) {
    finish_row(o, row, r, cols, a, mine, top);
  } else {
    if (lane_id() == 0) part[unit] = Part{a.m, a.s, a.t, 0.0f};
    if (TOP && (int)lane_id() < top) lists[(size_t)unit * top + lane_id()] = mine;
  }
}

// Joins the parts of a row: its first wavefront the sums, in their order; all of them every eighth list each, and what they
// have then pair by pair. A chain of exchanges bounds it (lists of 131072 columns' parts: 7.7 us).
constexpr int kJoinWaves = 8;
template <class T, bool TOP>
__global__ __launch_bounds__((TOP ? kJoinWaves : 1) * kWave) void k_label_join(const T* x, size_t ld, u32 cols, int top, u32 parts, LabelOut o,
                                                                              const Part* part, const u64* lists) {
  __shared__ u64 list[TOP ? kJoinWaves / 2 : 1][kWave];
  const u32 r = blockIdx.x, lane = lane_id(), wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  u64 mine = 0;
  if (TOP) {
    const int at = kWave - 1 - (int)lane;  // mirrored
    const u64* const mirrored = lists + (size_t)r * parts * top + at;
    u64 next = wave < parts && at < top ? mirrored[(size_t)wave * top] : 0;
    for (u32 p = wave; p < parts; p += kJoinWaves) {
      const u64 now = next;
      if (p + kJoinWaves < parts) next = at < top ? mirrored[(size_t)(p + kJoinWaves) * top] : 0;
      mine = top_merge(mine, now);
    }
#pragma unroll
    for (u32 half = kJoinWaves / 2; half >= 1; half >>= 1) {
      if (wave >= half && wave < 2 * half) list[wave - half][lane] = mine;
      __syncthreads();
      if (wave < half) mine = top_merge(mine, list[wave][kWave - 1 - lane]);
      __syncthreads();
    }
    if (wave != 0) return;
  }
  Soft a = {neg_inf(), 0.0f, 0.0f};
  for (u32 p = lane; p < parts; p += kWave) {
    const Part q = part[(size_t)r * parts + p];
    join(a, Soft{q.m, q.s, q.t});
  }
  finish_row(o, x + (size_t)r * ld, r, cols, wave_join(a), mine, top);
}

// a lane to a row of few columns, where a wavefront would be idle but for those (65536 x 2 float32: 3.2 us, a launch)
template <class T>
__global__ __launch_bounds__(kThreads) void k_labels_small(const T* x, size_t ld, u32 rows, u32 cols, int top, LabelOut o) {
  const u32 r = blockIdx.x * kThreads + threadIdx.x;
  if (r >= rows) return;
  const T* row = x + (size_t)r * ld;
  float most = neg_inf();
  for (u32 j = 0; j < cols; ++j) most = __builtin_fmaxf(most, (float)row[j]);
  const float m = shift_of(most);
  float s = 0.0f, t = 0.0f;
  for (u32 j = 0; j < cols; ++j) {
    const float d = (float)row[j] - m, e = __builtin_amdgcn_exp2f(d * kLog2e);
    s += e;
    t += e == 0.0f ? 0.0f : e * d;
  }
  const float log_s = logf(s);
  const bool empty = s == 0.0f;
  const int label = o.label[r];
  const bool has = (u32)label < cols;
  if (!has && label != -1 && o.status) atomicOr(o.status, HAFLO_ST_RANGE);
  o.logp[r] = !has ? 0.0f : empty ? neg_inf() : (float)row[label] - m - log_s;
  o.entropy[r] = empty ? 0.0f : log_s - t / s;
  o.lse[r] = empty ? neg_inf() : m + log_s;
  u64 last = ~0ull;
  for (int k = 0; k < top; ++k) {
    u64 best = 0;
    for (u32 j = 0; j < cols; ++j) {
      const u64 key = key_of((float)row[j], j);
      if (key < last && key > best) best = key;
    }
    o.top_logp[(size_t)r * top + k] = empty ? neg_inf() : value_of(best) - m - log_s;
    o.top_index[(size_t)r * top + k] = (int)~(u32)best;
    last = best;
  }
}

// a number below `count`, the last one for those behind it
__device__ __forceinline__ u32 lowest(u32 i, u32 count) { return i < count ? i : count - 1; }

struct GradIn {
  const int* label;
  const float *lse, *entropy, *dlogp, *dentropy;
  const int* top_index;
  const float* dtop;
};
// dx = -p (g + dentropy (ln p + entropy)), p = e^(x - lse) / z and g the sum of what label and alternatives are given, plus that at
// their columns. z, the row's sum of e^(x - lse), is formed here once more: float32 holds lse to 2^-24 of the logits' size, so that z is 1
// for small ones only (a row of the type's lowest value has lse equal to it, and z is the row's length).
// WAVES wavefronts take a row or, with WAVES = 0, a group of 2^shift lanes of one. A lane keeps its first HELD vectors of the row between
// the sum and the results and reads what is behind them twice; it writes only columns that it alone reads, after the sum. Memory bounds
// it, one reading and one writing (8192 x 32768 bfloat16: 201 to 213 us call after call, 5.0 to 5.3 TB/s, and with lse taken for exact, without
// the sum, 202; 2048 x 131072, three quarters of it read twice, 237 and 201); of a single row the one compute unit that it is on (131072 columns: 22).
template <class T, int WAVES, int HELD, bool TOP>
__global__ __launch_bounds__(WAVES > kWaves ? WAVES * kWave : kThreads, 4) void k_labels_grad(const T* x, size_t ld, u32 rows, u32 cols, int top, u32 shift,
                                                                                         GradIn g, T* dx, size_t lddx) {
  constexpr u32 kBlock = WAVES > kWaves ? WAVES * kWave : kThreads;
  __shared__ float sums[WAVES > 1 ? WAVES : 1];
  const u32 lanes = WAVES ? WAVES * kWave : 1u << shift, per = WAVES ? kBlock / (WAVES * kWave) : kBlock >> shift;
  // whole vectors, and what is left behind them, the next lane's
  const u32 q = threadIdx.x & (lanes - 1), vectors = cols / 8, rest = q == (vectors & (lanes - 1)) ? cols % 8 : 0;
  for (u32 r0 = blockIdx.x * per; r0 < rows; r0 += gridDim.x * per) {
    u32 mine = r0 + (WAVES ? threadIdx.x / (WAVES * kWave) : threadIdx.x >> shift);
    if (WAVES) mine = (u32)__builtin_amdgcn_readfirstlane((int)mine);
    const u32 r = mine < rows ? mine : rows - 1;
    const T* const row = x + (size_t)r * ld;
    T* const out = dx + (size_t)r * lddx;
    const float lse = g.lse[r];
    Vec8<T> held[HELD], tail = {};
    const auto load = [&](u32 base) {
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (base + i * lanes < vectors) held[i] = load_wide(row + (base + i * lanes) * 8);
    };
    float z = 0.0f;
    const auto add = [&](const Vec8<T>& v) {
#pragma unroll
      for (int j = 0; j < 8; ++j) z += __builtin_amdgcn_exp2f(((float)v.get(j) - lse) * kLog2e);
    };
    if (rest) tail = load_some(row + vectors * 8, (int)rest, (T)neg_inf());
    for (u32 base = q + HELD * lanes; base < vectors; base += HELD * lanes) {
      load(base);
#pragma unroll
      for (int i = 0; i < HELD; ++i)
        if (base + i * lanes < vectors) add(held[i]);
    }
    load(q);
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (q + i * lanes < vectors) add(held[i]);
    if (rest) add(tail);
    for (u32 d = 1; d < (lanes < kWave ? lanes : kWave); d <<= 1) z += lane_read(z, (int)(lane_id() ^ d));
    if (WAVES > 1) {
      if (lane_id() == 0) sums[threadIdx.x / kWave] = z;
      __syncthreads();
      z = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) z += sums[w];
      __syncthreads();
    }
    const float dh = g.dentropy ? g.dentropy[r] : 0.0f, by = 1.0f / z, log_p = g.entropy[r] - logf(z);
    const int label = g.label[r];
    const float dlogp = (u32)label < cols ? g.dlogp[r] : 0.0f;
    const int* const top_index = g.top_index + (size_t)r * top;
    const float* const dtop = g.dtop + (size_t)r * top;
    float given = dlogp;
    u32 hits = 0;  // which of this lane's vectors hold alternatives, bit by bit, the last bit for all from the 32nd on
    const auto turn_of = [&](u32 vector) { return lowest(WAVES ? vector / (WAVES * kWave) : vector >> shift, 32); };
    if (TOP) {
#pragma unroll 4
      for (int k = 0; k < top; ++k) {  // (without a branch: the loads of several are on their way together)
        const u32 at = (u32)top_index[k];
        const float d = dtop[k];
        given += at < cols ? d : 0.0f;
        hits |= (at / 8 & (lanes - 1)) == q ? 1u << turn_of(at / 8) : 0u;
      }
    }
    const auto result = [&](Vec8<T> v, u32 col) {
      // the words alone are kept, rather than the exponentials of all: registers are short
#pragma unroll
      for (u32 n = 0; n < sizeof(T) / 2; ++n) asm volatile("" : "+v"(v.w[n]));
      float d[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float far = (float)v.get(j) - lse, product = far * kLog2e;
        float p = __builtin_amdgcn_exp2f(product) * by;
        // what the product's rounding took from the exponent, 2^-24 of it, shows in 32-bit results alone
        const float more = sizeof(T) == 4 ? (fmaf(far, kLog2e, -product) + far * kLog2eRest) * kLn2 : 0.0f;
        d[j] = p == 0.0f ? 0.0f : fmaf(p, more, p) * (-given - dh * (far + log_p));
      }
      const auto give = [&](u32 at, float more) {
        const u32 place = at - col;
        if (place < 8u && at < cols) {
#pragma unroll
          for (u32 j = 0; j < 8; ++j) d[j] += place == j ? more : 0.0f;
        }
      };
      give((u32)label, dlogp);
      if (TOP && (hits >> turn_of(col / 8) & 1))
        for (int k = 0; k < top; ++k) {
          const u32 at = (u32)top_index[k];
          if (at - col < 8u) give(at, dtop[k]);
        }
      Vec8<T> res = {};
#pragma unroll
      for (int j = 0; j < 8; ++j) res.set(j, (T)(lse == neg_inf() ? 0.0f : d[j]));
      return res;
    };
    const auto put = [&](u32 base) {
#pragma unroll
      for (int i = 0; i < HELD; ++i) {
        if (base + i * lanes < vectors) store_wide(out + (base + i * lanes) * 8, result(held[i], (base + i * lanes) * 8));
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (mine >= rows) continue;
    put(q);
    for (u32 base = q + HELD * lanes; base < vectors; base += HELD * lanes) {
      load(base);
      put(base);
    }
    if (rest) store_some(out + vectors * 8, result(tail, vectors * 8), (int)rest);
  }
}

u32 label_parts(size_t rows, size_t cols) {
  if (cols <= kWaveCols || rows == 0 || rows >= kSplitBlocks) return 1;
  const size_t want = kSplitBlocks / rows, most = ceil_div(cols, kSplitCols);
  return (u32)(want < most ? (want ? want : 1) : most);
}

bool label_sizes(int type, size_t rows, size_t cols, size_t top) {
  return valid_type(type) && rows <= kMostCount && cols >= 1 && cols <= kMostCount - 16 && top <= HAFLO_LABEL_MAX_TOP && top <= cols;
}

size_t label_bytes(size_t rows, size_t cols, size_t top) {
  const size_t parts = label_parts(rows, cols);
  return parts == 1 ? 0 : align256(rows * parts * sizeof(Part)) + rows * parts * top * 8;
}

template <class T>
int label_forward(const T* x, size_t ld, size_t rows, size_t cols, size_t top, const LabelOut& o, void* ws, hipStream_t st) {
  const u32 parts = label_parts(rows, cols);
  Part* part = (Part*)ws;
  u64* lists = (u64*)((char*)ws + align256(rows * parts * sizeof(Part)));
  if (cols <= kSmallCols) {
    hipLaunchKernelGGL((k_labels_small<T>), dim3((unsigned)ceil_div(rows, kThreads)), dim3(kThreads), 0, st, x, ld, (u32)rows, (u32)cols, (int)top, o);
    return launched();
  }
#define HAFLO_LOCAL_RUN(W, TOP, BLOCKS)                                                                                                       \
  in_turns(BLOCKS, kThreads, [&](u32 first, dim3 grid, dim3 block) {                                                                         \
    hipLaunchKernelGGL((k_labels<T, W, TOP>), grid, block, 0, st, x, ld, (u32)rows, (u32)cols, (int)top, parts, o, part, lists, first);       \
  })
  if (cols <= kWaveCols || (cols <= kManyWaveCols && rows >= kManyRows)) {
    if (top) HAFLO_LOCAL_RUN(1, true, ceil_div(rows, kWaves));
    else HAFLO_LOCAL_RUN(1, false, ceil_div(rows, kWaves));
  } else {
    if (top) HAFLO_LOCAL_RUN(kWaves, true, rows * parts);
    else HAFLO_LOCAL_RUN(kWaves, false, rows * parts);
  }
#undef HAFLO_LOCAL_RUN
  if (parts > 1) {
    if (top)
      hipLaunchKernelGGL((k_label_join<T, true>), dim3((unsigned)rows), dim3(kJoinWaves * kWave), 0, st, x, ld, (u32)cols, (int)top, parts, o, part, lists);
    else
      hipLaunchKernelGGL((k_label_join<T, false>), dim3((unsigned)rows), dim3(kWave), 0, st, x, ld, (u32)cols, (int)top, parts, o, part, lists);
  }
  return launched();
}

template <class T>
int label_backward(const T* x, size_t ld, size_t rows, size_t cols, size_t top, const GradIn& g, T* dx, size_t lddx, hipStream_t st) {
  // Few rows to a wavefront where they fill its lanes, few wavefronts to a row where they hold it: barriers and idle lanes cost more than the
  // registers. us by groups and by wavefronts: 16384 x 2000 bfloat16 26 and 28, x 1000 float32 24 and 26. By one wavefront and by four: 16384
  // x 2500 bfloat16 37 and 53, x 4000 50 and 50, x 4100 54 and 62, x 5000 69 and 71; float32 x 2500 62 and 80, x 4000 101 and 93, x 5000 137 and
  // 117. By four and by eight: 8192 x 12000 bfloat16 76 and 90, x 16500 106 and 129; float32 x 16500 211 and 203. By eight and by
  // sixteen: 4096 x 32768 bfloat16 112 and 125, x 33000 120 and 133, 2048 x 131072 250 and 237; float32 x 131072 562 and 510. Rows of 16 bits
  // are so taken on to a quarter more than is held.
  constexpr int kHeld = sizeof(T) == 2 ? 4 : 2;  // vectors of a lane in a group: 64 bytes
  u32 shift = 0;  // of a group's lanes
  while ((size_t)(8 * kHeld) << shift < cols && shift < 6) ++shift;
#define HAFLO_LOCAL_RUN(WAVES, HELD, PER, THREADS)                                                                                     \
  do {                                                                                                                               \
    const size_t most = HAFLO_LOCAL_LANES / (THREADS) < kGradBlocks ? HAFLO_LOCAL_LANES / (THREADS) : kGradBlocks;                   \
    const dim3 grid((unsigned)(ceil_div(rows, PER) < most ? ceil_div(rows, PER) : most)), block(THREADS);                            \
    if (g.dtop)                                                                                                                      \
      hipLaunchKernelGGL((k_labels_grad<T, WAVES, HELD, true>), grid, block, 0, st, x, ld, (u32)rows, (u32)cols, (int)top, shift, g, dx, lddx); \
    else                                                                                                                             \
      hipLaunchKernelGGL((k_labels_grad<T, WAVES, HELD, false>), grid, block, 0, st, x, ld, (u32)rows, (u32)cols, 0, shift, g, dx, lddx); \
  } while (0)
  constexpr size_t kFull = 8 * kWave * 8, kPast = sizeof(T) == 2 ? kFull * 5 / 4 : kFull;  // what a wavefront holds, and how far it goes
  if (cols <= 8 * kWave * kHeld) HAFLO_LOCAL_RUN(0, kHeld, (size_t)kThreads >> shift, kThreads);
  else if (cols <= kPast) HAFLO_LOCAL_RUN(1, 8, kWaves, kThreads);
  else if (cols <= 4 * kPast) HAFLO_LOCAL_RUN(4, 8, 1, 4 * kWave);
  else if (cols <= 8 * kPast) HAFLO_LOCAL_RUN(8, 8, 1, 8 * kWave);
  else HAFLO_LOCAL_RUN(16, 4, 1, 16 * kWave);
#undef HAFLO_LOCAL_RUN
  return launched();
}

}  // namespace

extern "C" {

size_t haflo_label_workspace_bytes(int type, size_t rows, size_t cols, size_t top) {
  return label_sizes(type, rows, cols, top) ? label_bytes(rows, cols, top) : (size_t)-1;
}

int haflo_label_logprobs(int type, const void* d_logits, size_t ld, const int32_t* d_label, size_t rows, size_t cols,
                         size_t top, float* d_logp, float* d_entropy, float* d_lse, float* d_top_logp,
                         int32_t* d_top_index, uint32_t* d_status, void* d_workspace, size_t workspace_bytes, void* stream) {
  if (!label_sizes(type, rows, cols, top)) return HAFLO_EINVAL;
  if (rows == 0) return HAFLO_OK;
  if (!d_logits || ld < cols || !d_label || !d_logp || !d_entropy || !d_lse || (top && (!d_top_logp || !d_top_index))) return HAFLO_EINVAL;
  const size_t bytes = label_bytes(rows, cols, top);
  if (!enough(d_workspace, workspace_bytes, bytes)) return HAFLO_EINVAL;
  const LabelOut o = {d_label, d_logp, d_entropy, d_lse, d_top_logp, d_top_index, d_status};
  HAFLO_LOCAL_TYPES(type, return label_forward<T>((const T*)d_logits, ld, rows, cols, top, o, d_workspace, (hipStream_t)stream));
}

int haflo_label_logprobs_backward(int type, const void* d_logits, size_t ld, const int32_t* d_label, const float* d_lse,
                                  const float* d_entropy, const float* d_dlogp, const float* d_dentropy,
                                  const int32_t* d_top_index, const float* d_dtop, size_t rows, size_t cols, size_t top,
                                  void* d_dx, size_t lddx, void* stream) {
  if (!label_sizes(type, rows, cols, top)) return HAFLO_EINVAL;
  if (rows == 0) return HAFLO_OK;
  if (!d_logits || ld < cols || !d_label || !d_lse || !d_entropy || !d_dlogp || (d_dtop && top && !d_top_index) || !d_dx || lddx < cols)
    return HAFLO_EINVAL;
  if (!in_place(d_logits, ld, d_dx, lddx, rows)) return HAFLO_EINVAL;
  const GradIn g = {d_label, d_lse, d_entropy, d_dlogp, d_dentropy, d_top_index, top ? d_dtop : nullptr};
  HAFLO_LOCAL_TYPES(type, return label_backward<T>((const T*)d_logits, ld, rows, cols, top, g, (T*)d_dx, lddx, (hipStream_t)stream));
}

}  // extern "C"
