// A projection that all parties share with each row's own low-rank adapter beside it, and its gradients.
//
//   forward   h[t] = scale A[a] drop(x[t]),      y[t] = W x[t] + B[a] h[t]           a = the row's adapter
//   backward  g[t] = scale B[a]^T dy[t],         dx[t] = W^T dy[t] + drop'(A[a]^T g[t])
//             dA[a] = sum_t g[t] drop(x[t])^T,   dB[a] = sum_t dy[t] h[t]^T
//
// h and g, the rows' short vectors ("z" where a kernel serves both directions), come from k_shrink. k_project forms
// the large product and adds the adapters' part, k_few does for few rows. k_prepare lists the rows by
// adapter: a tile's rows are taken from that list, so that they share one adapter as a rule, whatever the order the
// caller has them in, and k_grad sums over the rows of one adapter. It also lays out anew what reduces along columns (W, A and B
// of the backward pass) and, for k_project, operands whose rows do not begin at 16-byte boundaries.
#include "local_common.hpp"

using namespace haflo::local;

namespace {

constexpr int kThreads = 256;

template <class T>
constexpr int step_elems() {  // of the reduction in one step of k_project: 128 bytes of a row
  return 128 / (int)sizeof(T);
}

__device__ __forceinline__ int party_of(const int* index, u32 t, u32 parties) {
  const int a = index[t];
  return (u32)a < parties ? a : -1;
}

// a place below `count`, the last one for those behind it
__device__ __forceinline__ u32 lowest(u32 i, u32 count) { return i < count ? i : count - 1; }

// Eight elements at column k of a row of `cols`, in two steps: a load without a branch, as the compiler waits for a load at the
// next branch around one, and where the elements pass the row's end, so the row's last eight were loaded, their moving to
// their places, with zeros behind them. Rows of less than eight are loaded element by element.
template <class T>
__device__ __forceinline__ Vec8<T> load_row(const T* row, u32 k, u32 cols) {
  return load_wide(row + (k + 8 <= cols ? k : cols - 8));
}
template <class T>
__device__ __forceinline__ Vec8<T> load_short(const T* row, u32 k, u32 cols) {
  return load_some(row, k == 0 ? (int)cols : 0);
}
template <class T>
__device__ __forceinline__ void settle(Vec8<T>& v, u32 k, u32 cols) {
  if (k + 8 <= cols || cols < 8) return;
  const u32 by = k + 8 - cols;
  const Vec8<T> was = v;
  v = Vec8<T>{};
#pragma unroll
  for (u32 n = 1; n < 8; ++n)
    if (by == n) {
#pragma unroll
      for (u32 j = 0; j + n < 8; ++j) v.set(j, was.get(j + n));
    }
}
template <class T>
__device__ __forceinline__ void apply_drop(Vec8<T>& v, const Drop& d, u32 row, u32 k) {
  const u32x4 draws = philox(d, k >> 3, row);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (sizeof(T) == 4) v.w[j >> 2][j & 3] = kept(d, draws, j) ? v.w[j >> 2][j & 3] : 0u;
    else v.w[0][j >> 1] &= kept(d, draws, j) ? 0xFFFFFFFFu : j & 1 ? 0x0000FFFFu : 0xFFFF0000u;
  }
}
// Rows that several wavefronts multiply go through LDS, 1024 bytes of each at a time.
constexpr int kRowBytes = 1024;
// eight elements, the q-th of a row in LDS; pieces of 16 bytes of sixteen rows lie on different banks
template <class T>
__device__ __forceinline__ T* row_piece(T* tile, u32 row, u32 q, u32 e) {
  constexpr u32 kPieces = sizeof(T) / 2;  // of eight elements
  return tile + row * (kRowBytes / sizeof(T)) + ((q * kPieces + e) ^ (row & 15)) * (16 / sizeof(T));
}
template <class T>
__device__ __forceinline__ void put_row(T* tile, u32 row, u32 q, const Vec8<T>& v) {
#pragma unroll
  for (u32 e = 0; e < sizeof(T) / 2; ++e) *(u32x4*)row_piece(tile, row, q, e) = v.w[e];
}
template <class T>
__device__ __forceinline__ Vec8<T> get_row(T* tile, u32 row, u32 q) {
  Vec8<T> v;
#pragma unroll
  for (u32 e = 0; e < sizeof(T) / 2; ++e) v.w[e] = *(const u32x4*)row_piece(tile, row, q, e);
  return v;
}

// z[t, r] = scale[a] s sum_k drop(x[t, k]) F[a][r, k], F rows f_ld apart; z rows z_ld long with zeros behind the rank, h without.
// A block takes sixteen rows of `order` and one part of the reduction, its wavefronts some steps in turn each; once for every
// party among the rows. Rows behind the last, of x and of F, are the last one again: what they give is left aside.
// Reading x bounds it: 8192 x 4096 bfloat16 with rank 16, 28 to 33 us, 2.0 to 2.4 TB/s; with the rows brought to LDS by all
// wavefronts first and multiplied from there 28 to 40.
constexpr int kShrinkWaves = 4;
template <class T, int RT>
__global__ __launch_bounds__(kShrinkWaves * kWave) void k_shrink(const T* x, size_t ldx, const T* f, size_t f_ld, const float* scale, const int* index,
                                                                 const u32* order, u32 rows, u32 inner, u32 rank, u32 parties, Drop d, u32 parts,
                                                                 u32 z_ld, float* z, float* h, u32* status, u32 first_block) {
  constexpr int kAhead = RT == 1 ? 4 : 2;  // steps whose operands are on their way together
  __shared__ float sum[kShrinkWaves][RT][16][17];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const u32 block = first_block + blockIdx.x, at0 = block / parts * 16, part = block % parts;
  const auto row_at = [&](u32 i) { return at0 + i >= rows ? rows : order[at0 + i]; };
  const u32 mine = row_at(lane % 16);
  const int raw = mine < rows ? index[mine] : -1;
  const int a = (u32)raw < parties ? raw : -1;
  if (status && part == 0 && threadIdx.x < 16 && raw != a && raw != -1) atomicOr(status, HAFLO_ST_RANGE);
  // the part's share of the reduction, in steps of 32
  const u32 steps = (inner + 31) / 32, first = (u32)((u64)steps * part / parts), end = (u32)((u64)steps * (part + 1) / parts);
  float own[RT];  // of row out_i, r = lane % 16
#pragma unroll
  for (int i = 0; i < RT; ++i) own[i] = 0.0f;
  const u32 out_i = lane / 16 * 4 + wave;
  const u32 out_t = row_at(out_i);
  const int out_a = out_t < rows ? party_of(index, out_t, parties) : -1;
  const T* const x_row = x + (size_t)lowest(mine, rows) * ldx;
  size_t f_at[RT];
#pragma unroll
  for (int i = 0; i < RT; ++i) f_at[i] = (size_t)lowest(i * 16 + lane % 16, rank) * f_ld;
  u64 left = __builtin_amdgcn_ballot_w64(a >= 0) & 0xFFFF;
  while (left) {
    const int who = __builtin_amdgcn_readlane(a, __builtin_ctzll(left));
    left &= ~__builtin_amdgcn_ballot_w64(a == who);
    const T* fa = f + (size_t)who * rank * f_ld;
    f32x4 acc[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (u32 s0 = first + wave * kAhead; s0 < end; s0 += kShrinkWaves * kAhead) {
      Vec8<T> xv[kAhead], fv[kAhead][RT];
      u32 k[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) k[u] = s0 + u < end ? (s0 + u) * 32 + lane / 16 * 8 : inner;
      if (inner >= 8) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          xv[u] = load_row(x_row, k[u], inner);
#pragma unroll
          for (int i = 0; i < RT; ++i) fv[u][i] = load_row(fa + f_at[i], k[u], inner);
        }
      } else {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          xv[u] = load_short(x_row, k[u], inner);
#pragma unroll
          for (int i = 0; i < RT; ++i) fv[u][i] = load_short(fa + f_at[i], k[u], inner);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        settle(xv[u], k[u], inner);
#pragma unroll
        for (int i = 0; i < RT; ++i) settle(fv[u][i], k[u], inner);
        if (d.threshold) apply_drop(xv[u], d, mine, (s0 + u) * 32 + lane / 16 * 8);
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[i] = mma32(fv[u][i], xv[u], acc[i]);
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
        const u32 r = lane % 16;
        float s = 0.0f;
#pragma unroll
        for (int v = 0; v < kShrinkWaves; ++v) s += sum[v][i][out_i][r];
        own[i] = s;
      }
    }
    __syncthreads();
  }
  if (out_t < rows) {
    const float by = out_a < 0 ? 0.0f : scale[out_a] * (d.threshold ? d.scale : 1.0f);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const u32 r = i * 16 + lane % 16;
      if (r < z_ld) z[((size_t)part * rows + out_t) * z_ld + r] = r < rank ? own[i] * by : 0.0f;
      if (h && r < rank) h[(size_t)out_t * rank + r] = own[i] * by;
    }
  }
}

// A lane an element (3001 rows, 3 us: a launch): z[i] = sum over parts, and without the places behind the rank to h
__global__ __launch_bounds__(kThreads) void k_join(const float* in, u32 parts, size_t count, u32 z_ld, u32 rank, float* z, float* h) {
  const size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= count) return;
  float s = 0.0f;
  for (u32 p = 0; p < parts; ++p) s += in[p * count + i];
  if (z) z[i] = s;
  const u32 r = (u32)(i % z_ld);
  if (h && r < rank) h[i / z_ld * rank + r] = s;
}

// ---------------------------------------------------------------------------------------------------
// The adapters' part of k_project: matrix instructions in 32 bits, as z is float32 and may cancel against the large product, and an
// infinity of z or of an adapter must meet the other's whole element. Lane l holds four ranks from 4 (l / 16) on of its row.
// z and the adapters' rows are `ranks` long, a multiple of sixteen, with zeros behind the rank.
constexpr u32 kRanks = 16;
__device__ __forceinline__ f32x4 low_of_z(const float* z) {
  f32x4 v;
  __builtin_memcpy(&v, __builtin_assume_aligned(z + lane_id() / 16 * 4, 16), sizeof(v));
  return v;
}
template <class T>
__device__ __forceinline__ f32x4 low_of_f(const T* f) {
  T t[4];
  __builtin_memcpy(t, __builtin_assume_aligned(f + lane_id() / 16 * 4, 4 * sizeof(T)), sizeof(t));
  return f32x4{(float)t[0], (float)t[1], (float)t[2], (float)t[3]};
}
__device__ __forceinline__ f32x4 low_mma(const f32x4& f, const f32x4& z, f32x4 acc) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(f[e], z[e], acc, 0, 0, 0);
  return acc;
}

// Where the rows of a tile are loaded from, sixteen bytes a lane straight into LDS, lane l's to `to` + 16 l. Matrices below
// 4 GiB are read as buffers, whose offsets are 32-bit words and whose loads the compiler counts one by one; FAR ones are not.
template <class T, bool FAR>
struct Source;
template <class T>
struct Source<T, false> {
  using At = u32;
  __amdgpu_buffer_rsrc_t buffer;
  __device__ __forceinline__ Source(const T* p, u32 bytes) : buffer(__builtin_amdgcn_make_buffer_rsrc((void*)p, 0, bytes, 0x00027000)) {}
  static __device__ __forceinline__ At at(u32 row, size_t ld, u32 k) { return (row * (u32)ld + k) * (u32)sizeof(T); }
  __device__ __forceinline__ void load(At at, u32 k, void* to) const {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer, (__attribute__((address_space(3))) void*)to, 16, (int)at, (int)(k * (u32)sizeof(T)), 0, 0);
  }
};
template <class T>
struct Source<T, true> {
  using At = size_t;
  const T* p;
  __device__ __forceinline__ Source(const T* p_, u32) : p(p_) {}
  static __device__ __forceinline__ At at(u32 row, size_t ld, u32 k) { return row * ld + k; }
  __device__ __forceinline__ void load(At at, u32 k, void* to) const {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p + at + k), (__attribute__((address_space(3))) void*)to, 16, 0, 0);
  }
};
// Until this wavefront's loads but the latest LATER have arrived and its reads of LDS are done, and all other
// wavefronts of the block are there too.
template <int LATER>
__device__ __forceinline__ void wait_for_tiles() {
  asm volatile("" ::: "memory");
  static_assert(LATER < 16, "");
  __builtin_amdgcn_s_waitcnt(0x70 + LATER);  // vmcnt(LATER) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// A tile's row in LDS is 128 bytes, eight pieces of 16; piece c of row r lies at place c ^ (r / 2) % 8, which spreads the
// sixteen rows that lanes read at once over all banks.
__device__ __forceinline__ u32 place_of(u32 row, u32 piece) { return piece ^ (row >> 1 & 7); }
template <class T>
__device__ __forceinline__ Vec8<T> load_frag(const T* tile, u32 row, u32 k) {  // eight elements from the k-th of a row
  constexpr u32 kPer = 16 / sizeof(T);
  Vec8<T> v;
#pragma unroll
  for (u32 i = 0; i < 8 / kPer; ++i)
    v.w[i] = *(const u32x4*)(tile + row * step_elems<T>() + place_of(row, k / kPer + i) * kPer);
  return v;
}

// Four sums with the draws that two words hold.
__device__ __forceinline__ void drop_four(f32x4& v, const Drop& d, u32 lo, u32 hi) {
  v[0] = (lo & 0xFFFFu) >= d.threshold ? v[0] * d.scale : 0.0f;
  v[1] = (lo >> 16) >= d.threshold ? v[1] * d.scale : 0.0f;
  v[2] = (hi & 0xFFFFu) >= d.threshold ? v[2] * d.scale : 0.0f;
  v[3] = (hi >> 16) >= d.threshold ? v[3] * d.scale : 0.0f;
}

// The operands that a wavefront multiplies next: its outputs by XN sixteens of its rows.
template <class T, int OT, int XN>
struct Frags {
  Vec8<T> w[OT], x[XN];
};
template <class T, int OT, int XN>
__device__ __forceinline__ void load_w(Frags<T, OT, XN>& f, const T* tile, u32 out0, u32 s) {
#pragma unroll
  for (int i = 0; i < OT; ++i) f.w[i] = load_frag(tile, out0 + i * 16 + lane_id() % 16, s * 32 + lane_id() / 16 * 8);
}
template <class T, int OT, int XN>
__device__ __forceinline__ void load_x(Frags<T, OT, XN>& f, const T* tile, u32 row0, u32 s, u32 part) {
#pragma unroll
  for (int j = 0; j < XN; ++j) f.x[j] = load_frag(tile, row0 + (part * XN + j) * 16 + lane_id() % 16, s * 32 + lane_id() / 16 * 8);
}

// Half (0: the first, 1: the second) of this wavefront's loads of both tiles at `k`, in LDS rows of whole steps.
template <class T, int TM, int TN, int WAVES, class From>
__device__ __forceinline__ void ask_tiles(int half, const From& x, const typename From::At (&at_x)[TM / 8 / WAVES], const From& w,
                                          const typename From::At (&at_w)[TN / 8 / WAVES], u32 k, u32 wave, T* lx, T* lw) {
  constexpr int LX = TM / 8 / WAVES, LW = TN / 8 / WAVES;
#pragma unroll
  for (int i = half * LX / 2; i < (half + 1) * LX / 2; ++i) x.load(at_x[i], k, lx + (i * WAVES + wave) * 8 * step_elems<T>());
#pragma unroll
  for (int i = half * LW / 2; i < (half + 1) * LW / 2; ++i) w.load(at_w[i], k, lw + (i * WAVES + wave) * 8 * step_elems<T>());
}

// One step of the reduction, with the first operands in `f`. Operands are read from LDS under the products before theirs, a
// read between every few of them. Before the last products the next step's tiles are waited for; the tiles after those are then asked for
// in place of this step's, one half under the last products and the other under the next step's first, so that the loads
// neither hold the products up at one place nor are waited for before three quarters of a step are over.
template <class T, int TM, int TN, int WAVES, class From, int XN, int RT, int OT>
__device__ __forceinline__ void project_step(const From& x, const typename From::At (&at_x)[TM / 8 / WAVES], const From& w,
                                             const typename From::At (&at_w)[TN / 8 / WAVES], u32 k_next, u32 k_after, u32 wave, u32 row0,
                                             u32 out0, T* cx, T* cw, T* nx, T* nw,
                                             Frags<T, OT, XN>& f, f32x4 (&acc)[OT][RT]) {
  constexpr int KE = step_elems<T>(), kSub = KE / 32, kParts = RT / XN, kAll = kSub * kParts;
  constexpr int kAsks = (TM + TN) / 8 / WAVES / 2, kReads = sizeof(T) / 2, kProducts = XN * OT * (sizeof(T) == 2 ? 1 : 8);
#pragma unroll
  for (int q = 0; q < kAll; ++q) {
    const int s = q / kParts, part = q % kParts;
    const bool last = q + 1 == kAll, new_w = last || (q + 1) / kParts != s;
    Frags<T, OT, XN> next;
    if (q == 0 && kAll > 1) ask_tiles<T, TM, TN, WAVES>(1, x, at_x, w, at_w, k_next, wave, nx, nw);
    if (last) {
      wait_for_tiles<0>();
      ask_tiles<T, TM, TN, WAVES>(0, x, at_x, w, at_w, k_after, wave, cx, cw);
      if (kAll == 1) ask_tiles<T, TM, TN, WAVES>(1, x, at_x, w, at_w, k_after, wave, cx, cw);
    }
    load_x(next, last ? nx : cx, row0, last ? 0 : (q + 1) / kParts, last ? 0 : (q + 1) % kParts);
    if (new_w) {
      load_w(next, last ? nw : cw, out0, last ? 0 : s + 1);
    } else {
#pragma unroll
      for (int i = 0; i < OT; ++i) next.w[i] = f.w[i];
    }
#pragma unroll
    for (int j = 0; j < XN; ++j)
#pragma unroll
      for (int i = 0; i < OT; ++i) acc[i][part * XN + j] = mma32(f.w[i], f.x[j], acc[i][part * XN + j]);
    // a load, where there are any, and one or more reads of LDS with products between them
    constexpr int kSlots = kAsks < 4 ? kAsks : 4;
#pragma unroll
    for (int n = 0; n < kSlots; ++n) {
      if (last || q == 0) __builtin_amdgcn_sched_group_barrier(0x010, kAsks / kSlots, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, kProducts / kSlots / 4, 0);
      if (new_w) __builtin_amdgcn_sched_group_barrier(0x100, (XN + OT) * kReads / kSlots, 0);
      else __builtin_amdgcn_sched_group_barrier(0x100, XN * kReads / kSlots, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, kProducts / kSlots / 2, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    f = next;
  }
}

// The whole reduction of a tile. That the four tiles in LDS are told apart here, and only here, is what lets the compiler see which reads
// need not wait for the loads on their way.
template <class T, int TM, int TN, int WAVES, class From, int RT, int OT>
__device__ __forceinline__ void reduce(const From& x, const typename From::At (&at_x)[TM / 8 / WAVES], const From& w,
                                       const typename From::At (&at_w)[TN / 8 / WAVES], u32 steps, u32 wave, u32 row0, u32 out0,
                                       T* __restrict__ lx0, T* __restrict__ lw0, T* __restrict__ lx1, T* __restrict__ lw1, f32x4 (&acc)[OT][RT]) {
  constexpr int KE = step_elems<T>(), XN = RT < 4 ? RT : 4;
  const u32 inner = steps * KE;
  const auto after = [&](u32 at) { return at + KE < inner ? at + KE : 0; };
  u32 k = after(0);
  ask_tiles<T, TM, TN, WAVES>(0, x, at_x, w, at_w, 0, wave, lx0, lw0);
  ask_tiles<T, TM, TN, WAVES>(1, x, at_x, w, at_w, 0, wave, lx0, lw0);
  ask_tiles<T, TM, TN, WAVES>(0, x, at_x, w, at_w, k, wave, lx1, lw1);
  if (KE / 32 * (RT / XN) == 1) ask_tiles<T, TM, TN, WAVES>(1, x, at_x, w, at_w, k, wave, lx1, lw1);
  Frags<T, OT, XN> frags;
  wait_for_tiles<(TM + TN) / 8 / WAVES / 2>();
  load_x(frags, lx0, row0, 0, 0);
  load_w(frags, lw0, out0, 0);
  // the loads go round past the last step, rather than that the loop has other forms for its end
  for (u32 i = 0;; i += 2) {
    const u32 k2 = after(k), k3 = after(k2);
    project_step<T, TM, TN, WAVES>(x, at_x, w, at_w, k, k2, wave, row0, out0, lx0, lw0, lx1, lw1, frags, acc);
    if (i + 1 >= steps) break;
    project_step<T, TM, TN, WAVES>(x, at_x, w, at_w, k2, k3, wave, row0, out0, lx1, lw1, lx0, lw0, frags, acc);
    if (i + 2 >= steps) break;
    k = k3;
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): none of them arrives after the block's end
}

// y[t, o] = drop'(sum_r z[t, r] F[a][o, r]) + sum_k x[t, k] W[o, k], inner a multiple of a step. A block takes TM rows (of
// `order`) by TN outputs, its WM x WN wavefronts a part of that each in products of 16 x 16. Two steps' tiles lie in LDS: one
// is filled while the other is read. Matrix instructions and the reads of LDS between them bound the large tiles (8192 x 4096
// to 4096, bfloat16: 231 us, 1190 TFLOP/s; a call 301 instead of 238 by tiles of 128 x 128), the wait for each step's loads the small
// ones (float16 3001 x 1001 to 515: 14 us, 221 TFLOP/s).
template <class T, int TM, int TN, int WM, int WN, bool DROP, bool FAR>
__global__ __launch_bounds__(WM * WN * kWave) void k_project(const T* x, size_t ldx, const T* w, size_t ldw, const T* f, const float* z,
                                                             const int* index, const u32* order, const u32* begin, u32 rows, u32 inner,
                                                             u32 outer, u32 parties, u32 ranks, Drop d, T* y, size_t ldy, u32 x_bytes, u32 w_bytes,
                                                             u32 first_block) {
  constexpr int KE = step_elems<T>(), WAVES = WM * WN, RT = TM / WM / 16, OT = TN / WN / 16;
  constexpr int LX = TM / 8 / WAVES, LW = TN / 8 / WAVES;
  __shared__ __align__(16) T lds[2 * (TM + TN) * KE];
  T* const lx0 = lds;
  T* const lw0 = lx0 + TM * KE;
  T* const lx1 = lw0 + TN * KE;
  T* const lw1 = lx1 + TM * KE;
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  // Blocks are dealt to the eight dies in turn: each gets neighbouring tiles, four tiles of rows by all outputs at a time,
  // whose operands its cache holds.
  const u32 tiles_m = (rows + TM - 1) / TM, tiles_n = (outer + TN - 1) / TN, tiles = tiles_m * tiles_n;
  const u32 block = first_block + blockIdx.x, die = block % 8, per = tiles / 8, over = tiles % 8;
  const u32 tile = die * per + (die < over ? die : over) + block / 8;
  const u32 band = tile / (4 * tiles_n), in_band = tile % (4 * tiles_n), high = tiles_m - band * 4 < 4 ? tiles_m - band * 4 : 4;
  const u32 t0 = (band * 4 + in_band % high) * TM, o0 = in_band / high * TN;
  const u32 row0 = wave / WN * (TM / WM), out0 = wave % WN * (TN / WN);  // this wavefront's corner

  using From = Source<T, FAR>;
  const From from_x(x, x_bytes), from_w(w, w_bytes);
  typename From::At at_x[LX], at_w[LW];  // this lane's pieces
#pragma unroll
  for (int i = 0; i < LX; ++i) {
    const u32 r = (i * WAVES + wave) * 8 + lane / 8, at = t0 + r < rows ? t0 + r : rows - 1;
    at_x[i] = From::at(order[at], ldx, place_of(r, lane % 8) * (16 / sizeof(T)));
  }
#pragma unroll
  for (int i = 0; i < LW; ++i) {
    const u32 r = (i * WAVES + wave) * 8 + lane / 8, o = o0 + r < outer ? o0 + r : outer - 1;
    at_w[i] = From::at(o, ldw, place_of(r, lane % 8) * (16 / sizeof(T)));
  }
  f32x4 acc[OT][RT];
  u32 t[RT];  // this lane's rows, `rows`: none
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    const u32 at = t0 + row0 + j * 16 + lane % 16;
    t[j] = at < rows ? order[at] : rows;
#pragma unroll
    for (int i = 0; i < OT; ++i) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  reduce<T, TM, TN, WAVES>(from_x, at_x, from_w, at_w, inner / KE, wave, row0, out0, lx0, lw0, lx1, lw1, acc);

  // the adapters' part, party by party along the list
  const u32 wave_at = t0 + row0, listed = begin[parties], wave_end = wave_at + TM / WM < rows ? wave_at + TM / WM : rows;
  for (u32 at = wave_at; at < wave_end && at < listed;) {
    const int who = index[order[at]];
    const u32 next = begin[who + 1];
#pragma unroll
    for (int j = 0; j < RT; j += 2) {
      const u32 p = wave_at + j * 16 + lane % 16;
      const bool mine0 = p >= at && p < next, mine1 = p + 16 >= at && p + 16 < next;
      if (__builtin_amdgcn_ballot_w64(mine0 || mine1) == 0) continue;
      f32x4 low0[OT], low1[OT];
#pragma unroll
      for (int i = 0; i < OT; ++i) low0[i] = low1[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      for (u32 r0 = 0; r0 < ranks; r0 += kRanks) {
        const f32x4 v0 = low_of_z(z + (size_t)(t[j] < rows ? t[j] : 0) * ranks + r0);
        const f32x4 v1 = low_of_z(z + (size_t)(t[j + 1] < rows ? t[j + 1] : 0) * ranks + r0);
#pragma unroll
        for (int i = 0; i < OT; ++i) {
          const u32 o = o0 + out0 + i * 16 + lane % 16;
          const f32x4 fv = low_of_f(f + ((size_t)who * outer + (o < outer ? o : outer - 1)) * ranks + r0);
          low0[i] = low_mma(fv, v0, low0[i]);
          low1[i] = low_mma(fv, v1, low1[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < OT; ++i) {
        if (DROP) {
          // A lane's four outputs are half of a generator's call, the other half is the lane's beside it: of two rows' calls
          // each makes one, and they exchange halves.
          const bool odd = (lane & 16) != 0;
          const u32x4 draws = philox(d, (o0 + out0 + i * 16 + lane / 16 * 4) >> 3, t[j] ^ ((t[j] ^ t[j + 1]) & (0u - (u32)odd)));
          const u32 give0 = odd ? draws[0] : draws[2], give1 = odd ? draws[1] : draws[3];
          const u32 keep0 = odd ? draws[2] : draws[0], keep1 = odd ? draws[3] : draws[1];
          const u32 got0 = lane_read(give0, (int)(lane ^ 16)), got1 = lane_read(give1, (int)(lane ^ 16));
          drop_four(low0[i], d, odd ? got0 : keep0, odd ? got1 : keep1);
          drop_four(low1[i], d, odd ? keep0 : got0, odd ? keep1 : got1);
        }
        // nothing is added to other parties' rows, not even zeros' products: an adapter may hold infinities
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[i][j][e] += mine0 ? low0[i][e] : 0.0f;
          acc[i][j + 1][e] += mine1 ? low1[i][e] : 0.0f;
        }
      }
      __builtin_amdgcn_sched_barrier(0);  // one pair of rows at a time: the sums hold half of the registers
    }
    at = next;
  }

  // A lane holds four outputs of each of its rows: results of 16 bits go through the tiles' place in LDS, a wavefront's through its
  // own part of it, and leave in 16-byte pieces, a whole line or half a line of a row at a time.
  constexpr u32 kPieces = OT * 16 * sizeof(T) / 16, kShift = kPieces == 8 ? 1 : 2;
  if (sizeof(T) == 2) {
    __syncthreads();  // other wavefronts have read the last tiles
    T* const own = lds + wave * (RT * 16 * OT * 16);
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int i = 0; i < OT; ++i) {
        T v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (T)acc[i][j][e];
        const u32 r = j * 16 + lane % 16, piece = i * 2 + lane / 32;
        __builtin_memcpy(own + r * (OT * 16) + (piece ^ (r >> kShift & (kPieces - 1))) * 8 + (lane / 16 & 1) * 4, v, sizeof(v));
        __builtin_amdgcn_sched_barrier(0);
      }
    __builtin_amdgcn_wave_barrier();
    constexpr u32 kRows = kWave / kPieces;  // of one store
#pragma unroll
    for (u32 n = 0; n < RT * 16 / kRows; ++n) {
      const u32 r = n * kRows + lane / kPieces, piece = lane % kPieces;
      Vec8<T> v;
      v.w[0] = *(const u32x4*)(own + r * (OT * 16) + (piece ^ (r >> kShift & (kPieces - 1))) * 8);
      const u32 row = lane_read(t[n * kRows / 16], (int)(r % 16)), o = o0 + out0 + piece * 8;
      if (row >= rows || o >= outer) continue;
      T* const to = y + (size_t)row * ldy + o;
      if (o + 8 <= outer) store_wide(to, v);
      else store_some(to, v, (int)(outer - o));
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    if (t[j] >= rows) continue;
#pragma unroll
    for (int i = 0; i < OT; ++i) {
      const u32 o = o0 + out0 + i * 16 + lane / 16 * 4;
      T* const to = y + (size_t)t[j] * ldy + o;
      T v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (T)acc[i][j][e];
      if (o + 4 <= outer) {
        __builtin_memcpy(to, v, sizeof(v));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (o + e < outer) to[e] = v[e];
      }
    }
  }
}

// The same for few rows, in two launches. k_few reads W once for 64 rows: a block takes them, 64 outputs and one part of the reduction, 1024 bytes of
// every row at a time, its wavefronts four sixteens of outputs in two halves of that; further blocks form the parts of z = h or
// g for one row each, as k_shrink does. k_few_join adds the parts, and the adapters' part to them. What bounds it is the
// reading of W: 64 rows of 4096 to 4096 in bfloat16 take 16 us and 6 for the joining, one row 9.7 and 4.7.
constexpr int kFewWaves = 8;
template <class T, int RT, bool SHORT>
__device__ __forceinline__ void few_product(const T* x, size_t ldx, const T* w, size_t ldw, u32 rows, u32 inner, u32 outer, u32 tile, u32 part,
                                            u32 parts, size_t part_step, float* sums, T* lx, f32x4* half) {
  constexpr u32 kElems = kRowBytes / sizeof(T), kSteps = kElems / 32 / 2, kLanes = kElems / 8, kRows = kWave / kLanes;  // rows of a load
  constexpr u32 kLoads = RT * 16 / (kFewWaves * kRows);
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const u32 o = tile * 64 + wave % 4 * 16 + lane % 16;
  const u32 turns = (inner + kElems - 1) / kElems, first = (u32)((u64)turns * part / parts), end = (u32)((u64)turns * (part + 1) / parts);
  size_t x_at[kLoads];
#pragma unroll
  for (u32 i = 0; i < kLoads; ++i) x_at[i] = (size_t)lowest((i * kFewWaves + wave) * kRows + lane / kLanes, rows) * ldx;
  const T* const w_row = w + (size_t)lowest(o, outer) * ldw;
  f32x4 acc[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (u32 n = first; n < end; ++n) {
    Vec8<T> wv[kSteps], xv[kLoads];
    const u32 kx = n * kElems + lane % kLanes * 8, kw = n * kElems + wave / 4 * kSteps * 32 + lane / 16 * 8;
    const auto load = [&](const T* row, u32 k) { return SHORT ? load_short(row, k, inner) : load_row(row, k, inner); };
#pragma unroll
    for (u32 i = 0; i < kLoads; ++i) xv[i] = load(x + x_at[i], kx);
#pragma unroll
    for (u32 s = 0; s < kSteps; ++s) wv[s] = load(w_row, kw + s * 32);
    if (n != first) __syncthreads();
#pragma unroll
    for (u32 i = 0; i < kLoads; ++i) {
      settle(xv[i], kx, inner);
      put_row(lx, (i * kFewWaves + wave) * kRows + lane / kLanes, lane % kLanes, xv[i]);
    }
    __syncthreads();
#pragma unroll
    for (u32 s = 0; s < kSteps; ++s) {
      settle(wv[s], kw + s * 32, inner);
#pragma unroll
      for (int j = 0; j < RT; ++j) acc[j] = mma32(wv[s], get_row(lx, j * 16 + lane % 16, (wave / 4 * kSteps + s) * 4 + lane / 16), acc[j]);
    }
  }
  __syncthreads();
  if (wave >= 4) {
#pragma unroll
    for (int j = 0; j < RT; ++j) half[((wave - 4) * RT + j) * kWave + lane] = acc[j];
  }
  __syncthreads();
  if (wave >= 4) return;
  const u32 o4 = tile * 64 + wave * 16 + lane / 16 * 4;
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    const u32 t = j * 16 + lane % 16;
    if (t >= rows) continue;
    const f32x4 s = acc[j] + half[(wave * RT + j) * kWave + lane];
    float* const to = sums + part * part_step + (size_t)t * outer + o4;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (o4 + e < outer) to[e] = s[e];
  }
}

template <class T, int RT, int ZT>
__global__ __launch_bounds__(kFewWaves * kWave) void k_few(const T* x, size_t ldx, const T* w, size_t ldw, const T* f, size_t f_ld,
                                                           const float* scale, const int* index, u32 rows, u32 inner, u32 outer, u32 rank,
                                                           u32 parties, Drop d, u32 parts, u32 z_parts, u32 z_ld, float* sums, float* z,
                                                           u32* status, u32 first_block) {
  __shared__ __align__(16) char lds[RT * 16 * kRowBytes];  // tiles of x, then halves of sums; or parts of z
  constexpr u32 kGroup = RT * 16;
  const u32 tiles = (outer + 63) / 64 * parts, products = (rows + kGroup - 1) / kGroup * tiles;
  const u32 block = first_block + blockIdx.x;
  if (block < products) {
    const u32 t0 = block / tiles * kGroup, at = block % tiles, count = rows - t0 < kGroup ? rows - t0 : kGroup;
    const T* const x0 = x + (size_t)t0 * ldx;
    float* const to = sums + (size_t)t0 * outer;
    const size_t step = (size_t)rows * outer;
    if (inner < 8) few_product<T, RT, true>(x0, ldx, w, ldw, count, inner, outer, at / parts, at % parts, parts, step, to, (T*)lds, (f32x4*)lds);
    else few_product<T, RT, false>(x0, ldx, w, ldw, count, inner, outer, at / parts, at % parts, parts, step, to, (T*)lds, (f32x4*)lds);
    return;
  }
  float(*const lz)[ZT * 16] = (float(*)[ZT * 16])lds;
  constexpr int kAhead = ZT == 1 ? 4 : 2;
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const u32 t = (block - products) / z_parts, part = (block - products) % z_parts;
  const int raw = index[t], a = party_of(index, t, parties);
  if (status && part == 0 && threadIdx.x == 0 && raw != a && raw != -1) atomicOr(status, HAFLO_ST_RANGE);
  float* const to = z + ((size_t)part * rows + t) * z_ld;
  if (a < 0) {
    if (threadIdx.x < z_ld) to[threadIdx.x] = 0.0f;
    return;
  }
  const T* const fa = f + (size_t)a * rank * f_ld;
  const u32 steps = (inner + 31) / 32, first = (u32)((u64)steps * part / z_parts), end = (u32)((u64)steps * (part + 1) / z_parts);
  size_t f_at[ZT];
#pragma unroll
  for (int i = 0; i < ZT; ++i) f_at[i] = (size_t)lowest(i * 16 + lane % 16, rank) * f_ld;
  f32x4 acc[ZT];
#pragma unroll
  for (int i = 0; i < ZT; ++i) acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (u32 s0 = first + wave * kAhead; s0 < end; s0 += kFewWaves * kAhead) {
    Vec8<T> xv[kAhead], fv[kAhead][ZT];
    u32 k[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) k[u] = s0 + u < end ? (s0 + u) * 32 + lane / 16 * 8 : inner;
    if (inner >= 8) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        xv[u] = load_row(x + (size_t)t * ldx, k[u], inner);
#pragma unroll
        for (int i = 0; i < ZT; ++i) fv[u][i] = load_row(fa + f_at[i], k[u], inner);
      }
    } else {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        xv[u] = load_short(x + (size_t)t * ldx, k[u], inner);
#pragma unroll
        for (int i = 0; i < ZT; ++i) fv[u][i] = load_short(fa + f_at[i], k[u], inner);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      settle(xv[u], k[u], inner);
#pragma unroll
      for (int i = 0; i < ZT; ++i) settle(fv[u][i], k[u], inner);
      if (d.threshold) apply_drop(xv[u], d, t, (s0 + u) * 32 + lane / 16 * 8);
#pragma unroll
      for (int i = 0; i < ZT; ++i) acc[i] = mma32(fv[u][i], xv[u], acc[i]);
    }
  }
  // all sixteen rows of the second operand were the same one: its first column has the sums
  if (lane % 16 == 0) {
#pragma unroll
    for (int i = 0; i < ZT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) lz[wave][i * 16 + lane / 16 * 4 + e] = acc[i][e];
  }
  __syncthreads();
  const u32 r = threadIdx.x;
  if (r >= z_ld) return;
  float s = 0.0f;
#pragma unroll
  for (int v = 0; v < kFewWaves; ++v) s += r < ZT * 16 ? lz[v][r] : 0.0f;
  to[r] = r < rank ? s * scale[a] * (d.threshold ? d.scale : 1.0f) : 0.0f;
}

// A block takes 256 outputs of a row, a lane one: the reading of the parts bounds it (64 rows of 4096, 8 parts: 6 us). Its z is written to `z_out` (z_ld places) or `h` (rank) by the first of the row.
template <class T, bool DROP>
__global__ __launch_bounds__(kThreads) void k_few_join(const float* sums, const float* z, const T* f, u32 f_ld, const int* index, u32 rows, u32 outer,
                                                       u32 parties, u32 rank, Drop d, u32 parts, u32 z_parts, u32 z_ld, T* y, size_t ldy,
                                                       float* z_out, float* h, u32 first_block) {
  __shared__ float zl[HAFLO_ADAPTER_MAX_RANK];
  const u32 block = first_block + blockIdx.x, blocks = (outer + kThreads - 1) / kThreads, t = block / blocks, o = block % blocks * kThreads + threadIdx.x;
  float m = 0.0f;
  if (o < outer && y)
#pragma unroll 4
    for (u32 p = 0; p < parts; ++p) m += sums[((size_t)p * rows + t) * outer + o];
  if (threadIdx.x < z_ld) {
    float s = 0.0f;
    for (u32 p = 0; p < z_parts; ++p) s += z[((size_t)p * rows + t) * z_ld + threadIdx.x];
    zl[threadIdx.x] = s;
    if (block % blocks == 0) {
      if (z_out) z_out[(size_t)t * z_ld + threadIdx.x] = s;
      if (h && threadIdx.x < rank) h[(size_t)t * rank + threadIdx.x] = s;
    }
  }
  __syncthreads();
  if (o >= outer || !y) return;
  const int a = party_of(index, t, parties);
  if (a >= 0) {
    const T* const fr = f + ((size_t)a * outer + o) * f_ld;
    float low = 0.0f;
    for (u32 r0 = 0; r0 < rank; r0 += 8) {
      const Vec8<T> v = r0 + 8 <= rank ? load_wide(fr + r0) : load_some(fr + r0, (int)(rank - r0));
#pragma unroll
      for (u32 r = 0; r < 8; ++r)
        if (r0 + r < rank) low += zl[r0 + r] * (float)v.get(r);
    }
    if (DROP) {
      const u32x4 draws = philox(d, o >> 3, t);
      const u32 word = o & 4 ? (o & 2 ? draws[3] : draws[2]) : (o & 2 ? draws[1] : draws[0]);
      low = (word >> (16 * (o & 1)) & 0xFFFFu) >= d.threshold ? low * d.scale : 0.0f;
    }
    m += low;
  }
  y[(size_t)t * ldy + o] = (T)m;
}

// rows of one chunk of a party's list: as many as leave some 512 blocks of k_grad
u32 chunk_rows(size_t rows, size_t cols, size_t rank) {
  const size_t blocks = rows * ceil_div(cols, 128) * ceil_div(rank, 64) / 512;
  u32 n = 16;
  while (n < 256 && 2 * n <= blocks) n *= 2;
  return n;
}
// What a call lays out before its products: matrices copied to rows of `out_ld` elements with zeros behind what they hold, or
// transposed to such rows (`count` of them one behind the other), and the rows grouped by adapter by the first block.
// Memory bounds it: W of 4096 x 4096 in bfloat16 transposed in 26 us, 2.6 TB/s. One launch, as a short one costs 3 us and more.
constexpr int kPrepareThreads = 1024;
constexpr u32 kGroupCounts = 16384;
__host__ __device__ inline u32 group_waves(u32 parties) { return parties < 1024 ? 16 : 3; }  // whose counts fit LDS
template <class T>
struct Layout {
  const T* in;
  T* out;
  size_t ld, in_step, out_step;
  u32 rows, cols, out_ld, first, transposed;  // `first`: of its blocks
};
struct Group {
  const int* index;
  u32 rows, parties, chunk_rows;
  u32 *begin, *chunk_begin, *chunk, *order, *status;
};
constexpr int kLayouts = 5;
template <class T>
struct Prepare {
  Layout<T> job[kLayouts];
  int jobs;
  bool grouped;
  Group group;
};

// `order` holds the rows of party 0 in ascending order, then those of party 1, ..., at last those without; begin[p] is where
// p's start, begin[parties] where the last begin; chunk_begin[p] the first of p's chunks of chunk_rows rows; chunk[c] = p.
// The block's wavefronts take a range of rows each, count them, and list them from where their counts say. One compute unit's
// vector instructions bound it (16384 rows: 13 us party by party, 18 when every 64 rows were taken as mixed; 3001 mixed rows:
// 11); more blocks would cost another launch.
__device__ void group_rows(const Group& g, u32* counts) {
  constexpr int kAhead = 8;
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id(), waves = group_waves(g.parties);
  const u32 rows = g.rows, parties = g.parties;
  const int* const index = g.index;
  const u32 bins = parties + 1, bits = 32 - (u32)__builtin_clz(parties);
  const u32 per = ((rows + waves - 1) / waves + kWave - 1) / kWave * kWave;
  const u32 first = wave < waves && (u64)wave * per < rows ? wave * per : rows, end = rows - first < per ? rows : first + per;
  for (u32 i = threadIdx.x; i < waves * bins; i += kPrepareThreads) counts[i] = 0;
  __syncthreads();
  int raw[kAhead];
  u32 at[kAhead], first_of[kAhead], below[kAhead];
  u32 held = ~0u;  // where the rows that raw holds begin
  for (int pass = 0; pass < 2; ++pass) {
    for (u32 base = first; base < end; base += kAhead * kWave) {
      if (base != held) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) raw[i] = index[lowest(base + i * kWave + lane, end)];
        held = base;
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const u32 t = base + i * kWave + lane;
        const u32 a = (u32)raw[i] < parties ? (u32)raw[i] : parties;
        if (pass == 0 && t < end && a == parties && raw[i] != -1 && g.status) atomicOr(g.status, HAFLO_ST_RANGE);
        u64 same = __builtin_amdgcn_ballot_w64(t < end);  // the lanes whose row has this one's party, bit by bit
        const u32 one = (u32)__builtin_amdgcn_readfirstlane((int)a);
        const bool mixed = __builtin_amdgcn_ballot_w64(t < end && a != one) != 0;  // (rows often come party by party)
        for (u32 b = 0; mixed && b < bits; ++b) {
          const u64 ones = __builtin_amdgcn_ballot_w64(a >> b & 1);
          same &= a >> b & 1 ? ones : ~ones;
        }
        // the first of them counts them; a wavefront's additions take place in their order, none waits for the one before
        at[i] = 0;
        first_of[i] = same ? (u32)__builtin_ctzll(same) : lane;
        below[i] = (u32)__builtin_popcountll(same & ((1ull << lane) - 1));
        if (t < end && first_of[i] == lane) at[i] = atomicAdd(&counts[wave * bins + a], (u32)__builtin_popcountll(same));
      }
      if (pass == 0) continue;
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const u32 t = base + i * kWave + lane, from = lane_read(at[i], (int)first_of[i]);
        if (t < end) g.order[from + below[i]] = t;
      }
    }
    __syncthreads();
    if (pass == 0 && wave == 0) {  // counts to places, 64 parties at a time
      u32 at = 0, chunks = 0;
      for (u32 p0 = 0; p0 < bins; p0 += kWave) {
        const u32 p = p0 + lane;
        u32 n = 0;
        for (u32 w = 0; w < waves; ++w) n += p < bins ? counts[w * bins + p] : 0;
        u32 to = n, c = p < parties ? (n + g.chunk_rows - 1) / g.chunk_rows : 0, c_to = c;
#pragma unroll
        for (int s = 1; s < kWave; s <<= 1) {  // sums up to each lane
          const u32 below = lane_read(to, (int)lane - s), c_below = lane_read(c_to, (int)lane - s);
          if ((int)lane >= s) {
            to += below;
            c_to += c_below;
          }
        }
        u32 place = at + to - n;
        if (p < bins) {
          g.begin[p] = place;
          g.chunk_begin[p] = chunks + c_to - c;
          for (u32 w = 0; w < waves; ++w) {
            const u32 m = counts[w * bins + p];
            counts[w * bins + p] = place;
            place += m;
          }
        }
        const u32 c_from = chunks + c_to - c;
        u64 many = __builtin_amdgcn_ballot_w64(c > 4);
        if (c <= 4)
          for (u32 i = 0; i < c; ++i) g.chunk[c_from + i] = p;
        for (; many; many &= many - 1) {  // all lanes for a party of many
          const int of = __builtin_ctzll(many);
          const u32 base = (u32)__builtin_amdgcn_readlane((int)c_from, of), n_of = (u32)__builtin_amdgcn_readlane((int)c, of);
          for (u32 i = lane; i < n_of; i += kWave) g.chunk[base + i] = p0 + of;
        }
        at += (u32)__builtin_amdgcn_readlane((int)to, kWave - 1);
        chunks += (u32)__builtin_amdgcn_readlane((int)c_to, kWave - 1);
      }
    }
    __syncthreads();
  }
}

template <class T>
__global__ __launch_bounds__(kPrepareThreads) void k_prepare(Prepare<T> p, u32 first_block) {
  __shared__ __align__(16) u32 lds[kGroupCounts];
  u32 block = first_block + blockIdx.x;
  if (p.grouped) {
    if (block == 0) {
      group_rows(p.group, lds);
      return;
    }
    --block;
  }
  int j = 0;
  while (j + 1 < p.jobs && block >= p.job[j + 1].first) ++j;
  const Layout<T> job = p.job[j];
  block -= job.first;
  if (!job.transposed) {
    const u32 groups = job.out_ld / 8;
    const u64 at = (u64)block * kPrepareThreads + threadIdx.x;
    if (at >= (u64)job.rows * groups) return;
    const u32 r = (u32)(at / groups), c = (u32)(at - (u64)r * groups) * 8;
    const T* const row = job.in + (size_t)r * job.ld;
    Vec8<T> v = job.cols < 8 ? load_short(row, c, job.cols) : load_row(row, c, job.cols);
    settle(v, c, job.cols);
    store_wide(job.out + (size_t)r * job.out_ld + c, v);
    return;
  }
  T(*const tile)[66] = (T(*)[66])lds;
  const u32 tiles_c = (job.cols + 63) / 64, tiles = tiles_c * ((job.out_ld + 63) / 64);
  const u32 which = block / tiles, at = block % tiles, r0 = at / tiles_c * 64, c0 = at % tiles_c * 64;
  const T* const in = job.in + which * job.in_step;
  T* const out = job.out + which * job.out_step;
  constexpr u32 kLoads = 64 * 64 / kPrepareThreads;
  T v[kLoads];
#pragma unroll
  for (u32 n = 0; n < kLoads; ++n) {
    const u32 i = n * kPrepareThreads + threadIdx.x;
    v[n] = in[(size_t)lowest(r0 + i / 64, job.rows) * job.ld + lowest(c0 + i % 64, job.cols)];
  }
#pragma unroll
  for (u32 n = 0; n < kLoads; ++n) {
    const u32 i = n * kPrepareThreads + threadIdx.x;
    tile[i / 64][i % 64] = r0 + i / 64 < job.rows ? v[n] : (T)0.0f;
  }
  __syncthreads();
  for (u32 i = threadIdx.x; i < 64 * 64; i += kPrepareThreads) {
    const u32 c = c0 + i / 64, r = r0 + i % 64;
    if (r < job.out_ld && c < job.cols) out[(size_t)c * job.out_ld + r] = tile[i % 64][i / 64];
  }
}

// out[chunk][r][col] = sum over the chunk's rows t of z[t, r] drop(m[t, col]) on matrix instructions in 32 bits, whose
// operands are one element a lane: lane l holds eight columns from 8 (l % 16) on of row l / 16 out of four, and element j of
// all lanes is one operand, for the columns 8 c + j. A block takes 128 columns and RT sixteens of z, its wavefronts every
// fourth four rows each. The next rows are on their way while the present ones are multiplied.
// Both gradients are formed by one launch. 8192 rows of 4096 and 4096 columns, rank 16, bfloat16: 56 us, 38 TFLOP/s and 2.4 TB/s, so
// bound by neither alone but by a row's way from memory to its sixteen products; four rows ahead in place of two gain nothing.
template <class T>
struct GradOf {
  const T* m;
  size_t ld;
  const float* z;
  float *out, *grad;
  size_t r_step, col_step;  // of the gradient
  u32 cols, z_ld;
  Drop d;
};
template <class T, int RT>
__global__ __launch_bounds__(kThreads) void k_grad(GradOf<T> a, GradOf<T> b, u32 rank, u32 parties, const u32* __restrict__ begin,
                                                   const u32* __restrict__ chunk_begin, const u32* __restrict__ chunk,
                                                   const u32* __restrict__ list, u32 chunk_rows, u32 first_block) {
  constexpr int kAhead = 2, kWaves = kThreads / kWave;
  __shared__ f32x4 sum[kWaves - 1][RT][8][kWave];
  const u32 wave = (u32)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = lane_id();
  const u32 tiles_r = (rank + RT * 16 - 1) / (RT * 16), of_a = (a.cols + 127) / 128 * tiles_r, of_b = (b.cols + 127) / 128 * tiles_r;
  const u32 block = first_block + blockIdx.x, c = block / (of_a + of_b), both = block % (of_a + of_b), at = both < of_a ? both : both - of_a;
  if (c >= chunk_begin[parties]) return;
  const GradOf<T> g = both < of_a ? a : b;
  const T* __restrict__ const m = g.m;
  const float* __restrict__ const z = g.z;
  float* __restrict__ const out = g.out;
  const size_t ld = g.ld;
  const u32 cols = g.cols, z_ld = g.z_ld;
  const Drop d = g.d;
  const u32 col = at / tiles_r * 128 + lane % 16 * 8, r0 = at % tiles_r * (RT * 16), r = r0 + lane % 16;
  const u32 p = chunk[c], first = begin[p] + (c - chunk_begin[p]) * chunk_rows;
  const u32 end = first + chunk_rows < begin[p + 1] ? first + chunk_rows : begin[p + 1];
  const u32 mine = first + wave * 4 + lane / 16, turns = (end - first + kWaves * 4 - 1) / (kWaves * 4);
  f32x4 acc[RT][8];
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  struct Rows4 {
    Vec8<T> v;
    float z[RT];
    u32 t;
  } ahead[kAhead];
  u32 listed[kAhead];  // the rows after those
  const auto look = [&](u32 n) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const u32 i = mine + (n + u) * (kWaves * 4);
      listed[u] = list[lowest(i, end)];
    }
  };
  const auto fetch = [&](u32 n) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) ahead[u].t = listed[u];
    look(n + kAhead);
    if (cols >= 8) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) ahead[u].v = load_row(m + (size_t)ahead[u].t * ld, col, cols);
    } else {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) ahead[u].v = load_short(m + (size_t)ahead[u].t * ld, col, cols);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
#pragma unroll
      for (int i = 0; i < RT; ++i) ahead[u].z[i] = z[(size_t)ahead[u].t * z_ld + lowest(r + i * 16, rank)];
    }
  };
  look(0);
  fetch(0);
  for (u32 n = 0; n < turns; n += kAhead) {
    Rows4 now[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) now[u] = ahead[u];
    if (n + kAhead < turns) fetch(n + kAhead);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      settle(now[u].v, col, cols);
      if (d.threshold) apply_drop(now[u].v, d, now[u].t, col);
      if (mine + (n + u) * (kWaves * 4) >= end) {  // the last row again
        now[u].v = Vec8<T>{};
#pragma unroll
        for (int i = 0; i < RT; ++i) now[u].z[i] = 0.0f;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float f = (float)now[u].v.get(j);
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(now[u].z[i], f, acc[i][j], 0, 0, 0);
      }
    }
  }
  if (wave != 0) {
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[wave - 1][i][j][lane] = acc[i][j];
  }
  __syncthreads();
  if (wave != 0) return;
  const float by = d.threshold ? d.scale : 1.0f;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < kWaves - 1; ++w) acc[i][j] += sum[w][i][j][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const u32 rr = r0 + i * 16 + lane / 16 * 4 + e;
      if (rr >= rank || col >= cols) continue;
      float* const to = out + ((size_t)c * rank + rr) * cols + col;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = acc[i][j][e] * by;
      if (col + 8 <= cols) {
        __builtin_memcpy(to, v, sizeof(v));
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col + j < cols) to[j] = v[j];
      }
    }
  }
}

// grad[p] = sum of the party's chunks, in their order. A lane takes an element; the chunks' reading bounds it (8192 rows, 8 parties,
// 16 x 8192 weights: 9 us).
template <class T>
__global__ __launch_bounds__(kThreads) void k_grad_join(GradOf<T> a, GradOf<T> b, const u32* __restrict__ chunk_begin, u32 rank,
                                                     u32 first_block) {
  const size_t n_a = (size_t)rank * a.cols, n_b = (size_t)rank * b.cols;
  const u32 of_a = (u32)((n_a + kThreads - 1) / kThreads), of_b = (u32)((n_b + kThreads - 1) / kThreads);
  const u32 block = first_block + blockIdx.x, p = block / (of_a + of_b), both = block % (of_a + of_b);
  const GradOf<T> g = both < of_a ? a : b;
  const size_t n = both < of_a ? n_a : n_b, i = (size_t)(both < of_a ? both : both - of_a) * kThreads + threadIdx.x;
  if (i >= n) return;
  const u32 end = chunk_begin[p + 1];
  float s = 0.0f;
#pragma unroll 8
  for (u32 c = chunk_begin[p]; c < end; ++c) s += g.out[c * n + i];
  g.grad[p * n + i / g.cols * g.r_step + i % g.cols * g.col_step] = s;
}

struct Sizes {
  size_t rows, inner, outer, parties, rank;
};
constexpr size_t kMostElements = (size_t)1 << 56;  // of a matrix, so that sums of sizes stay within 64 bits
bool adapter_sizes(int type, const Sizes& s) {
  return valid_type(type) && s.rows <= kMostCount && s.inner >= 1 && s.inner <= kMostCount - 512 && s.outer >= 1 &&
         s.outer <= kMostCount - 512 && s.parties >= 1 && s.parties <= HAFLO_ADAPTER_MAX_PARTIES && s.rank >= 1 &&
         s.rank <= HAFLO_ADAPTER_MAX_RANK && s.rows * s.inner <= kMostElements && s.rows * s.outer <= kMostElements &&
         s.inner * s.outer <= kMostElements;
}
// Whether k_few takes a product: up to 256 rows, where k_project's tiles would leave most of the chip idle; float32, whose matrix
// instructions bound it sooner, up to 2^31 products of elements. Forward, us by k_few and by k_project: bfloat16 4096 to 4096
// 128 rows 27 and 46, 256 rows 41 and 46, 4096 to 256 128 rows 17 and 33; float32 4096 to 4096 128 rows 61 and 89, 192 rows 98 and
// 92, 4096 to 256 256 rows 25 and 87.
bool few(int type, const Sizes& s) {
  return s.rows <= 256 && (type != HAFLO_F32 || s.rows * s.inner <= ((size_t)1 << 31) / s.outer);
}
// parts of k_shrink's reduction: enough blocks to fill the chip, at least 512 columns each
u32 shrink_parts(bool by_row, size_t rows, size_t k) {
  if (rows == 0) return 1;
  const size_t tiles = by_row ? rows : ceil_div(rows, 16), want = tiles < 512 ? ceil_div(512, tiles) : 1, most = ceil_div(k, 512);
  return (u32)(want < most ? want : most);
}
// parts of k_few's reduction: two blocks of it to a compute unit, at least 1024 bytes of a row each
u32 few_parts(int type, size_t rows, size_t k, size_t n) {
  if (rows == 0) return 1;
  const size_t want = ceil_div(512, ceil_div(rows, 64) * ceil_div(n, 64)), most = ceil_div(k * type_size(type), kRowBytes);
  return (u32)(want < most ? want : most);
}
size_t padded(int type, size_t k) { return ceil_div(k, 128 / type_size(type)) * (128 / type_size(type)); }
size_t whole_ranks(size_t rank) { return ceil_div(rank, kRanks) * kRanks; }
u32 grad_rows(const Sizes& s) { return chunk_rows(s.rows, s.inner + s.outer, s.rank); }
struct Plan {
  size_t z_parts, few_sums, z, x, w, low, f, begin, chunk_begin, chunk, order, sums_a, sums_b, total;
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
  const size_t e = type_size(type), ranks = whole_ranks(s.rank);
  const size_t k = backward ? s.outer : s.inner, n = backward ? s.inner : s.outer, kp = padded(type, k);  // the product's sizes
  p.z_parts = take(shrink_parts(few(type, s), s.rows, k) * s.rows * ranks * 4);
  if (few(type, s)) p.few_sums = take(few_parts(type, s.rows, k, n) * s.rows * n * 4);
  p.z = take(s.rows * ranks * 4);
  p.x = take(s.rows * kp * e);
  p.w = take(n * kp * e);
  if (backward) p.low = take(s.parties * s.rank * kp * e);
  p.f = take(s.parties * n * ranks * e);
  p.chunks = s.rows / grad_rows(s) + s.parties;
  p.begin = take((s.parties + 1) * 4);
  p.chunk_begin = take((s.parties + 1) * 4);
  p.chunk = take(p.chunks * 4);
  p.order = take(s.rows * 4);
  if (backward) {
    p.sums_a = take(p.chunks * s.rank * s.inner * 4);
    p.sums_b = take(p.chunks * s.rank * s.outer * 4);
  }
  p.total = b;
  return p;
}

template <class T>
struct Rows {
  const T* p;
  size_t ld;
};
// Collects what is to be laid out, and launches it.
template <class T>
struct Layouts {
  Prepare<T> p = {};
  size_t blocks = 0;

  Rows<T> add(const void* in, char* out, size_t ld, size_t in_step, size_t out_step, size_t rows, size_t cols, size_t out_ld, bool transposed, size_t need) {
    p.job[p.jobs++] = {(const T*)in, (T*)out, ld, in_step, out_step, (u32)rows, (u32)cols, (u32)out_ld, (u32)blocks, transposed ? 1u : 0u};
    blocks += need;
    return {(const T*)out, out_ld};
  }
  // A matrix with rows at 16-byte boundaries and of a multiple of `step` elements, zeros behind what they hold, as k_project
  // needs it: itself, or its copy at `room`.
  Rows<T> wide(const void* m, size_t ld, size_t rows, size_t cols, size_t step, char* room) {
    if ((uintptr_t)m % 16 == 0 && ld * sizeof(T) % 16 == 0 && cols % step == 0) return {(const T*)m, ld};
    const size_t to = ceil_div(cols, step) * step;
    return add(m, room, ld, 0, 0, rows, cols, to, false, ceil_div(rows * (to / 8), kPrepareThreads));
  }
  Rows<T> transposed(const void* in, size_t ld, size_t in_step, size_t rows, size_t cols, size_t count, char* room, size_t out_ld) {
    return add(in, room, ld, in_step, cols * out_ld, rows, cols, out_ld, true, ceil_div(out_ld, 64) * ceil_div(cols, 64) * count);
  }
  void launch(hipStream_t st) {
    blocks += p.grouped ? 1 : 0;
    in_turns(blocks, kPrepareThreads, [&](u32 first, dim3 grid, dim3 block) { hipLaunchKernelGGL((k_prepare<T>), grid, block, 0, st, p, first); });
  }
};
template <class T>
void add_group(Prepare<T>& to, const Sizes& s, const int* index, char* ws, const Plan& p, u32* status) {
  to.grouped = true;
  to.group = {index, (u32)s.rows, (u32)s.parties, grad_rows(s), (u32*)(ws + p.begin), (u32*)(ws + p.chunk_begin), (u32*)(ws + p.chunk),
          (u32*)(ws + p.order), status};
}

// What both directions do: z from x and the low-rank rows `low`, then x against `w` with `f` (outer x rank of every party).
template <class T>
struct Product {
  Rows<T> x, w, low, f;
  const float* scale;
  const int* index;
  Sizes s;  // `inner` is the reduction's length, `outer` the result's
  Drop before, after;
  char* ws;
  Plan plan;
  u32* status;
  hipStream_t st;

  u32 ranks() const { return (u32)whole_ranks(s.rank); }
  size_t padded_inner() const { return ceil_div(s.inner, step_elems<T>()) * step_elems<T>(); }
  const u32* order() const { return (const u32*)(ws + plan.order); }
  float* z_parts() const { return (float*)(ws + plan.z_parts); }
  float* z() const { return (float*)(ws + plan.z); }

  // z, dense as `h` too unless that is null
  void shrink(float* h) const {
    const u32 parts = shrink_parts(false, s.rows, s.inner);
    const size_t blocks = ceil_div(s.rows, 16) * parts;
    float* const to = parts > 1 ? z_parts() : z();
    float* const h_now = parts > 1 ? nullptr : h;
#define HAFLO_LOCAL_RUN(RT)                                                                                                             \
  in_turns(blocks, kShrinkWaves * kWave, [&](u32 first, dim3 grid, dim3 block) {                                                        \
    hipLaunchKernelGGL((k_shrink<T, RT>), grid, block, 0, st, x.p, x.ld, low.p, low.ld, scale, index, order(), (u32)s.rows, (u32)s.inner, \
                       (u32)s.rank, (u32)s.parties, before, parts, ranks(), to, h_now, status, first);                                  \
  })
    if (s.rank <= 16) HAFLO_LOCAL_RUN(1);
    else if (s.rank <= 64) HAFLO_LOCAL_RUN(4);
    else HAFLO_LOCAL_RUN(8);
#undef HAFLO_LOCAL_RUN
    const size_t count = s.rows * ranks();
    if (parts > 1)
      hipLaunchKernelGGL(k_join, dim3((unsigned)ceil_div(count, kThreads)), dim3(kThreads), 0, st, (const float*)z_parts(), parts, count, ranks(),
                         (u32)s.rank, z(), h);
  }

  // Few rows: y, unless it is null, and z; dense as `h` too unless that is null.
  void few_rows(float* h, T* y, size_t ldy) const {
    const u32 zp = shrink_parts(true, s.rows, s.inner), parts = few_parts(sizeof(T) == 4 ? HAFLO_F32 : HAFLO_F16, s.rows, s.inner, s.outer);
    const size_t blocks = (y ? ceil_div(s.rows, 64) * ceil_div(s.outer, 64) * parts : 0) + s.rows * zp;
    float* const sums = (float*)(ws + plan.few_sums);
#define HAFLO_LOCAL_RUN(RT, ZT)                                                                                                              \
  in_turns(blocks, kFewWaves * kWave, [&](u32 first, dim3 grid, dim3 block) {                                                                \
    hipLaunchKernelGGL((k_few<T, RT, ZT>), grid, block, 0, st, x.p, x.ld, w.p, w.ld, low.p, low.ld, scale, index, (u32)s.rows, (u32)s.inner, \
                       (u32)(y ? s.outer : 0), (u32)s.rank, (u32)s.parties, before, parts, zp, ranks(), sums, z_parts(), status, first);     \
  })
#define HAFLO_LOCAL_RANK(RT)                       \
  do {                                             \
    if (s.rank <= 16) HAFLO_LOCAL_RUN(RT, 1);      \
    else if (s.rank <= 64) HAFLO_LOCAL_RUN(RT, 4); \
    else HAFLO_LOCAL_RUN(RT, 8);                   \
  } while (0)
    if (s.rows <= 16) HAFLO_LOCAL_RANK(1);
    else if (s.rows <= 32) HAFLO_LOCAL_RANK(2);
    else HAFLO_LOCAL_RANK(4);
#undef HAFLO_LOCAL_RANK
#undef HAFLO_LOCAL_RUN
#define HAFLO_LOCAL_RUN(DROP)                                                                                                               \
  in_turns(s.rows * ceil_div(s.outer, kThreads), kThreads, [&](u32 first, dim3 grid, dim3 block) {                                          \
    hipLaunchKernelGGL((k_few_join<T, DROP>), grid, block, 0, st, (const float*)sums, (const float*)z_parts(), f.p, (u32)f.ld, index,       \
                       (u32)s.rows, (u32)s.outer, (u32)s.parties, (u32)s.rank, after, parts, zp, ranks(), y, ldy, z(), h, first);           \
  })
    if (after.threshold) HAFLO_LOCAL_RUN(true);
    else HAFLO_LOCAL_RUN(false);
#undef HAFLO_LOCAL_RUN
  }

  // The largest tiles that give every compute unit one: W and x are read once for a tile's side. Calls, us: bfloat16 8192 x 4096 to 4096 by
  // 256 x 256 238, by 128 x 128 301; 4096 x 1024 to 4096 55 and 69; 4096 x 4096 to 2048 by 128 x 128 97, by 64 x 64 123; 4096 x 512 to 2048
  // 33 and 35; too few tiles, float16 3001 x 1001 to 515, 38 and 32. float32 is bound by its matrix instructions and takes the small tiles,
  // which leave the fewest of them idle: 8192 x 4096 to 4096 by 256 x 256 2131, by 128 x 128 1970, by 64 x 64 1955; 4096 x 1024 to 1024 by
  // 128 x 128 96, by 64 x 64 90; 16384 x 1024 to 1024 310, 308 and 314.
  void project(T* y, size_t ldy) const {
    const size_t x_bytes = ((s.rows - 1) * x.ld + padded_inner()) * sizeof(T), w_bytes = ((s.outer - 1) * w.ld + padded_inner()) * sizeof(T);
    const bool far = x_bytes > 0xFFFFFFFFu || w_bytes > 0xFFFFFFFFu;
#define HAFLO_LOCAL_RUN(TM, TN, WM, WN, DROP, FAR)                                                                                        \
  in_turns(ceil_div(s.rows, TM) * ceil_div(s.outer, TN), WM * WN * kWave, [&](u32 first, dim3 grid, dim3 block) {                         \
    hipLaunchKernelGGL((k_project<T, TM, TN, WM, WN, DROP, FAR>), grid, block, 0, st, x.p, x.ld, w.p, w.ld, f.p, (const float*)z(), index, \
                       order(), (const u32*)(ws + plan.begin), (u32)s.rows, (u32)padded_inner(), (u32)s.outer, (u32)s.parties, ranks(),   \
                       after, y, ldy, (u32)x_bytes, (u32)w_bytes, first);                                                                 \
  })
#define HAFLO_LOCAL_TILE(DROP)                                                                                    \
  do {                                                                                                            \
    if (far) HAFLO_LOCAL_RUN(256, 256, 2, 4, DROP, true);                                                         \
    else if constexpr (sizeof(T) == 4) HAFLO_LOCAL_RUN(64, 64, 2, 2, DROP, false);                                \
    else if (ceil_div(s.rows, 256) * ceil_div(s.outer, 256) >= 256) HAFLO_LOCAL_RUN(256, 256, 2, 4, DROP, false); \
    else if (ceil_div(s.rows, 128) * ceil_div(s.outer, 128) >= 256) HAFLO_LOCAL_RUN(128, 128, 2, 2, DROP, false); \
    else HAFLO_LOCAL_RUN(64, 64, 2, 2, DROP, false);                                                              \
  } while (0)
    if (after.threshold) HAFLO_LOCAL_TILE(true);
    else HAFLO_LOCAL_TILE(false);
#undef HAFLO_LOCAL_TILE
#undef HAFLO_LOCAL_RUN
  }
};

template <class T>
void grads(const GradOf<T>& a, const GradOf<T>& b, const Sizes& s, const Plan& p, char* ws, hipStream_t st) {
  const u32* chunk_begin = (const u32*)(ws + p.chunk_begin);
  const size_t columns = ceil_div(a.cols, 128) + ceil_div(b.cols, 128);
#define HAFLO_LOCAL_RUN(RT)                                                                                                             \
  in_turns(p.chunks * columns * ceil_div(s.rank, RT * 16), kThreads, [&](u32 first, dim3 grid, dim3 block) {                            \
    hipLaunchKernelGGL((k_grad<T, RT>), grid, block, 0, st, a, b, (u32)s.rank, (u32)s.parties, (const u32*)(ws + p.begin), chunk_begin, \
                       (const u32*)(ws + p.chunk), (const u32*)(ws + p.order), grad_rows(s), first);                                    \
  })
  if (s.rank <= 16) HAFLO_LOCAL_RUN(1);
  else if (s.rank <= 32) HAFLO_LOCAL_RUN(2);
  else HAFLO_LOCAL_RUN(4);
#undef HAFLO_LOCAL_RUN
  const size_t need = ceil_div(s.rank * a.cols, kThreads) + ceil_div(s.rank * b.cols, kThreads);
  in_turns(s.parties * need, kThreads, [&](u32 first, dim3 grid, dim3 block) {
    hipLaunchKernelGGL((k_grad_join<T>), grid, block, 0, st, a, b, chunk_begin, (u32)s.rank, first);
  });
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
  if (!enough(d_workspace, workspace_bytes, plan.total)) return HAFLO_EINVAL;
  char* const ws = (char*)d_workspace;
  const hipStream_t st = (hipStream_t)stream;
  const Drop d = make_drop(p, seed, offset);
  Drop none = d;
  none.threshold = 0;
  HAFLO_LOCAL_TYPES(type, {
    const bool many = !few(type, s);
    Layouts<T> lay;
    Product<T> f = {{(const T*)d_x, ldx}, {(const T*)d_w, ldw}, {(const T*)d_a, inner}, {(const T*)d_b, rank}, d_scale, d_index, s, d, none, ws,
                    plan, many ? nullptr : d_status, st};
    if (many) {
      add_group(lay.p, s, d_index, ws, plan, d_status);
      f.x = lay.wide(d_x, ldx, rows, inner, step_elems<T>(), ws + plan.x);
      f.w = lay.wide(d_w, ldw, outer, inner, step_elems<T>(), ws + plan.w);
      f.f = lay.wide(d_b, rank, parties * outer, rank, kRanks, ws + plan.f);
    }
    lay.launch(st);
    if (many) {
      f.shrink(d_h);
      f.project((T*)d_y, ldy);
    } else {
      f.few_rows(d_h, (T*)d_y, ldy);
    }
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
  if (!enough(d_workspace, workspace_bytes, plan.total)) return HAFLO_EINVAL;
  char* const ws = (char*)d_workspace;
  const hipStream_t st = (hipStream_t)stream;
  const Drop d = make_drop(p, seed, offset);
  Drop none = d;
  none.threshold = 0;
  HAFLO_LOCAL_TYPES(type, {
    const bool many = !few(type, s);
    const size_t ranks = whole_ranks(rank);
    const size_t kp = padded(type, outer);
    const Sizes back = {rows, outer, inner, parties, rank};
    Layouts<T> lay;
    add_group(lay.p, s, d_index, ws, plan, d_status);
    Rows<T> dy = {(const T*)d_dy, lddy};
    if (rows) {
      if (many) dy = lay.wide(d_dy, lddy, rows, outer, step_elems<T>(), ws + plan.x);
      // B^T, W^T and A^T: what is reduced along columns here
      Product<T> f = {dy, {}, lay.transposed(d_b, rank, outer * rank, outer, rank, parties, ws + plan.low, kp), {}, d_scale, d_index, back, none, d,
                      ws, plan, nullptr, st};
      if (d_dx) {
        f.w = lay.transposed(d_w, ldw, 0, outer, inner, 1, ws + plan.w, kp);
        f.f = lay.transposed(d_a, inner, rank * inner, rank, inner, parties, ws + plan.f, ranks);
      }
      lay.launch(st);
      if (many) {
        f.shrink(nullptr);
        if (d_dx) f.project((T*)d_dx, lddx);
      } else {
        f.few_rows(nullptr, (T*)d_dx, lddx);
      }
    } else {
      lay.launch(st);
    }
    const GradOf<T> a = {(const T*)d_x, ldx, (const float*)(ws + plan.z), (float*)(ws + plan.sums_a), d_da, inner, 1, (u32)inner, (u32)ranks, d};
    const GradOf<T> b = {dy.p, dy.ld, d_h, (float*)(ws + plan.sums_b), d_db, 1, rank, (u32)outer, (u32)rank, none};
    grads<T>(a, b, s, plan, ws, st);
  });
  return launched();
}

}  // extern "C"
