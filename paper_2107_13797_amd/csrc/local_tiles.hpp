// Tiles of large products: two matrices' rows, 128 bytes of each at a time, from memory into LDS and from there into matrix
// instructions, whose sums stay in registers.
#pragma once
#include "local_common.hpp"

namespace haflo {
namespace local {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// What one lane brings to a product of 16 x 16 tiles, four lanes to a row, and what it holds of its result.
template <class T>
struct Multiplied {
  using Vec = Vec8<T>;
  using Sum = f32x4;
  static constexpr u32 kLane = 8, kProducts = sizeof(T) == 2 ? 1 : 8;  // elements; instructions
};
struct Bytes16 {
  u32x4 w[1];
};
template <>
struct Multiplied<int8_t> {
  using Vec = Bytes16;
  using Sum = i32x4;
  static constexpr u32 kLane = 16, kProducts = 1;
};
__device__ __forceinline__ i32x4 mma32(const Bytes16& a, const Bytes16& b, i32x4 acc) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), acc, 0, 0, 0);
}

template <class T>
constexpr int step_elems() {  // of the reduction in one step: 128 bytes of a row
  return 128 / (int)sizeof(T);
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
__device__ __forceinline__ typename Multiplied<T>::Vec load_frag(const T* tile, u32 row, u32 k) {  // a lane's elements from the k-th of a row
  constexpr u32 kPer = 16 / sizeof(T);
  typename Multiplied<T>::Vec v;
#pragma unroll
  for (u32 i = 0; i < Multiplied<T>::kLane / kPer; ++i)
    v.w[i] = *(const u32x4*)(tile + row * step_elems<T>() + place_of(row, k / kPer + i) * kPer);
  return v;
}

// The operands that a wavefront multiplies next: its outputs by XN sixteens of its rows.
template <class T, int OT, int XN>
struct Frags {
  typename Multiplied<T>::Vec w[OT], x[XN];
};
template <class T, int OT, int XN>
__device__ __forceinline__ void load_w(Frags<T, OT, XN>& f, const T* tile, u32 out0, u32 s) {
#pragma unroll
  for (int i = 0; i < OT; ++i) f.w[i] = load_frag(tile, out0 + i * 16 + lane_id() % 16, (s * 4 + lane_id() / 16) * Multiplied<T>::kLane);
}
template <class T, int OT, int XN>
__device__ __forceinline__ void load_x(Frags<T, OT, XN>& f, const T* tile, u32 row0, u32 s, u32 part) {
#pragma unroll
  for (int j = 0; j < XN; ++j) f.x[j] = load_frag(tile, row0 + (part * XN + j) * 16 + lane_id() % 16, (s * 4 + lane_id() / 16) * Multiplied<T>::kLane);
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
                                             Frags<T, OT, XN>& f, typename Multiplied<T>::Sum (&acc)[OT][RT]) {
  constexpr int KE = step_elems<T>(), kSub = KE / 4 / Multiplied<T>::kLane, kParts = RT / XN, kAll = kSub * kParts;
  constexpr int kAsks = (TM + TN) / 8 / WAVES / 2, kReads = Multiplied<T>::kLane * sizeof(T) / 16, kProducts = XN * OT * Multiplied<T>::kProducts;
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
                                       T* __restrict__ lx0, T* __restrict__ lw0, T* __restrict__ lx1, T* __restrict__ lw1, typename Multiplied<T>::Sum (&acc)[OT][RT]) {
  constexpr int KE = step_elems<T>(), XN = RT < 4 ? RT : 4;
  const u32 inner = steps * KE;
  const auto after = [&](u32 at) { return at + KE < inner ? at + KE : 0; };
  u32 k = after(0);
  ask_tiles<T, TM, TN, WAVES>(0, x, at_x, w, at_w, 0, wave, lx0, lw0);
  ask_tiles<T, TM, TN, WAVES>(1, x, at_x, w, at_w, 0, wave, lx0, lw0);
  ask_tiles<T, TM, TN, WAVES>(0, x, at_x, w, at_w, k, wave, lx1, lw1);
  if (KE / 4 / Multiplied<T>::kLane * (RT / XN) == 1) ask_tiles<T, TM, TN, WAVES>(1, x, at_x, w, at_w, k, wave, lx1, lw1);
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

// One step of a reduction whose tiles lie in LDS four steps deep: this one's tiles are waited for, the ones three steps on asked for
// in place of the last step's.
template <class T, int TM, int TN, int WAVES, class From, int RT, int OT>
__device__ __forceinline__ void deep_step(const From& x, const typename From::At (&at_x)[TM / 8 / WAVES], const From& w,
                                          const typename From::At (&at_w)[TN / 8 / WAVES], u32 k_later, u32 wave, u32 row0, u32 out0, T* cx, T* cw, T* lx,
                                          T* lw, typename Multiplied<T>::Sum (&acc)[OT][RT]) {
  constexpr int kSub = step_elems<T>() / 4 / Multiplied<T>::kLane;
  wait_for_tiles<2 * (TM + TN) / 8 / WAVES>();
  ask_tiles<T, TM, TN, WAVES>(0, x, at_x, w, at_w, k_later, wave, lx, lw);
  ask_tiles<T, TM, TN, WAVES>(1, x, at_x, w, at_w, k_later, wave, lx, lw);
  Frags<T, OT, RT> f[kSub];
#pragma unroll
  for (int s = 0; s < kSub; ++s) {
    load_x(f[s], cx, row0, s, 0);
    load_w(f[s], cw, out0, s);
  }
#pragma unroll
  for (int s = 0; s < kSub; ++s)
#pragma unroll
    for (int j = 0; j < RT; ++j)
#pragma unroll
      for (int i = 0; i < OT; ++i) acc[i][j] = mma32(f[s].w[i], f[s].x[j], acc[i][j]);
}
// The whole reduction of a small tile, of which few are on a compute unit: what bounds it is how long a load takes, so that three
// steps' are on their way. The eight tiles in LDS are told apart here, as in `reduce`.
template <class T, int TM, int TN, int WAVES, class From, int RT, int OT>
__device__ __forceinline__ void reduce_deep(const From& x, const typename From::At (&at_x)[TM / 8 / WAVES], const From& w,
                                            const typename From::At (&at_w)[TN / 8 / WAVES], u32 steps, u32 wave, u32 row0, u32 out0, T* __restrict__ x0,
                                            T* __restrict__ w0, T* __restrict__ x1, T* __restrict__ w1, T* __restrict__ x2, T* __restrict__ w2,
                                            T* __restrict__ x3, T* __restrict__ w3, typename Multiplied<T>::Sum (&acc)[OT][RT]) {
  constexpr u32 KE = step_elems<T>();
  const u32 inner = steps * KE;
  const auto after = [&](u32 at) { return at + KE < inner ? at + KE : 0; };
  const auto ask = [&](u32 k, T* lx, T* lw) {
    ask_tiles<T, TM, TN, WAVES>(0, x, at_x, w, at_w, k, wave, lx, lw);
    ask_tiles<T, TM, TN, WAVES>(1, x, at_x, w, at_w, k, wave, lx, lw);
  };
  u32 k = 0;
  ask(k, x0, w0);
  k = after(k);
  ask(k, x1, w1);
  k = after(k);
  ask(k, x2, w2);
  // the loads go round past the last step, rather than that the loop has other forms for its end
  for (u32 i = 0;; i += 4) {
    k = after(k);
    deep_step<T, TM, TN, WAVES>(x, at_x, w, at_w, k, wave, row0, out0, x0, w0, x3, w3, acc);
    if (i + 1 >= steps) break;
    k = after(k);
    deep_step<T, TM, TN, WAVES>(x, at_x, w, at_w, k, wave, row0, out0, x1, w1, x0, w0, acc);
    if (i + 2 >= steps) break;
    k = after(k);
    deep_step<T, TM, TN, WAVES>(x, at_x, w, at_w, k, wave, row0, out0, x2, w2, x1, w1, acc);
    if (i + 3 >= steps) break;
    k = after(k);
    deep_step<T, TM, TN, WAVES>(x, at_x, w, at_w, k, wave, row0, out0, x3, w3, x2, w2, acc);
    if (i + 4 >= steps) break;
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): none of them arrives after the block's end
}

}  // namespace local
}  // namespace haflo
