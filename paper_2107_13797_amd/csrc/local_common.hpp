// Helpers shared by the operators of a party's local step: element types, the dropout generator, wavefront
// reductions, matrix instructions.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/haflo_local.h"

namespace haflo {
namespace local {

using u16 = uint16_t;
using u32 = uint32_t;
using u64 = uint64_t;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32 u32x4 __attribute__((ext_vector_type(4), may_alias));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kWave = 64;
constexpr size_t kMostCount = 0x7FFFFFFF;

// Eight consecutive elements, the unit of loads, stores and of a dropout call. It is held in whole words, and elements are
// taken out where they are used: as eight elements it would be taken apart right behind its load, which would so be waited for.
template <class T>
struct Vec8 {
  u32x4 w[sizeof(T) / 2];
  __device__ __forceinline__ T get(int j) const {
    if constexpr (sizeof(T) == 4) {
      const u32 word = w[j >> 2][j & 3];  // (a copy: the cast of an element itself takes the vector's first)
      return __builtin_bit_cast(T, word);
    } else {
      return __builtin_bit_cast(T, (u16)(w[0][j >> 1] >> (16 * (j & 1))));
    }
  }
  __device__ __forceinline__ void set(int j, T v) {
    if constexpr (sizeof(T) == 4) {
      w[j >> 2][j & 3] = __builtin_bit_cast(u32, v);
    } else {
      const u32 b = __builtin_bit_cast(u16, v);
      w[0][j >> 1] = j & 1 ? (w[0][j >> 1] & 0xFFFFu) | b << 16 : (w[0][j >> 1] & 0xFFFF0000u) | b;
    }
  }
};

// Vector accesses of memory need no more alignment than an element's.
typedef u32x4 u32x4_of_2 __attribute__((aligned(2), may_alias));
typedef u32x4 u32x4_of_4 __attribute__((aligned(4), may_alias));
template <class T>
__device__ __forceinline__ Vec8<T> load_wide(const T* p) {
  Vec8<T> r;
#pragma unroll
  for (u32 i = 0; i < sizeof(T) / 2; ++i) {
    if constexpr (sizeof(T) == 2) r.w[i] = ((const u32x4_of_2*)p)[i];
    else r.w[i] = ((const u32x4_of_4*)p)[i];
  }
  return r;
}
template <class T>
__device__ __forceinline__ void store_wide(T* p, const Vec8<T>& r) {
#pragma unroll
  for (u32 i = 0; i < sizeof(T) / 2; ++i) {
    if constexpr (sizeof(T) == 2) ((u32x4_of_2*)p)[i] = r.w[i];
    else ((u32x4_of_4*)p)[i] = r.w[i];
  }
}
// The first `n` of eight elements; the others are `other`.
template <class T>
__device__ __forceinline__ Vec8<T> load_some(const T* p, int n, T other = (T)0.0f) {
  Vec8<T> r = {};
#pragma unroll
  for (int j = 0; j < 8; ++j) r.set(j, j < n ? p[j] : other);
  return r;
}
template <class T>
__device__ __forceinline__ void store_some(T* p, const Vec8<T>& v, int n) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < n) p[j] = v.get(j);
}

// Eight elements of a row from column `col` on, zeros behind its end; no element of another vector is read. Lanes past the end, as
// groups of a power of two have them, take no part in what the one across it does.
template <class T>
__device__ __forceinline__ Vec8<T> load_cols(const T* row, u32 col, u32 cols) {
  if (col + 8 <= cols) return load_wide(row + col);
  if (col >= cols) return Vec8<T>{};
  return load_some(row + col, (int)(cols - col));
}
// The same in two steps where nothing is written over the row, and it has eight elements: a load without a branch, as the compiler waits for
// a load at the next branch around one, of the row's last eight where the elements pass its end; and their moving to their places,
// with zeros behind them.
template <class T>
__device__ __forceinline__ Vec8<T> load_clamped(const T* row, u32 col, u32 cols) {
  return load_wide(row + (col + 8 <= cols ? col : cols - 8));
}
template <class T>
__device__ __forceinline__ void settle(Vec8<T>& v, u32 col, u32 cols) {
  if (col + 8 <= cols || cols < 8) return;
  const u32 by = col + 8 - cols;
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
__device__ __forceinline__ void store_cols(T* row, u32 col, u32 cols, const Vec8<T>& v) {
  if (col + 8 <= cols) store_wide(row + col, v);
  else if (col < cols) store_some(row + col, v, (int)(cols - col));
}

// The dropout of one call: what a kernel needs of (p, seed, offset).
struct Drop {
  u32 threshold;  // draws below it drop their element; 0: no dropout
  float scale;
  u32 k0, k1, o0, o1;
};
inline Drop make_drop(double p, u64 seed, u64 offset) {
  Drop d;
  d.threshold = (u32)__builtin_rint(p * 65536.0);
  d.scale = d.threshold >= 65536u ? 0.0f : (float)(65536.0 / (65536.0 - (double)d.threshold));
  d.k0 = (u32)seed;
  d.k1 = (u32)(seed >> 32);
  d.o0 = (u32)offset;
  d.o1 = (u32)(offset >> 32);
  return d;
}
// Philox4x32-10: ten rounds of two 32 x 32 -> 64-bit products.
__device__ __forceinline__ u32x4 philox(const Drop& d, u32 group, u32 row) {
  u32 c0 = group, c1 = row, c2 = d.o0, c3 = d.o1, k0 = d.k0, k1 = d.k1;
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const u64 x = (u64)c0 * 0xD2511F53u, y = (u64)c2 * 0xCD9E8D57u;
    c0 = (u32)(y >> 32) ^ c1 ^ k0;
    c1 = (u32)y;
    c2 = (u32)(x >> 32) ^ c3 ^ k1;
    c3 = (u32)x;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  u32x4 r = {c0, c1, c2, c3};
  return r;
}
__device__ __forceinline__ bool kept(const Drop& d, const u32x4& draws, int j) {
  return ((draws[j >> 1] >> (16 * (j & 1))) & 0xFFFFu) >= d.threshold;
}

__device__ __forceinline__ u32 lane_id() { return threadIdx.x & (kWave - 1); }
__device__ __forceinline__ u32 lane_read(u32 v, int lane) {
  return (u32)__builtin_amdgcn_ds_bpermute(lane << 2, (int)v);
}
__device__ __forceinline__ float lane_read(float v, int lane) {
  return __builtin_bit_cast(float, lane_read(__builtin_bit_cast(u32, v), lane));
}
__device__ __forceinline__ u64 lane_read(u64 v, int lane) {
  const u32 lo = lane_read((u32)v, lane), hi = lane_read((u32)(v >> 32), lane);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ double lane_read(double v, int lane) {
  return __builtin_bit_cast(double, lane_read(__builtin_bit_cast(u64, v), lane));
}

// What a lane of the same sixteen holds, by a move that the vector unit makes on the way (quad_perm, row_half_mirror, row_mirror)
template <int CTRL>
__device__ __forceinline__ u32 lane_swap(u32 v) {
  return (u32)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int CTRL>
__device__ __forceinline__ float lane_swap(float v) {
  return __builtin_bit_cast(float, lane_swap<CTRL>(__builtin_bit_cast(u32, v)));
}
template <int CTRL>
__device__ __forceinline__ double lane_swap(double v) {
  const u64 b = __builtin_bit_cast(u64, v);
  return __builtin_bit_cast(double, (u64)lane_swap<CTRL>((u32)(b >> 32)) << 32 | lane_swap<CTRL>((u32)b));
}
// `with` over a wavefront's groups of `lanes` lanes, a power of two: pairs, then pairs of what they hold, so that with a commutative `with` all
// lanes of a group hold the same bits.
template <class S, class F>
__device__ __forceinline__ S lanes_join(S v, u32 lanes, const F& with) {
  if (lanes >= 2) v = with(v, lane_swap<0xB1>(v));
  if (lanes >= 4) v = with(v, lane_swap<0x4E>(v));
  if (lanes >= 8) v = with(v, lane_swap<0x141>(v));
  if (lanes >= 16) v = with(v, lane_swap<0x140>(v));
  if (lanes >= 32) v = with(v, lane_read(v, (int)(lane_id() ^ 16)));
  if (lanes >= 64) v = with(v, lane_read(v, (int)(lane_id() ^ 32)));
  return v;
}

// acc += a b on 16 x 16 by 32: lane l holds rows l % 16 of both operands at elements 8 (l / 16) .. + 7, and in
// acc[r] row 4 (l / 16) + r of the first operand against row l % 16 of the second.
__device__ __forceinline__ f32x4 mma32(const Vec8<__bf16>& a, const Vec8<__bf16>& b, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma32(const Vec8<_Float16>& a, const Vec8<_Float16>& b, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}
// the same in 32 bits: each instruction takes one element of every lane, so that element j of lane group g stands for
// the reduction's place 8 g + j in both operands alike
__device__ __forceinline__ f32x4 mma32(const Vec8<float>& a, const Vec8<float>& b, f32x4 acc) {
#pragma unroll
  for (int j = 0; j < 8; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a.get(j), b.get(j), acc, 0, 0, 0);
  return acc;
}

inline bool valid_type(int type) { return type == HAFLO_F32 || type == HAFLO_F16 || type == HAFLO_BF16; }
inline size_t type_size(int type) { return type == HAFLO_F32 ? 4 : 2; }
inline size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }
inline size_t ceil_div(size_t a, size_t b) { return (a + b - 1) / b; }
// Whether an output may lie where an input does: each element over its own, so with rows equally far apart.
inline bool in_place(const void* in, size_t ld_in, const void* out, size_t ld_out, size_t rows) {
  return in != out || ld_in == ld_out || rows <= 1;
}
// Whether a workspace does for a call that needs `bytes`: its parts are read sixteen bytes at a time.
inline bool enough(const void* ws, size_t ws_bytes, size_t bytes) {
  return bytes == 0 || (ws && (uintptr_t)ws % 16 == 0 && ws_bytes >= bytes);
}
// Lanes of one launch at most: the runtime counts them in 32 bits. What takes more is launched in turns, each from the block on that
// the kernel's last argument names.
#ifndef HAFLO_LOCAL_LANES
#define HAFLO_LOCAL_LANES 0x80000000u
#endif
template <class F>
inline void in_turns(size_t blocks, u32 threads, const F& launch) {
  const size_t most = HAFLO_LOCAL_LANES / threads;
  for (size_t first = 0; first < blocks; first += most)
    launch((u32)first, dim3((unsigned)(blocks - first < most ? blocks - first : most)), dim3(threads));
}
inline int launched() { return hipGetLastError() == hipSuccess ? HAFLO_OK : HAFLO_EHIP; }

}  // namespace local
}  // namespace haflo

// Calls BODY with T as the element type that `type` names.
#define HAFLO_LOCAL_TYPES(type, ...)         \
  do {                                       \
    if ((type) == HAFLO_F32) {               \
      using T = float;                       \
      __VA_ARGS__;                           \
    } else if ((type) == HAFLO_F16) {        \
      using T = _Float16;                    \
      __VA_ARGS__;                           \
    } else {                                 \
      using T = __bf16;                      \
      __VA_ARGS__;                           \
    }                                        \
  } while (0)
