// CPU stand-in for <hip/hip_runtime.h> for the operators of a party's local step: the one of the ciphertext operators
// with the matrix instructions on floating-point types and the few other builtins that those kernels use. Compiled by
// clang, which knows the half types.
#pragma once
#include "../../include/hip/hip_runtime.h"

// A launch is limited in lanes, as on the card, and is noted by the kernel's name as the source has it.
#include <string>
#ifndef HIPEMU_LANES
#define HIPEMU_LANES 0xFFFFFFFFu
#endif
namespace hipemu_local {
inline std::string& launches() {
  static std::string s;
  return s;
}
inline bool& refused() {
  static bool r = false;
  return r;
}
inline bool& dry() {
  static bool d = false;
  return d;
}
inline bool may_launch(const char* kernel, dim3 grid, dim3 block) {
  launches() += std::string(kernel) + "\n";
  if (dry()) return false;
  if ((uint64_t)grid.x * block.x <= HIPEMU_LANES) return true;
  refused() = true;
  return false;
}
inline hipError_t last_error() {
  const bool r = refused();
  refused() = false;
  return r ? hipErrorInvalidValue : hipSuccess;
}
}  // namespace hipemu_local
// the kernels launched since the last call
extern "C" __attribute__((weak, used)) const char* hipemu_launches() {
  static std::string s;
  s.swap(hipemu_local::launches());
  hipemu_local::launches().clear();
  return s.c_str();
}
// kernels are noted but not run
extern "C" __attribute__((weak, used)) void hipemu_dry(int on) { hipemu_local::dry() = on != 0; }
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, shmem, stream, ...)                 \
  ((void)(stream), hipemu_local::may_launch(#kernel, (grid), (block))               \
                       ? hipemu::launch((grid), (block), [&]() { kernel(__VA_ARGS__); }) \
                       : (void)0)
#define hipGetLastError hipemu_local::last_error

namespace hipemu_local {
// what each lane of a wavefront brought to its current exchange; two sets, as a lane may be one exchange ahead
struct Slots {
  float a[64][8], b[64][8];
};
inline Slots& slots(int parity) {
  static Slots s[2][32];  // by wavefront of the block
  return s[parity][threadIdx.x / 64];
}
inline int& parity() {
  static int p[2048];  // by lane of the block
  return p[threadIdx.x];
}
// one 16 x 16 product of `k` elements a lane; lane l's stand for the reduction's places k (l / 16) ..
template <class C>
inline C mfma(const float* a, const float* b, C c, int k) {
  const int lane = (int)(threadIdx.x % 64), at = parity() ^= 1;
  Slots& s = slots(at);
  for (int j = 0; j < k; ++j) {
    s.a[lane][j] = a[j];
    s.b[lane][j] = b[j];
  }
  hipemu::ballot(true);
  for (int r = 0; r < 4; ++r) {
    float sum = c[r];
    for (int g = 0; g < 4; ++g)
      for (int j = 0; j < k; ++j) sum += s.a[16 * g + 4 * (lane / 16) + r][j] * s.b[16 * g + lane % 16][j];
    c[r] = sum;
  }
  return c;
}
template <class C>
inline C mfma1(float a, float b, C c) {
  return mfma(&a, &b, c, 1);
}
template <class V, class C>
inline C mfma8(V a, V b, C c) {
  float x[8], y[8];
  for (int j = 0; j < 8; ++j) {
    x[j] = (float)a[j];
    y[j] = (float)b[j];
  }
  return mfma(x, y, c, 8);
}
}  // namespace hipemu_local

// one 16 x 16 product by 4 in 64 bits: lane l's row of the result is 4 r + l / 16
typedef double hipemu_f64x4 __attribute__((ext_vector_type(4)));
static inline hipemu_f64x4 __builtin_amdgcn_mfma_f64_16x16x4f64(double a, double b, hipemu_f64x4 c, int, int, int) {
  struct Wave {
    double a[64], b[64];
  };
  static Wave waves[2][32];  // as Slots
  const int lane = (int)(threadIdx.x % 64), at = hipemu_local::parity() ^= 1;
  Wave& s = waves[at][threadIdx.x / 64];
  s.a[lane] = a;
  s.b[lane] = b;
  hipemu::ballot(true);
  for (int r = 0; r < 4; ++r)
    for (int g = 0; g < 4; ++g) c[r] += s.a[16 * g + 4 * r + lane / 16] * s.b[16 * g + lane % 16];
  return c;
}

#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) hipemu_local::mfma8((a), (b), (c))
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) hipemu_local::mfma8((a), (b), (c))
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) hipemu_local::mfma1((a), (b), (c))
// each lane's sixteen bytes to its place behind the wavefront's address; there when the call returns
#define __builtin_amdgcn_global_load_lds(from, to, size, offset, aux) \
  memcpy((char*)(void*)(to) + (threadIdx.x % 64) * (size), (const char*)(const void*)(from), (size))
struct hipemu_buffer {
  const char* p;
  uint32_t bytes;
};
#define __amdgpu_buffer_rsrc_t hipemu_buffer
#define __builtin_amdgcn_make_buffer_rsrc(p, stride, bytes, flags) (hipemu_buffer{(const char*)(p), (uint32_t)(bytes)})
// past the buffer's end a load gives zeros
static inline void hipemu_buffer_to_lds(hipemu_buffer b, void* to, uint32_t size, uint32_t at) {
  char* const mine = (char*)to + threadIdx.x % 64 * size;
  if ((uint64_t)at + size <= b.bytes) memcpy(mine, b.p + at, size);
  else memset(mine, 0, size);
}
#define __builtin_amdgcn_raw_ptr_buffer_load_lds(b, to, size, at, more, offset, aux) \
  hipemu_buffer_to_lds((b), (void*)(to), (size), (uint32_t)(at) + (uint32_t)(more))
static inline float __builtin_amdgcn_exp2f(float x) { return exp2f(x); }
static inline void __builtin_amdgcn_s_setprio(int) {}
static inline void __builtin_amdgcn_s_waitcnt(int) {}
static inline void __builtin_amdgcn_wave_barrier() { hipemu::ballot(true); }
static inline void __builtin_amdgcn_s_barrier() { hipemu::barrier(); }
