// Dropout from a counter-based generator: the mask is computed where it is used and never stored.
#include "local_common.hpp"

using namespace haflo::local;

namespace {

constexpr int kDropThreads = 256;
constexpr size_t kDropBlocks = HAFLO_LOCAL_LANES / kDropThreads < 4096 ? HAFLO_LOCAL_LANES / kDropThreads : 4096;

// A lane takes eight consecutive columns of a row: one generator call and 16-byte accesses. Memory bounds it (16384 x 4096 bfloat16 with
// a residual: 76 us, 5.3 TB/s).
template <class T, bool RESIDUAL>
__global__ __launch_bounds__(kDropThreads) void k_dropout(const T* x, size_t ldx, const T* res, size_t ldr, T* y, size_t ldy,
                                                          u32 rows, u32 cols, Drop d) {
  const u32 groups = (cols + 7) / 8;
  const u64 total = (u64)rows * groups, step = (u64)gridDim.x * kDropThreads;
  for (u64 at = (u64)blockIdx.x * kDropThreads + threadIdx.x; at < total; at += step) {
    const u32 row = (u32)(at / groups), g = (u32)(at - (u64)row * groups);
    const u32 col = g * 8;
    const int n = cols - col < 8 ? (int)(cols - col) : 8;
    const T* px = x + row * ldx + col;
    const T* pr = RESIDUAL ? res + row * ldr + col : nullptr;
    T* py = y + row * ldy + col;
    const bool wide = n == 8;
    Vec8<T> v = wide ? load_wide(px) : load_some(px, n), r = {};
    if (RESIDUAL) r = wide ? load_wide(pr) : load_some(pr, n);
    const u32x4 draws = philox(d, g, row);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float f = kept(d, draws, j) ? (float)v.get(j) * d.scale : 0.0f;
      if (RESIDUAL) f += (float)r.get(j);
      v.set(j, (T)f);
    }
    if (wide) store_wide(py, v);
    else store_some(py, v, n);
  }
}

template <class T>
int dropout(const void* x, size_t ldx, const void* res, size_t ldr, void* y, size_t ldy, size_t rows, size_t cols,
            const Drop& d, hipStream_t st) {
  const size_t need = ceil_div(rows * ceil_div(cols, 8), kDropThreads);
  const dim3 grid((unsigned)(need < kDropBlocks ? need : kDropBlocks)), block(kDropThreads);
  if (res)
    hipLaunchKernelGGL((k_dropout<T, true>), grid, block, 0, st, (const T*)x, ldx, (const T*)res, ldr, (T*)y, ldy, (u32)rows, (u32)cols, d);
  else
    hipLaunchKernelGGL((k_dropout<T, false>), grid, block, 0, st, (const T*)x, ldx, (const T*)res, ldr, (T*)y, ldy, (u32)rows, (u32)cols, d);
  return launched();
}

}  // namespace

extern "C" int haflo_dropout(int type, const void* d_x, size_t ldx, const void* d_residual, size_t ldr, void* d_y,
                             size_t ldy, size_t rows, size_t cols, double p, uint64_t seed, uint64_t offset, void* stream) {
  if (!valid_type(type) || !(p >= 0.0 && p <= 1.0) || rows > kMostCount || cols > kMostCount) return HAFLO_EINVAL;
  if (rows == 0 || cols == 0) return HAFLO_OK;
  if (!d_x || !d_y || ldx < cols || ldy < cols || (d_residual && ldr < cols)) return HAFLO_EINVAL;
  if (!in_place(d_x, ldx, d_y, ldy, rows) || !in_place(d_residual, ldr, d_y, ldy, rows)) return HAFLO_EINVAL;
  const Drop d = make_drop(p, seed, offset);
  HAFLO_LOCAL_TYPES(type, return dropout<T>(d_x, ldx, d_residual, ldr, d_y, ldy, rows, cols, d, (hipStream_t)stream));
}
