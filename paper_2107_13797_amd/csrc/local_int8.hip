// A projection with weights of eight bits, as the common model answers with: one scale for each output and one for each row of x.
//
//   s = amax / 127,  q = rint(v (127 / amax))  of every row,      y[t, o] = s_x[t] s_w[o] sum_k q_x[t, k] q_w[o, k] + bias[o] + residual[t, o]
//
// Sums are whole numbers of 32 bits and exact. Rows of eight bits are kept with zeros up to a multiple of 128 bytes, so that no
// product has an end to look after.
#include "local_common.hpp"

using namespace haflo::local;

namespace {

constexpr u32 kThreads = 256, kWaves = kThreads / kWave;
constexpr u32 kMostLanes = 1024;
constexpr size_t kRow = HAFLO_INT8_ROW, kMostInner = HAFLO_INT8_MAX_COLS;
typedef int i32x4 __attribute__((ext_vector_type(4)));

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

// Rows to eight bits: a group of `lanes` lanes a row, eight columns to a lane, and of a longer row the others again. Memory bounds it.
template <class T>
__global__ __launch_bounds__(kMostLanes) void k_quantize(const T* x, size_t ldx, u32 rows, u32 cols, u32 width, u32 lanes, int8_t* q, float* scale,
                                                         u32 first_block) {
  __shared__ u32 most[kMostLanes / kWave];
  const u32 groups = blockDim.x / lanes, at = threadIdx.x % lanes * 8;
  const u64 mine = (u64)(first_block + blockIdx.x) * groups + threadIdx.x / lanes;
  const u64 row = mine < rows ? mine : rows - 1;
  const T* const from = x + row * ldx;
  const Vec8<T> own = load_cols(from, at, cols);
  u32 m = most_of(own);
  for (u32 col = at + lanes * 8; col < cols; col += lanes * 8) {
    const u32 b = most_of(load_cols(from, col, cols));
    m = b > m ? b : m;
  }
  for (u32 d = 1; d < lanes && d < kWave; d <<= 1) {
    const u32 o = lane_read(m, (int)(lane_id() ^ d));
    m = o > m ? o : m;
  }
  if (lanes > kWave) {
    if (lane_id() == 0) most[threadIdx.x / kWave] = m;
    __syncthreads();
    for (u32 w = 0; w < lanes / kWave; ++w) m = most[w] > m ? most[w] : m;
  }
  if (mine >= rows) return;
  const Scale s = scale_of(m);
  u64* const to = (u64*)(q + row * width);
  if (at < width) to[at / 8] = eight_bits(own, s);
  for (u32 col = at + lanes * 8; col < width; col += lanes * 8) to[col / 8] = eight_bits(load_cols(from, col, cols), s);
  if (at == 0) scale[row] = s.scale;
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
// four outputs from `o` on of row t
template <class T>
__device__ __forceinline__ void store_four(const Out<T>& to, u32 t, u32 o, const i32x4& acc) {
  if (t >= to.rows) return;
  const float by = to.x_scale[t];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (o + r >= to.outer) return;
    float v = (float)acc[r] * (by * to.w_scale[o + r]);
    if (to.bias) v += to.bias[o + r];
    if (to.residual) v += (float)to.residual[t * to.ldr + o + r];
    to.y[t * to.ldy + o + r] = (T)v;
  }
}

// y of 16 outputs by 16 R rows, a wavefront each, its operands from memory as they are needed.
template <class T, int R>
__global__ __launch_bounds__(kThreads) void k_int8(const int8_t* x, const int8_t* w, u32 width, Out<T> to, u32 first_block) {
  const u32 wave = threadIdx.x / kWave, lane = lane_id(), tiles = (to.outer + 63) / 64, block = first_block + blockIdx.x;
  const u32 o0 = (block % tiles * kWaves + wave) * 16, t0 = block / tiles * 16 * R;
  const auto row = [&](u32 i, u32 n) { return i < n ? i : n - 1; };
  const int8_t* const wr = w + (size_t)row(o0 + lane % 16, to.outer) * width + lane / 16 * 16;
  const int8_t* xr[R];
  i32x4 acc[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    xr[j] = x + (size_t)row(t0 + 16 * j + lane % 16, to.rows) * width + lane / 16 * 16;
    acc[j] = i32x4{0, 0, 0, 0};
  }
  for (u32 k = 0; k < width; k += 64) {
    const i32x4 a = *(const i32x4*)(wr + k);
#pragma unroll
    for (int j = 0; j < R; ++j) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, *(const i32x4*)(xr[j] + k), acc[j], 0, 0, 0);
  }
#pragma unroll
  for (int j = 0; j < R; ++j) store_four(to, t0 + 16 * j + lane % 16, o0 + lane / 16 * 4, acc[j]);
}

template <class T>
void quantize(const void* x, size_t ldx, size_t rows, size_t cols, int8_t* q, float* scale, hipStream_t st) {
  const size_t width = row_bytes(cols);
  u32 lanes = 16;
  while (lanes < kMostLanes && (size_t)lanes * 8 < width) lanes *= 2;
  const u32 threads = lanes <= (u32)kWave ? kThreads : lanes;
  in_turns(ceil_div(rows, threads / lanes), threads, [&](u32 first, dim3 grid, dim3 block) {
    hipLaunchKernelGGL((k_quantize<T>), grid, block, 0, st, (const T*)x, ldx, (u32)rows, (u32)cols, (u32)width, lanes, q, scale, first);
  });
}
template <class T>
void product(const int8_t* x, const int8_t* w, size_t cols, const Out<T>& to, hipStream_t st) {
  in_turns(ceil_div(to.rows, 64) * ceil_div(to.outer, 64), kThreads, [&](u32 first, dim3 grid, dim3 block) {
    hipLaunchKernelGGL((k_int8<T, 4>), grid, block, 0, st, x, w, (u32)row_bytes(cols), to, first);
  });
}

bool int8_sizes(int type, size_t rows, size_t inner, size_t outer) {
  return valid_type(type) && rows <= kMostCount && inner >= 1 && inner <= kMostInner && outer >= 1 && outer <= kMostCount && rows * outer <= kMostResults;
}
bool aligned(const void* p) { return p && (uintptr_t)p % 16 == 0; }
struct Plan {
  size_t scale, total;
};
Plan int8_plan(size_t rows, size_t inner) {
  Plan p;
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
  return int8_sizes(type, rows, inner, outer) ? int8_plan(rows, inner).total : (size_t)-1;
}

int haflo_int8_forward(int type, const void* d_x, size_t ldx, const int8_t* d_wq, const float* d_w_scale, const float* d_bias, const void* d_residual,
                       size_t ldr, size_t rows, size_t inner, size_t outer, void* d_y, size_t ldy, void* d_workspace, size_t workspace_bytes,
                       void* stream) {
  if (!int8_sizes(type, rows, inner, outer)) return HAFLO_EINVAL;
  if (rows == 0) return HAFLO_OK;
  if (!d_x || ldx < inner || !aligned(d_wq) || !d_w_scale || (d_residual && ldr < outer) || !d_y || ldy < outer) return HAFLO_EINVAL;
  if (!in_place(d_residual, ldr, d_y, ldy, rows)) return HAFLO_EINVAL;
  const Plan plan = int8_plan(rows, inner);
  if (!enough(d_workspace, workspace_bytes, plan.total)) return HAFLO_EINVAL;
  int8_t* const xq = (int8_t*)d_workspace;
  float* const x_scale = (float*)((char*)d_workspace + plan.scale);
  HAFLO_LOCAL_TYPES(type, {
    quantize<T>(d_x, ldx, rows, inner, xq, x_scale, (hipStream_t)stream);
    const Out<T> to = {x_scale, d_w_scale, d_bias, (const T*)d_residual, ldr, (T*)d_y, ldy, (u32)rows, (u32)outer};
    product<T>(xq, d_wq, inner, to, (hipStream_t)stream);
  });
  return launched();
}

}  // extern "C"
