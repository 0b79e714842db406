// Matrices in 8-bit floating point with a scale for each block of 128 columns (lop_quantize_blocks).
//
// q = x * (448 / a), scale = a / 448 with a the block's largest magnitude: a block is read once, its maximum formed while it
// lies in registers. 16 lanes hold the 128 columns of a row's block, 8 values each, so that a load instruction covers four rows by 256
// bytes (bf16) and the maximum needs four exchanges inside 16 lanes. Bound by memory: 2 (4) bytes read and 1 written a value; 16384 x 4096
// values take 38 us in bf16 (5.3 TB/s), 58 us in fp32 (5.7 TB/s).
// A lane loads 32 bytes: with 64 and 128 bytes these take 40 us (bf16) and 66 us (fp32), and 64 rows 2.9 and 3.9 us instead of 2.3; with
// 16 bytes (bf16) 40 us. Blocks of 128 rows are spread over 1024 threads: 256 x 4096 values in bf16 take 3.7 us (4.4 with 256 threads), 16384 x 4096
// in fp32 59 us (66), in bf16 40 us (39).
#include <hip/hip_runtime.h>

#include "launch.hpp"
#include "lop.h"
#include "op_check.hpp"

namespace lop {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr float kMost = 448.f, kLeast = 0x1p-64f;
constexpr int kBlock = LOP_F8_BLOCK;

struct QuantizeParams {
  const char* x;
  char* q;
  float* scale;
  long long x_pitch, q_pitch, scale_row, scale_col;   // bytes, bytes, elements, elements
  int lo, hi, k, blocks;                              // rows of this launch; blocks of columns
};

template <typename T> struct Eight;   // eight values: 16 bytes of bf16, 32 of fp32
template <> struct Eight<__bf16> {
  u32x4 a;
  __device__ __forceinline__ void load(const char* p) { a = *(const u32x4*)p; }
  __device__ __forceinline__ void clear() { a = u32x4{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(a[i] << 16);
      v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
  }
};
template <> struct Eight<float> {
  u32x4 a, b;
  __device__ __forceinline__ void load(const char* p) { a = *(const u32x4*)p; b = *(const u32x4*)(p + 16); }
  __device__ __forceinline__ void clear() { a = b = u32x4{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = __uint_as_float(a[i]); v[4 + i] = __uint_as_float(b[i]); }
  }
};

__device__ __forceinline__ u32x2 to_e4m3(const float (&v)[8], float by) {
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i] * by, v[4 * i + 1] * by, 0, false);
    r[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2] * by, v[4 * i + 3] * by, w, true);
  }
  return r;
}

// A workgroup: GROUPS groups of 16 lanes, ROWS consecutive rows each, one block of columns. WHOLE: its rows share one scale.
template <typename T, int GROUPS, int ROWS, bool WHOLE>
__global__ __launch_bounds__(16 * GROUPS) void quantize_kernel(const QuantizeParams p) {
  constexpr int TILE = GROUPS * ROWS;
  static_assert(!WHOLE || TILE == kBlock, "a workgroup has a block");
  const int tile = blockIdx.x / p.blocks, kb = blockIdx.x - tile * p.blocks;
  const int group = threadIdx.x >> 4, lane = threadIdx.x & 15;
  const long long row0 = p.lo + (long long)tile * TILE + group * ROWS;
  const int col = kb * kBlock + lane * 8;
  Eight<T> in[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    if (row0 + i < p.hi && col < p.k) in[i].load(p.x + (row0 + i) * p.x_pitch + (long long)col * (int)sizeof(T));
    else in[i].clear();
  }
  float most[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    float v[8];
    in[i].get(v);
    float m = 0.f;   // (fmaxf passes a NaN over)
#pragma unroll
    for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(v[j]));
#pragma unroll
    for (int d = 1; d < 16; d *= 2) m = fmaxf(m, __shfl_xor(m, d, 64));
    most[i] = m;
  }
  if constexpr (WHOLE) {
    __shared__ float of_group[GROUPS];
    float m = most[0];
#pragma unroll
    for (int i = 1; i < ROWS; ++i) m = fmaxf(m, most[i]);
    if (lane == 0) of_group[group] = m;
    __syncthreads();
    m = of_group[0];
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) m = fmaxf(m, of_group[i]);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) most[i] = m;
  }
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const float a = fmaxf(most[i], kLeast);
    if (row0 + i < p.hi) {
      float v[8];
      in[i].get(v);
      if (col < p.k) *(u32x2*)(p.q + (row0 + i) * p.q_pitch + col) = to_e4m3(v, kMost / a);
      if (WHOLE ? (i == 0 && threadIdx.x == 0) : lane == i)
        p.scale[(WHOLE ? (row0 / kBlock) : row0 + i) * p.scale_row + kb * p.scale_col] = a / kMost;
    }
  }
}

template <typename T>
int quantize(const lop_quantize_t* op, lop_rows_t rows, hipStream_t s) {
  QuantizeParams p;
  p.x = (const char*)op->x;
  p.q = (char*)op->q;
  p.scale = op->scale;
  p.x_pitch = op->x_stride * (long long)sizeof(T);
  p.q_pitch = op->q_stride;
  p.scale_row = op->scale_row;
  p.scale_col = op->scale_col;
  p.lo = rows.lo;
  p.hi = rows.hi;
  p.k = op->k;
  p.blocks = (int)ceil_div(op->k, kBlock);
  const bool whole = op->block_rows != 1;
  constexpr int ROWS = 4 / (int)sizeof(T), GROUPS = 64;
  const int tile = whole ? kBlock : 16 * ROWS, threads = whole ? 16 * GROUPS : 256;
  const long long grid = ceil_div(rows.hi - rows.lo, tile) * p.blocks;
  if (grid > launch_blocks(threads)) return LOP_ERR_UNSUPPORTED;
  const dim3 g((unsigned)grid), b(threads);
  LOP_HIP(whole ? launch_kernel(quantize_kernel<T, GROUPS, kBlock / GROUPS, true>, g, b, s, nullptr, p)
                : launch_kernel(quantize_kernel<T, 16, ROWS, false>, g, b, s, nullptr, p));
  return LOP_OK;
}

}  // namespace
}  // namespace lop

extern "C" int lop_quantize_blocks(const lop_quantize_t* op, lop_rows_t rows, void* stream) {
  using namespace lop;
  if (!op || op->m < 0 || op->k < 1) return LOP_ERR_INVALID_ARG;
  if (!known_dtype(op->dtype) || (op->block_rows != 1 && op->block_rows != kBlock) || op->k % 16) return LOP_ERR_UNSUPPORTED;
  if (const int e = check_band(rows, op->m)) return e;
  if (op->block_rows != 1 && (rows.lo % kBlock || (rows.hi % kBlock && rows.hi != op->m))) return LOP_ERR_BAND_RANGE;
  if (rows.lo == rows.hi) return LOP_OK;
  if (!op->x || !op->q || !op->scale || !aligned16(op->x) || !aligned16(op->q) || ((uintptr_t)op->scale & 3)) return LOP_ERR_INVALID_ARG;
  if (!whole_vectors(op->x_stride, dtype_bytes(op->dtype), op->m > 1) || !whole_vectors(op->q_stride, 1, op->m > 1) || !apart(op->q_stride, op->k, op->m))
    return LOP_ERR_INVALID_ARG;
  if (op->scale_row < 0 || op->scale_col < 0 || !apart(1, op->scale_row, ceil_div(op->m, op->block_rows), op->scale_col, ceil_div(op->k, kBlock))) return LOP_ERR_INVALID_ARG;
  return op->dtype == LOP_BF16 ? quantize<__bf16>(op, rows, (hipStream_t)stream) : quantize<float>(op, rows, (hipStream_t)stream);
}
