// The row-wise operator on operands in 8-bit floating point with a scale for each block of 128 columns (lop_rowwise_f8).
//
//   y[m][n] = act( sum over blocks b of x_scale[m][b] * w_scale[n / 128][b] * (sum over the block of x[m][k] * w[n][k]) + bias[n] + residual[m][n] )
//
// The inner sum is one 16 x 16 x 128 matrix instruction with a zero accumulator; its 4 results a lane are multiplied by the two scales and added to the
// sums in fp32. (The 8-bit matrix instructions, of any shape, add up the products of a block to 1.4e-5 of the result in norm for normal values, less than the
// rounding to bf16 by a factor of 100. For fp32 outputs that would show: there the operands, which bf16 holds exactly, go through the bf16 instructions at
// half the rate, whose sums are off by 1e-7.) The weights are the instruction's rows and the matrix rows its columns, so that a lane's results
// share a matrix row, one product of two scales does for all of them, and they lie next to one another in y.
#include <hip/hip_runtime.h>

#include "act.hpp"
#include "conv_common.hpp"
#include "launch.hpp"
#include "lop.h"
#include "op_check.hpp"

namespace lop {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
constexpr unsigned kOut = 0x80000000u;   // past the end of every buffer resource here
constexpr int kBlock = LOP_F8_BLOCK;

struct F8Params {
  const char *x, *w;
  const float *x_scale, *w_scale, *bias;
  const char* res;
  char* y;
  long long x_stride, w_stride, y_stride, res_stride;              // bytes
  long long x_scale_row, x_scale_col, w_scale_row, w_scale_col;    // elements
  int lo, hi, n, k, act;
  int mx, ny;        // tiles
  int vectors;       // y, residual and n let four outputs travel together
  FastDiv by_group;
};

// 16 rows of 128 values: of a row, lane group g of four holds 16-byte chunks g and g + 4. W: the type of the matrix instruction's operands.
template <typename W> struct Operand;
template <> struct Operand<unsigned char> {
  u32x4 v[2];
  __device__ __forceinline__ void set(const u32x4& a, const u32x4& b) { v[0] = a; v[1] = b; }
  static __device__ __forceinline__ f32x4 product(const Operand& a, const Operand& b) {
    const auto whole = [](const Operand& o) __attribute__((always_inline)) {
      return i32x8{(int)o.v[0][0], (int)o.v[0][1], (int)o.v[0][2], (int)o.v[0][3], (int)o.v[1][0], (int)o.v[1][1], (int)o.v[1][2], (int)o.v[1][3]};
    };
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole(a), whole(b), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
  }
};
template <> struct Operand<__bf16> {
  bf16x8 v[4];
  __device__ __forceinline__ void set(const u32x4& a, const u32x4& b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned from = (i < 2 ? a : b)[(i & 1) * 2 + j / 2];
        const bf16x2 two = j & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(from, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(from, 1.f, false);
        w[j] = __builtin_bit_cast(unsigned, two);
      }
      v[i] = __builtin_bit_cast(bf16x8, w);
    }
  }
  static __device__ __forceinline__ f32x4 product(const Operand& a, const Operand& b) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], s, 0, 0, 0);
    return s;
  }
};
template <typename T> struct MulType { typedef unsigned char type; };
template <> struct MulType<float> { typedef __bf16 type; };

// (The median instruction of clamp_act makes the lower bound of a NaN. Here a NaN operand shows in its outputs.)
__device__ __forceinline__ float clamp_keeping_nan(float v, const Clamp& c) {
  v = v < c.lo ? c.lo : v;
  return v > c.hi ? c.hi : v;
}

// Four neighbouring outputs of one matrix row.
template <typename T>
__device__ __forceinline__ void put_four(const F8Params& p, f32x4 v, long long m, int n, const Clamp& cl) {
  if (n >= p.n) return;
  T* const y = (T*)(p.y + m * p.y_stride) + n;
  const T* const r = (const T*)(p.res + m * p.res_stride) + n;
  if (p.vectors) {
    alignas(16) T in[4], o[4];
    if (p.bias) v += *(const f32x4*)(p.bias + n);
    if (p.res) {
      __builtin_memcpy(in, __builtin_assume_aligned(r, 4 * sizeof(T)), sizeof(in));
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += to_f32(in[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = from_f32<T>(clamp_keeping_nan(v[i], cl));
    __builtin_memcpy(__builtin_assume_aligned(y, 4 * sizeof(T)), o, sizeof(o));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (n + i >= p.n) break;
      float s = v[i];
      if (p.bias) s += p.bias[n + i];
      if (p.res) s += to_f32(r[i]);
      y[i] = from_f32<T>(clamp_keeping_nan(s, cl));
    }
  }
}

// A workgroup: WM x WN wavefronts, BM matrix rows x BN outputs; stages of one block of columns of both operands in LDS, and of their scales.
// A row's 16-byte chunks lie at chunk ^ key(row): the 16 lanes that read one chunk of 16 rows at a time touch every bank once. Rows of
// the weights are dealt to the instructions so that a lane's results of four instructions are 16 neighbouring outputs: instruction
// t of four, its row r: 16 (r / 4) + 4 t + r mod 4 of 64.
template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void rowwise_f8_kernel(const F8Params p) {
  constexpr int NW = WM * WN, TM = BM / (16 * WM), TN = BN / (16 * WN);
  constexpr int A_LD = BM / (8 * NW), B_LD = BN / (8 * NW), LPS = A_LD + B_LD + 1;   // load instructions of a wavefront and stage
  constexpr int A_BYTES = BM * 128, S_AT = (BM + BN) * 128, STAGE = S_AT + NW * 256;
  static_assert(NW > BM / 64 && BM % 64 == 0 && TN % 4 == 0 && 128 % (BN / WN) == 0, "tile shape");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * STAGE];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM, wn = wave / WM;
  const TileId tile = xcd_tile_of(blockIdx.x, p.mx, p.ny, 1, p.by_group);
  const long long m0 = p.lo + (long long)tile.m * BM;
  const int n0 = tile.n * BN, ns = (p.k + kBlock - 1) / kBlock;

  const __amdgpu_buffer_rsrc_t xbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.x + m0 * p.x_stride), 0, 0x7fffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t wbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.w + n0 * p.w_stride), 0, 0x7fffffff, 0x00020000);
  unsigned a_off[A_LD], b_off[B_LD];
  bool a_past[A_LD], b_past[B_LD];   // the chunk lies past the end of the reduction in the last stage
#pragma unroll
  for (int i = 0; i < A_LD; ++i) {
    const int row = (wave + NW * i) * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
    a_off[i] = m0 + row < p.hi ? (unsigned)(row * (int)p.x_stride + chunk * 16) : kOut;
    a_past[i] = (ns - 1) * kBlock + chunk * 16 >= p.k;
  }
#pragma unroll
  for (int i = 0; i < B_LD; ++i) {
    const int row = (wave + NW * i) * 8 + (lane >> 3), chunk = (lane & 7) ^ (((row >> 1) & 1) | ((row >> 4) & 3) << 1);
    b_off[i] = n0 + row < p.n ? (unsigned)(row * (int)p.w_stride + chunk * 16) : kOut;
    b_past[i] = (ns - 1) * kBlock + chunk * 16 >= p.k;
  }
  // scales: wavefronts 0 .. BM / 64 - 1 those of 64 matrix rows each, the others those of the weights' blocks
  const bool of_x = wave < BM / 64;
  unsigned s_off;
  if (of_x) s_off = m0 + wave * 64 + lane < p.hi ? (unsigned)((wave * 64 + lane) * (int)p.x_scale_row * 4) : kOut;
  else s_off = lane < (BN + kBlock - 1) / kBlock && n0 + lane * kBlock < p.n ? (unsigned)(lane * (int)p.w_scale_row * 4) : kOut;
  const float* const s_base = of_x ? p.x_scale + m0 * p.x_scale_row : p.w_scale + n0 / kBlock * p.w_scale_row;
  const long long s_step = of_x ? p.x_scale_col : p.w_scale_col;

  auto issue = [&](int s) __attribute__((always_inline)) {
    unsigned char* const dst = smem + (s & 1) * STAGE;
    const bool last = s == ns - 1;
#pragma unroll
    for (int i = 0; i < A_LD; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(xbuf, (__attribute__((address_space(3))) void*)(dst + (wave + NW * i) * 1024), 16,
                                               (int)((last & a_past[i]) ? kOut : a_off[i]), s * kBlock, 0, 0);
#pragma unroll
    for (int i = 0; i < B_LD; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(wbuf, (__attribute__((address_space(3))) void*)(dst + A_BYTES + (wave + NW * i) * 1024), 16,
                                               (int)((last & b_past[i]) ? kOut : b_off[i]), s * kBlock, 0, 0);
    const __amdgpu_buffer_rsrc_t sbuf =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(s_base + s * s_step), 0, 0x7fffffff, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(sbuf, (__attribute__((address_space(3))) void*)(dst + S_AT + wave * 256), 4, (int)s_off, 0, 0, 0);
  };
  auto barrier = [&]() __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  const unsigned lds0 = (unsigned)(unsigned long)(__attribute__((address_space(3))) unsigned char*)smem;
  const int r16 = lane & 15, g = lane >> 4;
  // fragments: chunks g and g + 4 of a row
  const unsigned a_at = lds0 + (unsigned)((wm * TM * 16 + r16) * 128 + ((g ^ (r16 >> 1)) & 7) * 16);
  const int wrow = 16 * (r16 >> 2) + (r16 & 3);
  const unsigned b_at = lds0 + (unsigned)(A_BYTES + (wn * TN * 16 + wrow) * 128 + ((g ^ (((r16 >> 1) & 1) | (r16 >> 2) << 1)) & 7) * 16);
  const unsigned sx_at = lds0 + (unsigned)(S_AT + (wm * TM * 16 + r16) * 4);
  const unsigned sw_at = lds0 + (unsigned)(S_AT + BM * 4 + (wn * TN * 16 / kBlock) * 4);

  f32x4 acc[TN][TM];
#pragma unroll
  for (int a = 0; a < TN; ++a)
#pragma unroll
    for (int b = 0; b < TM; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};

  issue(0);
  if (ns > 1) issue(1);
  for (int s = 0; s < ns; ++s) {
    if (s + 1 < ns) __builtin_amdgcn_s_waitcnt(vmcnt_imm(LPS));
    else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    barrier();
    const unsigned at = (unsigned)((s & 1) * STAGE);
    u32x4 fx[TM][2];
    float sx[TM], sw;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(fx[i][0]) : "v"(a_at + at), "n"(i * 2048) : "memory");
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(fx[i][1]) : "v"((a_at + at) ^ 64u), "n"(i * 2048) : "memory");
      asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(sx[i]) : "v"(sx_at + at), "n"(i * 64) : "memory");
    }
    asm volatile("ds_read_b32 %0, %1" : "=v"(sw) : "v"(sw_at + at) : "memory");
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(fx[i][0]), "+v"(fx[i][1]), "+v"(sx[i]));
    asm volatile("" : "+v"(sw));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < TM; ++i) sx[i] *= sw;
    typedef Operand<typename MulType<T>::type> Op;
    Op ox[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) ox[i].set(fx[i][0], fx[i][1]);
#pragma unroll
    for (int t = 0; t < TN; ++t) {
      u32x4 fw[2];
      const int off = (t / 4) * 64 * 128 + (t % 4) * 4 * 128;
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(fw[0]) : "v"(b_at + at), "n"(off) : "memory");
      asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(fw[1]) : "v"((b_at + at) ^ 64u), "n"(off) : "memory");
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      asm volatile("" : "+v"(fw[0]), "+v"(fw[1]));
      Op ow;
      ow.set(fw[0], fw[1]);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const f32x4 part = Op::product(ow, ox[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][i][e] = fmaf(part[e], sx[i], acc[t][i][e]);
      }
    }
    if (s + 2 < ns) {
      barrier();   // (no wavefront reads this stage any more)
      issue(s + 2);
    }
  }

  const Clamp cl = make_clamp(p.act);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const long long m = m0 + wm * TM * 16 + i * 16 + r16;
    if (m >= p.hi) continue;
#pragma unroll
    for (int t = 0; t < TN; ++t) put_four<T>(p, acc[t][i], m, n0 + wn * TN * 16 + (t / 4) * 64 + g * 16 + (t % 4) * 4, cl);
  }
}

template <typename T>
int rowwise_f8(const lop_rowwise_f8_t* op, lop_rows_t rows, hipStream_t stream) {
  constexpr int E = (int)sizeof(T);
  F8Params p;
  p.x = (const char*)op->x; p.w = (const char*)op->w;
  p.x_scale = op->x_scale; p.w_scale = op->w_scale; p.bias = op->bias;
  p.res = (const char*)op->residual; p.y = (char*)op->y;
  p.x_stride = op->x_stride; p.w_stride = op->w_stride;
  p.y_stride = op->y_stride * E; p.res_stride = op->residual_stride * E;
  p.x_scale_row = op->x_scale_row; p.x_scale_col = op->x_scale_col;
  p.w_scale_row = op->w_scale_row; p.w_scale_col = op->w_scale_col;
  p.lo = rows.lo; p.hi = rows.hi; p.n = op->n; p.k = op->k; p.act = op->act;
  const uintptr_t bits = (uintptr_t)p.y | (uintptr_t)p.res | (uintptr_t)p.y_stride | (uintptr_t)(p.res ? p.res_stride : 0);
  p.vectors = bits % (4 * E) == 0 && op->n % 4 == 0 && aligned16(p.bias);
  constexpr int BM = 128, BN = 128;
  const long long mx = ceil_div(rows.hi - rows.lo, BM), ny = ceil_div(op->n, BN);
  if (mx * ny > launch_blocks(256) || ny > 65535) return LOP_ERR_UNSUPPORTED;
  p.mx = (int)mx; p.ny = (int)ny;
  p.by_group = make_fastdiv(kGroupM * p.ny);
  LOP_HIP(launch_kernel(rowwise_f8_kernel<T, BM, BN, 2, 2>, dim3((unsigned)(mx * ny)), dim3(256), stream, nullptr, p));
  return LOP_OK;
}

}  // namespace
}  // namespace lop

extern "C" int lop_rowwise_f8(const lop_rowwise_f8_t* op, lop_rows_t rows, void* stream) {
  using namespace lop;
  if (!op || op->m < 0 || op->n < 1 || op->k < 1) return LOP_ERR_INVALID_ARG;
  if (!known_dtype(op->dtype) || op->k % 16 || op->act < LOP_ACT_NONE || op->act > LOP_ACT_RELU6) return LOP_ERR_UNSUPPORTED;
  if (const int e = check_band(rows, op->m)) return e;
  if (rows.lo == rows.hi) return LOP_OK;
  const size_t E = dtype_bytes(op->dtype);
  if (!op->x || !op->w || !op->x_scale || !op->w_scale || !op->y || !aligned16(op->x) || !aligned16(op->w)) return LOP_ERR_INVALID_ARG;
  if (((uintptr_t)op->x_scale | (uintptr_t)op->w_scale | (uintptr_t)op->bias) & 3) return LOP_ERR_INVALID_ARG;
  if (((uintptr_t)op->y | (uintptr_t)op->residual) & (E - 1)) return LOP_ERR_INVALID_ARG;
  if (!whole_vectors(op->x_stride, 1, op->m > 1) || !whole_vectors(op->w_stride, 1, op->n > 1)) return LOP_ERR_INVALID_ARG;
  if (op->x_scale_row < 0 || op->x_scale_col < 0 || op->w_scale_row < 0 || op->w_scale_col < 0 || op->y_stride < 0 ||
      (op->residual && op->residual_stride < 0))
    return LOP_ERR_INVALID_ARG;
  // (offsets within a tile of at most 256 rows are 32 bits)
  constexpr long long far = (1LL << 31) / 256 - 1;
  if ((op->m > 1 && op->x_stride + op->k > far) || (op->n > 1 && op->w_stride + op->k > far) || (op->m > 1 && op->x_scale_row > far / 4) ||
      (op->n > kBlock && op->w_scale_row > far / 4) || op->k > far)
    return LOP_ERR_UNSUPPORTED;
  return op->dtype == LOP_BF16 ? rowwise_f8<__bf16>(op, rows, (hipStream_t)stream) : rowwise_f8<float>(op, rows, (hipStream_t)stream);
}
