// The row-wise operator on operands in 8-bit floating point with a scale for each block of 128 columns (lop_rowwise_f8).
//
//   y[m][n] = act( sum over blocks b of x_scale[m][b] * w_scale[n / 128][b] * (sum over the block of x[m][k] * w[n][k]) + bias[n] + residual[m][n] )
//
// The inner sum is one 16 x 16 x 128 matrix instruction with a zero accumulator; its 4 results a lane are multiplied by the two scales and added to the
// sums in fp32. (The 8-bit matrix instructions align the products of eight neighbouring columns at the largest sum of two exponents among them, E, and cut what is
// below 2^(E - 13) off towards zero; the eights are added in fp32. For normal values that is 1.4e-5 of the result in norm, less than the rounding to bf16 by a
// factor of 100; where large products cancel each other it is more than that of what is left. For fp32 outputs it would show always: there the operands, which bf16 holds exactly, go through the bf16
// instructions at half the rate, whose sums are off by 1e-7.) The weights are the instruction's rows and the matrix rows its columns, so that a lane's results
// share a matrix row, one product of two scales does for all of them, and they lie next to one another in y.
//
// Bound: large products by the matrix instructions and the scaling between them: 16384 x 4096 to 16384 outputs take 1013 us, 2.17 PFLOP/s (a library
// product without scales 2.6); few rows by reading the weights: 48 rows of 4096 to 4096 9.8 us, where the launch and the way to memory are most of it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>

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
  int vectors;       // rows of y and residual begin on 16 bytes and are a multiple of that
  FastDiv by_group;
};

// 16 rows of 128 values: of a row, lane group g of four holds 16-byte chunks g and g + 4. W: the type of the matrix instruction's operands.
template <typename W> struct Operand;
template <> struct Operand<unsigned char> {
  i32x8 v;
  // (Without the statement the compiler takes the upper half of an operand that is carried around a loop for dead.)
  __device__ __forceinline__ void set(const u32x4& a, const u32x4& b) {
    v = i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
    asm("" : "+v"(v));
  }
  static __device__ __forceinline__ f32x4 product(const Operand& a, const Operand& b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
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
    alignas(16) T o[4];
    if (p.bias)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += p.bias[n + i];
    if (p.res) {
      __builtin_memcpy(o, __builtin_assume_aligned(r, 4 * sizeof(T)), sizeof(o));
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += to_f32(o[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = from_f32<T>(clamp_keeping_nan(v[i], cl));
    __builtin_memcpy(__builtin_assume_aligned(y, 4 * sizeof(T)), o, sizeof(o));
  } else {
    float bias[4] = {0.f, 0.f, 0.f, 0.f}, add[4] = {0.f, 0.f, 0.f, 0.f};   // (first: one wait for all of them)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = min(i, p.n - 1 - n);
      if (p.bias) bias[i] = p.bias[n + at];
      if (p.res) add[i] = to_f32(r[at]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < p.n) y[i] = from_f32<T>(clamp_keeping_nan(v[i] + bias[i] + add[i], cl));
  }
}

// A workgroup: WM x WN wavefronts, BM matrix rows x BN outputs; stages of one block of columns of both operands in LDS, and of their scales.
// A row's 16-byte chunks lie at chunk ^ key(row): the 16 lanes that read one chunk of 16 rows at a time touch every bank once. Rows of
// the weights are dealt to the instructions so that a lane's results of four instructions are 16 neighbouring outputs: instruction
// t of four, its row r: 16 (r / 4) + 4 t + r mod 4 of 64.
//  - A wavefront goes through its weight tiles, TM products each: the next tile is read from LDS meanwhile, and the results of
//    the one before are scaled and added, four vector instructions under each matrix instruction.
//  - In front of the last weight tile there is a barrier: the stage's last operands are in registers, and the next stage's are
//    read, each matrix tile into the registers that its last product has left.
//  - Two stages are all that LDS holds of the large tile, and a stage lasts a microsecond. So its memory is refilled in two parts, as it falls free: that of the
//    matrix rows, the scales and the first half of the weights behind a barrier in the middle (HALVES), the rest behind the one at the end: every load is
//    issued a stage and a half ahead of its use.
//  - Where a workgroup fills a compute unit (HALVES) it takes tile after tile, and the next one's first stages are on their way while this one's sums leave.
//  - Where there are few tiles, KG groups of wavefronts take every KG-th stage each, and their sums are added in LDS in the order of the groups.
template <typename T, int BM, int BN, int WM, int WN, int KG>
__global__ __launch_bounds__(64 * WM * WN * KG) __attribute__((amdgpu_waves_per_eu(2))) void rowwise_f8_kernel(const F8Params p) {
  typedef Operand<typename MulType<T>::type> Op;
  constexpr int NW = WM * WN, TM = BM / (16 * WM), TN = BN / (16 * WN), E = (int)sizeof(T), VE = 16 / E;
  constexpr int A_LD = BM / (8 * NW), B_LD = BN / (8 * NW), LPS = A_LD + B_LD + 1;   // load instructions of a wavefront and stage
  constexpr int A_BYTES = BM * 128, S_AT = (BM + BN) * 128, STAGE = S_AT + NW * 256;
  constexpr bool HALVES = TN == 8;   // (a wavefront's first four weight tiles are the first 64 of its 128 rows)
  constexpr int END = HALVES ? B_LD / 2 : LPS, MID = LPS - END;   // loads behind the barrier at the end, in the middle
  static_assert(!HALVES || NW * 8 == 64, "a load instruction's rows are all of one half");
  static_assert(NW > BM / 64 && BM % 64 == 0 && TN % 4 == 0 && 128 % (BN / WN) == 0, "tile shape");
  static_assert(KG == 1 || !HALVES, "groups have a tile");
  __shared__ __attribute__((aligned(1024))) unsigned char smem[KG * 2 * STAGE];

  const int lane = threadIdx.x & 63;
  const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NW;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % NW;   // of the group
  unsigned char* const mine = smem + group * 2 * STAGE;
  const int wm = wave % WM, wn = wave / WM;
  const int ns = (p.k + KG * kBlock - 1) / (KG * kBlock);   // stages of a group (one past the reduction is zeros)
  long long m0;
  int n0;

  __amdgpu_buffer_rsrc_t xbuf, wbuf;
  // What this lane fetches: row lane / 8 of the groups of eight wave + NW i. (Its chunk of matrix rows, and so whether that lies past the end of the
  // reduction in the last stage, is the same for all of them: the keys repeat after NW groups.)
  static_assert(NW % 2 == 0, "keys");
  unsigned a_off[A_LD], b_off[B_LD];
  const int row8 = wave * 8 + (lane >> 3), a_chunk = (lane & 7) ^ ((row8 >> 1) & 7);
  int b_chunk[B_LD];
#pragma unroll
  for (int i = 0; i < B_LD; ++i) {
    const int row = row8 + NW * 8 * i;
    b_chunk[i] = (lane & 7) ^ (((row >> 1) & 1) | ((row >> 4) & 3) << 1);
  }
  // scales: wavefronts 0 .. BM / 64 - 1 those of 64 matrix rows each, the others those of the weights' blocks
  const bool of_x = wave < BM / 64;
  unsigned s_off;
  const float* s_base;
  const long long s_step = of_x ? p.x_scale_col : p.w_scale_col;
  auto set_tile = [&](int at) __attribute__((always_inline)) {
    const TileId tile = xcd_tile_of(at, p.mx, p.ny, 1, p.by_group);
    m0 = p.lo + (long long)tile.m * BM;
    n0 = tile.n * BN;
    xbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.x + m0 * p.x_stride), 0, 0x7fffffff, 0x00020000);
    wbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.w + n0 * p.w_stride), 0, 0x7fffffff, 0x00020000);
#pragma unroll
    for (int i = 0; i < A_LD; ++i) {
      const int row = row8 + NW * 8 * i;
      a_off[i] = m0 + row < p.hi ? (unsigned)(row * (int)p.x_stride + a_chunk * 16) : kOut;
    }
#pragma unroll
    for (int i = 0; i < B_LD; ++i) {
      const int row = row8 + NW * 8 * i;
      b_off[i] = n0 + row < p.n ? (unsigned)(row * (int)p.w_stride + b_chunk[i] * 16) : kOut;
    }
    if (of_x) s_off = m0 + wave * 64 + lane < p.hi ? (unsigned)((wave * 64 + lane) * (int)p.x_scale_row * 4) : kOut;
    else s_off = lane < (BN + kBlock - 1) / kBlock && n0 + lane * kBlock < p.n ? (unsigned)(lane * (int)p.w_scale_row * 4) : kOut;
    s_base = of_x ? p.x_scale + m0 * p.x_scale_row : p.w_scale + n0 / kBlock * p.w_scale_row;
  };

  auto issue = [&](int s, int j) __attribute__((always_inline)) {   // load instruction j of stage s
    unsigned char* const dst = mine + (s & 1) * STAGE;
    const int block = s * KG + group, chunks = (p.k - block * kBlock) / 16;   // (of this block, or more)
    if (j < A_LD) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(xbuf, (__attribute__((address_space(3))) void*)(dst + (wave + NW * j) * 1024), 16,
                                               (int)(a_chunk >= chunks ? kOut : a_off[j]), block * kBlock, 0, 0);
    } else if (j < A_LD + B_LD) {
      const int i = j - A_LD;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(wbuf, (__attribute__((address_space(3))) void*)(dst + A_BYTES + (wave + NW * i) * 1024), 16,
                                               (int)(b_chunk[i] >= chunks ? kOut : b_off[i]), block * kBlock, 0, 0);
    } else {
      const __amdgpu_buffer_rsrc_t sbuf =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(s_base + block * s_step), 0, 0x7fffffff, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(sbuf, (__attribute__((address_space(3))) void*)(dst + S_AT + wave * 256), 4, (int)(KG > 1 && chunks <= 0 ? kOut : s_off), 0, 0, 0);
    }
  };
  auto issue_mid = [&](int s, int j) __attribute__((always_inline)) {   // (halves: load instructions 0, 2, .. of the weights are first halves)
    issue(s, j < A_LD ? j : j < MID - 1 ? A_LD + 2 * (j - A_LD) : LPS - 1);
  };
  auto issue_end = [&](int s, int j) __attribute__((always_inline)) { issue(s, HALVES ? A_LD + 2 * j + 1 : j); };
  auto barrier = [&]() __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  const unsigned lds0 = (unsigned)(unsigned long)(__attribute__((address_space(3))) unsigned char*)mine;
  const int r16 = lane & 15, g = lane >> 4;
  // operands: chunks g and g + 4 of a row
  const unsigned a_at = lds0 + (unsigned)((wm * TM * 16 + r16) * 128 + ((g ^ (r16 >> 1)) & 7) * 16);
  const int wrow = 16 * (r16 >> 2) + (r16 & 3);
  const unsigned b_at = lds0 + (unsigned)(A_BYTES + (wn * TN * 16 + wrow) * 128 + ((g ^ (((r16 >> 1) & 1) | (r16 >> 2) << 1)) & 7) * 16);
  const unsigned sx_at = lds0 + (unsigned)(S_AT + (wm * TM * 16 + r16) * 4);
  const unsigned sw_at = lds0 + (unsigned)(S_AT + BM * 4 + (wn * TN * 16 / kBlock) * 4);

  u32x4 fx[TM][2], fw[2][2];
  float sx[TM], sw;
  // (what an asm names in a lambda of its own type of argument is not captured by that: hence the references)
  auto read_x = [&](unsigned at, auto i) __attribute__((always_inline)) {
    u32x4(&f)[2] = fx[i];
    float& scale = sx[i];
    const unsigned a0 = a_at + at, a1 = a0 ^ 64u, as = sx_at + at;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f[0]) : "v"(a0), "n"(i * 2048) : "memory");
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f[1]) : "v"(a1), "n"(i * 2048) : "memory");
    asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(scale) : "v"(as), "n"(i * 64) : "memory");
  };
  auto read_w = [&](unsigned at, auto t, u32x4 (&f)[2]) __attribute__((always_inline)) {
    constexpr int off = (t / 4) * 64 * 128 + (t % 4) * 4 * 128;
    const unsigned a0 = b_at + at, a1 = a0 ^ 64u;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f[0]) : "v"(a0), "n"(off) : "memory");
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(f[1]) : "v"(a1), "n"(off) : "memory");
  };
  auto read_scale = [&](unsigned at) __attribute__((always_inline)) {
    asm volatile("ds_read_b32 %0, %1" : "=v"(sw) : "v"(sw_at + at) : "memory");
  };
  auto wait_w = [&](u32x4 (&f)[2]) __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1])::"memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto wait_w2 = [&](u32x4 (&f)[2]) __attribute__((always_inline)) {   // the two reads behind it may be on their way
    asm volatile("s_waitcnt lgkmcnt(2)" : "+v"(f[0]), "+v"(f[1])::"memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  auto wait_all = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(fw[0][0]), "+v"(fw[0][1]), "+v"(fw[1][0]), "+v"(fw[1][1]), "+v"(sw)::"memory");
#pragma unroll
    for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(fx[i][0]), "+v"(fx[i][1]), "+v"(sx[i]));
    __builtin_amdgcn_sched_barrier(0);
  };

  f32x4 acc[TN][TM], part[TM];
  float by[TM];
  auto add = [&](auto t, auto i) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[t][i][e] = fmaf(part[i][e], by[i], acc[t][i][e]);
  };
  // One stage; `next`: another follows, `refill`: and one after that. MORE: stores that are younger than the loads it waits for in its middle,
  // and MORE_END at its end. (Memory instructions of a wavefront finish in order.)
  auto stage = [&](int s, bool next, bool refill, auto MORE, auto MORE_END) __attribute__((always_inline)) {
    const unsigned at = (unsigned)((s & 1) * STAGE), after = (unsigned)(STAGE - (s & 1) * STAGE);
    Op ox[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      ox[i].set(fx[i][0], fx[i][1]);
      by[i] = sx[i] * sw;
    }
    unroll<TN>([&](auto t) __attribute__((always_inline)) {
      constexpr bool last = t == TN - 1, before_last = t == TN - 2, middle = HALVES && t == TN / 2 - 2;
      Op ow;
      ow.set(fw[t & 1][0], fw[t & 1][1]);
      unroll<TM>([&](auto i) __attribute__((always_inline)) {
        if constexpr (t > 0) add(std::integral_constant<int, t - 1>{}, i);
        part[i] = Op::product(ow, ox[i]);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (last) {
          if (next) read_x(after, i);
          if (refill)
#pragma unroll
            for (int j = i * END / TM; j < (i + 1) * END / TM; ++j) issue_end(s + 2, j);
          __builtin_amdgcn_sched_barrier(0);
        } else if constexpr (HALVES && t == TN / 2 - 1) {
          if (refill)
#pragma unroll
            for (int j = i * MID / TM; j < (i + 1) * MID / TM; ++j) issue_mid(s + 2, j);
          __builtin_amdgcn_sched_barrier(0);
        }
      });
      // the weight tile after the next into the registers of this one
      if constexpr (middle) {
        wait_w(fw[(t + 1) & 1]);
        if (next) __builtin_amdgcn_s_waitcnt(vmcnt_imm(MID + END + MORE));
        else __builtin_amdgcn_s_waitcnt(vmcnt_imm(MORE));
        barrier();
        read_w(at, std::integral_constant<int, t + 2>{}, fw[t & 1]);
      } else if constexpr (before_last) {
        wait_w(fw[(t + 1) & 1]);
        if (next) {
          if (HALVES && refill) __builtin_amdgcn_s_waitcnt(vmcnt_imm(MID + END + MORE_END));
          else __builtin_amdgcn_s_waitcnt(vmcnt_imm(HALVES ? END + MORE_END : 0));
          barrier();
          read_w(after, std::integral_constant<int, 0>{}, fw[t & 1]);
          read_scale(after);
        }
      } else if constexpr (last) {
        if (next) read_w(after, std::integral_constant<int, 1>{}, fw[t & 1]);
      } else {
        read_w(at, std::integral_constant<int, t + 2>{}, fw[t & 1]);
        wait_w2(fw[(t + 1) & 1]);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    unroll<TM>([&](auto i) __attribute__((always_inline)) { add(std::integral_constant<int, TN - 1>{}, i); });
    if (next) wait_all();
  };
  static_assert(TN % 2 == 0, "a stage begins with the first set of weights");

  auto start = [&]() __attribute__((always_inline)) {   // a tile's first loads
    for (int s = 0; s < 2 && s < ns; ++s) {
#pragma unroll
      for (int j = 0; j < MID; ++j) issue_mid(s, j);
#pragma unroll
      for (int j = 0; j < END; ++j) issue_end(s, j);
    }
  };
  const Clamp cl = make_clamp(p.act);
  constexpr int STORES = TM * TN / 4 * E;   // of a tile: 16 values of a lane for four weight tiles
  static_assert(!HALVES || LPS + END + STORES < 64, "the counter's range");
  constexpr std::integral_constant<int, 0> none{};
  constexpr std::integral_constant<int, HALVES ? STORES : 0> stores{};
  int launch = blockIdx.x;
  bool behind = false;   // STORES stores are younger than the tile's first loads
  set_tile(launch);
  start();
  for (;;) {
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
      for (int b = 0; b < TM; ++b) acc[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (behind) {   // (two stages at least)
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(HALVES ? END + LPS + STORES : 0));
    } else if (ns > 1) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(HALVES ? END + LPS : LPS));
    } else {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(HALVES ? END : 0));
    }
    barrier();
    unroll<TM>([&](auto i) __attribute__((always_inline)) { read_x(0u, i); });
    read_w(0u, std::integral_constant<int, 0>{}, fw[0]);
    read_w(0u, std::integral_constant<int, 1>{}, fw[1]);
    read_scale(0u);
    wait_all();
    int s = 0;
    if (HALVES && behind) {
      stage(0, true, true, stores, stores);
      stage(1, true, true, stores, none);
      s = 2;
    }
    for (; s + 2 < ns; ++s) stage(s, true, true, none, none);
    for (; s + 1 < ns; ++s) stage(s, true, false, none, none);
    stage(s, false, false, none, none);

    if constexpr (KG > 1) {
      static_assert(KG == 2 && TN * TM * NW * 1024 <= KG * 2 * STAGE, "LDS");
      f32x4* const sums = (f32x4*)smem + wave * 64 + lane;
      __syncthreads();
#pragma unroll
      for (int u = 0; u < TN * TM; ++u)
        if (group == 1) sums[u * NW * 64] = acc[u / TM][u % TM];
      __syncthreads();
#pragma unroll
      for (int u = 0; u < TN * TM; ++u)
        if (group == 0) acc[u / TM][u % TM] += sums[u * NW * 64];
    }
    // The sums leave: y (and residual) are buffers that begin at the tile, what lies outside goes nowhere.
    const bool alone = !p.res && !p.bias;
    const int rows_left = group == 0 ? (int)min(p.hi - m0, (long long)BM) : 0, n_left = min(p.n - n0, BN), n_at = n0;
    const __amdgpu_buffer_rsrc_t ybuf = __builtin_amdgcn_make_buffer_rsrc(p.y + m0 * p.y_stride + (long long)n0 * E, 0, 0x7fffffff, 0x00020000);
    const __amdgpu_buffer_rsrc_t rbuf =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.res + m0 * p.res_stride + (long long)n0 * E), 0, 0x7fffffff, 0x00020000);
    launch += gridDim.x;
    const bool more = launch < p.mx * p.ny;
    auto go_on = [&]() __attribute__((always_inline)) {   // (no wavefront reads the last stages any more)
      barrier();
      set_tile(launch);
      start();
    };
    auto leave = [&](auto with_more) __attribute__((always_inline)) {   // with_more: bias or residual
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int row = wm * TM * 16 + i * 16 + r16;
#pragma unroll
        for (int t = 0; t < TN; t += 4) {
#pragma unroll
          for (int c = 0; c < 16; c += VE) {
            const int n = wn * TN * 16 + t * 16 + g * 16 + c;
            const bool ok = row < rows_left && n < n_left;
            alignas(16) T o[VE];
            float v[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) v[e] = acc[t + (c + e) / 4][i][e % 4];
            if constexpr (with_more) {
              if (p.bias && ok)
#pragma unroll
                for (int e = 0; e < VE; ++e) v[e] += p.bias[n_at + n + e];
              if (p.res) {
                *(u32x4*)o = __builtin_amdgcn_raw_buffer_load_b128(rbuf, (int)(ok ? (unsigned)(row * (int)p.res_stride + n * E) : kOut), 0, 0);
#pragma unroll
                for (int e = 0; e < VE; ++e) v[e] += to_f32(o[e]);
              }
            }
#pragma unroll
            for (int e = 0; e < VE; ++e) o[e] = from_f32<T>(clamp_keeping_nan(v[e], cl));
            __builtin_amdgcn_raw_buffer_store_b128(*(const u32x4*)o, ybuf, (int)(ok ? (unsigned)(row * (int)p.y_stride + n * E) : kOut), 0, 0);
          }
        }
      }
    };
    behind = false;
    if (p.vectors && alone) {
      behind = more && HALVES && ns >= 4;
      if (more) go_on();
      leave(std::false_type{});
    } else if (p.vectors) {
      leave(std::true_type{});
      if (more) go_on();
    } else {
      // Rows that do not begin on 16 bytes: through LDS, 16 rows of a wavefront at a time, so that a store's lanes are neighbouring outputs.
      constexpr int PITCH = TN * 16 + 4;
      static_assert(KG * NW * 16 * PITCH * 4 <= KG * 2 * STAGE, "LDS");
      __syncthreads();
      float* const to = (float*)smem + (group * NW + wave) * 16 * PITCH;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int t = 0; t < TN; ++t) *(f32x4*)(to + r16 * PITCH + (t / 4) * 64 + g * 16 + (t % 4) * 4) = acc[t][i];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 1
        for (int u = 0; u < 2 * (TN / 4); ++u) {   // eight rows of 64 outputs; bias and residual first: one wait for all of them
          const int c = u / 2 * 64 + lane, n = wn * TN * 16 + c, r0 = u % 2 * 8, row0 = wm * TM * 16 + i * 16 + r0;
          const bool in = n < n_left;
          const float bias = p.bias && in ? p.bias[n_at + n] : 0.f;
          float add[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) add[r] = 0.f;
          if (p.res)
#pragma unroll
            for (int r = 0; r < 8; ++r) {
              const int at = (int)(in && row0 + r < rows_left ? (unsigned)((row0 + r) * (int)p.res_stride + n * E) : kOut);
              if constexpr (E == 2) add[r] = to_f32(__builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(rbuf, at, 0, 0)));
              else add[r] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rbuf, at, 0, 0));
            }
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const T o = from_f32<T>(clamp_keeping_nan(to[(r0 + r) * PITCH + c] + bias + add[r], cl));
            const int at = (int)(in && row0 + r < rows_left ? (unsigned)((row0 + r) * (int)p.y_stride + n * E) : kOut);
            if constexpr (E == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, o), ybuf, at, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, o), ybuf, at, 0, 0);
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
      if (more) go_on();
    }
    if (!more) return;
  }
}

// Few matrix rows, or few tiles: the weights are read once and what counts is to have many loads on their way. A workgroup has TM x TN tiles of
// 16 x 16; its NW wavefronts take every NW-th block of columns each, straight from memory into operands, a block ahead, and their
// sums are added in LDS in the order of the wavefronts.
template <typename T, int TM, int TN, int NW>
__global__ __launch_bounds__(64 * NW) void rowwise_f8_few_kernel(const F8Params p) {
  typedef Operand<typename MulType<T>::type> Op;
  __shared__ f32x4 sums[NW][TN * TM][64];
  const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const TileId tile = xcd_tile_of(blockIdx.x, p.mx, p.ny, 1, p.by_group);
  const long long m0 = p.lo + (long long)tile.m * (TM * 16);
  const int n0 = tile.n * (TN * 16), ns = (p.k + kBlock - 1) / kBlock;
  const __amdgpu_buffer_rsrc_t xbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.x + m0 * p.x_stride), 0, 0x7fffffff, 0x00020000);
  const __amdgpu_buffer_rsrc_t wbuf = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(p.w + n0 * p.w_stride), 0, 0x7fffffff, 0x00020000);
  unsigned a_off[TM], b_off[TN];
  const float* sx_at[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const bool live = m0 + i * 16 + r16 < p.hi;
    a_off[i] = live ? (unsigned)((i * 16 + r16) * (int)p.x_stride + g * 16) : kOut;
    sx_at[i] = p.x_scale + (live ? m0 + i * 16 + r16 : m0) * p.x_scale_row;
  }
#pragma unroll
  for (int t = 0; t < TN; ++t) b_off[t] = n0 + t * 16 + r16 < p.n ? (unsigned)((t * 16 + r16) * (int)p.w_stride + g * 16) : kOut;
  const float* const sw_at = p.w_scale + n0 / kBlock * p.w_scale_row;

  struct Block { u32x4 x[TM][2], w[TN][2]; float sx[TM], sw; };
  auto load = [&](int s, Block& b) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool past = s * kBlock + (g + 4 * h) * 16 >= p.k;
#pragma unroll
      for (int t = 0; t < TN; ++t) b.w[t][h] = __builtin_amdgcn_raw_buffer_load_b128(wbuf, (int)(past || b_off[t] == kOut ? kOut : b_off[t] + h * 64), s * kBlock, 0);
#pragma unroll
      for (int i = 0; i < TM; ++i) b.x[i][h] = __builtin_amdgcn_raw_buffer_load_b128(xbuf, (int)(past || a_off[i] == kOut ? kOut : a_off[i] + h * 64), s * kBlock, 0);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) b.sx[i] = sx_at[i][s * p.x_scale_col];
    b.sw = sw_at[s * p.w_scale_col];
  };
  f32x4 acc[TN][TM];
#pragma unroll
  for (int t = 0; t < TN; ++t)
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const Block& b) __attribute__((always_inline)) {
    Op ox[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) ox[i].set(b.x[i][0], b.x[i][1]);
#pragma unroll
    for (int t = 0; t < TN; ++t) {
      Op ow;
      ow.set(b.w[t][0], b.w[t][1]);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const f32x4 part = Op::product(ow, ox[i]);
        const float by = b.sx[i] * b.sw;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][i][e] = fmaf(part[e], by, acc[t][i][e]);
      }
    }
  };
  int s = wave;
  if (s < ns) {
    Block a, b;
    load(s, a);
    for (;;) {
      if (s + NW >= ns) { multiply(a); break; }
      load(s + NW, b);
      multiply(a);
      s += NW;
      if (s + NW >= ns) { multiply(b); break; }
      load(s + NW, a);
      multiply(b);
      s += NW;
    }
  }
#pragma unroll
  for (int t = 0; t < TN; ++t)
#pragma unroll
    for (int i = 0; i < TM; ++i) sums[wave][t * TM + i][lane] = acc[t][i];
  __syncthreads();
  const Clamp cl = make_clamp(p.act);
  for (int u = wave; u < TN * TM; u += NW) {
    const int t = u / TM, i = u % TM;
    f32x4 v = sums[0][u][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) v += sums[w][u][lane];
    const long long m = m0 + i * 16 + r16;
    if (m < p.hi) put_four<T>(p, v, m, n0 + t * 16 + g * 4, cl);
  }
}

// Which kernel: the one that is estimated to be done first. Time of a launch, us = start + rounds * (each + blocks of columns * step), where a round is a
// workgroup (128 x 128: two) on every compute unit. Fitted to 217 products of 1 to 16384 rows, 256 to 8192 columns and 128 to 16384 outputs that were timed
// with every kernel: the chosen one is the fastest to 0.2 % in the mean, to 7 % at worst. Measured, us, bf16, 4096 columns: 48 rows to 4096 outputs 9.8 (32 x 32;
// 12.9 with 16 x 32, 13.9 with 32 x 64), 96 rows 14.0 (32 x 64; 18.1 with 64 x 128, 24.5 with 128 x 128), 512 rows 20.0 (64 x 128; 25.4 with 128 x 128, 45.7 with
// 32 x 64), 2048 rows 42 (128 x 128; 58.8 with 256 x 256, 87.6 with 64 x 128) and 4096 rows 69 (256 x 256; 80 with 128 x 128). Of few columns the stores are
// most of it: 256 columns, 10228 rows to 2983 outputs take 40 with 128 x 128, 47 with 256 x 256, 110 with 32 x 64, 135 with 64 x 128.
constexpr int kCus = 256;
int choose(long long m, long long n, int k, bool f32) {
  struct Shape { int bm, bn; double start, each, step, step_f32; };
  static constexpr Shape shapes[] = {{16, 32, 1.1, 0.4, 0.15, 0.17}, {32, 32, 0.3, 0.9, 0.28, 0.30}, {32, 64, 2.1, 0.4, 0.35, 0.36},
                                     {64, 128, 2.4, 3.1, 0.50, 0.96}, {128, 128, 3.6, 2.7, 1.32, 2.13}, {256, 256, 8.0, 5.2, 1.8, 0.0}};
  const double blocks = (double)ceil_div(k, kBlock);
  int best = 0;
  double least = 0.0;
  for (int i = 0; i < (f32 ? 5 : 6); ++i) {
    const Shape& s = shapes[i];
    const double groups = (double)ceil_div(m, s.bm) * (double)ceil_div(n, s.bn), step = f32 ? s.step_f32 : s.step;
    double rounds = std::ceil(groups / kCus);
    if (i == 4) {   // two to a unit: a last single one takes 0.6 of the time of two
      const double pairs = std::floor(rounds / 2);
      rounds = pairs + (rounds > 2 * pairs ? 0.6 : 0.0);
    }
    const double time = s.start + rounds * (s.each + blocks * step);
    if (i == 0 || time < least) { best = i; least = time; }
  }
  return best;
}

struct Kernel {
  void (*run)(const F8Params);
  const char* name;   // of the instance, with %s for the type of its results
  int bm, bn, threads;
  long long most;     // workgroups
};
template <typename T>
Kernel kernel_of(long long m, long long n, int k) {
  constexpr long long all = 1LL << 31;
  switch (choose(m, n, k, sizeof(T) == 4)) {
    case 0: return {rowwise_f8_few_kernel<T, 1, 2, 8>, "rowwise_f8_few_kernel<%s, 1, 2, 8>", 16, 32, 512, all};
    case 1: return {rowwise_f8_few_kernel<T, 2, 2, 8>, "rowwise_f8_few_kernel<%s, 2, 2, 8>", 32, 32, 512, all};
    case 2: return {rowwise_f8_few_kernel<T, 2, 4, 4>, "rowwise_f8_few_kernel<%s, 2, 4, 4>", 32, 64, 256, all};
    case 3: return {rowwise_f8_kernel<T, 64, 128, 1, 2, 2>, "rowwise_f8_kernel<%s, 64, 128, 1, 2, 2>", 64, 128, 256, all};
    case 4: break;
    default:   // (not chosen for fp32)
      if constexpr (sizeof(T) == 2) return {rowwise_f8_kernel<T, 256, 256, 4, 2, 1>, "rowwise_f8_kernel<%s, 256, 256, 4, 2, 1>", 256, 256, 512, kCus};
  }
  return {rowwise_f8_kernel<T, 128, 128, 2, 2, 1>, "rowwise_f8_kernel<%s, 128, 128, 2, 2, 1>", 128, 128, 256, all};
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
  p.vectors = bits % 16 == 0 && op->n % (16 / E) == 0;
  const int rows_in = rows.hi - rows.lo;
  const Kernel kernel = kernel_of<T>(rows_in, op->n, op->k);
  const long long mx = ceil_div(rows_in, kernel.bm), ny = ceil_div(op->n, kernel.bn);
  if (mx * ny > launch_blocks(kernel.threads) || ny > 65535) return LOP_ERR_UNSUPPORTED;
  p.mx = (int)mx; p.ny = (int)ny;
  p.by_group = make_fastdiv(kGroupM * p.ny);
  LOP_HIP(launch_kernel(kernel.run, dim3((unsigned)std::min(mx * ny, kernel.most)), dim3(kernel.threads), stream, nullptr, p));
  return LOP_OK;
}

int check_sizes(const lop_rowwise_f8_t* op, lop_rows_t rows) {
  if (!op || op->m < 0 || op->n < 1 || op->k < 1) return LOP_ERR_INVALID_ARG;
  if (!known_dtype(op->dtype) || op->k % 16 || op->act < LOP_ACT_NONE || op->act > LOP_ACT_RELU6) return LOP_ERR_UNSUPPORTED;
  return check_band(rows, op->m);
}

}  // namespace
}  // namespace lop

extern "C" int lop_rowwise_f8(const lop_rowwise_f8_t* op, lop_rows_t rows, void* stream) {
  using namespace lop;
  if (const int e = check_sizes(op, rows)) return e;
  if (rows.lo == rows.hi) return LOP_OK;
  const size_t E = dtype_bytes(op->dtype);
  if (!op->x || !op->w || !op->x_scale || !op->w_scale || !op->y || !aligned16(op->x) || !aligned16(op->w)) return LOP_ERR_INVALID_ARG;
  if (((uintptr_t)op->x_scale | (uintptr_t)op->w_scale | (uintptr_t)op->bias) & 3) return LOP_ERR_INVALID_ARG;
  if (((uintptr_t)op->y | (uintptr_t)op->residual) & (E - 1)) return LOP_ERR_INVALID_ARG;
  if (!apart(op->y_stride, op->n, op->m)) return LOP_ERR_INVALID_ARG;
  if (!whole_vectors(op->x_stride, 1, op->m > 1) || !whole_vectors(op->w_stride, 1, op->n > 1)) return LOP_ERR_INVALID_ARG;
  if (op->x_scale_row < 0 || op->x_scale_col < 0 || op->w_scale_row < 0 || op->w_scale_col < 0 || op->y_stride < 0 ||
      (op->residual && op->residual_stride < 0))
    return LOP_ERR_INVALID_ARG;
  // (offsets within a tile of at most 256 rows are 32 bits)
  constexpr long long far = (1LL << 31) / 256 - 1;
  if ((op->m > 1 && (op->y_stride + op->n) * (long long)E > far) || (op->m > 1 && op->residual && (op->residual_stride + op->n) * (long long)E > far) ||
      (long long)op->n * (long long)E > far)
    return LOP_ERR_UNSUPPORTED;
  if ((op->m > 1 && op->x_stride + op->k > far) || (op->n > 1 && op->w_stride + op->k > far) || (op->m > 1 && op->x_scale_row > far / 4) ||
      (op->n > kBlock && op->w_scale_row > far / 4) || op->k > far)
    return LOP_ERR_UNSUPPORTED;
  return op->dtype == LOP_BF16 ? rowwise_f8<__bf16>(op, rows, (hipStream_t)stream) : rowwise_f8<float>(op, rows, (hipStream_t)stream);
}

extern "C" int lop_rowwise_f8_kernel(const lop_rowwise_f8_t* op, lop_rows_t rows, char* name, size_t size) {
  using namespace lop;
  if (!name || size == 0) return LOP_ERR_INVALID_ARG;
  name[0] = 0;
  if (const int e = check_sizes(op, rows)) return e;
  const int m = rows.hi - rows.lo;
  if (m == 0) return LOP_OK;
  if (op->dtype == LOP_BF16) snprintf(name, size, kernel_of<__bf16>(m, op->n, op->k).name, "__bf16");
  else snprintf(name, size, kernel_of<float>(m, op->n, op->k).name, "float");
  return LOP_OK;
}
