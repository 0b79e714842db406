// Queries and keys normalized for each head and rotated by their positions (lop_head_norm_rope): element-wise but for a sum over
// a head, one pass over the data.
//
//   y = x * rsqrt(mean(x^2) + eps) * weight,   (a, b) -> amplitude * (a cos t - b sin t, a sin t + b cos t),   t = position * freq[pair]
//
// A lane holds two groups of four consecutive values that need no other lane's: of neighbouring pairs two groups side by side, of
// pairs half the rotated part apart the same place in both halves; what is not rotated follows eight by eight. A head is 8, 16 or 32 lanes, and the
// cosines of a lane's four pairs serve every head of its token that the wavefront goes through: they cost as much as several
// heads, since far positions need their angle reduced in 64 bits. Bound by memory: 16384 tokens of 40 heads of 128 values take 68 us in bf16
// (4.9 TB/s), 118 us in fp32 (5.7 TB/s); one token 3 us, which a launch in a graph and three loads one after the other take.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "launch.hpp"
#include "lop.h"
#include "op_check.hpp"

namespace lop {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct RopeParams {
  const char *q, *k;
  char *q_out, *k_out;
  long long q_token, q_head, k_token, k_head, q_out_token, q_out_head, k_out_token, k_out_head;   // bytes
  const float *q_weight, *k_weight, *freq;
  const int* positions;
  int lo, hi, heads_q, heads_k, head_dim, rot_dim, interleaved;
  int parts, per_part;   // wavefronts a token's heads are dealt to, heads of each
  float eps, amplitude, by_dim;
};

template <typename T> struct Four;
template <> struct Four<__bf16> {
  typedef u32x2 raw;
  static __device__ __forceinline__ void get(const raw& a, float (&v)[4]) {
    v[0] = __uint_as_float(a[0] << 16); v[1] = __uint_as_float(a[0] & 0xffff0000u);
    v[2] = __uint_as_float(a[1] << 16); v[3] = __uint_as_float(a[1] & 0xffff0000u);
  }
  static __device__ __forceinline__ raw put(const float (&v)[4]) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(u32x2, bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]});
  }
};
template <> struct Four<float> {
  typedef f32x4 raw;
  static __device__ __forceinline__ void get(const raw& a, float (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i];
  }
  static __device__ __forceinline__ raw put(const float (&v)[4]) { return f32x4{v[0], v[1], v[2], v[3]}; }
};

// LANES: lanes of a head, the power of two from head_dim / 8 on.
template <typename T, int LANES>
__global__ __launch_bounds__(256) void head_norm_rope_kernel(const RopeParams p) {
  typedef typename Four<T>::raw raw;
  constexpr int SIDE = 64 / LANES;   // heads side by side
  const int lane = threadIdx.x & 63, j = lane % LANES, side = lane / LANES;
  const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long long token = p.lo + wave / p.parts;
  const int part = (int)(wave % p.parts);
  if (token >= p.hi) return;   // (no barrier follows)
  const bool live = j * 8 < p.head_dim;
  const bool turns = j * 8 < p.rot_dim;
  // where the lane's two groups lie, and the pair of each of the four products
  const bool halves = turns && !p.interleaved;
  const int a_at = live ? (halves ? 4 * j : 8 * j) : 0, b_at = live ? (halves ? p.rot_dim / 2 + 4 * j : 8 * j + 4) : 0;
  float c[4], s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) { c[i] = 1.f; s[i] = 0.f; }
  if (turns) {
    // in turns: the whole ones leave before the angle is rounded to 32 bits
    const double position = (double)p.positions[token] * 0.15915494309189533577;   // 1 / (2 pi)
    const f32x4 f = *(const f32x4*)(p.freq + 4 * j);   // interleaved: pairs 4j .. 4j + 3, too
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double t = position * (double)f[i];
      float si, co;
      sincospif(2.f * (float)(t - rint(t)), &si, &co);
      c[i] = co * p.amplitude;
      s[i] = si * p.amplitude;
    }
  }
  f32x4 wq[2], wk[2];
  wq[0] = wq[1] = wk[0] = wk[1] = f32x4{1.f, 1.f, 1.f, 1.f};
  if (live && p.q_weight) { wq[0] = *(const f32x4*)(p.q_weight + a_at); wq[1] = *(const f32x4*)(p.q_weight + b_at); }
  if (live && p.k_weight && p.heads_k) { wk[0] = *(const f32x4*)(p.k_weight + a_at); wk[1] = *(const f32x4*)(p.k_weight + b_at); }

  const int heads = p.heads_q + p.heads_k, last = min(heads, (part + 1) * p.per_part);
  for (int h = part * p.per_part + side; h < last; h += SIDE) {   // (the lanes of a head go together)
    const bool here = live, is_k = h >= p.heads_q;
    const int n = is_k ? h - p.heads_q : h;
    const char* const x = is_k ? p.k + token * p.k_token + n * p.k_head : p.q + token * p.q_token + n * p.q_head;
    float a[4] = {0.f, 0.f, 0.f, 0.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
    if (here) {
      Four<T>::get(*(const raw*)(x + a_at * (int)sizeof(T)), a);
      Four<T>::get(*(const raw*)(x + b_at * (int)sizeof(T)), b);
    }
    if (is_k ? p.k_weight != nullptr : p.q_weight != nullptr) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += a[i] * a[i] + b[i] * b[i];
#pragma unroll
      for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d, 64);
      float mean = sum * p.by_dim + p.eps, by = 1.f;
      if (!(mean >= 0x1p-100f && mean <= 0x1p120f)) {   // values beyond 2^60 or below 2^-50, whose squares fp32 does not hold: of the values times a power of two
        by = mean < 1.f ? 0x1p70f : 0x1p-70f;           // (in a loop of its own for such heads: 80 registers, prompts 99 us instead of 70)
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += (a[i] * by) * (a[i] * by) + (b[i] * by) * (b[i] * by);
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) sum += __shfl_xor(sum, d, 64);
        mean = sum * p.by_dim + p.eps * by * by;
      }
      const float r = by / sqrtf(mean);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] *= r * (is_k ? wk[0][i] : wq[0][i]);
        b[i] *= r * (is_k ? wk[1][i] : wq[1][i]);
      }
    }
    float u[4], v[4];
    if (p.interleaved) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        u[2 * i] = a[2 * i] * c[i] - a[2 * i + 1] * s[i];
        u[2 * i + 1] = a[2 * i] * s[i] + a[2 * i + 1] * c[i];
        v[2 * i] = b[2 * i] * c[2 + i] - b[2 * i + 1] * s[2 + i];
        v[2 * i + 1] = b[2 * i] * s[2 + i] + b[2 * i + 1] * c[2 + i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u[i] = a[i] * c[i] - b[i] * s[i];
        v[i] = a[i] * s[i] + b[i] * c[i];
      }
    }
    if (!turns) {   // (not by way of cosines of 1 and sines of 0: an infinity beside a value is no part of it)
#pragma unroll
      for (int i = 0; i < 4; ++i) { u[i] = a[i]; v[i] = b[i]; }
    }
    if (here) {
      char* const y = is_k ? p.k_out + token * p.k_out_token + n * p.k_out_head : p.q_out + token * p.q_out_token + n * p.q_out_head;
      *(raw*)(y + a_at * (int)sizeof(T)) = Four<T>::put(u);
      *(raw*)(y + b_at * (int)sizeof(T)) = Four<T>::put(v);
    }
  }
}

template <typename T>
int rope(const lop_head_norm_rope_t* op, lop_rows_t rows, hipStream_t stream) {
  constexpr long long E = sizeof(T);
  RopeParams p;
  p.q = (const char*)op->q; p.k = (const char*)op->k; p.q_out = (char*)op->q_out; p.k_out = (char*)op->k_out;
  p.q_token = op->q_token * E; p.q_head = op->q_head * E; p.k_token = op->k_token * E; p.k_head = op->k_head * E;
  p.q_out_token = op->q_out_token * E; p.q_out_head = op->q_out_head * E;
  p.k_out_token = op->k_out_token * E; p.k_out_head = op->k_out_head * E;
  p.q_weight = op->q_weight; p.k_weight = op->k_weight; p.freq = op->freq; p.positions = op->positions;
  p.lo = rows.lo; p.hi = rows.hi;
  p.heads_q = op->heads_q; p.heads_k = op->heads_k; p.head_dim = op->head_dim; p.rot_dim = op->rot_dim; p.interleaved = op->interleaved != 0;
  p.eps = op->eps; p.amplitude = op->amplitude; p.by_dim = 1.f / (float)op->head_dim;
  const int lanes = op->head_dim <= 64 ? 8 : op->head_dim <= 128 ? 16 : 32;
  // A round: the heads that lie side by side in a wavefront. Several rounds to a wavefront share its cosines, but take as long as they do: as many as leave
  // 4096 wavefronts, of fp32, whose rounds outlast the cosines of another wavefront, two at most. Measured, us, 40 heads of 128 values (ten rounds), bf16: 64
  // tokens 3.5 with one round and 10.8 with all, 1024 tokens 8.4 with two, 10.0 with one, 15.6 with all, 4096 tokens 21.5 with all, 29 with one, 16384 tokens
  // 68 and 107; of fp32 4096 tokens 34 with two, 35 with one, 39 with all, 16384 tokens 118, 124 and 132.
  const long long tokens = rows.hi - rows.lo;
  const int heads = op->heads_q + op->heads_k, side = 64 / lanes, rounds = (heads + side - 1) / side;
  const int most = E == 4 ? 2 : rounds;
  const int each = (int)std::min<long long>(most, std::max<long long>(1, rounds * tokens / 4096));   // rounds of heads of a wavefront
  p.per_part = each * side;
  p.parts = (rounds + each - 1) / each;
  const long long grid = ceil_div(tokens * p.parts, 4);
  if (grid > launch_blocks(256)) return LOP_ERR_UNSUPPORTED;
  const dim3 g((unsigned)grid), b(256);
  LOP_HIP(lanes == 8    ? launch_kernel(head_norm_rope_kernel<T, 8>, g, b, stream, nullptr, p)
          : lanes == 16 ? launch_kernel(head_norm_rope_kernel<T, 16>, g, b, stream, nullptr, p)
                        : launch_kernel(head_norm_rope_kernel<T, 32>, g, b, stream, nullptr, p));
  return LOP_OK;
}

}  // namespace
}  // namespace lop

extern "C" int lop_head_norm_rope(const lop_head_norm_rope_t* op, lop_rows_t rows, void* stream) {
  using namespace lop;
  if (!op || op->tokens < 0 || op->heads_q < 0 || op->heads_k < 0 || op->heads_q > (1 << 20) || op->heads_k > (1 << 20) ||
      op->heads_q + op->heads_k < 1 || op->head_dim < 1 || op->rot_dim < 0)
    return LOP_ERR_INVALID_ARG;
  if (!known_dtype(op->dtype) || op->head_dim % 8 || op->head_dim > 256 || op->rot_dim % 8) return LOP_ERR_UNSUPPORTED;
  if (op->rot_dim > op->head_dim) return LOP_ERR_SHAPE;
  if (const int e = check_band(rows, op->tokens)) return e;
  if (rows.lo == rows.hi) return LOP_OK;
  const size_t E = dtype_bytes(op->dtype);
  const bool many = op->tokens > 1;
  auto good = [&](const void* p, long long token, long long head, int heads) {
    return heads == 0 || (p && aligned16(p) && whole_vectors(token, E, many) && whole_vectors(head, E, heads > 1));
  };
  if (!good(op->q, op->q_token, op->q_head, op->heads_q) || !good(op->q_out, op->q_out_token, op->q_out_head, op->heads_q) ||
      !good(op->k, op->k_token, op->k_head, op->heads_k) || !good(op->k_out, op->k_out_token, op->k_out_head, op->heads_k))
    return LOP_ERR_INVALID_ARG;
  for (int i = 0; i < 2; ++i)   // an output's heads do not overlap
    if (const int heads = i ? op->heads_k : op->heads_q; heads > 0 && !apart(op->head_dim, i ? op->k_out_token : op->q_out_token, op->tokens,
                                                                            i ? op->k_out_head : op->q_out_head, heads))
      return LOP_ERR_INVALID_ARG;
  if (!aligned16(op->q_weight) || !aligned16(op->k_weight)) return LOP_ERR_INVALID_ARG;
  if (op->rot_dim > 0 && (!op->positions || ((uintptr_t)op->positions & 3) || !op->freq || !aligned16(op->freq))) return LOP_ERR_INVALID_ARG;
  if ((op->q_weight || op->k_weight) && !(op->eps >= 0.f)) return LOP_ERR_INVALID_ARG;
  return op->dtype == LOP_BF16 ? rope<__bf16>(op, rows, (hipStream_t)stream) : rope<float>(op, rows, (hipStream_t)stream);
}
