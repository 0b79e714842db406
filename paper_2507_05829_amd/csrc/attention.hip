// Softmax attention of packed query rows with shared key heads (lop_attention).
//
//   out = sum over j of exp(c s_j - c m) v_j / sum over j of exp(c s_j - c m),   s_j = q . k_j,  m = max s_j,  c = scale
//
// in one pass over the keys: maximum, sum and unnormalized output of the keys so far are kept, and multiplied by exp(c m_old - c m_new)
// where the maximum grows. The query heads that share a key head are rows of one tile, so that its keys and values are read once for all of
// them, of a prompt as of single tokens.
//
// A wavefront holds 32 rows. It computes the scores transposed, keys x rows (k q^T), so that a row is a lane and its
// mirror image 32 lanes on: a maximum over keys is one over registers and one exchange, and the weights lie as the product with the values
// (v^T w^T) wants its second operand, whose order of keys is free as long as both operands have the same. Four
// wavefronts share tiles of KT keys and values, which travel from memory to LDS without passing through registers, one
// tile ahead. Where there are few workgroups the keys are cut into parts, and a second kernel joins their results.
//
// Bound: prompts by the matrix cores and the vector instructions of the weights, which one wavefront's products and the other's weights share a SIMD for: a
// causal prompt of 8192 rows of 32 heads (8 of keys) of 128 bf16 values takes 502 us, 1.09 PFLOP/s (a large library product 1.2), on a slower machine 549. Single rows
// by reading keys and values: 32 rows on caches of 2000 to 8000 keys of 8 heads of 128 bf16 values 149 us, 4.9 TB/s.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "conv_common.hpp"
#include "conv_split.hpp"
#include "launch.hpp"
#include "lop.h"
#include "op_check.hpp"

namespace lop {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr unsigned kOut = 0x80000000u;
constexpr int kRows = 128;            // of a workgroup: 32 for each of four wavefronts
constexpr float kMostOfTile = 4096.f;
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

struct AttnParams {
  const char *q, *k, *v;
  char* out;
  long long q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;   // bytes
  const int *q_offsets, *k_begin, *k_end;
  float* lse;
  float* part;       // of keys cut into parts: [split][row of the band][head][head_dim] of the part's mean, then [..][2] of maximum and sum
  int heads_k, group, head_dim, seqs, rows_q, rows_k, causal;
  int lo, hi;        // the band
  int tile0, tiles;  // of packed rows
  int splits;
  float scale;
};

__device__ __forceinline__ int clamp_to(int v, int most) { return min(max(v, 0), most); }

// Tiles of kRows packed rows (row of the sequence x group + head of the group) are numbered so that sequence i's begin at
// start(i) = floor(q_offsets[i] group / kRows) + i: at least as many numbers as it has tiles, whatever the lengths, and no list to make.
struct Place { int seq, tile; };
__device__ __forceinline__ Place find_tile(const AttnParams& p, int t) {
  const int lane = threadIdx.x & 63;
  auto start = [&](int i) { return (int)((long long)clamp_to(p.q_offsets[i], p.rows_q) * p.group / kRows) + i; };
  int lo = 0, hi = p.seqs;   // the last i with start(i) <= t lies in [lo, hi)
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const int n = __popcll(__ballot(i < hi && start(i) <= t));
    if (n == 0) return Place{-1, 0};   // (only where the first sequence does not begin at row 0)
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const int at = t - start(lo);
  return Place{at < 0 ? -1 : lo, at};
}

// Of 16 lanes, lane i gets value i % 4 of the four that lanes i / 4, i / 4 + 4, + 8 and + 12 point at.
__device__ __forceinline__ u32x2 transposed_read(const unsigned char* at) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at));
}

__device__ __forceinline__ float max_of_halves(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __builtin_elementwise_maximum(__uint_as_float((unsigned)s[0]), __uint_as_float((unsigned)s[1]));
}
__device__ __forceinline__ float sum_of_halves(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float((unsigned)s[0]) + __uint_as_float((unsigned)s[1]);
}

__device__ __forceinline__ bool of_either_half(bool v) {
  const unsigned long long lanes = __ballot(v);
  return (((unsigned)lanes | (unsigned)(lanes >> 32)) >> (threadIdx.x & 31)) & 1;
}

// a product with the sum of products before it, which is none
template <typename T>
__device__ __forceinline__ f32x16 mma_first(const u32x4& a, const u32x4& b) {
  const f32x16 none = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), none, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
    f32x16 s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[0], y[0], none, 0, 0, 0);
#pragma unroll
    for (int i = 1; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[i], s, 0, 0, 0);
    return s;
  }
}

// Scores become weights 2^(c s - m) of a row, which are added to its sum. What the exponents are relative to, m, need not be the maximum: as long as a tile's
// weights add up to no more than kMostOfTile in either lane of a row it stays, and nothing is lost: output and sum are at most that many times too large, which values
// below 2^115 leave room for (of larger ones an output may become infinite, and the row goes through the careful pass). Where they add up to more, as in the first
// tile, the row's m becomes the maximum so far and its output and sum are multiplied. So the maximum is hardly ever formed. (Another row's m stays, and its weights are formed again
// as they were: its bits do not depend on the rows beside it.)
template <int NB, int DT>
__device__ __forceinline__ void to_weights(f32x16 (&s)[NB], const float c, float& m, float& l, f32x16 (&o)[DT]) {
  f32x16 w[NB];
  auto weights = [&](float from) __attribute__((always_inline)) {
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        w[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], c, -from));
        part[i & 3] += w[b][i];
      }
    return (part[0] + part[1]) + (part[2] + part[3]);
  };
  float sum = weights(m);   // (no key so far: m is -infinity, and the sum infinite or a NaN)
  const bool many = !(sum <= kMostOfTile);
  if (__any(many)) {
    const bool grows = of_either_half(many);
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = b ? 0 : 1; i < 16; ++i) top = __builtin_elementwise_maximum(top, s[b][i]);
    const float most = max_of_halves(top) * c, grown = grows ? __builtin_elementwise_maximum(m, most) : m;
    const float by = !grows ? 1.f : m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - grown);
    m = grown;
    l *= by;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] *= by;
    sum = weights(m == -INFINITY ? 0.f : m);
  }
  l += sum;
#pragma unroll
  for (int b = 0; b < NB; ++b) s[b] = w[b];
}

// The same for the careful pass: m is the maximum of the unscaled scores so far, followed at every step, and weights are 2^(c (s - m)). Of scores from 2^31 on c s - m
// is off by a step of m, more than the exponential function's range, where c (s - m) of the maximum is 0. The output is the weighted mean so far and the weights
// are shares of their sum, l, which both lanes of a row have here: values that fp32 holds have a mean that it holds, while their sums may pass its range.
template <int NB, int DT>
__device__ __forceinline__ void to_shares(f32x16 (&s)[NB], const float c, float& m, float& l, f32x16 (&o)[DT]) {
  float top = m;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = __builtin_elementwise_maximum(top, s[b][i]);
  top = max_of_halves(top);
  const float before = m == -INFINITY ? 0.f : l * __builtin_amdgcn_exp2f((m - top) * c), from = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[b][i] = __builtin_amdgcn_exp2f((s[b][i] - from) * c);
      sum += s[b][i];
    }
  m = top;
  l = before + sum_of_halves(sum);
  const float by = l == 0.f ? 0.f : 1.f / l, keep = before * by;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] *= keep;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[b][i] *= by;
}

constexpr int attn_pitch(int bytes) { return bytes <= 128 ? 128 : bytes <= 256 ? 256 : bytes <= 512 ? 512 : 1024; }

// DP: head_dim rounded up to what is computed (a multiple of 32)
template <typename T, int DP>
struct AttnShape {
  static constexpr int E = (int)sizeof(T);
  static constexpr int PITCH = attn_pitch(DP * E);       // bytes of a key in LDS
  static constexpr int CP = PITCH / 16;                  // 16-byte chunks of it
  static constexpr int KT = E == 4 && PITCH >= 512 ? 32 : 64;   // keys of a tile (two workgroups' tiles fit a compute unit up to 128 values)
  static constexpr int BYTES = KT * PITCH;
  static constexpr int LDS = 4 * BYTES;                  // two tiles of keys and of values
  static constexpr int LD = BYTES / 4096;                // load instructions of a wavefront for one tile of either
  static constexpr int KS = DP * E / 32;                 // operands of a row: steps of 16 bytes in either half
  static constexpr int DT = DP / 32;
  static constexpr bool PARTS = E == 4 && DP <= 128;     // (of 256 values the rows' parts alone would take 192 registers)
  static constexpr int PITCH3 = attn_pitch(DP * 2), PART = 32 * PITCH3;   // a tile of 32 keys as three bf16 parts, keys and values
  static_assert(!PARTS || 6 * PART <= LDS, "LDS");
  // where chunk c of key `row` lies: at c ^ key. Keys: 16 lanes read one chunk of 16 keys. Values: 16 lanes read 32 bytes of four
  // keys, two such sets side by side (bf16); 32 lanes read 128 bytes of a key and the others of the fourth key on (fp32).
  static __device__ __forceinline__ int k_key(int row) { return CP == 8 ? (row >> 1) & 7 : row & 15; }
  static __device__ __forceinline__ int v_key(int row) {
    if constexpr (E == 4) return ((row >> 2) & 1) * 8;
    return CP == 8 ? ((row >> 1) & 1) * 4 : (row & 3) * 4;
  }
};

// (Where two workgroups fit the LDS of a compute unit their registers have to, too.)
template <typename T, int DP>
__global__ __launch_bounds__(256, (AttnShape<T, DP>::LDS <= 72 * 1024 ? 2 : 1)) void attention_kernel(const AttnParams p) {
  typedef AttnShape<T, DP> S;
  constexpr int PITCH = S::PITCH, KT = S::KT, NB = KT / 32, LD = S::LD, KS = S::KS, DT = S::DT, E = S::E;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[S::LDS];

  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // The last tiles first: with a causal mask they have the most keys. Key heads fastest: neighbouring workgroups go to different XCDs, whose L2
  // then holds the keys of one head each where there are eight.
  const int head = blockIdx.x % p.heads_k;
  const Place place = find_tile(p, p.tile0 + p.tiles - 1 - blockIdx.x / p.heads_k);
  if (place.seq < 0) return;
  const int q0 = clamp_to(p.q_offsets[place.seq], p.rows_q), nq = clamp_to(p.q_offsets[place.seq + 1], p.rows_q) - q0;
  const int k0 = clamp_to(p.k_begin[place.seq], p.rows_k), nk = max(clamp_to(p.k_end[place.seq], p.rows_k) - k0, 0);
  const long long packed = (long long)max(nq, 0) * p.group, first = (long long)place.tile * kRows;
  if (first >= packed) return;
  const int here = (int)min(packed - first, (long long)kRows);   // rows of this tile
  // this lane's row
  const int in_tile = wave * 32 + (lane & 31);
  const unsigned row = (unsigned)(first + min(in_tile, here - 1));
  const int token = (int)(row / (unsigned)p.group), qh = head * p.group + (int)(row - (unsigned)token * p.group);
  const long long at_row = (long long)q0 + token;
  const bool live = in_tile < here && at_row >= p.lo && at_row < p.hi;
  // (no row of the tile is in the band)
  if (q0 + first / p.group >= p.hi || q0 + (first + here - 1) / p.group < p.lo) return;
  const int sees = p.causal ? min(max(nk - nq + token + 1, 0), nk) : nk;   // keys of this row
  auto row_sees = [&](int r) {   // of the tile's row r (the same in all lanes)
    const int t = (int)((first + min(r, here - 1)) / p.group);
    return p.causal ? min(max(nk - nq + t + 1, 0), nk) : nk;
  };
  const bool busy = wave * 32 < here;
  const int least = row_sees(wave * 32), most = busy ? row_sees(wave * 32 + 31) : 0;
  const int all = row_sees(kRows - 1);
  // tiles of keys, and this workgroup's part of them
  int t0 = 0, t1 = (all + KT - 1) / KT;
  if (p.splits > 1) {
    const int each = (t1 + p.splits - 1) / p.splits;
    t0 = min(blockIdx.y * each, (unsigned)t1);
    t1 = min(t0 + each, t1);
  }

  // ---- the rows' operands: 16 bytes at 32 ks + 16 half
  // ---- and what this lane fetches of a tile
  u32x4 fq[KS];
  unsigned k_off[LD], v_off[LD];
  const char* const qp = p.q + at_row * p.q_token + qh * p.q_head;
  auto get_ready = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int at = ks * 32 + half * 16;
      fq[ks] = u32x4{0u, 0u, 0u, 0u};
      if (live && at < p.head_dim * E) fq[ks] = *(const u32x4*)(qp + at);
    }
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int at = (wave + 4 * i) * 1024 + lane * 16, r = at / PITCH, c = at % PITCH / 16;
      const int ck = c ^ S::k_key(r), cv = c ^ S::v_key(r);
      k_off[i] = ck * 16 < p.head_dim * E ? (unsigned)(r * (int)p.k_token + ck * 16) : kOut;
      v_off[i] = cv * 16 < p.head_dim * E ? (unsigned)(r * (int)p.v_token + cv * 16) : kOut;
    }
  };
  const char* const kp = p.k + (long long)k0 * p.k_token + head * p.k_head;
  const char* const vp = p.v + (long long)k0 * p.v_token + head * p.v_head;
  // (Said to be a scalar: where the compiler keeps it in a vector register, for the lanes' comparisons, every load below becomes a loop over the lanes' buffers.)
  const int row_bytes = __builtin_amdgcn_readfirstlane(p.head_dim * E);
  auto issue = [&](int t, int buf) __attribute__((always_inline)) {   // (keys past the sequence's last arrive as zeros)
    const int left = min(nk - t * KT, KT) - 1;
    const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(kp + (long long)t * KT * p.k_token), 0,
                                                                        left * (int)p.k_token + row_bytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vp + (long long)t * KT * p.v_token), 0,
                                                                        left * (int)p.v_token + row_bytes, 0x00020000);
    unsigned char* const dst = smem + buf * 2 * S::BYTES + wave * 1024;
#pragma unroll
    for (int i = 0; i < LD; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(kb, (__attribute__((address_space(3))) void*)(dst + i * 4096), 16, (int)k_off[i], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < LD; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(vb, (__attribute__((address_space(3))) void*)(dst + S::BYTES + i * 4096), 16, (int)v_off[i], 0, 0, 0);
  };
  auto barrier = [&]() __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // ---- where it reads: chunk 2 ks + half of key lane mod 32; of the values what the operand v^T wants
  const unsigned lds0 = (unsigned)(unsigned long)(__attribute__((address_space(3))) unsigned char*)smem;
  const unsigned k_at = lds0 + (lane & 31) * PITCH + ((half ^ S::k_key(lane & 31)) * 16);
  unsigned v_at;
  if constexpr (E == 2) {
    const int s = lane & 15, key = 4 * half + s / 4;   // (of 16 lanes, see transposed reads below)
    v_at = lds0 + S::BYTES + key * PITCH + ((2 * ((lane >> 4) & 1) + (s & 3) / 2) ^ S::v_key(key)) * 16 + (s & 1) * 8;
  } else {
    const int key = 4 * half;
    v_at = lds0 + S::BYTES + key * PITCH + (((lane & 31) / 4) ^ S::v_key(key)) * 16 + (lane & 3) * 4;
  }

  const float c = p.scale * kLog2e;
  f32x16 o[DT];
  float m, l;   // what the exponents of c s are relative to, in powers of two; sum
  auto pass = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    m = -INFINITY;
    l = 0.f;
    if (t0 < t1) issue(t0, 0);
    for (int t = t0; t < t1; ++t) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
      barrier();
      if (t + 1 < t1) issue(t + 1, (t + 1 - t0) & 1);
      if (t * KT >= most) continue;
      const unsigned buf = (unsigned)(((t - t0) & 1) * 2 * S::BYTES), kb = k_at + buf, vb = v_at + buf;

      // The values' operands come in chunks: of 16 keys (fp32: two) and up to 128 columns, two reads (one) for each 32 columns. A chunk is read while the one
      // before it is multiplied, the first one behind the keys.
      constexpr int G = E == 4 ? DT : DT % 4 == 0 ? 4 : DT, PER = E == 4 ? 1 : 2, CHUNK = G * PER, CHUNKS = (E == 4 ? NB * 16 : NB * 2) * (DT / G);
      u32x2 fv[2][CHUNK];   // (fp32: the first of two)
      auto read_v = [&](auto chunk, auto r) __attribute__((always_inline)) {   // read r of a chunk
        u32x2& to = fv[chunk & 1][r];
        constexpr int step = chunk / (DT / G), d = chunk % (DT / G) * G + r / PER;
        if constexpr (E == 2) {
          const unsigned at = vb ^ (unsigned)(d * 64);
          // Of 16 lanes, lane i gets value i % 4 of the four that lanes i / 4, i / 4 + 4, + 8 and + 12 point at: four keys of one of 16 columns.
          asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(to) : "v"(at), "n"((step * 16 + r % 2 * 8) * PITCH) : "memory");
        } else {
          const unsigned at = vb ^ (unsigned)(d * 128);
          float got;
          asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(got) : "v"(at), "n"((step / 16 * 32 + step % 16 / 4 * 8 + step % 4) * PITCH) : "memory");
          to[0] = __float_as_uint(got);
        }
      };

      // scores: steps of 16 bytes of 32 keys, RING reads ahead; the two blocks of keys in turn, so that no product waits for the one before it
      constexpr int STEPS = KS * NB, RING = STEPS < 8 ? STEPS : 8;
      f32x16 s[NB];
      u32x4 fk[RING];
      auto read_k = [&](auto step) __attribute__((always_inline)) {
        u32x4& to = fk[step % RING];
        const unsigned at = kb ^ (unsigned)(step / NB * 32);
        asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(to) : "v"(at), "n"(step % NB * 32 * PITCH) : "memory");
      };
      unroll<RING>([&](auto i) __attribute__((always_inline)) { read_k(i); });
      unroll<STEPS>([&](auto i) __attribute__((always_inline)) {
        constexpr int behind = i - (STEPS - RING);   // steps without a read of keys so far
        constexpr int younger = (i + RING <= STEPS ? RING - 1 : STEPS - 1 - i) + (careful || behind < 0 ? 0 : behind < CHUNK ? behind : CHUNK);
        u32x4& f = fk[i % RING];
        asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(f) : "n"(younger) : "memory");
        if constexpr (i < NB) s[i] = mma_first<T>(f, fq[0]);
        else mma<T>(f, fq[i / NB], s[i % NB]);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (i + RING < STEPS) read_k(std::integral_constant<int, i + RING>{});
        else if constexpr (!careful && behind < CHUNK) read_v(std::integral_constant<int, 0>{}, std::integral_constant<int, behind>{});
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (!careful) unroll<(CHUNK > RING ? CHUNK - RING : 0)>([&](auto r) __attribute__((always_inline)) { read_v(std::integral_constant<int, 0>{}, std::integral_constant<int, RING + r>{}); });

      const bool partly = t * KT + KT > least;
      if (partly) {
        const int upto = sees - t * KT - 4 * half;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[b][i] = b * 32 + (i / 4) * 8 + i % 4 < upto ? s[b][i] : -INFINITY;
      }
      if constexpr (careful) to_shares(s, c, m, l, o);
      else to_weights(s, c, m, l, o);
      // output
      if constexpr (careful) {
        const int upto = sees - t * KT;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll 1
          for (int i = 0; i < 16; ++i) {
            const float mine = s[b][i], other = __shfl_xor(mine, 32, 64);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
              const int key = b * 32 + (i / 4) * 8 + h * 4 + i % 4;
              const float w = half == h ? mine : other;
              const unsigned char* const vrow = smem + buf + S::BYTES + key * PITCH;
#pragma unroll
              for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const int at = (d * 32 + j * 8 + half * 4) * E;
                  const T* const x = (const T*)(vrow + (((at / 16) ^ S::v_key(key)) * 16) + at % 16);
#pragma unroll
                  for (int e = 0; e < 4; ++e) {
                    const float sum = fmaf(w, to_f32(x[e]), o[d][j * 4 + e]);
                    o[d][j * 4 + e] = key < upto ? sum : o[d][j * 4 + e];
                  }
                }
            }
          }
      } else {
        u32x4 fw;
        unroll<CHUNKS>([&](auto chunk) __attribute__((always_inline)) {
          constexpr bool last = chunk == CHUNKS - 1;
          constexpr int step = chunk / (DT / G), d0 = chunk % (DT / G) * G;
          if constexpr (!last) unroll<CHUNK>([&](auto r) __attribute__((always_inline)) { read_v(std::integral_constant<int, chunk + 1>{}, r); });
          if constexpr (E == 2 && d0 == 0) {   // 16 keys: the operand's eight of a lane are keys 4 half + {0..3} and 8 on of them
            alignas(16) __bf16 w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = (__bf16)s[step / 2][step % 2 * 8 + i];
            fw = *(const u32x4*)w;
          }
          __builtin_amdgcn_sched_barrier(0);
          unroll<G>([&](auto d) __attribute__((always_inline)) {
            constexpr int younger = PER * (G - 1 - d) + (last ? 0 : CHUNK);
            if constexpr (E == 2) {
              u32x2 &a = fv[chunk & 1][2 * d], &b = fv[chunk & 1][2 * d + 1];
              asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a), "+v"(b) : "n"(younger) : "memory");
              mma<T>(u32x4{a[0], a[1], b[0], b[1]}, fw, o[d0 + d]);
            } else {
              float a = __uint_as_float(fv[chunk & 1][d][0]);
              asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(a) : "n"(younger) : "memory");
              o[d0 + d] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, s[step / 16][step % 16], o[d0 + d], 0, 0, 0);
            }
          });
          __builtin_amdgcn_sched_barrier(0);
        });
      }
    }
    if constexpr (careful) m *= c;
  };
  // fp32 on the bf16 matrix cores: a value is the sum of three bf16 values, a product of two values the sum of the six largest partial products
  // (see conv_split.hpp): 192 cycles where the fp32 instructions take 512. Tiles of 32 keys pass through registers, where they are split, a tile ahead, into one
  // buffer. Scores are 2^48 times as large as they are, so that some are infinite here and finite in fp32: rows of such a score, which a weight of zero
  // would hide, and of an output that is not finite go through the fp32 instructions afterwards.
  float low = 0.f;   // the least score that the row sees, where it is negative
  auto pass_of_parts = [&]() __attribute__((always_inline)) {
    constexpr int P3 = S::PITCH3, PART = S::PART, CH = DP / 32, K3 = DP / 16;
    typedef AttnShape<__bf16, DP> B;   // (where chunks of a key lie)
    const float c3 = c * kSplitUnscale;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    m = -INFINITY;
    l = 0.f;
    // the rows' parts: 8 values from 16 ks + 8 half on
    u32x4 q3[K3][3];
#pragma unroll
    for (int ks = 0; ks < K3; ++ks) {
      const int at = ks * 64 + half * 32;
      u32x4 a = {0u, 0u, 0u, 0u}, b = a;
      if (live && at < p.head_dim * E) { a = *(const u32x4*)(qp + at); b = *(const u32x4*)(qp + at + 16); }
      split_bf16(a, b, q3[ks]);
    }
    // this thread's part of a tile: four values from 4 (tid mod 8 + 8 i) on of key tid / 8
    // (which lie at their first place ^ 64 i: chunks of 16 bytes, keys of chunks that leave the lowest two bits to 4 i)
    const int r = threadIdx.x >> 3, c8 = threadIdx.x & 7;
    const int to_k = r * P3 + ((c8 / 2) ^ B::k_key(r)) * 16 + (c8 & 1) * 8, to_v = 3 * PART + r * P3 + ((c8 / 2) ^ B::v_key(r)) * 16 + (c8 & 1) * 8;
    const unsigned k_row = r * (unsigned)p.k_token + c8 * 16, v_row = r * (unsigned)p.v_token + c8 * 16;
    u32x4 next[2][CH];
    auto fetch = [&](int t) __attribute__((always_inline)) {   // (keys past the sequence's last arrive as zeros)
      const int columns = t * 32 + r < nk ? p.head_dim - c8 * 4 : 0;
      const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(kp + (long long)t * 32 * p.k_token), 0, 0x7fffffff, 0x00020000);
      const __amdgpu_buffer_rsrc_t vb = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vp + (long long)t * 32 * p.v_token), 0, 0x7fffffff, 0x00020000);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        next[0][i] = __builtin_amdgcn_raw_buffer_load_b128(kb, (int)(i * 32 < columns ? k_row + i * 128 : kOut), 0, 0);
        next[1][i] = __builtin_amdgcn_raw_buffer_load_b128(vb, (int)(i * 32 < columns ? v_row + i * 128 : kOut), 0, 0);
      }
    };
    const int u0 = t0 * (KT / 32), u1 = min(t1 * (KT / 32), (all + 31) / 32);
    if (u0 < u1) fetch(u0);
    const unsigned char* const k_from = smem + (lane & 31) * P3;
    const int k_key = B::k_key(lane & 31), s16 = lane & 15, v_key0 = 4 * half + s16 / 4;
    const unsigned char* const v_from = smem + 3 * PART + v_key0 * P3 + (s16 & 1) * 8;
    const int v_chunk = (2 * ((lane >> 4) & 1) + (s16 & 3) / 2) ^ B::v_key(v_key0);
    for (int t = u0; t < u1; ++t) {
      barrier();   // (no wavefront reads the tile before)
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        uint2 part[3];
        split_bf16(__builtin_bit_cast(f32x4, next[0][i]), part);
#pragma unroll
        for (int e = 0; e < 3; ++e) *(uint2*)(smem + e * PART + (to_k ^ (i * 64))) = part[e];
        split_bf16(__builtin_bit_cast(f32x4, next[1][i]), part);
#pragma unroll
        for (int e = 0; e < 3; ++e) *(uint2*)(smem + e * PART + (to_v ^ (i * 64))) = part[e];
      }
      if (t + 1 < u1) fetch(t + 1);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      barrier();
      const int key0 = t * 32;
      if (key0 >= most) continue;
      f32x16 tile[1];
      f32x16& s = tile[0];
#pragma unroll
      for (int ks = 0; ks < K3; ++ks) {
        u32x4 k3[3];
#pragma unroll
        for (int e = 0; e < 3; ++e) k3[e] = *(const u32x4*)(k_from + e * PART + ((2 * ks + half) ^ k_key) * 16);
#pragma unroll
        for (int e = 0; e < 6; ++e) {
          if (ks == 0 && e == 0) s = mma_first<__bf16>(k3[kSplitW[e]], q3[ks][kSplitX[e]]);
          else mma<__bf16>(k3[kSplitW[e]], q3[ks][kSplitX[e]], s);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (key0 + 32 > least) {
        const int upto = sees - key0 - 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const bool seen = (i / 4) * 8 + i % 4 < upto;
          low = __builtin_elementwise_minimum(low, seen ? s[i] : 0.f);
          s[i] = seen ? s[i] : -INFINITY;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) low = __builtin_elementwise_minimum(low, s[i]);
      }
      to_weights(tile, c3, m, l, o);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 w3[3];
        split_bf16(__builtin_bit_cast(u32x4, f32x4{s[8 * h], s[8 * h + 1], s[8 * h + 2], s[8 * h + 3]}),
                   __builtin_bit_cast(u32x4, f32x4{s[8 * h + 4], s[8 * h + 5], s[8 * h + 6], s[8 * h + 7]}), w3);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          u32x4 v3[3];
#pragma unroll
          for (int e = 0; e < 3; ++e) {
            const unsigned char* const at = v_from + e * PART + h * 16 * P3 + (v_chunk ^ (4 * d)) * 16;
            const u32x2 a = transposed_read(at), b = transposed_read(at + 8 * P3);
            v3[e] = u32x4{a[0], a[1], b[0], b[1]};
          }
#pragma unroll
          for (int e = 0; e < 6; ++e) mma<__bf16>(v3[kSplitW[e]], w3[kSplitX[e]], o[d]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] *= kSplitUnscale;
  };
  // The rows that a pass got right leave; whether there are others. Odd are an output that is not finite, a score that was not (low), and a sum of weights near
  // zero: relative to a score far from zero (see to_shares) all weights may vanish, else the largest is at least 1. With the least sum here no weight of more than
  // 2^-62 of the largest is lost. A later pass writes odd rows only, so that a row's bits do not depend on the rows beside it.
  constexpr float kLeastSum = 0x1p-64f;
  bool open = live;   // the row is still to be written
  auto leave = [&](auto careful) __attribute__((always_inline)) {
    const float sum = careful ? l : sum_of_halves(l);
    bool odd = false;
    if constexpr (!careful) {
      odd = !(low > -INFINITY) || (sees > t0 * KT && !(sum >= kLeastSum));
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd |= !(fabsf(o[d][i]) < INFINITY);
      odd = of_either_half(odd);
    }
    if (open && !odd) {
      const float by = careful ? 1.f : sum == 0.f ? 0.f : 1.f / sum;   // (no key: a row that sees none, or none of this part)
      if (p.splits > 1) {
        const long long rows = (long long)(p.hi - p.lo) * (p.heads_k * p.group);
        const long long slot = blockIdx.y * rows + (at_row - p.lo) * (p.heads_k * p.group) + qh;
        float* const to = p.part + slot * p.head_dim;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int at = d * 32 + j * 8 + half * 4;
            if (at < p.head_dim) *(f32x4*)(to + at) = f32x4{o[d][j * 4] * by, o[d][j * 4 + 1] * by, o[d][j * 4 + 2] * by, o[d][j * 4 + 3] * by};
          }
        if (half == 0) *(float2*)(p.part + p.splits * rows * p.head_dim + slot * 2) = make_float2(m, sees > 0 ? sum : -1.f);
      } else {
        const float by_all = sum == 0.f ? NAN : by;   // (no seen score is one that fp32 holds)
        char* const op = p.out + at_row * p.out_token + qh * p.out_head;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int at = d * 32 + j * 8 + half * 4;
            if (at >= p.head_dim) continue;
            alignas(16) T w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = from_f32<T>(sees > 0 ? o[d][j * 4 + e] * by_all : 0.f);
            __builtin_memcpy(__builtin_assume_aligned(op + at * E, 4 * E), w, sizeof(w));
          }
        if (p.lse && half == 0) p.lse[(long long)qh * p.rows_q + at_row] = sees > 0 ? (m + log2f(sum)) * kLn2 : -INFINITY;
      }
    }
    open = open && odd;
    return careful ? 0 : __syncthreads_or(open);
  };
  if constexpr (S::PARTS) {
    pass_of_parts();
    if (!leave(std::false_type{})) return;
  }
  // Weights of zero times an infinity or a NaN of a value that the row does not see are NaNs. They are rare, and looked for at the end only: then the
  // keys are gone through again, one by one.
  get_ready();
  low = 0.f;
  pass(std::false_type{});
  if (!leave(std::false_type{})) return;
  pass(std::true_type{});
  leave(std::true_type{});
}

// Joins the parts of a row: a wavefront for each row and head, lane s has part s's maximum and sum. (A sum of -1: the row sees no key.)
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(const AttnParams p) {
  const int lane = threadIdx.x & 63, heads = p.heads_k * p.group;
  const long long rows = (long long)(p.hi - p.lo) * heads, at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (at >= rows) return;
  const int head = (int)(at % heads);
  const long long row = p.lo + at / heads;
  const int first = clamp_to(p.q_offsets[0], p.rows_q), last = clamp_to(p.q_offsets[p.seqs], p.rows_q);
  if (row < first || row >= last) return;
  const float2* const stats = (const float2*)(p.part + p.splits * rows * p.head_dim);
  const float2 mine = lane < p.splits ? stats[lane * rows + at] : make_float2(-INFINITY, 0.f);
  float m = mine.x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) m = __builtin_elementwise_maximum(m, __shfl_xor(m, d, 64));
  const float by = __builtin_amdgcn_exp2f(mine.x - (m == -INFINITY ? 0.f : m));
  const bool none = __any(mine.y < 0.f);
  float l = by * mine.y;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d, 64);
  const float share = by * mine.y / l;
  const bool here = lane * 4 < p.head_dim;
  const float* const from = p.part + at * p.head_dim + (here ? lane * 4 : 0);
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < p.splits; s0 += 8) {   // (the last part again where there are fewer, and nothing of it)
    f32x4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = *(const f32x4*)(from + min(s0 + i, p.splits - 1) * rows * p.head_dim);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (s0 + i < p.splits) o += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(share), s0 + i)) * x[i];
  }
  if (here) {
    alignas(16) T w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = from_f32<T>(none ? 0.f : o[i]);
    __builtin_memcpy(__builtin_assume_aligned(p.out + row * p.out_token + head * p.out_head + lane * 4 * (int)sizeof(T), 4 * sizeof(T)), w, sizeof(w));
  }
  if (p.lse && lane == 0) p.lse[(long long)head * p.rows_q + row] = none ? -INFINITY : (m + log2f(l)) * kLn2;
}

// How a call is cut: which tiles the rows of a band can have (see find_tile: a row's number lies between floor(row group / kRows) - 1 and floor(...) + its
// sequence), and parts of the keys: those with which the call is estimated to be done first. A workgroup takes `alone` us a tile of keys where it is alone on
// its compute unit and `shared` where it is one of two; joining reads and writes the parts' outputs and is a launch. Measured with 1, 2, 4, 8, 16, 32 and 64
// parts, us: a row of 32 heads (8 of keys) on 8 000 keys 144, 78, 44, 27, 19, 17, 21; 8 such rows on 4 000 keys 81, 52, 35, 34, 38, 46, 65; 256 rows on 4 000 keys 83,
// 52, 35, 37, 49, 73, 137; a prompt of 1 000 rows 27, 41, 47, 67, ..; in fp32 with 12 heads (4) 138, 66, 60, 70, ...
// Of 120 calls of all kinds the chosen number is within 3 % of the best in the mean, and 34 % off at worst (caches filled to a half on the average).
struct Cut { int tile0, tiles, splits; };
Cut cut(const lop_attention_t* op, lop_rows_t rows) {
  const long long group = op->heads_q / op->heads_k;
  Cut c;
  c.tile0 = (int)std::max(rows.lo * group / kRows - 1, 0LL);
  c.tiles = (int)((rows.hi * group - 1) / kRows + op->seqs - c.tile0);
  c.splits = 1;
  if (op->max_keys < (op->dtype == LOP_F32 ? LOP_ATTENTION_CUT_F32 : LOP_ATTENTION_CUT)) return c;
  struct Price { int keys; double alone, shared; };   // (shared 0: a workgroup has its compute unit for itself)
  static constexpr Price prices[2][4] = {{{64, 0.9, 1.2}, {64, 1.1, 1.7}, {64, 1.3, 2.0}, {64, 2.9, 0.0}},     // bf16: 64, 96, 128, 256 values a head
                                         {{32, 1.7, 3.0}, {32, 2.4, 4.3}, {32, 4.3, 5.9}, {32, 8.9, 0.0}}};    // fp32
  const Price& price = prices[op->dtype == LOP_F32][op->head_dim <= 64 ? 0 : op->head_dim <= 96 ? 1 : op->head_dim <= 128 ? 2 : 3];
  constexpr double kCus = 256.0;
  const double blocks = (double)c.tiles * op->heads_k, band = rows.hi - rows.lo, tiles = (double)ceil_div(op->max_keys, price.keys);
  // (of a causal prompt the average row sees half of the keys)
  const double seen = op->causal ? 1.0 - 0.5 * std::min(1.0, (double)op->rows_q / op->seqs / op->max_keys) : 1.0;
  double least = 0.0;
  for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
    const double each = std::ceil(tiles / s), units = blocks * s / kCus, full = price.shared > 0.0 ? units / 2 * price.shared : units * price.alone;
    double time = units <= 1.0 ? each * price.alone : each * std::max(price.alone, seen * full);
    if (s > 1) time += 5.0 + s * band * op->heads_q * op->head_dim * 8.0 / 3.5e6;
    if (s == 1 || time < least) { c.splits = s; least = time; }
  }
  return c;
}
unsigned long long workspace_of(const lop_attention_t* op, lop_rows_t rows, int splits) {
  return splits < 2 ? 0 : (unsigned long long)splits * (rows.hi - rows.lo) * op->heads_q * (op->head_dim + 2) * sizeof(float);
}

int check_sizes(const lop_attention_t* op, lop_rows_t rows) {
  if (!op || op->heads_q < 1 || op->heads_k < 1 || op->head_dim < 1 || op->seqs < 0 || op->rows_q < 0 || op->rows_k < 0 || op->max_keys < 0)
    return LOP_ERR_INVALID_ARG;
  if (!known_dtype(op->dtype) || op->head_dim % 8 || op->head_dim > 256) return LOP_ERR_UNSUPPORTED;
  if (op->heads_q % op->heads_k) return LOP_ERR_SHAPE;
  if (const int e = check_band(rows, op->rows_q)) return e;
  // (numbers of packed rows and of keys, up to the end of a tile, are 32 bits)
  const long long group = op->heads_q / op->heads_k, packed = (long long)op->rows_q * group;
  if (packed >= (1LL << 31) || op->rows_k > INT_MAX - 64 || (packed / kRows + op->seqs + 1) * op->heads_k > launch_blocks(256) ||
      ceil_div((long long)op->rows_q * op->heads_q, 4) > launch_blocks(256))
    return LOP_ERR_UNSUPPORTED;
  return LOP_OK;
}

template <typename T>
hipError_t launch_attention(const AttnParams& p, hipStream_t s) {
  const dim3 grid((unsigned)p.tiles * (unsigned)p.heads_k, (unsigned)p.splits), block(256);
  const hipError_t e = p.head_dim <= 64    ? launch_kernel(attention_kernel<T, 64>, grid, block, s, nullptr, p)
                       : p.head_dim <= 96  ? launch_kernel(attention_kernel<T, 96>, grid, block, s, nullptr, p)
                       : p.head_dim <= 128 ? launch_kernel(attention_kernel<T, 128>, grid, block, s, nullptr, p)
                                           : launch_kernel(attention_kernel<T, 256>, grid, block, s, nullptr, p);
  if (e != hipSuccess || p.splits < 2) return e;
  const long long waves = (long long)(p.hi - p.lo) * p.heads_k * p.group;
  return launch_kernel(attention_join_kernel<T>, dim3((unsigned)ceil_div(waves, 4)), block, s, nullptr, p);
}

}  // namespace
}  // namespace lop

extern "C" int lop_attention_workspace(const lop_attention_t* op, lop_rows_t rows, unsigned long long* bytes) {
  using namespace lop;
  if (!bytes) return LOP_ERR_INVALID_ARG;
  *bytes = 0;
  if (const int e = check_sizes(op, rows)) return e;
  if (rows.lo < rows.hi && op->seqs > 0) *bytes = workspace_of(op, rows, cut(op, rows).splits);
  return LOP_OK;
}

extern "C" int lop_attention(const lop_attention_t* op, lop_rows_t rows, void* stream) {
  using namespace lop;
  if (const int e = check_sizes(op, rows)) return e;
  if (!(op->scale > 0.f) || !(op->scale < INFINITY)) return LOP_ERR_INVALID_ARG;
  if (rows.lo == rows.hi || op->seqs == 0) return LOP_OK;
  const long long E = (long long)dtype_bytes(op->dtype);
  auto good = [&](const void* p, long long token, long long head, int rows_of, int heads) {
    return p && aligned16(p) && whole_vectors(token, E, rows_of > 1) && whole_vectors(head, E, heads > 1);
  };
  if (!good(op->q, op->q_token, op->q_head, op->rows_q, op->heads_q) || !good(op->out, op->out_token, op->out_head, op->rows_q, op->heads_q))
    return LOP_ERR_INVALID_ARG;
  if (op->rows_k > 0 && (!good(op->k, op->k_token, op->k_head, op->rows_k, op->heads_k) || !good(op->v, op->v_token, op->v_head, op->rows_k, op->heads_k)))
    return LOP_ERR_INVALID_ARG;
  if (!apart(op->head_dim, op->out_token, op->rows_q, op->out_head, op->heads_q)) return LOP_ERR_INVALID_ARG;
  if (!op->q_offsets || !op->k_begin || !op->k_end) return LOP_ERR_INVALID_ARG;
  if (((uintptr_t)op->q_offsets | (uintptr_t)op->k_begin | (uintptr_t)op->k_end | (uintptr_t)op->lse) & 3 || !aligned16(op->workspace)) return LOP_ERR_INVALID_ARG;
  // (a tile's keys are one buffer: its rows lie behind one another, and offsets in it are 32 bits)
  if (op->rows_k > 1 && (op->k_token < op->head_dim || op->v_token < op->head_dim)) return LOP_ERR_INVALID_ARG;
  if (op->rows_k > 1 && (op->k_token * E > (1LL << 31) / 128 || op->v_token * E > (1LL << 31) / 128)) return LOP_ERR_UNSUPPORTED;
  const Cut c = cut(op, rows);
  AttnParams p;
  p.q = (const char*)op->q; p.k = (const char*)op->k; p.v = (const char*)op->v; p.out = (char*)op->out;
  p.q_token = op->q_token * E; p.q_head = op->q_head * E; p.out_token = op->out_token * E; p.out_head = op->out_head * E;
  p.k_token = op->rows_k > 1 ? op->k_token * E : 0; p.k_head = op->k_head * E;
  p.v_token = op->rows_k > 1 ? op->v_token * E : 0; p.v_head = op->v_head * E;
  p.q_offsets = op->q_offsets; p.k_begin = op->k_begin; p.k_end = op->k_end;
  p.lse = op->lse;
  p.heads_k = op->heads_k; p.group = op->heads_q / op->heads_k; p.head_dim = op->head_dim;
  p.seqs = op->seqs; p.rows_q = op->rows_q; p.rows_k = op->rows_k; p.causal = op->causal != 0;
  p.lo = rows.lo; p.hi = rows.hi;
  p.tile0 = c.tile0; p.tiles = c.tiles;
  p.splits = c.splits > 1 && op->workspace && op->workspace_bytes >= workspace_of(op, rows, c.splits) ? c.splits : 1;
  p.part = (float*)op->workspace;
  p.scale = op->scale;
  LOP_HIP(op->dtype == LOP_BF16 ? launch_attention<__bf16>(p, (hipStream_t)stream) : launch_attention<float>(p, (hipStream_t)stream));
  return LOP_OK;
}
