// The decode step of slim attention over a K-cache in 4 or 8 bits (its format: kernels_quant.hip): scores, weighted sum of K, merge + projection through W_KV.
// Three launches; none of their workgroups waits for another.  What a code stands for is exact in bf16, so that K enters both products without a rounding.
// The codes are read twice: the numerators of all heads weigh every column, and the H x d sums of one pass would fill the registers of a compute unit each, whose partial
// results (512 KB a unit at 32 heads x 4096) are more bytes than the second pass.  1 x 16384 rows x 32 x 128 in 4 bits: 9 + 15 + 12.6 us.
#include <algorithm>

#include "device_common.h"
#include "slim_kernels.h"

namespace slim {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float scale_of(unsigned dw, int k) { return __uint_as_float(((dw >> (8 * k)) & 0xffu) << 23); }

// Eight codes of a row: columns 2 k and 2 k + 1 as floats, or as a pair of bf16 (exact)
template <int BITS> struct Codes8;
template <> struct Codes8<4> {
  unsigned w;
  __device__ __forceinline__ void load(const unsigned char* p) { w = *(const unsigned*)p; }
  template <int K> __device__ __forceinline__ f32x2 f32(float s) const { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, K); }
  template <int K> __device__ __forceinline__ unsigned bf16(float s) const {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, K));
  }
};
template <> struct Codes8<8> {
  u32x2 w;
  __device__ __forceinline__ void load(const unsigned char* p) { w = *(const u32x2*)p; }
  template <int K> __device__ __forceinline__ f32x2 f32(float s) const { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[K >> 1], s, (K & 1) != 0); }
  template <int K> __device__ __forceinline__ unsigned bf16(float s) const {
    return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[K >> 1], s, (K & 1) != 0));
  }
};

// ---- scores -------------------------------------------------------------------------------------------

template <int STEP>
__device__ __forceinline__ float from_partner(float v) {
  if constexpr (STEP == 1) return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xf, 0xf, true));
  else if constexpr (STEP == 2) return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xf, 0xf, true));
  else if constexpr (STEP == 4) return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true));     // 7 - lane
  else if constexpr (STEP == 8) return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xf, 0xf, true));     // 15 - lane
  else return __shfl_xor(v, STEP);
}
// Lane i of a head's P lanes gets the sum over these lanes of their v[i]: halves are exchanged from the widest step on.  (The mirrors that steps of
// 4 and 8 use flip the lower bits too; whom they join still differs in the step's own bit, and in every round from everyone joined before.)
template <int P>
__device__ __forceinline__ float sums_to_lanes(float (&v)[P], int lane) {
  if constexpr (P > 1) {
    constexpr int S = P / 2;
    float u[S];
    const bool upper = (lane & S) != 0;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      const float mine = upper ? v[k + S] : v[k], other = upper ? v[k] : v[k + S];
      u[k] = mine + from_partner<S>(other);
    }
    return sums_to_lanes<S>(u, lane);
  } else {
    return v[0];
  }
}
template <int P>
__device__ __forceinline__ float max_over_lanes(float v) {
  if constexpr (P > 1) { v = fmaxf(v, from_partner<P / 2>(v)); return max_over_lanes<P / 2>(v); }
  else return v;
}
template <int P>
__device__ __forceinline__ float sum_over_lanes(float v) {
  if constexpr (P > 1) { v = v + from_partner<P / 2>(v); return sum_over_lanes<P / 2>(v); }
  else return v;
}

// A wave takes 64 rows x 64 / P heads; a head is P lanes of eight columns (those past d_k are idle).  Rows go P at a time, lane i of a head ends with the
// 64 / P consecutive rows from i * 64 / P on, and the scale bytes of all 64 rows are one run of a lane's group.  From the scores come softmax numerators relative
// to a power of two per head and block: a whole exponent, so that a later change of reference is exact in every type.
// HBM-bound (0.53 or 1.03 bytes an element); about 20 instructions a row and lane, 37 with rotated keys, where the vector ALU bounds.  For heads of other widths than
// the next kernel's.
template <bool F32, int BITS, int P, bool ROPE>
__global__ __launch_bounds__(256) void qscores_kernel(QDecodeArgs a) {
  __shared__ f32x4 table[ROPE && P <= 16 ? QUANT_ROWS * P * 2 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  {
    const long wgs = (long)gridDim.x * gridDim.y * gridDim.z, wg = blockIdx.x + (long)gridDim.x * (blockIdx.y + (long)gridDim.y * blockIdx.z);
    for (long i = wg * 256 + tid; i < a.ncounters; i += wgs * 256) a.counters[i] = 0;
  }
  const int b = blockIdx.z, t0 = blockIdx.x * QUANT_ROWS;
  const int len = seq_len_of(a.seq_lens, b, a.T);
  if (t0 >= len) return;
  constexpr int HW = 64 / P, RP = 64 / P;
  const int h = (blockIdx.y * 4 + wave) * HW + lane / P, i = lane % P;
  const bool on = h < a.H && i * 8 < a.d_k;
  const int col = on ? h * a.d_k + i * 8 : 0;
  float qf[8];
  unsigned qb[4], qr[4];                          // pairs (q0, q1) and (-q1, q0)
  if constexpr (F32) {
    const f32x4* src = (const f32x4*)((const float*)a.q + (long)b * a.d + col);
    const f32x4 lo = src[0], hi = src[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) { qf[j] = lo[j]; qf[4 + j] = hi[j]; }
  } else {
    const u32x4 v = *(const u32x4*)((const uint16_t*)a.q + (long)b * a.d + col);
#pragma unroll
    for (int j = 0; j < 4; ++j) { qb[j] = v[j]; qr[j] = ((v[j] >> 16) ^ 0x8000u) | v[j] << 16; qf[2 * j] = __uint_as_float(v[j] << 16); qf[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u); }
  }
  if (!on) {                                      // (a lane past its head's columns counts nothing: a row that is not finite is that for its whole sequence)
#pragma unroll
    for (int j = 0; j < 4; ++j) { qb[j] = qr[j] = 0u; qf[2 * j] = qf[2 * j + 1] = 0.f; }
  }
  const unsigned char* codes = a.codes + ((long)b * a.stride + t0) * (a.d * BITS / 8);
  const unsigned at_col = (unsigned)(col * BITS / 8);
  const u32x4* sp = (const u32x4*)(a.scales + ((long)b * (a.d / 32) + col / 32) * a.stride + t0);
  u32x4 sc[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) sc[k] = sp[k];
  const long row_bytes = a.d * BITS / 8;
  float s[RP];
  Codes8<BITS> w[2][P];
  auto fetch = [&](int j, auto buf) {
#pragma unroll
    for (int r = 0; r < P; ++r) w[buf.value][r].load(codes + (long)(r * RP + j) * row_bytes + at_col);
  };
  auto step = [&](int j, auto J) {
    constexpr int cur = decltype(J)::value & 1;
    float v[P];
#pragma unroll
    for (int r = 0; r < P; ++r) {
      const int row = r * RP + decltype(J)::value;
      const float f = scale_of(sc[row >> 4][(row >> 2) & 3], row & 3);
      const Codes8<BITS>& c = w[cur][r];
      float x = 0.f;
      if constexpr (ROPE) {
        f32x4 t[2];
        if constexpr (P <= 16) {
          const f32x4* cs = table + (row * (P * 2) + i * 2);
          t[0] = cs[0]; t[1] = cs[1];
        } else {
          // (rows behind the sequence, whose score is masked, have no position in the table)
          const f32x4* cs = (const f32x4*)(a.rope + ((long)min(t0 + row, len - 1) * (a.d_k / 2) + (on ? i * 4 : 0)) * 2);
          t[0] = cs[0]; t[1] = cs[1];
        }
        auto pair = [&](auto K) {
          constexpr int k = decltype(K)::value;
          const float co = t[k >> 1][2 * (k & 1)], si = t[k >> 1][2 * (k & 1) + 1];
          float u, w;                              // q . y and q . (y turned by a quarter): the score is u cos + w sin
          if constexpr (F32) {
            const f32x2 y = c.template f32<k>(f);
            u = fmaf(qf[2 * k], y[0], qf[2 * k + 1] * y[1]);
            w = fmaf(qf[2 * k], y[1], -(qf[2 * k + 1] * y[0]));
          } else {
            const bf16x2 y = __builtin_bit_cast(bf16x2, c.template bf16<k>(f));
            u = __builtin_amdgcn_fdot2_f32_bf16(y, __builtin_bit_cast(bf16x2, qb[k]), 0.f, false);
            w = __builtin_amdgcn_fdot2_f32_bf16(y, __builtin_bit_cast(bf16x2, qr[k]), 0.f, false);
          }
          x = fmaf(co, u, x);
          x = fmaf(si, w, x);
        };
        pair(std::integral_constant<int, 0>{}); pair(std::integral_constant<int, 1>{});
        pair(std::integral_constant<int, 2>{}); pair(std::integral_constant<int, 3>{});
      } else if constexpr (F32) {
        auto pair = [&](auto K) {
          constexpr int k = decltype(K)::value;
          const f32x2 y = c.template f32<k>(f);
          x = fmaf(qf[2 * k], y[0], x);
          x = fmaf(qf[2 * k + 1], y[1], x);
        };
        pair(std::integral_constant<int, 0>{}); pair(std::integral_constant<int, 1>{});
        pair(std::integral_constant<int, 2>{}); pair(std::integral_constant<int, 3>{});
      } else {
        auto pair = [&](auto K) {
          constexpr int k = decltype(K)::value;
          x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, c.template bf16<k>(f)), __builtin_bit_cast(bf16x2, qb[k]), x, false);
        };
        pair(std::integral_constant<int, 0>{}); pair(std::integral_constant<int, 1>{});
        pair(std::integral_constant<int, 2>{}); pair(std::integral_constant<int, 3>{});
      }
      v[r] = x;
    }
    s[decltype(J)::value] = sums_to_lanes<P>(v, lane);
  };
  if ((int)(blockIdx.y * 4 + wave) * HW < a.H) fetch(0, std::integral_constant<int, 0>{});
  if constexpr (ROPE && P <= 16) {
    // The 64 rows' cos and sin, which 16 and more heads share: to LDS once (32 KB for 128 columns).  Asked for from memory by every head they took as long as the codes.
    const int per = a.d_k / 4;
    for (int x = tid; x < QUANT_ROWS * P * 2; x += 256) {
      const int row = x / (P * 2), k = x % (P * 2);
      table[x] = k < per ? *(const f32x4*)(a.rope + (long)min(t0 + row, len - 1) * a.d_k + k * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();
  }
  if ((int)(blockIdx.y * 4 + wave) * HW >= a.H) return;  // (no head for this wave)
  auto both = [&](int j, auto J) {
    if constexpr (decltype(J)::value + 1 < RP) fetch(decltype(J)::value + 1, std::integral_constant<int, (decltype(J)::value + 1) & 1>{});
    step(j, J);
  };
  full_steps<0, RP>(0, both);
  // numerators
  float m = NEG_INF;
#pragma unroll
  for (int j = 0; j < RP; ++j) {
    s[j] = t0 + i * RP + j < len ? s[j] * a.qscale : NEG_INF;
    m = fmaxf(m, s[j]);
  }
  m = max_over_lanes<P>(m);
  const float ref = m == NEG_INF ? 0.f : ceilf(m);
  float l = 0.f;
  const long o = ((long)b * a.H + h) * a.Tp + t0 + i * RP;
  float p[RP];
#pragma unroll
  for (int j = 0; j < RP; ++j) {
    p[j] = exp2f(s[j] - ref);
    if constexpr (!F32) p[j] = (float)(__bf16)p[j];       // rounded where it enters the product with K, and the sum is of what enters
    l += p[j];
  }
  l = sum_over_lanes<P>(l);
  if (h >= a.H) return;
  if constexpr (F32) {
#pragma unroll
    for (int j = 0; j < RP; ++j) ((float*)a.P)[o + j] = p[j];
  } else {
#pragma unroll
    for (int j = 0; j < RP; ++j) ((__bf16*)a.P)[o + j] = (__bf16)p[j];
  }
  if (i == 0) {
    const long at = ((long)b * a.H + h) * a.NB + blockIdx.x;
    a.ref[at] = ref;
    a.sum[at] = l;
  }
}

// The same for heads of 32 CH columns (32, 64, 96, 128): four lanes a head, 8 CH columns each, none idle.  A wave has eight heads x 16 rows, in two halves of the
// lanes eight rows each; the four waves have a block of 64 rows, and meet in LDS for its reference.
// With 16 lanes a head, heads of 96 columns kept a quarter of the lanes idle: 16 sequences of 600..5000 rows x 24 heads in 8 bits, rotary 35 us, without 22.7; now
// 24.6 and 19.3 (5.6 TB/s of codes).  Rotary, the vector ALU has 14 of it.  Eight waves, whose sixteen heads shared the table, had fewer workgroups to fill one's waits with
// another's work: 29.7, and 31.3 with q and the table behind the codes; registers for five waves a SIMD spill (37).  1 x 16384 x 32 x 128 in 4 bits 9 us.
template <bool F32, int BITS, int CH, bool ROPE>
__global__ __launch_bounds__(256) void qscores_even_kernel(QDecodeArgs a) {
  constexpr int P = 4, RP = 2, DK = 32 * CH;
  __shared__ f32x4 table[ROPE ? QUANT_ROWS * DK / 4 : 1];
  __shared__ float most[4][8], total[4][8];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  {
    const long wgs = (long)gridDim.x * gridDim.y * gridDim.z, wg = blockIdx.x + (long)gridDim.x * (blockIdx.y + (long)gridDim.y * blockIdx.z);
    for (long i = wg * 256 + tid; i < a.ncounters; i += wgs * 256) a.counters[i] = 0;
  }
  // Blocks of the same rows follow each other over the heads and sequences: they take cos and sin from the L2s.  (Which comes first moves on by one from rows to rows:
  // an XCD would get the same sequences and heads all along, and the others the short ones.)
  const int groups = (a.H + 7) / 8, blk = blockIdx.z * gridDim.y + blockIdx.y;
  const unsigned at_block = (blockIdx.x + (unsigned)blk) % gridDim.x;
  const int b = at_block / groups, hg = at_block % groups;
  const int len = seq_len_of(a.seq_lens, b, a.T);
  if (blk >= (len + QUANT_ROWS - 1) / QUANT_ROWS) return;
  const int t0 = blk * QUANT_ROWS;
  const int i = lane & 3, slot = (lane >> 2) & 7, half = lane >> 5;
  const int h = hg * 8 + slot, hc = min(h, a.H - 1);      // (heads past the last: the last again, not stored)
  const int col = hc * DK + i * 8 * CH, first = wave * 16 + half * 8;         // this lane's columns and first row of the block
  const long row_bytes = (long)a.d * BITS / 8;
  const unsigned char* codes = a.codes + ((long)b * a.stride + t0 + wave * 16) * row_bytes;
  const unsigned at = (unsigned)(half * 8 * (int)row_bytes + col * BITS / 8);
  constexpr int PER_THREAD = DK / 16;               // table entries: 64 DK / 4 over 256 threads
  f32x4 turn[ROPE ? PER_THREAD : 1];
  if constexpr (ROPE) {
    // (rows behind the sequence, whose score is masked, have no position in the table)
#pragma unroll
    for (int x = 0; x < PER_THREAD; ++x) {
      const int at_entry = tid + x * 256, row = at_entry / (DK / 4), k = at_entry % (DK / 4);
      turn[x] = *(const f32x4*)(a.rope + (long)min(t0 + row, len - 1) * DK + k * 4);
    }
  }
  constexpr int NSC = CH == 3 ? 3 : 1;             // groups that the chunks of eight columns lie in (24 columns: two, which of them is the lane's)
  u32x2 sc[NSC];
#pragma unroll
  for (int k = 0; k < NSC; ++k) sc[k] = *(const u32x2*)(a.scales + ((long)b * (a.d / 32) + (col + 8 * k) / 32) * a.stride + t0 + first);
  float qf[F32 ? 8 * CH : 1];
  unsigned qb[4 * CH], qr[4 * CH];
  if constexpr (F32) {
    const f32x4* src = (const f32x4*)((const float*)a.q + (long)b * a.d + col);
#pragma unroll
    for (int j = 0; j < 2 * CH; ++j) {
      const f32x4 v = src[j];
#pragma unroll
      for (int k = 0; k < 4; ++k) qf[4 * j + k] = v[k];
    }
  } else {
    const u32x4* src = (const u32x4*)((const uint16_t*)a.q + (long)b * a.d + col);
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const u32x4 v = src[j];
#pragma unroll
      for (int k = 0; k < 4; ++k) { qb[4 * j + k] = v[k]; qr[4 * j + k] = ((v[k] >> 16) ^ 0x8000u) | v[k] << 16; }
    }
  }
  // (Loads come back in order: what all rows need first, then the rows as they are taken.)
  Codes8<BITS> w[P * RP][CH];
#pragma unroll
  for (int j = 0; j < RP; ++j)
#pragma unroll
    for (int r = 0; r < P; ++r)
#pragma unroll
      for (int k = 0; k < CH; ++k) w[r * RP + j][k].load(codes + (long)(r * RP + j) * row_bytes + at + k * BITS);
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (ROPE) {
#pragma unroll
    for (int x = 0; x < PER_THREAD; ++x) table[tid + x * 256] = turn[x];
    lds_barrier();
  }
  float s[RP];
#pragma unroll
  for (int j = 0; j < RP; ++j) {
    float v[P];
#pragma unroll
    for (int r = 0; r < P; ++r) {
      const int row = r * RP + j;                  // lane i ends with rows 2 i and 2 i + 1
      float x = 0.f;
      auto chunk = [&](int, auto C) {
        constexpr int ch = decltype(C)::value;
        const float f = scale_of(sc[NSC == 1 ? 0 : ch][row >> 2], row & 3);
        const Codes8<BITS>& c = w[row][ch];
        f32x4 t[2];
        if constexpr (ROPE) {
          const f32x4* cs = table + (first + row) * (DK / 4) + (i * CH + ch) * 2;
          t[0] = cs[0]; t[1] = cs[1];
        }
        auto pair = [&](int, auto K) {
          constexpr int k = decltype(K)::value, kk = 4 * ch + k;
          if constexpr (ROPE) {
            const float co = t[k >> 1][2 * (k & 1)], si = t[k >> 1][2 * (k & 1) + 1];
            float u, y;                            // q . y and q . (y turned by a quarter): the score is u cos + w sin
            if constexpr (F32) {
              const f32x2 z = c.template f32<k>(f);
              u = fmaf(qf[2 * kk], z[0], qf[2 * kk + 1] * z[1]);
              y = fmaf(qf[2 * kk], z[1], -(qf[2 * kk + 1] * z[0]));
            } else {
              const bf16x2 z = __builtin_bit_cast(bf16x2, c.template bf16<k>(f));
              u = __builtin_amdgcn_fdot2_f32_bf16(z, __builtin_bit_cast(bf16x2, qb[kk]), 0.f, false);
              y = __builtin_amdgcn_fdot2_f32_bf16(z, __builtin_bit_cast(bf16x2, qr[kk]), 0.f, false);
            }
            x = fmaf(co, u, x);
            x = fmaf(si, y, x);
          } else if constexpr (F32) {
            const f32x2 z = c.template f32<k>(f);
            x = fmaf(qf[2 * kk], z[0], x);
            x = fmaf(qf[2 * kk + 1], z[1], x);
          } else {
            x = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, c.template bf16<k>(f)), __builtin_bit_cast(bf16x2, qb[kk]), x, false);
          }
        };
        full_steps<0, 4>(0, pair);
      };
      full_steps<0, CH>(0, chunk);
      v[r] = x;
    }
    s[j] = sums_to_lanes<P>(v, lane);
  }
  // numerators, against the block's reference
  float m = NEG_INF;
#pragma unroll
  for (int j = 0; j < RP; ++j) {
    s[j] = t0 + first + i * RP + j < len ? s[j] * a.qscale : NEG_INF;
    m = fmaxf(m, s[j]);
  }
  m = max_over_lanes<P>(m);
  m = fmaxf(m, __shfl_xor(m, 32));
  if (i == 0 && half == 0) most[wave][slot] = m;
  lds_barrier();
#pragma unroll
  for (int k = 0; k < 4; ++k) m = fmaxf(m, most[k][slot]);
  const float ref = m == NEG_INF ? 0.f : ceilf(m);
  float l = 0.f, p[RP];
#pragma unroll
  for (int j = 0; j < RP; ++j) {
    p[j] = exp2f(s[j] - ref);
    if constexpr (!F32) p[j] = (float)(__bf16)p[j];       // rounded where it enters the product with K, and the sum is of what enters
    l += p[j];
  }
  l = sum_over_lanes<P>(l);
  l += __shfl_xor(l, 32);
  if (i == 0 && half == 0) total[wave][slot] = l;
  const long o = ((long)b * a.H + hc) * a.Tp + t0 + first + i * RP;
  if (h < a.H) {
    if constexpr (F32) *(f32x2*)((float*)a.P + o) = f32x2{p[0], p[1]};
    else *(bf16x2*)((uint16_t*)a.P + o) = bf16x2{(__bf16)p[0], (__bf16)p[1]};
  }
  lds_barrier();
  if (wave == 0 && i == 0 && half == 0 && h < a.H) {
    const long x = ((long)b * a.H + h) * a.NB + blk;
    a.ref[x] = ref;
    a.sum[x] = (total[0][slot] + total[1][slot]) + (total[2][slot] + total[3][slot]);
  }
}

// ---- weighted sum of K ----------------------------------------------------------------------------------

// A split's blocks of one sequence: [blk0, blk1), none where the sequence is shorter
__device__ __forceinline__ bool split_blocks(const QDecodeArgs& a, int len, int split, int& blk0, int& blk1) {
  const int nb = (len + QUANT_ROWS - 1) / QUANT_ROWS;
  blk0 = split * a.per;
  blk1 = min(blk0 + a.per, nb);
  return blk0 < blk1;
}

// References of up to 32 heads for a split: the largest of its blocks, to LDS; the first column block notes them and the sums for the merge.
// Eight threads a head.  The first two blocks of a thread are asked for before the rows (loads come back in order).
struct SplitReferences {
  float ref[2], sum[2];
  __device__ __forceinline__ void ask(const QDecodeArgs& a, int b, int blk0, int blk1, int h0, int nh) {
    const int j = threadIdx.x >> 3, k = threadIdx.x & 7, h = min(h0 + j, a.H - 1);
    const long at = ((long)b * a.H + h) * a.NB;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int blk = min(blk0 + k + 8 * i, blk1 - 1);
      ref[i] = a.ref[at + blk];
      sum[i] = a.sum[at + blk];
    }
  }
  __device__ __forceinline__ void finish(const QDecodeArgs& a, int b, int split, int blk0, int blk1, int h0, int nh, bool note, float* mref) const {
    const int j = threadIdx.x >> 3, k = threadIdx.x & 7, h = min(h0 + j, a.H - 1);
    const long at = ((long)b * a.H + h) * a.NB;
    float m = fmaxf(ref[0], ref[1]), l = 0.f;          // (a block twice does not change the largest)
    for (int blk = blk0 + k + 16; blk < blk1; blk += 8) m = fmaxf(m, a.ref[at + blk]);
    m = max_over_lanes<8>(m);
    if (note) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (blk0 + k + 8 * i < blk1) l += sum[i] * exp2f(ref[i] - m);
      for (int blk = blk0 + k + 16; blk < blk1; blk += 8) l += a.sum[at + blk] * exp2f(a.ref[at + blk] - m);
      l = sum_over_lanes<8>(l);
    }
    if (k == 0 && j < nh) {
      mref[j] = m;
      if (note && h0 + j < a.H) {
        const long o = ((long)b * a.nsplit + split) * a.H + h0 + j;
        a.sref[o] = m;
        a.ssum[o] = l;
      }
    }
    lds_barrier();
  }
};

template <int BITS> struct Codes16;              // 16 columns of a row
template <> struct Codes16<4> { typedef u32x2 type; };
template <> struct Codes16<8> { typedef u32x4 type; };
template <int BITS, int K>
__device__ __forceinline__ unsigned bf16_pair(const typename Codes16<BITS>::type& w, float s) {
  if constexpr (BITS == 4) return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[K >> 2], s, K & 3));
  else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[K >> 1], s, (K & 1) != 0));
}

constexpr int QW_COLS = 256;                     // columns of a workgroup: 16 lanes x 16

// C[h][c] = sum_t p[h][t] K[t][c] on 16x16x32 matrix instructions: rows are heads, the contraction is over 32 cache rows, a lane holds eight rows x 16 columns and
// makes one column of operands after the other.  The four waves take every fourth 32 rows of the split and join through LDS in a fixed order.
// Bound by HBM for the codes where a sequence is long: 1 x 16384 rows x 32 x 128 in 4 bits 15 us, 7 of them the stream (5.1 TB/s), the rest the start (2.5), the waves'
// join and partial sums; 16 sequences of 600..5000 rows x 24 x 96 in 8 bits 28.6 us.
template <int BITS, int NT>
__global__ __launch_bounds__(256, 2) void qweighted_kernel(QDecodeArgs a) {
  typedef typename Codes16<BITS>::type W16;
  __shared__ float mref[32];
  __shared__ f32x4 join[4][3][4][64];            // [from][to: waves after it][operand]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ngroups = (a.H + 16 * NT - 1) / (16 * NT);
  const int b = blockIdx.z / ngroups, h0 = blockIdx.z % ngroups * 16 * NT, split = blockIdx.y;
  const int len = seq_len_of(a.seq_lens, b, a.T);
  int blk0, blk1;
  if (!split_blocks(a, len, split, blk0, blk1)) return;
  const int n = lane & 15, kg = lane >> 4;
  const int c = blockIdx.x * QW_COLS + n * 16;
  const int cc = min(c, a.d - 16);               // (columns past the row's end: anything, not stored)
  float m[NT];
  const uint16_t* P[NT];
  const float* R[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int h = min(h0 + t * 16 + n, a.H - 1);  // (heads past the last: anything, not stored)
    P[t] = (const uint16_t*)a.P + ((long)b * a.H + h) * a.Tp + kg * 8;
    R[t] = a.ref + ((long)b * a.H + h) * a.NB;
  }
  const long row_bytes = a.d * BITS / 8;
  // (a uniform pointer and a lane's offset: a pointer a lane and row would take 32 registers)
  const unsigned char* codes = a.codes + (long)b * a.stride * row_bytes;
  const unsigned at = (unsigned)(kg * 8 * (int)row_bytes + cc * BITS / 8);
  const unsigned char* scales = a.scales + ((long)b * (a.d / 32) + cc / 32) * a.stride + kg * 8;
  f32x4 acc[NT][16];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int step1 = min(blk1 * 2, (len + 31) / 32);
  struct Rows { W16 w[8]; u32x2 s; u32x4 p[NT]; float r[NT]; };
  auto fetch = [&](int k, Rows& x) {
    const long r0 = (long)k * 32;
#pragma unroll
    for (int i = 0; i < 8; ++i) x.w[i] = *(const W16*)(codes + (r0 + i) * row_bytes + at);
    x.s = *(const u32x2*)(scales + r0);
#pragma unroll
    for (int t = 0; t < NT; ++t) { x.p[t] = *(const u32x4*)(P[t] + r0); x.r[t] = R[t][k >> 1]; }
  };
  auto compute = [&](int k, Rows& x) {
    if (k * 32 + 32 > len) {
      // Rows behind the sequence may hold anything, and their numerators of zero would not make zero of a NaN.
      const int left = len - k * 32 - kg * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= left) {
          x.w[i] = W16{};
          x.s[i >> 2] &= ~(0xffu << (8 * (i & 3)));
        }
    }
    bf16x8 A[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      // relative to the split's reference: so many binades less
      const unsigned sh = (unsigned)fminf(fmaxf(m[t] - x.r[t], 0.f), 255.f) << 7;
      const u16x2 by = {(unsigned short)sh, (unsigned short)sh};
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned w = x.p[t][j];              // (a bit cast of the element itself takes the vector's first, whatever j is)
        v[j] = __builtin_bit_cast(unsigned, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, w), by));
      }
      A[t] = __builtin_bit_cast(bf16x8, v);
    }
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = scale_of(x.s[i >> 2], i & 3);
    auto pair = [&](int, auto K) {
      constexpr int kk = decltype(K)::value;
      unsigned y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = bf16_pair<BITS, kk>(x.w[i], s[i]);
      u32x4 lo, hi;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lo[i] = __builtin_amdgcn_perm(y[2 * i + 1], y[2 * i], 0x05040100u);
        hi[i] = __builtin_amdgcn_perm(y[2 * i + 1], y[2 * i], 0x07060302u);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        acc[t][2 * kk] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A[t], __builtin_bit_cast(bf16x8, lo), acc[t][2 * kk], 0, 0, 0);
        acc[t][2 * kk + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A[t], __builtin_bit_cast(bf16x8, hi), acc[t][2 * kk + 1], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);           // (all operands made ahead of the products do not fit the registers)
    };
    full_steps<0, 8>(0, pair);
  };
  // One loop with the next rows in a second set of registers, copied: with the two sets in turn the accumulators were copied instead, and went to scratch.
  int k = blk0 * 2 + wave;
  SplitReferences refs;
  refs.ask(a, b, blk0, blk1, h0, 16 * NT);
  Rows x;
  if (k < step1) fetch(k, x);
  refs.finish(a, b, split, blk0, blk1, h0, 16 * NT, blockIdx.x == 0, mref);
#pragma unroll
  for (int t = 0; t < NT; ++t) m[t] = mref[min(h0 + t * 16 + n, a.H - 1) - h0];
  if (k < step1) {
#pragma unroll 1
    for (;;) {
      Rows next;
      int kn = min(k + 4, step1 - 1);             // (past the wave's last step: rows that nothing takes)
      asm volatile("" : "+s"(kn));               // (pointers are made anew each time, from uniform ones: kept across the loop they take 40 registers)
      fetch(kn, next);
      compute(k, x);
      k += 4;
      if (k >= step1) break;
      x = next;
    }
  }
  // Wave w ends with operands 4 w .. 4 w + 3 of every tile: for each tile the waves hand the others their quarters and add what they get in the order
  // of the waves from their own on.  (Constant indices: with the wave's own quarter picked at run time the accumulators went to scratch, 27 us for a launch
  // that takes 8.  One quarter after the other, three waves looking on, took 3.6 us.)
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int qd = 0; qd < 4; ++qd)
      if (wave != qd) {
#pragma unroll
        for (int j = 0; j < 4; ++j) join[wave][(qd - wave - 1) & 3][j][lane] = acc[t][qd * 4 + j];
      }
    lds_barrier();
#pragma unroll
    for (int qd = 0; qd < 4; ++qd)
      if (wave == qd) {
        f32x4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[j] = acc[t][qd * 4 + j];
#pragma unroll
          for (int w = 1; w < 4; ++w) v[j] += join[(qd + w) & 3][3 - w][j][lane];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int h = h0 + t * 16 + kg * 4 + i;
          if (h < a.H && c < a.d)
            *(f32x4*)(a.C + (((long)b * a.nsplit + split) * a.H + h) * a.d + c + qd * 4) = f32x4{v[0][i], v[1][i], v[2][i], v[3][i]};
        }
      }
    if (t + 1 < NT) lds_barrier();
  }
}

// The same in fp32 on the vector ALU: a thread has eight columns and eight heads, numerators are uniform.  For caches of layers that are kept in full precision.
template <int BITS>
__global__ __launch_bounds__(256) void qweighted_f32_kernel(QDecodeArgs a) {
  __shared__ float mref[32];
  __shared__ float join[3][64][65];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int ngroups = (a.H + 7) / 8;
  const int b = blockIdx.z / ngroups, h0 = blockIdx.z % ngroups * 8, split = blockIdx.y;
  const int len = seq_len_of(a.seq_lens, b, a.T);
  int blk0, blk1;
  if (!split_blocks(a, len, split, blk0, blk1)) return;
  SplitReferences refs;
  refs.ask(a, b, blk0, blk1, h0, 8);
  refs.finish(a, b, split, blk0, blk1, h0, 8, blockIdx.x == 0, mref);
  const int c = blockIdx.x * 512 + lane * 8, cc = min(c, a.d - 8);
  const long row_bytes = a.d * BITS / 8;
  const unsigned char* codes = a.codes + (long)b * a.stride * row_bytes + (long)cc * BITS / 8;
  const unsigned char* scales = a.scales + ((long)b * (a.d / 32) + cc / 32) * a.stride;
  float acc[8][8];
#pragma unroll
  for (int h = 0; h < 8; ++h)
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[h][j] = 0.f;
  const float* P[8];
  float f[8];
#pragma unroll
  for (int h = 0; h < 8; ++h) P[h] = (const float*)a.P + ((long)b * a.H + min(h0 + h, a.H - 1)) * a.Tp;
  for (int blk = blk0; blk < blk1; ++blk) {
#pragma unroll
    for (int h = 0; h < 8; ++h) {
      const int hh = min(h0 + h, a.H - 1);
      f[h] = exp2f(a.ref[((long)b * a.H + hh) * a.NB + blk] - mref[hh - h0]);
    }
    const int t1 = min((blk + 1) * QUANT_ROWS, len);
    for (int t = blk * QUANT_ROWS + wave; t < t1; t += 4) {       // (the waves: every fourth row)
      Codes8<BITS> w;
      w.load(codes + t * row_bytes);
      const float s = __uint_as_float((unsigned)scales[t] << 23);
      const f32x2 y0 = w.template f32<0>(s), y1 = w.template f32<1>(s), y2 = w.template f32<2>(s), y3 = w.template f32<3>(s);
      const float y[8] = {y0[0], y0[1], y1[0], y1[1], y2[0], y2[1], y3[0], y3[1]};
#pragma unroll
      for (int h = 0; h < 8; ++h) {
        const float p = P[h][t] * f[h];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[h][j] = fmaf(p, y[j], acc[h][j]);
      }
    }
  }
  for (int w = 1; w < 4; ++w) {
    if (wave == w)
#pragma unroll
      for (int h = 0; h < 8; ++h)
#pragma unroll
        for (int j = 0; j < 8; ++j) join[w - 1][h * 8 + j][lane] = acc[h][j];
  }
  __syncthreads();
  if (wave != 0 || c >= a.d) return;
#pragma unroll
  for (int h = 0; h < 8; ++h) {
    if (h0 + h >= a.H) continue;
    float* o = a.C + (((long)b * a.nsplit + split) * a.H + h0 + h) * a.d + c;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = acc[h][j] + join[0][h * 8 + j][lane] + join[1][h * 8 + j][lane] + join[2][h * 8 + j][lane];
  }
}

// ---- merge of the splits and projection -------------------------------------------------------------------

constexpr int QP_BATCH = 16, QP_COLS = 128, QP_MAX_SPLITS = 64, QP_MAX_ROWS = 256;

// Weights of a batch tile's splits for head h: 2^(reference - largest) / sum; zero for splits that a sequence does not have, and for sequences without rows
__device__ __forceinline__ void split_weights(const QDecodeArgs& a, int b0, int h, float (&wt)[QP_BATCH][QP_MAX_SPLITS + 1]) {
  // 16 threads a sequence
  const int j = threadIdx.x >> 4, k = threadIdx.x & 15, b = b0 + j;
  const int len = b < a.B ? seq_len_of(a.seq_lens, b, a.T) : 0;
  const int nb = (len + QUANT_ROWS - 1) / QUANT_ROWS, used = (nb + a.per - 1) / a.per;
  const long at = (long)min(b, a.B - 1) * a.nsplit * a.H + h;
  float ref[QP_MAX_SPLITS / 16], sum[QP_MAX_SPLITS / 16], m = NEG_INF, l = 0.f;
#pragma unroll
  for (int i = 0; i < QP_MAX_SPLITS / 16; ++i) {       // (all on their way at once; splits that the sequence does not have hold anything)
    const long s = at + (long)min(k + 16 * i, a.nsplit - 1) * a.H;
    ref[i] = a.sref[s];
    sum[i] = a.ssum[s];
  }
#pragma unroll
  for (int i = 0; i < QP_MAX_SPLITS / 16; ++i) {
    if (k + 16 * i >= used) { ref[i] = NEG_INF; sum[i] = 0.f; }
    m = fmaxf(m, ref[i]);
  }
  m = max_over_lanes<16>(m);
#pragma unroll
  for (int i = 0; i < QP_MAX_SPLITS / 16; ++i)
    if (k + 16 * i < used) l += sum[i] * (ref[i] = exp2f(ref[i] - m));
  l = sum_over_lanes<16>(l);
#pragma unroll
  for (int i = 0; i < QP_MAX_SPLITS / 16; ++i)
    if (k + 16 * i < a.nsplit) wt[j][k + 16 * i] = k + 16 * i < used ? ref[i] / l : 0.f;
  if (k == 0) wt[j][QP_MAX_SPLITS] = __int_as_float(used);
}

// out[b][h d_k + j] = sum_c C[b][h][c] W[c][h d_k + j].  A workgroup takes a head, up to 128 of its columns, 16 sequences and a row split of W: it merges the
// splits' partial sums into LDS (as bf16 hi + lo, which keeps 16 bits of them; W is bf16), multiplies on 16x16x32 matrix instructions, and whoever of a
// head's row splits comes last adds their results in the order of their numbers.  HBM-bound on W for small batches: 1 x 4096 x 4096 12.6 us, 6.4 of them W at 5.2 TB/s, 2 the
// start, 3 the meeting of the row splits.  (Sixteen columns and all rows a workgroup, which needs no meeting, took 16: pieces of 32 bytes.)
template <bool F32>
__global__ __launch_bounds__(256) void qproject_kernel(QDecodeArgs a) {
  __shared__ float wt[QP_BATCH][QP_MAX_SPLITS + 1];
  __shared__ __align__(16) char operand[F32 ? QP_BATCH * QP_MAX_ROWS * 4 : 2 * QP_BATCH * (QP_MAX_ROWS + 8) * 2];
  __shared__ f32x4 join[4][8][64];
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ct = (a.d_k + QP_COLS - 1) / QP_COLS;
  const int h = blockIdx.x / ct, j0 = blockIdx.x % ct * QP_COLS, rs = blockIdx.y, b0 = blockIdx.z * QP_BATCH;
  const int cr0 = rs * a.crows, rows = min(a.crows, a.d - cr0);
  // W's first rows are on their way while the splits are merged: all of a workgroup's, 256 at the most.
  const int nj = min(QP_COLS, a.d_k - j0), n = lane & 15, kg = lane >> 4;
  const bool in = n * 8 < nj;
  u32x4 w[F32 ? 1 : 2][8];
  if constexpr (!F32) {
    const uint16_t* W = (const uint16_t*)a.W + (long)h * a.d_k + j0 + (in ? n * 8 : 0);
#pragma unroll
    for (int x = 0; x < 2; ++x)
      if (wave * 32 + x * 128 < rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[x][i] = *(const u32x4*)(W + (long)(cr0 + wave * 32 + x * 128 + kg * 8 + i) * a.d);      // (32 rows: all there or none)
      }
  }
  split_weights(a, b0, h, wt);
  __syncthreads();
  // Merge: four columns a lane.  A wave takes four sequences, or with one or two of them a quarter or half of the splits; sixteen loads are on their way at once.
  {
    const int seqs = min(QP_BATCH, a.B - b0), padded = F32 ? rows : (rows + 31) / 32 * 32, r = lane * 4;
    const float* src = a.C + (long)h * a.d + cr0 + min(r, rows - 4);
    const long step = (long)a.H * a.d;
    auto store = [&](int j, f32x4 v) {
      if (r >= padded) return;
      if constexpr (F32) {
        *(f32x4*)(operand + (j * QP_MAX_ROWS + r) * 4) = v;
      } else {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        bf16x4 hi, lo;
#pragma unroll
        for (int k = 0; k < 4; ++k) { hi[k] = (__bf16)v[k]; lo[k] = (__bf16)(v[k] - (float)hi[k]); }
        *(bf16x4*)(operand + (j * (QP_MAX_ROWS + 8) + r) * 2) = hi;
        *(bf16x4*)(operand + ((QP_BATCH + j) * (QP_MAX_ROWS + 8) + r) * 2) = lo;
      }
    };
    // (behind the last split: the last again, with a weight of zero)
    if (seqs > 2) {
      int used[4], most = 0;
      f32x4 v[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        used[y] = __builtin_amdgcn_readfirstlane(__float_as_int(wt[wave * 4 + y][QP_MAX_SPLITS]));
        most = max(most, used[y]);
        v[y] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      for (int s0 = 0; s0 < most; s0 += 4) {
        f32x4 x[4][4];
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[y][i] = *(const f32x4*)(src + ((long)min(b0 + wave * 4 + y, a.B - 1) * a.nsplit + max(min(s0 + i, used[y] - 1), 0)) * step);
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (s0 + i < used[y]) {
              const float f = wt[wave * 4 + y][s0 + i];
#pragma unroll
              for (int k = 0; k < 4; ++k) v[y][k] = fmaf(f, x[y][i][k], v[y][k]);
            }
      }
#pragma unroll
      for (int y = 0; y < 4; ++y) store(wave * 4 + y, v[y]);
    } else {
      f32x4* parts = &join[0][0][0];
      const int G = seqs == 2 ? 2 : 4, j = wave / G;
      const int used = __builtin_amdgcn_readfirstlane(__float_as_int(wt[j][QP_MAX_SPLITS]));
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      for (int s0 = wave % G; s0 < used; s0 += 16 * G) {
        f32x4 x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = *(const f32x4*)(src + ((long)(b0 + j) * a.nsplit + min(s0 + i * G, used - 1)) * step);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (s0 + i * G < used) {
            const float f = wt[j][s0 + i * G];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = fmaf(f, x[i][k], v[k]);
          }
      }
      parts[wave * 64 + lane] = v;
      __syncthreads();
      if (wave % G == 0) {
        for (int g = 1; g < G; ++g) v += parts[(wave + g) * 64 + lane];
        store(j, v);
      }
      for (int z = 4 / G + wave; z < QP_BATCH; z += 4) store(z, f32x4{0.f, 0.f, 0.f, 0.f});       // (rows of the operand without a sequence)
    }
  }
  __syncthreads();
  float mine[8];                                 // this thread's results: sequence tid / 16, columns 8 (tid % 16) ...
  if constexpr (!F32) {
    f32x4 acc[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int r = wave * 32 + x * 128;
      if (r >= rows) break;
      u32x4 t[8];
      transpose8x8(w[x], t);
      const bf16x8 hi = *(const bf16x8*)(operand + (n * (QP_MAX_ROWS + 8) + r + kg * 8) * 2);
      const bf16x8 lo = *(const bf16x8*)(operand + ((QP_BATCH + n) * (QP_MAX_ROWS + 8) + r + kg * 8) * 2);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hi, __builtin_bit_cast(bf16x8, t[j]), acc[j], 0, 0, 0);
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lo, __builtin_bit_cast(bf16x8, t[j]), acc[j], 0, 0, 0);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) join[wave][j][lane] = acc[j];
    __syncthreads();
    // row m of a product is lane group m / 4, element m % 4
    const int m = tid >> 4, from = (m >> 2) * 16 + (tid & 15);
#pragma unroll
    for (int j = 0; j < 8; ++j) mine[j] = (join[0][j][from][m & 3] + join[1][j][from][m & 3]) + (join[2][j][from][m & 3] + join[3][j][from][m & 3]);
  } else {
    const float* C = (const float*)operand + (tid >> 4) * QP_MAX_ROWS;
    const int c = (tid & 15) * 8;
    const float* W = (const float*)a.W + (long)cr0 * a.d + (long)h * a.d_k + j0 + (c < nj ? c : 0);
#pragma unroll
    for (int j = 0; j < 8; ++j) mine[j] = 0.f;
    for (int r = 0; r < rows; ++r) {
      const f32x4 lo = *(const f32x4*)(W + (long)r * a.d), hi = *(const f32x4*)(W + (long)r * a.d + 4);
      const float x = C[r];
#pragma unroll
      for (int k = 0; k < 4; ++k) { mine[k] = fmaf(x, lo[k], mine[k]); mine[4 + k] = fmaf(x, hi[k], mine[4 + k]); }
    }
  }
  const int b = b0 + (tid >> 4), c = (tid & 15) * 8;
  const bool mine_there = b < a.B && c < nj;
  const long o = (long)b * a.d + (long)h * a.d_k + j0 + c;
  if (a.csw > 1) {
    // Partial results go past the L2s (each XCD has its own) and are read past them: a fence would write all of an L2 back, 60 us for the launch.
    if (mine_there) {
      unsigned long long* p = (unsigned long long*)(a.part + (long)rs * a.B * a.d + o);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        __hip_atomic_store(p + j, (unsigned long long)__float_as_uint(mine[2 * j]) | (unsigned long long)__float_as_uint(mine[2 * j + 1]) << 32, __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0)
      last = __hip_atomic_fetch_add(a.counters + blockIdx.z * gridDim.x + blockIdx.x, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.csw - 1;
    __syncthreads();
    if (!last) return;
    if (mine_there) {
#pragma unroll
      for (int j = 0; j < 8; ++j) mine[j] = 0.f;
#pragma unroll 8
      for (int s = 0; s < a.csw; ++s) {
        const unsigned long long* p = (const unsigned long long*)(a.part + (long)s * a.B * a.d + o);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const unsigned long long x = __hip_atomic_load(p + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          mine[2 * j] += __uint_as_float((unsigned)x);
          mine[2 * j + 1] += __uint_as_float((unsigned)(x >> 32));
        }
      }
    }
  }
  if (!mine_there) return;
  if constexpr (F32) {
    f32x4* p = (f32x4*)((float*)a.out + o);
    p[0] = f32x4{mine[0], mine[1], mine[2], mine[3]};
    p[1] = f32x4{mine[4], mine[5], mine[6], mine[7]};
  } else {
    bf16x8 v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (__bf16)mine[j];
    *(bf16x8*)((uint16_t*)a.out + o) = v;
  }
}

template <bool F32, int BITS, int P>
void scores_of(const QDecodeArgs& a, hipStream_t st) {
  const int hw = 4 * 64 / P;
  const dim3 grid(a.NB, (a.H + hw - 1) / hw, a.B);
  if (a.rope) qscores_kernel<F32, BITS, P, true><<<grid, 256, 0, st>>>(a);
  else qscores_kernel<F32, BITS, P, false><<<grid, 256, 0, st>>>(a);
}
template <bool F32, int BITS, int CH>
void even_scores(const QDecodeArgs& a, hipStream_t st) {
  const dim3 grid((a.H + 7) / 8 * a.B, a.NB < 32768 ? a.NB : 32768, (a.NB + 32767) / 32768);
  if (a.rope) qscores_even_kernel<F32, BITS, CH, true><<<grid, 256, 0, st>>>(a);
  else qscores_even_kernel<F32, BITS, CH, false><<<grid, 256, 0, st>>>(a);
}
template <bool F32, int BITS>
void scores_by_width(const QDecodeArgs& a, hipStream_t st) {
  if (a.d_k == 32) even_scores<F32, BITS, 1>(a, st);
  else if (a.d_k == 64) even_scores<F32, BITS, 2>(a, st);
  else if (a.d_k == 96) even_scores<F32, BITS, 3>(a, st);
  else if (a.d_k == 128) even_scores<F32, BITS, 4>(a, st);
  else if (a.d_k <= 32) scores_of<F32, BITS, 4>(a, st);
  else if (a.d_k <= 64) scores_of<F32, BITS, 8>(a, st);
  else if (a.d_k <= 128) scores_of<F32, BITS, 16>(a, st);
  else if (a.d_k <= 256) scores_of<F32, BITS, 32>(a, st);
  else scores_of<F32, BITS, 64>(a, st);
}

}  // namespace

int qdecode_counters(int B, int H, int d) { return H * ((d / H + QP_COLS - 1) / QP_COLS) * ((B + QP_BATCH - 1) / QP_BATCH); }

// How the work is cut.  Splits of the weighted sum: a workgroup for every compute unit (with two, one sequence of 16384 rows x 4096 took 18.6 us instead of 15.9, as
// much more to write and merge), but of 1024 rows at the most where that does not make more than four a unit: sequences of a batch are not equally long (16 of up
// to 5000 rows x 2304 in 8 bits: two splits 38.6 us, four 28.6).  128 rows at least: a step of 32 for every wave.  Row splits of W: a workgroup a unit, 256 rows at the most.
static long weighted_units(int dtype, int H, int d) {          // workgroups of a split of one sequence
  return dtype == DT_F32 ? (long)((d + 511) / 512) * ((H + 7) / 8) : (long)((d + QW_COLS - 1) / QW_COLS) * ((H + 31) / 32);
}
static long wanted_splits(int nb, long units) {
  const long want = (256 + units - 1) / units, even = std::min<long>((nb + 15) / 16, 1024 / units);
  return std::min<long>(std::max(want, even), QP_MAX_SPLITS);
}
static long wanted_row_splits(int d, long tiles) {
  return std::min<long>(std::max<long>((256 + tiles - 1) / tiles, (d + QP_MAX_ROWS - 1) / QP_MAX_ROWS), d / 32);
}
void qdecode_cut(int dtype, int B, int H, int T, int d, int* per, int* nsplit, int* csw, int* crows) {
  const int nb = (T + QUANT_ROWS - 1) / QUANT_ROWS;
  const long want = wanted_splits(nb, B * weighted_units(dtype, H, d));
  *per = std::max((int)((nb + want - 1) / want), 2);
  *nsplit = (nb + *per - 1) / *per;
  const long c = wanted_row_splits(d, qdecode_counters(B, H, d));
  *crows = (int)(((d + c - 1) / c + 31) / 32 * 32);
  *csw = (d + *crows - 1) / *crows;
}

// The splits themselves go up and down with T, and with B they go down faster than it goes up: B ceil(x / B) <= x + B - 1, B floor(y / B) <= y, and a sequence has no more
// splits in a larger batch than by itself.
size_t qdecode_most_splits(int dtype, int B, int H, int T, int d) {
  const int nb = (T + QUANT_ROWS - 1) / QUANT_ROWS;
  const long units = weighted_units(dtype, H, d), alone = std::min<long>((nb + 1) / 2, wanted_splits(nb, units));
  return std::min(B * alone, std::max((256 + units - 1) / units + B - 1, std::min((long)B * ((nb + 15) / 16), 1024 / units)));
}
// The same for the row splits of W, sixteen sequences at a time.
size_t qdecode_most_row_splits(int B, int H, int d) {
  const long tiles = qdecode_counters(1, H, d), least = (d + QP_MAX_ROWS - 1) / QP_MAX_ROWS, groups = (B + QP_BATCH - 1) / QP_BATCH;
  const long alone = wanted_row_splits(d, tiles);
  return alone > 1 ? std::min(B * alone, std::max(QP_BATCH * ((256 + tiles - 1) / tiles + groups - 1), B * least)) : 0;
}

void launch_qdecode_scores(int dtype, const QDecodeArgs& a, hipStream_t st) {
  if (dtype == DT_F32) {
    if (a.bits == 4) scores_by_width<true, 4>(a, st); else scores_by_width<true, 8>(a, st);
  } else {
    if (a.bits == 4) scores_by_width<false, 4>(a, st); else scores_by_width<false, 8>(a, st);
  }
}

void launch_qdecode_weighted(int dtype, const QDecodeArgs& a, hipStream_t st) {
  if (dtype == DT_F32) {
    const dim3 grid((a.d + 511) / 512, a.nsplit, a.B * ((a.H + 7) / 8));
    if (a.bits == 4) qweighted_f32_kernel<4><<<grid, 256, 0, st>>>(a);
    else qweighted_f32_kernel<8><<<grid, 256, 0, st>>>(a);
    return;
  }
  const int cols = (a.d + QW_COLS - 1) / QW_COLS;
  if (a.H <= 16) {
    const dim3 grid(cols, a.nsplit, a.B);
    if (a.bits == 4) qweighted_kernel<4, 1><<<grid, 256, 0, st>>>(a);
    else qweighted_kernel<8, 1><<<grid, 256, 0, st>>>(a);
  } else {
    const dim3 grid(cols, a.nsplit, a.B * ((a.H + 31) / 32));
    if (a.bits == 4) qweighted_kernel<4, 2><<<grid, 256, 0, st>>>(a);
    else qweighted_kernel<8, 2><<<grid, 256, 0, st>>>(a);
  }
}

void launch_qdecode_project(int dtype, const QDecodeArgs& a, hipStream_t st) {
  const int ct = (a.d_k + QP_COLS - 1) / QP_COLS;
  const dim3 grid(a.H * ct, a.csw, (a.B + QP_BATCH - 1) / QP_BATCH);
  if (dtype == DT_F32) qproject_kernel<true><<<grid, 256, 0, st>>>(a);
  else qproject_kernel<false><<<grid, 256, 0, st>>>(a);
}

}  // namespace slim
