// K-caches held in 4 or 8 bits: rows quantised as they are written, rows read back, and the decode step that reads them.
//
// A row's columns form groups of 32 that share a power of two 2^s; an element is an e2m1 (4 bits: 0, 0.5, 1, 1.5, 2, 3, 4, 6) or e4m3 (8 bits, up to 448) value
// times it.  Codes lie row by row, the scale bytes (s + 127; 255: the group is not a number) group by group, so that the scales of consecutive rows are
// consecutive bytes: whoever reads R rows of a group takes its R scales in one load.
//
// The conversions are the CU's own (v_cvt_scalef32_*): they round to the nearest value, ties to even, take 2^s from the exponent of a float (255 there
// gives NaN, 0 is 2^-127), and what they make of a code is exact in bf16, a significand of four bits at most under any exponent.
#include "device_common.h"
#include "slim_kernels.h"

namespace slim {
namespace {

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int TILE_T = 64, TILE_C = 256;      // rows and columns of a workgroup that converts

__device__ __forceinline__ float pow2_of(unsigned byte) { return __uint_as_float(byte << 23); }

// Where packed row r goes: sequence and row of its cache (b < 0: nowhere).  Without offsets the sequences bring the same number of rows each.
__device__ __forceinline__ void place_of(const QuantArgs& a, int r, int& b, long& t) {
  b = -1;
  t = 0;
  if (r >= a.n_rows) return;
  int first;
  if (a.cu) {
    int lo = 0, hi = a.B;                      // the last sequence that starts at or before r (empty ones before it share its start)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.cu[mid] <= r) lo = mid; else hi = mid;
    }
    first = a.cu[lo];
    if (r < first || r >= a.cu[lo + 1]) return;
    b = lo;
  } else {
    const int per = a.n_rows / a.B;
    b = r / per;
    first = b * per;
  }
  t = (long)(a.start ? a.start[b] : 0) + ((long)r - first);      // (offsets may be anything: 32 bits could wrap into the cache)
  if (t < 0 || t >= a.T) t = -1;
}

// Rows -> codes and scales.  A workgroup takes 64 packed rows x 256 columns: eight columns a thread (16 bytes of bf16 in, four or eight bytes of codes out), a group is
// four lanes.  The scale bytes go through LDS, so that a group's bytes of consecutive rows leave in one store.  HBM-bound: 2 + 0.53 bytes an element; 18560 rows x
// 4096 in 4 bits 47 us, 4.1 TB/s (reading the rows alone takes 28.5).  The rows are read past the caches, which they fill to no use: 52 us without.
template <bool F32, int BITS>
__global__ __launch_bounds__(256) void quant_append_kernel(QuantArgs a) {
  __shared__ long at[TILE_T];                  // row of all caches, -1: nowhere
  __shared__ unsigned char sc[TILE_C / 32][TILE_T];
  const int tid = threadIdx.x, cols = (a.d + TILE_C - 1) / TILE_C, r0 = blockIdx.x / cols * TILE_T, c0 = blockIdx.x % cols * TILE_C;
  const int c = c0 + (tid & 31) * 8, rr = tid >> 5;
  const bool in = c < a.d;
  // (all loads without a branch, so that they are on their way together: rows and columns past the end are the last ones again, and not stored)
  const int cc = in ? c : 0;
  u32x4 v[8][F32 ? 2 : 1];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long r = min(r0 + rr + 8 * i, a.n_rows - 1);
    const u32x4* src = F32 ? (const u32x4*)((const float*)a.rows + r * a.pitch + cc) : (const u32x4*)((const uint16_t*)a.rows + r * a.pitch + cc);
#pragma unroll
    for (int k = 0; k < (F32 ? 2 : 1); ++k) v[i][k] = __builtin_nontemporal_load(src + k);
  }
  if (tid < TILE_T) {
    int b; long t;
    place_of(a, r0 + tid, b, t);
    at[tid] = b < 0 || t < 0 ? -1 : b * a.stride + t;
  }
  __syncthreads();
  constexpr int EMAX = BITS == 4 ? 2 : 8;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // The largest magnitude as bits: of floats without a sign the order is that of the integers, and what is not finite is above all others.
    float x[8];
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (F32) x[j] = __uint_as_float(v[i][j >> 2][j & 3]);
      else x[j] = __uint_as_float(j & 1 ? v[i][0][j >> 1] & 0xffff0000u : v[i][0][j >> 1] << 16);
      m = max(m, __float_as_uint(x[j]) & 0x7fffffffu);
    }
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true));
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true));
    // Its exponent, one more over a significand of 1.75: 6 and 448 are that much of their binade, so that an element is cut off by a seventh of itself at the
    // most (4 bits; at 8 bits nothing is).  Under 2^-126 floats have no exponent: the smallest scale holds there all the same.
    unsigned s = m >= 0x7f800000u ? 255u : (unsigned)min(max((int)((m + 0x1fffffu) >> 23) - EMAX, 0), 254 - EMAX);
    const float scale = pow2_of(s);
    const int row = rr + 8 * i;
    const long to = at[row];
    if (in && to >= 0) {
      if constexpr (BITS == 4) {
        unsigned w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
        *(unsigned*)(a.codes + to * (a.d / 2) + c / 2) = s == 255u ? 0u : w;
      } else {
        // (Only magnitudes above 1.75 x 2^127 are over 448 of the largest scale; the conversion would make NaN of them.)
        const float top = 448.f * pow2_of(254 - EMAX);
        s16x2 w0 = {0, 0}, w1 = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fminf(fmaxf(x[j], -top), top);
        w0 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w0, x[0], x[1], scale, false);
        w0 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w0, x[2], x[3], scale, true);
        w1 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w1, x[4], x[5], scale, false);
        w1 = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w1, x[6], x[7], scale, true);
        const u32x2 w = {__builtin_bit_cast(unsigned, w0), __builtin_bit_cast(unsigned, w1)};
        *(u32x2*)(a.codes + to * a.d + c) = s == 255u ? u32x2{0u, 0u} : w;
      }
    }
    if ((tid & 3) == 0) sc[(tid & 31) >> 2][row] = (unsigned char)s;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < TILE_C / 32 / 4; ++k) {
    const int row = tid & 63, g = (tid >> 6) + 4 * k;
    const long to = at[row];
    if (to < 0 || c0 + g * 32 >= a.d) continue;
    const long b = to / a.stride, t = to - b * a.stride;
    a.scales[(b * (a.d / 32) + c0 / 32 + g) * a.stride + t] = sc[g][row];
  }
}

// Codes and scales -> rows, the same tiles.  Rows past the cache's T are zeros; rows of no sequence are left as they are.  HBM-bound: 7777 rows x 4096 in 8 bits to
// bf16 16 us, 6 TB/s; 18560 rows in 4 bits 38 us, 5.1 TB/s.
template <bool F32, int BITS>
__global__ __launch_bounds__(256) void quant_read_kernel(QuantArgs a) {
  __shared__ long at[TILE_T];                  // row of all caches, -1: a row of zeros, -2: no row
  __shared__ unsigned char sc[TILE_C / 32][TILE_T];
  const int tid = threadIdx.x, cols = (a.d + TILE_C - 1) / TILE_C, r0 = blockIdx.x / cols * TILE_T, c0 = blockIdx.x % cols * TILE_C;
  if (tid < TILE_T) {
    int b; long t;
    place_of(a, r0 + tid, b, t);
    at[tid] = b < 0 ? -2 : t < 0 ? -1 : b * a.stride + t;
  }
  __syncthreads();
  const int c = c0 + (tid & 31) * 8, rr = tid >> 5;
  const bool in = c < a.d;
  u32x2 w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long from = max(at[rr + 8 * i], 0l);   // (without a branch: a row of zeros or none reads the first row's codes, for nothing)
    if constexpr (BITS == 4) w[i][0] = *(const unsigned*)(a.codes + from * (a.d / 2) + (in ? c : 0) / 2);
    else w[i] = *(const u32x2*)(a.codes + from * a.d + (in ? c : 0));
  }
#pragma unroll
  for (int k = 0; k < TILE_C / 32 / 4; ++k) {
    const int row = tid & 63, g = (tid >> 6) + 4 * k;
    const long from = at[row];
    unsigned char s = 0;
    if (from >= 0 && c0 + g * 32 < a.d) {
      const long b = from / a.stride, t = from - b * a.stride;
      s = a.scales[(b * (a.d / 32) + c0 / 32 + g) * a.stride + t];
    }
    sc[g][row] = s;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = rr + 8 * i;
    if (!in || at[row] == -2) continue;
    const float scale = pow2_of(sc[(tid & 31) >> 2][row]);
    const long o = (long)(r0 + row) * a.pitch + c;
    if (at[row] == -1) w[i] = u32x2{0u, 0u};
    if constexpr (F32) {
      f32x2 v[4];
      if constexpr (BITS == 4) {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i][0], scale, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i][0], scale, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i][0], scale, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[i][0], scale, 3);
      } else {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i][0], scale, false);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i][0], scale, true);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i][1], scale, false);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i][1], scale, true);
      }
      f32x4* dst = (f32x4*)((float*)a.out + o);
      dst[0] = f32x4{v[0][0], v[0][1], v[1][0], v[1][1]};
      dst[1] = f32x4{v[2][0], v[2][1], v[3][0], v[3][1]};
    } else {
      u32x4 v;
      if constexpr (BITS == 4) {
        v[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i][0], scale, 0));
        v[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i][0], scale, 1));
        v[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i][0], scale, 2));
        v[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i][0], scale, 3));
      } else {
        v[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i][0], scale, false));
        v[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i][0], scale, true));
        v[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i][1], scale, false));
        v[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i][1], scale, true));
      }
      *(u32x4*)((uint16_t*)a.out + o) = v;
    }
  }
}

// Neighbouring workgroups have neighbouring columns: with neighbouring rows instead, 18560 rows of 4096 columns were read in pieces 8 KB apart at any one time.
unsigned tiles_of(const QuantArgs& a) { return (unsigned)((a.n_rows + TILE_T - 1) / TILE_T) * (unsigned)((a.d + TILE_C - 1) / TILE_C); }

}  // namespace

void launch_quant_append(int dtype, int bits, const QuantArgs& a, hipStream_t st) {
  const unsigned grid = tiles_of(a);
  if (dtype == DT_F32) {
    if (bits == 4) quant_append_kernel<true, 4><<<grid, 256, 0, st>>>(a);
    else quant_append_kernel<true, 8><<<grid, 256, 0, st>>>(a);
  } else {
    if (bits == 4) quant_append_kernel<false, 4><<<grid, 256, 0, st>>>(a);
    else quant_append_kernel<false, 8><<<grid, 256, 0, st>>>(a);
  }
}

void launch_quant_read(int dtype, int bits, const QuantArgs& a, hipStream_t st) {
  const unsigned grid = tiles_of(a);
  if (dtype == DT_F32) {
    if (bits == 4) quant_read_kernel<true, 4><<<grid, 256, 0, st>>>(a);
    else quant_read_kernel<true, 8><<<grid, 256, 0, st>>>(a);
  } else {
    if (bits == 4) quant_read_kernel<false, 4><<<grid, 256, 0, st>>>(a);
    else quant_read_kernel<false, 8><<<grid, 256, 0, st>>>(a);
  }
}

}  // namespace slim
