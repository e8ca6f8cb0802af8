// Attention over whole prompts in bf16: causal or full, grouped heads, packed sequences.
#include <algorithm>

#include "prompt_common.h"

namespace slim {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int PK = 64;                         // keys of a tile

// 16-byte pieces of a row in LDS: a power of two, so that they can be swapped among themselves by the row's number.  Keys are read with lanes on consecutive
// rows, 16 bytes each; values with four rows x 32 bytes for every 16 lanes.  Either way the rows of one access shall lie in different banks.
template <int DKP> struct Pitch { static constexpr int pieces = DKP <= 32 ? 4 : DKP <= 64 ? 8 : DKP <= 128 ? 16 : 32; };
template <int PC> __device__ __forceinline__ int k_swap(int row) { return PC >= 16 ? row & 15 : PC == 8 ? (row >> 1) & 7 : (row >> 2) & 3; }
template <int PC> __device__ __forceinline__ int v_swap(int row) { return PC >= 16 ? (row & 3) << 2 : PC == 8 ? (row & 2) << 1 : 0; }

// One pass over the keys with a running reference and sum a query; 128 queries a workgroup, 32 a wave, tiles of 64 keys in two LDS buffers (two workgroups a compute
// unit).  Products are 32x32x16: S^T = K Q^T, whose result has a query's scores in two lanes, so that
// maxima and sums are the lane's own but for one exchange; its registers, rounded to bf16, are the operand of O^T += V^T P^T as they are, V's
// operand being read in the same order of keys (transposed reads of four rows).
// Bound by the matrix cores and the vector ALU together: a tile of 128 columns is 1024 cycles of products and 990 of numerators (an exponential takes 16) a wave.
// 16384 queries x 32 heads x 128, causal: 2.02 ms, 1.09 PFLOP/s, as a library product of 8192^3; heads of 96 and 64 columns have the same numerators for fewer products:
// 0.70 to 0.88.
// QW = 2: 64 queries a workgroup, for prompts that do not fill the chip: the waves are two pairs, each with half of every tile's keys, joined at the end.  A sequence's longest
// workgroup then takes half as long (777 queries x 32 heads 22 -> 18 us).  With 128, four buffers, the next tile's scores beside the numerators, operands read further
// ahead: no gain in any combination, a tile takes 1.1 us of the matrix cores' 0.9.
template <int DKP, bool WHOLE, int QW>
__global__ __launch_bounds__(256, DKP <= 128 ? 2 : 1) void prompt_kernel(PromptArgs a) {
  constexpr int PC = Pitch<DKP>::pieces, NS = DKP / 16, NV = DKP / 32, PQ = 32 * QW, KW = 4 / QW, NH = 2 / KW;   // NH: 32 keys of a tile, NH times
  __shared__ __align__(16) char tiles[2][2][PK * PC * 16];       // [buffer][keys, values]
  PromptTile t;
  if (!prompt_tile(a, PQ, t)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, half = lane >> 5;
  const int qw = wave % QW, kw = wave / QW;                       // the wave's 32 queries, and which 32 NH keys of a tile are its own
  const int i = min(t.i0 + qw * 32 + n, t.n_q - 1);          // this lane's query (past the last: the last, not stored)
  const int off = t.n_k - t.n_q;
  const int sees = a.causal ? i + off : t.n_k - 1;               // its last key
  const int wave_last = t.i0 + qw * 32 >= t.n_q ? -1                  // (no query: the wave only takes part in the loads)
                        : a.causal ? min(t.i0 + qw * 32 + 31, t.n_q - 1) + off : t.n_k - 1;
  const int end = a.causal ? min(t.i0 + PQ, t.n_q) + off : t.n_k;     // keys that the workgroup needs
  const int all = end > 0 ? (end + PK - 1) / PK : 0, per = __builtin_amdgcn_readfirstlane((all + a.nsplit - 1) / a.nsplit);
  const int tile0 = t.split * per, tile1 = min(tile0 + per, all);

  const uint16_t* K = (const uint16_t*)a.k + t.k0 * a.k_pitch + (long)t.hk * a.d_k;
  const uint16_t* V = (const uint16_t*)a.v + t.k0 * a.v_pitch + (long)t.hk * a.d_k;
  if constexpr (!WHOLE) {                                          // pieces past d_k: zeros that nothing is loaded over
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (int x = tid; x < 4 * PK * PC; x += 256) ((u32x4*)tiles)[x] = zero;
    __syncthreads();
  }
  const int pieces = a.d_k / 8;
  constexpr int NX = PK * PC / 256, XR = 256 / PC;                 // loads of a wave for a tile's keys, rows between them
  constexpr unsigned PAIR = 2 * PK * PC * 16;                      // a buffer: keys, then values
  const int row0 = (wave * 64 + lane) / PC, place = lane % PC;
  // (rows of one lane are 16 or more apart, or pairs of them are: their pieces are swapped alike)
  constexpr int NC = PC == 32 ? 2 : 1;
  unsigned ko[NC], vo[NC];
  int ck[NC], cv[NC];
#pragma unroll
  for (int x = 0; x < NC; ++x) {
    ck[x] = place ^ k_swap<PC>(row0 + x * XR);
    cv[x] = place ^ v_swap<PC>(row0 + x * XR);
    ko[x] = (unsigned)(row0 * (int)a.k_pitch + ck[x] * 8) * 2;
    vo[x] = (unsigned)(row0 * (int)a.v_pitch + cv[x] * 8) * 2;
  }
  const uint64_t k_first = scalar((uint64_t)K), v_first = scalar((uint64_t)V), k_step = scalar((uint64_t)a.k_pitch * (2 * XR)), v_step = scalar((uint64_t)a.v_pitch * (2 * XR));
  const unsigned lds0 = lds_address(tiles) + wave * 1024;
  auto load = [&](int tile, int buf) {
    const unsigned to = lds0 + buf * PAIR;
    const int key0 = tile * PK;
    if (key0 + PK <= t.n_k) {
      uint64_t kp = k_first + (uint64_t)(unsigned)(tile * NX) * k_step, vp = v_first + (uint64_t)(unsigned)(tile * NX) * v_step;
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        if (WHOLE || ck[x % NC] < pieces) load_to_lds(kp, ko[x % NC], to + x * 4096);
        if (WHOLE || cv[x % NC] < pieces) load_to_lds(vp, vo[x % NC], to + PAIR / 2 + x * 4096);
        kp += k_step;
        vp += v_step;
      }
    } else {                                                       // rows past the last: the last, masked
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const long key = min(key0 + row0 + x * XR, t.n_k - 1);
        if (WHOLE || ck[x % NC] < pieces) load_to_lds(K + key * a.k_pitch + ck[x % NC] * 8, to + x * 4096);
        if (WHOLE || cv[x % NC] < pieces) load_to_lds(V + key * a.v_pitch + cv[x % NC] * 8, to + PAIR / 2 + x * 4096);
      }
    }
  };

  if (tile0 < tile1) load(tile0, 0);
  bf16x8 q[NS];
  {
    const uint16_t* src = (const uint16_t*)a.q + (t.q0 + i) * a.q_pitch + (long)t.h * a.d_k;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int c = s * 16 + half * 8;
      u32x4 x = {0u, 0u, 0u, 0u};
      if (c < a.d_k) x = *(const u32x4*)(src + c);
      q[s] = __builtin_bit_cast(bf16x8, x);
    }
    own_loads_done();
  }
  f32x16 o[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[v][r] = 0.f;
  float ref = NEG_INF, sum = 0.f;

  // This lane's places in the buffer of the present tile: a key's pieces, and four rows of values (rows 8 and more further on are swapped alike)
  unsigned ka[NS], va[NV];
#pragma unroll
  for (int k = 0; k < NS; ++k) ka[k] = kw * (NH * 32 * PC * 16) + (unsigned)(n * PC + ((2 * k + half) ^ k_swap<PC>(n))) * 16;
  {
    const int row = 4 * half + ((lane & 15) >> 2), byte = ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
#pragma unroll
    for (int v = 0; v < NV; ++v) va[v] = PAIR / 2 + kw * (NH * 32 * PC * 16) + (unsigned)(row * PC + ((v * 4 + (byte >> 4)) ^ v_swap<PC>(row))) * 16 + (byte & 15);
  }
  // One tile, this wave's keys of it.  MASKED: some queries of the wave do not see all of its keys.
  const char* const lds = (const char*)tiles;
  auto attend = [&](int key0, int buf, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    const char* const vt = lds + buf * PAIR + PAIR / 2 + kw * (NH * 32 * PC * 16);
    f32x16 s[NH];
    __builtin_amdgcn_s_setprio(1);                 // (the SIMD's other wave fills in: 8000 and 6854 keys x 24 heads x 96 75 -> 71 us)
#pragma unroll
    for (int x = 0; x < NH; ++x) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[x][r] = 0.f;
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        const bf16x8 A = *(const bf16x8*)(lds + ka[k] + x * (32 * PC * 16));
        s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, q[k], s[x], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    unsigned long long bad = 0;                                  // rows of values that are not finite
    if constexpr (MASKED) {
#pragma unroll
      for (int x = 0; x < NH; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + x * 32 + 8 * (r >> 2) + 4 * half + (r & 3) > sees) s[x][r] = NEG_INF;
      // (a lane a row, or half a row: zero times what is not finite is NaN, and stays)
      float top = 0.f;
      const bf16x2 zero = {(__bf16)0.f, (__bf16)0.f};
      const int row = NH == 2 ? lane : n, c0 = NH == 2 ? 0 : half * (PC / 2);
#pragma unroll 4
      for (int c = 0; c < PC * NH / 2; ++c) {
        const u32x4 v = *(const u32x4*)(vt + (row * PC + c0 + (c ^ (row & (PC * NH / 2 - 1)))) * 16);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const unsigned two = v[y];
          top = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), zero, top, false);
        }
      }
      bad = __ballot(top != 0.f);
      if constexpr (NH == 1) bad = (bad | bad >> 32) & 0xffffffffull;
    }
    float m = NEG_INF;
#pragma unroll
    for (int x = 0; x < NH; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, s[x][r]);
    m = max_of_halves(m) * a.scale;
    // The reference moves only when a score leaves it 2^8 behind: numerators up to that are as exact, and the sums have room for them.  (Each query's own: a
    // neighbour's may have moved for a key that this one does not see, which shall not change a bit of its result.)
    const bool moves = m > ref + 8.f;
    if (__any(moves)) {
      const float f = __builtin_amdgcn_exp2f(moves ? ref - m : 0.f);
      ref = moves ? m : ref;
      sum *= f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[v][r] *= f;
    }
    const float base = ref == NEG_INF ? 0.f : ref;
#pragma unroll
    for (int x = 0; x < NH; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[x][r] = __builtin_amdgcn_exp2f(fmaf(s[x][r], a.scale, -base));
        sum += s[x][r];
      }
#pragma unroll
    for (int k = 0; k < 2 * NH; ++k) {
      bf16x8 p;
#pragma unroll
      for (int r = 0; r < 8; ++r) p[r] = (__bf16)s[k >> 1][(k & 1) * 8 + r];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        u32x4 A;
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          const char* at = lds + va[v] + (k * 16 + g * 8) * PC * 16;
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at));
          A[2 * g] = x[0];
          A[2 * g + 1] = x[1];
        }
        if (MASKED && bad) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {                          // pairs of rows: which of them are finite
            const unsigned two = (unsigned)(bad >> (k * 16 + (j >> 1) * 8 + 2 * (j & 1))) >> (4 * half);
            A[j] &= (two & 1 ? 0u : 0xffffu) | (two & 2 ? 0u : 0xffff0000u);
          }
        }
        o[v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, A), p, o[v], 0, 0, 0);
      }
    }
    if constexpr (MASKED) {
      // A row with a value that is not finite goes to the queries that see it one by one.
      while (bad) {
        const int row = __ffsll((long long)bad) - 1;
        bad &= bad - 1;
        const int reg = (row >> 5) * 16 + ((row & 31) >> 3) * 4 + (row & 3);
        float p = 0.f;
#pragma unroll
        for (int x = 0; x < 16 * NH; ++x) p = x == reg ? s[x >> 4][x & 15] : p;
        p = __shfl(p, n + 32 * ((row >> 2) & 1));
        if (key0 + row <= sees) {
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int c = v * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
              const uint16_t x = *(const uint16_t*)(vt + (row * PC + ((c >> 3) ^ v_swap<PC>(row))) * 16 + (c & 7) * 2);
              o[v][r] = fmaf(p, __uint_as_float((unsigned)x << 16), o[v][r]);
            }
        }
      }
    }
  };
  // Tiles that all queries of the workgroup see, then the rest
  const int seen = (a.causal ? t.i0 + off + 1 : t.n_k) / PK, whole = min(max(seen, tile0), tile1);
  auto turn = [&](int tile, auto masked) {
    const int buf = (tile - tile0) & 1;
    tiles_barrier<0>();
    if (tile + 1 < tile1) load(tile + 1, buf ^ 1);
    const int key0 = tile * PK + kw * (NH * 32);
    if (key0 <= wave_last) attend(key0, buf, masked);
#pragma unroll
    for (int k = 0; k < NS; ++k) ka[k] ^= PAIR;
#pragma unroll
    for (int v = 0; v < NV; ++v) va[v] ^= PAIR;
  };
#pragma unroll 1
  for (int tile = tile0; tile < whole; ++tile) turn(tile, std::false_type{});
#pragma unroll 1
  for (int tile = whole; tile < tile1; ++tile) turn(tile, std::true_type{});
  sum = sum_of_halves(sum);
  if constexpr (KW == 2) {
    // The keys' two halves, joined where the tiles were
    f32x4* const J = (f32x4*)(lds + qw * ((NV * 16 + 2) * 256));
    float* const rs = (float*)(J + NV * 4 * 64);
    tiles_barrier<0>();
    if (kw == 1) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r) J[(v * 4 + r) * 64 + lane] = f32x4{o[v][4 * r], o[v][4 * r + 1], o[v][4 * r + 2], o[v][4 * r + 3]};
      rs[lane] = ref;
      rs[64 + lane] = sum;
    }
    lds_barrier();
    if (kw == 1) return;
    const float r2 = rs[lane], m = fmaxf(ref, r2);
    // (no reference: no key, or keys that are not a number)
    const float f = ref == NEG_INF ? 1.f : exp2f(ref - m), g = r2 == NEG_INF ? 1.f : exp2f(r2 - m);
    sum = sum * f + rs[64 + lane] * g;
    ref = m;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x4 y = J[(v * 4 + r) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[v][4 * r + e] = o[v][4 * r + e] * f + y[e] * g;
      }
  }
  if (t.i0 + qw * 32 + n >= t.n_q) return;
  const long row = (t.q0 + i) * a.H + t.h;
  if (a.nsplit > 1) {
    if (half == 0) {
      float* ml = a.ml + ((long)t.split * a.rows_q * a.H + row) * 2;
      ml[0] = ref;
      ml[1] = sum;
    }
    float* dst = a.O + ((long)t.split * a.rows_q * a.H + row) * a.d_k;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int c = v * 32 + 8 * r + 4 * half;
        if (c < a.d_k) *(f32x4*)(dst + c) = f32x4{o[v][4 * r], o[v][4 * r + 1], o[v][4 * r + 2], o[v][4 * r + 3]};
      }
    return;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;                // (no key: zeros)
  uint16_t* dst = (uint16_t*)a.out + row * a.d_k;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      const int c = v * 32 + 8 * r + 4 * half;
      bf16x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (__bf16)(o[v][4 * r + e] * inv);
      if (c < a.d_k) *(bf16x4*)(dst + c) = x;
    }
}

// The splits of the keys joined: four columns a thread.  Rows of no sequence stay as they are.
template <bool F32>
__global__ __launch_bounds__(256) void prompt_merge_kernel(PromptArgs a) {
  const long x = (long)blockIdx.x * 256 + threadIdx.x, per = a.d_k / 4;
  const long row = x / per, n = (long)a.rows_q * a.H;          // row: query * H + head
  if (row >= n) return;
  const int c = (int)(x % per) * 4, i = (int)(row / a.H);
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.cu_q[mid] <= i) lo = mid; else hi = mid;
  }
  if (i < a.cu_q[lo] || i >= a.cu_q[lo + 1]) return;
  float m = NEG_INF;
  for (int s = 0; s < a.nsplit; ++s) m = fmaxf(m, a.ml[(s * n + row) * 2]);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
  for (int s = 0; s < a.nsplit; ++s) {
    const float r = a.ml[(s * n + row) * 2], l = a.ml[(s * n + row) * 2 + 1];
    if (r == NEG_INF && l == 0.f) continue;                      // no key there
    const float f = r == NEG_INF ? 1.f : exp2f(r - m);           // (keys that are not a number leave no reference)
    const f32x4 y = *(const f32x4*)(a.O + (s * n + row) * a.d_k + c);
    sum = fmaf(l, f, sum);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = fmaf(y[k], f, v[k]);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if constexpr (F32) {
    *(f32x4*)((float*)a.out + row * a.d_k + c) = f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
  } else {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    bf16x4 y;
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = (__bf16)(v[k] * inv);
    *(bf16x4*)((uint16_t*)a.out + row * a.d_k + c) = y;
  }
}

template <int DKP, int QW>
void prompt_of(const PromptArgs& a, hipStream_t st) {
  if (a.d_k == Pitch<DKP>::pieces * 8) prompt_kernel<DKP, true, QW><<<prompt_grid(a, 32 * QW), 256, 0, st>>>(a);
  else prompt_kernel<DKP, false, QW><<<prompt_grid(a, 32 * QW), 256, 0, st>>>(a);
}
template <int QW>
void prompt_by_width(const PromptArgs& a, hipStream_t st) {
  if (a.d_k <= 32) prompt_of<32, QW>(a, st);
  else if (a.d_k <= 64) prompt_of<64, QW>(a, st);
  else if (a.d_k <= 96) prompt_of<96, QW>(a, st);
  else if (a.d_k <= 128) prompt_of<128, QW>(a, st);
  else if constexpr (QW == 4) {
    if (a.d_k <= 192) prompt_of<192, QW>(a, st);
    else prompt_of<256, QW>(a, st);
  }
}

}  // namespace

// How a call is cut: queries a workgroup and parts of the keys, by what they are expected to take (us).  A workgroup's tiles come one after the other, and a compute
// unit's workgroups share its matrix cores; parts have to be joined by another launch.  128 queries a tile of 128 columns: 1.13 one after the other, 0.88 of a compute
// unit's time; 64 queries: 0.77 and 0.53.  (777 queries x 32 heads x 128 22 and 18, 128 behind 5000 keys x 16 heads over 2 40 and 30, each with its best parts, 1500 x 20 x 64
// without a mask 33 and 23; where 128 fill the chip, 4000 x 32 x 128, 148 and 167.)  Keys and values that the last-level cache does not keep come a tile of 64 keys in 1.05 us for
// either, and fewer queries read them more often: 128 then (the last 300 of 8000 and 6854 rows x 24 heads x 96 77 and 82).  Over 154 shapes with their cuts timed this one takes
// 1.8 % longer than the best of each (profiles/prompt_cuts.txt);
// the fp32 kernel has one form, and its own times.
PromptCut prompt_cut(int dtype, int B, int rows_q, int rows_k, int H, int H_kv, int d_k) {
  const bool f32 = dtype == DT_F32;
  const int busy = rows_q < B ? rows_q : B;                        // sequences that can have queries; the others' places are empty
  const double keys = (double)rows_k / B / PK;                     // (as if the sequences were equally long, and so the queries of those)
  const double seen = rows_k > 0 && busy > 0 ? keys * (1 - 0.5 * fmin(1.0, (double)rows_q / rows_k * ((double)B / busy))) : 0;
  const double width = 0.45 + 0.55 * (d_k < 32 ? 32 : d_k) / 128;
  const bool cached = 4.0 * rows_k * H_kv * d_k <= 1e8;
  const int most = f32 ? prompt_f32_rows(d_k) : 128, fewest = !f32 && d_k <= 128 && cached ? 64 : most;
  PromptCut best{most, 1};
  if (busy == 0) return best;
  double least = 1e30;
  for (int rows = most; rows >= fewest; rows /= 2) {
    const double tiles = (double)busy * ((rows_q / busy + rows - 1) / rows) * H;
    const long places = ((long)rows_q / rows + B + 7) / 8 * 8 * H;   // workgroups of a part, the empty ones among them
    for (int n = 1; n <= PROMPT_MAX_PARTS; ++n) {
      if (n > 1 && (keys * PK < PROMPT_PART_KEYS * n || tiles * n > PROMPT_PART_TILES || places * n >= 1 << 24)) break;      // (a launch has 32 bits of threads)
      const double per = ceil(keys / n);
      double t;
      if (f32) {
        const double alone = 3.4 * d_k / 64, merge = n > 1 ? 4 + n * (double)rows_q * H * d_k * 8 / 4e6 : 0;
        t = (tiles * n <= 256 ? per * alone : ceil(tiles * n / 512) * per * 2 * alone) + merge;
      } else {
        const double alone = rows == 64 ? 0.77 : 1.13, one = rows == 64 ? 0.53 : 0.88, left = fmod(tiles * n, 512);      // (two a compute unit at once)
        const double rounds = floor(tiles * n / 512) * 2 * one + (left == 0 ? 0 : left <= 256 ? fmax(one, 0.9 * alone) : 2 * one);
        const double chain = per * alone * width, shared = rounds * width * seen / n;
        t = fmax(chain, shared) + 0.14 * fmin(chain, shared) + 0.75 * ceil(tiles * n / 256);
        if (n > 1) t += 6.5 + 0.65 * n + n * (double)rows_q * H * d_k * 8 / 4.1e6;
      }
      if (t < least) { least = t; best = PromptCut{rows, n}; }
    }
  }
  return best;
}

// A sequence has at most `rows` queries for each of its workgroups, and one more in the mean, which the cut rounds off.
size_t prompt_most_part_rows(int dtype, int rows_q, int rows_k, int H, int d_k) {
  const size_t parts = std::min(rows_k / PROMPT_PART_KEYS, PROMPT_MAX_PARTS), rows = dtype == DT_F32 ? prompt_f32_rows(d_k) : 128;
  return parts > 1 ? std::min(parts * rows_q * H, PROMPT_PART_TILES * (rows + 1)) : 0;
}

void launch_prompt(int dtype, const PromptArgs& a, hipStream_t st) {
  if (dtype == DT_F32) launch_prompt_f32(a, st);
  else if (a.rows == 64) prompt_by_width<2>(a, st);
  else prompt_by_width<4>(a, st);
}

void launch_prompt_merge(int dtype, const PromptArgs& a, hipStream_t st) {
  const long n = (long)a.rows_q * a.H * (a.d_k / 4);
  const unsigned grid = (unsigned)((n + 255) / 256);
  if (dtype == DT_F32) prompt_merge_kernel<true><<<grid, 256, 0, st>>>(a);
  else prompt_merge_kernel<false><<<grid, 256, 0, st>>>(a);
}

}  // namespace slim
