// Attention over whole prompts in fp32 (kernels_prompt.hip has it in bf16).
#include "prompt_common.h"

namespace slim {
namespace {

constexpr int PK = 32;                         // keys of a tile; 16 queries a wave

template <int DKP> struct Pitch { static constexpr int pieces = DKP <= 64 ? 16 : DKP <= 128 ? 32 : 64; };

__device__ __forceinline__ float max_of_groups(float v) {
  const unsigned u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return max_of_halves(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
}

// As in bf16, on 16x16x4 products: S^T = K Q^T has a query in the four lanes l % 16, four consecutive keys in the registers of each; register i of all four
// is the operand of a product over the keys 4 g + i (g the lane's group), V's rows are read to fit.  Operands of the first product come four at a time: lane
// group g holds columns 4 g .. 4 g + 3 of 16, a product takes one of the four from each.  Bound by the matrix cores' fp32 rate.
template <int DKP>
__global__ __launch_bounds__(256, DKP <= 128 ? 2 : 1) void prompt_f32_kernel(PromptArgs a) {
  constexpr int PC = Pitch<DKP>::pieces, NS = DKP / 16, NV = (DKP + 63) / 64;
  __shared__ __align__(16) char tiles[2][2][PK * PC * 16];       // [buffer][keys, values]
  PromptTile t;
  if (!prompt_tile(a, PROMPT_F32_ROWS, t)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  const int i = min(t.i0 + wave * 16 + n, t.n_q - 1);
  const int off = t.n_k - t.n_q;
  const int sees = a.causal ? i + off : t.n_k - 1;
  const int wave_first = a.causal ? min(t.i0 + wave * 16, t.n_q - 1) + off : t.n_k - 1;
  const int wave_last = a.causal ? min(t.i0 + wave * 16 + 15, t.n_q - 1) + off : t.n_k - 1;
  const int end = a.causal ? min(t.i0 + PROMPT_F32_ROWS, t.n_q) + off : t.n_k;
  const int all = end > 0 ? (end + PK - 1) / PK : 0, per = __builtin_amdgcn_readfirstlane((all + a.nsplit - 1) / a.nsplit);
  const int tile0 = t.split * per, tile1 = min(tile0 + per, all);
  const float* K = (const float*)a.k + t.k0 * a.k_pitch + (long)t.hk * a.d_k;
  const float* V = (const float*)a.v + t.k0 * a.v_pitch + (long)t.hk * a.d_k;
  const bool clear = a.d_k < PC * 4;
  if (clear) {
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (int x = tid; x < 4 * PK * PC; x += 256) ((u32x4*)tiles)[x] = zero;
    __syncthreads();
  }
  const int pieces = a.d_k / 4;
  auto load = [&](int tile, int buf) {
    const int key0 = tile * PK;
#pragma unroll
    for (int x = 0; x < PK * PC / 256; ++x) {
      const int at = (x * 4 + wave) * 64 + lane, row = at / PC, place = at % PC;
      const long key = min(key0 + row, t.n_k - 1);
      const int ck = place ^ (row & 15);
      if (!clear || ck < pieces) load_to_lds(K + key * a.k_pitch + ck * 4, lds_address(tiles[buf][0]) + (x * 4 + wave) * 1024);
      if (!clear || place < pieces) load_to_lds(V + key * a.v_pitch + place * 4, lds_address(tiles[buf][1]) + (x * 4 + wave) * 1024);
    }
  };
  if (tile0 < tile1) load(tile0, 0);
  f32x4 q[NS];
  {
    const float* src = (const float*)a.q + (t.q0 + i) * a.q_pitch + (long)t.h * a.d_k;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int c = s * 16 + g * 4;
      q[s] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (c < a.d_k) q[s] = *(const f32x4*)(src + c);
    }
    own_loads_done();
  }
  f32x4 o[NV][4];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[v][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float ref = NEG_INF, sum = 0.f;
  for (int tile = tile0; tile < tile1; ++tile) {
    const int buf = (tile - tile0) & 1, key0 = tile * PK;
    tiles_barrier<0>();
    if (tile + 1 < tile1) load(tile + 1, buf ^ 1);
    if (key0 > wave_last) continue;
    const char* kt = tiles[buf][0];
    const char* vt = tiles[buf][1];
    f32x4 s[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
      const int row = x * 16 + n;
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        const f32x4 A = *(const f32x4*)(kt + (row * PC + ((4 * k + g) ^ (row & 15))) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[e], q[k][e], s[x], 0, 0, 0);
      }
    }
    const bool masked = key0 + PK - 1 > wave_first;
    unsigned bad = 0;                                            // rows of values that are not finite, where some queries do not see all rows
    if (masked) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (key0 + x * 16 + 4 * g + r > sees) s[x][r] = NEG_INF;
      unsigned top = 0;                                          // (two lanes a row)
      for (int c = 0; c < PC / 2; ++c) {
        const u32x4 v = *(const u32x4*)(vt + ((lane >> 1) * PC + (lane & 1) * (PC / 2) + ((c + lane) & (PC / 2 - 1))) * 16);
#pragma unroll
        for (int y = 0; y < 4; ++y) top = max(top, v[y] & 0x7fffffffu);
      }
      const unsigned long long lanes = __ballot(top >= 0x7f800000u);
#pragma unroll
      for (int r = 0; r < PK; ++r) bad |= (unsigned)((lanes >> (2 * r) & 3) != 0) << r;
    }
    float m = NEG_INF;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r) m = fmaxf(m, s[x][r]);
    m = max_of_groups(m) * a.scale;
    if (__any(m > ref)) {
      const float to = fmaxf(ref, m);
      const float f = to == NEG_INF ? 1.f : exp2f(ref - to);
      ref = to;
      sum *= f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[v][j] *= f;
    }
    const float base = ref == NEG_INF ? 0.f : ref;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[x][r] = exp2f(fmaf(s[x][r], a.scale, -base));
        sum += s[x][r];
      }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = x * 16 + 4 * g + r;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          f32x4 A = *(const f32x4*)(vt + (row * PC + v * 16 + n) * 16);
          if (bad >> row & 1) A = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 4; ++j) o[v][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[j], s[x][r], o[v][j], 0, 0, 0);
        }
      }
    while (bad) {
      const int row = __ffs((int)bad) - 1;
      bad &= bad - 1;
      const int reg = (row >> 4) * 4 + (row & 3);
      float p = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) p = x == reg ? s[x >> 2][x & 3] : p;
      p = __shfl(p, n + 16 * ((row >> 2) & 3));
      if (key0 + row <= sees) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const f32x4 x = *(const f32x4*)(vt + (row * PC + v * 16 + 4 * g + r) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[v][j][r] = fmaf(p, x[j], o[v][j][r]);
          }
      }
    }
  }
  sum = sum_over_row_groups(sum);
  if (t.i0 + wave * 16 + n >= t.n_q) return;
  const long row = (t.q0 + i) * a.H + t.h;
  const bool whole = a.nsplit == 1;
  if (!whole && g == 0) {
    float* ml = a.ml + ((long)t.split * a.rows_q * a.H + row) * 2;
    ml[0] = ref;
    ml[1] = sum;
  }
  const float f = !whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
  float* dst = whole ? (float*)a.out + row * a.d_k : a.O + ((long)t.split * a.rows_q * a.H + row) * a.d_k;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int c = v * 64 + 16 * g + 4 * r;
      if (c < a.d_k) *(f32x4*)(dst + c) = f32x4{o[v][0][r] * f, o[v][1][r] * f, o[v][2][r] * f, o[v][3][r] * f};
    }
}

template <int DKP>
void prompt_of(const PromptArgs& a, hipStream_t st) { prompt_f32_kernel<DKP><<<prompt_grid(a, PROMPT_F32_ROWS), 256, 0, st>>>(a); }

}  // namespace

void launch_prompt_f32(const PromptArgs& a, hipStream_t st) {
  if (a.d_k <= 32) prompt_of<32>(a, st);
  else if (a.d_k <= 64) prompt_of<64>(a, st);
  else if (a.d_k <= 96) prompt_of<96>(a, st);
  else if (a.d_k <= 128) prompt_of<128>(a, st);
  else if (a.d_k <= 192) prompt_of<192>(a, st);
  else prompt_of<256>(a, st);
}

}  // namespace slim
