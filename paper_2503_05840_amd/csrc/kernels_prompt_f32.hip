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
// group g holds columns 4 g .. 4 g + 3 of 16, a product takes one of the four from each.  QT tiles of queries a wave share what is read of K and V.
// Bound by the matrix cores' fp32 rate: 4 x 1500 queries x 20 heads x 64, full, 387 us, 119 TFLOP/s of 154.
template <int DKP, bool WHOLE, int QT>
__global__ __launch_bounds__(256, DKP <= 128 ? 2 : 1) void prompt_f32_kernel(PromptArgs a) {
  constexpr int PC = Pitch<DKP>::pieces, NS = DKP / 16, NV = (DKP + 63) / 64, PQ = 64 * QT;
  __shared__ __align__(16) char tiles[2][2][PK * PC * 16];       // [buffer][keys, values]
  PromptTile t;
  if (!prompt_tile(a, PQ, t)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  const int off = t.n_k - t.n_q, i0 = t.i0 + wave * 16 * QT;
  int i[QT], sees[QT];                                            // this lane's queries (past the last: the last, not stored) and their last keys
#pragma unroll
  for (int y = 0; y < QT; ++y) {
    i[y] = min(i0 + y * 16 + n, t.n_q - 1);
    sees[y] = a.causal ? i[y] + off : t.n_k - 1;
  }
  const int wave_last = i0 >= t.n_q ? -1                                // (no query: the wave only takes part in the loads)
                        : a.causal ? min(i0 + 16 * QT - 1, t.n_q - 1) + off : t.n_k - 1;
  const int end = a.causal ? min(t.i0 + PQ, t.n_q) + off : t.n_k;     // keys that the workgroup needs
  const int all = end > 0 ? (end + PK - 1) / PK : 0, per = __builtin_amdgcn_readfirstlane((all + a.nsplit - 1) / a.nsplit);
  const int tile0 = t.split * per, tile1 = min(tile0 + per, all);
  const float* K = (const float*)a.k + t.k0 * a.k_pitch + (long)t.hk * a.d_k;
  const float* V = (const float*)a.v + t.k0 * a.v_pitch + (long)t.hk * a.d_k;
  if constexpr (!WHOLE) {                                          // pieces past d_k: zeros that nothing is loaded over
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (int x = tid; x < 4 * PK * PC; x += 256) ((u32x4*)tiles)[x] = zero;
    __syncthreads();
  }
  const int pieces = a.d_k / 4;
  constexpr int NX = PK * PC / 256, XR = 256 / PC;                 // loads of a wave for a tile's keys, rows between them
  constexpr int NC = XR < 16 ? 16 / XR : 1;                        // (rows of one lane 16 apart are swapped alike)
  constexpr unsigned PAIR = 2 * PK * PC * 16;
  const int row0 = (wave * 64 + lane) / PC, place = lane % PC;
  unsigned ko[NC];
  int ck[NC];
#pragma unroll
  for (int x = 0; x < NC; ++x) {
    ck[x] = place ^ ((row0 + x * XR) & 15);
    ko[x] = (unsigned)(row0 * (int)a.k_pitch + ck[x] * 4) * 4;
  }
  const unsigned vo = (unsigned)(row0 * (int)a.v_pitch + place * 4) * 4;
  const uint64_t k_first = scalar((uint64_t)K), v_first = scalar((uint64_t)V), k_step = scalar((uint64_t)a.k_pitch * (4 * XR)),
                 v_step = scalar((uint64_t)a.v_pitch * (4 * XR));
  const unsigned lds0 = lds_address(tiles) + wave * 1024;
  auto load = [&](int tile, int buf) {
    const int key0 = tile * PK;
    const unsigned to = lds0 + buf * PAIR;
    if (key0 + PK <= t.n_k) {
      uint64_t kp = k_first + (uint64_t)(unsigned)(tile * NX) * k_step, vp = v_first + (uint64_t)(unsigned)(tile * NX) * v_step;
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        if (WHOLE || ck[x % NC] < pieces) load_to_lds(kp, ko[x % NC], to + x * 4096);
        if (WHOLE || place < pieces) load_to_lds(vp, vo, to + PAIR / 2 + x * 4096);
        kp += k_step;
        vp += v_step;
      }
    } else {                                                       // rows past the last: the last, masked
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const long key = min(key0 + row0 + x * XR, t.n_k - 1);
        if (WHOLE || ck[x % NC] < pieces) load_to_lds(K + key * a.k_pitch + ck[x % NC] * 4, to + x * 4096);
        if (WHOLE || place < pieces) load_to_lds(V + key * a.v_pitch + place * 4, to + PAIR / 2 + x * 4096);
      }
    }
  };
  if (tile0 < tile1) load(tile0, 0);
  f32x4 q[QT][NS];
#pragma unroll
  for (int y = 0; y < QT; ++y) {
    const float* src = (const float*)a.q + (t.q0 + i[y]) * a.q_pitch + (long)t.h * a.d_k;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int c = s * 16 + g * 4;
      q[y][s] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (c < a.d_k) q[y][s] = *(const f32x4*)(src + c);
    }
  }
  own_loads_done();
  f32x4 o[QT][NV][4];
  float ref[QT], sum[QT];
#pragma unroll
  for (int y = 0; y < QT; ++y) {
    ref[y] = NEG_INF;
    sum[y] = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[y][v][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  unsigned ka[NS], va = PAIR / 2 + (unsigned)(4 * g * PC + n) * 16;
#pragma unroll
  for (int k = 0; k < NS; ++k) ka[k] = (unsigned)(n * PC + ((4 * k + g) ^ n)) * 16;
  const char* const lds = (const char*)tiles;
  // One tile.  MASKED: some queries of the wave do not see all of its keys.
  auto attend = [&](int key0, int buf, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    const char* const vt = lds + buf * PAIR + PAIR / 2;
    f32x4 s[QT][2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int y = 0; y < QT; ++y) s[y][x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        const f32x4 A = *(const f32x4*)(lds + ka[k] + x * (16 * PC * 16));
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int y = 0; y < QT; ++y) s[y][x] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[e], q[y][k][e], s[y][x], 0, 0, 0);
      }
    }
    unsigned bad = 0;                                            // rows of values that are not finite
    if constexpr (MASKED) {
#pragma unroll
      for (int y = 0; y < QT; ++y)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (key0 + x * 16 + 4 * g + r > sees[y]) s[y][x][r] = NEG_INF;
      float top = 0.f;                                           // (two lanes a row: zero times what is not finite is NaN, and stays)
#pragma unroll 4
      for (int c = 0; c < PC / 2; ++c) {
        const f32x4 v = *(const f32x4*)(vt + ((lane >> 1) * PC + (lane & 1) * (PC / 2) + ((c + lane) & (PC / 2 - 1))) * 16);
#pragma unroll
        for (int y = 0; y < 4; ++y) top = fmaf(v[y], 0.f, top);
      }
      unsigned long long lanes = __ballot(top != 0.f);
      for (lanes |= lanes >> 1; lanes; lanes &= lanes - 1) {     // (an even lane's bit: its row's)
        const int l = __ffsll((long long)lanes) - 1;
        if (!(l & 1)) bad |= 1u << (l >> 1);
      }
    }
#pragma unroll
    for (int y = 0; y < QT; ++y) {
      float m = NEG_INF;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) m = fmaxf(m, s[y][x][r]);
      m = max_of_groups(m) * a.scale;
      // (the reference moves only when a score leaves it 2^8 behind: numerators up to that are as exact; each query's own, or unseen keys would show in its bits)
      const bool moves = m > ref[y] + 8.f;
      if (__any(moves)) {
        const float f = __builtin_amdgcn_exp2f(moves ? ref[y] - m : 0.f);
        ref[y] = moves ? m : ref[y];
        sum[y] *= f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[y][v][j] *= f;
      }
      const float base = ref[y] == NEG_INF ? 0.f : ref[y];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[y][x][r] = __builtin_amdgcn_exp2f(fmaf(s[y][x][r], a.scale, -base));
          sum[y] += s[y][x][r];
        }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          f32x4 A = *(const f32x4*)(lds + va + ((x * 16 + r) * PC + v * 16) * 16);
          if (MASKED && bad)
            if (bad >> (x * 16 + 4 * g + r) & 1) A = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int y = 0; y < QT; ++y) o[y][v][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(A[j], s[y][x][r], o[y][v][j], 0, 0, 0);
        }
    if constexpr (MASKED) {
      // A row with a value that is not finite goes to the queries that see it one by one.
      while (bad) {
        const int row = __ffs((int)bad) - 1;
        bad &= bad - 1;
        const int reg = (row >> 4) * 4 + (row & 3);
#pragma unroll
        for (int y = 0; y < QT; ++y) {
          float p = 0.f;
#pragma unroll
          for (int x = 0; x < 8; ++x) p = x == reg ? s[y][x >> 2][x & 3] : p;
          p = __shfl(p, n + 16 * ((row >> 2) & 3));
          if (key0 + row <= sees[y]) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const f32x4 x = *(const f32x4*)(vt + (row * PC + v * 16 + 4 * g + r) * 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[y][v][j][r] = fmaf(p, x[j], o[y][v][j][r]);
              }
          }
        }
      }
    }
  };
  const int seen = (a.causal ? t.i0 + off + 1 : t.n_k) / PK, whole = min(max(seen, tile0), tile1);
  auto turn = [&](int tile, auto masked) {
    const int buf = (tile - tile0) & 1;
    tiles_barrier<0>();
    if (tile + 1 < tile1) load(tile + 1, buf ^ 1);
    if (tile * PK <= wave_last) attend(tile * PK, buf, masked);
#pragma unroll
    for (int k = 0; k < NS; ++k) ka[k] ^= PAIR;
    va ^= PAIR;
  };
#pragma unroll 1
  for (int tile = tile0; tile < whole; ++tile) turn(tile, std::false_type{});
#pragma unroll 1
  for (int tile = whole; tile < tile1; ++tile) turn(tile, std::true_type{});
#pragma unroll
  for (int y = 0; y < QT; ++y) {
    const float l = sum_over_row_groups(sum[y]);
    if (i0 + y * 16 + n >= t.n_q) continue;
    const long row = (t.q0 + i[y]) * a.H + t.h;
    const bool last = a.nsplit == 1;
    if (!last && g == 0) {
      float* ml = a.ml + ((long)t.split * a.rows_q * a.H + row) * 2;
      ml[0] = ref[y];
      ml[1] = l;
    }
    const float f = !last ? 1.f : l == 0.f ? 0.f : 1.f / l;
    float* dst = last ? (float*)a.out + row * a.d_k : a.O + ((long)t.split * a.rows_q * a.H + row) * a.d_k;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int c = v * 64 + 16 * g + 4 * r;
        if (c < a.d_k) *(f32x4*)(dst + c) = f32x4{o[y][v][0][r] * f, o[y][v][1][r] * f, o[y][v][2][r] * f, o[y][v][3][r] * f};
      }
  }
}

template <int DKP, int QT>
void prompt_of(const PromptArgs& a, hipStream_t st) {
  if (a.d_k == Pitch<DKP>::pieces * 4) prompt_f32_kernel<DKP, true, QT><<<prompt_grid(a, 64 * QT), 256, 0, st>>>(a);
  else prompt_f32_kernel<DKP, false, QT><<<prompt_grid(a, 64 * QT), 256, 0, st>>>(a);
}

}  // namespace

int prompt_f32_rows(int d_k) { return d_k <= 32 || (d_k > 64 && d_k <= 128) ? 128 : 64; }     // queries of a workgroup

void launch_prompt_f32(const PromptArgs& a, hipStream_t st) {
  if (a.d_k <= 32) prompt_of<32, 2>(a, st);
  else if (a.d_k <= 64) prompt_of<64, 1>(a, st);
  else if (a.d_k <= 96) prompt_of<96, 2>(a, st);
  else if (a.d_k <= 128) prompt_of<128, 2>(a, st);
  else if (a.d_k <= 192) prompt_of<192, 1>(a, st);
  else prompt_of<256, 1>(a, st);
}

}  // namespace slim
