// Attention of a tree of drafted tokens over a K-cache: N <= 64 query rows per sequence at once, each of which sees the whole context and
// those drafted tokens that it hangs on.  Three steps for both element types: scores and softmax numerators (tree_scores_kernel), the
// weighted sum of whole K rows as one matrix product of all heads (tree_weighted_kernel), merge and projection (tree_project_kernel).
#include "slim_kernels.h"

#include "device_common.h"

#include <algorithm>

namespace slim {
namespace {

// The two element types: a lane's 16 bytes hold VEC elements, a matrix product of two such operands runs over 4 * VEC of them
// (lane / 16 takes VEC each), on bf16 in one instruction, on fp32 in four of four elements.
template <int DT> struct Elem;
template <> struct Elem<DT_BF16> {
  static constexpr int VEC = 8;
  typedef uint16_t T;
};
template <> struct Elem<DT_F32> {
  static constexpr int VEC = 4;
  typedef float T;
};

constexpr int TREE_BLOCK = TREE_BLOCK_ROWS;      // rows that share a reference of the numerators
constexpr float REF_STEP = 32.f;                 // references are multiples of this (log2 domain)

template <int DT>
__device__ __forceinline__ f32x4 mma(const u32x4& a, const u32x4& b, f32x4 acc) {
  if constexpr (DT == DT_BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], acc, 0, 0, 0);
    return acc;
  }
}

// VEC rows x VEC columns per lane -> VEC operands (one per column), each VEC rows of that column
template <int DT, int VEC = Elem<DT>::VEC>
__device__ __forceinline__ void transpose(const u32x4 (&k)[VEC], u32x4 (&a)[VEC]) {
  if constexpr (DT == DT_BF16) {
    transpose8x8(k, a);
  } else {
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int j = 0; j < 4; ++j) a[c][j] = k[j][c];
  }
}

// Row of a chunk (4 * VEC rows) that slot (g, j) of an operand stands for: the rows that a score tile leaves in lane group g, so that numerators
// become operands where they are made
__device__ __forceinline__ int slot_row(int g, int j) { return 16 * (j >> 2) + 4 * g + (j & 3); }

// Element offset inside a sequence's cache of row t, piece at `po`: rp the pitch of a row inside a band of 32, d whole rows
__device__ __forceinline__ size_t row_at(int t, int rp, int d) { return (size_t)(t >> 5) * 32 * d + (size_t)((t & 31) * rp); }
__device__ __forceinline__ int piece_at(int col, int d_k, bool banded) { return banded ? col / d_k * (32 * d_k) + col % d_k : col; }

// The tree of one sequence, one node a lane: which nodes it sees (itself and its ancestors; bit j: node j), 0 for an unused slot.  A parent is
// -1 (a root) or an earlier node; any other value makes the slot unused, and the slots that hang on it.  By doubling: six rounds
// reach 64 nodes.
__device__ __forceinline__ uint64_t ancestors(const int32_t* parents, int N, int lane) {
  const int par = lane < N ? parents[lane] : -2;
  const bool ok = par >= -1 && par < lane;
  int up = ok && par >= 0 ? par : lane;
  uint64_t anc = 1ull << lane;
  int bad = !ok;
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    anc |= (uint64_t)__shfl((unsigned)anc, up) | (uint64_t)__shfl((unsigned)(anc >> 32), up) << 32;
    bad |= __shfl(bad, up);
    up = __shfl(up, up);
  }
  return bad ? 0 : anc;
}

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// max / sum over the four lanes that share lane % 16, the same in all four
__device__ __forceinline__ float max_over_groups(float v) {
  const unsigned u = __float_as_uint(v);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const unsigned w = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ float bf16_value(unsigned bits) { return __uint_as_float(bits << 16); }

// A rotated piece of a key row (adjacent pairs, VEC / 2 of them; cs: their cos and sin).  bf16: the rotated values as hi + lo, so that
// rounding them costs no accuracy that the stored keys have.
template <int DT>
__device__ __forceinline__ void rotate_piece(u32x4 x, const f32x4* cs, u32x4& hi, u32x4& lo) {
  if constexpr (DT == DT_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x1 = bf16_value(x[i] & 0xffffu), x2 = __uint_as_float(x[i] & 0xffff0000u);
      const float c = cs[i >> 1][2 * (i & 1)], s = cs[i >> 1][2 * (i & 1) + 1];
      const float y1 = x1 * c + x2 * s, y2 = x2 * c - x1 * s;
      const unsigned h1 = bf16_bits(y1), h2 = bf16_bits(y2);
      hi[i] = h1 | h2 << 16;
      lo[i] = (unsigned)bf16_bits(y1 - bf16_value(h1)) | (unsigned)bf16_bits(y2 - bf16_value(h2)) << 16;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float x1 = __uint_as_float(x[2 * i]), x2 = __uint_as_float(x[2 * i + 1]);
      const float c = cs[0][2 * i], s = cs[0][2 * i + 1];
      hi[2 * i] = __float_as_uint(x1 * c + x2 * s);
      hi[2 * i + 1] = __float_as_uint(x2 * c - x1 * s);
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Scores and numerators.  A workgroup of four waves takes 64 query rows (row m = h N + i: the nodes of head h one after the other, so
// that small trees of many heads fill the tiles) and 256 rows of the cache, a wave 64 of these:
// S^T = K_h q_h^T for every head of the query rows, with the query operand zero where a row is another head's.  As references the
// numerators 2^(s - ref) take the block's maximum rounded up to a multiple of 32: a bf16 or fp32 numerator is as exact at 2^-32 as at 1,
// and blocks whose maxima differ by less than that have the same reference, so that the weighted sum hardly ever rescales.  They
// leave as operands of that sum (lane l of a 1 KB fragment: query row l % 16, cache rows slot_row(l / 16, j)).
// ------------------------------------------------------------------------------------------------
template <int DT, bool ROPE>
__global__ __launch_bounds__(256) void tree_scores_kernel(TreeArgs a) {
  constexpr int VEC = Elem<DT>::VEC, KW = 4 * VEC;
  typedef typename Elem<DT>::T T;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n16 = lane & 15, g = lane >> 4;
  const int group = blockIdx.x, blk = blockIdx.y, b = blockIdx.z;
  const int rows = a.N * a.H;
  const int len = seq_len_of(a.seq_lens, b, a.T), L = len + a.N;
  if (blk * TREE_BLOCK >= L) return;
  __shared__ float red[2][4][64];
  const T* K = (const T*)a.K + (size_t)b * a.k_bstride;
  const int rp = a.banded ? a.d_k : a.d;
  const uint64_t anc = ancestors(a.parents + (size_t)b * a.N, a.N, lane);
  const int depth = __popcll(anc) - 1;

  const int t0 = blk * TREE_BLOCK + wave * 64;
  int trow[4], pos[4];
#pragma unroll
  for (int ts = 0; ts < 4; ++ts) {
    const int t = min(t0 + 16 * ts + n16, L - 1);          // (rows past the end: a valid address, masked below)
    trow[ts] = t;
    if constexpr (ROPE) {
      const int dj = __shfl(depth, t - len & 63);
      pos[ts] = t < len ? t : len + max(dj, 0);
    }
  }
  f32x4 acc[4][4];
  int head[4], qoff[4];
#pragma unroll
  for (int mt = 0; mt < 4; ++mt) {
    const int m = min(group * 64 + mt * 16 + n16, rows - 1);
    head[mt] = m / a.N;
    qoff[mt] = (m % a.N) * a.d;
#pragma unroll
    for (int ts = 0; ts < 4; ++ts) acc[ts][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const T* q = (const T*)a.q + (size_t)b * a.N * a.d;
  const int h0 = group * 64 / a.N, h1 = min(group * 64 + 63, rows - 1) / a.N;
  for (int h = h0; h <= h1; ++h) {
    for (int kk = 0; kk * KW < a.d_k; ++kk) {
      const int j = kk * KW + g * VEC;
      const bool in = j < a.d_k;                           // (d_k is whole pieces, not whole steps)
      const int col = h * a.d_k + (in ? j : 0), po = piece_at(col, a.d_k, a.banded);
      u32x4 kf[4], kl[4];
#pragma unroll
      for (int ts = 0; ts < 4; ++ts) {
        kf[ts] = *(const u32x4*)(K + row_at(trow[ts], rp, a.d) + po);
        if constexpr (ROPE) {
          f32x4 cs[VEC / 4];
#pragma unroll
          for (int i = 0; i < VEC / 4; ++i) cs[i] = *(const f32x4*)(a.rope + (size_t)pos[ts] * a.d_k + (in ? j : 0) + 4 * i);
          rotate_piece<DT>(kf[ts], cs, kf[ts], kl[ts]);
          if (!in) kl[ts] = u32x4{0, 0, 0, 0};
        }
        if (!in) kf[ts] = u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) {
        const int lo = group * 64 + mt * 16;
        if (lo >= rows || lo / a.N > h || min(lo + 15, rows - 1) / a.N < h) continue;      // (no row of this head)
        u32x4 qf = *(const u32x4*)(q + qoff[mt] + col);
        if (head[mt] != h || !in) qf = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int ts = 0; ts < 4; ++ts) {
          acc[ts][mt] = mma<DT>(kf[ts], qf, acc[ts][mt]);
          if constexpr (ROPE && DT == DT_BF16) acc[ts][mt] = mma<DT>(kl[ts], qf, acc[ts][mt]);
        }
      }
    }
  }
  // a lane has query row n16 of each tile and the cache rows 4 g .. 4 g + 3 of each score tile
  float mx[4];
#pragma unroll
  for (int mt = 0; mt < 4; ++mt) {
    const int m = group * 64 + mt * 16 + n16;
    const uint64_t mine = __shfl((unsigned)anc, m % a.N) | (uint64_t)__shfl((unsigned)(anc >> 32), m % a.N) << 32;
    const uint64_t see = m < rows ? mine : 0;
    mx[mt] = NEG_INF;
#pragma unroll
    for (int ts = 0; ts < 4; ++ts)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = t0 + 16 * ts + 4 * g + r - len;
        const bool on = j < 0 ? see != 0 : j < a.N && (see >> (j & 63) & 1);
        const float s = on ? acc[ts][mt][r] * a.qscale : NEG_INF;
        acc[ts][mt][r] = s;
        mx[mt] = fmaxf(mx[mt], s);
      }
    mx[mt] = max_over_groups(mx[mt]);
    if (g == 0) red[0][wave][mt * 16 + n16] = mx[mt];
  }
  lds_barrier();
  constexpr int FR = 64 / KW;                              // fragments of a wave's 64 rows
#pragma unroll
  for (int mt = 0; mt < 4; ++mt) {
    const int at = mt * 16 + n16;
    const float m4 = fmaxf(fmaxf(red[0][0][at], red[0][1][at]), fmaxf(red[0][2][at], red[0][3][at]));
    const float ref = m4 == NEG_INF ? NEG_INF : REF_STEP * ceilf(m4 * (1.f / REF_STEP));
    const float sub = m4 == NEG_INF ? 0.f : ref;           // (nothing visible: numerators of 0, and of NaN scores NaN)
    mx[mt] = ref;
    float l = 0.f;
#pragma unroll
    for (int ts = 0; ts < 4; ++ts)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float p = exp2_of(acc[ts][mt][r] - sub);
        if constexpr (DT == DT_BF16) p = (float)(__bf16)p; // the weighted sum takes bf16 numerators; their sum is of the same values
        acc[ts][mt][r] = p;
        l += p;
      }
    l = sum_over_row_groups(l);
    if (g == 0) red[1][wave][at] = l;
    const int tile = group * 4 + mt;
    if (tile * 16 >= rows) continue;
    u32x4* P = (u32x4*)a.P + (((size_t)b * a.MT + tile) * a.CT + (size_t)blk * (TREE_BLOCK / KW) + wave * FR) * 64 + lane;
    if constexpr (DT == DT_BF16) {
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[i] = __float_as_uint(acc[2 * f + (i >> 1)][mt][2 * (i & 1)]) >> 16 | (__float_as_uint(acc[2 * f + (i >> 1)][mt][2 * (i & 1) + 1]) & 0xffff0000u);
        P[f * 64] = v;
      }
    } else {
#pragma unroll
      for (int f = 0; f < 4; ++f) P[f * 64] = __builtin_bit_cast(u32x4, acc[f][mt]);
    }
  }
  lds_barrier();
  if (wave == 0) {
    const int tile = group * 4 + lane / 16;
    if (tile * 16 < rows) {
      const size_t at = ((size_t)b * a.NB + blk) * a.MT * 16 + group * 64 + lane;
      a.lsum[at] = red[1][0][lane] + red[1][1][lane] + red[1][2][lane] + red[1][3][lane];
      const float m4 = fmaxf(fmaxf(red[0][0][lane], red[0][1][lane]), fmaxf(red[0][2][lane], red[0][3][lane]));
      a.ref[at] = m4 == NEG_INF ? NEG_INF : REF_STEP * ceilf(m4 * (1.f / REF_STEP));
    }
  }
}

// Blocks of sequence b that split s sums: the sequence's own blocks, cut evenly
__device__ __forceinline__ void split_blocks(const TreeArgs& a, int L, int s, int& first, int& end) {
  const int nb = (L + TREE_BLOCK - 1) / TREE_BLOCK, per = (nb + a.S - 1) / a.S;
  first = min(nb, s * per);
  end = min(nb, first + per);
}

template <int DT>
__device__ __forceinline__ u32x4 scaled(u32x4 p, float f) {
  if constexpr (DT == DT_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      p[i] = (unsigned)bf16_bits(bf16_value(p[i] & 0xffffu) * f) | (unsigned)bf16_bits(__uint_as_float(p[i] & 0xffff0000u) * f) << 16;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = __float_as_uint(__uint_as_float(p[i]) * f);
  }
  return p;
}

template <int DT>
__device__ __forceinline__ bool not_finite(u32x4 x) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == DT_BF16) bad |= (x[i] & 0x7f80u) == 0x7f80u || (x[i] & 0x7f800000u) == 0x7f800000u;
    else bad |= (x[i] & 0x7f800000u) == 0x7f800000u;
  }
  return bad;
}

// ------------------------------------------------------------------------------------------------
// Weighted sum: C^T = K^T P^T over a split of the context, for all heads together: every query row sums whole rows of K.  A wave owns
// 16 VEC columns of K (128 in bf16) and NT tiles of 16 query rows; a workgroup's four waves are four neighbouring column blocks of the same query
// rows.  K goes from memory to the wave's registers and is transposed there (no other wave of the workgroup needs it); the numerators arrive as
// operands.  Rows of the context need no mask; the chunks that hold drafted tokens or the cache's end are taken one by one behind them.
// ------------------------------------------------------------------------------------------------
template <int DT, int NT>
__global__ __launch_bounds__(256, NT > 4 ? 1 : 2) void tree_weighted_kernel(TreeArgs a) {
  constexpr int VEC = Elem<DT>::VEC, CW = 16 * VEC, CH = 4 * VEC, CPB = TREE_BLOCK / CH;
  typedef typename Elem<DT>::T T;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n16 = lane & 15, g = lane >> 4;
  const int mgroups = (a.MT + NT - 1) / NT, dgroups = (a.DB + 3) / 4;
  int unit, mg;
  if (!unit_of_workgroup(blockIdx.x, mgroups, a.B * a.S * dgroups, true, unit, mg)) return;
  const int block = unit % dgroups * 4 + wave, s = unit / dgroups % a.S, b = unit / dgroups / a.S;
  if (block >= a.DB) return;
  const int len = seq_len_of(a.seq_lens, b, a.T), L = len + a.N;
  int first, end;
  split_blocks(a, L, s, first, end);
  if (first >= end) return;

  const int col = min(block * CW + n16 * VEC, a.d - VEC);  // (columns past the row's end are not used by anybody)
  const int rp = a.banded ? a.d_k : a.d;
  const T* K = (const T*)a.K + (size_t)b * a.k_bstride + piece_at(col, a.d_k, a.banded);
  const u32x4* P[NT];
  int tile[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    tile[nt] = min(mg * NT + nt, a.MT - 1);
    P[nt] = (const u32x4*)a.P + ((size_t)b * a.MT + tile[nt]) * a.CT * 64 + lane;
  }
  f32x4 acc[VEC][NT];
  float ref[NT], l[NT], fac[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    ref[nt] = NEG_INF;
    l[nt] = 0.f;
    fac[nt] = 1.f;
#pragma unroll
    for (int c = 0; c < VEC; ++c) acc[c][nt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool rescaled = false;                                   // whether some numerators of the present block need a factor
  auto next_block = [&](int blk) {
    float nref[NT], nl[NT];
    bool differ = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const size_t at = (((size_t)b * a.NB + blk) * a.MT + tile[nt]) * 16 + n16;
      nref[nt] = a.ref[at];
      nl[nt] = a.lsum[at];
      differ |= nref[nt] != ref[nt];
    }
    rescaled = __any(differ);
    if (rescaled) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float top = fmaxf(ref[nt], nref[nt]);
        const float old = top == ref[nt] ? 1.f : exp2_of(ref[nt] - top);
        fac[nt] = top == nref[nt] ? 1.f : exp2_of(nref[nt] - top);
        ref[nt] = top;
        l[nt] = l[nt] * old + nl[nt] * fac[nt];
#pragma unroll
        for (int c = 0; c < VEC; ++c) acc[c][nt] *= old;
      }
      bool less = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) less |= fac[nt] != 1.f;
      rescaled = __any(less);
    } else {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) l[nt] += nl[nt];
    }
  };
  auto load = [&](int chunk, u32x4 (&k)[VEC], u32x4 (&p)[NT]) {
    const T* at = K + row_at(chunk * CH, rp, a.d);
#pragma unroll
    for (int j = 0; j < VEC; ++j) k[j] = *(const u32x4*)(at + slot_row(g, j) * rp);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) p[nt] = P[nt][(size_t)chunk * 64];
  };
  auto sum = [&](const u32x4 (&k)[VEC], u32x4 (&p)[NT]) {
    u32x4 kt[VEC];
    transpose<DT>(k, kt);
    if (rescaled) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) p[nt] = scaled<DT>(p[nt], fac[nt]);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < VEC; ++c) acc[c][nt] = mma<DT>(kt[c], p[nt], acc[c][nt]);
  };

  const int c0 = first * CPB, cend = min(end * CPB, (L + CH - 1) / CH), cfull = min(cend, max(c0, len / CH));
  u32x4 k[2][VEC], p[2][NT];
  if (c0 < cfull) load(c0, k[0], p[0]);
  auto step = [&](int chunk, auto I) {
    if (chunk % CPB == 0) next_block(chunk / CPB);
    load(min(chunk + 1, cfull - 1), k[1 - I], p[1 - I]);
    sum(k[I], p[I]);
  };
  int chunk = c0;
  for (; chunk < cfull; chunk += 2) unrolled_steps<0, 2>(chunk, cfull, step);
  for (chunk = max(c0, cfull); chunk < cend; ++chunk) {
    if (chunk % CPB == 0) next_block(chunk / CPB);
    // rows past the last drafted token are no part of the cache; a drafted key that is not finite must not reach nodes that do not see it
    // (0 times infinity is no 0): it enters the sum as 0, and nodes that do see it get NaN
    bool bad = false;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int t = chunk * CH + slot_row(g, j);
      k[0][j] = *(const u32x4*)(K + row_at(min(t, L - 1), rp, a.d));
      if (t >= L) k[0][j] = u32x4{0, 0, 0, 0};
      if (t >= len && not_finite<DT>(k[0][j])) {
        bad = true;
        k[0][j] = u32x4{0, 0, 0, 0};
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) p[0][nt] = P[nt][(size_t)chunk * 64];
    if (__any(bad)) {
      const uint64_t anc = ancestors(a.parents + (size_t)b * a.N, a.N, lane);
      for (int t = max(len, chunk * CH); t < min(L, chunk * CH + CH); ++t) {
        if (!__any(not_finite<DT>(*(const u32x4*)(K + row_at(t, rp, a.d))))) continue;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int m = tile[nt] * 16 + n16, i = m % a.N, j = t - len;
          const unsigned half = __shfl(j < 32 ? (unsigned)anc : (unsigned)(anc >> 32), i);
          const bool sees = m < a.N * a.H && (half >> (j & 31) & 1);
#pragma unroll
          for (int c = 0; c < VEC; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[c][nt][r] = sees ? __builtin_nanf("") : acc[c][nt][r];
        }
      }
    }
    sum(k[0], p[0]);
  }

  // a lane has query row n16 of each tile and the columns 4 VEC g + VEC r + c of the block, which the projection reads as operands
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (mg * NT + nt >= a.MT) continue;
    const size_t row = ((size_t)b * a.S + s) * a.MT + tile[nt];
    f32x4* C = (f32x4*)a.C + (row * a.DB + block) * VEC * 64 + lane;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int hf = 0; hf < VEC / 4; ++hf)
        C[(r * (VEC / 4) + hf) * 64] = f32x4{acc[hf * 4][nt][r], acc[hf * 4 + 1][nt][r], acc[hf * 4 + 2][nt][r], acc[hf * 4 + 3][nt][r]};
    if (block == 0 && g == 0) {
      a.sref[row * 16 + n16] = ref[nt];
      a.sl[row * 16 + n16] = l[nt];
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Merge of the splits and projection: out[i, h] = (sum_s w_s C_s[h N + i]) W_KV[:, h].  A workgroup of eight waves takes one head (or 16 VEC
// columns of one), NM of the query tiles that hold rows of it (of any sequence) and a range of rows of W_KV, which the waves share out in
// blocks of 16 VEC; their sums meet in LDS.  In bf16 C enters as hi + lo: W_KV = W_K^-1 W_V can make a rounding of C larger.
// ------------------------------------------------------------------------------------------------
template <int DT, int NM>
__global__ __launch_bounds__(512) void tree_project_kernel(TreeArgs a) {
  constexpr int VEC = Elem<DT>::VEC, CW = 16 * VEC, PITCH = CW + 4;
  typedef typename Elem<DT>::T T;
  __shared__ float weight[NM * TREE_MAX_SPLITS * 16];      // [tile][split][row]
  __shared__ __align__(16) float sums[8 * 16 * PITCH];     // [wave][row][column]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n16 = lane & 15, g = lane >> 4;
  const int cblocks = (a.d_k + CW - 1) / CW;               // column blocks of a head
  const int cs = blockIdx.x % a.csw, hc = blockIdx.x / a.csw, h = hc / cblocks, cb = hc % cblocks;
  const int tile0 = h * a.N / 16, ntiles = (h * a.N + a.N - 1) / 16 - tile0 + 1;
  const int x0 = blockIdx.y * NM;
  if (x0 >= a.B * ntiles) return;
  int tb[NM], tt[NM];
#pragma unroll
  for (int i = 0; i < NM; ++i) {
    const int x = min(x0 + i, a.B * ntiles - 1);
    tb[i] = x / ntiles;
    tt[i] = tile0 + x % ntiles;
  }
  // weights of the splits: 2^(ref_s - max) over the whole sum; 0 where a split or a row has nothing (its C may be unwritten)
  for (int e = threadIdx.x; e < NM * 16; e += 512) {
    const int i = e / 16, x = min(x0 + i, a.B * ntiles - 1), b = x / ntiles, t = tile0 + x % ntiles;
    const int L = seq_len_of(a.seq_lens, b, a.T) + a.N;
    const int nb = (L + TREE_BLOCK - 1) / TREE_BLOCK, per = (nb + a.S - 1) / a.S, ns = (nb + per - 1) / per;
    float top = NEG_INF, sum = 0.f;
    for (int s = 0; s < ns; ++s) top = fmaxf(top, a.sref[(((size_t)b * a.S + s) * a.MT + t) * 16 + e % 16]);
    for (int s = 0; s < ns; ++s) {
      const size_t at = (((size_t)b * a.S + s) * a.MT + t) * 16 + e % 16;
      sum += a.sl[at] * (top == NEG_INF ? 1.f : exp2_of(a.sref[at] - top));
    }
    for (int s = 0; s < a.S; ++s) {
      float w = 0.f;
      if (s < ns && sum != 0.f) w = (top == NEG_INF ? 1.f : exp2_of(a.sref[(((size_t)b * a.S + s) * a.MT + t) * 16 + e % 16] - top)) / sum;
      weight[(i * a.S + s) * 16 + e % 16] = w;
    }
  }
  lds_barrier();
  const int hcol = cb * CW + n16 * VEC;                    // column of the head that the lane loads
  const bool in = hcol < a.d_k;
  const T* W = (const T*)a.W + h * a.d_k + (in ? hcol : 0);
  f32x4 acc[NM][VEC];
#pragma unroll
  for (int i = 0; i < NM; ++i)
#pragma unroll
    for (int c = 0; c < VEC; ++c) acc[i][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int per = (a.DB + a.csw - 1) / a.csw, first = cs * per, end = min(a.DB, first + per);
  for (int blk = first + wave; blk < end; blk += 8) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = blk * CW + 4 * VEC * g + VEC * r;    // of W_KV, column of C
      u32x4 w[VEC], wt[VEC];
      const bool there = row < a.d;                        // (d is whole pieces)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        w[j] = *(const u32x4*)(W + (size_t)((there ? row : 0) + j) * a.d);
        if (!there) w[j] = u32x4{0, 0, 0, 0};
      }
      transpose<DT>(w, wt);
#pragma unroll
      for (int i = 0; i < NM; ++i) {
        float c[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) c[j] = 0.f;
        for (int s = 0; s < a.S; ++s) {
          const float f = weight[(i * a.S + s) * 16 + n16];
          const f32x4* C = (const f32x4*)a.C + ((((size_t)tb[i] * a.S + s) * a.MT + tt[i]) * a.DB + blk) * VEC * 64 + lane;
#pragma unroll
          for (int hf = 0; hf < VEC / 4; ++hf) {
            const f32x4 v = C[(r * (VEC / 4) + hf) * 64];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[hf * 4 + j] += f == 0.f || !there ? 0.f : v[j] * f;
          }
        }
        if constexpr (DT == DT_BF16) {
          u32x4 hi, lo;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const unsigned h1 = bf16_bits(c[2 * j]), h2 = bf16_bits(c[2 * j + 1]);
            hi[j] = h1 | h2 << 16;
            lo[j] = (unsigned)bf16_bits(c[2 * j] - bf16_value(h1)) | (unsigned)bf16_bits(c[2 * j + 1] - bf16_value(h2)) << 16;
          }
#pragma unroll
          for (int cc = 0; cc < VEC; ++cc) acc[i][cc] = mma<DT>(wt[cc], lo, mma<DT>(wt[cc], hi, acc[i][cc]));
        } else {
          u32x4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) v[j] = __float_as_uint(c[j]);
#pragma unroll
          for (int cc = 0; cc < VEC; ++cc) acc[i][cc] = mma<DT>(wt[cc], v, acc[i][cc]);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NM; ++i) {
    if (x0 + i >= a.B * ntiles) break;
    // (a lane has query row n16 and the columns VEC (4 g + r) + c)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int hf = 0; hf < VEC / 4; ++hf)
        *(f32x4*)(sums + (wave * 16 + n16) * PITCH + VEC * (4 * g + r) + hf * 4) =
            f32x4{acc[i][hf * 4][r], acc[i][hf * 4 + 1][r], acc[i][hf * 4 + 2][r], acc[i][hf * 4 + 3][r]};
    lds_barrier();
    for (int e = threadIdx.x; e < 16 * CW / 4; e += 512) {
      const int row = e / (CW / 4), c4 = e % (CW / 4) * 4, m = tt[i] * 16 + row;
      if (m / a.N == h && cb * CW + c4 < a.d_k) {
        f32x4 v = *(const f32x4*)(sums + row * PITCH + c4);
#pragma unroll
        for (int w = 1; w < 8; ++w) v += *(const f32x4*)(sums + (w * 16 + row) * PITCH + c4);
        const size_t node = (size_t)tb[i] * a.N + m % a.N;
        const int at = h * a.d_k + cb * CW + c4;
        if (a.csw > 1) {
          *(f32x4*)(a.part + ((size_t)cs * a.B * a.N + node) * a.d + at) = v;
        } else if constexpr (DT == DT_BF16) {
          *(uint2*)((uint16_t*)a.out + node * a.d + at) =
              uint2{(unsigned)bf16_bits(v[0]) | (unsigned)bf16_bits(v[1]) << 16, (unsigned)bf16_bits(v[2]) | (unsigned)bf16_bits(v[3]) << 16};
        } else {
          *(f32x4*)((float*)a.out + node * a.d + at) = v;
        }
      }
    }
    lds_barrier();
  }
}

// Sums of the row splits of W_KV, always in the same order, rounded once
template <int DT>
__global__ __launch_bounds__(256) void tree_sum_kernel(const float* part, int csw, size_t n4, void* out) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n4) return;
  f32x4 v = ((const f32x4*)part)[i];
  for (int c = 1; c < csw; ++c) v += ((const f32x4*)part)[c * n4 + i];
  if constexpr (DT == DT_BF16)
    ((uint2*)out)[i] = uint2{(unsigned)bf16_bits(v[0]) | (unsigned)bf16_bits(v[1]) << 16, (unsigned)bf16_bits(v[2]) | (unsigned)bf16_bits(v[3]) << 16};
  else
    ((f32x4*)out)[i] = v;
}

template <int DT>
void launch_tree_scores_t(const TreeArgs& a, hipStream_t st) {
  const dim3 grid((a.N * a.H + 63) / 64, a.NB, a.B);
  if (a.rope) hipLaunchKernelGGL((tree_scores_kernel<DT, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((tree_scores_kernel<DT, false>), grid, dim3(256), 0, st, a);
}

template <int DT>
void launch_tree_weighted_t(const TreeArgs& a, int nt, hipStream_t st) {
  const int mgroups = (a.MT + nt - 1) / nt, units = a.B * a.S * ((a.DB + 3) / 4);
  const dim3 grid((units + 7) / 8 * 8 * mgroups);
  switch (nt) {
    case 1: hipLaunchKernelGGL((tree_weighted_kernel<DT, 1>), grid, dim3(256), 0, st, a); break;
    case 2: hipLaunchKernelGGL((tree_weighted_kernel<DT, 2>), grid, dim3(256), 0, st, a); break;
    case 4: hipLaunchKernelGGL((tree_weighted_kernel<DT, 4>), grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL((tree_weighted_kernel<DT, 8>), grid, dim3(256), 0, st, a); break;
  }
}

template <int DT>
void launch_tree_project_t(const TreeArgs& a, hipStream_t st) {
  constexpr int CW = 16 * Elem<DT>::VEC;
  const int heads = a.H * ((a.d_k + CW - 1) / CW);
  const int tiles = a.B * ((a.N + 14) / 16 + 1);
  if (tiles > 2) hipLaunchKernelGGL((tree_project_kernel<DT, 4>), dim3(heads * a.csw, (tiles + 3) / 4), dim3(512), 0, st, a);
  else hipLaunchKernelGGL((tree_project_kernel<DT, 1>), dim3(heads * a.csw, tiles), dim3(512), 0, st, a);
  if (a.csw > 1) {
    const size_t n4 = (size_t)a.B * a.N * a.d / 4;
    hipLaunchKernelGGL(tree_sum_kernel<DT>, dim3((n4 + 255) / 256), dim3(256), 0, st, a.part, a.csw, n4, a.out);
  }
}

}  // namespace

// Query tiles of 16 rows that a wave of the weighted sum takes together: as many as there are, up to eight (all 512 registers).
int tree_tiles(int H, int N) {
  const int mt = (H * N + 15) / 16;
  return mt >= 5 ? 8 : mt >= 3 ? 4 : mt;
}

// Context splits of the weighted sum: until there is a workgroup for every compute unit, a block of rows each at least.  Grows with T.
int tree_splits(int dtype, int B, int N, int H, int T, int d) {
  const int nt = tree_tiles(H, N), mt = (H * N + 15) / 16, cw = 16 * vec_elems(dtype);
  const long wgs = (long)B * ((mt + nt - 1) / nt) * ((d + 4 * cw - 1) / (4 * cw));
  const int nb = (T + N + TREE_BLOCK_ROWS - 1) / TREE_BLOCK_ROWS;
  return (int)std::max(1l, std::min<long>({(256 + wgs - 1) / wgs, nb, TREE_MAX_SPLITS}));
}

// Row splits of W_KV in the projection: until there is a workgroup for every compute unit, a block of rows for each wave at least.
int tree_row_splits(int dtype, int B, int N, int H, int d) {
  const int cw = 16 * vec_elems(dtype), d_k = d / H, db = (d + cw - 1) / cw;
  const long tiles = (long)B * ((N + 14) / 16 + 1), wgs = (long)H * ((d_k + cw - 1) / cw) * (tiles > 2 ? (tiles + 3) / 4 : tiles);
  return (int)std::max(1l, std::min<long>({(256 + wgs - 1) / wgs, (db + 7) / 8, 16}));
}

void launch_tree_scores(int dtype, const TreeArgs& a, hipStream_t st) {
  if (dtype == DT_BF16) launch_tree_scores_t<DT_BF16>(a, st);
  else launch_tree_scores_t<DT_F32>(a, st);
}
void launch_tree_weighted(int dtype, const TreeArgs& a, hipStream_t st) {
  const int nt = tree_tiles(a.H, a.N);
  if (dtype == DT_BF16) launch_tree_weighted_t<DT_BF16>(a, nt, st);
  else launch_tree_weighted_t<DT_F32>(a, nt, st);
}
void launch_tree_project(int dtype, const TreeArgs& a, hipStream_t st) {
  if (dtype == DT_BF16) launch_tree_project_t<DT_BF16>(a, st);
  else launch_tree_project_t<DT_F32>(a, st);
}

}  // namespace slim
