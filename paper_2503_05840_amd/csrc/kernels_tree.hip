// Attention of a tree of drafted tokens over a K-cache: N <= 64 query rows per sequence at once, each of which sees the whole context and
// those drafted tokens that it hangs on.  Three steps for both element types: scores and softmax numerators (tree_scores_kernel), the
// weighted sum of whole K rows as one matrix product of all heads (tree_weighted_kernel), merge and projection (tree_project_kernel).
#include "slim_kernels.h"

#include "device_common.h"

#include <algorithm>
#include <climits>

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

// Two of them, the first in the lower half (one instruction; a pair of single ones is three)
__device__ __forceinline__ unsigned bf16_pair(float x, float y) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{x, y}, bf16x2));
}
__device__ __forceinline__ float bf16_value(unsigned bits) { return __uint_as_float(bits << 16); }

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

// Which drafted keys of sequence b hold anything that is not finite (bit j: node j), the same in every lane
__device__ __forceinline__ uint64_t odd_keys(const TreeArgs& a, int b, int lane) {
  uint64_t m = 0;
  for (int i = lane; i < 2 * a.H; i += 64) m |= a.odd[(size_t)b * 2 * a.H + i];
  if (!__any(m != 0)) return 0;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) m |= (uint64_t)__shfl_xor((unsigned)m, k) | (uint64_t)__shfl_xor((unsigned)(m >> 32), k) << 32;
  return m;
}

// VEC consecutive columns of a row of C as the projection's operand, 64 lanes apart: in bf16 hi and lo, since W_KV = W_K^-1 W_V can make a rounding
// of C larger
template <int DT, int VEC = Elem<DT>::VEC>
__device__ __forceinline__ void store_operand(const float (&v)[VEC], u32x4* out) {
  u32x4 hi, lo;
  if constexpr (DT == DT_BF16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      hi[j] = bf16_pair(v[2 * j], v[2 * j + 1]);
      lo[j] = bf16_pair(v[2 * j] - bf16_value(hi[j] & 0xffffu), v[2 * j + 1] - __uint_as_float(hi[j] & 0xffff0000u));
    }
    out[0] = hi;
    out[64] = lo;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) hi[j] = __float_as_uint(v[j]);
    out[0] = hi;
  }
}

// acc += a b, the accumulator staying where it is.  With as many accumulators as there are accumulation registers the compiler gives a product
// another destination than its addend and moves hundreds of registers a step to put that right.  In an asm statement the wait states
// are this code's: two between a vector instruction that writes an operand and the product -- operands_ready() where operands may be that
// new --, those of reading a result in settle().
template <int DT>
__device__ __forceinline__ void mma_in_place(const u32x4& a, const u32x4& b, f32x4& acc) {
  if constexpr (DT == DT_BF16) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
  else acc = mma<DT>(a, b, acc);
}
// (An operand that has just been written is named: an asm statement keeps its place among others of its kind only.)
__device__ __forceinline__ void operands_ready(u32x4& x) { asm volatile("s_nop 1" : "+v"(x)); }
// (and for the accumulators of a tile's products: where registers are short the compiler parks one elsewhere and brings it back right before its product)
template <int VEC, int NT>
__device__ __forceinline__ void operands_ready(f32x4 (&acc)[VEC][NT], int nt) {
  if constexpr (VEC == 8)
    asm volatile("s_nop 1" : "+a"(acc[0][nt]), "+a"(acc[1][nt]), "+a"(acc[2][nt]), "+a"(acc[3][nt]), "+a"(acc[4][nt]), "+a"(acc[5][nt]), "+a"(acc[6][nt]), "+a"(acc[7][nt]));
}
__device__ __forceinline__ void settle() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

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

// The same, element pair by element pair: what rows 2 jp and 2 jp + 1 (bf16) or row jp (fp32) give operand c.
template <int DT, int VEC = Elem<DT>::VEC>
__device__ __forceinline__ void transpose_one(const u32x4 (&k)[VEC], u32x4 (&a)[VEC], int jp, int c) {
  if constexpr (DT == DT_BF16) a[c][jp] = __builtin_amdgcn_perm(k[2 * jp + 1][c / 2], k[2 * jp][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
  else a[c][jp] = k[jp][c];
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

// How the sequences share the slots of the weighted sum: the fewest steps of 64 rows a slot that leave enough of them (ragged batches: 8 sequences of 600
// to 5000 rows in 16 slots take 30 steps, where as many slots for each take 40).  By one wave, which has up to four sequences a lane.
__device__ void plan_splits(const TreeArgs& a, int lane) {
  int steps[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = i * 64 + lane;
    steps[i] = b < a.B ? (seq_len_of(a.seq_lens, b, a.T) + a.N + TREE_STEP_ROWS - 1) / TREE_STEP_ROWS : 0;
  }
  auto total = [](int v) {
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) v += __shfl_xor(v, k);
    return v;
  };
  int lo = a.per_min, hi = (a.T + a.N + TREE_STEP_ROWS - 1) / TREE_STEP_ROWS;      // (as many a slot as the longest may have: B slots)
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    int n = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) n += (steps[i] + mid - 1) / mid;
    if (total(n) <= a.slots) hi = mid;
    else lo = mid + 1;
  }
  int at = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = (steps[i] + lo - 1) / lo;
    int upto = n;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
      const int o = __shfl_up(upto, k);
      if (lane >= k) upto += o;
    }
    const int b = i * 64 + lane, first = at + upto - n;
    if (b < a.B) {
      a.plan[1 + a.slots + b] = first * 2 * TREE_MAX_SPLITS + n;
      for (int s = 0; s < n; ++s) a.plan[1 + first + s] = b * TREE_MAX_SPLITS + s;
    }
    at += __shfl(upto, 63);
  }
  for (int i = at + lane; i < a.slots; i += 64) a.plan[1 + i] = -1;
  if (lane == 0) a.plan[0] = lo;
}
// (called by every workgroup of the scores' launch)
__device__ __forceinline__ void plan_once(const TreeArgs& a, int lane, int wave) {
  if (a.slots > a.B && wave == 0 && blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) plan_splits(a, lane);
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
      hi[i] = bf16_pair(y1, y2);
      lo[i] = bf16_pair(y1 - bf16_value(hi[i] & 0xffffu), y2 - __uint_as_float(hi[i] & 0xffff0000u));
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

template <int DT>
__device__ __forceinline__ bool not_finite(u32x4 x) {
  int bad = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == DT_BF16) bad |= (x[i] & 0x7f80u) == 0x7f80u;
    bad |= (x[i] & 0x7f800000u) == 0x7f800000u;
  }
  return bad != 0;
}

// ------------------------------------------------------------------------------------------------
// Scores and numerators.  A workgroup takes one head and 256 rows of the cache, a wave 16 TS of these: S^T = K_h q_h^T.  The head's
// query rows (m = h N + i: the nodes of a head one after the other, so that small trees of many heads fill the tiles of the weighted sum) lie in up
// to MAXT tiles of 16, whose other rows are other heads': zero in the query operand and written by their own workgroups.  As references the
// numerators 2^(s - ref) take the block's maximum rounded up to a multiple of 32: a bf16 or fp32 numerator is as exact at 2^-32 as at 1,
// and blocks whose maxima differ by less than that have the same reference, so that the weighted sum hardly ever needs a factor.  They
// leave as operands of that sum (lane l of a 1 KB fragment: query row l % 16, cache rows slot_row(l / 16, j)).  Bound by the chain of a short workgroup:
// lengths, keys, maxima, numerators.  16 x 21 nodes x 500..1504 x 20 x 64 28 us, 8 x 16 x 600..5000 x 24 x 96 rotary 68, 1 x 1 x 777 x 32 x 128 8.
// ------------------------------------------------------------------------------------------------
template <int DT, bool ROPE, int TS, int MAXT>
__global__ __launch_bounds__(1024 / TS) void tree_scores_kernel(TreeArgs a) {
  constexpr int VEC = Elem<DT>::VEC, KW = 4 * VEC, WV = 16 / TS, KU = 4;
  typedef typename Elem<DT>::T T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x, blk = blockIdx.y, b = blockIdx.z;
  const int len = __builtin_amdgcn_readfirstlane(seq_len_of(a.seq_lens, b, a.T)), L = len + a.N;
  plan_once(a, lane, wave);
  if (blk * TREE_BLOCK >= L) return;
  __shared__ float red[2][WV][MAXT * 16];
  __shared__ uint64_t odd[WV];
  const T* K = (const T*)a.K + (size_t)b * a.k_bstride + piece_at(h * a.d_k, a.d_k, a.banded);
  const int rp = a.banded ? a.d_k : a.d;
  const int m0 = h * a.N, m1 = h + 1 == a.H ? a.MT * 16 : m0 + a.N;      // the last head also has the rows that fill its last tile
  const int tile0 = m0 / 16, ntiles = (m1 + 15) / 16 - tile0;

  const int t0 = blk * TREE_BLOCK + wave * 16 * TS;
  int trow[TS], pos[TS];
  const uint64_t anc = ancestors(a.parents + (size_t)b * a.N, a.N, lane);
  const int depth = __popcll(anc) - 1;
#pragma unroll
  for (int ts = 0; ts < TS; ++ts) {
    const int t = min(t0 + 16 * ts + n16, L - 1);          // (rows past the end: a valid address, masked below)
    trow[ts] = t;
    if constexpr (ROPE) {
      const int dj = __shfl(depth, t - len & 63);
      pos[ts] = t < len ? t : len + max(dj, 0);
    }
  }
  f32x4 acc[TS][MAXT];
  const T* q[MAXT];
  bool mine[MAXT];
#pragma unroll
  for (int mt = 0; mt < MAXT; ++mt) {
    const int i = (tile0 + mt) * 16 + n16 - m0;
    mine[mt] = i >= 0 && i < a.N;
    q[mt] = (const T*)a.q + ((size_t)b * a.N + (mine[mt] ? i : 0)) * a.d + h * a.d_k;
#pragma unroll
    for (int ts = 0; ts < TS; ++ts) acc[ts][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bool bad[TS] = {};                                       // whether the piece of a drafted key is not finite
  for (int k0 = 0; k0 * KW < a.d_k; k0 += KU) {
    u32x4 kf[KU][TS], kl[KU][TS];
#pragma unroll
    for (int ku = 0; ku < KU; ++ku) {
      if ((k0 + ku) * KW >= a.d_k) break;
      const int j = (k0 + ku) * KW + g * VEC;
      const int at = j < a.d_k ? j : 0;                    // (d_k is whole pieces, not whole steps)
#pragma unroll
      for (int ts = 0; ts < TS; ++ts) kf[ku][ts] = *(const u32x4*)(K + row_at(trow[ts], rp, a.d) + at);
    }
#pragma unroll
    for (int ku = 0; ku < KU; ++ku) {
      if ((k0 + ku) * KW >= a.d_k) break;
      const int j = (k0 + ku) * KW + g * VEC;
      const bool in = j < a.d_k;
#pragma unroll
      for (int ts = 0; ts < TS; ++ts) {
        if (t0 + 16 * ts + 16 > len) bad[ts] |= trow[ts] >= len && not_finite<DT>(kf[ku][ts]);
        if constexpr (ROPE) {
          f32x4 cs[VEC / 4];
#pragma unroll
          for (int i = 0; i < VEC / 4; ++i) cs[i] = *(const f32x4*)(a.rope + (size_t)pos[ts] * a.d_k + (in ? j : 0) + 4 * i);
          rotate_piece<DT>(kf[ku][ts], cs, kf[ku][ts], kl[ku][ts]);
          if (!in) kl[ku][ts] = u32x4{0, 0, 0, 0};
        }
        if (!in) kf[ku][ts] = u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int mt = 0; mt < MAXT; ++mt) {
        if (mt >= ntiles) break;
        u32x4 qf = *(const u32x4*)(q[mt] + (in ? j : 0));
        if (!mine[mt] || !in) qf = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int ts = 0; ts < TS; ++ts) {
          acc[ts][mt] = mma<DT>(kf[ku][ts], qf, acc[ts][mt]);
          if constexpr (ROPE && DT == DT_BF16) acc[ts][mt] = mma<DT>(kl[ku][ts], qf, acc[ts][mt]);
        }
      }
    }
  }
  // a lane has query row n16 of each tile and the cache rows 4 g .. 4 g + 3 of each score tile
#pragma unroll
  for (int mt = 0; mt < MAXT; ++mt) {
    if (mt >= ntiles) break;
    const int i = (tile0 + mt) * 16 + n16 - m0;
    const uint64_t own = __shfl((unsigned)anc, i & 63) | (uint64_t)__shfl((unsigned)(anc >> 32), i & 63) << 32;
    const uint64_t see = mine[mt] ? own : 0;
    float mx = NEG_INF;
#pragma unroll
    for (int ts = 0; ts < TS; ++ts)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = t0 + 16 * ts + 4 * g + r - len;
        const bool on = j < 0 ? see != 0 : j < a.N && (see >> (j & 63) & 1);
        const float s = on ? acc[ts][mt][r] * a.qscale : NEG_INF;
        acc[ts][mt][r] = s;
        mx = fmaxf(mx, s);
      }
    mx = max_over_groups(mx);
    if (g == 0) red[0][wave][mt * 16 + n16] = mx;
  }
  uint64_t mask = 0;                                       // drafted rows of the wave that are not finite
#pragma unroll
  for (int ts = 0; ts < TS; ++ts) {
    uint64_t m = __ballot(bad[ts]);
    m = (m | m >> 16 | m >> 32 | m >> 48) & 0xffff;
    const int at = t0 + 16 * ts - len;
    mask |= at >= 64 || at <= -16 ? 0 : at >= 0 ? m << at : m >> -at;
  }
  if (lane == 0) odd[wave] = mask;
  lds_barrier();
  auto block_ref = [&](int at) {
    float m = red[0][0][at];
#pragma unroll
    for (int w = 1; w < WV; ++w) m = fmaxf(m, red[0][w][at]);
    return m == NEG_INF ? NEG_INF : REF_STEP * ceilf(m * (1.f / REF_STEP));
  };
#pragma unroll
  for (int mt = 0; mt < MAXT; ++mt) {
    if (mt >= ntiles) break;
    const int at = mt * 16 + n16, m = (tile0 + mt) * 16 + n16;
    const float ref = block_ref(at), sub = ref == NEG_INF ? 0.f : ref;     // (nothing visible: numerators of 0, and of NaN scores NaN)
    float l = 0.f;
#pragma unroll
    for (int ts = 0; ts < TS; ++ts)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float p = exp2_of(acc[ts][mt][r] - sub);
        if constexpr (DT == DT_BF16) p = (float)(__bf16)p; // the weighted sum takes bf16 numerators; their sum is of the same values
        acc[ts][mt][r] = p;
        l += p;
      }
    l = sum_over_row_groups(l);
    if (g == 0) red[1][wave][at] = l;
    if (m < m0 || m >= m1) continue;
    // (a wave of one score tile has half of a bf16 fragment's rows: 8 of the lane's 16 bytes)
    char* P = (char*)a.P + ((((size_t)b * a.MT + tile0 + mt) * a.CT + (size_t)blk * (TREE_BLOCK / KW)) * 64 + lane) * 16;
#pragma unroll
    for (int ts = 0; ts < TS; ++ts) {
      const int sub16 = wave * TS + ts;
      if constexpr (DT == DT_BF16) {
        const uint2 v = {__float_as_uint(acc[ts][mt][0]) >> 16 | (__float_as_uint(acc[ts][mt][1]) & 0xffff0000u),
                         __float_as_uint(acc[ts][mt][2]) >> 16 | (__float_as_uint(acc[ts][mt][3]) & 0xffff0000u)};
        if constexpr (TS % 2 == 0) {
          if (ts % 2 == 0) continue;
          const uint2 u = {__float_as_uint(acc[ts - 1][mt][0]) >> 16 | (__float_as_uint(acc[ts - 1][mt][1]) & 0xffff0000u),
                           __float_as_uint(acc[ts - 1][mt][2]) >> 16 | (__float_as_uint(acc[ts - 1][mt][3]) & 0xffff0000u)};
          *(u32x4*)(P + sub16 / 2 * 1024) = u32x4{u.x, u.y, v.x, v.y};
        } else {
          *(uint2*)(P + sub16 / 2 * 1024 + sub16 % 2 * 8) = v;
        }
      } else {
        *(u32x4*)(P + sub16 * 1024) = __builtin_bit_cast(u32x4, acc[ts][mt]);
      }
    }
  }
  lds_barrier();
  for (int at = threadIdx.x; at < ntiles * 16; at += WV * 64) {
    const int m = tile0 * 16 + at;
    if (m < m0 || m >= m1) continue;
    float l = red[1][0][at];
#pragma unroll
    for (int w = 1; w < WV; ++w) l += red[1][w][at];
    const size_t to = ((size_t)b * a.NB + blk) * a.MT * 16 + m;
    a.lsum[to] = l;
    a.ref[to] = block_ref(at);
  }
  // which drafted keys are not finite in this head's columns: they lie in this block, or in this and the next
  const int at = blk - len / TREE_BLOCK;
  if (threadIdx.x == 0 && at >= 0) {
    uint64_t any = 0;
    for (int w = 0; w < WV; ++w) any |= odd[w];
    a.odd[((size_t)b * 2 + at) * a.H + h] = any;
    if (at == 0 && (L - 1) / TREE_BLOCK == blk) a.odd[((size_t)b * 2 + 1) * a.H + h] = 0;
  }
}

// ------------------------------------------------------------------------------------------------
// The same for many rows: a workgroup of eight waves walks a range of 256-row blocks of one head, a wave 32 rows of each, with the
// head's queries resident as operands (heads of up to four steps: 128 columns in bf16, 64 in fp32) and the next block's keys in flight
// while this one's are scored.  One barrier a block, for the maxima; the sums of a block are put together behind the next one's, and its
// numerators stored behind the wait for the next one's keys, which would else be a wait for them as well.  Blocks of context alone need
// no mask.  8 x 64 nodes x 4096 x 32 x 128: 97 us, of which K (270 MB) would take 55 at a copy's rate; 1 x 26 x 16384 43.  (A workgroup's range is cut by T, not
// by the sequence's length: one short sequence of a large T is walked by few workgroups.)
// ------------------------------------------------------------------------------------------------
template <int DT, int MAXT>
__global__ __launch_bounds__(512, 1) void tree_scores_stream_kernel(TreeArgs a, int per) {
  constexpr int VEC = Elem<DT>::VEC, KW = 4 * VEC, WV = 8, TS = 2, KU = 4;
  typedef typename Elem<DT>::T T;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
  const int h = blockIdx.x, b = blockIdx.z;
  const int len = __builtin_amdgcn_readfirstlane(seq_len_of(a.seq_lens, b, a.T)), L = len + a.N;
  const int blk0 = blockIdx.y * per, blk1 = min(blk0 + per, (L + TREE_BLOCK - 1) / TREE_BLOCK);
  plan_once(a, lane, wave);
  if (blk0 >= blk1) return;
  // [block parity][maximum, sum], and the odd keys of a block, each wave's in its own place.  Two barriers without one between them leave no wave more than
  // a block ahead of another (wave 0 alone finishes blocks for all), so a place is read for the last time before the barrier behind which it may be
  // written again, two blocks on: maxima and odd keys are written before their block's barrier, read between that and the next and written again
  // behind the next; sums are written behind their block's barrier, read between the next and the one after and written again behind that.
  __shared__ float red[2][2][WV][MAXT * 16];
  __shared__ uint64_t odd[2][WV];
  const int rp = a.banded ? a.d_k : a.d, nk = (a.d_k + KW - 1) / KW;
  const T* K = (const T*)a.K + (size_t)b * a.k_bstride + piece_at(h * a.d_k, a.d_k, a.banded);
  const int m0 = h * a.N, m1 = h + 1 == a.H ? a.MT * 16 : m0 + a.N;
  const int tile0 = m0 / 16, ntiles = (m1 + 15) / 16 - tile0;

  u32x4 kf[2][KU][TS];
  auto load = [&](int blk, u32x4 (&to)[KU][TS]) {
#pragma unroll
    for (int ts = 0; ts < TS; ++ts) {
      const int t = min(blk * TREE_BLOCK + (wave * TS + ts) * 16 + n16, L - 1);
      const T* at = K + row_at(t, rp, a.d);
#pragma unroll
      for (int ku = 0; ku < KU; ++ku) {
        const int j = ku * KW + g * VEC;
        to[ku][ts] = *(const u32x4*)(at + (j < a.d_k ? j : 0));
      }
    }
  };
  load(blk0, kf[0]);
  const uint64_t anc = ancestors(a.parents + (size_t)b * a.N, a.N, lane);
  u32x4 qf[MAXT][KU];
  uint64_t see[MAXT];
#pragma unroll
  for (int mt = 0; mt < MAXT; ++mt) {
    const int i = (tile0 + mt) * 16 + n16 - m0;
    const bool mine = i >= 0 && i < a.N;
    const T* q = (const T*)a.q + ((size_t)b * a.N + (mine ? i : 0)) * a.d + h * a.d_k;
#pragma unroll
    for (int ku = 0; ku < KU; ++ku) {
      const int j = ku * KW + g * VEC;
      qf[mt][ku] = *(const u32x4*)(q + (j < a.d_k ? j : 0));
      if (!mine || j >= a.d_k) qf[mt][ku] = u32x4{0, 0, 0, 0};
    }
    const uint64_t own = __shfl((unsigned)anc, i & 63) | (uint64_t)__shfl((unsigned)(anc >> 32), i & 63) << 32;
    see[mt] = mine ? own : 0;
  }
  // the sums of a block whose waves are all past it
  auto finish = [&](int blk, int par) {
    for (int at = threadIdx.x; at < ntiles * 16; at += WV * 64) {
      const int m = tile0 * 16 + at;
      if (m < m0 || m >= m1) continue;
      float l = red[par][1][0][at];
#pragma unroll
      for (int w = 1; w < WV; ++w) l += red[par][1][w][at];
      a.lsum[((size_t)b * a.NB + blk) * a.MT * 16 + m] = l;
    }
  };
  // the odd keys of a block, between its barrier and the next
  auto note_odd = [&](int blk, int par) {
    const int at = blk - len / TREE_BLOCK;
    if (threadIdx.x == 0 && at >= 0) {
      uint64_t any = 0;
      for (int w = 0; w < WV; ++w) any |= odd[par][w];
      a.odd[((size_t)b * 2 + at) * a.H + h] = any;
      if (at == 0 && (L - 1) / TREE_BLOCK == blk) a.odd[((size_t)b * 2 + 1) * a.H + h] = 0;
    }
  };
  constexpr int PF = TS * 16 / KW;
  u32x4 pend[MAXT][PF];                                    // the last block's numerators
  auto store = [&](int blk) {
#pragma unroll
    for (int mt = 0; mt < MAXT; ++mt) {
      const int m = (tile0 + mt) * 16 + n16;
      if (m < m0 || m >= m1) continue;
      u32x4* P = (u32x4*)a.P + (((size_t)b * a.MT + tile0 + mt) * a.CT + (size_t)blk * (TREE_BLOCK / KW) + wave * PF) * 64 + lane;
#pragma unroll
      for (int f = 0; f < PF; ++f) P[f * 64] = pend[mt][f];
    }
  };
  auto step = [&](int blk, auto I) {
    const int par = I, t0 = blk * TREE_BLOCK + wave * 16 * TS;
#pragma unroll
    for (int ku = 0; ku < KU; ++ku)
#pragma unroll
      for (int ts = 0; ts < TS; ++ts) asm volatile("" : "+v"(kf[I][ku][ts]));      // (this block's keys are waited for here)
    if (blk > blk0) store(blk - 1);
    load(min(blk + 1, blk1 - 1), kf[1 - I]);
    f32x4 acc[TS][MAXT];
#pragma unroll
    for (int ts = 0; ts < TS; ++ts)
#pragma unroll
      for (int mt = 0; mt < MAXT; ++mt) acc[ts][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bool drafted = t0 + 16 * TS > len;               // (uniform) some rows are drafted ones, or past the end
    bool bad[TS] = {};
#pragma unroll
    for (int ku = 0; ku < KU; ++ku) {
      if (ku >= nk) break;
      const int j = ku * KW + g * VEC;
      const bool in = j < a.d_k;
#pragma unroll
      for (int ts = 0; ts < TS; ++ts) {
        u32x4 kx = kf[I][ku][ts];
        const int t = min(t0 + 16 * ts + n16, L - 1);
        if (drafted) bad[ts] |= t >= len && not_finite<DT>(kx);
        if (!in) kx = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int mt = 0; mt < MAXT; ++mt) {
          acc[ts][mt] = mma<DT>(kx, qf[mt][ku], acc[ts][mt]);
        }
      }
    }
#pragma unroll
    for (int mt = 0; mt < MAXT; ++mt) {
      float mx = NEG_INF;
#pragma unroll
      for (int ts = 0; ts < TS; ++ts)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (drafted) {
            const int j = t0 + 16 * ts + 4 * g + r - len;
            if (j >= 0 && !(j < a.N && (see[mt] >> (j & 63) & 1))) acc[ts][mt][r] = NEG_INF;
          }
          mx = fmaxf(mx, acc[ts][mt][r]);
        }
      mx = max_over_groups(mx);
      if (g == 0) red[par][0][wave][mt * 16 + n16] = see[mt] ? mx * a.qscale : NEG_INF;
    }
    if (drafted) {
      uint64_t mask = 0;
#pragma unroll
      for (int ts = 0; ts < TS; ++ts) {
        uint64_t m = __ballot(bad[ts]);
        m = (m | m >> 16 | m >> 32 | m >> 48) & 0xffff;
        const int at = t0 + 16 * ts - len;
        mask |= at >= 64 || at <= -16 ? 0 : at >= 0 ? m << at : m >> -at;
      }
      if (lane == 0) odd[par][wave] = mask;
    } else if (lane == 0) {
      odd[par][wave] = 0;
    }
    lds_barrier();
    if (blk > blk0) finish(blk - 1, 1 - par);
    note_odd(blk, par);
#pragma unroll
    for (int mt = 0; mt < MAXT; ++mt) {
      const int at = mt * 16 + n16, m = (tile0 + mt) * 16 + n16;
      float top = red[par][0][0][at];
#pragma unroll
      for (int w = 1; w < WV; ++w) top = fmaxf(top, red[par][0][w][at]);
      const float ref = REF_STEP * ceilf(top * (1.f / REF_STEP));
      const float sub = top == NEG_INF ? 0.f : ref;        // (nothing visible, or nothing but NaN: numerators of 0 or NaN)
      if (wave == 0 && g == 0 && m >= m0 && m < m1) a.ref[((size_t)b * a.NB + blk) * a.MT * 16 + m] = ref;
      u32x4 (&v)[PF] = pend[mt];
      float l = 0.f;
#pragma unroll
      for (int ts = 0; ts < TS; ++ts) {
        float p[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = see[mt] ? exp2_of(fmaf(acc[ts][mt][r], a.qscale, -sub)) : 0.f;
        if constexpr (DT == DT_BF16) {
          // (the weighted sum takes bf16 numerators; their sum is of the same values)
          v[0][2 * ts] = bf16_pair(p[0], p[1]);
          v[0][2 * ts + 1] = bf16_pair(p[2], p[3]);
#pragma unroll
          for (int i = 0; i < 2; ++i) l += bf16_value(v[0][2 * ts + i] & 0xffffu) + __uint_as_float(v[0][2 * ts + i] & 0xffff0000u);
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            v[ts][r] = __float_as_uint(p[r]);
            l += p[r];
          }
        }
      }
      l = sum_over_row_groups(l);
      if (g == 0) red[par][1][wave][at] = l;
    }
  };
  for (int blk = blk0; blk < blk1; blk += 2) unrolled_steps<0, 2>(blk, blk1, step);
  store(blk1 - 1);
  lds_barrier();
  finish(blk1 - 1, (blk1 - 1 - blk0) & 1);
}

// Chunks [first, end) of a sequence of L rows that its split s sums, `per` steps of 64 rows each.
constexpr int TREE_STEP = TREE_STEP_ROWS;
struct Share { int first, end; };
__device__ __forceinline__ Share split_share(int L, int s, int per, int ch) {
  const int steps = (L + TREE_STEP - 1) / TREE_STEP;
  return {min(steps, s * per) * (TREE_STEP / ch), min(min(steps, (s + 1) * per) * (TREE_STEP / ch), (L + ch - 1) / ch)};
}

// Numerators times 2^-e, e >= 0 a whole number: e off their exponents, down to 0.  (They are >= 0; one that is NaN is no longer, but then its row's
// sum is, and the row's result with it.)
__device__ __forceinline__ float lower_by(float ref, float fin) { return fin == ref ? 0.f : fminf(fin - ref, 255.f); }
template <int DT>
__device__ __forceinline__ u32x4 lowered(u32x4 p, float e) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  const unsigned n = (unsigned)e, by = DT == DT_BF16 ? n << 7 | n << 23 : n << 23;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned x = p[i];                               // (a bit cast of the element itself takes element 0)
    if constexpr (DT == DT_BF16)
      p[i] = __builtin_bit_cast(unsigned, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, by)));
    else
      p[i] = __builtin_elementwise_sub_sat(x, by);
  }
  return p;
}

// ------------------------------------------------------------------------------------------------
// Weighted sum: C^T = K^T P^T over a split of the context, for all heads together: every query row sums whole rows of K.  A wave owns
// 16 VEC columns of K (128 in bf16) and NT tiles of 16 query rows; a workgroup's four waves, one per SIMD, are four neighbouring column blocks
// of the same query rows.  K goes from memory to the wave's registers and is transposed there (no other wave of the workgroup needs it), RK
// steps of 64 rows ahead; the numerators are the same for the four waves and go through LDS, a step ahead, one barrier a step.  Bound by the matrix cores and
// what has to be issued beside them: 8 x 64 nodes x 4096 x 32 x 128 508 us (479 to
// 563), 1.10 PFLOP/s (a library product of 8192^3: 1.08 to 1.16 from run to run), 54 % of their cycles.  With eight tiles in bf16 the epilogue, not the loop, keeps 92 bytes
// a lane in scratch.
// ------------------------------------------------------------------------------------------------
template <int DT, int NT> struct Weighted {
  static constexpr int VEC = Elem<DT>::VEC, CH = 4 * VEC, SC = TREE_STEP / CH;    // chunks of a step
  static constexpr int PF = (SC * NT + 3) / 4;                                    // fragments of a step that a wave brings
  static constexpr int KR = VEC * NT > 48 ? 2 : 2 * SC;                           // chunks of K in registers, besides the one in use
  static constexpr int UN = 2 * SC == KR ? 2 : 1;                                 // steps after which the registers' roles are the same again
  static_assert(UN * SC % KR == 0 && SC % 2 == 0, "");
};

// Workgroup i -> its query tiles (mg), column blocks (dg), split and sequence.  An XCD's workgroups at one time share rows of K (same dg) and
// numerators (same mg) through its L2: it gets blocks of up to 8 mg x 6 dg.  Four neighbouring dg are 4 KB of every row, all channels of
// the L2 where rows are a multiple of that long; the 16 mg x 2 dg of before drew on a quarter of them.  An XCD gets every eighth unit: the blocks
// of a slot turn on by what that passes, or blocks of unlike size would always be the same XCDs'.
struct WeightedPlace { bool any; int mg, dg, slot; };
__host__ __device__ __forceinline__ int weighted_units(const TreeArgs& a, int NT, int* mblocks, int* dblocks) {
  *mblocks = ((a.MT + NT - 1) / NT + 7) / 8;
  *dblocks = ((a.DB + 3) / 4 + 5) / 6;
  return a.slots * *mblocks * *dblocks;
}
__device__ __forceinline__ WeightedPlace weighted_place(const TreeArgs& a, int NT, int i) {
  const int mgroups = (a.MT + NT - 1) / NT, dgroups = (a.DB + 3) / 4;
  int mblocks, dblocks;
  const int units = weighted_units(a, NT, &mblocks, &dblocks);
  const int mper = (mgroups + mblocks - 1) / mblocks, dper = (dgroups + dblocks - 1) / dblocks;
  int unit, inner;
  WeightedPlace p;
  p.any = unit_of_workgroup(i, mper * dper, units, colocate_units(units), unit, inner);
  const int blocks = mblocks * dblocks;
  p.slot = unit / blocks;
  const int block = (unit + p.slot * blocks / 8) % blocks;
  p.mg = block / dblocks * mper + inner / dper;
  p.dg = block % dblocks * dper + inner % dper;
  p.any = p.any && p.mg < mgroups && p.dg < dgroups;
  return p;
}

template <int PART, int N, class I, class F>
__device__ __forceinline__ void every_part(int st, I i, F& f) {
  if constexpr (PART < N) {
    f(st, i, std::integral_constant<int, PART>{});
    every_part<PART + 1, N>(st, i, f);
  }
}

template <int DT, int NT>
__global__ __launch_bounds__(256, 1) void tree_weighted_kernel(TreeArgs a) {
  typedef Weighted<DT, NT> G;
  constexpr int VEC = G::VEC, CW = 16 * VEC, CH = G::CH, SC = G::SC, PF = G::PF, KR = G::KR, UN = G::UN, CPB = TREE_BLOCK / CH, ROWS = NT * 16, SUB = 256 / ROWS;
  typedef typename Elem<DT>::T T;
  __shared__ u32x4 ring[2][SC * NT * 64];
  __shared__ float red[SUB][ROWS], fin[ROWS], wrow[ROWS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
  const WeightedPlace at = weighted_place(a, NT, blockIdx.x);
  if (!at.any) return;
  const int mg = at.mg, dg = at.dg, block = dg * 4 + wave;
  const bool whole = a.slots == a.B;                       // a sequence each
  int b = at.slot, s = 0, per = INT_MAX / TREE_STEP;
  if (!whole) {
    const int entry = __builtin_amdgcn_readfirstlane(a.plan[1 + at.slot]);
    if (entry < 0) return;                                 // (a slot that no sequence needs)
    b = entry / TREE_MAX_SPLITS;
    s = entry % TREE_MAX_SPLITS;
    per = __builtin_amdgcn_readfirstlane(a.plan[0]);
  }
  const int len = __builtin_amdgcn_readfirstlane(seq_len_of(a.seq_lens, b, a.T)), L = len + a.N;
  const Share share = split_share(L, s, per, CH);
  if (share.first >= share.end) return;
  const int c0 = share.first;

  const int rp = a.banded ? a.d_k : a.d;
  const T* K = (const T*)a.K + (size_t)b * a.k_bstride;
  const int piece = piece_at(min(block * CW + n16 * VEC, a.d - VEC), a.d_k, a.banded);     // (columns past the row's end are not used by anybody)
  unsigned voff[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) voff[j] = (unsigned)(piece + slot_row(g, j) * rp) * sizeof(T);
  // (addresses of loads: a uniform pointer and 32 bits of a lane)
  const char *pp[PF], *rfp[PF];
#pragma unroll
  for (int i = 0; i < PF; ++i) {
    const int f = min(wave + 4 * i, SC * NT - 1), tile = min(mg * NT + f / SC, a.MT - 1);      // (the last wave may bring a fragment twice)
    pp[i] = (const char*)a.P + (((size_t)b * a.MT + tile) * a.CT + f % SC) * 1024;
    rfp[i] = (const char*)(a.ref + ((size_t)b * a.NB * a.MT + tile) * 16);
  }
  const unsigned lane16 = lane * 16, row4 = n16 * 4;
  const size_t ref_pitch = (size_t)a.MT * 64;
  // drafted keys that are not finite: the steps that hold drafted ones are taken one by one behind the others
  const uint64_t odd = odd_keys(a, b, lane);
  const int cend = __builtin_amdgcn_readfirstlane(odd ? min(share.end, max(c0, len / TREE_STEP * SC)) : share.end), nsteps = (cend - c0 + SC - 1) / SC;

  u32x4 k[KR][VEC], kt[2][VEC], pr[PF];
  float rr[PF];
  // (rows past the cache's end: its last row, whose numerators there are 0)
  const char* kp = nullptr;                                // the chunk that is loaded
  unsigned lim = 0;
  auto load_chunk = [&](int i) {
    const int chunk = min(c0 + i, cend - 1);
    kp = (const char*)(K + row_at(chunk * CH, rp, a.d));
    lim = (unsigned)(piece + min(L - 1 - chunk * CH, CH - 1) * rp) * sizeof(T);
  };
  auto load_row = [&](int j) { return *(const u32x4*)(kp + min(voff[j], lim)); };
  auto load_p = [&](int step, int i) {
    const int chunk = c0 + min(step, nsteps - 1) * SC;
    pr[i] = *(const u32x4*)(pp[i] + (size_t)chunk * 1024 + lane16);
    rr[i] = *(const float*)(rfp[i] + chunk / CPB * ref_pitch + row4);
  };
  if (nsteps > 0) {
#pragma unroll
    for (int i = 0; i < PF; ++i) load_p(0, i);
#pragma unroll
    for (int i = 0; i < KR; ++i) {
      load_chunk(i);
#pragma unroll
      for (int j = 0; j < VEC; ++j) k[i][j] = load_row(j);
    }
  }

  // the split's reference and sum of every row
  {
    const int row = threadIdx.x % ROWS, sub = threadIdx.x / ROWS;
    const int b0 = c0 / CPB, b1 = (share.end - 1) / CPB + 1;
    const size_t first = (size_t)b * a.NB * a.MT * 16 + min(mg * NT + row / 16, a.MT - 1) * 16 + row % 16;
    const size_t pitch = (size_t)a.MT * 16;
    float top = NEG_INF;
    if (sub < SUB) {
#pragma unroll 4
      for (int blk = b0 + sub; blk < b1; blk += SUB) top = fmaxf(top, a.ref[first + blk * pitch]);
      red[sub][row] = top;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SUB; ++i) top = fmaxf(top, red[i][row]);
    if (sub == 0) fin[row] = top;
    __syncthreads();
    // (one split: its sum makes the weights; more: the first column blocks' workgroups note reference and sum for the merge)
    if (whole || dg == 0) {
      float l = 0.f;
      if (sub < SUB) {
#pragma unroll 4
        for (int blk = b0 + sub; blk < b1; blk += SUB) {
          const float r = a.ref[first + blk * pitch];
          if (blk * CPB >= c0) l += a.lsum[first + blk * pitch] * (r == top ? 1.f : exp2_of(r - top));   // (a block's sum: with its first row)
        }
        red[sub][row] = l;
      }
      __syncthreads();
      l = 0.f;
#pragma unroll
      for (int i = 0; i < SUB; ++i) l += red[i][row];
      if (!whole && sub == 0 && mg * NT + row / 16 < a.MT) {
        const size_t to = ((size_t)at.slot * a.MT + mg * NT + row / 16) * 16 + row % 16;
        a.sref[to] = top;
        a.sl[to] = l;
      }
      if (whole && sub == 0) wrow[row] = l != 0.f ? 1.f / l : 0.f;
      lds_barrier();                                       // (wrow is read by all; without steps before the odd keys' there is no other barrier in between)
    }
  }
  f32x4 acc[VEC][NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < VEC; ++c) acc[c][nt] = f32x4{0.f, 0.f, 0.f, 0.f};

  float fr[PF];
#pragma unroll
  for (int i = 0; i < PF; ++i) fr[i] = fin[min(wave + 4 * i, SC * NT - 1) / SC * 16 + n16];
  // Operands of the tiles to come: read AHEAD tiles early
  constexpr int TILES = SC * NT, AHEAD = TILES > 2 ? 2 : 1, PQ = TILES == 2 ? 2 : TILES % 3 == 0 ? 3 : 4;
  static_assert(TILES % PQ == 0, "");
  u32x4 pf[PQ];
  auto fragment = [](int at) constexpr { return at % NT * SC + at / NT; };
  if (nsteps > 0) {
#pragma unroll
    for (int i = 0; i < PF; ++i) {
      ring[0][min(wave + 4 * i, SC * NT - 1) * 64 + lane] = lowered<DT>(pr[i], lower_by(rr[i], fr[i]));
      load_p(1, i);
    }
    transpose<DT>(k[0], kt[0]);
    load_chunk(KR);
#pragma unroll
    for (int j = 0; j < VEC; ++j) k[0][j] = load_row(j);
    lds_barrier();
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) pf[i] = ring[0][fragment(i) * 64 + lane];
  }
  // One step: its products, and between them, an instruction or three behind each -- what fits beside a product of 16 cycles --, what the next
  // ones need: the next chunk's keys transposed, those of the chunk KR later requested into their registers, the next step's numerators parked and
  // those of the step after requested.  A tile's operand is read AHEAD tiles early; AHEAD tiles before the end the waves meet, so that the next
  // step's first can be.
  // the PART-th of the places of a step: product CC of its tile AT
  auto place = [&](int st, auto I, auto PART) __attribute__((always_inline)) {
    constexpr int at = PART / VEC, cc = PART % VEC, c = at / NT, nt = at % NT;
    u32x4 (&next)[VEC] = k[(I * SC + c + 1) % KR], (&ktn)[VEC] = kt[(c + 1) & 1];
    if constexpr (cc == 0) {
      if constexpr (at == TILES - AHEAD) lds_barrier();
      if constexpr (at + AHEAD < TILES) pf[(at + AHEAD) % PQ] = ring[st & 1][fragment(at + AHEAD) * 64 + lane];
      else pf[(at + AHEAD) % PQ] = ring[st + 1 & 1][fragment(at + AHEAD - TILES) * 64 + lane];
      operands_ready(acc, nt);
      __builtin_amdgcn_sched_barrier(0);
    }
    mma_in_place<DT>(kt[c & 1][cc], pf[at % PQ], acc[cc][nt]);
    if constexpr (nt == 0 && cc == 0) load_chunk(st * SC + c + 1 + KR);
    // of this tile: row groups [j0, j1) of the next chunk, transposed in the first `slots` places, their registers filled again in the others
    constexpr int j0 = 4 * nt / NT, n = 4 * (nt + 1) / NT - j0, slots = n <= 1 ? VEC / 2 : n <= 2 ? VEC * 3 / 4 : VEC, rows = n * VEC / 4;
    if constexpr (cc < slots) {
#pragma unroll
      for (int t = n * VEC * cc / slots; t < n * VEC * (cc + 1) / slots; ++t) transpose_one<DT>(next, ktn, j0 + t / VEC, t % VEC);
    }
#pragma unroll
    for (int r = 0; r < rows; ++r)
      if (cc == (slots < VEC ? slots + r * (VEC - slots) / (rows ? rows : 1) : VEC - 1)) next[j0 * VEC / 4 + r] = load_row(j0 * VEC / 4 + r);
    // fragments parked beside this tile
    constexpr int i0 = PF * at / (TILES - AHEAD), i1 = at < TILES - AHEAD ? PF * (at + 1) / (TILES - AHEAD) : i0;
#pragma unroll
    for (int i = i0; i < i1; ++i) {
      if constexpr (cc == 0) pr[i] = lowered<DT>(pr[i], lower_by(rr[i], fr[i]));
      if constexpr (cc == VEC / 2) ring[st + 1 & 1][min(wave + 4 * i, TILES - 1) * 64 + lane] = pr[i];
      if constexpr (cc == VEC - 1) load_p(st + 2, i);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](int st, auto I) __attribute__((always_inline)) { every_part<0, TILES * VEC>(st, I, place); };
  int st = 0;
  for (; st + UN <= nsteps; st += UN) full_steps<0, UN>(st, step);
  unrolled_steps<0, UN>(st, nsteps, step);

  if (odd) {
    // A drafted key that is not finite must not reach nodes that do not see it (0 times infinity is no 0): it enters the sum as 0, and the
    // projection makes NaN of the nodes that do see it.
    for (int chunk = max(c0, len / TREE_STEP * SC); chunk < share.end; ++chunk) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const int t = min(chunk * CH + slot_row(g, j), L - 1);
        k[0][j] = *(const u32x4*)(K + piece + row_at(t, rp, a.d));
        if (t >= len && (odd >> (t - len) & 1)) k[0][j] = u32x4{0, 0, 0, 0};
      }
      transpose<DT>(k[0], kt[0]);
#pragma unroll
      for (int c = 0; c < VEC; ++c) operands_ready(kt[0][c]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        u32x4 pf = ((const u32x4*)a.P)[(((size_t)b * a.MT + min(mg * NT + nt, a.MT - 1)) * a.CT + chunk) * 64 + lane];
        pf = lowered<DT>(pf, lower_by(a.ref[((size_t)b * a.NB + chunk / CPB) * a.MT * 16 + min(mg * NT + nt, a.MT - 1) * 16 + n16], fin[nt * 16 + n16]));
        operands_ready(pf);
        operands_ready(acc, nt);
#pragma unroll
        for (int c = 0; c < VEC; ++c) mma_in_place<DT>(kt[0][c], pf, acc[c][nt]);
      }
    }
  }

  settle();
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int c = 0; c < VEC; ++c) asm volatile("" : "+a"(acc[c][nt]));      // (nothing reads them before that wait)
  // a lane has query row n16 of each tile and the columns 4 VEC g + VEC r + c of the block, which the projection reads as operands
  if (block >= a.DB) return;
  uint64_t anc = 0;
  if (odd && whole) anc = ancestors(a.parents + (size_t)b * a.N, a.N, lane);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (mg * NT + nt >= a.MT) continue;
    const size_t row = (size_t)at.slot * a.MT + mg * NT + nt;
    if (whole) {
      float w = wrow[nt * 16 + n16];
      if (odd && __shfl((anc & odd) != 0 ? 1 : 0, ((mg * NT + nt) * 16 + n16) % a.N)) w = __builtin_nanf("");
      u32x4* out = (u32x4*)a.Cop + (row * a.DB + block) * VEC * 64 + lane;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v[VEC];
#pragma unroll
        for (int c = 0; c < VEC; ++c) v[c] = w == 0.f ? 0.f : acc[c][nt][r] * w;
        store_operand<DT>(v, out + r * (VEC / 4) * 64);
      }
    } else {
      f32x4* C = (f32x4*)a.C + (row * a.DB + block) * VEC * 64 + lane;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int hf = 0; hf < VEC / 4; ++hf)
          C[(r * (VEC / 4) + hf) * 64] = f32x4{acc[hf * 4][nt][r], acc[hf * 4 + 1][nt][r], acc[hf * 4 + 2][nt][r], acc[hf * 4 + 3][nt][r]};
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Merge of the splits: C = sum_s w_s C_s, w_s = 2^(ref_s - max) over the whole sum, into operands of the projection.  A workgroup takes one query
// tile and `per` column blocks of it.  (The projection itself read a tile once for every head that has rows in it, every split of it: 1 x 2
// nodes x 16384 x 32 x 128 54 us.)
// ------------------------------------------------------------------------------------------------
template <int DT>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, int per) {
  constexpr int VEC = Elem<DT>::VEC;
  const int lane = threadIdx.x & 63, n16 = lane & 15, r = threadIdx.x >> 6, tile = blockIdx.x, b = blockIdx.z;
  __shared__ float weight[TREE_MAX_SPLITS][16];
  __shared__ bool nothing[16];                             // an unused slot's row: its sums may be anything
  const int entry = a.plan[1 + a.slots + b], slot0 = entry / (2 * TREE_MAX_SPLITS), ns = entry % (2 * TREE_MAX_SPLITS);
  if (r == 0) {
    bool nan = false;                                      // (a node that sees a drafted key that is not finite)
    if (const uint64_t odd = odd_keys(a, b, lane)) {
      const uint64_t anc = ancestors(a.parents + (size_t)b * a.N, a.N, lane);
      nan = __shfl((anc & odd) != 0 ? 1 : 0, (tile * 16 + n16) % a.N);
    }
    const size_t at = ((size_t)slot0 * a.MT + tile) * 16 + n16, pitch = (size_t)a.MT * 16;
    float top = NEG_INF, sum = 0.f;
#pragma unroll 4
    for (int s = 0; s < ns; ++s) top = fmaxf(top, a.sref[at + s * pitch]);
#pragma unroll 4
    for (int s = 0; s < ns; ++s) sum += a.sl[at + s * pitch] * (top == NEG_INF ? 1.f : exp2_of(a.sref[at + s * pitch] - top));
    for (int s = lane >> 4; s < ns; s += 4) {
      const float w = sum == 0.f ? 0.f : (top == NEG_INF ? 1.f : exp2_of(a.sref[at + s * pitch] - top)) / sum;
      weight[s][n16] = nan ? __builtin_nanf("") : w;
    }
    if (lane < 16) nothing[n16] = sum == 0.f && !nan;
  }
  lds_barrier();
  const int end = min(a.DB, (int)(blockIdx.y + 1) * per);
  for (int blk = blockIdx.y * per; blk < end; ++blk) {
    const f32x4* C = (const f32x4*)a.C + (((size_t)slot0 * a.MT + tile) * a.DB + blk) * VEC * 64 + r * (VEC / 4) * 64 + lane;
    const size_t pitch = (size_t)a.MT * a.DB * VEC * 64;
    float v[VEC] = {};
#pragma unroll 4
    for (int s = 0; s < ns; ++s) {
      const float w = weight[s][n16];
#pragma unroll
      for (int hf = 0; hf < VEC / 4; ++hf) {
        const f32x4 x = C[s * pitch + hf * 64];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[hf * 4 + j] += x[j] * w;      // (a weight may vanish, but not a value that is not finite)
      }
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[j] = nothing[n16] ? 0.f : v[j];
    store_operand<DT>(v, (u32x4*)a.Cop + (((size_t)b * a.MT + tile) * a.DB + blk) * VEC * 64 + r * (VEC / 4) * 64 + lane);
  }
}

// ------------------------------------------------------------------------------------------------
// Projection: out[i, h] = C[h N + i] W_KV[:, h].  A workgroup of four waves, one per SIMD, takes one head (or 16 VEC columns of one), NM of the query
// tiles that hold rows of it (of any sequence) and a range of rows of W_KV, which the waves share out 4 VEC at a time; what they load lies
// RD turns ahead in registers, and their sums meet in LDS.  1 x 1 node x 32 x 128: W_KV (33.5 MB) in 13 us, 2.5 TB/s, half of it the start and the end;
// 8 x 64 71 us, C read once for every head that has rows in a tile.
// ------------------------------------------------------------------------------------------------
template <int DT, int NM>
__global__ __launch_bounds__(256, 1) void tree_project_kernel(TreeArgs a) {
  constexpr int VEC = Elem<DT>::VEC, CW = 16 * VEC, PITCH = CW + 4, OPS = VEC / 4, RD = NM == 4 ? 2 : 4;
  typedef typename Elem<DT>::T T;
  __shared__ __align__(16) float sums[4 * 16 * PITCH];     // [wave][row][column]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
  const int cblocks = (a.d_k + CW - 1) / CW;               // column blocks of a head
  const int cs = blockIdx.x % a.csw, hc = blockIdx.x / a.csw, h = hc / cblocks, cb = hc % cblocks;
  const int tile0 = h * a.N / 16, ntiles = (h * a.N + a.N - 1) / 16 - tile0 + 1;
  const int x0 = blockIdx.y * NM;
  if (x0 >= a.B * ntiles) return;
  int tb[NM], tt[NM];
  const u32x4* C[NM];
#pragma unroll
  for (int i = 0; i < NM; ++i) {
    const int x = min(x0 + i, a.B * ntiles - 1);
    tb[i] = x / ntiles;
    tt[i] = tile0 + x % ntiles;
    C[i] = (const u32x4*)a.Cop + ((size_t)tb[i] * a.MT + tt[i]) * a.DB * VEC * 64 + lane;
  }
  const int hcol = cb * CW + n16 * VEC;                    // column of the head that the lane loads
  const T* W = (const T*)a.W + h * a.d_k + (hcol < a.d_k ? hcol : 0);
  const int turns = a.DB * 4, per = (turns + a.csw * 4 - 1) / (a.csw * 4) * 4, first = cs * per + wave, end = min(turns, cs * per + per);
  u32x4 w[RD][VEC], c[RD][NM][OPS];
  auto load = [&](int turn, u32x4 (&wr)[VEC], u32x4 (&cr)[NM][OPS]) {
    const int t = min(turn, turns - 1);
    const int row = t / 4 * CW + 4 * VEC * g + VEC * (t % 4);      // of W_KV, column of C
#pragma unroll
    for (int j = 0; j < VEC; ++j) wr[j] = *(const u32x4*)(W + (size_t)((row < a.d ? row : 0) + j) * a.d);   // (d is whole pieces)
#pragma unroll
    for (int i = 0; i < NM; ++i)
#pragma unroll
      for (int o = 0; o < OPS; ++o) cr[i][o] = C[i][(size_t)t * OPS * 64 + o * 64];
  };
  f32x4 acc[NM][VEC];
#pragma unroll
  for (int i = 0; i < NM; ++i)
#pragma unroll
    for (int k = 0; k < VEC; ++k) acc[i][k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < RD; ++i) load(first + 4 * i, w[i], c[i]);
  auto step = [&](int n, auto I) {
    const int t = first + 4 * n;
    const bool there = t / 4 * CW + 4 * VEC * g + VEC * (t % 4) < a.d;
    u32x4 wt[VEC], x[NM][OPS];
    transpose<DT>(w[I], wt);
#pragma unroll
    for (int i = 0; i < NM; ++i)
#pragma unroll
      for (int o = 0; o < OPS; ++o) x[i][o] = there ? c[I][i][o] : u32x4{0, 0, 0, 0};      // (columns past C's end may hold anything)
    load(t + 4 * RD, w[I], c[I]);
#pragma unroll
    for (int i = 0; i < NM; ++i)
#pragma unroll
      for (int o = 0; o < OPS; ++o)
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[i][k] = mma<DT>(wt[k], x[i][o], acc[i][k]);
  };
  const int nsteps = (end - first + 3) / 4;
  int n = 0;
  for (; n + RD <= nsteps; n += RD) full_steps<0, RD>(n, step);
  unrolled_steps<0, RD>(n, nsteps, step);
#pragma unroll
  for (int i = 0; i < NM; ++i) {
    if (x0 + i >= a.B * ntiles) break;
    // (a lane has query row n16 and the columns VEC (4 g + r) + k)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int hf = 0; hf < VEC / 4; ++hf)
        *(f32x4*)(sums + (wave * 16 + n16) * PITCH + VEC * (4 * g + r) + hf * 4) =
            f32x4{acc[i][hf * 4][r], acc[i][hf * 4 + 1][r], acc[i][hf * 4 + 2][r], acc[i][hf * 4 + 3][r]};
    lds_barrier();
    for (int e = threadIdx.x; e < 16 * CW / 4; e += 256) {
      const int row = e / (CW / 4), c4 = e % (CW / 4) * 4, m = tt[i] * 16 + row;
      if (m / a.N == h && cb * CW + c4 < a.d_k) {
        f32x4 v = *(const f32x4*)(sums + row * PITCH + c4);
#pragma unroll
        for (int w = 1; w < 4; ++w) v += *(const f32x4*)(sums + (w * 16 + row) * PITCH + c4);
        const size_t node = (size_t)tb[i] * a.N + m % a.N;
        const int at = h * a.d_k + cb * CW + c4;
        if (a.csw > 1) {
          *(f32x4*)(a.part + ((size_t)cs * a.B * a.N + node) * a.d + at) = v;
        } else if constexpr (DT == DT_BF16) {
          *(uint2*)((uint16_t*)a.out + node * a.d + at) =
              uint2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
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
    ((uint2*)out)[i] = uint2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
  else
    ((f32x4*)out)[i] = v;
}

// Tiles of 16 query rows that a head's rows can lie in at most: they begin at multiples of the common divisor of N and 16.
int tree_head_tiles(int N) {
  int div = 16;
  while (N % div) div /= 2;
  return (16 - div + N + 15) / 16;
}
// Query tiles that a workgroup of the projection takes together.
int tree_project_tiles(long tiles) { return tiles <= 1 ? 1 : tiles <= 2 ? 2 : 4; }

template <int DT, bool ROPE, int TS>
void launch_tree_scores_s(const TreeArgs& a, hipStream_t st) {
  const dim3 grid(a.H, a.NB, a.B), block(1024 / TS);
  if (a.N <= 17) hipLaunchKernelGGL((tree_scores_kernel<DT, ROPE, TS, 2>), grid, block, 0, st, a);      // (a head's rows touch two tiles at most)
  else hipLaunchKernelGGL((tree_scores_kernel<DT, ROPE, TS, 5>), grid, block, 0, st, a);
}
// Two score tiles a wave and twice the waves where a wave of four keeps more than two query tiles' sums, 200 registers: 16 x 21 nodes x 1504 x 20 x 64
// 104.9 -> 99.0 us for the call, 4 x 40 x 8000 x 12 x 72 113.9 -> 107.8; of two query tiles 319.6 -> 336.3 (24 x 5 x 6000 x 16 x 128), 157.5 -> 161.3 (8 x 16 x
// 3000 x 32 x 80).  And for rotary keys, with two tiles 72 -> 70 (8 x 16 x 5000 x 24 x 96; cos and sin asked for together with the keys 88).
template <int DT, bool ROPE>
void launch_tree_scores_w(const TreeArgs& a, hipStream_t st) {
  if constexpr (ROPE) {
    launch_tree_scores_s<DT, ROPE, 2>(a, st);
  } else {
    if (a.N > 17) launch_tree_scores_s<DT, ROPE, 2>(a, st);
    else launch_tree_scores_s<DT, ROPE, 4>(a, st);
  }
}
template <int DT, bool ROPE>
void launch_tree_scores_r(const TreeArgs& a, hipStream_t st) {
  const long blocks = (long)a.H * a.NB * a.B;
  if (blocks <= 512) return launch_tree_scores_s<DT, ROPE, 1>(a, st);     // few workgroups: more waves of fewer rows
  // The walk where its four steps of a row are all used, there is no rotation to wait for, and a round of workgroups holds every head: 8 x 64
  // nodes x 4096 x 32 x 128 175 -> 105 us, 4 ragged x 32 x 8000 86 -> 62, 1 x 2 x 16384 40 -> 31; but heads of 64 columns 34 -> 38 (16 x 21 x
  // 1504 x 20), rotary ones 72 -> 100 (8 x 16 x 5000 x 24 x 96), 384 heads in a batch 112 -> 119 (24 x 5 x 6000 x 16 x 128).
  constexpr int W = 16 * Elem<DT>::VEC;
  const int tiles = tree_head_tiles(a.N);
  if (ROPE || a.d_k > W || a.d_k <= W * 3 / 4 || tiles > 4 || a.H * a.B > 256) return launch_tree_scores_w<DT, ROPE>(a, st);
  const int z = std::min(a.NB, 256 / (a.H * a.B)), per = (a.NB + z - 1) / z;
  const dim3 grid(a.H, (a.NB + per - 1) / per, a.B);
  switch (tiles) {
    case 1: hipLaunchKernelGGL((tree_scores_stream_kernel<DT, 1>), grid, dim3(512), 0, st, a, per); break;
    case 2: hipLaunchKernelGGL((tree_scores_stream_kernel<DT, 2>), grid, dim3(512), 0, st, a, per); break;
    case 3: hipLaunchKernelGGL((tree_scores_stream_kernel<DT, 3>), grid, dim3(512), 0, st, a, per); break;
    default: hipLaunchKernelGGL((tree_scores_stream_kernel<DT, 4>), grid, dim3(512), 0, st, a, per); break;
  }
}
template <int DT>
void launch_tree_scores_t(const TreeArgs& a, hipStream_t st) {
  if (a.rope) launch_tree_scores_r<DT, true>(a, st);
  else launch_tree_scores_r<DT, false>(a, st);
}

template <int DT>
void launch_tree_weighted_t(const TreeArgs& a, int nt, hipStream_t st) {
  int mblocks, dblocks;
  const int units = weighted_units(a, nt, &mblocks, &dblocks);
  const int mper = ((a.MT + nt - 1) / nt + mblocks - 1) / mblocks, dper = ((a.DB + 3) / 4 + dblocks - 1) / dblocks;
  const dim3 grid(unit_grid(units, mper * dper, colocate_units(units)));
  switch (nt) {
    case 1: hipLaunchKernelGGL((tree_weighted_kernel<DT, 1>), grid, dim3(256), 0, st, a); break;
    case 2: hipLaunchKernelGGL((tree_weighted_kernel<DT, 2>), grid, dim3(256), 0, st, a); break;
    case 3: hipLaunchKernelGGL((tree_weighted_kernel<DT, 3>), grid, dim3(256), 0, st, a); break;
    case 4: hipLaunchKernelGGL((tree_weighted_kernel<DT, 4>), grid, dim3(256), 0, st, a); break;
    case 6: hipLaunchKernelGGL((tree_weighted_kernel<DT, 6>), grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL((tree_weighted_kernel<DT, 8>), grid, dim3(256), 0, st, a); break;
  }
}

template <int DT>
void launch_tree_merge_t(const TreeArgs& a, hipStream_t st) {
  const int per = (int)std::max(1l, (long)a.B * a.MT * a.DB / 2048);
  hipLaunchKernelGGL(tree_merge_kernel<DT>, dim3(a.MT, (a.DB + per - 1) / per, a.B), dim3(256), 0, st, a, per);
}

template <int DT>
void launch_tree_project_t(const TreeArgs& a, hipStream_t st) {
  constexpr int CW = 16 * Elem<DT>::VEC;
  const int heads = a.H * ((a.d_k + CW - 1) / CW), tiles = a.B * tree_head_tiles(a.N), nm = tree_project_tiles(tiles);
  const dim3 grid(heads * a.csw, (tiles + nm - 1) / nm), block(256);
  if (nm == 1) hipLaunchKernelGGL((tree_project_kernel<DT, 1>), grid, block, 0, st, a);
  else if (nm == 2) hipLaunchKernelGGL((tree_project_kernel<DT, 2>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((tree_project_kernel<DT, 4>), grid, block, 0, st, a);
  if (a.csw > 1) {
    const size_t n4 = (size_t)a.B * a.N * a.d / 4;
    hipLaunchKernelGGL(tree_sum_kernel<DT>, dim3((n4 + 255) / 256), dim3(256), 0, st, a.part, a.csw, n4, a.out);
  }
}

}  // namespace

// How the weighted sum is cut: NT query tiles of 16 rows to a wave, and slots, each a range of a sequence's rows.  The fewest tiles of the sizes that
// there are in the fewest groups of eight at most; more slots than sequences where there are two for each before the workgroups are as many as the
// compute units (the merge that they need takes 5-16 us, which fewer would hardly gain), in whole rounds over the XCDs, and of `per_min` steps at least.
void tree_cut(int dtype, int B, int N, int H, int T, int d, int* nt, int* slots, int* per_min) {
  const int mt = (H * N + 15) / 16, groups = (mt + 7) / 8, each = (mt + groups - 1) / groups, cw = 16 * vec_elems(dtype);
  *nt = each > 6 ? 8 : each > 4 ? 6 : each;
  const int mgroups = (mt + *nt - 1) / *nt, dgroups = (d + 4 * cw - 1) / (4 * cw), blocks = (mgroups + 7) / 8 * ((dgroups + 5) / 6);
  const int steps = (T + N + TREE_STEP - 1) / TREE_STEP, least = dtype == DT_F32 ? 2 : 4;
  *per_min = std::max(least, (steps + TREE_MAX_SPLITS - 1) / TREE_MAX_SPLITS);
  const long room = 256 / ((long)mgroups * dgroups), whole = blocks % 8 == 0 ? 1 : blocks % 4 == 0 ? 2 : blocks % 2 == 0 ? 4 : 8;
  *slots = B;
  if (room < 2 * (long)B) return;
  const long most = std::min(room, (long)B * std::min((steps + least - 1) / least, TREE_MAX_SPLITS));
  *slots = (int)std::max<long>(B, most >= whole ? most / whole * whole : most);
}

// Row splits of W_KV in the projection: until there is a workgroup for every compute unit, a turn for each wave at least.
int tree_row_splits(int dtype, int B, int N, int H, int d) {
  const int cw = 16 * vec_elems(dtype), d_k = d / H, db = (d + cw - 1) / cw;
  const long tiles = (long)B * tree_head_tiles(N), nm = tree_project_tiles(tiles), wgs = (long)H * ((d_k + cw - 1) / cw) * ((tiles + nm - 1) / nm);
  return (int)std::max(1l, std::min<long>({(256 + wgs - 1) / wgs, db, 16}));
}

// A sequence has `cuts` slots at most (tree_cut's `most`), and room * MT <= 256 MT / (mgroups dgroups), where MT / mgroups <= min(MT, 8).
size_t tree_most_split_tiles(int dtype, int B, int N, int H, int T, int d) {
  const int mt = (H * N + 15) / 16, cw = 16 * vec_elems(dtype), dgroups = (d + 4 * cw - 1) / (4 * cw), steps = (T + N + TREE_STEP - 1) / TREE_STEP;
  const int least = dtype == DT_F32 ? 2 : 4, cuts = std::min((steps + least - 1) / least, TREE_MAX_SPLITS);
  return cuts > 1 ? std::min<size_t>((size_t)B * cuts * mt, 256 * std::min(mt, 8) / dgroups) : 0;
}

// With csw > 1 there are fewer than 256 workgroups, so csw <= 256 / wgs + 1 <= 512 / wgs, and wgs >= H cblocks B N / 64 (four tiles of 16 rows a workgroup at most).
size_t tree_most_split_rows(int dtype, int B, int N, int H, int d) {
  const int cw = 16 * vec_elems(dtype), cblocks = (d / H + cw - 1) / cw, db = (d + cw - 1) / cw;
  return db > 1 ? std::min<size_t>((size_t)std::min(db, 16) * B * N, 512 * 64 / ((long)H * cblocks)) : 0;
}

void launch_tree_scores(int dtype, const TreeArgs& a, hipStream_t st) {
  if (dtype == DT_BF16) launch_tree_scores_t<DT_BF16>(a, st);
  else launch_tree_scores_t<DT_F32>(a, st);
}
void launch_tree_weighted(int dtype, const TreeArgs& a, hipStream_t st) {
  if (dtype == DT_BF16) launch_tree_weighted_t<DT_BF16>(a, a.NT, st);
  else launch_tree_weighted_t<DT_F32>(a, a.NT, st);
}
void launch_tree_merge(int dtype, const TreeArgs& a, hipStream_t st) {
  if (dtype == DT_BF16) launch_tree_merge_t<DT_BF16>(a, st);
  else launch_tree_merge_t<DT_F32>(a, st);
}
void launch_tree_project(int dtype, const TreeArgs& a, hipStream_t st) {
  if (dtype == DT_BF16) launch_tree_project_t<DT_BF16>(a, st);
  else launch_tree_project_t<DT_F32>(a, st);
}

}  // namespace slim
