// What follows the attention of a tree of drafted tokens: the walk down the tree that accepts or rejects them, the draw of the next token,
// and the move of the accepted path's keys to their places in the cache.
#include "slim_kernels.h"

#include "device_common.h"

namespace slim {
namespace {

constexpr int VW = 16;                       // waves of a verifying workgroup
constexpr int RUN = 4;                       // pieces of 16 bytes that a thread takes at most where the next token is looked for

template <int DT> struct Prob;
template <> struct Prob<DT_F32> {
  static constexpr int VEC = 4;
  typedef float T;
  static __device__ __forceinline__ float value(float x) { return x; }
  static __device__ __forceinline__ float get(const u32x4& x, int j) { return __uint_as_float(x[j]); }
  static __device__ __forceinline__ void clear(u32x4& x, int j) { x[j] = 0; }
  static __device__ __forceinline__ void set(u32x4& x, int j, float v) { x[j] = __float_as_uint(v); }
};
template <> struct Prob<DT_BF16> {
  static constexpr int VEC = 8;
  typedef uint16_t T;
  static __device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((unsigned)x << 16); }
  static __device__ __forceinline__ float get(const u32x4& x, int j) { return __uint_as_float(j & 1 ? x[j >> 1] & 0xffff0000u : x[j >> 1] << 16); }
  static __device__ __forceinline__ void clear(u32x4& x, int j) { x[j >> 1] &= j & 1 ? 0xffffu : 0xffff0000u; }
  static __device__ __forceinline__ void set(u32x4& x, int j, uint16_t v) { x[j >> 1] |= (unsigned)v << (j & 1 ? 16 : 0); }
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s);
  return v;
}

// What is left of a node's distribution: max(p - a q, 0) with a draft, p without the excluded tokens else.  The rows are read in pieces of 16 bytes
// on 16-byte boundaries (p and draft are aligned, so a row of p and its row of the draft begin alike): the first may begin with `skip` elements of the
// row before, which count as 0, and what does not fill the last is read one by one.
template <int DT, bool DRAFT>
struct Residual {
  typedef Prob<DT> E;
  typedef typename E::T T;
  static constexpr int VEC = E::VEC, U = DRAFT ? 4 : 8;     // pieces of each that a lane has in flight
  const T *p, *q;                            // the row's first piece
  int skip, V, full, pieces;                 // whole pieces, all pieces
  double am;
  int lane, tok;                             // excluded: tokens of the lanes in `out`
  uint64_t out, near;                        // near: bit piece / 64 % 64 of every excluded one

  __device__ Residual(const VerifyArgs& a, int b, int node, double am_, uint64_t out_, int tok_) : am(am_), tok(tok_), out(out_), near(0) {
    const size_t at = ((size_t)b * a.N + node) * a.V;
    lane = threadIdx.x & 63;
    skip = (int)(at % VEC);
    V = a.V;
    p = (const T*)a.p + at - skip;
    q = DRAFT ? (const T*)a.draft + at - skip : nullptr;
    full = (skip + V) / VEC;
    pieces = (skip + V + VEC - 1) / VEC;
    if constexpr (!DRAFT)
      for (uint64_t m = out; m; m &= m - 1) near |= 1ull << (__builtin_amdgcn_readlane(tok, __ffsll((unsigned long long)m) - 1) + skip) / VEC / 64 % 64;
  }
  __device__ __forceinline__ void mask(int k, u32x4& x, u32x4& y) const {
    if (k == 0) {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (j < skip) {
          E::clear(x, j);
          E::clear(y, j);
        }
    }
    if constexpr (!DRAFT) {
      if (near >> (k / 64 % 64) & 1)
        for (uint64_t m = out; m; m &= m - 1) {
          const int v = __builtin_amdgcn_readlane(tok, __ffsll((unsigned long long)m) - 1) + skip - k * VEC;
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (j == v) E::clear(x, j);
        }
    }
  }
  template <bool USEQ>
  __device__ __forceinline__ double value(const u32x4& x, const u32x4& y, int j) const {
    if constexpr (USEQ) return fmax((double)E::get(x, j) - am * (double)E::get(y, j), 0.0);
    else return (double)E::get(x, j);
  }
  // piece k of the two rows, zeros past the end
  template <bool USEQ>
  __device__ __forceinline__ void piece(int k, u32x4& x, u32x4& y) const {
    x = y = u32x4{0, 0, 0, 0};
    if (k < full) {
      x = ((const u32x4*)p)[k];
      if constexpr (USEQ) y = ((const u32x4*)q)[k];
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (k * VEC + j < skip + V) {
          E::set(x, j, p[k * VEC + j]);
          if constexpr (USEQ) E::set(y, j, q[k * VEC + j]);
        }
    }
    mask(k, x, y);
  }
  // sum over the pieces [ka, kb), the same in every lane of the wave
  template <bool USEQ>
  __device__ double sum(int ka, int kb) const {
    const int fb = min(kb, full);
    double s = 0;
    for (int k = ka; k < fb; k += 64 * U) {
      u32x4 x[U], y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = min(k + u * 64 + lane, fb - 1);
        x[u] = ((const u32x4*)p)[at];
        if constexpr (USEQ) y[u] = ((const u32x4*)q)[at];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = k + u * 64 + lane;
        if (at >= fb) break;
        mask(at, x[u], y[u]);
#pragma unroll
        for (int j = 0; j < VEC; ++j) s += value<USEQ>(x[u], y[u], j);
      }
    }
    if (kb > full && ka <= full && lane == 0) {
      u32x4 x, y;
      piece<USEQ>(full, x, y);
#pragma unroll
      for (int j = 0; j < VEC; ++j) s += value<USEQ>(x, y, j);
    }
    return wave_sum(s);
  }
};

// The pieces [k0, k1) in VW parts, one a wave; their sums into part[].  Returns the whole sum.
template <bool USEQ, class R>
__device__ double sum_parts(const R& r, int k0, int k1, double* part) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), per = (k1 - k0 + VW - 1) / VW, ka = k0 + wave * per;
  const double s = ka < k1 ? r.template sum<USEQ>(ka, min(k1, ka + per)) : 0.0;
  __syncthreads();                           // (what part[] held has been read)
  if (r.lane == 0) part[wave] = s;
  __syncthreads();
  double all = 0;
#pragma unroll
  for (int w = 0; w < VW; ++w) all += part[w];
  return all;
}

// The lowest token whose running sum is over u times the whole sum, or the last with any weight where there is none; -1 where nothing has weight.
// The sums of a pass over the row say which of VW parts holds it; a part of up to 1024 RUN pieces (a vocabulary of 262144 in fp32, 524288 in bf16) is then scanned,
// a few pieces a thread, a larger one is summed in parts again.
template <bool USEQ, class R>
__device__ int draw(const R& r, double u, double* part) {
  constexpr int VEC = R::VEC;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int k0 = 0, k1 = r.pieces;
  double run = 0, border = 0;
  for (bool first = true;; first = false) {
    const double all = sum_parts<USEQ>(r, k0, k1, part);
    if (first) {
      if (!(all > 0)) return -1;
      border = u * all;
    }
    const int per = (k1 - k0 + VW - 1) / VW;
    int at = -1, with = 0;
    double before = run, acc = run;
    for (int w = 0; w < VW; ++w) {
      const double s = part[w];
      if (s > 0 && at < 0) {
        with = w;
        before = acc;
        if (acc + s > border) at = w;
      }
      acc += s;
    }
    if (at < 0) at = with;                   // (rounding, or u = 1: the last part with any weight)
    run = before;
    const int lo = k0 + at * per;
    k1 = min(k1, lo + per);
    k0 = lo;
    if (k1 - k0 <= VW * 64 * RUN) break;
  }
  // a thread's neighbouring pieces, the running sum before and after them
  const int each = (k1 - k0 + VW * 64 - 1) / (VW * 64);
  u32x4 x[RUN], y[RUN];
  double own = 0;
#pragma unroll
  for (int i = 0; i < RUN; ++i) {
    const int k = k0 + tid * each + i;
    x[i] = y[i] = u32x4{0, 0, 0, 0};
    if (i < each && k < k1) r.template piece<USEQ>(k, x[i], y[i]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) own += r.template value<USEQ>(x[i], y[i], j);
  }
  double incl = own;
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const double o = __shfl_up(incl, k);
    if (lane >= k) incl += o;
  }
  double excl = __shfl_up(incl, 1);
  if (lane == 0) excl = 0;
  __syncthreads();
  if (lane == 63) part[wave] = incl;
  __syncthreads();
  double base = run;
  for (int w = 0; w < wave; ++w) base += part[w];
  incl += base;
  excl += base;
  // the first thread over the border, the last with any weight; of the one that counts, the token
  __shared__ int over[VW], any[VW], found;
  const unsigned long long mo = __ballot(own > 0 && incl > border), ma = __ballot(own > 0);
  if (lane == 0) {
    over[wave] = mo ? wave * 64 + __ffsll(mo) - 1 : VW * 64;
    any[wave] = ma ? wave * 64 + 63 - __clzll(ma) : -1;
  }
  __syncthreads();
  int to = VW * 64, ta = -1;
#pragma unroll
  for (int w = 0; w < VW; ++w) {
    to = min(to, over[w]);
    ta = max(ta, any[w]);
  }
  if (tid == (to < VW * 64 ? to : ta)) {
    int hit = -1, last = 0;
    double s = excl;
#pragma unroll
    for (int i = 0; i < RUN; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const double v = r.template value<USEQ>(x[i], y[i], j);
        const int at = (k0 + tid * each + i) * VEC + j - r.skip;
        s += v;
        if (v > 0) {
          last = at;
          if (hit < 0 && s > border) hit = at;
        }
      }
    found = hit >= 0 ? hit : last;
  }
  __syncthreads();
  return found;
}

// ------------------------------------------------------------------------------------------------
// One workgroup per sequence.  After k rejections at a node the residual distribution is max(p - a_k q, 0) / F(a_k) with F(a) = sum max(p - a q, 0),
// a_0 = 0, F(a_0) = 1 and a_{k+1} = a_k + F(a_k): one scalar stands for the chain of residual vectors, and only F of the last one needs
// a pass over the vocabulary.  Every product and sum in 64 bits.  A node is a lane of every wave, which has asked for the node's p and q
// before the walk begins, so that the walk itself reads registers.  Bound by one compute unit's passes over a row: 8 x 26 nodes x 128000 chosen, one pass of
// 512 KB, 15 us; 32 x 16 x 50257 bf16 24; 1 x 8 x 32000 8.
// ------------------------------------------------------------------------------------------------
template <int DT, bool DRAFT>
__global__ __launch_bounds__(VW * 64) void tree_verify_kernel(VerifyArgs a) {
  typedef Prob<DT> E;
  typedef typename E::T T;
  typedef Residual<DT, DRAFT> R;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  __shared__ double part[VW];
  const size_t mine = (size_t)b * a.N + min(lane, a.N - 1);
  const int tok = a.tokens[mine], par = a.parents[mine];
  const float un = a.u[mine];
  const bool there = lane > 0 && lane < a.N && par >= 0 && par < lane && tok >= 0 && tok < a.V;
  float pn = 0.f, qn = 0.f;
  if (there) {
    const size_t at = ((size_t)b * a.N + par) * a.V + tok;
    pn = E::value(((const T*)a.p)[at]);
    if constexpr (DRAFT) qn = E::value(((const T*)a.draft)[at]);
  }
  auto of = [](float v, int i) { return (double)__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), i)); };
  int cur = 0;
  uint64_t path = 1, out = 0;
  double am = 0.0, F = 1.0;
  bool have = true;                          // whether F is that of am
  for (uint64_t next = __ballot(there && par == 0); next;) {
    const int i = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)next) - 1);
    next &= next - 1;
    const double px = of(pn, i), ui = of(un, i);
    bool yes;
    if constexpr (DRAFT) {
      const double qx = of(qn, i);
      if (!have) {
        const R r(a, b, cur, am, 0, tok);
        F = sum_parts<true>(r, 0, r.pieces, part);
        have = true;
      }
      yes = ui * F * qx < px - am * qx;
      if (!yes) {
        am += F;
        have = false;
      }
    } else {
      const bool gone = __any((out >> lane & 1) && tok == __builtin_amdgcn_readlane(tok, i));
      const double left = gone ? 0.0 : px;
      yes = ui * F < left;
      if (!yes) {
        F -= left;
        out |= 1ull << i;
      }
    }
    if (yes) {
      path |= 1ull << i;
      cur = i;
      am = 0.0;
      F = 1.0;
      have = true;
      out = 0;
      next = __ballot(there && par == i);
    }
  }
  const int n = __popcll(path);
  if (tid < 64) {
    if (path >> lane & 1) a.path[(size_t)b * a.N + __popcll(path & ((1ull << lane) - 1))] = lane;
    if (lane >= n && lane < a.N) a.path[(size_t)b * a.N + lane] = -1;
    if (lane == 0) a.n_path[b] = n;
  }
  const R r(a, b, cur, am, out, tok);
  const double u0 = of(un, 0);
  int hit;
  if (DRAFT && am != 0.0) hit = draw<DRAFT>(r, u0, part);
  else hit = draw<false>(r, u0, part);
  if (hit < 0) {
    // nothing has any weight: the likeliest of the target's, lowest first
    const T* row = (const T*)a.p + ((size_t)b * a.N + cur) * a.V;
    float top = -1.f;
    int arg = 0x7fffffff;
    for (int v = tid; v < a.V; v += VW * 64) {
      const float pv = E::value(row[v]);
      if (pv > top) {
        top = pv;
        arg = v;
      }
    }
    __shared__ float tops[VW];
    __shared__ int args[VW];
    auto take = [&](float t, int v) {
      if (t > top || (t == top && v < arg)) {
        top = t;
        arg = v;
      }
    };
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
      const float t = __shfl_xor(top, k);
      const int v = __shfl_xor(arg, k);
      take(t, v);
    }
    if (lane == 0) {
      tops[tid >> 6] = top;
      args[tid >> 6] = arg;
    }
    __syncthreads();
    for (int w = 0; w < VW; ++w) take(tops[w], args[w]);
    hit = arg == 0x7fffffff ? 0 : arg;
  }
  if (tid == 0) a.next[b] = hit;
}

// ------------------------------------------------------------------------------------------------
// One workgroup per sequence.  A thread moves 16-byte column pieces of the path's rows, in the path's order: row j goes to len + j < len + path[j], so
// no row is overwritten before it has been read, and no thread reads what another writes.  The new length may take the old one's place:
// it is written when every thread has read that.  Eight rows are asked for before the first is stored (each is read from a later place than any of them is
// written to): 64 sequences of 16 rows x 1280 in 7 us, one of two rows x 4096 in 2.
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(1024) void tree_commit_kernel(u32x4* K, long bstride, const int32_t* path, const int32_t* n_path, const int32_t* seq_lens,
                                                           int32_t* new_lens, int N, int T, int pieces, int head_pieces, int banded) {
  const int b = blockIdx.x;
  __shared__ int from[TREE_MAX_NODES];
  const int len = seq_len_of(seq_lens, b, T);
  const int n = min(max(n_path[b], 0), N);
  static_assert(TREE_MAX_NODES <= 64, "a wave brings the whole path");
  if ((int)threadIdx.x < n) from[threadIdx.x] = path[(size_t)b * N + threadIdx.x];
  __syncthreads();
  if (threadIdx.x == 0) new_lens[b] = len + n;
  const int rp = banded ? head_pieces : pieces;
  constexpr int AHEAD = 8;
  auto moves = [&](int j) { return j < n && from[j] > j && from[j] < N; };      // (else in place already, or no slot)
  for (int piece = threadIdx.x; piece < pieces; piece += blockDim.x) {
    u32x4* base = K + (size_t)b * bstride + (banded ? piece / head_pieces * (32 * head_pieces) + piece % head_pieces : piece);
    auto row = [&](int t) { return base + (size_t)(t >> 5) * 32 * pieces + (size_t)(t & 31) * rp; };
    for (int j = 0; j < n; j += AHEAD) {
      u32x4 x[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) x[i] = *row(len + (moves(j + i) ? from[j + i] : 0));
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (moves(j + i)) *row(len + j + i) = x[i];
    }
  }
}

}  // namespace

void launch_tree_verify(int dtype, const VerifyArgs& a, hipStream_t st) {
  const dim3 grid(a.B), block(VW * 64);
  if (dtype == DT_BF16) {
    if (a.draft) hipLaunchKernelGGL((tree_verify_kernel<DT_BF16, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((tree_verify_kernel<DT_BF16, false>), grid, block, 0, st, a);
  } else {
    if (a.draft) hipLaunchKernelGGL((tree_verify_kernel<DT_F32, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((tree_verify_kernel<DT_F32, false>), grid, block, 0, st, a);
  }
}

void launch_tree_commit(int dtype, void* K, long k_bstride, const int32_t* path, const int32_t* n_path, const int32_t* seq_lens, int32_t* new_lens,
                        int B, int N, int T, int d, int d_k, int banded, hipStream_t st) {
  const int vec = vec_elems(dtype), pieces = d / vec;
  const int threads = pieces >= 1024 ? 1024 : (pieces + 63) / 64 * 64;
  hipLaunchKernelGGL(tree_commit_kernel, dim3(B), dim3(threads), 0, st, (u32x4*)K, k_bstride / vec, path, n_path, seq_lens, new_lens, N, T, pieces,
                     d_k / vec, banded);
}

}  // namespace slim
