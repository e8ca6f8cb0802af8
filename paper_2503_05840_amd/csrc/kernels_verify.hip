// What follows the attention of a tree of drafted tokens: the walk down the tree that accepts or rejects them, the draw of the next token,
// and the move of the accepted path's keys to their places in the cache.
#include "slim_kernels.h"

#include "device_common.h"

namespace slim {
namespace {

constexpr int VW = 16;                       // waves of a verifying workgroup

template <int DT> struct Prob;
template <> struct Prob<DT_F32> {
  static constexpr int VEC = 4;
  typedef float T;
  static __device__ __forceinline__ float value(float x) { return x; }
};
template <> struct Prob<DT_BF16> {
  static constexpr int VEC = 8;
  typedef uint16_t T;
  static __device__ __forceinline__ float value(uint16_t x) { return __uint_as_float((unsigned)x << 16); }
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s);
  return v;
}

// Sum over the workgroup, the same bits in every thread.
__device__ double group_sum(double v, double* red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_sum(v);
  if (lane == 0) red[wave] = v;
  __syncthreads();
  double s = 0;
#pragma unroll
  for (int w = 0; w < VW; ++w) s += red[w];
  __syncthreads();
  return s;
}

// ------------------------------------------------------------------------------------------------
// One workgroup per sequence.  After k rejections at a node the residual distribution is max(p - a_k q, 0) / F(a_k) with F(a) = sum max(p - a q, 0),
// a_0 = 0, F(a_0) = 1 and a_{k+1} = a_k + F(a_k): one scalar stands for the chain of residual vectors, and only F of the last one needs
// a pass over the vocabulary.  Every product and sum in 64 bits.
// ------------------------------------------------------------------------------------------------
template <int DT, bool DRAFT>
__global__ __launch_bounds__(VW * 64) void tree_verify_kernel(VerifyArgs a) {
  typedef Prob<DT> E;
  typedef typename E::T T;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ int tok[TREE_MAX_NODES], par[TREE_MAX_NODES], out[TREE_MAX_NODES];
  __shared__ float un[TREE_MAX_NODES];
  __shared__ double red[VW], before[VW];
  __shared__ int found[VW];
  if (tid < a.N) {
    tok[tid] = a.tokens[(size_t)b * a.N + tid];
    par[tid] = a.parents[(size_t)b * a.N + tid];
    un[tid] = a.u[(size_t)b * a.N + tid];
  }
  __syncthreads();
  const T* P = (const T*)a.p + (size_t)b * a.N * a.V;
  const T* Q = DRAFT ? (const T*)a.draft + (size_t)b * a.N * a.V : nullptr;
  int cur = 0, n = 1, nout = 0;
  double am = 0.0, F = 1.0;
  bool have = true;                          // whether F is that of am
  if (tid == 0) a.path[(size_t)b * a.N] = 0;
  for (int i = 1; i < a.N; ++i) {
    const int x = tok[i];
    if (par[i] != cur || x < 0 || x >= a.V) continue;
    const double px = E::value(P[(size_t)cur * a.V + x]);
    bool yes;
    if constexpr (DRAFT) {
      const double qx = E::value(Q[(size_t)cur * a.V + x]);
      if (!have) {
        double s = 0;
        for (int v = tid; v < a.V; v += VW * 64)
          s += fmax((double)E::value(P[(size_t)cur * a.V + v]) - am * (double)E::value(Q[(size_t)cur * a.V + v]), 0.0);
        F = group_sum(s, red);
        have = true;
      }
      yes = (double)un[i] * F * qx < px - am * qx;
      if (!yes) {
        am += F;
        have = false;
      }
    } else {
      double left = px;
      for (int k = 0; k < nout; ++k) left = out[k] == x ? 0.0 : left;
      yes = (double)un[i] * F < left;
      if (!yes) {
        F -= left;
        __syncthreads();
        if (tid == 0) out[nout] = x;
        ++nout;
        __syncthreads();
      }
    }
    if (yes) {
      if (tid == 0) a.path[(size_t)b * a.N + n] = i;
      ++n;
      cur = i;
      am = 0.0;
      F = 1.0;
      have = true;
      nout = 0;
    }
  }
  for (int i = n + tid; i < a.N; i += VW * 64) a.path[(size_t)b * a.N + i] = -1;
  if (tid == 0) a.n_path[b] = n;

  // the next token: the waves have neighbouring stretches of the vocabulary, sum them, and the wave whose stretch holds the border looks for it
  const T* Pc = P + (size_t)cur * a.V;
  const T* Qc = DRAFT ? Q + (size_t)cur * a.V : nullptr;
  auto residual = [&](int v) -> double {
    const double pv = E::value(Pc[v]);
    if constexpr (DRAFT) return am == 0.0 ? pv : fmax(pv - am * (double)E::value(Qc[v]), 0.0);
    for (int k = 0; k < nout; ++k)
      if (out[k] == v) return 0.0;
    return pv;
  };
  const int per = (a.V + VW - 1) / VW, v0 = wave * per, v1 = min(a.V, v0 + per);
  double s = 0;
  for (int v = v0 + lane; v < v1; v += 64) s += residual(v);
  s = wave_sum(s);
  if (lane == 0) red[wave] = s;
  __syncthreads();
  double total = 0, mine = 0;
  for (int w = 0; w < VW; ++w) {
    if (w == wave) mine = total;
    total += red[w];
  }
  const double border = (double)un[0] * total;
  // first token past the border in the own stretch; the last one with any weight stands in where rounding leaves none
  int hit = 0x7fffffff, last = -1;
  if (total > 0 && mine + s > border && mine <= border) {
    double run = mine;
    for (int v = v0; v < v1 && hit == 0x7fffffff; v += 64) {
      const int at = v + lane;
      double r = at < v1 ? residual(at) : 0.0;
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) {
        const double o = __shfl_up(r, k);
        if (lane >= k) r += o;
      }
      const unsigned long long over = __ballot(at < v1 && run + r > border);
      if (over) hit = v + __ffsll(over) - 1;
      run += __shfl(r, 63);
    }
  }
  __shared__ int hits[VW];
  if (lane == 0) hits[wave] = hit;
  __syncthreads();
  hit = 0x7fffffff;
  for (int w = 0; w < VW; ++w) hit = min(hit, hits[w]);
  if (hit == 0x7fffffff) {
    // nothing past the border: the last token with any weight, or, where nothing has any, the likeliest of the target's
    float top = -1.f;
    int arg = 0x7fffffff;
    for (int v = tid; v < a.V; v += VW * 64) {
      if (residual(v) > 0) last = v;
      const float pv = E::value(Pc[v]);
      if (pv > top) {
        top = pv;
        arg = v;
      }
    }
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
      last = max(last, __shfl_xor(last, k));
      const float t2 = __shfl_xor(top, k);
      const int a2 = __shfl_xor(arg, k);
      if (t2 > top || (t2 == top && a2 < arg)) {
        top = t2;
        arg = a2;
      }
    }
    __shared__ float tops[VW];
    __shared__ int args[VW], lasts[VW];
    if (lane == 0) {
      tops[wave] = top;
      args[wave] = arg;
      lasts[wave] = last;
    }
    __syncthreads();
    for (int w = 0; w < VW; ++w) {
      last = max(last, lasts[w]);
      if (tops[w] > top || (tops[w] == top && args[w] < arg)) {
        top = tops[w];
        arg = args[w];
      }
    }
    hit = total > 0 && last >= 0 ? last : arg == 0x7fffffff ? 0 : arg;
  }
  if (tid == 0) a.next[b] = hit;
}

// ------------------------------------------------------------------------------------------------
// One workgroup per sequence.  A thread moves 16-byte column pieces of the path's rows, in the path's order: row j goes to len + j < len + path[j], so
// no row is overwritten before it has been read, and no thread reads what another writes.  The new length may take the old one's place:
// it is written when every thread has read that.
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
  for (int piece = threadIdx.x; piece < pieces; piece += blockDim.x) {
    u32x4* base = K + (size_t)b * bstride + (banded ? piece / head_pieces * (32 * head_pieces) + piece % head_pieces : piece);
    auto row = [&](int t) { return base + (size_t)(t >> 5) * 32 * pieces + (size_t)(t & 31) * rp; };
    for (int j = 0; j < n; ++j)
      if (from[j] > j && from[j] < N) *row(len + j) = *row(len + from[j]);      // (else in place already, or no slot)
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
