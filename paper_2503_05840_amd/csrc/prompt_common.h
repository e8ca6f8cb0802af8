// What the kernels of prompt attention share (kernels_prompt.hip, kernels_prompt_f32.hip): which rows a workgroup has, rows from memory into LDS, the merge's inputs.
#pragma once
#include "device_common.h"
#include "slim_kernels.h"

namespace slim {

// 16 bytes a lane from memory to LDS: lane l's go to lds + 16 l.  The caller waits (vmcnt) before it, or another wave behind a barrier, reads them.
// (As asm: the compiler would wait for all of them before the first LDS read that follows, of another buffer too.)
__device__ __forceinline__ void load_to_lds(const void* p, unsigned lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "s"(__builtin_amdgcn_readfirstlane((int)lds)) : "memory");
}
// A value that is the same for the whole wave, in scalar registers
__device__ __forceinline__ uint64_t scalar(uint64_t v) {
  uint64_t u = (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)v) | (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32;
  asm volatile("" : "+s"(u));
  return u;
}
// The same from such a pointer and a lane's offset in bytes
__device__ __forceinline__ void load_to_lds(uint64_t base, unsigned offset, unsigned lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(base), "s"(__builtin_amdgcn_readfirstlane((int)lds)) : "memory");
}
__device__ __forceinline__ unsigned lds_address(const void* p) {
  return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// The tiles that this wave asked for are there but for the last LEFT loads, then everybody's; and everybody is done with the buffer that is filled next.
template <int LEFT>
__device__ __forceinline__ void tiles_barrier() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LEFT) : "memory"); }

// This wave's own loads are there.  (The builtin, which the compiler counts: it would wait for them at their first use, inside a loop, and for the tiles on their way too.)
__device__ __forceinline__ void own_loads_done() { __builtin_amdgcn_s_waitcnt(0x0f70); }

struct PromptTile {
  long q0, k0;            // first rows of the sequence
  int n_q, n_k, i0;       // its rows, and the tile's first query
  int h, hk, split;       // head, its keys' head, part of the keys
};

__device__ __forceinline__ int clamped(int v, int hi) { return v < 0 ? 0 : (v > hi ? hi : v); }

// Workgroup -> head, tile of `rows` queries, split of the keys.  Sequence b's tiles have places from cu_q[b] / rows + b on: never more tiles than places up to the
// next one's, so that no workgroup needs a sum over the batch; places behind a sequence's last tile are empty.
// Workgroups are dealt to the 8 XCDs round robin, each with an L2 of its own: an XCD has whole key heads (8 places of `full` of them at a time) and its share of the
// `rem` heads that are left, whose places go to the XCDs in turn.  Of all these the last places come first: the tiles of a causal sequence that see the
// most keys, so that what is left at the end is short (6000 queries x 32 heads x 128, heads one after the other 381 us, this way 352).
struct PromptPlaces {
  int places, full, rem, block;                   // block: key heads' places of an XCD in eight places
  __host__ __device__ PromptPlaces(const PromptArgs& a, int rows) {
    places = a.rows_q / rows + a.B;
    full = a.H_kv / 8;
    rem = a.H_kv % 8;
    block = 8 * full + rem;
  }
};
__device__ __forceinline__ bool prompt_tile(const PromptArgs& a, int rows, PromptTile& t) {
  const PromptPlaces pp(a, rows);
  // (All of it is the same for the whole wave, and is told so: pointers made from it stay in scalar registers.)
  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  const int xcd = (int)blockIdx.x & 7, slot = (int)blockIdx.x >> 3;
  const int G = uniform(a.H / a.H_kv), u = uniform(slot / G), w = uniform(u / a.nsplit);
  t.split = u - w * a.nsplit;
  const int blk = uniform(w / pp.block), x = w - blk * pp.block;
  int place;
  if (x < 8 * pp.full) {
    const int p = uniform(x / pp.full);
    place = blk * 8 + p;
    t.hk = xcd * pp.full + x - p * pp.full;
  } else {
    const int v = (x - 8 * pp.full) * 8 + xcd, p = uniform(v / pp.rem);
    place = blk * 8 + p;
    t.hk = 8 * pp.full + v - p * pp.rem;
  }
  if (place >= pp.places) return false;
  place = pp.places - 1 - place;
  t.h = t.hk * G + slot - u * G;
  int lo = 0, hi = a.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (clamped(a.cu_q[mid], a.rows_q) / rows + mid <= place) lo = mid; else hi = mid;
  }
  const int q0 = uniform(clamped(a.cu_q[lo], a.rows_q)), q1 = uniform(clamped(a.cu_q[lo + 1], a.rows_q));
  const int k0 = uniform(clamped(a.cu_k[lo], a.rows_k)), k1 = uniform(clamped(a.cu_k[lo + 1], a.rows_k));
  t.q0 = q0; t.n_q = q1 - q0;
  t.k0 = k0; t.n_k = max(k1 - k0, 0);
  const int j = place - uniform(q0 / rows + lo);
  t.i0 = j * rows;
  return j >= 0 && t.i0 < t.n_q;
}
inline unsigned prompt_grid(const PromptArgs& a, int rows) {
  const PromptPlaces pp(a, rows);
  return 8u * (unsigned)((pp.places + 7) / 8) * (unsigned)pp.block * (unsigned)(a.H / a.H_kv * a.nsplit);
}

// max / sum over the lanes l and l ^ 32
__device__ __forceinline__ float max_of_halves(float v) {
  const unsigned u = __float_as_uint(v);
  const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float sum_of_halves(float v) {
  const unsigned u = __float_as_uint(v);
  const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

void launch_prompt_f32(const PromptArgs& a, hipStream_t st);
int prompt_f32_rows(int d_k);

}  // namespace slim
