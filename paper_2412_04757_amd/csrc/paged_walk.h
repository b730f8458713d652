// How a launch over the tokens of many sequences is shared out: the sequences' pieces of work lie one after the other, workgroup w takes
// pieces [w share, (w + 1) share), whatever the lengths. Every workgroup finds its place from the lengths on the device.
#pragma once
#include "device_common.h"
#include "paged_internal.h"

namespace ltri {

// Place in the row of all pieces: `before` pieces lie in front of sequence `seq`, of `total`.
struct PagedPlace { long long before, total; int seq; };

constexpr int WALK_T = 256;      // threads of a workgroup that walks

// Sum over a workgroup's threads of those in front, and of all.
__device__ __forceinline__ void paged_scan(unsigned long long mine, unsigned long long& before, unsigned long long& total) {
  __shared__ unsigned long long s_wave[WALK_T / 64];
  const int tid = threadIdx.x;
  const unsigned long long incl = wave_scan_u64(mine);
  if ((tid & 63) == 63) s_wave[tid >> 6] = incl;
  __syncthreads();
  before = incl - mine;
  total = 0;
  for (int i = 0; i < WALK_T / 64; ++i) {
    if (i < tid >> 6) before += s_wave[i];
    total += s_wave[i];
  }
}

// pieces(s) of sequence s; x_of(total): the piece to find. All threads call; seq = -1 where there is no such piece.
template <class Pieces, class Find>
__device__ __forceinline__ PagedPlace paged_find(int n_seqs, Pieces pieces, Find x_of) {
  __shared__ long long s_before;
  __shared__ int s_seq;
  const int tid = threadIdx.x, per = (n_seqs + WALK_T - 1) / WALK_T;
  unsigned long long mine = 0, before, total;
  for (int s = tid * per; s < min(n_seqs, (tid + 1) * per); ++s) mine += (unsigned long long)pieces(s);
  if (tid == 0) s_seq = -1;
  paged_scan(mine, before, total);
  const long long x = x_of((long long)total);
  if (x >= (long long)before && x < (long long)(before + mine)) {
    int s = tid * per;
    long long at = (long long)before;
    for (long long p = pieces(s); x >= at + p; p = pieces(++s)) at += p;
    s_seq = s;
    s_before = at;
  }
  __syncthreads();
  PagedPlace r{0, (long long)total, s_seq};
  if (r.seq >= 0) r.before = s_before;
  __syncthreads();
  return r;
}

// The place of sequence seq. All threads call.
template <class Pieces>
__device__ __forceinline__ PagedPlace paged_place(int n_seqs, Pieces pieces, int seq) {
  __shared__ unsigned long long s_before;
  if (threadIdx.x == 0) s_before = 0;
  __syncthreads();
  unsigned long long mine = 0, ahead = 0, before, total;
  for (int s = threadIdx.x; s < n_seqs; s += WALK_T) {
    const unsigned long long p = (unsigned long long)pieces(s);
    mine += p;
    if (s < seq) ahead += p;
  }
  if (ahead) atomicAdd(&s_before, ahead);
  paged_scan(mine, before, total);                 // (its barrier is behind the additions)
  return PagedPlace{(long long)s_before, (long long)total, seq};
}

}  // namespace ltri
