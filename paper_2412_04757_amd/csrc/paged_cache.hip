// Writing of new tokens into a key-value cache in pages, and its eviction by accumulated attention weight.
#include "device_common.h"
#include "paged_internal.h"

namespace ltri {

// New rows to their places: a thread moves 16 bytes of a key row and of a value row. Bound by memory: every byte is read
// and written once.
__global__ __launch_bounds__(256) void paged_append_kernel(PagedCall a) {
  const PagedDims& D = a.D;
  const int s = blockIdx.z, h = blockIdx.y, per = D.d * D.elt / 16;      // pieces of a row: 8, 16 or 32
  const int len = paged_len(a, s);
  for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < (long long)a.n * per; t += (long long)gridDim.x * 256) {
    const int i = (int)(t / per), c = (int)(t % per), at = len - a.n + i;
    if (at < 0) continue;
    const int page = paged_page(a, s, at);
    if (page < 0) continue;
    const size_t src = (((size_t)s * D.Hkv + h) * a.n + i) * per + c;
    const size_t dst = (size_t)paged_row(D, page, h, at) * D.elt + 16 * c;
    *(uint4*)(a.k + dst) = ((const uint4*)a.k_new)[src];
    *(uint4*)(a.v + dst) = ((const uint4*)a.v_new)[src];
    if (D.weights && c == 0) {
      const size_t mark = paged_mark(D, page, h, at);
      a.weight[mark] = a.w_new ? a.w_new[((size_t)s * D.Hkv + h) * a.n + i] : 0.f;
      a.pos[mark] = a.seen[s] - a.n + i;
    }
  }
}

// ------------------------------------------------------------------ eviction

// A token's order: larger stays sooner. Protected tokens above all weights, NaN below.
__device__ __forceinline__ uint32_t evict_key(const PagedCall& a, int s, size_t mark) {
  const int pos = a.pos[mark];
  if (pos < a.n_sink || (long long)pos >= (long long)a.seen[s] - a.n_recent) return 0xFFFFFFFFu;
  const float w = a.weight[mark];
  if (!(w == w)) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

constexpr int EV_T = 1024, EV_W = EV_T / 64;

// Exclusive sum over the workgroup's threads, and the total.
__device__ __forceinline__ int block_scan(int x, int* total) {
  __shared__ int sums[EV_W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int incl = wave_scan_i32(x);
  if (lane == 63) sums[wave] = incl;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < EV_W; ++i) {
    if (i < wave) before += sums[i];
    all += sums[i];
  }
  __syncthreads();
  *total = all;
  return before + incl - x;
}

// One workgroup per (sequence, KV head). The keep-th largest key is found digit by digit (8 bits at a time, a histogram
// of the keys that share the digits found so far); of the tokens with that key the first ones stay. Then two lists: places
// below keep that became free, and places beyond that stay.
__global__ __launch_bounds__(EV_T) void paged_select_kernel(PagedCall a) {
  const PagedDims& D = a.D;
  const int s = blockIdx.y, h = blockIdx.x, slot = s * D.Hkv + h, tid = threadIdx.x;
  __shared__ int hist[256];
  __shared__ int s_digit, s_rank, s_bad;
  __shared__ unsigned long long s_before;
  if (tid == 0) { s_bad = 0; s_before = 0; a.move_head[2 * slot + 1] = 0; }
  __syncthreads();
  unsigned long long tiles = 0;
  for (int i = tid; i < s; i += EV_T) tiles += (unsigned long long)paged_tiles(paged_len(a, i));
  if (tiles) atomicAdd(&s_before, tiles);
  const int n = paged_len(a, s), keep = a.keep;
  if (n <= keep) return;
  for (int i = tid << D.page_shift; i < n && i >= 0; i += EV_T << D.page_shift)
    if (paged_page(a, s, i) < 0) s_bad = 1;
  __syncthreads();
  if (s_bad) return;
  const long long before = (long long)s_before;
  if (before + paged_tiles(n) > D.score_tiles) {
    atomicCAS(a.err, 0, LTRI_ECAPACITY);
    return;
  }
  auto key_at = [&](int i) { return evict_key(a, s, paged_mark(D, a.table[(size_t)s * D.table_pages + (i >> D.page_shift)], h, i)); };
  uint32_t prefix = 0;
  int rank = keep;                                   // of the keys that share the prefix, how many stay
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += EV_T) {
      const uint32_t k = key_at(i);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int left = rank, b = 255;
      while (hist[b] < left) left -= hist[b--];
      s_digit = b; s_rank = left;
    }
    __syncthreads();
    prefix |= (uint32_t)s_digit << shift;
    rank = s_rank;
  }
  int32_t* list = a.moves + ((size_t)before * D.Hkv + (size_t)h * paged_tiles(n)) * PAGED_TILE;
  const int half = min(keep, n - keep);              // both lists have as many entries, at most this
  int ties = 0, holes = 0, movers = 0;
  for (int base = 0; base < n; base += EV_T) {
    const int i = base + tid;
    const uint32_t k = i < n ? key_at(i) : 0u;
    int total;
    const int tie = i < n && k == prefix;
    const int before_me = block_scan(tie, &total);
    const bool stays = i < n && (k > prefix || (tie && ties + before_me < rank));
    ties += total;
    const int hole = i < keep && !stays, mover = i >= keep && stays;
    const int a0 = block_scan(hole, &total);
    if (hole) list[holes + a0] = i;
    holes += total;
    const int b0 = block_scan(mover, &total);
    if (mover) list[half + movers + b0] = i;
    movers += total;
  }
  if (tid == 0) {
    a.move_head[2 * slot] = (long long)(list - a.moves);
    a.move_head[2 * slot + 1] = (long long)movers << 32 | half;
  }
}

// The moves: a wavefront takes one row after the other; the first workgroup of a sequence also writes its length.
__global__ __launch_bounds__(256) void paged_move_kernel(PagedCall a) {
  const PagedDims& D = a.D;
  const int h = blockIdx.y, s = blockIdx.z, slot = s * D.Hkv + h, lane = threadIdx.x & 63;
  const long long head = a.move_head[2 * slot + 1];
  const int count = (int)(head >> 32), half = (int)head;
  if (head == 0) return;
  const int32_t* list = a.moves + a.move_head[2 * slot];
  const int per = D.d * D.elt / 16;
  for (int i = blockIdx.x * 4 + (threadIdx.x >> 6); i < count; i += gridDim.x * 4) {
    const int to = list[i], from = list[half + i];
    const int pt = a.table[(size_t)s * D.table_pages + (to >> D.page_shift)], pf = a.table[(size_t)s * D.table_pages + (from >> D.page_shift)];
    const size_t dst = (size_t)paged_row(D, pt, h, to) * D.elt, src = (size_t)paged_row(D, pf, h, from) * D.elt;
    if (lane < per) *(uint4*)(a.k + dst + 16 * lane) = *(const uint4*)(a.k + src + 16 * lane);
    if (lane < per) *(uint4*)(a.v + dst + 16 * lane) = *(const uint4*)(a.v + src + 16 * lane);
    if (lane == 0) a.weight[paged_mark(D, pt, h, to)] = a.weight[paged_mark(D, pf, h, from)];
    if (lane == 1) a.pos[paged_mark(D, pt, h, to)] = a.pos[paged_mark(D, pf, h, from)];
  }
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) a.lens[s] = a.keep;
}

hipError_t launch_paged_append(const PagedCall& a, hipStream_t s) {
  const long long pieces = (long long)a.n * (a.D.d * a.D.elt / 16);
  const int wgs = (int)(pieces > 256 * 1024 ? 1024 : (pieces + 255) / 256);
  paged_append_kernel<<<dim3(wgs, a.D.Hkv, a.seq_count), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_evict(const PagedCall& a, hipStream_t s) {
  paged_select_kernel<<<dim3(a.D.Hkv, a.seq_count), EV_T, 0, s>>>(a);
  paged_move_kernel<<<dim3(32, a.D.Hkv, a.seq_count), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ltri
