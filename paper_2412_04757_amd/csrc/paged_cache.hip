// Writing of new tokens into a key-value cache in pages, and its eviction by accumulated attention weight.
#include <algorithm>

#include "device_common.h"
#include "paged_internal.h"

namespace ltri {

// New rows to their places: a thread moves 16 bytes of a key row and of a value row. Bound by memory: every byte is read
// and written once. 4 x 2048 rows of 8 KV heads x 128 in bf16: 67 MB in 12 us.
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
//
// Which tokens stay is the selection of the keep-th largest of n 32-bit keys per (sequence, KV head), ties by place: a radix selection,
// 11 + 11 + 10 bits, each step a histogram of the keys that share the digits found so far. Then the places below keep that
// became free and the places beyond that stay, both in order, are the two ends of the moves; they never overlap, so
// the moves need no order among themselves. What it must read is 8 bytes a token, and the rows that move; what bounds it are the
// steps one after the other: of 5125 tokens, 128 times, 12 us in one launch, 1.4 the loads, 1.2 and 0.8 a step, 1.5 the ranks, 1.6
// the move; 10240 tokens, 8 times, 19 us and 6.7 for the moves of 8 MB.

// A token's order: larger stays sooner. Protected tokens above all weights, NaN below.
__device__ __forceinline__ uint32_t evict_key(const PagedCall& a, int pos, float w, int seen) {
  if (pos < a.n_sink || (long long)pos >= (long long)seen - a.n_recent) return 0xFFFFFFFFu;
  if (!(w == w)) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

constexpr int EV_T = 1024, EV_W = EV_T / 64;
constexpr int EV_BINS = 2048;

__device__ __forceinline__ int mask_rank(unsigned long long m) {           // set bits below the lane
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// Digits of a key from the top: shift and value of step K.
constexpr int digit_shift(int k) { return k == 0 ? 21 : k == 1 ? 10 : 0; }
template <int K> __device__ __forceinline__ uint32_t digit_of(uint32_t key) { return K == 2 ? key & 1023u : (key >> digit_shift(K)) & 2047u; }
template <int K> __device__ __forceinline__ bool same_above(uint32_t key, uint32_t prefix) {
  if constexpr (K == 0) return true;
  else return ((key ^ prefix) >> digit_shift(K - 1)) == 0;
}
template <int K> using Step = std::integral_constant<int, K>;

// Counts a key in a step's histogram, whole wavefronts (`in`: the lane has one). Protected tokens, which share a bin, as one addition.
template <int K>
__device__ __forceinline__ void count_key(int* hist, uint32_t key, bool in, uint32_t prefix) {
  in = in && same_above<K>(key, prefix);
  const bool top = in && key == 0xFFFFFFFFu;
  const unsigned long long m = __ballot(top);
  if (m && (threadIdx.x & 63) == 0) atomicAdd(&hist[digit_of<K>(0xFFFFFFFFu)], __popcll(m));
  if (in && !top) atomicAdd(&hist[digit_of<K>(key)], 1);
}

// A step's bin, from the histogram in LDS: the one in which the rank-th largest key lies. The first wavefront looks, a lane at 32
// bins from the top, then at the bins of the lane that has it; the whole workgroup calls, behind a barrier. (Two bins a thread and a scan
// over the workgroup: 1.6 us, this: 0.8.)
struct Picked { int bin, left, all; };
template <int K>
__device__ __forceinline__ void pick_bin(const int* hist, Picked* s_pick, uint32_t& prefix, int& rank, bool& all) {
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {
    const int top = EV_BINS - 32 * (lane + 1);     // the lane's bins: top .. top + 31
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {                  // (each lane begins elsewhere: other banks)
      const int4 c = *(const int4*)&hist[top + 4 * ((lane + i) & 7)];
      sum += (c.x + c.y) + (c.z + c.w);
    }
    const int incl = wave_scan_i32(sum);
    const unsigned long long has = __ballot(incl >= rank);
    const int l = (int)__builtin_ctzll(has), left = rank - (__shfl(incl, l, 64) - __shfl(sum, l, 64));
    const int bin = EV_BINS - 32 * l - 1 - min(lane, 31), c = lane < 32 ? hist[bin] : 0;
    const int seen = wave_scan_i32(c);
    const unsigned long long in = __ballot(seen >= left);
    if (lane == (int)__builtin_ctzll(in)) *s_pick = Picked{bin, left - (seen - c), seen == left};
  }
  __syncthreads();
  const Picked p = *s_pick;
  prefix |= (uint32_t)p.bin << digit_shift(K);
  rank = p.left;
  all = p.all != 0;                               // the whole bin stays: no need to look into it
}

// The keys of PER tokens at first, first + stride, ..., below n (others: 0): places, then marks, all on their way together (one
// after the other ten tokens took 8.7 us, so 2.9). bad: a page is not in the pool.
template <int PER>
__device__ __forceinline__ void load_keys(const PagedCall& a, int s, int h, int n, int first, int stride, uint32_t (&key)[PER], bool& bad) {
  const PagedDims& D = a.D;
  const int32_t* table = a.table + (size_t)s * D.table_pages;
  const int seen = a.seen[s];
  int page[PER], pos[PER];
  float w[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) page[e] = table[min(first + e * stride, n - 1) >> D.page_shift];
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const bool good = (unsigned)page[e] < (unsigned)D.n_pages;
    bad |= !good;
    const size_t mark = paged_mark(D, good ? page[e] : 0, h, min(first + e * stride, n - 1));
    pos[e] = a.pos[mark];
    w[e] = a.weight[mark];
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) key[e] = first + e * stride < n ? evict_key(a, pos[e], w[e], seen) : 0u;
}

// Tiles of scratch in front of a sequence (each (sequence, KV head) has PAGED_TILE entries a tile); every wavefront adds for itself.
__device__ __forceinline__ long long list_tiles_before(const PagedCall& a, int s) {
  unsigned long long tiles = 0;
  for (int i = threadIdx.x & 63; i < s; i += 64) tiles += (unsigned long long)paged_tiles(paged_len(a, i));
  return __shfl((long long)wave_scan_u64(tiles), 63, 64);
}
__device__ __forceinline__ size_t list_base(const PagedCall& a, long long before, int n, int h) {
  return ((size_t)before * a.D.Hkv + (size_t)h * paged_tiles(n)) * PAGED_TILE;
}

// Moves one row after the other, several in flight: to(i), from(i) are places of sequence s, i = first, first + step, ...
template <class To, class From>
__device__ __forceinline__ void move_rows(const PagedCall& a, int s, int h, int first, int step, int count, To to, From from) {
  const PagedDims& D = a.D;
  const int lane = threadIdx.x & 63, per = D.d * D.elt / 16, side = lane / per, c = lane % per;     // side 0: keys, 1: values
  const int at_once = 32 / per;                                                                    // rows of a wavefront: 4, 2, 1
  const int32_t* table = a.table + (size_t)s * D.table_pages;
  const int sub = side / 2;
  char* pool = side & 1 ? a.v : a.k;
  constexpr int DEEP = 4;
  for (int i = first * at_once; i < count; i += step * at_once * DEEP) {
    u32x4_t row[DEEP];
    size_t dst[DEEP], mt[DEEP];
    float w[DEEP];
    int pos[DEEP];
    bool on[DEEP];
#pragma unroll
    for (int u = 0; u < DEEP; ++u) {
      const int m = i + u * step * at_once + sub;
      on[u] = m < count;
      const int t = to(on[u] ? m : 0), f = from(on[u] ? m : 0);
      const int pt = table[t >> D.page_shift], pf = table[f >> D.page_shift];
      dst[u] = (size_t)paged_row(D, pt, h, t) * D.elt + 16 * c;
      mt[u] = paged_mark(D, pt, h, t);
      const size_t mf = paged_mark(D, pf, h, f);
      row[u] = *(const u32x4_t*)(pool + (size_t)paged_row(D, pf, h, f) * D.elt + 16 * c);
      w[u] = a.weight[mf];
      pos[u] = a.pos[mf];
    }
#pragma unroll
    for (int u = 0; u < DEEP; ++u) {
      if (!on[u]) continue;
      *(u32x4_t*)(pool + dst[u]) = row[u];
      if (c == 0 && !(side & 1)) a.weight[mt[u]] = w[u];
      if (c == 0 && (side & 1)) a.pos[mt[u]] = pos[u];
    }
  }
}

// One workgroup per (sequence, KV head), its keys in registers (up to PER a thread): a wavefront has 64 per tokens in a row, so the
// ranks of free places and of comers are counts of set bits. FEW: the workgroup also makes the moves (the host knows of no more
// than EV_FEW), and the last one of a sequence writes its length; else two lists in scratch for paged_move_kernel.
constexpr int EV_FEW = 256;
template <int PER, bool FEW>
__global__ __launch_bounds__(EV_T) void paged_select_kernel(PagedCall a) {
  const PagedDims& D = a.D;
  const int s = blockIdx.y, h = blockIdx.x, slot = s * D.Hkv + h, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __shared__ __align__(16) int hist[3][EV_BINS];  // one for each step, cleared together
  __shared__ Picked s_pick[3];
  __shared__ int s_count[3][EV_W], s_bad;
  __shared__ int s_to[FEW ? EV_FEW : 1], s_from[FEW ? EV_FEW : 1];
  const int n = paged_len(a, s), keep = a.keep;
  if (!FEW && tid == 0) a.move_head[2 * slot + 1] = 0;
  if (n <= keep) return;
  if (tid == 0) s_bad = 0;
  for (int b = tid; b < 3 * EV_BINS; b += EV_T) ((int*)hist)[b] = 0;
  const int per = (n + EV_T - 1) / EV_T, base = wave * 64 * per + lane;
  uint32_t key[PER];
  bool bad = false;
  load_keys(a, s, h, n, base, 64, key, bad);
  __syncthreads();
  if (bad) s_bad = 1;
  uint32_t prefix = 0u;
  int rank = keep;
  bool all = false;
  auto step = [&](auto k) __attribute__((always_inline)) {
    constexpr int K = decltype(k)::value;
    if (all) return;
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (e < per) count_key<K>(hist[K], key[e], base + 64 * e < n, prefix);
    __syncthreads();
    pick_bin<K>(hist[K], &s_pick[K], prefix, rank, all);
  };
  step(Step<0>{});
  step(Step<1>{});
  step(Step<2>{});
  if (s_bad) {                                    // (left as it is)
    if (tid == 0) atomicCAS(a.err, 0, LTRI_EINVAL);
    if constexpr (!FEW) return;
  }
  // ties in front of the wavefront's tokens
  int ties = 0;
  if (!all) {
    int mine = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (e < per) mine += __popcll(__ballot(base + 64 * e < n && key[e] == prefix));
    if (lane == 0) s_count[0][wave] = mine;
    __syncthreads();
    for (int i = 0; i < EV_W; ++i) ties += i < wave ? s_count[0][i] : 0;
  }
  // bits of the lane's tokens that stay
  static_assert(PER <= 32, "");
  uint32_t stays = 0u;
  int holes = 0, comers = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    if (e >= per) continue;
    const int i = base + 64 * e;
    const bool tie = i < n && key[e] == prefix;
    bool stay = i < n && (all ? key[e] >= prefix : key[e] > prefix);
    if (!all) {
      const unsigned long long m = __ballot(tie);
      stay |= tie && ties + mask_rank(m) < rank;
      ties += __popcll(m);
    }
    stays |= (uint32_t)stay << e;
    holes += __popcll(__ballot(i < keep && !stay));
    comers += __popcll(__ballot(i >= keep && stay));
  }
  if (lane == 0) { s_count[1][wave] = holes; s_count[2][wave] = comers; }
  __syncthreads();
  holes = comers = 0;
  int count = 0;
  for (int i = 0; i < EV_W; ++i) {
    if (i < wave) { holes += s_count[1][i]; comers += s_count[2][i]; }
    count += s_count[2][i];
  }
  int32_t *to = s_to, *from = s_from;
  int half = 0;
  if constexpr (!FEW) {
    half = min(keep, n - keep);                   // both lists have `count` entries, at most this
    const long long before = list_tiles_before(a, s);
    if (before + paged_tiles(n) > D.score_tiles) {
      if (tid == 0) atomicCAS(a.err, 0, PAGED_NO_ROOM);
      return;
    }
    to = a.moves + list_base(a, before, n, h);
    from = to + half;
    if (tid == 0) {
      a.move_head[2 * slot] = (long long)(to - a.moves);
      a.move_head[2 * slot + 1] = (long long)count << 32 | half;
    }
  }
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    if (e >= per) continue;
    const int i = base + 64 * e;
    const bool stay = (stays >> e) & 1;
    const unsigned long long mh = __ballot(i < keep && !stay), mc = __ballot(i >= keep && i < n && stay);
    if (i < keep && !stay) to[holes + mask_rank(mh)] = i;
    if (i >= keep && stay) from[comers + mask_rank(mc)] = i;
    holes += __popcll(mh);
    comers += __popcll(mc);
  }
  if constexpr (FEW) {
    __syncthreads();
    if (!s_bad) move_rows(a, s, h, wave, EV_W, count, [&](int i) { return s_to[i]; }, [&](int i) { return s_from[i]; });
    if (tid == 0 && atomicAdd(a.tickets + s, 1) == D.Hkv - 1) {       // every workgroup of the sequence has read its length
      a.tickets[s] = 0;
      if (!s_bad) a.lens[s] = keep;
    }
  }
}

// The moves of two lists; the first workgroup of a sequence also writes its length.
__global__ __launch_bounds__(256) void paged_move_kernel(PagedCall a) {
  const int h = blockIdx.y, s = blockIdx.z, slot = s * a.D.Hkv + h;
  const long long head = a.move_head[2 * slot + 1];
  if (head == 0) return;
  const int32_t* list = a.moves + a.move_head[2 * slot];
  const int half = (int)head;
  move_rows(a, s, h, blockIdx.x * 4 + (threadIdx.x >> 6), gridDim.x * 4, (int)(head >> 32), [&](int i) { return list[i]; },
            [&](int i) { return list[half + i]; });
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) a.lens[s] = a.keep;
}

// ---- long sequences: several workgroups per (sequence, KV head), EV_CHUNK tokens each, the steps as launches ----
//   1  keys to scratch, the first digit's histogram; the workgroup that finishes last picks the bin
//   2  keys of that bin to a list; the last one finishes the selection on the list
//   3  per piece how many keys are above the threshold, and how many equal it (pieces end at `keep`)
//   4  the two lists of moves, each piece behind what the counts say of those in front
// and paged_move_kernel.

struct LongSlot {                                  // of a (sequence, KV head)
  long long base;                                  // of its keys, candidates and moves in scratch
  uint32_t key; int ties, all;                     // keys above `key` stay and the first `ties` equal to it, or (all) those >= key;
                                                   // after launch 1: of the bin
  int live;                                        // 0: nothing to do
};
static_assert(sizeof(LongSlot) == EV_SLOT_BYTES, "");
__device__ __forceinline__ LongSlot* long_slot(const PagedCall& a, int slot) { return (LongSlot*)a.long_slots + slot; }

// Takes a ticket of `parts`; true for the workgroup that finishes last, for all of whose threads what the others stored at device scope
// is then to be read. The counter is left at zero.
__device__ __forceinline__ bool last_of(int32_t* ticket, int parts) {
  __shared__ int s_last;
  wait_for_own_stores();
  __syncthreads();
  if (threadIdx.x == 0) {
    s_last = atomicAdd(ticket, 1) == parts - 1;
    if (s_last) *ticket = 0;
  }
  __syncthreads();
  const bool r = s_last != 0;
  __syncthreads();
  return r;
}

__global__ __launch_bounds__(EV_T) void paged_long_keys_kernel(PagedCall a) {
  const PagedDims& D = a.D;
  const int s = blockIdx.z, h = blockIdx.y, slot = s * D.Hkv + h, tid = threadIdx.x;
  const int n = paged_len(a, s), first = blockIdx.x * EV_CHUNK;
  LongSlot* L = long_slot(a, slot);
  if (n <= a.keep) {
    if (blockIdx.x == 0 && tid == 0) { L->live = 0; a.move_head[2 * slot + 1] = 0; }
    return;
  }
  if (first >= n) return;
  __shared__ __align__(16) int hist[EV_BINS];
  __shared__ Picked s_pick;
  for (int b = tid; b < EV_BINS; b += EV_T) hist[b] = 0;
  const long long before = list_tiles_before(a, s);
  const bool room = before + paged_tiles(n) <= D.score_tiles;
  const size_t base = list_base(a, before, n, h);
  int32_t* state = a.long_state + (size_t)slot * EV_LONG_WORDS;         // [0] ticket, [1] bad pages, [2] candidates, from [4] on the histogram
  bool bad = false;
  uint32_t key[EV_CHUNK / EV_T];
  load_keys(a, s, h, n, first + tid, EV_T, key, bad);
  __syncthreads();
#pragma unroll
  for (int e = 0; e < EV_CHUNK / EV_T; ++e) {
    const int i = first + e * EV_T + tid;
    if (room && i < n) a.keys[base + i] = key[e];
    count_key<0>(hist, key[e], i < n, 0u);
  }
  if (bad) { atomicOr(state + 1, 1); atomicCAS(a.err, 0, LTRI_EINVAL); }
  __syncthreads();
  for (int b = tid; b < EV_BINS; b += EV_T)
    if (hist[b]) atomicAdd(state + 4 + b, hist[b]);
  if (!last_of(state, (n + EV_CHUNK - 1) / EV_CHUNK)) return;
  for (int b = tid; b < EV_BINS; b += EV_T) {
    hist[b] = __hip_atomic_load(state + 4 + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    state[4 + b] = 0;
  }
  __syncthreads();
  uint32_t prefix = 0u;
  int rank = a.keep;
  bool all = false;
  pick_bin<0>(hist, &s_pick, prefix, rank, all);
  if (tid == 0) {
    const bool live = room && !__hip_atomic_load(state + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (!room) atomicCAS(a.err, 0, PAGED_NO_ROOM);
    state[1] = 0;
    *L = LongSlot{(long long)base, prefix, rank, (int)all, (int)live};
    a.move_head[2 * slot + 1] = 0;
  }
}

__global__ __launch_bounds__(EV_T) void paged_long_select_kernel(PagedCall a) {
  const PagedDims& D = a.D;
  const int s = blockIdx.z, h = blockIdx.y, slot = s * D.Hkv + h, tid = threadIdx.x, lane = tid & 63;
  LongSlot* L = long_slot(a, slot);
  if (!L->live || L->all) return;
  const int n = paged_len(a, s), first = blockIdx.x * EV_CHUNK;
  if (first >= n) return;
  uint32_t prefix = L->key;
  int rank = L->ties;
  const uint32_t* keys = (const uint32_t*)a.keys + L->base;
  uint32_t* found = (uint32_t*)a.candidates + L->base;
  int32_t* state = a.long_state + (size_t)slot * EV_LONG_WORDS;
  __shared__ __align__(16) int hist[EV_BINS];
  __shared__ Picked s_pick;
  __shared__ int s_n, s_at;
  if (tid == 0) s_n = 0;
  __syncthreads();
  // candidates of the piece, in any order
  uint32_t key[EV_CHUNK / EV_T];
  int mine = 0;
#pragma unroll
  for (int e = 0; e < EV_CHUNK / EV_T; ++e) {
    const int i = first + e * EV_T + tid;
    key[e] = keys[min(i, n - 1)];
    mine += i < n && same_above<1>(key[e], prefix);
  }
  const int incl = wave_scan_i32(mine);
  int at = 0;
  if (lane == 63 && incl) at = atomicAdd(&s_n, incl);
  at = __shfl(at, 63, 64) + incl - mine;
  __syncthreads();
  if (tid == 0) s_at = s_n ? atomicAdd(state + 2, s_n) : 0;
  __syncthreads();
  at += s_at;
#pragma unroll
  for (int e = 0; e < EV_CHUNK / EV_T; ++e) {
    const int i = first + e * EV_T + tid;
    if (i < n && same_above<1>(key[e], prefix)) __hip_atomic_store(found + at++, key[e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (!last_of(state, (n + EV_CHUNK - 1) / EV_CHUNK)) return;
  const int m = __hip_atomic_load(state + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  bool all = false;
  auto step = [&](auto k_c) __attribute__((always_inline)) {
    constexpr int K = decltype(k_c)::value;
    if (all) return;
    for (int b = tid; b < EV_BINS; b += EV_T) hist[b] = 0;
    __syncthreads();
    for (int i0 = 0; i0 < m; i0 += 8 * EV_T) {
      uint32_t k[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = __hip_atomic_load(found + min(i0 + e * EV_T + tid, m - 1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
      for (int e = 0; e < 8; ++e) count_key<K>(hist, k[e], i0 + e * EV_T + tid < m, prefix);
    }
    __syncthreads();
    pick_bin<K>(hist, &s_pick, prefix, rank, all);
  };
  step(Step<1>{});
  step(Step<2>{});
  if (tid == 0) {
    state[2] = 0;
    L->key = prefix;
    L->ties = rank;
    L->all = all;
  }
}

// Pieces of launches 3 and 4: those of [0, keep), then those of [keep, n).
struct Piece { int first, count; };
__device__ __forceinline__ Piece piece_of(int n, int keep, int c) {
  const int front = (keep + EV_CHUNK - 1) / EV_CHUNK;
  const int first = c < front ? c * EV_CHUNK : keep + (c - front) * EV_CHUNK, end = c < front ? min(keep, first + EV_CHUNK) : n;
  return Piece{first, max(0, min(EV_CHUNK, end - first))};
}

__global__ __launch_bounds__(EV_T) void paged_long_count_kernel(PagedCall a) {
  const int s = blockIdx.z, h = blockIdx.y, slot = s * a.D.Hkv + h, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const LongSlot L = *long_slot(a, slot);
  if (!L.live) return;
  const Piece p = piece_of(paged_len(a, s), a.keep, blockIdx.x);
  if (p.count == 0) return;
  const uint32_t* keys = (const uint32_t*)a.keys + L.base + p.first;
  int above = 0, ties = 0;
#pragma unroll
  for (int e = 0; e < EV_CHUNK / EV_T; ++e) {
    const int i = e * EV_T + tid;
    const uint32_t k = keys[min(i, p.count - 1)];
    above += i < p.count && (L.all ? k >= L.key : k > L.key);
    ties += i < p.count && !L.all && k == L.key;
  }
  __shared__ int s_count[2][EV_W];
  above = wave_scan_i32(above);
  ties = wave_scan_i32(ties);
  if (lane == 63) { s_count[0][wave] = above; s_count[1][wave] = ties; }
  __syncthreads();
  if (tid < 2) {
    int x = 0;
    for (int i = 0; i < EV_W; ++i) x += s_count[tid][i];
    a.long_counts[((size_t)slot * a.D.long_pieces + blockIdx.x) * 2 + tid] = x;
  }
}

__global__ __launch_bounds__(EV_T) void paged_long_lists_kernel(PagedCall a) {
  const int s = blockIdx.z, h = blockIdx.y, slot = s * a.D.Hkv + h, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const LongSlot L = *long_slot(a, slot);
  if (!L.live) return;
  const int n = paged_len(a, s), keep = a.keep, c = blockIdx.x, front = (keep + EV_CHUNK - 1) / EV_CHUNK;
  const Piece p = piece_of(n, keep, c);
  if (p.count == 0) return;
  // ties in front of the piece, then what stays in front of it: piece by piece, 64 at a time
  __shared__ int s_ties, s_rank, s_total, s_count[2][EV_W];
  if (wave == 0) {
    const int pieces = front + (n - keep + EV_CHUNK - 1) / EV_CHUNK;
    const int32_t* counts = a.long_counts + (size_t)slot * a.D.long_pieces * 2;
    int ties = 0, rank = 0, comers = 0;             // free places (front) or comers (behind) in front of the piece; all comers
    for (int b = 0; b < pieces; b += 64) {
      const int i = b + lane;
      const Piece q = piece_of(n, keep, min(i, pieces - 1));
      const int above = i < pieces ? counts[2 * i] : 0, t = i < pieces ? counts[2 * i + 1] : 0;
      const int scan = wave_scan_i32(t), t0 = ties + scan - t;
      const int stay = above + max(0, min(t, L.ties - t0));
      if (i == c) s_ties = t0;
      const int part = c < front ? (i < front && i < c ? q.count - stay : 0) : (i >= front && i < c ? stay : 0);
      const int sum = wave_scan_i32(part), all = wave_scan_i32(i >= front && i < pieces ? stay : 0);
      rank += __shfl(sum, 63, 64);
      comers += __shfl(all, 63, 64);
      ties += __shfl(scan, 63, 64);
    }
    if (lane == 0) { s_rank = rank; s_total = comers; }
  }
  __syncthreads();
  const int half = min(keep, n - keep);
  int32_t* list = a.moves + L.base + (c < front ? 0 : half);
  if (c == 0 && tid == 0) {
    a.move_head[2 * slot] = L.base;
    a.move_head[2 * slot + 1] = (long long)s_total << 32 | half;
  }
  const uint32_t* keys = (const uint32_t*)a.keys + L.base + p.first;
  constexpr int PER = EV_CHUNK / EV_T;
  uint32_t key[PER];
  const int base = wave * 64 * PER + lane;
  int mine = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    key[e] = keys[min(base + 64 * e, p.count - 1)];
    mine += __popcll(__ballot(base + 64 * e < p.count && key[e] == L.key));
  }
  if (lane == 0) s_count[0][wave] = mine;
  __syncthreads();
  int ties = s_ties, rank = s_rank;
  for (int i = 0; i < EV_W; ++i) ties += i < wave ? s_count[0][i] : 0;
  uint32_t picks = 0u;
  int picked = 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const bool in = base + 64 * e < p.count, tie = in && key[e] == L.key;
    bool stay = in && (L.all ? key[e] >= L.key : key[e] > L.key);
    const unsigned long long m = __ballot(tie);
    if (!L.all) stay |= tie && ties + mask_rank(m) < L.ties;
    ties += __popcll(m);
    const bool pick = in && (c < front ? !stay : stay);
    picks |= (uint32_t)pick << e;
    picked += __popcll(__ballot(pick));
  }
  if (lane == 0) s_count[1][wave] = picked;
  __syncthreads();
  for (int i = 0; i < EV_W; ++i) rank += i < wave ? s_count[1][i] : 0;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const bool pick = (picks >> e) & 1;
    const unsigned long long m = __ballot(pick);
    if (pick) list[rank + mask_rank(m)] = p.first + base + 64 * e;
    rank += __popcll(m);
  }
}

hipError_t launch_paged_append(const PagedCall& a, hipStream_t s) {
  const long long pieces = (long long)a.n * (a.D.d * a.D.elt / 16);
  const int wgs = (int)(pieces > 256 * 1024 ? 1024 : (pieces + 255) / 256);
  paged_append_kernel<<<dim3(wgs, a.D.Hkv, a.seq_count), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <bool FEW>
static void launch_select(const PagedCall& a, hipStream_t s) {
  const dim3 grid(a.D.Hkv, a.seq_count);
  if (a.D.cap_tokens <= 4 * EV_T) paged_select_kernel<4, FEW><<<grid, EV_T, 0, s>>>(a);
  else if (a.D.cap_tokens <= 8 * EV_T) paged_select_kernel<8, FEW><<<grid, EV_T, 0, s>>>(a);
  else paged_select_kernel<EV_LONG / EV_T, FEW><<<grid, EV_T, 0, s>>>(a);
}

// Which way goes by what the table could hold, as the host does not know the lengths: 16 sequences of 5125 tokens, one of which goes, take
// 14 us with a table of 5184 tokens (one launch), 18 with 8192 (two), 54 with 32768 (five) and 138 with 131072 (five, of whose workgroups
// most find nothing).
hipError_t launch_paged_evict(const PagedCall& a, hipStream_t s) {
  const PagedDims& D = a.D;
  const long long most = std::min<long long>(a.keep, D.cap_tokens - a.keep);      // moves of a sequence and KV head
  if (D.cap_tokens <= EV_LONG && most <= EV_FEW) {
    launch_select<true>(a, s);
    return hipGetLastError();
  }
  if (D.cap_tokens <= EV_LONG) {
    launch_select<false>(a, s);
  } else {
    const dim3 grid((unsigned)((D.cap_tokens + EV_CHUNK - 1) / EV_CHUNK), D.Hkv, a.seq_count);
    const dim3 pieces((unsigned)a.D.long_pieces, D.Hkv, a.seq_count);
    paged_long_keys_kernel<<<grid, EV_T, 0, s>>>(a);
    paged_long_select_kernel<<<grid, EV_T, 0, s>>>(a);
    paged_long_count_kernel<<<pieces, EV_T, 0, s>>>(a);
    paged_long_lists_kernel<<<pieces, EV_T, 0, s>>>(a);
  }
  // a wavefront has four of its rows in flight; as many workgroups as that needs, up to a few per compute unit
  const int at_once = 32 / (D.d * D.elt / 16) * 16;
  const int wgs = (int)std::max<long long>(1, std::min<long long>((most + at_once - 1) / at_once, 8ll * a.n_cus / (D.Hkv * a.seq_count)));
  paged_move_kernel<<<dim3(wgs, D.Hkv, a.seq_count), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ltri
