// Attention over a key-value cache in pages: o = sum_j softmax_j(q.k_j / sqrt(d)) v_j over a sequence's tokens, one pass
// with a running maximum and sum; with weights every token's share p_j = exp(s_j - lse) is added up per KV head.
//
// What bounds it: the key and value rows, each read once (512 bytes of bf16 rows and 4 G n products of 128 a token and KV head).
// So nothing is staged where one wavefront needs it: a lane loads 16-byte pieces in the order in which the matrix cores take them, and while a tile of 32
// tokens (fp32: 16) is used, the next one's rows come into the registers as they fall free: eight wavefronts a compute unit, 128 KB
// on their way. 16 sequences of 128K tokens, 8 KV heads x 128 in bf16: 1253 us, 6.9 TB/s (a large copy 5.9, a large read 6.9);
// 2 of 128K in fp32 327 us; one of 1000 tokens 10.9 us, of which the place in the row of tiles takes 1.3, the first rows 3.3, join
// and partial results 0.8, the ticket 0.9, the merge 3.5 and the launch the rest.
//   S^T = K Q^T    A = 16 tokens (lane % 16) x head_dim pieces (lane / 16), B = 16 (query row, head) pairs: a lane gets
//                  tokens 4 (lane / 16) + j, j < 4, of pair lane % 16. All query rows and heads of a KV head share the rows.
//   O^T = V^T P^T  A = V^T: lane % 16 stands for the CP columns whose piece of a row the lane has loaded, and one product per
//                  column of a piece takes that column of its tokens 4 (lane / 16) + j: in bf16 byte permutes inside the lane,
//                  no transposition. B = P^T is what the first product left in the lane. O^T and the running maximum both have
//                  the pair in lane % 16, so a rescale needs no exchange either.
// bf16 probabilities enter as p = hi + lo, two bf16 parts (the matrix cores are idle otherwise): the result is off by its own
// rounding only. fp32 runs the fp32 matrix cores.
// The tiles of all sequences, KV heads and blocks of pairs lie in one row, of which every workgroup takes an even share, whatever
// the lengths (paged_walk.h); its wavefronts take its tiles in turn and merge in LDS. Where a problem's tiles lie in several shares,
// the workgroup that finishes last (a ticket), or a launch of its own, adds the partial results up in order, so results do not
// depend on who that was. Two workgroups a compute unit: with three the tile loop spills (1839 us for the first case above), and at
// head_dim 64, where it does not, 16 sequences of 64K tokens took 172 us against 169, 16 rows over 4 of 32K 51.7 against 48.4. The
// last tenth of the row in short shares for whoever is done first (dies end 5 to 10 % apart): what a share costs to begin is more.
#include <algorithm>

#include "device_common.h"
#include "paged_internal.h"
#include "paged_walk.h"

namespace ltri {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int PA_WAVES = 4;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

template <int DT> struct PagedTile { static constexpr int N = DT == LTRI_F32 ? 16 : 32; };       // tokens per tile

// A KV head's problems: blocks of `size` pairs.
__host__ __device__ __forceinline__ int pair_blocks(const PagedCall& a, int size) { return (a.n * a.D.G + size - 1) / size; }
__device__ __forceinline__ int tiles_of(int len, int tile) { return (len + tile - 1) / tile; }
// What a problem counts as when work is shared out: its tiles and PAGED_EXTRA, which its beginning and end cost.
__device__ __forceinline__ int units_of(int len, int tile) { return len ? tiles_of(len, tile) + PAGED_EXTRA : 0; }

__device__ __forceinline__ long long share_of(long long total, int wgs, int min_share) { return max((total + wgs - 1) / wgs, (long long)min_share); }

// Scores of sequence s: [KV head][pair][tokens, padded to the tile], behind the units of the sequences in front; NULL: no room.
__device__ __forceinline__ float* score_rows(const PagedCall& a, long long before, int nt, int tile, int h) {
  if ((before + nt) * tile > a.D.score_tiles * PAGED_TILE) return nullptr;
  return a.scores + ((size_t)before * a.D.Hkv + (size_t)h * nt) * tile * (a.n * a.D.G);
}

// An element of an array that does not change while a launch runs, at an index that the wavefront shares.
__device__ __forceinline__ int scalar_load(const int32_t* p, int i) {
  typedef const __attribute__((address_space(4))) int32_t* constant_ptr;
  return ((constant_ptr)(uintptr_t)p)[i];
}
// The same value, as one that is only known here: what is computed from it stays here and is not kept in registers from before a loop.
__device__ __forceinline__ int only_here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
// 16 bytes a lane from base + off into LDS at to + 16 lane, without registers; M0 needs a cycle before it is used.
__device__ __forceinline__ void to_lds(const char* base, uint32_t off, uint32_t to) {
  const uint64_t b = (uint64_t)(uintptr_t)base;
  const uint64_t all = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)b);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(all) : "m0", "memory");
}
// Until the wavefront has N loads under way at most and its reads of LDS are done, then for the other wavefronts.
template <int N> __device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float over_quarters(float v) {        // sum over the four lanes of a pair
  v += __uint_as_float(lane_xor_c<16>(__float_as_uint(v)));
  return v + __uint_as_float(lane_xor_c<32>(__float_as_uint(v)));
}
__device__ __forceinline__ float max_quarters(float v) {
  v = fmaxf(v, __uint_as_float(lane_xor_c<16>(__float_as_uint(v))));
  return fmaxf(v, __uint_as_float(lane_xor_c<32>(__float_as_uint(v))));
}
__device__ __forceinline__ bool not_finite_f32(uint32_t x) { return (x & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool not_finite_bf16x2(uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ unsigned long long two_floats(float x, float y) {
  return ((unsigned long long)__float_as_uint(y) << 32) | __float_as_uint(x);
}
__device__ __forceinline__ float first_float(unsigned long long v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float second_float(unsigned long long v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ float safe_ref(float m) { return m == -INFINITY ? 0.f : m; }

// A wavefront's matrix products of one tile, by type. NU: groups of 16 tokens in a tile; VW: 32-bit words of a lane's piece of a value row.
// ONCE: no other wavefront of the problem reads these rows: they pass the caches by. 16 x 128K tokens 1394 -> 1268 us, 64 ragged sequences
// 193 -> 180; where wavefronts share rows (16 query rows over 32K) it is 59 -> 85. It knows nothing of pages that sequences share: 64 of 8704
// tokens, 8192 of them the same pages, take 201 us with it and 159 without, with pages of their own 340 and 382.
template <bool ONCE, class T> __device__ __forceinline__ T load_row(const char* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load((const T*)p);
  else return *(const T*)p;
}
template <int DT, int DIM, bool ONCE> struct TileOps;

template <int DIM, bool ONCE> struct TileOps<LTRI_BF16, DIM, ONCE> {
  static constexpr int NU = 2, NK = DIM / 32, NT = DIM / 16, CP = NT, VW = CP / 2;
  typedef u32x4_t Piece;
  Piece q[NK], k[NU][NK];
  uint32_t v[NU][4][VW];
  f32x4_t o[NT];
  __device__ __forceinline__ void load_q(const char* row, int g, bool there) {
#pragma unroll
    for (int i = 0; i < NK; ++i) q[i] = there ? *(const u32x4_t*)(row + i * 64 + g * 16) : u32x4_t{0u, 0u, 0u, 0u};
  }
  __device__ __forceinline__ void load_k(int u, const char* row, int g) {            // row: of token 16 u + lane % 16
#pragma unroll
    for (int i = 0; i < NK; ++i) k[u][i] = load_row<ONCE, u32x4_t>(row + i * 64 + g * 16);
  }
  __device__ __forceinline__ void store_k(int u, char* row, int g) const {
#pragma unroll
    for (int i = 0; i < NK; ++i) *(u32x4_t*)(row + i * 64 + g * 16) = k[u][i];
  }
  __device__ __forceinline__ void load_v(int u, int j, const char* row, int kl) {    // row: of token 16 u + 4 (lane / 16) + j
    if constexpr (VW == 4) {
      const u32x4_t x = load_row<ONCE, u32x4_t>(row + kl * 16);
      v[u][j][0] = x[0]; v[u][j][1] = x[1]; v[u][j][2] = x[2]; v[u][j][3] = x[3];
    } else {
      const u32x2_t x = load_row<ONCE, u32x2_t>(row + kl * 8);
      v[u][j][0] = x[0]; v[u][j][1] = x[1];
    }
  }
  __device__ __forceinline__ void store_v(int u, int j, char* row, int kl) const {
    if constexpr (VW == 4) *(u32x4_t*)(row + kl * 16) = u32x4_t{v[u][j][0], v[u][j][1], v[u][j][2], v[u][j][3]};
    else *(u32x2_t*)(row + kl * 8) = u32x2_t{v[u][j][0], v[u][j][1]};
  }
  __device__ __forceinline__ void zero_v(int u, int j) {
#pragma unroll
    for (int w = 0; w < VW; ++w) v[u][j][w] = 0u;
  }
  __device__ __forceinline__ bool odd_v(int u, int j) const {
    bool odd = false;
#pragma unroll
    for (int w = 0; w < VW; ++w) odd |= not_finite_bf16x2(v[u][j][w]);
    return odd;
  }
  __device__ __forceinline__ void scores(f32x4_t (&s)[NU]) const {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      s[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NK; ++i)
        s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k[u][i]), __builtin_bit_cast(bf16x8_t, q[i]), s[u], 0, 0, 0);
    }
  }
  // o += V^T P^T. APART: only the lane's tokens [u][j] whose bit 4 u + j of vis is set count, and only lanes with `mine` take the sum.
  template <bool APART>
  __device__ __forceinline__ void values(const f32x4_t (&p)[NU], uint32_t vis, bool mine) {
    u32x4_t hi, lo;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float x = p[u][2 * c], y = p[u][2 * c + 1];
        const uint32_t h = pack2(x, y);
        hi[2 * u + c] = h;
        lo[2 * u + c] = pack2(x - __uint_as_float(h << 16), y - __uint_as_float(h & 0xFFFF0000u));
      }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      u32x4_t col;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t x = __builtin_amdgcn_perm(v[u][2 * c + 1][t / 2], v[u][2 * c][t / 2], t & 1 ? 0x07060302u : 0x05040100u);
          if (APART) x &= ((vis >> (4 * u + 2 * c)) & 1 ? 0xFFFFu : 0u) | ((vis >> (4 * u + 2 * c + 1)) & 1 ? 0xFFFF0000u : 0u);
          col[2 * u + c] = x;
        }
      const bf16x8_t A = __builtin_bit_cast(bf16x8_t, col);
      f32x4_t sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, __builtin_bit_cast(bf16x8_t, lo), o[t], 0, 0, 0);
      sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, __builtin_bit_cast(bf16x8_t, hi), sum, 0, 0, 0);
      if constexpr (APART) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][e] = mine ? sum[e] : o[t][e];
      } else {
        o[t] = sum;
      }
    }
  }
};

template <int DIM, bool ONCE> struct TileOps<LTRI_F32, DIM, ONCE> {
  static constexpr int NU = 1, NK = DIM / 16, NT = DIM / 16, CP = 4, VW = DIM / 16;
  typedef f32x4_t Piece;
  Piece q[NK], k[NU][NK];
  uint32_t v[NU][4][VW];
  f32x4_t o[NT];
  __device__ __forceinline__ void load_q(const char* row, int g, bool there) {
#pragma unroll
    for (int i = 0; i < NK; ++i) q[i] = there ? *(const f32x4_t*)(row + i * 64 + g * 16) : f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void load_k(int u, const char* row, int g) {
#pragma unroll
    for (int i = 0; i < NK; ++i) k[u][i] = load_row<ONCE, f32x4_t>(row + i * 64 + g * 16);
  }
  __device__ __forceinline__ void store_k(int u, char* row, int g) const {
#pragma unroll
    for (int i = 0; i < NK; ++i) *(f32x4_t*)(row + i * 64 + g * 16) = k[u][i];
  }
  __device__ __forceinline__ void load_v(int u, int j, const char* row, int kl) {
#pragma unroll
    for (int c = 0; c < VW / 4; ++c) {
      const u32x4_t x = load_row<ONCE, u32x4_t>(row + c * 256 + kl * 16);
      v[u][j][4 * c] = x[0]; v[u][j][4 * c + 1] = x[1]; v[u][j][4 * c + 2] = x[2]; v[u][j][4 * c + 3] = x[3];
    }
  }
  __device__ __forceinline__ void store_v(int u, int j, char* row, int kl) const {
#pragma unroll
    for (int c = 0; c < VW / 4; ++c)
      *(u32x4_t*)(row + c * 256 + kl * 16) = u32x4_t{v[u][j][4 * c], v[u][j][4 * c + 1], v[u][j][4 * c + 2], v[u][j][4 * c + 3]};
  }
  __device__ __forceinline__ void zero_v(int u, int j) {
#pragma unroll
    for (int w = 0; w < VW; ++w) v[u][j][w] = 0u;
  }
  __device__ __forceinline__ bool odd_v(int u, int j) const {
    bool odd = false;
#pragma unroll
    for (int w = 0; w < VW; ++w) odd |= not_finite_f32(v[u][j][w]);
    return odd;
  }
  __device__ __forceinline__ void scores(f32x4_t (&s)[NU]) const {
    s[0] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[0][i][e], q[i][e], s[0], 0, 0, 0);
  }
  template <bool APART>
  __device__ __forceinline__ void values(const f32x4_t (&p)[NU], uint32_t vis, bool mine) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4_t sum = o[t];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        sum = __builtin_amdgcn_mfma_f32_16x16x4f32(!APART || ((vis >> j) & 1) ? __uint_as_float(v[0][j][t]) : 0.f, p[0][j], sum, 0, 0, 0);
      if constexpr (APART) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[t][e] = mine ? sum[e] : o[t][e];
      } else {
        o[t] = sum;
      }
    }
  }
};

// Sum of a problem's partial results of four columns of a pair: the parts first, first + step, ..., eight in flight. block: pairs of a
// problem. SAME: written by the same launch (device scope, see wait_for_own_stores).
template <int DIM, bool SAME>
__device__ __forceinline__ void add_parts(const PagedCall& a, int block, int w0, int parts, int first, int step, int p, int c, f32x4_t& o, float& top,
                                          float& sum) {
  constexpr int DEEP = 8;
  top = -INFINITY;
  sum = 0.f;
  o = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int k0 = first; k0 < parts; k0 += step * DEEP) {
    unsigned long long ml[DEEP];
    f32x4_t part[DEEP];
#pragma unroll
    for (int u = 0; u < DEEP; ++u) {
      const int k = min(k0 + step * u, parts - 1);
      const size_t at_part = (2 * (size_t)(w0 + k) + (k == 0)) * block + p;
      const float* from = a.part + at_part * DIM + c;
      if constexpr (SAME) {
        const unsigned long long* two = (const unsigned long long*)from;
        ml[u] = __hip_atomic_load(a.part_ml + at_part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const unsigned long long lo = __hip_atomic_load(two, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const unsigned long long hi = __hip_atomic_load(two + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        part[u] = f32x4_t{first_float(lo), second_float(lo), first_float(hi), second_float(hi)};
      } else {
        ml[u] = a.part_ml[at_part];
        part[u] = *(const f32x4_t*)from;
      }
    }
    float most = top;
#pragma unroll
    for (int u = 0; u < DEEP; ++u) most = fmaxf(most, first_float(ml[u]));     // (past the end: the last part's again)
    const float ref = safe_ref(most), back = __builtin_amdgcn_exp2f(top - ref);
    sum *= back;
    o *= back;
    top = most;
#pragma unroll
    for (int u = 0; u < DEEP; ++u) {
      if (k0 + step * u >= parts) continue;
      const float e = __builtin_amdgcn_exp2f(first_float(ml[u]) - ref);
      sum = fmaf(e, second_float(ml[u]), sum);
      o += e * part[u];
    }
  }
}

// A result's four columns, and with the first of them its log-sum-exp.
template <int DT, int DIM>
__device__ __forceinline__ void write_result(const PagedCall& a, size_t r, int c, f32x4_t o, float top, float sum) {
  if (sum == 0.f) o = f32x4_t{0.f, 0.f, 0.f, 0.f};
  else o *= 1.f / sum;
  if constexpr (DT == LTRI_F32) *(f32x4_t*)((float*)a.out + r * DIM + c) = o;
  else *(uint2*)((uint16_t*)a.out + r * DIM + c) = make_uint2(pack2(o[0], o[1]), pack2(o[2], o[3]));
  if (c == 0) {
    const float lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
    a.lse2[r] = lse2;
    if (a.lse) a.lse[r] = lse2 * LN2;
  }
}

// WB blocks of 16 pairs to a problem: a wavefront has block wave % WB, and every (PA_WAVES / WB)-th tile of the share. The blocks'
// wavefronts go through the same tiles side by side, so that one reads from memory what the others find in the compute unit's
// cache (two or four blocks to a wavefront need more registers than there are: 16 rows of 4 heads over 32K tokens 80 us, this 55).
// SHARED: four blocks of 128 columns read each tile from LDS, where all four wavefronts have brought it, three tiles ahead: 96 KB on
// their way a compute unit instead of 32, a quarter of the requests. The same 40.5 us with its merge, without 58; one workgroup a compute
// unit 43.8. 64 rows 98: a tile's 24 products a wavefront and the exponentials of 64 pairs take the compute unit 0.66 us, its bytes 0.7.
// SMALL: pages of fewer than 16 tokens, whose page is looked up lane by lane; else a group of 16 tokens lies in one page.
template <int DT, int DIM, int WB, bool SMALL>
__global__ __launch_bounds__(64 * PA_WAVES, 2) void paged_attend_kernel(PagedCall a, int min_share, int merge_later) {
  typedef TileOps<DT, DIM, WB == 1> Ops;
  constexpr int T = PagedTile<DT>::N, NU = Ops::NU, NT = Ops::NT, CP = Ops::CP, ELT = DT == LTRI_F32 ? 4 : 2;
  constexpr int PITCH = DIM + 4;
  static_assert(NU * 16 == T && WALK_T == 64 * PA_WAVES, "");
  constexpr int PB = 16 * WB, STEP = PA_WAVES / WB;                  // pairs of a problem, wavefronts of a block
  // SHARED: tiles in LDS, 16 KB each, in the pieces that lanes take: STAGES in a ring; afterwards the wavefronts' O.
  constexpr bool SHARED = WB == PA_WAVES && DIM == 128 && !SMALL;
  constexpr int STAGES = 4, STAGE_BYTES = 16384, O_BYTES = sizeof(float) * PA_WAVES * 16 * PITCH;
  static_assert(!SHARED || T * 2 * DIM * ELT == STAGE_BYTES, "");
  __shared__ __align__(16) char s_mem[SHARED && STAGES * STAGE_BYTES > O_BYTES ? STAGES * STAGE_BYTES : O_BYTES];
  float (*s_o)[16][PITCH] = (float (*)[16][PITCH])s_mem;
  __shared__ float s_m[PA_WAVES][16], s_l[PA_WAVES][16];
  __shared__ int s_last;
  const PagedDims& D = a.D;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kl = lane & 15, g = lane >> 4;
  const int w = blockIdx.x, pairs = a.n * D.G, blocks = pair_blocks(a, PB), per_tile = D.Hkv * blocks;
  const int page_mask = (1 << D.page_shift) - 1;
  const long long page_bytes = D.page_stride * ELT;
  const int tok_bytes = (int)D.token_stride * ELT;                   // 16 of them lie within 32 bits
  const uint32_t k_off = (uint32_t)(kl * tok_bytes + g * 16), v_off = (uint32_t)(4 * g * tok_bytes + kl * (CP * ELT));
  const float sc = LOG2E / sqrtf((float)DIM);

  long long share = 0;
  const PagedPlace at = paged_find(a.seq_count, [&](int s) { return (long long)units_of(paged_len(a, s), T) * per_tile; },
                                   [&](long long total) {
                                     share = share_of(total, gridDim.x, min_share);
                                     return share * w;
                                   });
  // sequences without tokens
  for (int s = w; s < a.seq_count; s += gridDim.x) {
    if (paged_len(a, s) > 0) continue;
    for (int i = tid; i < a.n * D.Hq; i += WALK_T) {
      const size_t r = (size_t)s * a.n * D.Hq + i;
      for (int c = 0; c < DIM * ELT / 16; ++c) ((uint4*)a.out)[r * (DIM * ELT / 16) + c] = make_uint4(0, 0, 0, 0);
      a.lse2[r] = -INFINITY;
      if (a.lse) a.lse[r] = -INFINITY;
    }
  }
  if (at.seq < 0) return;
  long long x = share * w, x_end = min(x + share, at.total), before = at.before;
  int s = at.seq;
  while (x < x_end) {
    const int len = paged_len(a, s), nt = tiles_of(len, T);
    const long long mine = (long long)units_of(len, T) * per_tile;
    if (x >= before + mine) {                            // on to the next sequence
      before += mine;
      ++s;
      continue;
    }
    const int hp = (int)((x - before) / (nt + PAGED_EXTRA)), h = hp / blocks, pb = hp % blocks;
    const long long problem = before + (long long)hp * (nt + PAGED_EXTRA) + PAGED_EXTRA; // its first tile
    const int t0 = (int)max(x - problem, 0ll), t1 = (int)min((long long)nt, x_end - problem);
    x = problem + max(t1, 0);
    if (t0 >= t1) continue;

    const int first_new = a.k_new ? max(len - a.n, 0) : len;         // tokens from here on come with the call
    const int np = min(PB, pairs - pb * PB);
    const int pair0 = pb * PB + 16 * (wave % WB);                    // the wavefront's pairs: from here on
    const int pair = min(pair0 + kl, pairs - 1), query_row = pair / D.G;
    const int sees = len - a.n + 1 + query_row;                      // tokens that the lane's pair sees
    const int all_see = len - a.n + 1 + min(pair0, pairs - 1) / D.G; // ... that every pair of the block sees
    // Tiles from here on: some token is not seen by some pair, or comes with the call. They take a way of their own, without the next
    // tile's rows on theirs; with SMALL pages every tile does, and has them.
    // (SHARED: the same for all wavefronts.)
    const int edge = SMALL ? t0 : min(t1, max(0, min(SHARED ? len - a.n + 1 + pb * PB / D.G : all_see, first_new)) / T);
    const int32_t* table = a.table + (size_t)s * D.table_pages;
    const char* kh = a.k + (size_t)h * D.head_stride * ELT;
    const char* vh = a.v + (size_t)h * D.head_stride * ELT;
    float* scores = nullptr;
    if (a.decay >= 0.f && paged_keeps_scores(pairs)) {
      scores = score_rows(a, before / per_tile, nt, T, h);
      if (scores) scores += (size_t)(pair0 + kl) * nt * T + 4 * g;
    }

    Ops ops;
    ops.load_q((const char*)a.q + (((size_t)s * a.n + query_row) * D.Hq + h * D.G + pair % D.G) * DIM * ELT, g, pair0 + kl < pairs);
#pragma unroll
    for (int t = 0; t < NT; ++t) ops.o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    // Pages of a tile: of its groups of 16 tokens, by scalar loads (the table does not change while a launch runs), or (SMALL) of the
    // token that the lane loads of every group's keys and of its four of the values. Past the sequence's end the last token's. They
    // are asked for before the rows of the tile in front, so that the loads, which come back in order, need not be waited for.
    struct Pages { int k[NU], v[NU][SMALL ? 4 : 1]; };
    auto look_up = [&](int t, Pages& p) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const int i0 = t * T + 16 * u;
        if constexpr (SMALL) {
          p.k[u] = table[min(i0 + kl, len - 1) >> D.page_shift];
#pragma unroll
          for (int j = 0; j < 4; ++j) p.v[u][j] = table[min(i0 + 4 * g + j, len - 1) >> D.page_shift];
        } else {
          p.k[u] = p.v[u][0] = scalar_load(table, __builtin_amdgcn_readfirstlane(min(i0, len - 1) >> D.page_shift));
        }
      }
    };
    auto good = [&](int page) { return (unsigned)page < (unsigned)D.n_pages; };
    auto row = [&](const char* base, int page, int i) __attribute__((always_inline)) {
      return base + ((long long)(good(page) ? page : 0) * page_bytes + (long long)(i & page_mask) * tok_bytes);
    };
    // rows of an edge tile, lane by lane; new tokens are read from the call's rows
    auto new_row = [&](const void* rows, int i) { return (const char*)rows + (((size_t)s * D.Hkv + h) * a.n + (i - (len - a.n))) * DIM * ELT; };
    auto edge_row = [&](const char* base, const void* rows, int page, int i) __attribute__((always_inline)) {
      i = min(i, len - 1);                                           // (the page is that of this token, too)
      return i >= first_new ? new_row(rows, i) : row(base, page, i);
    };
    auto load_k = [&](int t, const Pages& p, auto edge_c) __attribute__((always_inline)) {
      if constexpr (decltype(edge_c)::value) {
        const int kl_ = only_here(kl), g_ = only_here(g);
#pragma unroll
        for (int u = 0; u < NU; ++u) ops.load_k(u, edge_row(kh, a.k_new, p.k[u], t * T + 16 * u + kl_), g_);
      } else {
#pragma unroll
        for (int u = 0; u < NU; ++u) ops.load_k(u, row(kh, p.k[u], t * T + 16 * u) + k_off, 0);
      }
    };
    auto load_v = [&](int t, const Pages& p, auto edge_c) __attribute__((always_inline)) {
      if constexpr (decltype(edge_c)::value) {
        const int kl_ = only_here(kl), g_ = only_here(g);
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) ops.load_v(u, j, edge_row(vh, a.v_new, p.v[u][SMALL ? j : 0], t * T + 16 * u + 4 * g_ + j), kl_);
      } else {
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) ops.load_v(u, j, row(vh, p.v[u][0], t * T + 16 * u) + j * tok_bytes + v_off, 0);
      }
    };

    Pages now, next;
    // One tile; EDGE: see `edge`; MORE: the wavefront's next tile follows, and its rows are asked for. (With a condition in the loop in
    // its place the compiler, which then cannot count the loads on their way, waits for the values before the keys are used.)
    auto tile = [&](int t, auto edge_c, auto more_c, const char* staged = nullptr) __attribute__((always_inline)) {
      constexpr bool EDGE = decltype(edge_c)::value, MORE = decltype(more_c)::value;
      if constexpr (SHARED && !EDGE) {
#pragma unroll
        for (int e = 0; e < NU * Ops::NK; ++e) ops.k[e / Ops::NK][e % Ops::NK] = *(const typename Ops::Piece*)(staged + e * 1024 + lane * 16);
      } else if constexpr (EDGE && !SMALL) {
        look_up(t, now);
        load_k(t, now, edge_c);
        load_v(t, now, edge_c);
      }
      f32x4_t sv[NU];
      const int kl_ = EDGE ? only_here(kl) : kl, g_ = EDGE ? only_here(g) : g;
      const bool writes = EDGE && a.k_new && pb == 0 && wave % WB == 0;
      ops.scores(sv);
      if (writes) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          const int i = t * T + 16 * u + kl_;
          const int page = i >= first_new && i < len ? paged_page(a, s, i) : -1;
          if (page < 0) continue;
          ops.store_k(u, const_cast<char*>(row(kh, page, i)), g_);
          if (D.weights && g_ == 0) {
            const size_t mark = paged_mark(D, page, h, i);
            a.weight[mark] = 0.f;
            a.pos[mark] = a.seen[s] - (len - i);
          }
        }
      }
      Pages after;
      if constexpr (MORE) {
        look_up(min(t + 2 * STEP, nt - 1), after);
        load_k(t + STEP, next, edge_c);
        __builtin_amdgcn_sched_barrier(0);
      }

      // of the lane's tokens 16 u + 4 g + j (bit 4 u + j): which are there at all, and which its pair sees
      uint32_t there = 0xFFu, vis = 0xFFu;
      if constexpr (EDGE) {
        there = vis = 0u;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = t * T + 16 * u + 4 * g_ + j;
            const bool ok = i < len && good(now.v[u][SMALL ? j : 0]);
            if (i < len && !ok) atomicCAS(a.err, 0, LTRI_EINVAL);
            there |= (uint32_t)ok << (4 * u + j);
            vis |= (uint32_t)(ok && i < sees) << (4 * u + j);
          }
      } else {
        bool bad = false;
#pragma unroll
        for (int u = 0; u < NU; ++u) bad |= !good(now.k[u]);
        if (bad) {                                                   // (uniform)
          atomicCAS(a.err, 0, LTRI_EINVAL);
#pragma unroll
          for (int u = 0; u < NU; ++u)
            if (!good(now.k[u])) {
              there &= ~(0xFu << (4 * u));
#pragma unroll
              for (int j = 0; j < 4; ++j) ops.zero_v(u, j);
              sv[u] = f32x4_t{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            }
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sv[u][j] *= sc;
          if constexpr (EDGE) sv[u][j] = (vis >> (4 * u + j)) & 1 ? sv[u][j] : -INFINITY;
          mx = fmaxf(mx, sv[u][j]);
        }
      if (!SHARED && scores && pair0 + kl < pairs) {
#pragma unroll
        for (int u = 0; u < NU; ++u) *(f32x4_t*)(scores + (size_t)t * T + 16 * u) = sv[u];
      }
      const float m_new = fmaxf(m, max_quarters(mx)), ref = safe_ref(m_new);
      if (__any(m_new > m)) {                                        // rare after the first tiles
        const float alpha = __builtin_amdgcn_exp2f(m - ref);
        l *= alpha;
#pragma unroll
        for (int c = 0; c < NT; ++c) ops.o[c] *= alpha;
        m = m_new;
      }
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sv[u][j] = __builtin_amdgcn_exp2f(sv[u][j] - ref);
          l += sv[u][j];
        }
      if constexpr (SHARED && !EDGE) {
        constexpr int PER = Ops::VW / 4;         // pieces of a lane's part of a value row
#pragma unroll
        for (int e = 0; e < NU * 4 * PER; ++e) {
          const u32x4_t x = *(const u32x4_t*)(staged + STAGE_BYTES / 2 + e * 1024 + lane * 16);
#pragma unroll
          for (int i = 0; i < 4; ++i) ops.v[e / (4 * PER)][e / PER % 4][e % PER * 4 + i] = x[i];
        }
        if (there != 0xFFu) {                                        // (uniform)
#pragma unroll
          for (int u = 0; u < NU; ++u)
            if (!((there >> (4 * u)) & 1)) {
#pragma unroll
              for (int j = 0; j < 4; ++j) ops.zero_v(u, j);
            }
        }
      }
      bool apart = false;                        // an infinity or NaN in a token that some pair of the block does not see
      if constexpr (EDGE) {
        if (writes) {
#pragma unroll
          for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int i = t * T + 16 * u + 4 * g_ + j;
              const int page = i >= first_new && i < len ? now.v[u][SMALL ? j : 0] : -1;
              if (good(page)) ops.store_v(u, j, const_cast<char*>(row(vh, page, i)), kl_);
            }
        }
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (!((there >> (4 * u + j)) & 1)) ops.zero_v(u, j);
            else if (t * T + 16 * u + 4 * g_ + j >= all_see) apart |= ops.odd_v(u, j);
          }
        apart = (bool)__any(apart);
        if (apart) {
          // query row by query row, which takes the tokens it sees (0 times infinity would not be 0)
          const int r0 = pair0 / D.G, r1 = min(pair0 + 15, pairs - 1) / D.G;
          for (int r = r0; r <= r1; ++r) {
            uint32_t seen_bits = 0u;
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
              for (int j = 0; j < 4; ++j) seen_bits |= (uint32_t)(t * T + 16 * u + 4 * g_ + j < len - a.n + 1 + r) << (4 * u + j);
            ops.template values<true>(sv, seen_bits, query_row == r);
          }
        }
      }
      if (!apart) ops.template values<false>(sv, 0u, true);
      if constexpr (MORE) {
        __builtin_amdgcn_sched_barrier(0);
        load_v(t + STEP, next, edge_c);
        __builtin_amdgcn_sched_barrier(0);
        now = next;
        next = after;
      }
    };
    int t = t0 + wave / WB;
    if (pair0 >= pairs) t = t1;                                      // a block without pairs
    constexpr std::integral_constant<bool, SMALL> small_c{};
    const int end = SMALL ? t1 : edge;
    if constexpr (SHARED) {
      // Every wavefront brings a quarter of each tile, STAGES - 1 tiles ahead, from a page that it has looked up one tile sooner.
      const int last = __builtin_amdgcn_readfirstlane(end), begin = __builtin_amdgcn_readfirstlane(t0);
      const int u = wave * NU / PA_WAVES;        // the group of 16 tokens it brings some of
      const uint32_t ring = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)s_mem;
      auto page_of = [&](int x) { return scalar_load(table, (min(x, last - 1) * T + 16 * u) >> D.page_shift); };
      auto fetch = [&](int x, int page) __attribute__((always_inline)) {
        const char *kb = row(kh, page, x * T + 16 * u), *vb = row(vh, page, x * T + 16 * u);
        const uint32_t to = ring + (x - begin) % STAGES * STAGE_BYTES;
        constexpr int PER = Ops::VW / 4;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int piece = 2 * wave + e;
          to_lds(kb, k_off + piece % Ops::NK * 64, to + piece * 1024);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int piece = 2 * wave + e;
          to_lds(vb, v_off + piece / PER % 4 * tok_bytes + piece % PER * 256, to + STAGE_BYTES / 2 + piece * 1024);
        }
      };
      if (begin < last) {
        __syncthreads();                         // (the problem before has been read)
        int page[STAGES];
#pragma unroll
        for (int i = 0; i < STAGES; ++i) page[i] = page_of(begin + i);
        look_up(begin, now);
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i)
          if (begin + i < last) fetch(begin + i, page[i]);
        int ahead = page[STAGES - 1];
#pragma unroll
        for (int i = 0; i < Ops::NK; ++i) asm volatile("" : "+v"(ops.q[i]));      // (here and not in the loop, which counts its loads itself)
        for (int x = begin; x < last; ++x) {
          if (x + STAGES - 1 < last) {
            meet<4 * (STAGES - 2)>();            // tile x is there, and tile x - 1 has been read
            fetch(x + STAGES - 1, ahead);
          } else {
            meet<0>();
          }
          ahead = page_of(x + STAGES);
          look_up(min(x + 1, last - 1), next);
          if (pair0 < pairs) tile(x, small_c, std::false_type{}, s_mem + (x - begin) % STAGES * STAGE_BYTES);
          now = next;
        }
      }
      if (t < t1) t = last;
      if (t < t0) t = t0;
    } else if (t < end) {
      look_up(t, now);
      look_up(min(t + STEP, nt - 1), next);
      load_k(t, now, small_c);
      __builtin_amdgcn_sched_barrier(0);                             // keys before values, as in the loop: what is waited for first comes first
      load_v(t, now, small_c);
      __builtin_amdgcn_sched_barrier(0);
      for (; t + STEP < end; t += STEP) tile(t, small_c, std::true_type{});
      tile(t, small_c, std::false_type{});
      t += STEP;
    }
    if constexpr (!SMALL)
      for (; t < t1; t += STEP) tile(t, std::true_type{}, std::false_type{});

    // the wavefronts' results: own maximum, sum and O
    l = over_quarters(l);
    __syncthreads();                             // (the problem before has been read)
    const int tid_ = only_here(tid), lane_ = tid_ & 63, kl_ = lane_ & 15, g_ = lane_ >> 4;
    if (pair0 + kl_ < pairs) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int c = 0; c < NT; c += 4) {
          const int col = 16 * CP * (c / CP) + CP * (4 * g_ + j) + c % CP;
          *(f32x4_t*)&s_o[wave][kl_][col] = f32x4_t{ops.o[c][j], ops.o[c + 1][j], ops.o[c + 2][j], ops.o[c + 3][j]};
        }
      if (g_ == 0) { s_m[wave][kl_] = m; s_l[wave][kl_] = l; }
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == nt;
    const size_t slot = 2 * (size_t)w + (t0 == 0);
    // adds up those of a block, by threads that each take four columns of a pair, and hands (pair, column, O, maximum, sum) on
    auto join = [&](auto take) __attribute__((always_inline)) {
      for (int i = tid_; i < np * (DIM / 4); i += WALK_T) {
        const int p = i / (DIM / 4), c = i % (DIM / 4) * 4, w0 = p / 16, pl = p % 16;
        float top = s_m[w0][pl];
#pragma unroll
        for (int k = 1; k < STEP; ++k) top = fmaxf(top, s_m[w0 + k * WB][pl]);
        const float ref = safe_ref(top);
        float sum = 0.f;
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < STEP; ++k) {
          const float e = __builtin_amdgcn_exp2f(s_m[w0 + k * WB][pl] - ref);
          sum = fmaf(e, s_l[w0 + k * WB][pl], sum);
          o += e * *(const f32x4_t*)&s_o[w0 + k * WB][pl][c];
        }
        take(p, c, o, top, sum);
      }
    };
    auto result = [&](int p, int c, f32x4_t o, float top, float sum) __attribute__((always_inline)) {
      const int pr = pb * PB + p;
      write_result<DT, DIM>(a, ((size_t)s * a.n + pr / D.G) * D.Hq + h * D.G + pr % D.G, c, o, top, sum);
    };
    if (whole) {
      join(result);
      continue;
    }
    if (merge_later) {
      join([&](int p, int c, f32x4_t o, float top, float sum) __attribute__((always_inline)) {
        *(f32x4_t*)(a.part + (slot * PB + p) * DIM + c) = o;
        if (c == 0) a.part_ml[slot * PB + p] = two_floats(top, sum);
      });
      continue;
    }
    join([&](int p, int c, f32x4_t o, float top, float sum) __attribute__((always_inline)) {       // device scope (see wait_for_own_stores)
      unsigned long long* to = (unsigned long long*)(a.part + (slot * PB + p) * DIM + c);
      __hip_atomic_store(to, two_floats(o[0], o[1]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(to + 1, two_floats(o[2], o[3]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (c == 0) __hip_atomic_store(a.part_ml + slot * PB + p, two_floats(top, sum), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    const int w0 = (int)(problem / share), parts = (int)((problem + nt - 1) / share) - w0 + 1;      // the workgroups that share the problem
    wait_for_own_stores();
    __syncthreads();
    int32_t* ticket = a.tickets + ((size_t)s * D.Hkv + h) * blocks + pb;
    if (tid == 0) s_last = atomicAdd(ticket, 1) == parts - 1;
    __syncthreads();
    if (!s_last) continue;
    if (tid == 0) *ticket = 0;
    if constexpr (WB == 1) {                     // few pairs: every fourth part by one wavefront, then their sums as above
      for (int i = lane_; i < np * (DIM / 4); i += 64) {
        const int p = i / (DIM / 4), c = i % (DIM / 4) * 4;
        f32x4_t o;
        float top, sum;
        add_parts<DIM, true>(a, PB, w0, parts, wave, PA_WAVES, p, c, o, top, sum);
        *(f32x4_t*)&s_o[wave][p][c] = o;
        if (c == 0) { s_m[wave][p] = top; s_l[wave][p] = sum; }
      }
      __syncthreads();
      join(result);
    } else {
      for (int i = tid_; i < np * (DIM / 4); i += WALK_T) {
        const int p = i / (DIM / 4), c = i % (DIM / 4) * 4;
        f32x4_t o;
        float top, sum;
        add_parts<DIM, true>(a, PB, w0, parts, 0, 1, p, c, o, top, sum);
        result(p, c, o, top, sum);
      }
    }
  }
}

// The partial results of problems that several workgroups share, a workgroup per query row and head: where there are many of them,
// the workgroup that finishes last is too slow at it (128 KB through one compute unit take 9 us).
template <int DT, int DIM>
__global__ __launch_bounds__(WALK_T) void paged_merge_kernel(PagedCall a, int wgs, int min_share, int block) {
  constexpr int T = PagedTile<DT>::N;
  const PagedDims& D = a.D;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t r = blockIdx.x;
  const int head = (int)(r % D.Hq), q_row = (int)(r / D.Hq) % a.n, s = (int)(r / D.Hq / a.n), h = head / D.G, pair = q_row * D.G + head % D.G;
  const int blocks = pair_blocks(a, block), per_tile = D.Hkv * blocks;
  const int len = paged_len(a, s), nt = tiles_of(len, T);
  if (len == 0) return;
  const PagedPlace at = paged_place(a.seq_count, [&](int i) { return (long long)units_of(paged_len(a, i), T) * per_tile; }, s);
  const long long share = share_of(at.total, wgs, min_share);
  const long long problem = at.before + (long long)(h * blocks + pair / block) * (nt + PAGED_EXTRA) + PAGED_EXTRA;
  const int w0 = (int)(problem / share), parts = (int)((problem + nt - 1) / share) - w0 + 1;
  if (parts == 1) return;
  __shared__ __align__(16) float s_o[WALK_T / 64][2][DIM];
  __shared__ float s_m[WALK_T / 64][2], s_l[WALK_T / 64][2];
  constexpr int LANES = DIM / 4, SIDES = 2;      // lanes of a row; so many of them side by side take other parts
  const int side = lane / LANES, c = lane % LANES * 4;
  if (side < SIDES) {
    f32x4_t o;
    float top, sum;
    add_parts<DIM, false>(a, block, w0, parts, wave * SIDES + side, WALK_T / 64 * SIDES, pair % block, c, o, top, sum);
    *(f32x4_t*)&s_o[wave][side][c] = o;
    if (c == 0) { s_m[wave][side] = top; s_l[wave][side] = sum; }
  }
  __syncthreads();
  if (tid >= LANES) return;
  float top = -INFINITY, sum = 0.f;
  f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < WALK_T / 64 * SIDES; ++k) top = fmaxf(top, s_m[k / SIDES][k % SIDES]);
  const float ref = safe_ref(top);
#pragma unroll
  for (int k = 0; k < WALK_T / 64 * SIDES; ++k) {
    const float e = __builtin_amdgcn_exp2f(s_m[k / SIDES][k % SIDES] - ref);
    sum = fmaf(e, s_l[k / SIDES][k % SIDES], sum);
    o += e * *(const f32x4_t*)&s_o[k / SIDES][k % SIDES][c];
  }
  write_result<DT, DIM>(a, r, c, o, top, sum);
}

// Weights from the scores: w <- decay w + sum over the KV head's pairs of exp(s - lse). A wavefront takes 256 tokens of a KV head at a
// time, a lane four of them; the pieces are shared out like the tiles above. 16 x 16K tokens of 32 heads: 16 us for 50 MB.
constexpr int PW_TOKENS = 256;
template <int TILE>
__global__ __launch_bounds__(WALK_T) void paged_weights_kernel(PagedCall a) {
  const PagedDims& D = a.D;
  const int pairs = a.n * D.G, w = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  auto pieces = [&](int len) { return (len + PW_TOKENS - 1) / PW_TOKENS; };
  long long share = 0;
  const PagedPlace at = paged_find(a.seq_count, [&](int s) { return (long long)pieces(paged_len(a, s)) * D.Hkv; },
                                   [&](long long total) { share = (total + gridDim.x - 1) / gridDim.x; return share * w; });
  if (at.seq < 0) return;
  // units in front of the sequence
  long long units = paged_find(a.seq_count, [&](int s) { return s < at.seq ? (long long)units_of(paged_len(a, s), TILE) : 0; },
                               [&](long long) { return -1ll; }).total;
  long long before = at.before;
  const long long x_end = min(share * (w + 1), at.total);
  int s = at.seq;
  for (long long x = share * w + wave; x < x_end;) {
    const int len = paged_len(a, s), nt = tiles_of(len, TILE), np = pieces(len);
    if (x >= before + (long long)np * D.Hkv) {
      before += (long long)np * D.Hkv;
      units += units_of(len, TILE);
      ++s;
      continue;
    }
    const int h = (int)((x - before) / np), piece = (int)((x - before) % np);
    x += WALK_T / 64;
    const float* scores = score_rows(a, units, nt, TILE, h);
    if (!scores) {
      if (lane == 0) atomicCAS(a.err, 0, PAGED_NO_ROOM);
      continue;
    }
    const int i0 = piece * PW_TOKENS + 4 * lane, at_most = nt * TILE - 4;
    const size_t pitch = (size_t)nt * TILE;
    scores += min(i0, at_most);
    const float* lse = a.lse2 + (size_t)s * a.n * D.Hq + h * D.G;
    f32x4_t got = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < pairs; p0 += 4) {
      f32x4_t v[4];
      float l[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int p = min(p0 + u, pairs - 1);
        l[u] = lse[(size_t)(p / D.G) * D.Hq + p % D.G];
        v[u] = *(const f32x4_t*)(scores + p * pitch);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (p0 + u >= pairs || l[u] == -INFINITY) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) got[j] += __builtin_amdgcn_exp2f(v[u][j] - l[u]);
      }
    }
    for (int j = 0; j < 4; ++j) {
      if (i0 + j >= len) break;
      const int page = paged_page(a, s, i0 + j);
      if (page < 0) continue;
      float* to = a.weight + paged_mark(D, page, h, i0 + j);
      *to = a.decay == 0.f ? got[j] : fmaf(a.decay, *to, got[j]);
    }
  }
}

// The same from the keys, for many pairs (see paged_keeps_scores): the scores again, one tile of keys after the other, with the
// log-sum-exps at hand. The queries of 64 pairs stay in registers; the next tile's keys are on their way while one is used.
// 64 pairs over 32K tokens, 8 KV heads: 18 us for 67 MB of keys. More pairs go over the keys again for every 64, and over the weights:
// 512 pairs over 32K tokens, one KV head: 35 us (28 with loads that stay in the caches), 2048 pairs 122 (94).
template <int DT, int DIM>
__global__ __launch_bounds__(WALK_T, 2) void paged_key_weights_kernel(PagedCall a) {
  constexpr int T = PagedTile<DT>::N, ELT = DT == LTRI_F32 ? 4 : 2, WAVES = WALK_T / 64, NB = 4;
  typedef TileOps<DT, DIM, true> Ops;
  constexpr int NU = Ops::NU;
  const PagedDims& D = a.D;
  const int pairs = a.n * D.G, w = blockIdx.x, lane = threadIdx.x & 63, kl = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float sc = LOG2E / sqrtf((float)DIM);
  const int tok_bytes = (int)D.token_stride * ELT;
  long long share = 0;
  const PagedPlace at = paged_find(a.seq_count, [&](int s) { return (long long)tiles_of(paged_len(a, s), T) * D.Hkv; },
                                   [&](long long total) { share = share_of(total, gridDim.x, WAVES); return share * w; });
  if (at.seq < 0) return;
  long long x = share * w, before = at.before;
  const long long x_end = min(x + share, at.total);
  int s = at.seq;
  while (x < x_end) {
    const int len = paged_len(a, s), nt = tiles_of(len, T);
    if (x >= before + (long long)nt * D.Hkv) {
      before += (long long)nt * D.Hkv;
      ++s;
      continue;
    }
    const int h = (int)((x - before) / nt), t0 = (int)((x - before) % nt), t1 = (int)min((long long)nt, t0 + (x_end - x));
    x += t1 - t0;
    const int32_t* table = a.table + (size_t)s * D.table_pages;
    const char* kh = a.k + h * D.head_stride * ELT;
    struct Pages { int p[NU]; };                   // of the tokens 16 u + lane % 16; -1: none in the pool
    auto look_up = [&](int t, Pages& p) {
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        p.p[u] = table[min(t * T + 16 * u + kl, len - 1) >> D.page_shift];
        if ((unsigned)p.p[u] >= (unsigned)D.n_pages) p.p[u] = -1;
      }
    };
    Ops ops;
    auto load_k = [&](int t, const Pages& p) {
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const int i = min(t * T + 16 * u + kl, len - 1);
        ops.load_k(u, kh + (max(p.p[u], 0) * D.page_stride * ELT + (long long)(i & ((1 << D.page_shift) - 1)) * tok_bytes), g);
      }
    };
    for (int p0 = 0; p0 < pairs; p0 += 16 * NB) {
      typename Ops::Piece q[NB][Ops::NK];
      float lse2[NB];
      int sees[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int pair = min(p0 + 16 * b + kl, pairs - 1), row = pair / D.G;
        const size_t r = ((size_t)s * a.n + row) * D.Hq + h * D.G + pair % D.G;
        ops.load_q((const char*)a.q + r * DIM * ELT, g, true);
#pragma unroll
        for (int i = 0; i < Ops::NK; ++i) q[b][i] = ops.q[i];
        lse2[b] = a.lse2[r];
        sees[b] = p0 + 16 * b + kl < pairs && lse2[b] != -INFINITY ? len - a.n + 1 + row : 0;
      }
      int t = t0 + wave;
      Pages now, next;
      if (t < t1) {
        look_up(t, now);
        look_up(min(t + WAVES, nt - 1), next);
        load_k(t, now);
      }
      for (; t < t1; t += WAVES) {
        f32x4_t sv[NB][NU];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
          for (int i = 0; i < Ops::NK; ++i) ops.q[i] = q[b][i];
          ops.scores(sv[b]);
        }
        Pages after;
        look_up(min(t + 2 * WAVES, nt - 1), after);
        if (t + WAVES < t1) load_k(t + WAVES, next);
        // a lane's sums of its tokens 16 u + 4 g + j over the blocks, then over the 16 lanes that hold a token's pairs; lane 4 u + j
        // keeps token 4 g + j of group u
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float got = 0.f;
#pragma unroll
            for (int b = 0; b < NB; ++b) got += t * T + 16 * u + 4 * g + j < sees[b] ? __builtin_amdgcn_exp2f(fmaf(sv[b][u][j], sc, -lse2[b])) : 0.f;
            got += __uint_as_float(lane_xor_c<8>(__float_as_uint(got)));
            got += __uint_as_float(lane_xor_c<4>(__float_as_uint(got)));
            got += __uint_as_float(lane_xor_c<2>(__float_as_uint(got)));
            got += __uint_as_float(lane_xor_c<1>(__float_as_uint(got)));
            if (kl == 4 * u + j) sum = got;
          }
        const int u = kl >> 2, i = t * T + 16 * u + 4 * g + (kl & 3);
        const int page0 = __shfl(now.p[0], 4 * g + (kl & 3), 64), page1 = __shfl(now.p[NU - 1], 4 * g + (kl & 3), 64);
        const int page = u == 0 ? page0 : page1;
        if (u < NU && i < len && page >= 0) {
          float* to = a.weight + paged_mark(D, page, h, i);
          *to = p0 == 0 && a.decay == 0.f ? sum : fmaf(p0 == 0 ? a.decay : 1.f, *to, sum);
        }
        now = next;
        next = after;
      }
    }
  }
}

template <int DT, int DIM, int WB>
static void launch_pages(const PagedCall& a, int wgs, int min_share, bool later, hipStream_t s) {
  if (a.D.page_shift < 4) paged_attend_kernel<DT, DIM, WB, true><<<wgs, 64 * PA_WAVES, 0, s>>>(a, min_share, later);
  else paged_attend_kernel<DT, DIM, WB, false><<<wgs, 64 * PA_WAVES, 0, s>>>(a, min_share, later);
}
template <int DT, int DIM>
static void launch_blocks(const PagedCall& a, int wb, int wgs, int min_share, bool later, hipStream_t s) {
  if (wb == 1) launch_pages<DT, DIM, 1>(a, wgs, min_share, later, s);
  else if (wb == 2) launch_pages<DT, DIM, 2>(a, wgs, min_share, later, s);
  else launch_pages<DT, DIM, 4>(a, wgs, min_share, later, s);
}
template <int DT>
static void launch_dim(const PagedCall& a, int wb, int wgs, int min_share, bool later, hipStream_t s) {
  if (a.D.d == 64) launch_blocks<DT, 64>(a, wb, wgs, min_share, later, s);
  else launch_blocks<DT, 128>(a, wb, wgs, min_share, later, s);
  if (!later) return;
  const unsigned rows = (unsigned)a.seq_count * a.n * a.D.Hq;
  if (a.D.d == 64) paged_merge_kernel<DT, 64><<<rows, WALK_T, 0, s>>>(a, wgs, min_share, 16 * wb);
  else paged_merge_kernel<DT, 128><<<rows, WALK_T, 0, s>>>(a, wgs, min_share, 16 * wb);
}
template <int DT>
static void launch_key_weights(const PagedCall& a, int wgs, hipStream_t s) {
  if (a.D.d == 64) paged_key_weights_kernel<DT, 64><<<wgs, WALK_T, 0, s>>>(a);
  else paged_key_weights_kernel<DT, 128><<<wgs, WALK_T, 0, s>>>(a);
}

// A launch of its own for the merge from this many bytes of a problem's partial results on. One sequence, 8 KV heads of 4: 128K
// tokens (131 KB) 107.5 us with the last workgroup, 104.9 with the launch; 32K tokens of 16 rows (2 MB) 147 and 60; fp32, 2 x 4097
// tokens of one KV head, 64 wide (66 KB) 12.7 and 15.3. The host does not know the lengths: a long sequence among empty or short ones is
// merged by the last workgroup (16 rows over 32K tokens alone 40 us, beside 63 empty sequences 124, beside 63 of 100 tokens 97).
constexpr long long MERGE_BYTES = 96 << 10;

hipError_t launch_paged_attend(const PagedCall& a, hipStream_t s) {
  const int tile = a.D.dtype == LTRI_F32 ? 16 : 32, pairs = a.n * a.D.G;
  const int wb = pairs <= 16 ? 1 : pairs <= 32 ? 2 : 4, min_share = PA_WAVES / wb;
  // as many workgroups as the chip holds, or as the tables can have work for
  const long long tiles = (long long)a.seq_count * a.D.Hkv * ((a.D.cap_tokens + tile - 1) / tile + PAGED_EXTRA);
  const long long most = tiles * pair_blocks(a, 16 * wb);
  const int wgs = (int)std::min<long long>(std::min(a.n_cus * 2, PAGED_MAX_WGS), (most + min_share - 1) / min_share);
  // bytes of partial results of a problem, if its sequence is as long as the others
  const long long problems = (long long)a.seq_count * a.D.Hkv * pair_blocks(a, 16 * wb);
  const bool later = (wgs + problems - 1) / problems * std::min(pairs, 16 * wb) * a.D.d * 4 > MERGE_BYTES;
  if (a.D.dtype == LTRI_F32) launch_dim<LTRI_F32>(a, wb, wgs, min_share, later, s);
  else launch_dim<LTRI_BF16>(a, wb, wgs, min_share, later, s);
  if (a.decay < 0.f) return hipGetLastError();
  if (paged_keeps_scores(pairs)) {
    const long long pieces = (long long)a.seq_count * a.D.Hkv * ((a.D.cap_tokens + PW_TOKENS - 1) / PW_TOKENS);
    const int n = (int)std::min<long long>(a.n_cus * 8, pieces);
    if (tile == 16) paged_weights_kernel<16><<<n, WALK_T, 0, s>>>(a);
    else paged_weights_kernel<32><<<n, WALK_T, 0, s>>>(a);
  } else {
    const int n = (int)std::min<long long>(a.n_cus * 2, (tiles + PA_WAVES - 1) / PA_WAVES);
    if (a.D.dtype == LTRI_F32) launch_key_weights<LTRI_F32>(a, n, s);
    else launch_key_weights<LTRI_BF16>(a, n, s);
  }
  return hipGetLastError();
}

}  // namespace ltri
