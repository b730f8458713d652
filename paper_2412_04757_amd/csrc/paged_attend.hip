// Attention over a key-value cache in pages: o = sum_j softmax_j(q.k_j / sqrt(d)) v_j over a sequence's tokens, one pass
// with a running maximum and sum; with weights every token's share p_j = exp(s_j - lse) is added up per KV head.
//
// What bounds it: the key and value rows, each read once (512 bytes of bf16 rows and 4 G n products of 128 a token and KV head).
// So nothing is staged: a lane loads 16-byte pieces in the order in which the matrix cores take them, and while a tile of 32
// tokens (fp32: 16) is used, the next one's rows come into the registers as they fall free; three wavefronts a SIMD hide the rest.
//   S^T = K Q^T    A = 16 tokens (lane % 16) x head_dim pieces (lane / 16), B = 16 (query row, head) pairs: a lane gets tokens
//                  4 (lane / 16) + j, j < 4, of pair lane % 16. All query rows and heads of a KV head share the rows that way.
//   O^T = V^T P^T  A = V^T: lane % 16 stands for the CP columns whose piece of a row the lane has loaded, and one product per
//                  column of a piece takes that column of its tokens 4 (lane / 16) + j: in bf16 byte permutes inside the
//                  lane, no transposition. B = P^T is what the first product left in the lane. O^T and the running maximum have the pair in
//                  lane % 16 both, so a rescale needs no exchange either.
// bf16 probabilities enter as p = hi + lo, two bf16 parts (the matrix cores are idle otherwise): the result is off by its own
// rounding only. fp32 runs the fp32 matrix cores.
// The tiles of all sequences, KV heads and blocks of 16 pairs lie in one row, of which every workgroup takes an even share, whatever
// the lengths (paged_walk.h); its four wavefronts take every fourth tile and merge in LDS. Where a problem's tiles lie in several shares,
// the workgroup that finishes last (a ticket) adds the partial results up in order, so results do not depend on who that was.
#include <algorithm>

#include "device_common.h"
#include "paged_internal.h"
#include "paged_walk.h"

namespace ltri {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int PA_WAVES = 4;
// Workgroups of a compute unit, by registers (their tiles and results: 112 at head_dim 128 with one block of pairs, 160 with two).
constexpr int paged_occupancy(int dim, int blocks) { return dim == 128 && blocks == 2 ? 1 : 2; }
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

template <int DT> struct PagedTile { static constexpr int N = DT == LTRI_F32 ? 16 : 32; };       // tokens per tile

// A KV head's problems: blocks of `size` pairs.
__host__ __device__ __forceinline__ int pair_blocks(const PagedCall& a, int size) { return (a.n * a.D.G + size - 1) / size; }
__device__ __forceinline__ int tiles_of(int len, int tile) { return (len + tile - 1) / tile; }
// What a problem counts as when work is shared out: its tiles and PAGED_EXTRA, which its beginning and end cost.
__device__ __forceinline__ int units_of(int len, int tile) { return len ? tiles_of(len, tile) + PAGED_EXTRA : 0; }

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
__device__ __forceinline__ unsigned long long two_floats(float x, float y) { return ((unsigned long long)__float_as_uint(y) << 32) | __float_as_uint(x); }
__device__ __forceinline__ float first_float(unsigned long long v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float second_float(unsigned long long v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ float safe_ref(float m) { return m == -INFINITY ? 0.f : m; }

// A wavefront's matrix products of one tile, by type. NU: groups of 16 tokens in a tile; VW: 32-bit words of a lane's piece of a value row.
// NB: blocks of 16 pairs that share a tile's rows.
template <int DT, int DIM, int NB> struct TileOps;

template <int DIM, int NB> struct TileOps<LTRI_BF16, DIM, NB> {
  static constexpr int NU = 2, NK = DIM / 32, NT = DIM / 16, CP = NT, VW = CP / 2;
  u32x4_t q[NB][NK], k[NU][NK];
  uint32_t v[NU][4][VW];
  f32x4_t o[NB][NT];
  __device__ __forceinline__ void load_q(int b, const char* row, int g, bool there) {
#pragma unroll
    for (int i = 0; i < NK; ++i) q[b][i] = there ? *(const u32x4_t*)(row + i * 64 + g * 16) : u32x4_t{0u, 0u, 0u, 0u};
  }
  __device__ __forceinline__ void load_k(int u, const char* row, int g) {            // row: of token 16 u + lane % 16
#pragma unroll
    for (int i = 0; i < NK; ++i) k[u][i] = *(const u32x4_t*)(row + i * 64 + g * 16);
  }
  __device__ __forceinline__ void store_k(int u, char* row, int g) const {
#pragma unroll
    for (int i = 0; i < NK; ++i) *(u32x4_t*)(row + i * 64 + g * 16) = k[u][i];
  }
  __device__ __forceinline__ void load_v(int u, int j, const char* row, int kl) {    // row: of token 16 u + 4 (lane / 16) + j
    if constexpr (VW == 4) { const u32x4_t x = *(const u32x4_t*)(row + kl * 16); v[u][j][0] = x[0]; v[u][j][1] = x[1]; v[u][j][2] = x[2]; v[u][j][3] = x[3]; }
    else { const u32x2_t x = *(const u32x2_t*)(row + kl * 8); v[u][j][0] = x[0]; v[u][j][1] = x[1]; }
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
  __device__ __forceinline__ void scores(f32x4_t (&s)[NB][NU]) const {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        s[b][u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NK; ++i)
          s[b][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k[u][i]), __builtin_bit_cast(bf16x8_t, q[b][i]), s[b][u], 0, 0, 0);
      }
  }
  // o += V^T P^T. APART: only the lane's tokens [u][j] whose bit 4 u + j of vis is set count, and only the pairs of lanes with mine[b] take the sum.
  template <bool APART>
  __device__ __forceinline__ void values(const f32x4_t (&p)[NB][NU], uint32_t vis, const bool (&mine)[NB]) {
    u32x4_t hi[NB], lo[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float x = p[b][u][2 * c], y = p[b][u][2 * c + 1];
          const uint32_t h = pack2(x, y);
          hi[b][2 * u + c] = h;
          lo[b][2 * u + c] = pack2(x - __uint_as_float(h << 16), y - __uint_as_float(h & 0xFFFF0000u));
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
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x4_t sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, __builtin_bit_cast(bf16x8_t, lo[b]), o[b][t], 0, 0, 0);
        sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, __builtin_bit_cast(bf16x8_t, hi[b]), sum, 0, 0, 0);
        if constexpr (APART) {
#pragma unroll
          for (int e = 0; e < 4; ++e) o[b][t][e] = mine[b] ? sum[e] : o[b][t][e];
        } else {
          o[b][t] = sum;
        }
      }
    }
  }
};

template <int DIM, int NB> struct TileOps<LTRI_F32, DIM, NB> {
  static constexpr int NU = 1, NK = DIM / 16, NT = DIM / 16, CP = 4, VW = DIM / 16;
  f32x4_t q[NB][NK], k[NU][NK];
  uint32_t v[NU][4][VW];
  f32x4_t o[NB][NT];
  __device__ __forceinline__ void load_q(int b, const char* row, int g, bool there) {
#pragma unroll
    for (int i = 0; i < NK; ++i) q[b][i] = there ? *(const f32x4_t*)(row + i * 64 + g * 16) : f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void load_k(int u, const char* row, int g) {
#pragma unroll
    for (int i = 0; i < NK; ++i) k[u][i] = *(const f32x4_t*)(row + i * 64 + g * 16);
  }
  __device__ __forceinline__ void store_k(int u, char* row, int g) const {
#pragma unroll
    for (int i = 0; i < NK; ++i) *(f32x4_t*)(row + i * 64 + g * 16) = k[u][i];
  }
  __device__ __forceinline__ void load_v(int u, int j, const char* row, int kl) {
#pragma unroll
    for (int c = 0; c < VW / 4; ++c) {
      const u32x4_t x = *(const u32x4_t*)(row + c * 256 + kl * 16);
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
  __device__ __forceinline__ void scores(f32x4_t (&s)[NB][NU]) const {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      s[b][0] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[b][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[0][i][e], q[b][i][e], s[b][0], 0, 0, 0);
    }
  }
  template <bool APART>
  __device__ __forceinline__ void values(const f32x4_t (&p)[NB][NU], uint32_t vis, const bool (&mine)[NB]) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        f32x4_t sum = o[b][t];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          sum = __builtin_amdgcn_mfma_f32_16x16x4f32(!APART || ((vis >> j) & 1) ? __uint_as_float(v[0][j][t]) : 0.f, p[b][0][j], sum, 0, 0, 0);
        if constexpr (APART) {
#pragma unroll
          for (int e = 0; e < 4; ++e) o[b][t][e] = mine[b] ? sum[e] : o[b][t][e];
        } else {
          o[b][t] = sum;
        }
      }
  }
};

// SMALL: pages of fewer than 16 tokens, whose page is looked up lane by lane; else a group of 16 tokens lies in one page.
template <int DT, int DIM, int NB, bool SMALL>
__global__ __launch_bounds__(64 * PA_WAVES, paged_occupancy(DIM, NB)) void paged_attend_kernel(PagedCall a, int min_share) {
  typedef TileOps<DT, DIM, NB> Ops;
  constexpr int T = PagedTile<DT>::N, NU = Ops::NU, NT = Ops::NT, CP = Ops::CP, ELT = DT == LTRI_F32 ? 4 : 2;
  constexpr int PITCH = DIM + 4;
  static_assert(NU * 16 == T && WALK_T == 64 * PA_WAVES, "");
  constexpr int PB = 16 * NB;                    // pairs of a problem
  __shared__ __align__(16) float s_o[PA_WAVES][PB][PITCH];
  __shared__ float s_m[PA_WAVES][PB], s_l[PA_WAVES][PB];
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
                                     share = max((total + gridDim.x - 1) / gridDim.x, (long long)min_share);
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
    const int all_see = len - a.n + 1 + pb * PB / D.G;               // tokens that every pair of the block sees
    // tiles from here on: some token is not seen by some pair, or comes with the call (SMALL: every tile takes that way)
    const int first_edge = SMALL ? t0 : max(0, min(all_see, first_new)) / T;
    const int32_t* table = a.table + (size_t)s * D.table_pages;
    const char* kh = a.k + (size_t)h * D.head_stride * ELT;
    const char* vh = a.v + (size_t)h * D.head_stride * ELT;
    float* scores = nullptr;
    if (a.decay >= 0.f) {
      scores = score_rows(a, before / per_tile, nt, T, h);
      if (scores) scores += (size_t)(pb * PB + kl) * nt * T + 4 * g;
    }

    Ops ops;
    float m[NB], l[NB];
    int row_of[NB];                                                  // query rows of the lane's pairs
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int pair = min(pb * PB + 16 * b + kl, pairs - 1);
      row_of[b] = pair / D.G;
      ops.load_q(b, (const char*)a.q + (((size_t)s * a.n + row_of[b]) * D.Hq + h * D.G + pair % D.G) * DIM * ELT, g, 16 * b + kl < np);
#pragma unroll
      for (int t = 0; t < NT; ++t) ops.o[b][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      m[b] = -INFINITY;
      l[b] = 0.f;
    }

    // Pages of a tile: of its groups of 16 tokens, by scalar loads (the table does not change while a launch runs), or (SMALL) of the token that
    // the lane loads of every group's keys and of its four of the values. Past the sequence's end the last token's. They are asked for before the
    // rows of the tile in front, so that the loads, which come back in order, need not be waited for to have them.
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
    auto load_k = [&](int t, const Pages& p) __attribute__((always_inline)) {
      if (t >= first_edge) {
        const int kl_ = only_here(kl), g_ = only_here(g);
#pragma unroll
        for (int u = 0; u < NU; ++u) ops.load_k(u, edge_row(kh, a.k_new, p.k[u], t * T + 16 * u + kl_), g_);
      } else {
#pragma unroll
        for (int u = 0; u < NU; ++u) ops.load_k(u, row(kh, p.k[u], t * T + 16 * u) + k_off, 0);
      }
    };
    auto load_v = [&](int t, const Pages& p) __attribute__((always_inline)) {
      if (t >= first_edge) {
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
    // One tile; EDGE: see first_edge.
    auto tile = [&](int t, auto edge_c) __attribute__((always_inline)) {
      constexpr bool EDGE = decltype(edge_c)::value;
      f32x4_t sv[NB][NU];
      const int kl_ = EDGE ? only_here(kl) : kl, g_ = EDGE ? only_here(g) : g;
      ops.scores(sv);
      if constexpr (EDGE) {
        if (pb == 0 && a.k_new) {
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
      }
      const bool more = t + PA_WAVES < t1;
      Pages after;
      look_up(min(t + 2 * PA_WAVES, nt - 1), after);
      if (more) load_k(t + PA_WAVES, next);
      __builtin_amdgcn_sched_barrier(0);

      // of the lane's tokens 16 u + 4 g + j (bit 4 u + j): which are there at all, and which block b's pair sees
      uint32_t there = 0xFFu, vis[NB];
      if constexpr (EDGE) {
        there = 0u;
#pragma unroll
        for (int b = 0; b < NB; ++b) vis[b] = 0u;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = t * T + 16 * u + 4 * g_ + j;
            const bool ok = i < len && good(now.v[u][SMALL ? j : 0]);
            if (i < len && !ok) atomicCAS(a.err, 0, LTRI_EINVAL);
            there |= (uint32_t)ok << (4 * u + j);
#pragma unroll
            for (int b = 0; b < NB; ++b) vis[b] |= (uint32_t)(ok && i < len - a.n + 1 + row_of[b]) << (4 * u + j);
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
#pragma unroll
              for (int b = 0; b < NB; ++b) sv[b][u] = f32x4_t{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            }
        }
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float mx = -INFINITY;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            sv[b][u][j] *= sc;
            if constexpr (EDGE) sv[b][u][j] = (vis[b] >> (4 * u + j)) & 1 ? sv[b][u][j] : -INFINITY;
            mx = fmaxf(mx, sv[b][u][j]);
          }
        if (scores && 16 * b + kl < np) {
#pragma unroll
          for (int u = 0; u < NU; ++u) *(f32x4_t*)(scores + (size_t)(16 * b * nt + t) * T + 16 * u) = sv[b][u];
        }
        const float m_new = fmaxf(m[b], max_quarters(mx)), ref = safe_ref(m_new);
        if (__any(m_new > m[b])) {                                   // rare after the first tiles
          const float alpha = __builtin_amdgcn_exp2f(m[b] - ref);
          l[b] *= alpha;
#pragma unroll
          for (int c = 0; c < NT; ++c) ops.o[b][c] *= alpha;
          m[b] = m_new;
        }
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            sv[b][u][j] = __builtin_amdgcn_exp2f(sv[b][u][j] - ref);
            l[b] += sv[b][u][j];
          }
      }
      bool mine[NB];
      bool apart = false;                        // an infinity or NaN in a token that some pair of the block does not see
      if constexpr (EDGE) {
        if (pb == 0 && a.k_new) {
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
          const int r0 = pb * PB / D.G, r1 = (pb * PB + np - 1) / D.G;
          for (int r = r0; r <= r1; ++r) {
            uint32_t seen_bits = 0u;
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
              for (int j = 0; j < 4; ++j) seen_bits |= (uint32_t)(t * T + 16 * u + 4 * g_ + j < len - a.n + 1 + r) << (4 * u + j);
#pragma unroll
            for (int b = 0; b < NB; ++b) mine[b] = row_of[b] == r;
            ops.template values<true>(sv, seen_bits, mine);
          }
        }
      }
      if (!apart) ops.template values<false>(sv, 0u, mine);
      __builtin_amdgcn_sched_barrier(0);
      if (more) load_v(t + PA_WAVES, next);
      __builtin_amdgcn_sched_barrier(0);
      now = next;
      next = after;
    };
    int t = t0 + wave;
    if (t < t1) {
      look_up(t, now);
      look_up(min(t + PA_WAVES, nt - 1), next);
      load_k(t, now);
      __builtin_amdgcn_sched_barrier(0);                             // keys before values, as in the loop: what is waited for first comes first
      load_v(t, now);
      __builtin_amdgcn_sched_barrier(0);
    }
    for (; t < min(t1, first_edge); t += PA_WAVES) tile(t, std::false_type{});
    for (; t < t1; t += PA_WAVES) tile(t, std::true_type{});

    // the four wavefronts' results: own maximum, sum and O
    __syncthreads();                             // (the problem before has been read)
    const int tid_ = only_here(tid), lane_ = tid_ & 63, kl_ = lane_ & 15, g_ = lane_ >> 4;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int p = 16 * b + kl_;
      l[b] = over_quarters(l[b]);
      if (p >= np) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int c = 0; c < NT; c += 4) {
          const int col = 16 * CP * (c / CP) + CP * (4 * g_ + j) + c % CP;
          *(f32x4_t*)&s_o[wave][p][col] = f32x4_t{ops.o[b][c][j], ops.o[b][c + 1][j], ops.o[b][c + 2][j], ops.o[b][c + 3][j]};
        }
      if (g_ == 0) { s_m[wave][p] = m[b]; s_l[wave][p] = l[b]; }
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == nt;
    const size_t slot = 2 * (size_t)w + (t0 == 0);
    // adds the four up, by threads that each take four columns of a pair, and hands (pair, column, O, maximum, sum) on
    auto join = [&](auto take) __attribute__((always_inline)) {
      for (int i = tid_; i < np * (DIM / 4); i += WALK_T) {
        const int p = i / (DIM / 4), c = i % (DIM / 4) * 4;
        float top = s_m[0][p];
#pragma unroll
        for (int k = 1; k < PA_WAVES; ++k) top = fmaxf(top, s_m[k][p]);
        const float ref = safe_ref(top);
        float sum = 0.f;
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < PA_WAVES; ++k) {
          const float e = __builtin_amdgcn_exp2f(s_m[k][p] - ref);
          sum = fmaf(e, s_l[k][p], sum);
          o += e * *(const f32x4_t*)&s_o[k][p][c];
        }
        take(p, c, o, top, sum);
      }
    };
    auto result = [&](int p, int c, f32x4_t o, float top, float sum) __attribute__((always_inline)) {
      const int pr = pb * PB + p;
      const size_t r = ((size_t)s * a.n + pr / D.G) * D.Hq + h * D.G + pr % D.G;
      if (sum == 0.f) o = f32x4_t{0.f, 0.f, 0.f, 0.f};
      else o *= 1.f / sum;
      if constexpr (DT == LTRI_F32) *(f32x4_t*)((float*)a.out + r * DIM + c) = o;
      else *(uint2*)((uint16_t*)a.out + r * DIM + c) = make_uint2(pack2(o[0], o[1]), pack2(o[2], o[3]));
      if (c == 0) {
        const float lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
        a.lse2[r] = lse2;
        if (a.lse) a.lse[r] = lse2 * LN2;
      }
    };
    if (whole) {
      join(result);
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
    // the parts, every fourth by one wavefront, DEEP in flight; then the four wavefronts' sums as above
    constexpr int DEEP = 8;
    for (int i = lane_; i < np * (DIM / 4); i += 64) {
      const int p = i / (DIM / 4), c = i % (DIM / 4) * 4;
      float top = -INFINITY, sum = 0.f;
      f32x4_t o = {0.f, 0.f, 0.f, 0.f};
      for (int k0 = wave; k0 < parts; k0 += PA_WAVES * DEEP) {
        unsigned long long ml[DEEP], lo[DEEP], hi[DEEP];
#pragma unroll
        for (int u = 0; u < DEEP; ++u) {
          const int k = min(k0 + PA_WAVES * u, parts - 1);
          const size_t at_part = (2 * (size_t)(w0 + k) + (k == 0)) * PB + p;
          const unsigned long long* from = (const unsigned long long*)(a.part + at_part * DIM + c);
          ml[u] = __hip_atomic_load(a.part_ml + at_part, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          lo[u] = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          hi[u] = __hip_atomic_load(from + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
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
          if (k0 + PA_WAVES * u >= parts) continue;
          const float e = __builtin_amdgcn_exp2f(first_float(ml[u]) - ref);
          sum = fmaf(e, second_float(ml[u]), sum);
          o += e * f32x4_t{first_float(lo[u]), second_float(lo[u]), first_float(hi[u]), second_float(hi[u])};
        }
      }
      *(f32x4_t*)&s_o[wave][p][c] = o;
      if (c == 0) { s_m[wave][p] = top; s_l[wave][p] = sum; }
    }
    __syncthreads();
    join(result);
  }
}

// Weights from the scores: w <- decay w + sum over the KV head's pairs of exp(s - lse). A thread takes four tokens of a KV head;
// pieces of 1024 tokens are shared out like the tiles above.
constexpr int PW_TOKENS = 4 * WALK_T;
template <int TILE>
__global__ __launch_bounds__(WALK_T) void paged_weights_kernel(PagedCall a) {
  const PagedDims& D = a.D;
  const int pairs = a.n * D.G, w = blockIdx.x;
  auto pieces = [&](int len) { return (len + PW_TOKENS - 1) / PW_TOKENS; };
  long long share = 0;
  const PagedPlace at = paged_find(a.seq_count, [&](int s) { return (long long)pieces(paged_len(a, s)) * D.Hkv; },
                                   [&](long long total) { share = (total + gridDim.x - 1) / gridDim.x; return share * w; });
  if (at.seq < 0) return;
  __shared__ float s_lse[LTRI_PAGED_MAX_ROWS * 128];
  long long x = share * w, x_end = min(x + share, at.total), before = at.before;
  // units in front of the sequence
  long long units = paged_find(a.seq_count, [&](int s) { return s < at.seq ? (long long)units_of(paged_len(a, s), TILE) : 0; },
                               [&](long long) { return -1ll; }).total;
  int s = at.seq;
  while (x < x_end) {
    const int len = paged_len(a, s), nt = tiles_of(len, TILE), np = pieces(len);
    if (x >= before + (long long)np * D.Hkv) {
      before += (long long)np * D.Hkv;
      units += units_of(len, TILE);
      ++s;
      continue;
    }
    const int h = (int)((x - before) / np), piece = (int)((x - before) % np);
    ++x;
    const float* scores = score_rows(a, units, nt, TILE, h);
    if (!scores) {
      if (threadIdx.x == 0) atomicCAS(a.err, 0, LTRI_ECAPACITY);
      continue;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < pairs; p += WALK_T) s_lse[p] = a.lse2[((size_t)s * a.n + p / D.G) * D.Hq + h * D.G + p % D.G];
    __syncthreads();
    const int i0 = piece * PW_TOKENS + 4 * threadIdx.x;
    f32x4_t got = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < pairs && i0 < len; ++p) {
      const float lse2 = s_lse[p];
      const f32x4_t v = *(const f32x4_t*)(scores + (size_t)p * nt * TILE + i0);
      if (lse2 != -INFINITY) {
#pragma unroll
        for (int j = 0; j < 4; ++j) got[j] += __builtin_amdgcn_exp2f(v[j] - lse2);
      }
    }
    for (int j = 0; j < min(4, len - i0); ++j) {
      const int page = paged_page(a, s, i0 + j);
      if (page < 0) continue;
      float* to = a.weight + paged_mark(D, page, h, i0 + j);
      *to = a.decay == 0.f ? got[j] : fmaf(a.decay, *to, got[j]);
    }
  }
}

template <int DT, int DIM, int NB>
static void launch_pages(const PagedCall& a, int wgs, int min_share, hipStream_t s) {
  if (a.D.page_shift < 4) paged_attend_kernel<DT, DIM, NB, true><<<wgs, 64 * PA_WAVES, 0, s>>>(a, min_share);
  else paged_attend_kernel<DT, DIM, NB, false><<<wgs, 64 * PA_WAVES, 0, s>>>(a, min_share);
}
template <int DT>
static void launch_tiles(const PagedCall& a, bool two, int wgs, int min_share, hipStream_t s) {
  if (a.D.d == 64) two ? launch_pages<DT, 64, 2>(a, wgs, min_share, s) : launch_pages<DT, 64, 1>(a, wgs, min_share, s);
  else two ? launch_pages<DT, 128, 2>(a, wgs, min_share, s) : launch_pages<DT, 128, 1>(a, wgs, min_share, s);
}

hipError_t launch_paged_attend(const PagedCall& a, hipStream_t s) {
  const int tile = a.D.dtype == LTRI_F32 ? 16 : 32, min_share = PA_WAVES;
  const bool two = a.n * a.D.G > 16;             // two blocks of pairs share the rows of a tile
  // as many workgroups as the chip holds, or as the tables can have work for
  const long long most = (long long)a.seq_count * a.D.Hkv * pair_blocks(a, two ? 32 : 16) * ((a.D.cap_tokens + tile - 1) / tile + PAGED_EXTRA);
  const int wgs = (int)std::min<long long>(std::min(a.n_cus * paged_occupancy(a.D.d, two ? 2 : 1), PAGED_MAX_WGS), (most + min_share - 1) / min_share);
  if (a.D.dtype == LTRI_F32) launch_tiles<LTRI_F32>(a, two, wgs, min_share, s);
  else launch_tiles<LTRI_BF16>(a, two, wgs, min_share, s);
  if (a.decay >= 0.f) {
    const long long pieces = (long long)a.seq_count * a.D.Hkv * ((a.D.cap_tokens + PW_TOKENS - 1) / PW_TOKENS);
    const int n = (int)std::min<long long>(a.n_cus * 4, pieces);
    if (tile == 16) paged_weights_kernel<16><<<n, WALK_T, 0, s>>>(a);
    else paged_weights_kernel<32><<<n, WALK_T, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace ltri
