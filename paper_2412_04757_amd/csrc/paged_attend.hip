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

template <int DT> struct PagedTile { static constexpr int N = DT == LTRI_F32 ? 16 : 32; };       // tokens per tile

// Blocks of 16 pairs of a KV head.
__host__ __device__ __forceinline__ int pair_blocks(const PagedCall& a) { return (a.n * a.D.G + 15) / 16; }
__device__ __forceinline__ int tiles_of(int len, int tile) { return (len + tile - 1) / tile; }

// Scores of sequence s: [KV head][pair][tokens, padded to the tile], behind those of the sequences in front (`before` tiles); NULL: no room.
__device__ __forceinline__ float* score_rows(const PagedCall& a, long long before, int nt, int tile, int h) {
  if ((before + nt) * tile > a.D.score_tiles * PAGED_TILE) return nullptr;
  return a.scores + ((size_t)before * a.D.Hkv + (size_t)h * nt) * tile * (a.n * a.D.G);
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
__device__ __forceinline__ float safe_ref(float m) { return m == -INFINITY ? 0.f : m; }

// A wavefront's matrix products of one tile, by type. NU: groups of 16 tokens in a tile; VW: 32-bit words of a lane's piece of a value row.
template <int DT, int DIM> struct TileOps;

template <int DIM> struct TileOps<LTRI_BF16, DIM> {
  static constexpr int NU = 2, NK = DIM / 32, NT = DIM / 16, CP = NT, VW = CP / 2;
  uint4 q[NK], k[NU][NK];
  uint32_t v[NU][4][VW];
  f32x4_t o[NT];
  __device__ __forceinline__ void load_q(const char* row, int g, bool there) {
#pragma unroll
    for (int u = 0; u < NK; ++u) q[u] = there ? *(const uint4*)(row + u * 64 + g * 16) : make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void load_k(int u, const char* row, int g) {            // row: of token 16 u + lane % 16
#pragma unroll
    for (int i = 0; i < NK; ++i) k[u][i] = *(const uint4*)(row + i * 64 + g * 16);
  }
  __device__ __forceinline__ void store_k(int u, char* row, int g) const {
#pragma unroll
    for (int i = 0; i < NK; ++i) *(uint4*)(row + i * 64 + g * 16) = k[u][i];
  }
  __device__ __forceinline__ void load_v(int u, int j, const char* row, int kl) {    // row: of token 16 u + 4 (lane / 16) + j
    if constexpr (VW == 4) { const uint4 x = *(const uint4*)(row + kl * 16); v[u][j][0] = x.x; v[u][j][1] = x.y; v[u][j][2] = x.z; v[u][j][3] = x.w; }
    else { const uint2 x = *(const uint2*)(row + kl * 8); v[u][j][0] = x.x; v[u][j][1] = x.y; }
  }
  __device__ __forceinline__ void store_v(int u, int j, char* row, int kl) const {
    if constexpr (VW == 4) *(uint4*)(row + kl * 16) = make_uint4(v[u][j][0], v[u][j][1], v[u][j][2], v[u][j][3]);
    else *(uint2*)(row + kl * 8) = make_uint2(v[u][j][0], v[u][j][1]);
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
  // o += V^T P^T; vis: of the lane's tokens [u][j] (bit 4 u + j) those that count; takes: whether the lane's pair takes the sum
  __device__ __forceinline__ void values(const f32x4_t (&p)[NU], uint32_t vis = 0xFFu, bool takes = true) {
    uint4 hi, lo;
    uint32_t* ph = (uint32_t*)&hi;
    uint32_t* pl = (uint32_t*)&lo;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float x = p[u][2 * c], y = p[u][2 * c + 1];
        ph[2 * u + c] = pack2(x, y);
        pl[2 * u + c] = pack2(x - __uint_as_float(ph[2 * u + c] << 16), y - __uint_as_float(ph[2 * u + c] & 0xFFFF0000u));
      }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      uint4 col;
      uint32_t* pc = (uint32_t*)&col;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          pc[2 * u + c] = __builtin_amdgcn_perm(v[u][2 * c + 1][t / 2], v[u][2 * c][t / 2], t & 1 ? 0x07060302u : 0x05040100u);
          if (vis != 0xFFu) pc[2 * u + c] &= ((vis >> (4 * u + 2 * c)) & 1 ? 0xFFFFu : 0u) | ((vis >> (4 * u + 2 * c + 1)) & 1 ? 0xFFFF0000u : 0u);
        }
      const bf16x8_t A = __builtin_bit_cast(bf16x8_t, col);
      f32x4_t sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, __builtin_bit_cast(bf16x8_t, lo), o[t], 0, 0, 0);
      sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, __builtin_bit_cast(bf16x8_t, hi), sum, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[t][e] = takes ? sum[e] : o[t][e];
    }
  }
};

template <int DIM> struct TileOps<LTRI_F32, DIM> {
  static constexpr int NU = 1, NK = DIM / 16, NT = DIM / 16, CP = 4, VW = DIM / 16;
  f32x4_t q[NK], k[NU][NK];
  uint32_t v[NU][4][VW];
  f32x4_t o[NT];
  __device__ __forceinline__ void load_q(const char* row, int g, bool there) {
#pragma unroll
    for (int u = 0; u < NK; ++u) q[u] = there ? *(const f32x4_t*)(row + u * 64 + g * 16) : f32x4_t{0.f, 0.f, 0.f, 0.f};
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
      const uint4 x = *(const uint4*)(row + c * 256 + kl * 16);
      v[u][j][4 * c] = x.x; v[u][j][4 * c + 1] = x.y; v[u][j][4 * c + 2] = x.z; v[u][j][4 * c + 3] = x.w;
    }
  }
  __device__ __forceinline__ void store_v(int u, int j, char* row, int kl) const {
#pragma unroll
    for (int c = 0; c < VW / 4; ++c)
      *(uint4*)(row + c * 256 + kl * 16) = make_uint4(v[u][j][4 * c], v[u][j][4 * c + 1], v[u][j][4 * c + 2], v[u][j][4 * c + 3]);
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
  __device__ __forceinline__ void values(const f32x4_t (&p)[NU], uint32_t vis = 0xFFu, bool takes = true) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      f32x4_t sum = o[t];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        sum = __builtin_amdgcn_mfma_f32_16x16x4f32((vis >> j) & 1 ? __uint_as_float(v[0][j][t]) : 0.f, p[0][j], sum, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[t][e] = takes ? sum[e] : o[t][e];
    }
  }
};

// SMALL: pages of fewer than 16 tokens, whose page is looked up lane by lane; else a group of 16 tokens lies in one page.
template <int DT, int DIM, bool SMALL>
__global__ __launch_bounds__(64 * PA_WAVES, 2) void paged_attend_kernel(PagedCall a, int min_share) {
  typedef TileOps<DT, DIM> Ops;
  constexpr int T = PagedTile<DT>::N, NU = Ops::NU, NT = Ops::NT, CP = Ops::CP, ELT = DT == LTRI_F32 ? 4 : 2;
  constexpr int PITCH = DIM + 4;
  static_assert(NU * 16 == T && WALK_T == 64 * PA_WAVES, "");
  __shared__ __align__(16) float s_o[PA_WAVES][16][PITCH];
  __shared__ float s_m[PA_WAVES][16], s_l[PA_WAVES][16];
  __shared__ int s_last;
  const PagedDims& D = a.D;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kl = lane & 15, g = lane >> 4;
  const int w = blockIdx.x, pairs = a.n * D.G, blocks = pair_blocks(a), per_tile = D.Hkv * blocks;
  const int page_mask = (1 << D.page_shift) - 1;
  const long long tok_bytes = D.token_stride * ELT;
  const float sc = LOG2E / sqrtf((float)DIM);

  long long share = 0;
  const PagedPlace at = paged_find(a.seq_count, [&](int s) { return (long long)tiles_of(paged_len(a, s), T) * per_tile; },
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
    const long long mine = (long long)nt * per_tile;
    if (x >= before + mine) {                            // on to the next sequence
      before += mine;
      ++s;
      continue;
    }
    const int hp = (int)((x - before) / nt), h = hp / blocks, pb = hp % blocks;
    const long long problem = before + (long long)hp * nt;           // its first tile
    const int t0 = (int)(x - problem), t1 = (int)min((long long)nt, t0 + (x_end - x));
    x += t1 - t0;

    const int first_new = a.k_new ? max(len - a.n, 0) : len;         // tokens from here on come with the call
    const int pair = min(pb * 16 + kl, pairs - 1), np = min(16, pairs - pb * 16);
    const int sees = len - a.n + 1 + pair / D.G;                     // tokens that the lane's pair sees
    const int all_see = len - a.n + 1 + pb * 16 / D.G;               // ... that every pair of the block sees
    const int32_t* table = a.table + (size_t)s * D.table_pages;
    const char* kh = a.k + (size_t)h * D.head_stride * ELT;
    const char* vh = a.v + (size_t)h * D.head_stride * ELT;
    float* scores = nullptr;
    if (a.decay >= 0.f) {
      scores = score_rows(a, before / per_tile, nt, T, h);
      if (scores) scores += (size_t)(pb * 16 + kl) * nt * T;
    }

    Ops ops;
    ops.load_q((const char*)a.q + (((size_t)s * a.n + pair / D.G) * D.Hq + h * D.G + pair % D.G) * DIM * ELT, g, kl < np);
#pragma unroll
    for (int t = 0; t < NT; ++t) ops.o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    // Pages of a tile: of its groups of 16 tokens, or (SMALL) of the token that the lane loads of every group's keys and of its four
    // of the values. Past the sequence's end the last token's.
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
          p.k[u] = p.v[u][0] = table[min(i0, len - 1) >> D.page_shift];
        }
      }
    };
    auto good = [&](int page) { return (unsigned)page < (unsigned)D.n_pages; };
    auto row = [&](const char* base, int page, int i) __attribute__((always_inline)) {
      return base + ((long long)(good(page) ? page : 0) * D.page_stride * ELT + (long long)(i & page_mask) * tok_bytes);
    };
    // New tokens are read from the call's rows: their tiles take this way for every lane.
    auto new_row = [&](const void* rows, int i) { return (const char*)rows + (((size_t)s * D.Hkv + h) * a.n + (i - (len - a.n))) * DIM * ELT; };
    auto load_k = [&](int t, const Pages& p) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const int i0 = t * T + 16 * u;
        const char* at_row;
        if constexpr (SMALL) at_row = row(kh, p.k[u], min(i0 + kl, len - 1));
        else at_row = row(kh, __builtin_amdgcn_readfirstlane(p.k[u]), i0) + (uint32_t)(kl * (int)tok_bytes);
        if (i0 + 16 > first_new) {
          const int i = min(i0 + kl, len - 1);
          if (i >= first_new) at_row = new_row(a.k_new, i);
        }
        ops.load_k(u, at_row, g);
      }
    };
    auto load_v = [&](int t, const Pages& p) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const int i0 = t * T + 16 * u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const char* at_row;
          if constexpr (SMALL) at_row = row(vh, p.v[u][j], min(i0 + 4 * g + j, len - 1));
          else at_row = row(vh, __builtin_amdgcn_readfirstlane(p.v[u][0]), i0) + (uint32_t)((4 * g + j) * (int)tok_bytes);
          if (i0 + 16 > first_new) {
            const int i = min(i0 + 4 * g + j, len - 1);
            if (i >= first_new) at_row = new_row(a.v_new, i);
          }
          ops.load_v(u, j, at_row, kl);
        }
      }
    };

    Pages now, next;
    int t = t0 + wave;
    if (t < t1) {
      look_up(t, now);
      load_k(t, now);
      load_v(t, now);
      look_up(min(t + PA_WAVES, nt - 1), next);
    }
    for (; t < t1; t += PA_WAVES) {
      f32x4_t sv[NU];
      ops.scores(sv);
      const bool takes = (t + 1) * T > first_new;                    // the tile has new tokens (uniform)
      if (takes && pb == 0) {
#pragma unroll
        for (int u = 0; u < NU; ++u) {
          const int i = t * T + 16 * u + kl;
          const int page = i >= first_new && i < len ? paged_page(a, s, i) : -1;
          if (page < 0) continue;
          ops.store_k(u, const_cast<char*>(row(kh, page, i)), g);
          if (D.weights && g == 0) {
            const size_t mark = paged_mark(D, page, h, i);
            a.weight[mark] = 0.f;
            a.pos[mark] = a.seen[s] - (len - i);
          }
        }
      }
      const bool more = t + PA_WAVES < t1;
      if (more) load_k(t + PA_WAVES, next);

      // which of the lane's tokens 16 u + 4 g + j count for its pair, and which are there at all
      uint32_t vis = 0xFFu, there = 0xFFu;
      bool edge = (t + 1) * T > all_see;
      {
        bool bad = false;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < (SMALL ? 4 : 1); ++j) bad |= !good(now.v[u][j]);
        edge |= (bool)__any(bad);
      }
      if (edge) {
        vis = there = 0u;
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = t * T + 16 * u + 4 * g + j;
            const bool ok = i < len && good(now.v[u][SMALL ? j : 0]);
            if (i < len && !ok) atomicCAS(a.err, 0, LTRI_EINVAL);
            there |= (uint32_t)ok << (4 * u + j);
            vis |= (uint32_t)(ok && i < sees) << (4 * u + j);
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sv[u][j] = (vis >> (4 * u + j)) & 1 ? sv[u][j] * sc : -INFINITY;
          mx = fmaxf(mx, sv[u][j]);
        }
      if (scores && kl < np) {
#pragma unroll
        for (int u = 0; u < NU; ++u) *(f32x4_t*)(scores + (size_t)t * T + 16 * u + 4 * g) = sv[u];
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
      if (takes && pb == 0) {
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = t * T + 16 * u + 4 * g + j;
            const int page = i >= first_new && i < len ? now.v[u][SMALL ? j : 0] : -1;
            if (good(page)) ops.store_v(u, j, const_cast<char*>(row(vh, page, i)), kl);
          }
      }
      bool apart = false;                        // an infinity or NaN in a token that some pair of the block does not see
      if (edge) {
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (!((there >> (4 * u + j)) & 1)) ops.zero_v(u, j);
            else if (t * T + 16 * u + 4 * g + j >= all_see) apart |= ops.odd_v(u, j);
          }
        apart = (bool)__any(apart);
      }
      if (!apart) {
        ops.values(sv);
      } else {
        // query row by query row, which takes the tokens it sees (0 times infinity would not be 0)
        const int r0 = pb * 16 / D.G, r1 = (pb * 16 + np - 1) / D.G;
        for (int r = r0; r <= r1; ++r) {
          uint32_t seen_bits = 0u;
#pragma unroll
          for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) seen_bits |= (uint32_t)(t * T + 16 * u + 4 * g + j < len - a.n + 1 + r) << (4 * u + j);
          ops.values(sv, seen_bits, pair / D.G == r);
        }
      }
      if (more) load_v(t + PA_WAVES, next);
      now = next;
      look_up(min(t + 2 * PA_WAVES, nt - 1), next);
    }

    // the four wavefronts' results: own maximum, sum and O
    l = over_quarters(l);
    __syncthreads();                             // (the problem before has been read)
    if (kl < np) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int c = 0; c < NT; c += 4) {
          const int col = 16 * CP * (c / CP) + CP * (4 * g + j) + c % CP;
          *(f32x4_t*)&s_o[wave][kl][col] = f32x4_t{ops.o[c][j], ops.o[c + 1][j], ops.o[c + 2][j], ops.o[c + 3][j]};
        }
      if (g == 0) { s_m[wave][kl] = m; s_l[wave][kl] = l; }
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == nt;
    const size_t slot = 2 * (size_t)w + (t0 == 0);
    for (int i = tid; i < np * (DIM / 4); i += WALK_T) {
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
      if (whole) {
        const int pr = pb * 16 + p;
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
      } else {                                   // device scope (see wait_for_own_stores)
        unsigned long long* to = (unsigned long long*)(a.part + (slot * 16 + p) * DIM + c);
        __hip_atomic_store(to, ((unsigned long long)__float_as_uint(o[1]) << 32) | __float_as_uint(o[0]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(to + 1, ((unsigned long long)__float_as_uint(o[3]) << 32) | __float_as_uint(o[2]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (c == 0)
          __hip_atomic_store(a.part_ml + slot * 16 + p, ((unsigned long long)__float_as_uint(sum) << 32) | __float_as_uint(top), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    if (whole) continue;
    const long long w0 = problem / share, w1 = (problem + nt - 1) / share;       // the workgroups that share the problem
    wait_for_own_stores();
    __syncthreads();
    int32_t* ticket = a.tickets + ((size_t)s * D.Hkv + h) * blocks + pb;
    if (tid == 0) s_last = atomicAdd(ticket, 1) == (int)(w1 - w0);
    __syncthreads();
    if (!s_last) continue;
    if (tid == 0) *ticket = 0;
    auto slot_of_part = [&](long long i) { return 2 * (size_t)i + (i == w0); };
    for (int i = tid; i < np * (DIM / 2); i += WALK_T) {
      const int p = i / (DIM / 2), c = i % (DIM / 2) * 2;
      float top = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
      for (long long k = w0; k <= w1; ++k) {
        const unsigned long long ml = __hip_atomic_load(a.part_ml + slot_of_part(k) * 16 + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const unsigned long long oo = __hip_atomic_load((const unsigned long long*)(a.part + (slot_of_part(k) * 16 + p) * DIM + c), __ATOMIC_RELAXED,
                                                        __HIP_MEMORY_SCOPE_AGENT);
        const float mk = __uint_as_float((uint32_t)ml), top_new = fmaxf(top, mk), ref = safe_ref(top_new);
        const float ea = __builtin_amdgcn_exp2f(top - ref), eb = __builtin_amdgcn_exp2f(mk - ref);
        sum = sum * ea + eb * __uint_as_float((uint32_t)(ml >> 32));
        o0 = o0 * ea + eb * __uint_as_float((uint32_t)oo);
        o1 = o1 * ea + eb * __uint_as_float((uint32_t)(oo >> 32));
        top = top_new;
      }
      const int pr = pb * 16 + p;
      const size_t r = ((size_t)s * a.n + pr / D.G) * D.Hq + h * D.G + pr % D.G;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      if (sum == 0.f) o0 = o1 = 0.f;
      if constexpr (DT == LTRI_F32) *(float2*)((float*)a.out + r * DIM + c) = make_float2(o0 * inv, o1 * inv);
      else *(uint32_t*)((uint16_t*)a.out + r * DIM + c) = pack2(o0 * inv, o1 * inv);
      if (c == 0) {
        const float lse2 = sum == 0.f ? -INFINITY : top + log2f(sum);
        a.lse2[r] = lse2;
        if (a.lse) a.lse[r] = lse2 * LN2;
      }
    }
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
  // tiles of scores in front of the sequence
  long long tiles = paged_find(a.seq_count, [&](int s) { return s < at.seq ? (long long)tiles_of(paged_len(a, s), TILE) : 0; },
                               [&](long long) { return -1ll; }).total;
  int s = at.seq;
  while (x < x_end) {
    const int len = paged_len(a, s), nt = tiles_of(len, TILE), np = pieces(len);
    if (x >= before + (long long)np * D.Hkv) {
      before += (long long)np * D.Hkv;
      tiles += nt;
      ++s;
      continue;
    }
    const int h = (int)((x - before) / np), piece = (int)((x - before) % np);
    ++x;
    const float* scores = score_rows(a, tiles, nt, TILE, h);
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

template <int DT, int DIM>
static void launch_pages(const PagedCall& a, int wgs, int min_share, hipStream_t s) {
  if (a.D.page_shift < 4) paged_attend_kernel<DT, DIM, true><<<wgs, 64 * PA_WAVES, 0, s>>>(a, min_share);
  else paged_attend_kernel<DT, DIM, false><<<wgs, 64 * PA_WAVES, 0, s>>>(a, min_share);
}

hipError_t launch_paged_attend(const PagedCall& a, hipStream_t s) {
  const int tile = a.D.dtype == LTRI_F32 ? 16 : 32, min_share = PA_WAVES;
  // as many workgroups as the chip holds, or as the tables can have work for
  const long long most = (long long)a.seq_count * a.D.Hkv * pair_blocks(a) * ((a.D.cap_tokens + tile - 1) / tile);
  const int wgs = (int)std::min<long long>(std::min(a.n_cus * 2, PAGED_MAX_WGS), (most + min_share - 1) / min_share);
  if (a.D.dtype == LTRI_F32) {
    if (a.D.d == 64) launch_pages<LTRI_F32, 64>(a, wgs, min_share, s);
    else launch_pages<LTRI_F32, 128>(a, wgs, min_share, s);
  } else {
    if (a.D.d == 64) launch_pages<LTRI_BF16, 64>(a, wgs, min_share, s);
    else launch_pages<LTRI_BF16, 128>(a, wgs, min_share, s);
  }
  if (a.decay >= 0.f) {
    const long long pieces = (long long)a.seq_count * a.D.Hkv * ((a.D.cap_tokens + PW_TOKENS - 1) / PW_TOKENS);
    const int n = (int)std::min<long long>(a.n_cus * 4, pieces);
    if (tile == 16) paged_weights_kernel<16><<<n, WALK_T, 0, s>>>(a);
    else paged_weights_kernel<32><<<n, WALK_T, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace ltri
