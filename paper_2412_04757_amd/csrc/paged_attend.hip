// Attention over a key-value cache in pages: o = sum_j softmax_j(q.k_j / sqrt(d)) v_j over a sequence's tokens, one pass
// with a running maximum and sum; with weights every token's share p_j = exp(s_j - lse) is added up per KV head.
//
// One workgroup per (query row, head), four wavefronts that take every fourth token, a lane's share of the row in
// registers. Scores of every token go to scratch in the log2 domain, and a second launch turns them into weights.
#include "device_common.h"
#include "paged_internal.h"

namespace ltri {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Tiles of the sequences in front of s, and (whole batch) whether its scores fit the scratch.
__device__ __forceinline__ long long score_tiles_before(const PagedCall& a, int s) {
  __shared__ long long sum[4];
  long long n = 0;
  for (int i = threadIdx.x; i < s; i += 256) n += paged_tiles(paged_len(a, i));
  for (int m = 32; m; m >>= 1) n += __shfl_xor(n, m, 64);
  if ((threadIdx.x & 63) == 0) sum[threadIdx.x >> 6] = n;
  __syncthreads();
  n = sum[0] + sum[1] + sum[2] + sum[3];
  __syncthreads();
  return n;
}

template <int DT, int DIM>
__global__ __launch_bounds__(256) void paged_attend_kernel(PagedCall a) {
  typedef typename Elt<DT>::type T;
  constexpr int N = DIM / 64;
  const PagedDims& D = a.D;
  const int s = blockIdx.z, h = blockIdx.y, pair = blockIdx.x, row = pair / D.G, head = h * D.G + pair % D.G;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int len = paged_len(a, s), sees = max(len - a.n + 1 + row, 0);
  const long long before = a.decay >= 0.f ? score_tiles_before(a, s) : 0;
  const int nt = paged_tiles(len);
  float* scores = nullptr;
  if (a.decay >= 0.f && before + nt <= D.score_tiles)
    scores = a.scores + ((size_t)before * D.Hkv + (size_t)h * nt) * PAGED_TILE * (a.n * D.G) + (size_t)pair * nt * PAGED_TILE;
  const size_t orow = ((size_t)s * a.n + row) * D.Hq + head;
  float q[N], o[N], m = -INFINITY, l = 0.f;
  for (int e = 0; e < N; ++e) {
    q[e] = Elt<DT>::to_f32(((const T*)a.q)[orow * DIM + lane * N + e]);
    o[e] = 0.f;
  }
  const float sc = LOG2E / sqrtf((float)DIM);
  for (int j = wave; j < len; j += 4) {
    float x = -INFINITY;
    const int page = j < sees ? paged_page(a, s, j) : -1;
    if (page >= 0) {
      const long long at = paged_row(D, page, h, j) + lane * N;
      x = 0.f;
      for (int e = 0; e < N; ++e) x = fmaf(q[e], Elt<DT>::to_f32(((const T*)a.k)[at + e]), x);
      for (int b = 32; b; b >>= 1) x += __shfl_xor(x, b, 64);
      x *= sc;
      const float m_new = fmaxf(m, x), ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = exp2f(m - ref), p = exp2f(x - ref);
      l = l * alpha + p;
      for (int e = 0; e < N; ++e) o[e] = fmaf(p, Elt<DT>::to_f32(((const T*)a.v)[at + e]), o[e] * alpha);
      m = m_new;
    }
    if (scores && lane == 0) scores[j] = x;
  }
  __shared__ float s_o[4][DIM], s_m[4], s_l[4];
  for (int e = 0; e < N; ++e) s_o[wave][lane * N + e] = o[e];
  if (lane == 0) { s_m[wave] = m; s_l[wave] = l; }
  __syncthreads();
  const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3])), ref = top == -INFINITY ? 0.f : top;
  float total = 0.f, w[4];
  for (int i = 0; i < 4; ++i) { w[i] = exp2f(s_m[i] - ref); total += w[i] * s_l[i]; }
  for (int c = threadIdx.x; c < DIM; c += 256) {
    float x = 0.f;
    for (int i = 0; i < 4; ++i) x += w[i] * s_o[i][c];
    x = total == 0.f ? 0.f : x / total;
    if constexpr (DT == LTRI_F32) ((float*)a.out)[orow * DIM + c] = x;
    else ((__bf16*)a.out)[orow * DIM + c] = (__bf16)x;
  }
  if (threadIdx.x == 0) {
    const float lse2 = total == 0.f ? -INFINITY : top + log2f(total);
    a.lse2[orow] = lse2;
    if (a.lse) a.lse[orow] = lse2 * LN2;
  }
}

__global__ __launch_bounds__(256) void paged_weights_kernel(PagedCall a) {
  const PagedDims& D = a.D;
  const int s = blockIdx.z, h = blockIdx.y, pairs = a.n * D.G;
  const int len = paged_len(a, s), nt = paged_tiles(len);
  const long long before = score_tiles_before(a, s);
  if (before + nt > D.score_tiles) {
    atomicCAS(a.err, 0, LTRI_ECAPACITY);
    return;
  }
  const float* scores = a.scores + ((size_t)before * D.Hkv + (size_t)h * nt) * PAGED_TILE * pairs;
  for (int j = blockIdx.x * 256 + threadIdx.x; j < len; j += gridDim.x * 256) {
    const int page = paged_page(a, s, j);
    if (page < 0) continue;
    float got = 0.f;
    for (int pair = 0; pair < pairs; ++pair) {
      const float lse2 = a.lse2[((size_t)s * a.n + pair / D.G) * D.Hq + h * D.G + pair % D.G];
      if (lse2 != -INFINITY) got += exp2f(scores[(size_t)pair * nt * PAGED_TILE + j] - lse2);
    }
    float* w = a.weight + paged_mark(D, page, h, j);
    *w = a.decay == 0.f ? got : fmaf(a.decay, *w, got);
  }
}

template <int DT>
static void launch_dim(const PagedCall& a, dim3 grid, hipStream_t s) {
  if (a.D.d == 64) paged_attend_kernel<DT, 64><<<grid, 256, 0, s>>>(a);
  else paged_attend_kernel<DT, 128><<<grid, 256, 0, s>>>(a);
}

hipError_t launch_paged_attend(const PagedCall& a, hipStream_t s) {
  const dim3 grid(a.n * a.D.G, a.D.Hkv, a.seq_count);
  if (a.D.dtype == LTRI_F32) launch_dim<LTRI_F32>(a, grid, s);
  else launch_dim<LTRI_BF16>(a, grid, s);
  if (a.decay >= 0.f) paged_weights_kernel<<<dim3(16, a.D.Hkv, a.seq_count), 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ltri
