// Declarations shared by the host side and the kernels of the paged cache (ltri_paged.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>
#include "ltri_paged.h"

namespace ltri {

constexpr int PAGED_TILE = 32;             // rows of scores are padded to at most this many tokens
// Tiles that the beginning and end of a (sequence, KV head, block of pairs) are as long as. 256 sequences of up to 2000 tokens, us:
// 2: 144, 4: 121, 8: 114, 14: 121; 64 of up to 4096: 72, 67, 67, 68; even batches do not depend on it.
constexpr int PAGED_EXTRA = 8;
constexpr int PAGED_MAX_WGS = 1024;        // workgroups of an attention launch, at most
// Whether an attention with weights leaves its scores in scratch for them (8 bytes a token and pair, written and read), or the keys
// are read again (2 to 4 head_dim bytes a token): from 32 pairs on that is less, and the scratch need not hold scores of many rows.
// 16 rows of 4 heads over 32K tokens, 8 KV heads: scores 54 us (20 of it their writes), keys 18; 8 rows: keys 15; 4 rows: scores 16.
constexpr int PAGED_SCORE_PAIRS = 31;
__host__ __device__ constexpr bool paged_keeps_scores(int pairs) { return pairs <= PAGED_SCORE_PAIRS; }

// Eviction: tables of up to EV_LONG tokens are selected from by one workgroup per (sequence, KV head), longer ones by several, EV_CHUNK
// tokens each. One sequence of 8 KV heads, us with its append of 2K: one workgroup 16K tokens 43, 22K 52, 32K 60; several 22K tokens
// 46, 32K 46. (The rule looks at the table alone: with more sequences one workgroup each fills more of the chip.)
constexpr int EV_LONG = 16384, EV_CHUNK = 4096;
constexpr int EV_LONG_WORDS = 4 + 2048;    // counters of a (sequence, KV head), zero between launches
constexpr int EV_SLOT_BYTES = 24;          // what the launches of a long selection tell each other

// In the device's error word beside the statuses: a sequence whose scores or lists of moves find no room in scratch, which holds the
// pool's tokens. Told as LTRI_ECAPACITY.
constexpr int PAGED_NO_ROOM = 1;

struct PagedDims {
  int Hq, Hkv, G, d, dtype, elt;
  int page_shift, n_pages, table_pages, max_seqs, rows_max, weights;
  long long page_stride, head_stride, token_stride;    // elements
  long long cap_tokens;                                // table_pages * page_tokens
  int long_pieces;                                     // pieces of EV_CHUNK tokens of a table, and one
  long long score_tiles;                               // tiles of scores, and of lists of moves, the scratch has room for
};

// Byte offsets in the caller's buffers.
struct PagedLayout {
  size_t err;          // int32 [4]
  size_t tickets;      // int32 [max_seqs][Hkv][blocks of 16 pairs]  zero between launches
  size_t long_state;   // int32 [max_seqs * Hkv][EV_LONG_WORDS]  zero between launches (tables of more than EV_LONG tokens)
  size_t state_total;
  size_t lse;          // float [max_seqs][rows_max][Hq]  log-sum-exp, log2 domain
  size_t part;         // float [2 PAGED_MAX_WGS][16, 32 or 64][d]  partial results of a workgroup's first and last problem
  size_t part_ml;      // float2 [2 PAGED_MAX_WGS][16, 32 or 64]    their maxima and sums
  size_t scores;       // float [score_tiles][Hkv][pairs][PAGED_TILE]   (ordered otherwise, see score_rows)
  size_t move_head;    // int64 [max_seqs * Hkv][2]  offset of a list of moves and its length
  size_t moves;        // int32 [score_tiles][Hkv][PAGED_TILE]
  size_t keys, candidates;   // uint32, the same (tables of more than EV_LONG tokens, and the next two)
  size_t long_slots;   // [max_seqs * Hkv] of EV_SLOT_BYTES
  size_t long_counts;  // int32 [max_seqs * Hkv][long_pieces][2]
  size_t scratch_total;
};

struct PagedCall {
  PagedDims D;
  char* k; char* v; float* weight; int32_t* pos;
  int32_t* err; int32_t* tickets;
  float* lse2; float* part; unsigned long long* part_ml; float* scores; long long* move_head; int32_t* moves;
  uint32_t* keys; uint32_t* candidates; char* long_slots; int32_t* long_counts; int32_t* long_state;
  const int32_t* table; int32_t* lens; const int32_t* seen;
  int seq_count;
  int n_cus;                 // compute units of the device
  // append, step
  const void* k_new; const void* v_new; const float* w_new;
  // append, attend, step: new rows
  int n;
  const void* q; void* out; float* lse; float decay;
  // evict
  int keep, n_sink, n_recent;
};

hipError_t launch_paged_append(const PagedCall& a, hipStream_t s);
hipError_t launch_paged_attend(const PagedCall& a, hipStream_t s);      // k_new != NULL: the rows are written, too
hipError_t launch_paged_evict(const PagedCall& a, hipStream_t s);
hipError_t launch_fill_zero(void* p, size_t bytes, hipStream_t s);      // seg.hip

#if defined(__HIPCC__)
// Length of a sequence; one that the table cannot hold is reported and taken as empty.
__device__ __forceinline__ int paged_len(const PagedCall& a, int s) {
  const int n = a.lens[s];
  if (n > a.D.cap_tokens) {
    atomicCAS(a.err, 0, LTRI_ECAPACITY);
    return 0;
  }
  return n > 0 ? n : 0;
}
// Page of the token at place i of a sequence, or -1 (reported) if the table names none in the pool.
__device__ __forceinline__ int paged_page(const PagedCall& a, int s, int i) {
  const int p = a.table[(size_t)s * a.D.table_pages + (i >> a.D.page_shift)];
  if ((unsigned)p < (unsigned)a.D.n_pages) return p;
  atomicCAS(a.err, 0, LTRI_EINVAL);
  return -1;
}
// Element offset of a token's row in the pools, and its index in weight and pos.
__device__ __forceinline__ long long paged_row(const PagedDims& D, int page, int h, int i) {
  return page * D.page_stride + h * D.head_stride + (i & ((1 << D.page_shift) - 1)) * D.token_stride;
}
__device__ __forceinline__ size_t paged_mark(const PagedDims& D, int page, int h, int i) {
  return (((size_t)page * D.Hkv + h) << D.page_shift) + (i & ((1 << D.page_shift) - 1));
}
__device__ __forceinline__ int paged_tiles(int len) { return (len + PAGED_TILE - 1) / PAGED_TILE; }
#endif

}  // namespace ltri
