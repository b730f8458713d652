// Host side of the paged cache (ltri_paged.h): handle, argument checks, buffer layout.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>

#include "paged_internal.h"

using namespace ltri;

struct ltri_paged {
  PagedDims D;
  PagedLayout L;
  PagedCall base;            // what every call passes on
  char* state;
  hipStream_t stream;
  int device;
  bool dry;
  char err[512];
};

static int32_t fail(ltri_paged* c, int32_t code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(c->err, sizeof c->err, fmt, ap);
  va_end(ap);
  return code;
}

static size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

static int32_t derive(const ltri_paged_config* cfg, PagedDims& D, PagedLayout& L) {
  if (!cfg) return LTRI_EINVAL;
  const ltri_paged_config& c = *cfg;
  if (c.n_q_heads < 1 || c.n_q_heads > 4096 || c.n_kv_heads < 1 || c.n_q_heads % c.n_kv_heads || c.n_q_heads / c.n_kv_heads > 128)
    return LTRI_EINVAL;
  if (c.head_dim != 64 && c.head_dim != 128) return LTRI_EINVAL;
  if (c.dtype != LTRI_F32 && c.dtype != LTRI_BF16) return LTRI_EINVAL;
  if (c.page_tokens < 1 || c.page_tokens > 4096 || (c.page_tokens & (c.page_tokens - 1))) return LTRI_EINVAL;
  if (c.n_pages < 1 || c.table_pages < 1 || (long long)c.table_pages * c.page_tokens > (1ll << 30)) return LTRI_EINVAL;
  if (c.max_seqs < 1 || c.max_seqs > LTRI_PAGED_MAX_SEQS) return LTRI_EINVAL;
  if (c.rows_max < 1 || c.rows_max > LTRI_PAGED_MAX_ROWS) return LTRI_EINVAL;
  if (c.weights != 0 && c.weights != 1) return LTRI_EINVAL;
  D.Hq = c.n_q_heads; D.Hkv = c.n_kv_heads; D.G = c.n_q_heads / c.n_kv_heads;
  D.d = c.head_dim; D.dtype = c.dtype; D.elt = c.dtype == LTRI_F32 ? 4 : 2;
  D.page_shift = __builtin_ctz((unsigned)c.page_tokens);
  D.n_pages = c.n_pages; D.table_pages = c.table_pages; D.max_seqs = c.max_seqs; D.rows_max = c.rows_max;
  D.weights = c.weights;
  D.cap_tokens = (long long)c.table_pages * c.page_tokens;
  if (!c.page_stride && !c.head_stride && !c.token_stride) {
    D.token_stride = D.d;
    D.head_stride = (long long)c.page_tokens * D.d;
    D.page_stride = D.Hkv * D.head_stride;
  } else {
    D.page_stride = c.page_stride; D.head_stride = c.head_stride; D.token_stride = c.token_stride;
    const long long step = 16 / D.elt;
    struct Axis { long long* stride; long long count; };
    Axis ax[3] = {{&D.page_stride, c.n_pages}, {&D.head_stride, D.Hkv}, {&D.token_stride, c.page_tokens}};
    for (const Axis& x : ax) {
      if (x.count == 1) *x.stride = 0;                  // never stepped over, whatever was given
      else if (*x.stride < 1 || *x.stride % step || *x.stride > 1ll << 40) return LTRI_EINVAL;
      if ((double)x.count * *x.stride * D.elt > 4e18) return LTRI_EINVAL;      // (sums of three stay within 63 bits)
    }
    if (D.token_stride > 1ll << 24) return LTRI_EINVAL;     // 16 tokens lie within 32-bit byte offsets
    // no two rows may overlap: in the order of the strides, each steps over all that the axes below it reach
    for (int i = 0; i < 3; ++i)
      for (int j = i + 1; j < 3; ++j)
        if (*ax[j].stride < *ax[i].stride) { const Axis t = ax[i]; ax[i] = ax[j]; ax[j] = t; }
    long long reach = D.d;
    for (const Axis& x : ax) {
      if (x.count == 1) continue;
      if (*x.stride < reach) return LTRI_EINVAL;
      reach += *x.stride * (x.count - 1);
    }
  }
  if ((double)c.n_pages * D.page_stride * D.elt > 4e18) return LTRI_EINVAL;

  size_t o = 0;
  L.err = o;     o = align_up(o + 16);
  L.tickets = o; o = align_up(o + (size_t)c.max_seqs * D.Hkv * ((D.rows_max * D.G + 15) / 16) * 4);
  const bool is_long = D.weights && D.cap_tokens > EV_LONG;
  const size_t slots = (size_t)c.max_seqs * D.Hkv;
  L.long_state = o; o = align_up(o + (is_long ? slots * EV_LONG_WORDS * 4 : 0));
  L.state_total = o;

  // with weights no page is named twice in a call: its tokens are at most the pool's, and a sequence's last tile is padded
  D.score_tiles = 0;
  D.long_pieces = (int)((D.cap_tokens + EV_CHUNK - 1) / EV_CHUNK + 1);    // (one more: pieces end at the budget)
  if (D.weights) {
    const long long pool = (((long long)c.n_pages << D.page_shift) + PAGED_TILE - 1) / PAGED_TILE + (long long)c.max_seqs * (1 + PAGED_EXTRA);
    const long long tables = ((D.cap_tokens + PAGED_TILE - 1) / PAGED_TILE + PAGED_EXTRA) * c.max_seqs;
    D.score_tiles = pool < tables ? pool : tables;
  }
  if ((double)D.score_tiles * D.Hq * D.rows_max * PAGED_TILE * 4 > 1e15) return LTRI_EINVAL;
  o = 0;
  const int pairs = D.rows_max * D.G, block = pairs <= 16 ? 16 : pairs <= 32 ? 32 : 64;      // of a problem, at most
  const int scored = pairs < PAGED_SCORE_PAIRS ? pairs : PAGED_SCORE_PAIRS;                  // pairs whose scores are kept, at most
  L.lse = o;    o = align_up(o + (size_t)c.max_seqs * D.rows_max * D.Hq * 4);
  L.part = o;   o = align_up(o + (size_t)2 * PAGED_MAX_WGS * block * D.d * 4);
  L.part_ml = o; o = align_up(o + (size_t)2 * PAGED_MAX_WGS * block * 8);
  L.scores = o; o = align_up(o + (size_t)D.score_tiles * D.Hkv * scored * PAGED_TILE * 4);
  const size_t attend_end = o;
  o = 0;                                                 // the two kinds of call share the scratch
  L.move_head = o; o = align_up(o + (D.weights ? (size_t)c.max_seqs * D.Hkv * 16 : 0));
  const size_t list = (size_t)D.score_tiles * D.Hkv * PAGED_TILE * 4;
  L.moves = o;     o = align_up(o + list);
  L.keys = o;      o = align_up(o + (is_long ? list : 0));
  L.candidates = o; o = align_up(o + (is_long ? list : 0));
  L.long_slots = o; o = align_up(o + (is_long ? slots * EV_SLOT_BYTES : 0));
  L.long_counts = o; o = align_up(o + (is_long ? slots * D.long_pieces * 8 : 0));
  L.scratch_total = o > attend_end ? o : attend_end;
  return LTRI_OK;
}

namespace {
// The handle's device for the length of a call.
struct OnDevice {
  int before = -1;
  hipError_t e;
  explicit OnDevice(int device) {
    e = hipGetDevice(&before);
    if (e == hipSuccess && before != device) e = hipSetDevice(device);
    else before = -1;
  }
  ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};
}  // namespace

static int32_t check_hip(ltri_paged* c, hipError_t e, const char* what) {
  if (e == hipSuccess) return LTRI_OK;
  return fail(c, LTRI_EHIP, "%s: %s", what, hipGetErrorString(e));
}

static bool misaligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

extern "C" {

const char* ltri_paged_last_error(const ltri_paged* c) { return c ? c->err : ""; }

int32_t ltri_paged_workspace_bytes(const ltri_paged_config* cfg, size_t* state_bytes, size_t* scratch_bytes) {
  PagedDims D; PagedLayout L;
  const int32_t r = derive(cfg, D, L);
  if (r != LTRI_OK) return r;
  if (state_bytes) *state_bytes = L.state_total;
  if (scratch_bytes) *scratch_bytes = L.scratch_total;
  return LTRI_OK;
}

static int32_t create_impl(const ltri_paged_config* cfg, void* k_pages, void* v_pages, float* weight, int32_t* pos, void* state,
                           void* scratch, void* hip_stream, bool dry, ltri_paged** out) {
  if (!out) return LTRI_EINVAL;
  *out = nullptr;
  PagedDims D; PagedLayout L;
  const int32_t r = derive(cfg, D, L);
  if (r != LTRI_OK) return r;
  if (!dry) {
    if (!k_pages || !v_pages || !state || !scratch || misaligned(k_pages, 16) || misaligned(v_pages, 16) ||
        misaligned(state, 256) || misaligned(scratch, 256))
      return LTRI_EINVAL;
    if (D.weights ? (!weight || !pos || misaligned(weight, 4) || misaligned(pos, 4)) : (weight || pos)) return LTRI_EINVAL;
  }
  ltri_paged* c = new (std::nothrow) ltri_paged();
  if (!c) return LTRI_EINVAL;
  c->D = D; c->L = L; c->dry = dry; c->stream = (hipStream_t)hip_stream; c->device = 0; c->state = (char*)state;
  c->err[0] = 0;
  PagedCall& b = c->base;
  memset(&b, 0, sizeof b);
  b.D = D;
  b.k = (char*)k_pages; b.v = (char*)v_pages; b.weight = weight; b.pos = pos;
  char* t = (char*)scratch;
  b.err = (int32_t*)(c->state + L.err); b.tickets = (int32_t*)(c->state + L.tickets);
  b.lse2 = (float*)(t + L.lse); b.part = (float*)(t + L.part); b.part_ml = (unsigned long long*)(t + L.part_ml); b.scores = (float*)(t + L.scores);
  b.move_head = (long long*)(t + L.move_head); b.moves = (int32_t*)(t + L.moves);
  b.keys = (uint32_t*)(t + L.keys); b.candidates = (uint32_t*)(t + L.candidates); b.long_slots = t + L.long_slots;
  b.long_counts = (int32_t*)(t + L.long_counts); b.long_state = (int32_t*)(c->state + L.long_state);
  if (!dry) {
    hipError_t e = hipGetDevice(&c->device);
    if (e == hipSuccess) e = hipDeviceGetAttribute(&b.n_cus, hipDeviceAttributeMultiprocessorCount, c->device);
    if (e == hipSuccess) e = launch_fill_zero(c->state, L.state_total, c->stream);
    if (e != hipSuccess) { delete c; return LTRI_EHIP; }
  }
  *out = c;
  return LTRI_OK;
}

int32_t ltri_paged_create(const ltri_paged_config* cfg, void* k_pages, void* v_pages, float* weight, int32_t* pos, void* state,
                          void* scratch, void* hip_stream, ltri_paged** out) {
  return create_impl(cfg, k_pages, v_pages, weight, pos, state, scratch, hip_stream, false, out);
}

int32_t ltri_paged_create_dry(const ltri_paged_config* cfg, ltri_paged** out) {
  return create_impl(cfg, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, true, out);
}

int32_t ltri_paged_destroy(ltri_paged* c) {
  if (!c) return LTRI_EINVAL;
  delete c;
  return LTRI_OK;
}

int32_t ltri_paged_set_stream(ltri_paged* c, void* hip_stream) {
  if (!c) return LTRI_EINVAL;
  c->stream = (hipStream_t)hip_stream;
  return LTRI_OK;
}

// What every call is checked for; the call's arguments so far to a.
static int32_t begin(ltri_paged* c, int32_t seq_count, const int32_t* table, const int32_t* lens, const int32_t* seen,
                     bool needs_seen, PagedCall& a) {
  if (seq_count < 1 || seq_count > c->D.max_seqs)
    return fail(c, LTRI_EINVAL, "seq_count %d outside [1, max_seqs %d]", seq_count, c->D.max_seqs);
  if (!table || !lens) return fail(c, LTRI_EINVAL, "table or lens is NULL");
  if (needs_seen && !seen) return fail(c, LTRI_EINVAL, "seen is NULL, and the cache keeps positions");
  if (misaligned(table, 4) || misaligned(lens, 4) || misaligned(seen, 4)) return fail(c, LTRI_EINVAL, "table, lens or seen is not aligned");
  a = c->base;
  a.table = table; a.lens = const_cast<int32_t*>(lens); a.seen = seen; a.seq_count = seq_count;
  return LTRI_OK;
}

static int32_t check_rows(ltri_paged* c, const void* k_new, const void* v_new) {
  if (!k_new || !v_new) return fail(c, LTRI_EINVAL, "k_new or v_new is NULL");
  if (misaligned(k_new, 16) || misaligned(v_new, 16)) return fail(c, LTRI_EINVAL, "k_new and v_new must be 16-byte aligned");
  return LTRI_OK;
}

static int32_t check_query(ltri_paged* c, int32_t seq_count, const void* q, int32_t n_q, void* out, float* lse, float decay) {
  if (n_q < 1 || n_q > c->D.rows_max) return fail(c, LTRI_EINVAL, "%d query rows outside [1, rows_max %d]", n_q, c->D.rows_max);
  if (!q || !out) return fail(c, LTRI_EINVAL, "q or out is NULL");
  if (misaligned(q, 16) || misaligned(out, 16) || misaligned(lse, 4)) return fail(c, LTRI_EINVAL, "q and out must be 16-byte aligned, lse 4-byte");
  const uintptr_t bytes = (uintptr_t)seq_count * n_q * c->D.Hq * c->D.d * c->D.elt, from = (uintptr_t)q, to = (uintptr_t)out;
  if (from < to + bytes && to < from + bytes) return fail(c, LTRI_EINVAL, "q and out overlap");      // (weights read q again)
  if (!(std::fabs(decay) <= 3.4028234e38f)) return fail(c, LTRI_EINVAL, "decay is not a finite number");
  if (decay >= 0.0f && !c->D.weights) return fail(c, LTRI_EINVAL, "decay %g, but the cache keeps no weights", (double)decay);
  return LTRI_OK;
}

int32_t ltri_paged_append(ltri_paged* c, int32_t seq_count, const int32_t* table, const int32_t* lens, const int32_t* seen,
                          const void* k_new, const void* v_new, const float* w_new, int32_t n_new) {
  if (!c) return LTRI_EINVAL;
  PagedCall a;
  int32_t r = begin(c, seq_count, table, lens, seen, c->D.weights != 0, a);
  if (r != LTRI_OK) return r;
  if (n_new < 1) return fail(c, LTRI_EINVAL, "n_new %d", n_new);
  if (n_new > c->D.cap_tokens) return fail(c, LTRI_ECAPACITY, "%d new tokens exceed the table's %lld", n_new, c->D.cap_tokens);
  r = check_rows(c, k_new, v_new);
  if (r != LTRI_OK) return r;
  if (w_new && !c->D.weights) return fail(c, LTRI_EINVAL, "w_new given, but the cache keeps no weights");
  if (misaligned(w_new, 4)) return fail(c, LTRI_EINVAL, "w_new is not aligned");
  a.k_new = k_new; a.v_new = v_new; a.w_new = w_new; a.n = n_new;
  if (c->dry) return LTRI_OK;
  OnDevice on(c->device);
  r = check_hip(c, on.e, "device");
  return r != LTRI_OK ? r : check_hip(c, launch_paged_append(a, c->stream), "append to pages");
}

int32_t ltri_paged_attend(ltri_paged* c, int32_t seq_count, const int32_t* table, const int32_t* lens, const void* q, int32_t n_q,
                          void* out, float* lse, float decay) {
  if (!c) return LTRI_EINVAL;
  PagedCall a;
  int32_t r = begin(c, seq_count, table, lens, nullptr, false, a);
  if (r == LTRI_OK) r = check_query(c, seq_count, q, n_q, out, lse, decay);
  if (r != LTRI_OK) return r;
  a.q = q; a.n = n_q; a.out = out; a.lse = lse; a.decay = decay;
  if (c->dry) return LTRI_OK;
  OnDevice on(c->device);
  r = check_hip(c, on.e, "device");
  return r != LTRI_OK ? r : check_hip(c, launch_paged_attend(a, c->stream), "attend over pages");
}

int32_t ltri_paged_step(ltri_paged* c, int32_t seq_count, const int32_t* table, const int32_t* lens, const int32_t* seen,
                        const void* k_new, const void* v_new, const void* q, int32_t n_new, void* out, float* lse, float decay) {
  if (!c) return LTRI_EINVAL;
  PagedCall a;
  int32_t r = begin(c, seq_count, table, lens, seen, c->D.weights != 0, a);
  if (r == LTRI_OK) r = check_query(c, seq_count, q, n_new, out, lse, decay);
  if (r == LTRI_OK) r = check_rows(c, k_new, v_new);
  if (r != LTRI_OK) return r;
  a.k_new = k_new; a.v_new = v_new; a.q = q; a.n = n_new; a.out = out; a.lse = lse; a.decay = decay;
  if (c->dry) return LTRI_OK;
  OnDevice on(c->device);
  r = check_hip(c, on.e, "device");
  return r != LTRI_OK ? r : check_hip(c, launch_paged_attend(a, c->stream), "step over pages");
}

int32_t ltri_paged_evict(ltri_paged* c, int32_t seq_count, const int32_t* table, int32_t* lens, const int32_t* seen, int32_t keep,
                         int32_t n_sink, int32_t n_recent) {
  if (!c) return LTRI_EINVAL;
  if (!c->D.weights) return fail(c, LTRI_EINVAL, "the cache keeps no weights to evict by");
  PagedCall a;
  int32_t r = begin(c, seq_count, table, lens, seen, true, a);
  if (r != LTRI_OK) return r;
  if (keep < 1 || n_sink < 0 || n_recent < 0 || (long long)n_sink + n_recent > keep)
    return fail(c, LTRI_EINVAL, "keep %d, n_sink %d, n_recent %d: keep >= 1 and n_sink + n_recent <= keep are wanted", keep, n_sink, n_recent);
  a.keep = keep; a.n_sink = n_sink; a.n_recent = n_recent;
  if (c->dry || keep >= c->D.cap_tokens) return LTRI_OK;        // no sequence can hold more
  OnDevice on(c->device);
  r = check_hip(c, on.e, "device");
  return r != LTRI_OK ? r : check_hip(c, launch_paged_evict(a, c->stream), "evict");
}

int32_t ltri_paged_sync_status(ltri_paged* c) {
  if (!c) return LTRI_EINVAL;
  if (c->dry) return LTRI_OK;
  OnDevice on(c->device);
  int32_t r = check_hip(c, on.e, "device");
  if (r == LTRI_OK) r = check_hip(c, hipStreamSynchronize(c->stream), "synchronise");
  if (r != LTRI_OK) return r;
  int32_t e[4] = {0, 0, 0, 0};
  r = check_hip(c, hipMemcpy(e, c->state + c->L.err, sizeof e, hipMemcpyDeviceToHost), "read the error word");
  if (r != LTRI_OK || e[0] == 0) return r;
  r = check_hip(c, launch_fill_zero(c->state + c->L.err, 16, c->stream), "clear the error word");
  if (r != LTRI_OK) return r;
  if (e[0] == PAGED_NO_ROOM)
    return fail(c, LTRI_ECAPACITY, "raised on the device: more tokens in a call than the pool holds (a page named twice?); weights or evictions are left out");
  return fail(c, e[0], "raised on the device: %s", e[0] == LTRI_ECAPACITY ? "a length beyond the page table"
                                                                          : "a page outside the pool");
}

}  // extern "C"
