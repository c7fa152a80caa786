// C ABI of the operators on the full cache: argument checks, workspace layout, launches.
#include "../../include/sagekv_cache.h"

#include <math.h>
#include <stdint.h>

#include "device_utils.h"
#include "full_cache.h"

using namespace sagekv;

namespace {

constexpr int64_t kMaxTokens = 1ll << 25;    // rotary_kernel's grid: 64 threads a token, less than 2^32 in all
constexpr int64_t kMaxStride = 1ll << 44;    // elements: no product of a stride and an index leaves 64 bits

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
sagekv_status dev(hipError_t e) { return e == hipSuccess ? SAGEKV_OK : SAGEKV_ERR_DEVICE; }
int element_bytes(int dtype) { return dtype == SAGEKV_BF16 ? 2 : 4; }

sagekv_status check_type(int dtype, int head_dim) {
  if (dtype != SAGEKV_BF16 && dtype != SAGEKV_F32) return SAGEKV_ERR_UNSUPPORTED;
  return head_dim == 64 || head_dim == 128 ? SAGEKV_OK : SAGEKV_ERR_UNSUPPORTED;
}

// Strides of one operand: 16-byte multiples, not negative.
bool strides_ok(const int64_t* s, int n, int dtype) {
  for (int i = 0; i < n; ++i)
    if (s[i] < 0 || s[i] > kMaxStride || s[i] % (16 / element_bytes(dtype))) return false;
  return true;
}

// Rows of `dim` elements at n[i] steps of s[i] each: do two of them overlap?  Sorted by stride, each has to step over all that lies
// within the smaller ones.  (Strides that interleave without meeting do not occur in a tensor's layout.)
bool rows_overlap(const int64_t* s, const int64_t* n, int dims, int64_t dim) {
  int64_t extent = dim;
  bool done[3] = {false, false, false};
  for (int k = 0; k < dims; ++k) {
    int least = -1;
    for (int i = 0; i < dims; ++i)
      if (!done[i] && (least < 0 || s[i] < s[least])) least = i;
    done[least] = true;
    if (n[least] <= 1) continue;
    if (s[least] < extent) return true;
    if (n[least] - 1 > (1ll << 62) / s[least]) return true;  // leaves 64 bits: no such memory
    extent += (n[least] - 1) * s[least];
    if (extent > (1ll << 62)) return true;
  }
  return false;
}

sagekv_status check_map(const sagekvc_rotary_map* m, int head_dim) {
  if (m->rotary_dim < 2 || m->rotary_dim > head_dim || m->rotary_dim % 2 || !m->inv_freq) return SAGEKV_ERR_INVALID_ARG;
  if (m->layout != SAGEKVC_ROTARY_HALF && m->layout != SAGEKVC_ROTARY_PAIRS) return SAGEKV_ERR_INVALID_ARG;
  if ((m->transpose != 0 && m->transpose != 1) || !isfinite(m->amplitude)) return SAGEKV_ERR_INVALID_ARG;
  return aligned(m->inv_freq, 8) ? SAGEKV_OK : SAGEKV_ERR_UNSUPPORTED;
}

void set_map(const sagekvc_rotary_map* m, RotaryParams* p) {
  p->r = m ? m->rotary_dim : 0;
  p->pairs_layout = m && m->layout == SAGEKVC_ROTARY_PAIRS;
  p->amplitude = m ? m->amplitude : 1.f;
  p->sign = m && m->transpose ? -1.f : 1.f;
  p->freq = m ? m->inv_freq : nullptr;
}

// A read-only operand's place in memory, in bytes.
TokenRows rows_of(const void* base, int64_t token, int64_t head, int dtype) {
  return {(char*)const_cast<void*>(base), token * element_bytes(dtype), head * element_bytes(dtype)};
}

// Output rows [n][heads] of a rotation: apart from each other, and the input itself if they are in its place.
sagekv_status check_out(const void* in, int64_t in_token, int64_t in_head, const void* out, int64_t out_token, int64_t out_head, int64_t n,
                        int64_t heads, int dim) {
  const int64_t s[2] = {out_token, out_head}, count[2] = {n, heads};
  if (rows_overlap(s, count, 2, dim)) return SAGEKV_ERR_INVALID_ARG;
  if (in == out && ((n > 1 && in_token != out_token) || (heads > 1 && in_head != out_head))) return SAGEKV_ERR_INVALID_ARG;
  return SAGEKV_OK;
}

sagekv_status check_cache(const sagekvc_desc* d, const sagekv_paged_kv* pg, const void* K, const void* V, bool written, FullCache* c) {
  if (!d || !K || !V) return SAGEKV_ERR_INVALID_ARG;
  if (d->n_problems < 1 || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->n_q_heads % d->n_kv_heads) return SAGEKV_ERR_INVALID_ARG;
  if (d->capacity < 1) return SAGEKV_ERR_INVALID_ARG;
  if (d->capacity > 1ll << 30) return SAGEKV_ERR_UNSUPPORTED;  // a length and a block beside it stay within 32 bits
  if (check_type(d->dtype, d->head_dim) != SAGEKV_OK) return SAGEKV_ERR_UNSUPPORTED;
  if (d->n_q_heads / d->n_kv_heads > 64 || (int64_t)d->n_problems * d->n_kv_heads > 65535) return SAGEKV_ERR_UNSUPPORTED;
  int64_t k[3] = {d->k_stride_problem, d->k_stride_head, d->k_stride_token};
  int64_t v[3] = {d->v_stride_problem, d->v_stride_head, d->v_stride_token};
  int64_t n[3] = {d->n_problems, d->n_kv_heads, d->capacity};
  c->table = nullptr;
  c->pitch = 0;
  c->shift = 31;
  c->n_blocks = d->n_problems;
  if (pg) {
    const int ps = pg->page_size;
    if (!pg->block_table || pg->n_pages < 1 || ps < 16 || (ps & (ps - 1))) return SAGEKV_ERR_INVALID_ARG;
    if (pg->table_pitch < (d->capacity + ps - 1) / ps || pg->table_pitch > kMaxStride) return SAGEKV_ERR_INVALID_ARG;
    if (!aligned(pg->block_table, 4)) return SAGEKV_ERR_UNSUPPORTED;
    k[0] = pg->k_stride_page;
    v[0] = pg->v_stride_page;
    n[0] = pg->n_pages;
    n[2] = ps;
    c->table = pg->block_table;
    c->pitch = pg->table_pitch;
    c->shift = __builtin_ctz((unsigned)ps);
    c->n_blocks = pg->n_pages;
  }
  if (!strides_ok(k, 3, d->dtype) || !strides_ok(v, 3, d->dtype) || !aligned(K, 16) || !aligned(V, 16)) return SAGEKV_ERR_UNSUPPORTED;
  if (k[2] < d->head_dim || v[2] < d->head_dim) return SAGEKV_ERR_UNSUPPORTED;  // as in the eviction pass
  const int64_t most = (1 << 24) / element_bytes(d->dtype);  // 24 bits: see load_token in cache_attn.hip
  if (k[2] >= most || v[2] >= most) return SAGEKV_ERR_UNSUPPORTED;
  if (written && (rows_overlap(k, n, 3, d->head_dim) || rows_overlap(v, n, 3, d->head_dim))) return SAGEKV_ERR_INVALID_ARG;
  const int eb = element_bytes(d->dtype);
  c->K = (char*)const_cast<void*>(K);
  c->V = (char*)const_cast<void*>(V);
  c->ks_block = k[0] * eb, c->ks_head = k[1] * eb, c->ks_token = (int)k[2] * eb;
  c->vs_block = v[0] * eb, c->vs_head = v[1] * eb, c->vs_token = (int)v[2] * eb;
  return SAGEKV_OK;
}

struct AttnLayout {
  size_t acc, ml, joins, total;
};
// Scratch for kAttnGroups workgroups, however many a call has: sizes are part of the interface.
AttnLayout attn_layout(const sagekvc_desc* d) {
  const size_t heads = (size_t)2 * kAttnGroups * (d->n_q_heads / d->n_kv_heads);
  AttnLayout l;
  l.acc = 0;
  l.ml = heads * d->head_dim * sizeof(float);
  l.joins = l.ml + heads * sizeof(float2);
  l.total = l.joins + kAttnGroups * sizeof(JoinRecord);
  return l;
}

}  // namespace

extern "C" {

sagekv_status sagekvc_rotary_frequencies(int32_t rotary_dim, double base, const sagekvc_rotary_scaling* sc, double* inv_freq,
                                         float* amplitude) {
  if (rotary_dim < 2 || rotary_dim % 2 || !(base > 1.0) || !isfinite(base) || !inv_freq || !amplitude) return SAGEKV_ERR_INVALID_ARG;
  const int kind = sc ? sc->kind : SAGEKVC_SCALING_NONE;
  if (kind < SAGEKVC_SCALING_NONE || kind > SAGEKVC_SCALING_YARN) return SAGEKV_ERR_INVALID_ARG;
  if (kind != SAGEKVC_SCALING_NONE && (!(sc->factor >= 1.0) || !isfinite(sc->factor))) return SAGEKV_ERR_INVALID_ARG;
  const bool by_turns = kind == SAGEKVC_SCALING_PARTS || kind == SAGEKVC_SCALING_YARN;
  if (by_turns && (!(sc->low > 0.0) || !(sc->high > sc->low) || !isfinite(sc->high) || !(sc->original_len > 0.0) || !isfinite(sc->original_len)))
    return SAGEKV_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925;
  double first = 0.0, last = 0.0;
  if (kind == SAGEKVC_SCALING_YARN) {
    // original_len * base^(-2j/r) / (2 pi) = turns, solved for j
    auto pair = [&](double turns) { return rotary_dim * log(sc->original_len / (turns * two_pi)) / (2.0 * log(base)); };
    first = fmax(floor(pair(sc->high)), 0.0);
    last = fmin(ceil(pair(sc->low)), (double)rotary_dim - 1.0);
  }
  for (int j = 0; j < rotary_dim / 2; ++j) {
    const double f = pow(base, -2.0 * j / rotary_dim);
    double kept = 1.0;  // share of the unstretched frequency
    if (kind == SAGEKVC_SCALING_LINEAR) kept = 0.0;
    if (kind == SAGEKVC_SCALING_PARTS) kept = (sc->original_len * f / two_pi - sc->low) / (sc->high - sc->low);
    if (kind == SAGEKVC_SCALING_YARN) kept = last > first ? 1.0 - (j - first) / (last - first) : (double)(j <= first);
    kept = fmin(fmax(kept, 0.0), 1.0);
    inv_freq[j] = kind == SAGEKVC_SCALING_NONE ? f : f * kept + f / sc->factor * (1.0 - kept);
  }
  *amplitude = kind == SAGEKVC_SCALING_YARN ? (float)(0.1 * log(sc->factor) + 1.0) : 1.f;
  return SAGEKV_OK;
}

sagekv_status sagekvc_rotary(const sagekvc_rotary_desc* d, const sagekvc_rotary_map* m, const void* x, const int32_t* positions, void* out,
                             void* hip_stream) {
  if (!d || !m || d->n_tokens < 0 || d->n_heads < 1) return SAGEKV_ERR_INVALID_ARG;
  if (check_type(d->dtype, d->head_dim) != SAGEKV_OK || d->n_tokens > kMaxTokens || d->n_heads > 65535) return SAGEKV_ERR_UNSUPPORTED;
  sagekv_status st = check_map(m, d->head_dim);
  if (st != SAGEKV_OK) return st;
  const int64_t strides[4] = {d->x_stride_token, d->x_stride_head, d->out_stride_token, d->out_stride_head};
  if (!strides_ok(strides, 4, d->dtype)) return SAGEKV_ERR_UNSUPPORTED;
  if (d->n_tokens == 0) return SAGEKV_OK;
  if (!x || !positions || !out) return SAGEKV_ERR_INVALID_ARG;
  if (!aligned(x, 16) || !aligned(out, 16) || !aligned(positions, 4)) return SAGEKV_ERR_UNSUPPORTED;
  st = check_out(x, d->x_stride_token, d->x_stride_head, out, d->out_stride_token, d->out_stride_head, d->n_tokens, d->n_heads, d->head_dim);
  if (st != SAGEKV_OK) return st;
  RotaryParams p = {};
  p.q = rows_of(x, d->x_stride_token, d->x_stride_head, d->dtype);
  p.q_out = rows_of(out, d->out_stride_token, d->out_stride_head, d->dtype);
  p.n_tokens = d->n_tokens;
  p.Hq = d->n_heads;
  p.D = d->head_dim;
  p.dtype = d->dtype;
  p.positions = positions;
  set_map(m, &p);
  return dev(launch_rotary(p, (hipStream_t)hip_stream));
}

sagekv_status sagekvc_write(const sagekvc_desc* d, const sagekv_paged_kv* pages, const sagekvc_tokens* tk, const sagekvc_rotary_map* m,
                            const void* q, const void* k_new, const void* v_new, const int32_t* token_offsets, const int32_t* seq_lens,
                            const int32_t* positions, void* q_out, void* K, void* V, void* hip_stream) {
  RotaryParams p = {};
  sagekv_status st = check_cache(d, pages, K, V, true, &p.cache);
  if (st != SAGEKV_OK) return st;
  if (!tk || tk->n_tokens < 0 || !seq_lens || (q == nullptr) != (q_out == nullptr)) return SAGEKV_ERR_INVALID_ARG;
  if (!token_offsets && tk->n_tokens != d->n_problems) return SAGEKV_ERR_INVALID_ARG;
  if (tk->n_tokens > kMaxTokens) return SAGEKV_ERR_UNSUPPORTED;
  if (m) {
    st = check_map(m, d->head_dim);
    if (st != SAGEKV_OK) return st;
  }
  const int64_t kv[4] = {tk->k_stride_token, tk->k_stride_head, tk->v_stride_token, tk->v_stride_head};
  const int64_t qs[4] = {tk->q_stride_token, tk->q_stride_head, tk->q_out_stride_token, tk->q_out_stride_head};
  if (!strides_ok(kv, 4, d->dtype) || (q && !strides_ok(qs, 4, d->dtype))) return SAGEKV_ERR_UNSUPPORTED;
  if (tk->n_tokens == 0) return SAGEKV_OK;
  if (!k_new || !v_new) return SAGEKV_ERR_INVALID_ARG;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(q, 16) || !aligned(q_out, 16) || !aligned(token_offsets, 4) ||
      !aligned(seq_lens, 4) || !aligned(positions, 4))
    return SAGEKV_ERR_UNSUPPORTED;
  if (q) {
    st = check_out(q, qs[0], qs[1], q_out, qs[2], qs[3], tk->n_tokens, d->n_q_heads, d->head_dim);
    if (st != SAGEKV_OK) return st;
    p.q = rows_of(q, qs[0], qs[1], d->dtype);
    p.q_out = rows_of(q_out, qs[2], qs[3], d->dtype);
  }
  p.k = rows_of(k_new, kv[0], kv[1], d->dtype);
  p.v = rows_of(v_new, kv[2], kv[3], d->dtype);
  p.n_tokens = tk->n_tokens;
  p.capacity = d->capacity;
  p.Hq = d->n_q_heads;
  p.Hkv = d->n_kv_heads;
  p.D = d->head_dim;
  p.dtype = d->dtype;
  p.P = d->n_problems;
  p.offsets = token_offsets;
  p.lens = seq_lens;
  p.positions = positions;
  set_map(m, &p);
  return dev(launch_rotary(p, (hipStream_t)hip_stream));
}

size_t sagekvc_attn_workspace_bytes(const sagekvc_desc* d) {
  FullCache c;
  // (the strides of a paged cache's problems are not looked at, and the caches' addresses neither)
  sagekvc_desc one = d ? *d : sagekvc_desc{};
  one.k_stride_problem = one.k_stride_head = one.v_stride_problem = one.v_stride_head = 0;
  one.k_stride_token = one.v_stride_token = one.head_dim;
  const void* any = (const void*)16;
  if (check_cache(d ? &one : nullptr, nullptr, any, any, false, &c) != SAGEKV_OK) return 0;
  return attn_layout(d).total;
}

sagekv_status sagekvc_attn(const sagekvc_desc* d, const sagekv_paged_kv* pages, const void* q, const void* K, const void* V,
                           const int32_t* seq_lens, int32_t max_len, int32_t n_sink, int32_t n_recent, float* out, float* lse,
                           void* workspace, size_t workspace_bytes, void* hip_stream) {
  CacheAttnParams p = {};
  sagekv_status st = check_cache(d, pages, K, V, false, &p.cache);
  if (st != SAGEKV_OK) return st;
  if (!q || !seq_lens || !out || max_len < 1 || max_len > d->capacity || n_sink < 0 || n_recent < 0 || (n_recent == 0 && n_sink > 0))
    return SAGEKV_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(seq_lens, 4) || !aligned(out, 4) || !aligned(lse, 4) || !aligned(workspace, 16)) return SAGEKV_ERR_UNSUPPORTED;
  const AttnLayout l = attn_layout(d);
  if (!workspace || workspace_bytes < l.total) return SAGEKV_ERR_WORKSPACE;
  p.q = (const char*)q;
  p.out = out;
  p.lse = lse;
  p.lens = seq_lens;
  p.P = d->n_problems;
  p.Hq = d->n_q_heads;
  p.Hkv = d->n_kv_heads;
  p.G = d->n_q_heads / d->n_kv_heads;
  p.D = d->head_dim;
  p.dtype = d->dtype;
  p.S = n_sink < max_len ? n_sink : max_len;
  p.W = n_recent < max_len ? n_recent : max_len;
  p.max_len = max_len;
  p.scale = (float)(1.0 / sqrt((double)d->head_dim));
  p.join_scale = d->dtype == SAGEKV_BF16 ? p.scale : 1.f;
  // blocks of the longest row: all of its tokens, or those of the window's two ends
  const int bt = attn_block(d->dtype, d->head_dim);
  int64_t blocks = ((int64_t)max_len + bt - 1) / bt;
  if (p.W > 0) {
    const int64_t ends = (p.S + bt - 1) / bt + (p.W + bt - 2) / bt + 1;
    if (ends < blocks) blocks = ends;
  }
  const int64_t rows = (int64_t)d->n_problems * d->n_kv_heads, weight = rows * (blocks + 4);
  if (weight > 0x7FFFFFFF) return SAGEKV_ERR_UNSUPPORTED;
  p.n_waves = weight < kAttnWaves ? (int)weight : kAttnWaves;
  p.by_row = rows <= kAttnGroups;
  p.part_acc = (float*)((char*)workspace + l.acc);
  p.part_ml = (float2*)((char*)workspace + l.ml);
  p.joins = (JoinRecord*)((char*)workspace + l.joins);
  const bool short_rows = RowCuts(rows).rounds(blocks) <= kWholeRounds;  // none will be split, whatever the lengths are
  return dev(launch_cache_attn(p, !short_rows, (hipStream_t)hip_stream));
}

}  // extern "C"
