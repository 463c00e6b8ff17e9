// Host side of the rotary and paged-cache entry points: validation, scratch planning, launches.
#include <climits>
#include <cmath>

#include "snap_internal.cuh"

namespace snap {

namespace {

constexpr int kMaxTokens = INT_MAX - 255;      // a block of the rotary pass has 256 tokens at most: the last one's numbers stay within 32 bits
constexpr double kTwoPi = 6.283185307179586;

}  // namespace

// The fields the kernels use: snap_rope_table checks the rest.
int check_rope(const snap_rope_config_t* r) {
  if (!r) return SNAP_ERR_NULL_POINTER;
  if (r->rot_dim < 2 || r->rot_dim % 2 || r->rot_offset < 0) return SNAP_ERR_INVALID_ARG;
  if (r->interleaved != 0 && r->interleaved != 1) return SNAP_ERR_INVALID_ARG;
  if (r->scaling < SNAP_ROPE_PLAIN || r->scaling > SNAP_ROPE_YARN) return SNAP_ERR_INVALID_ARG;
  if (!std::isfinite(r->magnitude) || r->magnitude < 0) return SNAP_ERR_INVALID_ARG;
  if (r->magnitude == 0 && r->scaling == SNAP_ROPE_YARN && !(r->factor >= 1 && std::isfinite(r->factor))) return SNAP_ERR_INVALID_ARG;
  return SNAP_OK;
}

double rope_magnitude(const snap_rope_config_t* r) {
  if (r->magnitude > 0) return r->magnitude;
  return r->scaling == SNAP_ROPE_YARN ? 0.1 * std::log(r->factor) + 1.0 : 1.0;
}

// Strides of a [tokens][heads][d] tensor: multiples of 16 bytes, not negative.
bool strides_ok(long long tok, long long head, int eb) { return tok >= 0 && head >= 0 && (tok * eb) % 16 == 0 && (head * eb) % 16 == 0; }
// ... and, of one that is written, no two heads on the same memory: token-major or head-major.
bool out_strides_ok(long long tok, long long head, int tokens, int heads, int d, int eb) {
  if (!strides_ok(tok, head, eb)) return false;
  const bool one_t = tokens == 1, one_h = heads == 1;
  const bool token_major = (one_h || head >= d) && (one_t || tok >= (one_h ? 0 : (heads - 1) * head) + d);
  const bool head_major = (one_t || tok >= d) && (one_h || head >= (one_t ? 0 : (tokens - 1) * tok) + d);
  return token_major || head_major;
}

int check_page_counts(const snap_config_t* cfg, const snap_paged_t* p) {
  const int rc = validate_config(cfg);
  if (rc != SNAP_OK) return rc;
  if (!p) return SNAP_ERR_NULL_POINTER;
  if (p->page_tokens < 1 || p->n_pages < 1 || p->max_pages < 1 || p->reserved != 0) return SNAP_ERR_INVALID_ARG;
  if ((long long)p->page_tokens * p->max_pages > (1LL << 30)) return SNAP_ERR_INVALID_ARG;
  return SNAP_OK;
}

int check_paged(const snap_config_t* cfg, const snap_paged_t* p, int eb) {
  const int rc = check_page_counts(cfg, p);
  if (rc != SNAP_OK) return rc;
  const long long st[6] = {p->k_page_stride, p->k_head_stride, p->k_row_stride, p->v_page_stride, p->v_head_stride, p->v_row_stride};
  for (const long long x : st)
    if (x < 0 || x > (1LL << 40) || (x * eb) % 16) return SNAP_ERR_INVALID_ARG;
  if ((p->page_tokens > 1 && (p->k_row_stride < cfg->d_qk || p->v_row_stride < cfg->d_v)) ||
      (cfg->n_kv_heads > 1 && (p->k_head_stride < cfg->d_qk || p->v_head_stride < cfg->d_v)) ||
      (p->n_pages > 1 && (p->k_page_stride < cfg->d_qk || p->v_page_stride < cfg->d_v)))
    return SNAP_ERR_INVALID_ARG;
  if (cfg->v_aliases_k || cfg->d_qk > 256 || cfg->d_v > 256) return SNAP_ERR_UNSUPPORTED;
  return SNAP_OK;
}

PageMap page_map(const snap_paged_t* p, const int* table) {
  PageMap m;
  m.page = p->page_tokens; m.n_pages = p->n_pages; m.max_pages = p->max_pages; m.cap = p->page_tokens * p->max_pages;
  m.kp = p->k_page_stride; m.kh = p->k_head_stride; m.kr = p->k_row_stride;
  m.vp = p->v_page_stride; m.vh = p->v_head_stride; m.vr = p->v_row_stride;
  m.table = table;
  return m;
}

namespace {

// Do the blocks that move a call's rows (64 or more rows each) fit one grid, and its KV heads and sequences the selection's?
bool evict_countable(const snap_config_t* c, int n_seqs) {
  const long long keep = (long long)c->l_sink + c->l_recent + c->topk;
  return c->n_kv_heads <= 65535 && (keep / 64 + 1) * c->n_kv_heads * n_seqs <= 0x7fffffffLL;
}

}  // namespace

int status_of(cudaError_t e) { return e == cudaSuccess ? SNAP_OK : SNAP_ERR_CUDA; }

}  // namespace snap

using namespace snap;

extern "C" {

int snap_rope_table(const snap_rope_config_t* r, double* freqs_host, double* magnitude_host) {
  const int rc = check_rope(r);
  if (rc != SNAP_OK) return rc;
  if (!(r->base > 1) || !std::isfinite(r->base)) return SNAP_ERR_INVALID_ARG;
  const bool scaled = r->scaling != SNAP_ROPE_PLAIN;
  if (scaled && !(r->factor >= 1 && std::isfinite(r->factor))) return SNAP_ERR_INVALID_ARG;
  if ((r->scaling == SNAP_ROPE_LLAMA3 || r->scaling == SNAP_ROPE_YARN) && !(r->original_len > 0 && std::isfinite(r->original_len)))
    return SNAP_ERR_INVALID_ARG;
  if (r->scaling == SNAP_ROPE_LLAMA3 && !(r->low_freq > 0 && r->high_freq > r->low_freq && std::isfinite(r->high_freq)))
    return SNAP_ERR_INVALID_ARG;
  if (r->scaling == SNAP_ROPE_YARN && !(r->beta_slow > 0 && r->beta_fast > r->beta_slow && std::isfinite(r->beta_fast)))
    return SNAP_ERR_INVALID_ARG;
  double lo = 0, hi = 0;
  if (r->scaling == SNAP_ROPE_YARN) {
    const auto turns_at = [&](double n) { return r->rot_dim * std::log(r->original_len / (n * kTwoPi)) / (2.0 * std::log(r->base)); };
    lo = std::fmax(std::floor(turns_at(r->beta_fast)), 0.0);
    hi = std::fmin(std::ceil(turns_at(r->beta_slow)), r->rot_dim - 1.0);
    if (hi - lo < 1e-3) hi = lo + 1e-3;                        // both ends on one pair: a step there
  }
  for (int i = 0; freqs_host && i < r->rot_dim / 2; ++i) {
    double f = std::pow(r->base, -2.0 * i / r->rot_dim);
    if (r->scaling == SNAP_ROPE_LINEAR) f /= r->factor;
    if (r->scaling == SNAP_ROPE_LLAMA3) {
      const double turns = r->original_len * f / kTwoPi;       // original_len / wavelength
      const double s = std::fmin(std::fmax((turns - r->low_freq) / (r->high_freq - r->low_freq), 0.0), 1.0);
      f *= s + (1.0 - s) / r->factor;
    }
    if (r->scaling == SNAP_ROPE_YARN) {
      const double ramp = std::fmin(std::fmax((i - lo) / (hi - lo), 0.0), 1.0);
      f *= (1.0 - ramp) + ramp / r->factor;
    }
    freqs_host[i] = f;
  }
  if (magnitude_host) *magnitude_host = rope_magnitude(r);
  return SNAP_OK;
}

int snap_rope(const snap_config_t* cfg, const snap_rope_config_t* rope, const double* freqs_dev,
              const int32_t* positions_dev, int32_t n_tokens,
              const void* q_dev, int64_t q_token_stride, int64_t q_head_stride,
              void* q_out_dev, int64_t q_out_token_stride, int64_t q_out_head_stride,
              const void* k_dev, int64_t k_token_stride, int64_t k_head_stride,
              void* k_out_dev, int64_t k_out_token_stride, int64_t k_out_head_stride,
              int32_t inverse, void* cuda_stream) {
  int rc = validate_config(cfg);
  if (rc != SNAP_OK) return rc;
  rc = check_rope(rope);
  if (rc != SNAP_OK) return rc;
  if (rope->rot_dim > cfg->d_qk - rope->rot_offset || n_tokens < 0 || n_tokens > kMaxTokens || (inverse != 0 && inverse != 1)) return SNAP_ERR_INVALID_ARG;
  if (n_tokens == 0) return SNAP_OK;
  if (!freqs_dev || !positions_dev || !q_dev != !q_out_dev || !k_dev != !k_out_dev || (!q_dev && !k_dev)) return SNAP_ERR_NULL_POINTER;
  if (misaligned(q_dev, q_out_dev, k_dev, k_out_dev)) return SNAP_ERR_INVALID_ARG;
  const int eb = elt_bytes(cfg->dtype);
  if (q_dev && (!strides_ok(q_token_stride, q_head_stride, eb) ||
                !out_strides_ok(q_out_token_stride, q_out_head_stride, n_tokens, cfg->n_q_heads, cfg->d_qk, eb) ||
                (q_dev == q_out_dev && (q_token_stride != q_out_token_stride || q_head_stride != q_out_head_stride))))
    return SNAP_ERR_INVALID_ARG;
  if (k_dev && (!strides_ok(k_token_stride, k_head_stride, eb) ||
                !out_strides_ok(k_out_token_stride, k_out_head_stride, n_tokens, cfg->n_kv_heads, cfg->d_qk, eb) ||
                (k_dev == k_out_dev && (k_token_stride != k_out_token_stride || k_head_stride != k_out_head_stride))))
    return SNAP_ERR_INVALID_ARG;
  RopeArgs a = {};
  a.q = q_dev; a.q_out = q_out_dev; a.k = k_dev; a.k_out = k_out_dev;
  a.q_tok = q_token_stride; a.q_head = q_head_stride; a.qo_tok = q_out_token_stride; a.qo_head = q_out_head_stride;
  a.k_tok = k_token_stride; a.k_head = k_head_stride; a.ko_tok = k_out_token_stride; a.ko_head = k_out_head_stride;
  a.freqs = freqs_dev; a.positions = positions_dev; a.n_tokens = n_tokens;
  a.Hq = q_dev ? cfg->n_q_heads : 0; a.Hkv = k_dev ? cfg->n_kv_heads : 0; a.d_qk = cfg->d_qk; a.d_v = cfg->d_v;
  a.rot = rope->rot_dim; a.offset = rope->rot_offset; a.interleaved = rope->interleaved;
  a.magnitude = (float)rope_magnitude(rope); a.sign = inverse ? -1.f : 1.f;
  return status_of(launch_rope(cfg->dtype, a, static_cast<cudaStream_t>(cuda_stream)));
}

int snap_paged_append(const snap_config_t* cfg, const snap_paged_t* paged,
                      const int32_t* slot_ids_dev, const int32_t* rows_dev, int32_t n_tokens,
                      const snap_rope_config_t* rope, const double* freqs_dev, const int32_t* positions_dev,
                      const void* q_dev, int64_t q_token_stride, int64_t q_head_stride, void* q_out_dev,
                      const void* k_dev, int64_t k_token_stride, int64_t k_head_stride, void* k_out_dev,
                      const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                      void* k_pages_dev, void* v_pages_dev, const int32_t* page_table_dev,
                      int32_t* seq_len_dev, float* weights_dev, uint32_t* status_dev, void* cuda_stream) {
  int rc = check_paged(cfg, paged, cfg ? elt_bytes(cfg->dtype) : 0);
  if (rc != SNAP_OK) return rc;
  if (rope) {
    rc = check_rope(rope);
    if (rc != SNAP_OK) return rc;
    if (rope->rot_dim > cfg->d_qk - rope->rot_offset) return SNAP_ERR_INVALID_ARG;
  }
  if (n_tokens < 0 || n_tokens > kMaxTokens || (!rows_dev && n_tokens > 65536)) return SNAP_ERR_INVALID_ARG;   // (each token looks for its slot among those before it)
  if (n_tokens == 0) return SNAP_OK;
  if (!slot_ids_dev || !k_dev || !v_dev || !k_pages_dev || !v_pages_dev || !page_table_dev || !seq_len_dev || (rope && !freqs_dev) ||
      !q_dev != !q_out_dev)
    return SNAP_ERR_NULL_POINTER;
  if (misaligned(q_dev, q_out_dev, k_dev, k_out_dev, v_dev, k_pages_dev, v_pages_dev)) return SNAP_ERR_INVALID_ARG;
  const int eb = elt_bytes(cfg->dtype), Hq = cfg->n_q_heads, Hkv = cfg->n_kv_heads, d = cfg->d_qk;
  if ((q_dev && !strides_ok(q_token_stride, q_head_stride, eb)) || !strides_ok(k_token_stride, k_head_stride, eb) ||
      !strides_ok(v_token_stride, v_head_stride, eb))
    return SNAP_ERR_INVALID_ARG;
  // an output that is its own input has to be dense, like the output
  const auto dense = [&](long long tok, long long head, int heads) {
    return (heads == 1 || head == d) && (n_tokens == 1 || tok == (long long)heads * d);
  };
  if ((q_dev && q_dev == q_out_dev && !dense(q_token_stride, q_head_stride, Hq)) ||
      (k_dev == k_out_dev && !dense(k_token_stride, k_head_stride, Hkv)))
    return SNAP_ERR_INVALID_ARG;
  RopeArgs a = {};
  a.q = q_dev; a.q_out = q_out_dev; a.k = k_dev; a.k_out = k_out_dev; a.v = v_dev;
  a.q_tok = q_token_stride; a.q_head = q_head_stride; a.qo_tok = (long long)Hq * d; a.qo_head = d;
  a.k_tok = k_token_stride; a.k_head = k_head_stride; a.ko_tok = (long long)Hkv * d; a.ko_head = d;
  a.v_tok = v_token_stride; a.v_head = v_head_stride;
  a.freqs = freqs_dev; a.positions = positions_dev; a.n_tokens = n_tokens;
  a.Hq = q_dev ? Hq : 0; a.Hkv = Hkv; a.d_qk = d; a.d_v = cfg->d_v;
  a.magnitude = 1.f; a.sign = 1.f;
  if (rope) {
    a.rot = rope->rot_dim; a.offset = rope->rot_offset; a.interleaved = rope->interleaved;
    a.magnitude = (float)rope_magnitude(rope);
  }
  a.k_pages = k_pages_dev; a.v_pages = v_pages_dev; a.slots = slot_ids_dev; a.rows = rows_dev; a.seq_len = seq_len_dev;
  a.weights = weights_dev; a.max_seqs = cfg->max_seqs; a.map = page_map(paged, page_table_dev); a.status = status_dev;
  return status_of(launch_rope(cfg->dtype, a, static_cast<cudaStream_t>(cuda_stream)));
}

int64_t snap_paged_decode_workspace_bytes(const snap_config_t* cfg, const snap_paged_t* paged, int32_t n_active, int32_t with_weights) {
  const int rc = check_paged(cfg, paged, cfg ? elt_bytes(cfg->dtype) : 0);
  if (rc != SNAP_OK) return rc;
  if (n_active < 0) return SNAP_ERR_INVALID_ARG;
  PagedDecodePlan p;
  const int rp = paged_decode_plan(cfg->dtype, make_shape(cfg), page_map(paged, nullptr), n_active, with_weights != 0, sm_count(), &p);
  return rp == SNAP_OK ? (int64_t)p.bytes : rp;
}

int snap_paged_decode_attn(const snap_config_t* cfg, const snap_paged_t* paged, const void* q_dev,
                           const int32_t* slot_ids_dev, int32_t n_active,
                           const void* k_pages_dev, const void* v_pages_dev, const int32_t* page_table_dev,
                           const int32_t* seq_len_dev, const float* weights_in_dev, float* weights_out_dev,
                           void* out_dev, void* workspace_dev, size_t workspace_bytes,
                           uint32_t* status_dev, void* cuda_stream) {
  const int rc = check_paged(cfg, paged, cfg ? elt_bytes(cfg->dtype) : 0);
  if (rc != SNAP_OK) return rc;
  if (n_active < 0) return SNAP_ERR_INVALID_ARG;
  if (n_active == 0) return SNAP_OK;
  if (!q_dev || !slot_ids_dev || !k_pages_dev || !v_pages_dev || !page_table_dev || !seq_len_dev || !out_dev || !workspace_dev ||
      (weights_in_dev && !weights_out_dev))
    return SNAP_ERR_NULL_POINTER;
  if (misaligned(q_dev, k_pages_dev, v_pages_dev, out_dev, workspace_dev)) return SNAP_ERR_INVALID_ARG;
  const Shape s = make_shape(cfg);
  const PageMap m = page_map(paged, page_table_dev);
  PagedDecodePlan p;
  const int rp = paged_decode_plan(cfg->dtype, s, m, n_active, weights_out_dev != nullptr, sm_count(), &p);
  if (rp != SNAP_OK) return rp;
  if (workspace_bytes < p.bytes) return SNAP_ERR_WORKSPACE_TOO_SMALL;
  return status_of(launch_paged_decode(cfg->dtype, s, m, p, q_dev, slot_ids_dev, n_active, k_pages_dev, v_pages_dev, seq_len_dev,
                                       weights_in_dev, weights_out_dev, out_dev, static_cast<char*>(workspace_dev), status_dev,
                                       static_cast<cudaStream_t>(cuda_stream)));
}

int64_t snap_paged_evict_workspace_bytes(const snap_config_t* cfg, const snap_paged_t* paged, int32_t n_seqs) {
  const int rc = check_paged(cfg, paged, cfg ? elt_bytes(cfg->dtype) : 0);
  if (rc != SNAP_OK) return rc;
  if (n_seqs < 0 || n_seqs > 65535) return SNAP_ERR_INVALID_ARG;
  if (!evict_countable(cfg, n_seqs)) return SNAP_ERR_UNSUPPORTED;
  return (int64_t)paged_evict_scratch_bytes(make_shape(cfg), n_seqs);
}

int snap_paged_evict(const snap_config_t* cfg, const snap_paged_t* paged, const int32_t* src_slots_dev,
                     const int32_t* dst_slots_dev, int32_t n_seqs, void* k_pages_dev, void* v_pages_dev,
                     const int32_t* page_table_dev, int32_t* seq_len_dev, const float* weights_in_dev,
                     float* weights_out_dev, int32_t* kept_rows_dev, void* workspace_dev, size_t workspace_bytes,
                     uint32_t* status_dev, void* cuda_stream) {
  const int rc = check_paged(cfg, paged, cfg ? elt_bytes(cfg->dtype) : 0);
  if (rc != SNAP_OK) return rc;
  if (n_seqs < 0 || n_seqs > 65535) return SNAP_ERR_INVALID_ARG;
  if (n_seqs == 0) return SNAP_OK;
  if (!src_slots_dev || !dst_slots_dev || !k_pages_dev || !v_pages_dev || !page_table_dev || !seq_len_dev || !weights_in_dev ||
      !workspace_dev)
    return SNAP_ERR_NULL_POINTER;
  if (misaligned(k_pages_dev, v_pages_dev, workspace_dev)) return SNAP_ERR_INVALID_ARG;
  if (!evict_countable(cfg, n_seqs)) return SNAP_ERR_UNSUPPORTED;
  const Shape s = make_shape(cfg);
  if (workspace_bytes < paged_evict_scratch_bytes(s, n_seqs)) return SNAP_ERR_WORKSPACE_TOO_SMALL;
  return status_of(launch_paged_evict(cfg->dtype, s, page_map(paged, page_table_dev), src_slots_dev, dst_slots_dev, n_seqs, k_pages_dev,
                                      v_pages_dev, seq_len_dev, weights_in_dev, weights_out_dev, kept_rows_dev,
                                      static_cast<char*>(workspace_dev), status_dev, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
