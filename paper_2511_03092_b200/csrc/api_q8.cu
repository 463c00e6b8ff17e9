// Host side of the page plan and of the cache in pages of 8-bit numbers: validation, scratch planning, launches.
#include <climits>
#include <cmath>

#include "snap_internal.cuh"

namespace snap {
namespace {

constexpr int kMaxRequests = 65536;
constexpr int kMaxRowTokens = INT_MAX - 65535; // token numbers of a block's spare places stay within 32 bits

int check_q8(const snap_config_t* cfg, const snap_paged_q8_t* p) {
  const int rc = check_paged(cfg, p ? &p->pages : nullptr, 1);
  if (rc != SNAP_OK) return rc;
  if (p->block_tokens < 1 || p->pages.page_tokens % p->block_tokens || p->reserved != 0) return SNAP_ERR_INVALID_ARG;
  return SNAP_OK;
}

Q8Map q8_map(const snap_paged_q8_t* p, const int* table) {
  return {page_map(&p->pages, table), p->block_tokens, p->pages.page_tokens / p->block_tokens};
}

Q8Rows q8_rows(const snap_config_t* cfg, const snap_paged_q8_t* p, const int* slots, const int* cu, const int* first, int n_seqs,
               int n_tokens, const void* kp, const void* vp, const float* ks, const float* vs, const int* table, uint32_t* status) {
  Q8Rows r;
  r.slots = slots; r.cu = cu; r.first = first; r.n_seqs = n_seqs; r.n_tokens = n_tokens;
  r.Hq = cfg->n_q_heads; r.Hkv = cfg->n_kv_heads; r.d_qk = cfg->d_qk; r.d_v = cfg->d_v; r.max_seqs = cfg->max_seqs;
  r.map = q8_map(p, table);
  r.k_pages = static_cast<uint8_t*>(const_cast<void*>(kp)); r.v_pages = static_cast<uint8_t*>(const_cast<void*>(vp));
  r.k_scales = const_cast<float*>(ks); r.v_scales = const_cast<float*>(vs);
  r.status = status;
  return r;
}

}  // namespace
}  // namespace snap

using namespace snap;

extern "C" {

int64_t snap_paged_plan_workspace_bytes(const snap_config_t* cfg, const snap_paged_t* paged, int32_t n_seqs) {
  const int rc = check_page_counts(cfg, paged);
  if (rc != SNAP_OK) return rc;
  if (n_seqs < 0 || n_seqs > kMaxRequests) return SNAP_ERR_INVALID_ARG;
  return (int64_t)paged_plan_scratch_bytes(cfg->max_seqs, n_seqs);
}

int snap_paged_plan(const snap_config_t* cfg, const snap_paged_t* paged, const int32_t* slot_ids_dev,
                    const int32_t* new_tokens_dev, int32_t n_seqs, const int32_t* page_table_in_dev,
                    int32_t* page_table_out_dev, int32_t* seq_len_dev, int32_t* free_pages_dev,
                    const int32_t* n_free_in_dev, int32_t* n_free_out_dev, int32_t n_tokens_max, int32_t* granted_dev,
                    int32_t* first_rows_dev, int32_t* cu_tokens_dev, int32_t* token_slots_dev, int32_t* token_rows_dev,
                    void* workspace_dev, size_t workspace_bytes, uint32_t* status_dev, void* cuda_stream) {
  const int rc = check_page_counts(cfg, paged);
  if (rc != SNAP_OK) return rc;
  if (n_seqs < 0 || n_seqs > kMaxRequests || n_tokens_max < 0) return SNAP_ERR_INVALID_ARG;
  if (!cu_tokens_dev || !n_free_in_dev || !n_free_out_dev || !workspace_dev ||
      (n_tokens_max > 0 && (!token_slots_dev || !token_rows_dev)) ||
      (n_seqs > 0 && (!slot_ids_dev || !new_tokens_dev || !page_table_in_dev || !page_table_out_dev || !seq_len_dev || !free_pages_dev || !first_rows_dev)))
    return SNAP_ERR_NULL_POINTER;
  if (misaligned(token_slots_dev, token_rows_dev) || misaligned(workspace_dev)) return SNAP_ERR_INVALID_ARG;
  const uintptr_t in = reinterpret_cast<uintptr_t>(page_table_in_dev), out = reinterpret_cast<uintptr_t>(page_table_out_dev),
                  size = sizeof(int32_t) * (uintptr_t)cfg->max_seqs * (uintptr_t)paged->max_pages;
  if (n_seqs > 0 && in != out && (in < out ? out - in : in - out) < size) return SNAP_ERR_INVALID_ARG;   // a row would be read after it was written
  if (workspace_bytes < paged_plan_scratch_bytes(cfg->max_seqs, n_seqs)) return SNAP_ERR_WORKSPACE_TOO_SMALL;
  PlanArgs a = {};
  a.slots = slot_ids_dev; a.new_tokens = new_tokens_dev; a.table_in = page_table_in_dev; a.table_out = page_table_out_dev;
  a.seq_len = seq_len_dev; a.stack = free_pages_dev; a.n_free_in = n_free_in_dev; a.n_free_out = n_free_out_dev;
  a.granted = granted_dev; a.first_rows = first_rows_dev; a.cu = cu_tokens_dev; a.token_slots = token_slots_dev; a.token_rows = token_rows_dev;
  a.n = n_seqs; a.n_tokens_max = n_tokens_max; a.max_seqs = cfg->max_seqs;
  a.page = paged->page_tokens; a.n_pages = paged->n_pages; a.max_pages = paged->max_pages;
  a.scratch = static_cast<char*>(workspace_dev); a.status = status_dev;
  return status_of(launch_paged_plan(a, static_cast<cudaStream_t>(cuda_stream)));
}

int snap_paged_q8_append(const snap_config_t* cfg, const snap_paged_q8_t* paged,
                         const int32_t* slot_ids_dev, const int32_t* cu_tokens_dev, const int32_t* first_rows_dev,
                         int32_t n_seqs, int32_t n_tokens,
                         const snap_rope_config_t* rope, const double* freqs_dev, const int32_t* positions_dev,
                         const void* q_dev, int64_t q_token_stride, int64_t q_head_stride, void* q_out_dev,
                         const void* k_dev, int64_t k_token_stride, int64_t k_head_stride, void* k_out_dev,
                         const void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                         void* k_pages_dev, void* v_pages_dev, float* k_scales_dev, float* v_scales_dev,
                         const int32_t* page_table_dev, int32_t* seq_len_dev, uint32_t* status_dev, void* cuda_stream) {
  int rc = check_q8(cfg, paged);
  if (rc != SNAP_OK) return rc;
  if (rope) {
    rc = check_rope(rope);
    if (rc != SNAP_OK) return rc;
    if (rope->rot_dim > cfg->d_qk - rope->rot_offset) return SNAP_ERR_INVALID_ARG;
  }
  if (n_seqs < 0 || n_seqs > kMaxRequests || n_tokens < 0 || n_tokens > kMaxRowTokens) return SNAP_ERR_INVALID_ARG;
  if (n_seqs == 0 || n_tokens == 0) return SNAP_OK;
  if (!slot_ids_dev || !cu_tokens_dev || !first_rows_dev || !k_dev || !v_dev || !k_pages_dev || !v_pages_dev || !k_scales_dev || !v_scales_dev ||
      !page_table_dev || !seq_len_dev || (rope && !freqs_dev) || !q_dev != !q_out_dev)
    return SNAP_ERR_NULL_POINTER;
  if (misaligned(q_dev, q_out_dev, k_dev, k_out_dev, v_dev, k_pages_dev, v_pages_dev) || first_rows_dev == seq_len_dev) return SNAP_ERR_INVALID_ARG;
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
  Q8AppendArgs a = {};
  a.r = q8_rows(cfg, paged, slot_ids_dev, cu_tokens_dev, first_rows_dev, n_seqs, n_tokens, k_pages_dev, v_pages_dev, k_scales_dev, v_scales_dev,
                page_table_dev, status_dev);
  if (!q_dev) a.r.Hq = 0;
  a.q = q_dev; a.k = k_dev; a.v = v_dev; a.q_out = q_out_dev; a.k_out = k_out_dev;
  a.q_tok = q_token_stride; a.q_head = q_head_stride; a.k_tok = k_token_stride; a.k_head = k_head_stride;
  a.v_tok = v_token_stride; a.v_head = v_head_stride;
  a.freqs = freqs_dev; a.positions = positions_dev; a.seq_len = seq_len_dev;
  a.magnitude = 1.f; a.growth = 1.f;
  if (rope) {
    a.rot = rope->rot_dim; a.offset = rope->rot_offset; a.interleaved = rope->interleaved;
    a.magnitude = (float)rope_magnitude(rope);
    a.growth = std::fmax(1.f, (float)(std::sqrt(2.0) * rope_magnitude(rope)));
  }
  return status_of(launch_q8_append(cfg->dtype, a, static_cast<cudaStream_t>(cuda_stream)));
}

int64_t snap_paged_q8_decode_workspace_bytes(const snap_config_t* cfg, const snap_paged_q8_t* paged, int32_t n_active,
                                             int32_t q_len) {
  const int rc = check_q8(cfg, paged);
  if (rc != SNAP_OK) return rc;
  if (n_active < 0 || q_len < 1 || q_len > 1024) return SNAP_ERR_INVALID_ARG;
  Q8DecodePlan p;
  const int rp = q8_decode_plan(make_shape(cfg), q8_map(paged, nullptr), n_active, q_len, sm_count(), &p);
  return rp == SNAP_OK ? (int64_t)p.bytes : rp;
}

int snap_paged_q8_decode_attn(const snap_config_t* cfg, const snap_paged_q8_t* paged, const void* q_dev,
                              const int32_t* slot_ids_dev, int32_t n_active, int32_t q_len,
                              const void* k_pages_dev, const void* v_pages_dev, const float* k_scales_dev,
                              const float* v_scales_dev, const int32_t* page_table_dev, const int32_t* seq_len_dev,
                              void* out_dev, void* workspace_dev, size_t workspace_bytes, uint32_t* status_dev,
                              void* cuda_stream) {
  const int rc = check_q8(cfg, paged);
  if (rc != SNAP_OK) return rc;
  if (n_active < 0 || q_len < 1 || q_len > 1024) return SNAP_ERR_INVALID_ARG;
  if (n_active == 0) return SNAP_OK;
  if (!q_dev || !slot_ids_dev || !k_pages_dev || !v_pages_dev || !k_scales_dev || !v_scales_dev || !page_table_dev || !seq_len_dev || !out_dev ||
      !workspace_dev)
    return SNAP_ERR_NULL_POINTER;
  if (misaligned(q_dev, k_pages_dev, v_pages_dev, out_dev, workspace_dev)) return SNAP_ERR_INVALID_ARG;
  const Shape s = make_shape(cfg);
  const Q8Map m = q8_map(paged, page_table_dev);
  Q8DecodePlan p;
  const int rp = q8_decode_plan(s, m, n_active, q_len, sm_count(), &p);
  if (rp != SNAP_OK) return rp;
  if (workspace_bytes < p.bytes) return SNAP_ERR_WORKSPACE_TOO_SMALL;
  return status_of(launch_q8_decode(cfg->dtype, s, m, p, q_dev, slot_ids_dev, n_active, q_len, k_pages_dev, v_pages_dev, k_scales_dev, v_scales_dev,
                                    seq_len_dev, out_dev, static_cast<char*>(workspace_dev), status_dev, static_cast<cudaStream_t>(cuda_stream)));
}

int snap_paged_q8_gather(const snap_config_t* cfg, const snap_paged_q8_t* paged,
                         const int32_t* slot_ids_dev, const int32_t* cu_tokens_dev, const int32_t* first_rows_dev,
                         int32_t n_seqs, int32_t n_tokens,
                         const void* k_pages_dev, const void* v_pages_dev, const float* k_scales_dev, const float* v_scales_dev,
                         const int32_t* page_table_dev,
                         void* k_dev, int64_t k_token_stride, int64_t k_head_stride,
                         void* v_dev, int64_t v_token_stride, int64_t v_head_stride,
                         uint32_t* status_dev, void* cuda_stream) {
  const int rc = check_q8(cfg, paged);
  if (rc != SNAP_OK) return rc;
  if (n_seqs < 0 || n_seqs > kMaxRequests || n_tokens < 0 || n_tokens > kMaxRowTokens) return SNAP_ERR_INVALID_ARG;
  if (n_seqs == 0 || n_tokens == 0) return SNAP_OK;
  if (!slot_ids_dev || !cu_tokens_dev || !first_rows_dev || !k_pages_dev || !v_pages_dev || !k_scales_dev || !v_scales_dev || !page_table_dev ||
      !k_dev || !v_dev)
    return SNAP_ERR_NULL_POINTER;
  if (misaligned(k_dev, v_dev, k_pages_dev, v_pages_dev)) return SNAP_ERR_INVALID_ARG;
  const int eb = elt_bytes(cfg->dtype);
  if (!out_strides_ok(k_token_stride, k_head_stride, n_tokens, cfg->n_kv_heads, cfg->d_qk, eb) ||
      !out_strides_ok(v_token_stride, v_head_stride, n_tokens, cfg->n_kv_heads, cfg->d_v, eb))
    return SNAP_ERR_INVALID_ARG;
  Q8GatherArgs a;
  a.r = q8_rows(cfg, paged, slot_ids_dev, cu_tokens_dev, first_rows_dev, n_seqs, n_tokens, k_pages_dev, v_pages_dev, k_scales_dev, v_scales_dev,
                page_table_dev, status_dev);
  a.k = k_dev; a.v = v_dev; a.k_tok = k_token_stride; a.k_head = k_head_stride; a.v_tok = v_token_stride; a.v_head = v_head_stride;
  return status_of(launch_q8_gather(cfg->dtype, a, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
