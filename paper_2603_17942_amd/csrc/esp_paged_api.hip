// C ABI of the paged KV cache: argument validation.
#include <algorithm>
#include <cmath>

#include "esp_paged.h"

namespace {

#define ESP_HIP(expr)                          \
  do {                                         \
    hipError_t e__ = (expr);                   \
    if (e__ != hipSuccess) return ESP_EDEVICE; \
  } while (0)

inline size_t elt(int dtype) { return dtype == ESP_F32 ? 4 : 2; }

esp_status check_paged(const esp_paged_kv* kv) {
  if (!kv || !kv->k || !kv->v || !kv->page_table || !kv->len) return ESP_EINVAL;
  if (kv->dtype != ESP_F32 && kv->dtype != ESP_BF16) return ESP_EDTYPE;
  if (kv->n_layers < 1 || kv->n_kv_heads < 1 || kv->page_size < 1 || kv->n_pages < 1 || kv->batch < 1 || kv->table_stride < 1 || kv->len_bound < 0)
    return ESP_EINVAL;
  if ((uintptr_t)kv->k % 16 || (uintptr_t)kv->v % 16) return ESP_EINVAL;
  if (kv->head_dim != 64 && kv->head_dim != 128) return ESP_ESHAPE;
  if (kv->page_size % 32) return ESP_ESHAPE;
  // places are counted in blocks of 32 slots, and slots of a sequence, in 31 bits
  if ((int64_t)kv->n_pages * kv->n_kv_heads > INT32_MAX / (kv->page_size / 32)) return ESP_ECAPACITY;
  if ((int64_t)kv->table_stride * kv->page_size > INT32_MAX) return ESP_ECAPACITY;
  if (kv->n_layers > 65535 || kv->batch > 65535 || (int64_t)kv->n_layers * kv->n_kv_heads > MOST_WORKGROUPS) return ESP_ECAPACITY;
  return ESP_OK;
}
esp_status check_chunk(const esp_paged_kv* kv, const esp_chunk* c) {
  if (!c || !c->row0 || c->total_rows < 0 || c->max_rows < 0) return ESP_EINVAL;
  if ((int64_t)kv->len_bound + c->max_rows > INT32_MAX - 65536) return ESP_ECAPACITY;
  return ESP_OK;
}
PagedDev to_dev(const esp_paged_kv* kv, int layer) {
  const size_t off = (size_t)layer * kv->n_pages * kv->n_kv_heads * kv->page_size * kv->head_dim * elt(kv->dtype);
  return {(char*)kv->k + off, (char*)kv->v + off, kv->page_table, kv->len, kv->status, kv->n_kv_heads, kv->page_size, kv->n_pages,
          kv->batch, kv->table_stride, kv->len_bound};
}
// four rows a workgroup; pieces and elements of four rows are counted in 31 bits
bool too_many(int64_t heads, int64_t rows) { return rows > 4 * MOST_WORKGROUPS || heads * std::max<int64_t>(rows, 512) > INT32_MAX; }
// columns of a sequence and kv head are counted in 31 bits
bool too_many_columns(const esp_paged_kv* kv, const esp_chunk* c, int n_q) { return (int64_t)c->max_rows * (n_q / kv->n_kv_heads) > INT32_MAX / 2; }
bool bad_eps(float eps) { return !(eps >= 0.f) || !std::isfinite(eps); }
// (may be null: no rotation)
esp_status check_rope(const esp_rope* r) {
  if (!r) return ESP_OK;
  if (r->head_dim != 64 && r->head_dim != 128) return ESP_ESHAPE;
  if (r->rot_dim < 16 || r->rot_dim > r->head_dim || r->rot_dim % 16) return ESP_ESHAPE;
  if (!std::isfinite(r->amplitude)) return ESP_EINVAL;
  return ESP_OK;
}
void take_rope(RopeRows& a, const esp_rope* r) {
  a.rot = r ? r->rot_dim : 0;
  a.interleaved = r ? r->interleaved != 0 : 0;
  a.amplitude = r ? r->amplitude : 1.f;
  for (int i = 0; i < 64; ++i) a.turns[i] = i < a.rot / 2 ? r->turns[i] : 0.0;
}

}  // namespace

extern "C" {

esp_status esp_rope_make(int32_t head_dim, int32_t rot_dim, int32_t interleaved, double theta, double factor, int32_t orig_len,
                         double low_turns, double high_turns, double amplitude, esp_rope* out) {
  if (!out) return ESP_EINVAL;
  if (head_dim != 64 && head_dim != 128) return ESP_ESHAPE;
  if (rot_dim < 16 || rot_dim > head_dim || rot_dim % 16) return ESP_ESHAPE;
  if (!(theta > 0) || !std::isfinite(theta) || !(factor > 0) || !std::isfinite(factor) || orig_len < 0 || !std::isfinite((float)amplitude))
    return ESP_EINVAL;
  if (orig_len > 0 && !(std::isfinite(low_turns) && std::isfinite(high_turns - low_turns) && low_turns < high_turns)) return ESP_EINVAL;
  const double two_pi = 6.283185307179586476925286766559;
  esp_rope r{};
  r.head_dim = head_dim; r.rot_dim = rot_dim; r.interleaved = interleaved != 0; r.amplitude = (float)amplitude;
  for (int i = 0; i < rot_dim / 2; ++i) {
    const double f = std::pow(theta, -2.0 * i / rot_dim) / two_pi;
    const double keep = orig_len > 0 ? std::min(1.0, std::max(0.0, (orig_len * f - low_turns) / (high_turns - low_turns))) : 0.0;
    r.turns[i] = f * (keep + (1.0 - keep) / factor);
    if (!std::isfinite(r.turns[i])) return ESP_EINVAL;
  }
  *out = r;
  return ESP_OK;
}

esp_status esp_rope_qk(void* stream, int32_t dtype, const esp_rope* rope, int32_t rows, int32_t n_q, int32_t n_kv, const void* q,
                       int64_t q_stride, const void* k, int64_t k_stride, const int32_t* positions, const void* q_gain, const void* k_gain,
                       float eps, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride) {
  if (!rope || !positions || rows < 0 || (!q && !k) || !q != !q_out || !k != !k_out || bad_eps(eps)) return ESP_EINVAL;
  if (dtype != ESP_F32 && dtype != ESP_BF16) return ESP_EDTYPE;
  if ((q && n_q < 1) || (k && n_kv < 1)) return ESP_EINVAL;
  const esp_status st = check_rope(rope);
  if (st != ESP_OK) return st;
  const int hd = rope->head_dim;
  if (q && (q_stride < (int64_t)n_q * hd || q_out_stride < (int64_t)n_q * hd)) return ESP_ESHAPE;
  if (k && (k_stride < (int64_t)n_kv * hd || k_out_stride < (int64_t)n_kv * hd)) return ESP_ESHAPE;
  if ((q == q_out && q && q_stride != q_out_stride) || (k == k_out && k && k_stride != k_out_stride)) return ESP_EINVAL;
  if (too_many((int64_t)(q ? n_q : 0) + (k ? n_kv : 0), rows)) return ESP_ECAPACITY;
  if (rows == 0) return ESP_OK;
  RopeRows a{};
  a.q = q; a.k = k; a.q_stride = q_stride; a.k_stride = k_stride; a.q_out = q_out; a.k_out = k_out;
  a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride; a.q_gain = q_gain; a.k_gain = k_gain;
  a.positions = positions; a.eps = eps; a.rows = rows; a.hq = q ? n_q : 0; a.hkv = k ? n_kv : 0;
  take_rope(a, rope);
  ESP_HIP(launch_rope_rows((hipStream_t)stream, dtype, hd, a));
  return ESP_OK;
}

esp_status esp_paged_append(void* stream, const esp_paged_kv* kv, int32_t layer, const esp_chunk* rows, const esp_rope* rope,
                            const int32_t* positions, int32_t n_q, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                            const void* v, int64_t v_stride, const void* q_gain, const void* k_gain, float eps, void* q_out,
                            int64_t q_out_stride) {
  esp_status st = check_paged(kv);
  if (st != ESP_OK) return st;
  st = check_chunk(kv, rows);
  if (st != ESP_OK) return st;
  if (layer < 0 || layer >= kv->n_layers || !k || !v || !q != !q_out || (q && n_q < 1) || bad_eps(eps)) return ESP_EINVAL;
  st = check_rope(rope);
  if (st != ESP_OK) return st;
  const int hd = kv->head_dim, hkv = kv->n_kv_heads;
  if (rope && rope->head_dim != hd) return ESP_ESHAPE;
  if (q && (q_stride < (int64_t)n_q * hd || q_out_stride < (int64_t)n_q * hd)) return ESP_ESHAPE;
  if (k_stride < (int64_t)hkv * hd || v_stride < (int64_t)hkv * hd) return ESP_ESHAPE;
  if (q && q == q_out && q_stride != q_out_stride) return ESP_EINVAL;
  if (too_many((int64_t)(q ? n_q : 0) + 2 * (int64_t)hkv, rows->total_rows)) return ESP_ECAPACITY;
  if (rows->total_rows == 0 || rows->max_rows == 0) return ESP_OK;
  RopeRows a{};
  a.q = q; a.k = k; a.v = v; a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride;
  a.q_out = q_out; a.q_out_stride = q_out_stride; a.q_gain = q_gain; a.k_gain = k_gain;
  a.positions = positions; a.eps = eps; a.rows = rows->total_rows; a.hq = q ? n_q : 0; a.hkv = hkv;
  take_rope(a, rope);
  ESP_HIP(launch_paged_append((hipStream_t)stream, kv->dtype, hd, to_dev(kv, layer), {rows->row0, rows->total_rows, rows->max_rows}, a));
  return ESP_OK;
}

size_t esp_paged_attn_scratch_bytes(const esp_paged_kv* kv, const esp_chunk* rows, int32_t n_q) {
  if (check_paged(kv) != ESP_OK || check_chunk(kv, rows) != ESP_OK || n_q < 1 || n_q % kv->n_kv_heads) return 0;
  if (rows->total_rows == 0 || rows->max_rows == 0) return 0;
  const PagedAttnPlan p = paged_attn_plan(kv->dtype, kv->head_dim, kv->batch, n_q, kv->n_kv_heads, rows->total_rows, rows->max_rows, kv->len_bound);
  return paged_attn_partial_floats(p, kv->head_dim) * 4;
}

esp_status esp_paged_attn(void* stream, const esp_paged_kv* kv, int32_t layer, const esp_chunk* rows, int32_t n_q, const void* q,
                          int64_t q_stride, float scale, const uint64_t* anc, int32_t anc_words, void* out, void* scratch,
                          size_t scratch_bytes) {
  esp_status st = check_paged(kv);
  if (st != ESP_OK) return st;
  st = check_chunk(kv, rows);
  if (st != ESP_OK) return st;
  // a hidden key's score is -1e30: with less than this as scale its exponent would not be out of range
  if (layer < 0 || layer >= kv->n_layers || n_q < 1 || !q || !out || !(scale >= 1e-20f) || !std::isfinite(scale)) return ESP_EINVAL;
  if (n_q % kv->n_kv_heads) return ESP_ESHAPE;
  if (q_stride < (int64_t)n_q * kv->head_dim) return ESP_ESHAPE;
  if (anc && (int64_t)anc_words * 64 < rows->max_rows) return ESP_ESHAPE;
  if (too_many_columns(kv, rows, n_q)) return ESP_ECAPACITY;
  if (rows->total_rows == 0 || rows->max_rows == 0) return ESP_OK;
  const PagedAttnPlan p = paged_attn_plan(kv->dtype, kv->head_dim, kv->batch, n_q, kv->n_kv_heads, rows->total_rows, rows->max_rows, kv->len_bound);
  if (paged_attn_workgroups(p, kv->batch, kv->n_kv_heads) > MOST_WORKGROUPS) return ESP_ECAPACITY;
  const size_t need = paged_attn_partial_floats(p, kv->head_dim) * 4;
  if (need && (!scratch || scratch_bytes < need)) return ESP_ECAPACITY;
  if (need && (uintptr_t)scratch % 16) return ESP_EINVAL;
  PagedAttnArgs a{q, q_stride, out, anc, anc_words, n_q, scale, (float*)scratch};
  ESP_HIP(launch_paged_attn((hipStream_t)stream, kv->dtype, kv->head_dim, to_dev(kv, layer), {rows->row0, rows->total_rows, rows->max_rows}, a, p));
  return ESP_OK;
}

esp_status esp_paged_commit(void* stream, const esp_paged_kv* kv, const int32_t* n_emit, const int32_t* accepted_row, int32_t* len_out) {
  const esp_status st = check_paged(kv);
  if (st != ESP_OK) return st;
  if (!n_emit || !accepted_row || !len_out) return ESP_EINVAL;
  ESP_HIP(launch_paged_commit((hipStream_t)stream, kv->dtype, kv->head_dim, to_dev(kv, 0), kv->n_layers, n_emit, accepted_row, len_out));
  return ESP_OK;
}

esp_status esp_paged_load(void* stream, const esp_paged_kv* kv, int32_t layer, int32_t seq, int32_t first_slot, int32_t n_slots, void* k_rows,
                          void* v_rows) {
  const esp_status st = check_paged(kv);
  if (st != ESP_OK) return st;
  if (layer < 0 || layer >= kv->n_layers || seq < 0 || seq >= kv->batch || first_slot < 0 || n_slots < 0 || !k_rows || !v_rows) return ESP_EINVAL;
  if ((int64_t)first_slot + n_slots > (int64_t)kv->table_stride * kv->page_size) return ESP_ECAPACITY;
  ESP_HIP(launch_paged_load((hipStream_t)stream, kv->dtype, kv->head_dim, to_dev(kv, layer), seq, first_slot, n_slots, k_rows, v_rows));
  return ESP_OK;
}

size_t esp_paged_weigh_scratch_bytes(const esp_paged_kv* kv, const esp_chunk* rows, int32_t n_q, int32_t last_rows) {
  if (check_paged(kv) != ESP_OK || check_chunk(kv, rows) != ESP_OK || n_q < 1 || n_q % kv->n_kv_heads || last_rows < 0) return 0;
  if (rows->total_rows == 0 || rows->max_rows == 0 || too_many_columns(kv, rows, n_q)) return 0;
  const WeighPlan p = weigh_plan(kv->dtype, kv->batch, n_q, kv->n_kv_heads, rows->total_rows, rows->max_rows, last_rows, kv->len_bound);
  return (size_t)p.scratch_floats * 4;
}

esp_status esp_paged_weigh(void* stream, const esp_paged_kv* kv, int32_t layer, const esp_chunk* rows, int32_t n_q, const void* q, int64_t q_stride,
                           float scale, int32_t last_rows, const float* before, float* mass, int32_t mass_slots, void* scratch,
                           size_t scratch_bytes) {
  esp_status st = check_paged(kv);
  if (st != ESP_OK) return st;
  st = check_chunk(kv, rows);
  if (st != ESP_OK) return st;
  if (layer < 0 || layer >= kv->n_layers || n_q < 1 || !q || !mass || mass_slots < 1 || last_rows < 0 || !(scale >= 1e-20f) || !std::isfinite(scale))
    return ESP_EINVAL;
  if (n_q % kv->n_kv_heads) return ESP_ESHAPE;
  if (q_stride < (int64_t)n_q * kv->head_dim) return ESP_ESHAPE;
  if (kv->n_kv_heads > 65535 || too_many_columns(kv, rows, n_q)) return ESP_ECAPACITY;
  if (rows->total_rows == 0 || rows->max_rows == 0) return ESP_OK;
  const WeighPlan p = weigh_plan(kv->dtype, kv->batch, n_q, kv->n_kv_heads, rows->total_rows, rows->max_rows, last_rows, kv->len_bound);
  if (weigh_workgroups(p, kv->batch, kv->n_kv_heads, n_q / kv->n_kv_heads) > MOST_WORKGROUPS) return ESP_ECAPACITY;
  const size_t need = (size_t)p.scratch_floats * 4;
  if (!scratch || scratch_bytes < need) return ESP_ECAPACITY;
  if ((uintptr_t)scratch % 16) return ESP_EINVAL;
  const int64_t off = (int64_t)layer * kv->batch * kv->n_kv_heads * mass_slots;
  const WeighArgs a{q, q_stride, before ? before + off : nullptr, mass + off, (float*)scratch, n_q, last_rows, mass_slots,
                    (float)((double)scale * 1.4426950408889634), (uintptr_t)q % 16 == 0 && q_stride * (int64_t)elt(kv->dtype) % 16 == 0};
  ESP_HIP(launch_paged_weigh((hipStream_t)stream, kv->dtype, kv->head_dim, to_dev(kv, layer), {rows->row0, rows->total_rows, rows->max_rows}, a, p));
  return ESP_OK;
}

esp_status esp_paged_evict(void* stream, const esp_paged_kv* kv, const float* mass, int32_t mass_slots, int32_t keep, int32_t first, int32_t recent,
                           const int32_t* table_out, int32_t table_out_stride, float* mass_out, int32_t mass_out_slots, int32_t* len_out,
                           int32_t* kept) {
  const esp_status st = check_paged(kv);
  if (st != ESP_OK) return st;
  if (!mass || !table_out || !mass_out || !len_out || !kept || mass_slots < 1 || mass_out_slots < 1 || table_out_stride < 1 || keep < 1 || first < 0 ||
      recent < 0 || (int64_t)first + recent > keep)
    return ESP_EINVAL;
  if ((mass == mass_out && mass_slots != mass_out_slots) || (table_out == kv->page_table && table_out_stride != kv->table_stride)) return ESP_EINVAL;
  if (keep > INT32_MAX - 65536 || kv->len_bound > INT32_MAX - 65536 || mass_out_slots < keep || (int64_t)table_out_stride * kv->page_size < keep) return ESP_ECAPACITY;
  // four times 256 threads a layer, sequence and kv head
  if (kv->n_kv_heads > 65535 || (int64_t)kv->n_layers * kv->batch * kv->n_kv_heads > MOST_WORKGROUPS / 4) return ESP_ECAPACITY;
  const EvictArgs a{mass, mass_out, table_out, len_out, kept, kv->n_layers, mass_slots, mass_out_slots, table_out_stride, keep, first, recent};
  ESP_HIP(launch_paged_evict((hipStream_t)stream, kv->dtype, kv->head_dim, to_dev(kv, 0), a));
  return ESP_OK;
}

}  // extern "C"
