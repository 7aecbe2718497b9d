// Internal declarations of the paged KV cache: device-side views, launchers.
#pragma once

#include "esp_internal.h"

struct PagedDev {             // of one layer
  void *k, *v;
  const int32_t *table, *len;
  int32_t* status;
  int hkv, page_size, n_pages, batch, stride, len_bound;
};
struct ChunkDev {
  const int32_t* row0;
  int total, max_rows;
};
// a sequence's rows and length; ok: they fit each other, the buffers and the table
struct ChunkSeq { int row0, rows, len; bool ok; };
__device__ __forceinline__ bool chunk_rows_ok(const ChunkDev& ch, int a, int b) {
  const int64_t rows = (int64_t)b - a;
  return (a >= 0) & (rows >= 0) & (rows <= ch.max_rows) & (b <= ch.total);
}
__device__ __forceinline__ ChunkSeq chunk_seq(const PagedDev& kv, const ChunkDev& ch, int seq) {
  const int a = ch.row0[seq], b = ch.row0[seq + 1], len = kv.len[seq];
  const int64_t rows = (int64_t)b - a;
  const bool rows_ok = chunk_rows_ok(ch, a, b);
  const bool len_ok = (len >= 0) & (len <= kv.len_bound) & ((int64_t)len + rows <= (int64_t)kv.stride * kv.page_size);
  return {a, (int)rows, len, rows_ok && len_ok};
}
// the bits that belong to a sequence that is not ok
__device__ __forceinline__ int chunk_fault(const ChunkDev& ch, int seq) {
  return chunk_rows_ok(ch, ch.row0[seq], ch.row0[seq + 1]) ? ESP_DEV_LEN_OVER_BOUND : ESP_DEV_BAD_ROWS;
}
__device__ __forceinline__ void set_status(int32_t* status, int bits) {
  if (status) atomicOr(status, bits);
}
// first element of a page's plane
__host__ __device__ __forceinline__ size_t page_plane(int page, int kvh, int hkv, int page_size, int hd) {
  return ((size_t)page * hkv + kvh) * page_size * hd;
}

// workgroups of 256 threads that a launch can have: threads are counted in 32 bits
constexpr int64_t MOST_WORKGROUPS = (1 << 24) - 1;

struct RopeRows {             // what the row kernels are told
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
  void *q_out, *k_out;
  const void *q_gain, *k_gain;
  const int32_t* positions;
  float eps, amplitude;
  int rows, hq, hkv;          // heads of q, and of k and of v; 0: not there
  int rot, interleaved;       // rot 0: no rotation
  double turns[64];
};
hipError_t launch_rope_rows(hipStream_t st, int dtype, int hd, const RopeRows& a);
hipError_t launch_paged_append(hipStream_t st, int dtype, int hd, const PagedDev& kv, const ChunkDev& ch, const RopeRows& a);
hipError_t launch_paged_commit(hipStream_t st, int dtype, int hd, const PagedDev& kv, int layers, const int32_t* n_emit,
                               const int32_t* accepted, int32_t* len_out);
hipError_t launch_paged_load(hipStream_t st, int dtype, int hd, const PagedDev& kv, int seq, int first_slot, int n_slots, void* k_rows,
                             void* v_rows);

struct PagedAttnPlan {
  int cap = 1;                // column tiles of an item at most; 1: k_paged_stream
  int q_tiles = 1;            // items of a sequence and kv head at most
  int shares = 0;             // 0: a workgroup an item
  int least = 1;              // key tiles of a share at least
};
PagedAttnPlan paged_attn_plan(int dtype, int hd, int batch, int hq, int hkv, int total_rows, int max_rows, int len_bound);
int64_t paged_attn_workgroups(const PagedAttnPlan& p, int batch, int hkv);
size_t paged_attn_partial_floats(const PagedAttnPlan& p, int hd);
struct PagedAttnArgs {
  const void* q;
  int64_t q_stride;
  void* out;
  const uint64_t* anc;        // null: causal
  int anc_words, hq;
  float scale;                // with log2 e
  float* partials;
};
hipError_t launch_paged_attn(hipStream_t st, int dtype, int hd, const PagedDev& kv, const ChunkDev& ch, const PagedAttnArgs& a,
                             const PagedAttnPlan& p);

struct WeighPlan {
  int width = 0;              // columns that scores are kept for; 0: many, scores are computed twice
  int share_units = 1, shares = 1;       // units of 32 keys of a share of the statistics
  int parts = 1;              // many: of the columns, each with sums of its own
  bool join_here = false;     // many: the shares' statistics are joined where they are used
  int most_rows = 0;          // counted rows of a sequence at most
  bool packed = false;        // many: statistics lie by rows of the chunk, not by most_rows a sequence
  int64_t tokens = 0;         // of a sequence at most, in whole units
  int64_t columns = 0;        // many: of a share's statistics
  int64_t stats_floats = 0, scratch_floats = 0;
};
struct WeighArgs {
  const void* q;
  int64_t q_stride;
  const float* before;        // of the layer, as mass; null: nothing
  float* mass;
  float* scratch;
  int hq, last, slots;        // slots: of a sequence and kv head in mass
  float scale;                // with log2 e
  bool whole;                 // q can be read 16 bytes at a time
};
WeighPlan weigh_plan(int dtype, int batch, int hq, int hkv, int total_rows, int max_rows, int last, int len_bound);
int64_t weigh_workgroups(const WeighPlan& p, int batch, int hkv, int G);
hipError_t launch_paged_weigh(hipStream_t st, int dtype, int hd, const PagedDev& kv, const ChunkDev& ch, const WeighArgs& a, const WeighPlan& p);

struct EvictArgs {
  const float* mass;
  float* mass_out;
  const int32_t* table_out;
  int32_t *len_out, *kept;
  int layers, slots, out_slots, out_stride, keep, first, recent;
};
hipError_t launch_paged_evict(hipStream_t st, int dtype, int hd, const PagedDev& kv, const EvictArgs& a);
