// C entry points of the operators over the paged cache: argument checks, then the launchers.
#include <math.h>

#include "attn_paged.cuh"
#include "cache_ops.cuh"
#include "gemm_tc.cuh"

using namespace hyp;

namespace {

bool shape_ok(const hyp_attn_shape* s) {
  if (!s || s->n_kv_heads < 1 || s->n_kv_heads > 65535 || s->n_q_heads < s->n_kv_heads || s->n_q_heads % s->n_kv_heads) return false;
  const int G = s->n_q_heads / s->n_kv_heads;
  return (G == 1 || G == 2 || G == 4 || G == 8) && (s->head_dim == 64 || s->head_dim == 128);
}
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
// Pages of a table row: token positions stay below 2^30, so that a position plus a tile never leaves 32 bits.
bool pages_ok(int32_t n) { return n >= 1 && n <= (1 << 26); }
// Sequences and groups: a dimension of the grid.
bool count_ok(int32_t n) { return n >= 1 && n <= 65535; }
bool mod_ok(const hyp_attn_mod* m) {
  // the cap's powers stay within fp32 and its rounding below that of the scores
  if (!m || !(m->softcap == 0.f || (m->softcap >= 0x1p-10f && m->softcap <= 0x1p20f))) return false;
  return m->window >= 0 && aligned(m->slopes, 4) && aligned(m->prefix_lens, 4);
}
bool query_ok(const hyp_attn_shape* s, const void* q, int64_t q_stride, const void* out) {
  return q && out && q_stride >= (int64_t)s->n_q_heads * s->head_dim && q_stride % 8 == 0 && aligned(q, 16) && aligned(out, 16);
}
CacheView view(const hyp_attn_shape* s, int32_t n_seqs, const void* pool, const int32_t* table, int32_t table_stride, const int32_t* ctx) {
  return CacheView{(const __half*)pool, table, table_stride, ctx, n_seqs, s->n_q_heads, s->n_kv_heads, s->head_dim};
}
int finish(int rc) {
  if (rc < 0) return rc;
  cudaError_t e = cudaPeekAtLastError();
  if (e != cudaSuccess) {
    set_last_cuda_error((int)e);
    return HYP_ECUDA;
  }
  return HYP_OK;
}

}  // namespace

extern "C" size_t hyp_op_attn_mod_scratch_bytes(const hyp_attn_shape* shape, int32_t n_seqs, int32_t max_pages_per_seq) {
  if (!shape_ok(shape) || !count_ok(n_seqs) || !pages_ok(max_pages_per_seq)) return 0;
  return 4 * paged_scratch_floats(n_seqs, shape->n_q_heads, shape->head_dim,
                                  paged_splits(n_seqs, shape->n_kv_heads, max_pages_per_seq));
}

extern "C" int hyp_op_attn_decode_mod(const hyp_attn_shape* shape, const hyp_attn_mod* mod, int32_t n_seqs, const void* q,
                                      int64_t q_stride, const void* kv_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                                      const int32_t* ctx_lens, void* scratch, size_t scratch_bytes, void* out, void* stream) {
  if (!shape_ok(shape) || !mod_ok(mod) || !query_ok(shape, q, q_stride, out)) return HYP_EINVAL;
  if (!kv_pages || !block_table || !ctx_lens || !scratch || !count_ok(n_seqs) || !pages_ok(max_pages_per_seq)) return HYP_EINVAL;
  if (!aligned(kv_pages, 16) || !aligned(scratch, 16)) return HYP_EINVAL;
  if (scratch_bytes < hyp_op_attn_mod_scratch_bytes(shape, n_seqs, max_pages_per_seq)) return HYP_ECAPACITY;
  const int rc = tc_prepare();
  if (rc) return rc;
  return finish(launch_decode_mod(view(shape, n_seqs, kv_pages, block_table, max_pages_per_seq, ctx_lens), *mod, (const __half*)q,
                                  q_stride, (float*)scratch, (__half*)out, tc_err_flag_ptr(), (cudaStream_t)stream));
}

extern "C" int hyp_op_attn_prefill_mod(const hyp_attn_shape* shape, const hyp_attn_mod* mod, int32_t n_seqs, int32_t M, const void* q,
                                       int64_t q_stride, const void* kv_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                                       const int32_t* cu_q, const int32_t* ctx_lens, void* out, void* stream) {
  if (!shape_ok(shape) || !mod_ok(mod) || !query_ok(shape, q, q_stride, out)) return HYP_EINVAL;
  if (!kv_pages || !block_table || !cu_q || !ctx_lens || n_seqs < 1 || M < 1 || M > (1 << 26) || !pages_ok(max_pages_per_seq)) return HYP_EINVAL;
  if (!aligned(kv_pages, 16)) return HYP_EINVAL;
  const int rc = tc_prepare();
  if (rc) return rc;
  return finish(launch_prefill_mod(view(shape, n_seqs, kv_pages, block_table, max_pages_per_seq, ctx_lens), *mod, M, (const __half*)q,
                                   q_stride, cu_q, (__half*)out, tc_err_flag_ptr(), (cudaStream_t)stream));
}

extern "C" size_t hyp_op_attn_scored_scratch_bytes(const hyp_attn_shape* shape, int32_t n_seqs, int32_t max_pages_per_seq) {
  if (!shape_ok(shape) || !count_ok(n_seqs) || !pages_ok(max_pages_per_seq)) return 0;
  return 4 * (scored_scores_offset(n_seqs, shape->n_q_heads, shape->n_kv_heads, shape->head_dim, max_pages_per_seq) +
              (size_t)n_seqs * shape->n_q_heads * 16 * (size_t)max_pages_per_seq);
}

extern "C" int hyp_op_attn_decode_scored(const hyp_attn_shape* shape, int32_t n_seqs, const void* q, int64_t q_stride,
                                         const void* kv_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                                         const int32_t* ctx_lens, float decay, const float* weights_in, float* weights_out,
                                         int64_t weights_stride, void* scratch, size_t scratch_bytes, void* out, void* stream) {
  if (!shape_ok(shape) || !query_ok(shape, q, q_stride, out)) return HYP_EINVAL;
  if (!kv_pages || !block_table || !ctx_lens || !weights_out || !scratch || !count_ok(n_seqs) || !pages_ok(max_pages_per_seq)) return HYP_EINVAL;
  if (!aligned(kv_pages, 16) || !aligned(scratch, 16) || !aligned(weights_in, 4) || !aligned(weights_out, 4)) return HYP_EINVAL;
  if (!isfinite(decay) || weights_stride < 16 * (int64_t)max_pages_per_seq) return HYP_EINVAL;
  if (scratch_bytes < hyp_op_attn_scored_scratch_bytes(shape, n_seqs, max_pages_per_seq)) return HYP_ECAPACITY;
  const int rc = tc_prepare();
  if (rc) return rc;
  return finish(launch_decode_scored(view(shape, n_seqs, kv_pages, block_table, max_pages_per_seq, ctx_lens), (const __half*)q, q_stride,
                                     decay, weights_in, weights_out, weights_stride, (float*)scratch, (__half*)out,
                                     tc_err_flag_ptr(), (cudaStream_t)stream));
}

extern "C" int hyp_op_kv_evict(const hyp_attn_shape* shape, int32_t n_seqs, const void* kv_pages, const int32_t* block_table,
                               int32_t max_pages_per_seq, const int32_t* n_cached, const float* weights_in, int64_t weights_stride,
                               int32_t n_keep, int32_t n_sink, int32_t n_recent, void* dst_pages, const int32_t* dst_table,
                               int32_t dst_pages_per_seq, int32_t* kept, int32_t* new_lens, float* weights_out,
                               int64_t weights_out_stride, void* stream) {
  if (!shape_ok(shape) || !kv_pages || !block_table || !n_cached || !weights_in || !dst_pages || !dst_table || !kept || !new_lens || !weights_out)
    return HYP_EINVAL;
  if (!count_ok(n_seqs) || shape->n_kv_heads > 32767 || !pages_ok(max_pages_per_seq) || !pages_ok(dst_pages_per_seq)) return HYP_EINVAL;
  if (n_keep < 1 || n_sink < 0 || n_recent < 0 || n_sink > n_keep || n_recent > n_keep - n_sink) return HYP_EINVAL;
  if (16 * (int64_t)dst_pages_per_seq < n_keep || weights_stride < 16 * (int64_t)max_pages_per_seq || weights_out_stride < n_keep) return HYP_EINVAL;
  if (!aligned(kv_pages, 16) || !aligned(dst_pages, 16) || !aligned(weights_in, 4) || !aligned(weights_out, 4)) return HYP_EINVAL;
  const bool in_place = kv_pages == dst_pages && block_table == dst_table;
  if (in_place && dst_pages_per_seq != max_pages_per_seq) return HYP_EINVAL;
  if (weights_in == weights_out && weights_stride != weights_out_stride) return HYP_EINVAL;
  if (new_lens == n_cached) return HYP_EINVAL;  // the lengths are read until the last row has moved
  EvictArgs a{};
  a.pool = (const __half*)kv_pages; a.table = block_table; a.table_stride = max_pages_per_seq; a.cached = n_cached;
  a.w_in = weights_in; a.w_stride = weights_stride;
  a.n_keep = n_keep; a.n_sink = n_sink; a.n_recent = n_recent;
  a.dst = (__half*)dst_pages; a.dst_table = dst_table; a.dst_stride = dst_pages_per_seq;
  a.kept = kept; a.new_lens = new_lens; a.w_out = weights_out; a.w_out_stride = weights_out_stride;
  a.n_seqs = n_seqs; a.Hkv = shape->n_kv_heads; a.D = shape->head_dim; a.in_place = in_place;
  return finish(launch_kv_evict(a, (cudaStream_t)stream));
}

extern "C" size_t hyp_op_attn_shared_scratch_bytes(const hyp_attn_shape* shape, int32_t n_seqs, int32_t n_groups,
                                                   int32_t max_prefix_pages, int32_t max_pages_per_seq) {
  if (!shape_ok(shape) || !count_ok(n_seqs) || !count_ok(n_groups) || !pages_ok(max_prefix_pages) || !pages_ok(max_pages_per_seq)) return 0;
  const SharedPlan p = shared_plan(n_seqs, shape->n_q_heads, shape->n_kv_heads, shape->head_dim, n_groups, max_prefix_pages, max_pages_per_seq);
  return 4 * paged_scratch_floats(n_seqs, shape->n_q_heads, shape->head_dim, p.prefix_splits + p.own_splits);
}

extern "C" int hyp_op_attn_decode_shared(const hyp_attn_shape* shape, int32_t n_seqs, const void* q, int64_t q_stride,
                                         const void* kv_pages, int32_t n_groups, const int32_t* cu_group, const int32_t* prefix_table,
                                         int32_t max_prefix_pages, const int32_t* prefix_lens, const int32_t* block_table,
                                         int32_t max_pages_per_seq, const int32_t* ctx_lens, void* scratch, size_t scratch_bytes,
                                         void* out, void* stream) {
  if (!shape_ok(shape) || !query_ok(shape, q, q_stride, out)) return HYP_EINVAL;
  if (!kv_pages || !cu_group || !prefix_table || !prefix_lens || !block_table || !ctx_lens || !scratch) return HYP_EINVAL;
  if (!count_ok(n_seqs) || !count_ok(n_groups) || !pages_ok(max_prefix_pages) || !pages_ok(max_pages_per_seq)) return HYP_EINVAL;
  if (!aligned(kv_pages, 16) || !aligned(scratch, 16)) return HYP_EINVAL;
  if (scratch_bytes < hyp_op_attn_shared_scratch_bytes(shape, n_seqs, n_groups, max_prefix_pages, max_pages_per_seq)) return HYP_ECAPACITY;
  const SharedPlan p = shared_plan(n_seqs, shape->n_q_heads, shape->n_kv_heads, shape->head_dim, n_groups, max_prefix_pages, max_pages_per_seq);
  if ((double)shape->n_kv_heads * ((double)p.prefix_splits * p.row_tiles + (double)p.own_splits * n_seqs) > 2147483647.0) return HYP_ECAPACITY;
  const int rc = tc_prepare();
  if (rc) return rc;
  return finish(launch_decode_shared(view(shape, n_seqs, kv_pages, block_table, max_pages_per_seq, ctx_lens), (const __half*)q, q_stride,
                                     n_groups, cu_group, prefix_table, max_prefix_pages, prefix_lens, (float*)scratch, (__half*)out,
                                     tc_err_flag_ptr(), (cudaStream_t)stream));
}
