// C entry points of the operators in few bits: argument checks, then the launchers.
#include "cache_ops.cuh"
#include "gemm_tc.cuh"
#include "kv8.cuh"
#include "mx4.cuh"

using namespace hyp;

namespace {

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool shape_ok(const hyp_attn_shape* s, int32_t format) {
  if (!s || s->n_kv_heads < 1 || s->n_kv_heads > 32767 || s->n_q_heads < s->n_kv_heads || s->n_q_heads % s->n_kv_heads) return false;
  if (format != HYP_KV8_INT8 && format != HYP_KV8_E4M3) return false;
  const int G = s->n_q_heads / s->n_kv_heads;
  return (G == 1 || G == 2 || G == 4 || G == 8) && (s->head_dim == 64 || s->head_dim == 128);
}
bool pages_ok(int32_t n) { return n >= 1 && n <= (1 << 26); }
bool count_ok(int32_t n) { return n >= 1 && n <= 65535; }
Kv8View view(const hyp_attn_shape* s, int32_t format, int32_t n_seqs, const void* pool, const int32_t* table, int32_t table_stride) {
  return Kv8View{(uint8_t*)pool, table, table_stride, n_seqs, s->n_q_heads, s->n_kv_heads, s->head_dim, format};
}
bool type_ok(int32_t t) { return t == HYP_TYPE_F32 || t == HYP_TYPE_F16 || t == HYP_TYPE_BF16; }
// (up to 2^25 columns: what the grids' second dimension takes; 2^31 - 8 rows: whole CTAs of eight count them in 31 bits)
bool matrix_ok(int32_t N, int32_t K) { return N >= 1 && N <= 0x7ffffff8 && K >= 8 && K <= (1 << 25) && K % 8 == 0; }
// The tensor map counts lines of 64 bytes in 31 bits.
bool mx4_lines_ok(int32_t N, int32_t K, int halves) {
  return (long long)halves * mx_row_tiles(N) * mx_kb(K) * (MX_PACK_BYTES / 64) <= 0x7fffffffll;
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

extern "C" int hyp_op_mx4_quantize(const void* x, int32_t type, int32_t N, int32_t K, int64_t x_stride, void* codes, void* scales,
                                   void* stream) {
  if (!x || !codes || !scales || !type_ok(type) || !matrix_ok(N, K) || x_stride < K) return HYP_EINVAL;
  if (!aligned(x, 16) || !aligned(codes, 16) || x_stride % (type == HYP_TYPE_F32 ? 4 : 8)) return HYP_EINVAL;
  return finish(launch_mx4_quantize(x, type, N, K, x_stride, (uint8_t*)codes, (uint8_t*)scales, (cudaStream_t)stream));
}

extern "C" int hyp_op_mx4_dequantize(const void* codes, const void* scales, int32_t N, int32_t K, int32_t type, void* out,
                                     int64_t out_stride, void* stream) {
  if (!out || !codes || !scales || !type_ok(type) || !matrix_ok(N, K) || out_stride < K) return HYP_EINVAL;
  if (!aligned(out, 16) || !aligned(codes, 16) || out_stride % (type == HYP_TYPE_F32 ? 4 : 8)) return HYP_EINVAL;
  return finish(launch_mx4_dequantize((const uint8_t*)codes, (const uint8_t*)scales, N, K, type, out, out_stride, (cudaStream_t)stream));
}

extern "C" size_t hyp_op_mx4_packed_bytes(int32_t N, int32_t K, int32_t swiglu) {
  if (!matrix_ok(N, K) || !mx4_lines_ok(N, K, swiglu ? 2 : 1)) return 0;
  return mx4_packed_bytes(N, K, swiglu ? 2 : 1);
}

extern "C" int hyp_op_mx4_pack(const void* codes, const void* scales, int32_t N, int32_t K, int32_t swiglu, void* packed,
                               size_t packed_bytes, void* stream) {
  if (!codes || !scales || !packed || !matrix_ok(N, K) || !aligned(codes, 16) || !aligned(packed, 128)) return HYP_EINVAL;
  const size_t need = hyp_op_mx4_packed_bytes(N, K, swiglu);
  if (!need || packed_bytes < need) return HYP_ECAPACITY;
  return finish(launch_mx4_pack((const uint8_t*)codes, (const uint8_t*)scales, N, K, swiglu ? 2 : 1, (uint8_t*)packed, (cudaStream_t)stream));
}

extern "C" size_t hyp_op_gemm_mx4_scratch_bytes(int32_t M, int32_t K, int32_t terms) {
  if (!matrix_ok(M, K) || M > (1 << 26) || terms < 1 || terms > 3) return 0;
  return mx4_scratch_bytes(M, K, terms);
}

extern "C" int hyp_op_gemm_mx4_plan(int32_t M, int32_t N, int32_t K, int32_t terms, int32_t epilogue, int32_t* plan) {
  if (!plan || !matrix_ok(N, K) || M < 1 || M > (1 << 26) || terms < 1 || terms > 3) return HYP_EINVAL;
  if (epilogue < HYP_EPI_STORE_BF16 || epilogue > HYP_EPI_STORE_F32) return HYP_EINVAL;
  const bool swiglu = epilogue == HYP_EPI_SWIGLU_BF16;
  if (!mx4_lines_ok(N, K, swiglu ? 2 : 1)) return HYP_ECAPACITY;
  int32_t v[8];
  mx4_plan(M, N, K, terms, swiglu, v);
  for (int i = 0; i < 8; ++i) plan[i] = v[i];
  return HYP_OK;
}

extern "C" int hyp_op_gemm_mx4(const void* a, int32_t a_type, int64_t a_stride, const void* w_packed, int32_t M, int32_t N, int32_t K,
                               int32_t terms, int32_t epilogue, void* out, int32_t ldo, void* scratch, size_t scratch_bytes, void* stream) {
  if (!a || !w_packed || !out || !scratch || (a_type != HYP_TYPE_F16 && a_type != HYP_TYPE_BF16)) return HYP_EINVAL;
  if (!matrix_ok(N, K) || M < 1 || M > (1 << 26) || terms < 1 || terms > 3 || ldo < N || a_stride < K || a_stride % 8) return HYP_EINVAL;
  if (epilogue < HYP_EPI_STORE_BF16 || epilogue > HYP_EPI_STORE_F32) return HYP_EINVAL;
  const bool wide = epilogue == HYP_EPI_RESID_F32 || epilogue == HYP_EPI_STORE_F32;
  if (!aligned(a, 16) || !aligned(w_packed, 128) || !aligned(scratch, 128) || !aligned(out, wide ? 4 : 2)) return HYP_EINVAL;
  if (!mx4_lines_ok(N, K, epilogue == HYP_EPI_SWIGLU_BF16 ? 2 : 1) || scratch_bytes < mx4_scratch_bytes(M, K, terms)) return HYP_ECAPACITY;
  const int rc = tc_prepare();
  if (rc) return rc;
  return finish(launch_gemm_mx4(a, a_type, a_stride, (const uint8_t*)w_packed, M, N, K, terms, epilogue, out, ldo, (uint8_t*)scratch,
                                (cudaStream_t)stream));
}

extern "C" int hyp_op_kv8_write(const hyp_attn_shape* shape, int32_t format, int32_t n_seqs, int32_t M, const void* qkv, int32_t type,
                                int64_t stride, const float* rope_table, int32_t rope_positions, void* kv8_pages,
                                const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* cu_q, const int32_t* ctx_lens,
                                void* q_out, void* stream) {
  if (!shape_ok(shape, format) || !qkv || !kv8_pages || !block_table || !cu_q || !ctx_lens || !type_ok(type)) return HYP_EINVAL;
  if (!count_ok(n_seqs) || M < 1 || M > (1 << 26) || !pages_ok(max_pages_per_seq) || (rope_table && rope_positions < 1)) return HYP_EINVAL;
  if (stride < ((int64_t)shape->n_q_heads + 2 * shape->n_kv_heads) * shape->head_dim || stride % 8) return HYP_EINVAL;
  if (!aligned(qkv, 16) || !aligned(kv8_pages, 16) || !aligned(rope_table, 16) || !aligned(q_out, 16)) return HYP_EINVAL;
  const int rc = tc_prepare();
  if (rc) return rc;
  return finish(launch_kv8_write(view(shape, format, n_seqs, kv8_pages, block_table, max_pages_per_seq), M, qkv, type, stride, rope_table,
                                 rope_positions, cu_q, ctx_lens, (__half*)q_out, tc_err_flag_ptr(), (cudaStream_t)stream));
}

extern "C" int hyp_op_kv8_read(const hyp_attn_shape* shape, int32_t format, int32_t n_seqs, const void* kv8_pages, const int32_t* block_table,
                               int32_t max_pages_per_seq, const int32_t* first, const int32_t* lens, void* dst_pages,
                               const int32_t* dst_table, int32_t dst_pages_per_seq, void* stream) {
  if (!shape_ok(shape, format) || !kv8_pages || !block_table || !lens || !dst_pages || !dst_table) return HYP_EINVAL;
  if (!count_ok(n_seqs) || !pages_ok(max_pages_per_seq) || !pages_ok(dst_pages_per_seq)) return HYP_EINVAL;
  if (!aligned(kv8_pages, 16) || !aligned(dst_pages, 16)) return HYP_EINVAL;
  // a sequence's half pages, and the step of the warps that share them, are counted in 31 bits
  const int64_t pages = max_pages_per_seq < dst_pages_per_seq ? max_pages_per_seq : dst_pages_per_seq;
  if (pages * 2 * shape->n_kv_heads > 0x7fffffff - (1 << 16)) return HYP_ECAPACITY;
  return finish(launch_kv8_read(view(shape, format, n_seqs, kv8_pages, block_table, max_pages_per_seq), first, lens, (__half*)dst_pages,
                                dst_table, dst_pages_per_seq, (cudaStream_t)stream));
}

extern "C" size_t hyp_op_attn_kv8_scratch_bytes(const hyp_attn_shape* shape, int32_t n_seqs, int32_t max_pages_per_seq) {
  if (!shape_ok(shape, HYP_KV8_INT8) || !count_ok(n_seqs) || !pages_ok(max_pages_per_seq)) return 0;
  return 4 * paged_scratch_floats(n_seqs, shape->n_q_heads, shape->head_dim, kv8_splits(n_seqs, shape->n_kv_heads, max_pages_per_seq));
}

extern "C" int hyp_op_attn_decode_kv8(const hyp_attn_shape* shape, int32_t format, int32_t n_seqs, const void* q, int64_t q_stride,
                                      const void* kv8_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                                      const int32_t* ctx_lens, void* scratch, size_t scratch_bytes, void* out, void* stream) {
  if (!shape_ok(shape, format) || !q || !out || !kv8_pages || !block_table || !ctx_lens || !scratch) return HYP_EINVAL;
  if (!count_ok(n_seqs) || !pages_ok(max_pages_per_seq)) return HYP_EINVAL;
  if (q_stride < (int64_t)shape->n_q_heads * shape->head_dim || q_stride % 8) return HYP_EINVAL;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(kv8_pages, 16) || !aligned(scratch, 16)) return HYP_EINVAL;
  if (scratch_bytes < hyp_op_attn_kv8_scratch_bytes(shape, n_seqs, max_pages_per_seq)) return HYP_ECAPACITY;
  const int rc = tc_prepare();
  if (rc) return rc;
  return finish(launch_attn_kv8(view(shape, format, n_seqs, kv8_pages, block_table, max_pages_per_seq), (const __half*)q, q_stride, ctx_lens,
                                (float*)scratch, (__half*)out, tc_err_flag_ptr(), (cudaStream_t)stream));
}
