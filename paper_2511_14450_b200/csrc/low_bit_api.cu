// C entry points of the operators in few bits: argument checks, then the launchers.
#include "gemm_tc.cuh"
#include "mx4.cuh"

using namespace hyp;

namespace {

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool type_ok(int32_t t) { return t == HYP_TYPE_F32 || t == HYP_TYPE_F16 || t == HYP_TYPE_BF16; }
bool matrix_ok(int32_t N, int32_t K) { return N >= 1 && K >= 8 && K % 8 == 0; }
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
