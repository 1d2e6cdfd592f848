// The paged cache in 8 bits: layout, launchers.
//
// Pool [n_pages][2 (K, V)][Hkv] half pages of 16 tokens of one head: 16 rows of D one-byte codes, then the 16 tokens' fp32 scales.
// A half page is one run of 16 D + 64 bytes, so one copy brings codes and scales.  At D = 128 the 16-byte chunk c of slot t's row sits
// at chunk position c ^ (4 (t & 1)), so that eight lanes reading four chunks of two neighbouring rows meet all banks; rows of 64
// bytes do so as they are.  HYP_KV8_INT8: value = (code - 128) * scale.  HYP_KV8_E4M3: value = code * scale, scale a power of two.
#pragma once
#include "common.cuh"
#include "hyperion_ops.h"

namespace hyp {

__host__ __device__ constexpr int kv8_half_page(int D) { return 16 * D + 64; }
__host__ __device__ __forceinline__ size_t kv8_half_offset(long long page, int kind, int head, int Hkv, int D) {
  return ((size_t)(page * 2 + kind) * Hkv + head) * kv8_half_page(D);
}
// Byte offset of chunk c in slot t's row.
template <int D>
__host__ __device__ __forceinline__ int kv8_chunk(int c, int t) { return (D == 128 ? c ^ (4 * (t & 1)) : c) << 4; }

struct Kv8View {
  uint8_t* pool;
  const int32_t* table;
  int table_stride;
  int n_seqs, Hq, Hkv, D, fmt;
};

int launch_kv8_write(const Kv8View& c, int M, const void* qkv, int type, long long stride, const float* rope, int rope_positions,
                     const int32_t* cu_q, const int32_t* ctx, __half* q_out, int* err, cudaStream_t st);
int launch_kv8_read(const Kv8View& c, const int32_t* first, const int32_t* lens, __half* dst, const int32_t* dst_table, int dst_stride,
                    cudaStream_t st);
int kv8_splits(int n_seqs, int Hkv, int max_pages);
int launch_attn_kv8(const Kv8View& c, const __half* q, long long q_stride, const int32_t* ctx, float* scratch, __half* out, int* err,
                    cudaStream_t st);

}  // namespace hyp
