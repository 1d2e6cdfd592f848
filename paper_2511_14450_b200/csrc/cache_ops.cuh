// Launchers of the operators over the paged cache that the stage itself does not run: attention with modified scores,
// attention that returns its weights' sums, shared-prefix attention, eviction.  Each enqueues on `st` and returns the
// number of kernels launched or a negative status.
#pragma once
#include "common.cuh"
#include "hyperion_ops.h"

namespace hyp {

// cudaFuncSetAttribute is per device; asked once for each kernel and device.
template <auto kernel>
inline int allow_smem(int bytes) {
  static bool done[64] = {};
  int dev = 0;
  HYP_CUDA_TRY(cudaGetDevice(&dev));
  if (dev >= 0 && dev < 64 && done[dev]) return HYP_OK;
  HYP_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (dev >= 0 && dev < 64) done[dev] = true;
  return HYP_OK;
}

struct CacheView {
  const __half* pool;
  const int32_t* table;
  int table_stride;
  const int32_t* ctx;
  int n_seqs, Hq, Hkv, D;
};

int paged_splits(int n_seqs, int Hkv, int max_pages);
size_t paged_scratch_floats(int n_seqs, int Hq, int D, int n_slots);
// Where the scores of the scored operator start in its scratch: behind the partial rows, on the next 16-byte boundary (a partial
// row is D + 2 floats, so an odd number of rows ends 8 bytes off one, and the scores are read four at a time).
size_t scored_scores_offset(int n_seqs, int Hq, int Hkv, int D, int max_pages);

int launch_decode_mod(const CacheView& c, const hyp_attn_mod& mod, const __half* q, long long q_stride, float* scratch,
                      __half* out, int* err, cudaStream_t st);
int launch_decode_scored(const CacheView& c, const __half* q, long long q_stride, float decay, const float* w_in, float* w_out,
                         long long w_stride, float* scratch, __half* out, int* err, cudaStream_t st);
struct SharedPlan {
  bool flat;  // no row tiles: every sequence walks its prefix itself
  bool even;  // the prefix kernel hands its CTAs out by the lengths it finds
  int prefix_splits, own_splits, row_tiles, prefix_ctas;
};
SharedPlan shared_plan(int n_seqs, int Hq, int Hkv, int D, int n_groups, int prefix_pages, int own_pages);
int launch_decode_shared(const CacheView& c, const __half* q, long long q_stride, int n_groups, const int32_t* cu_group,
                         const int32_t* prefix_table, int prefix_stride, const int32_t* prefix_lens, float* scratch,
                         __half* out, int* err, cudaStream_t st);
int launch_prefill_mod(const CacheView& c, const hyp_attn_mod& mod, int M, const __half* q, long long q_stride,
                       const int32_t* cu_q, __half* out, int* err, cudaStream_t st);

struct EvictArgs {
  const __half* pool;
  const int32_t* table;
  int table_stride;
  const int32_t* cached;
  const float* w_in;
  long long w_stride;
  int n_keep, n_sink, n_recent;
  __half* dst;
  const int32_t* dst_table;
  int dst_stride;
  int32_t* kept;
  int32_t* new_lens;
  float* w_out;
  long long w_out_stride;
  int n_seqs, Hkv, D;
  bool in_place;
};
int launch_kv_evict(const EvictArgs& a, cudaStream_t st);

}  // namespace hyp
